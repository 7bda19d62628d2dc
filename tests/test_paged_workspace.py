"""Workspaces that a paged cache refuses to share."""
import pytest
import torch


@pytest.mark.parametrize("bad", [torch.zeros(64, dtype=torch.float32), torch.zeros(64, dtype=torch.uint8, device="meta"),
                                 torch.zeros(128, dtype=torch.uint8)[::2]])
def test_workspaces_of_other_types_and_devices(bad):
    from paper_2607_05061_gb300.paged import PagedCache
    PagedCache.empty(2, 2, 64, page=16, device="cpu", workspace=torch.zeros(64, dtype=torch.uint8))
    with pytest.raises(ValueError):
        PagedCache.empty(2, 2, 64, page=16, device="cpu", workspace=bad)
