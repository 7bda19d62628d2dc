"""More rows than the paged attention can number."""
import pytest

from test_paged_arguments import PTR, attend, batch, kv, pool, rows  # noqa: F401


@pytest.mark.parametrize("tokens,heads,H", [(2 ** 31 - 1, 4, 2), (2 ** 30, 4, 2), (2 ** 20, 1 << 15, 8), (2 ** 31 - 1, 2, 2)])
def test_more_rows_than_can_be_counted(kv, tokens, heads, H):  # noqa: F811
    b = batch(kv, starts_dev=PTR, n_tokens=tokens)
    shared = rows(kv, token_stride=0, head_stride=0)    # one row for all
    assert attend(kv, p=pool(kv, n_kv_heads=H), b=b, q=shared, heads=heads, out=PTR + 1024) == 1
