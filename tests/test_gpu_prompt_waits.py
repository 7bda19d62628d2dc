"""Tiles of few key blocks of the prompt attention on tcgen05, whose last products are on their way
when the rows are done with the last logits: right, and the same bits in every call.  (The barriers'
rule is modelled in test_gpu_paged_waits.py.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G", [1, 2, 4])
@pytest.mark.parametrize("S", [17, 70, 200, 500, 1500])
def test_tiles_of_few_blocks(cuda_device, S, G):
    from paper_2607_05061_gb300 import kvpop
    n, H, d = 2, 2, 128
    g = torch.Generator().manual_seed(S + G)
    Q, K, V = (torch.randn((n, h, S, d), generator=g).bfloat16().to(cuda_device) for h in (H * G, H, H))
    prio = torch.rand((n * H, S), generator=g).to(cuda_device)
    rank, tau = (t.view(n, H, S) for t in kvpop.topk_cutoff(prio, 4, S, 8))
    first, lse = kvpop.prompt_attention(Q, K, V, rank, tau, 4, S, 8)     # the window holds every key
    x = torch.einsum("nhgsd,nhtd->nhgst", Q.double().view(n, H, G, S, d), K.double()) / d ** 0.5
    x = x.masked_fill(torch.ones(S, S, dtype=torch.bool, device=cuda_device).triu(1), float("-inf"))
    y = (torch.softmax(x, -1) @ V.double()[:, :, None]).view(n, H * G, S, d)
    # weights of 8 bits, averaged: 2^-9 of the largest value at most; fp32 sums of the logits
    assert (first.double() - y).abs().max() <= 2.0 ** -8 * V.double().abs().max()
    assert (lse.double() - torch.logsumexp(x, -1).view(n, H * G, S)).abs().max() <= 1e-5
    flush = torch.empty(160 << 20, dtype=torch.uint8, device=cuda_device)
    for i in range(30):
        if i % 2:
            flush.fill_(i)
        again, lse2 = kvpop.prompt_attention(Q, K, V, rank, tau, 4, S, 8)
        assert torch.equal(again, first) and torch.equal(lse2, lse)
    assert kvpop.kvpop_standalone_status(torch.cuda.current_stream().cuda_stream) == 0
