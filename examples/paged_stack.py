"""A small stack of attention layers that keep every token in paged 8-bit caches.

Per layer: q, k, v projections, ``PagedCache.append`` (rotation and write), ``PagedCache.attend``,
output projection and residual; no norms and no MLP blocks, as in ``DecodeStack``.  Prompts of
different lengths come in chunks, other sequences' single tokens among them; then every sequence
takes one token a step, captured into a CUDA graph.

    python examples/paged_stack.py --layers 4 --batch 16 --prompt 2000 --steps 64
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2607_05061_gb300 import kvpop  # noqa: E402
from paper_2607_05061_gb300.paged import PagedCache, PageTable  # noqa: E402


def rotation_tables(positions: int, rot: int, base: float = 10000.0, device="cuda"):
    """cos, sin [positions][rot / 2] in fp32."""
    half = rot // 2
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (
        -torch.arange(half, dtype=torch.float64) / half)
    return angle.cos().float().to(device), angle.sin().float().to(device)


class PagedStack:
    """``layers`` layers of random weights; all share one page table, each has its own pages."""

    def __init__(self, layers: int, batch: int, hidden: int, n_kv_heads: int, q_per_kv: int, head_dim: int,
                 max_tokens: int, page: int = 64, seed: int = 0, device="cuda"):
        self.H, self.HQ, self.d, self.hidden, self.b = n_kv_heads, n_kv_heads * q_per_kv, head_dim, hidden, batch
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn((rows, cols), generator=g, device=device) / rows ** 0.5).bfloat16()
        nq, nkv = self.HQ * head_dim, self.H * head_dim
        self.layers = [{"Wqkv": weight(hidden, nq + 2 * nkv), "Wo": weight(nq, hidden)} for _ in range(layers)]
        per = -(-max_tokens // page)
        self.table = PageTable(batch, per, batch * per, page, device=device)
        self.caches = []
        for _ in range(layers):                    # calls of one stack follow each other: one workspace
            self.caches.append(PagedCache.empty(batch * per, n_kv_heads, head_dim, page, device=device,
                                                workspace=self.caches[0].workspace if self.caches else None))
        self.cos, self.sin = rotation_tables(max_tokens, head_dim, device=device)
        self.graph = None

    def forward(self, x, starts=None, max_new=None, lse=None):
        """Hidden states ``x [tokens][hidden]`` (bf16) of the new tokens through all layers; the
        table has pages for them, and ``advance`` is the caller's."""
        n, HQ, H, d = x.shape[0], self.HQ, self.H, self.d
        for W, cache in zip(self.layers, self.caches):
            qkv = torch.matmul(x, W["Wqkv"]).view(n, HQ + 2 * H, d)
            q = cache.append(self.table.dev, self.table.lens, qkv[:, :HQ], qkv[:, HQ:HQ + H], qkv[:, HQ + H:],
                             self.cos, self.sin, starts=starts, max_new=max_new)
            o, _ = cache.attend(self.table.dev, self.table.lens, q, starts=starts, max_new=max_new,
                                out_dtype=torch.bfloat16, lse=lse)
            x = x + torch.matmul(o.view(n, HQ * d), W["Wo"])
        return x

    def chunk(self, x, new):
        """``new[s]`` more tokens of every open place, their rows in ``x`` one place after the other
        (idle places have none)."""
        counts = self.table.counts(new)
        if x.shape[0] != sum(counts):
            raise ValueError(f"PagedStack.chunk: {x.shape[0]} rows for {sum(counts)} tokens of the open places")
        self.table.grow(new)
        y = self.forward(x, self.table.starts(new), max(counts))
        self.table.advance(new)
        return y

    def step(self, x):
        """One more token of every place (an idle one's row passes through the residual only)."""
        self.table.grow(1)
        y = self.forward(x)
        self.table.advance(1)
        return y

    def capture(self, x_in):
        """A step's layers as a CUDA graph on static ``x_in``; returns the hidden states it leaves.
        ``replay`` runs it."""
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream):
            torch.matmul(x_in, self.layers[0]["Wqkv"])          # cuBLAS sets itself up outside a capture only
            with torch.cuda.graph(self.graph, stream=stream):
                y = self.forward(x_in)
                self.table.advance_lens()
        torch.cuda.current_stream().wait_stream(stream)
        return y

    def replay(self):
        """The captured step: one more token of every open place, as ``step``."""
        self.table.grow(1)
        self.graph.replay()
        self.table.advance_held(1)

    def check(self):
        """Raises what a kernel recorded (bad tables, a wait that ran out)."""
        kvpop._ck(kvpop.kvpop_standalone_status(kvpop._stream()), "kvpop_standalone_status")


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("batch", 16), ("hidden", 4096), ("kv-heads", 8), ("q-per-kv", 4),
                        ("head-dim", 128), ("prompt", 2000), ("chunk", 512), ("steps", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    st = PagedStack(a.layers, a.batch, a.hidden, a.kv_heads, a.q_per_kv, a.head_dim, a.prompt + a.steps + 2)
    g = torch.Generator(device="cuda").manual_seed(1)
    left = [max(1, a.prompt - 37 * s) for s in range(a.batch)]
    for s in range(a.batch):
        st.table.open(s)
    torch.cuda.synchronize()
    t0, tokens = time.perf_counter(), sum(left)
    while any(left):
        new = [min(a.chunk, k) for k in left]
        st.chunk(torch.randn((sum(new), a.hidden), generator=g, device="cuda").bfloat16(), new)
        left = [k - c for k, c in zip(left, new)]
    st.check()
    t1 = time.perf_counter()
    print(f"prompts: {tokens} tokens through {a.layers} layers in {1e3 * (t1 - t0):.1f} ms")
    x = torch.randn((a.batch, a.hidden), generator=g, device="cuda").bfloat16()
    st.table.grow(a.steps + 1)
    st.capture(x)
    st.replay()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(a.steps):
        st.replay()
    st.check()
    t1 = time.perf_counter()
    print(f"decode: {a.steps} steps of {a.batch} tokens, {1e6 * (t1 - t0) / a.steps:.1f} us a step, "
          f"{a.batch * a.steps / (t1 - t0):.0f} tokens/s")


if __name__ == "__main__":
    main()
