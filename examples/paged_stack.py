"""A small stack of attention layers that keep every token in paged 8-bit caches.

Per layer: q, k, v projections, ``PagedCache.append`` (rotation and write), ``PagedCache.attend``,
output projection and residual; no norms and no MLP blocks, as in ``DecodeStack``.  Prompts of
different lengths come in chunks, other sequences' single tokens among them; then every sequence
takes one token a step, captured into a CUDA graph.  With ``--shared`` all prompts begin with the same
tokens, which are read once for all of them; with ``--keep`` the weights of positions are added up, and
the caches cut down to the heaviest ones before the steps.

    python examples/paged_stack.py --layers 4 --batch 16 --prompt 2000 --steps 64
    python examples/paged_stack.py --batch 32 --shared 8192 --prompt 300 --keep 1024
"""
from __future__ import annotations

import argparse
import os
import sys
import time
from typing import Optional

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
                 max_tokens: int, page: int = 64, seed: int = 0, device="cuda", weights: bool = False,
                 keep: Optional[int] = None):
        self.H, self.HQ, self.d, self.hidden, self.b = n_kv_heads, n_kv_heads * q_per_kv, head_dim, hidden, batch
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn((rows, cols), generator=g, device=device) / rows ** 0.5).bfloat16()
        nq, nkv = self.HQ * head_dim, self.H * head_dim
        self.layers = [{"Wqkv": weight(hidden, nq + 2 * nkv), "Wo": weight(nq, hidden)} for _ in range(layers)]
        per = -(-max_tokens // page)
        # with `weights` there is room for what ``shed`` moves, `keep` tokens of every place at most (none given: all)
        move = -(-min(max_tokens if keep is None else keep, max_tokens) // page) if weights else 0
        n_pages = batch * (per + move)
        self.table = PageTable(batch, per, n_pages, page, device=device)
        self.caches = []
        for _ in range(layers):                    # calls of one stack follow each other: one workspace
            self.caches.append(PagedCache.empty(n_pages, n_kv_heads, head_dim, page, device=device,
                                                workspace=self.caches[0].workspace if self.caches else None))
        self.cos, self.sin = rotation_tables(max_tokens, head_dim, device=device)
        self.graph = None
        # with `weights`: what each position of each layer and KV head has been given
        self.mass = [torch.zeros((batch, n_kv_heads, per * page), device=device) for _ in range(layers if weights else 0)]
        self.groups, self._grouped = (None, None), 0        # and the table's changes that they are of
        self._captured = (None, None)                       # groups that the captured step reads

    def forward(self, x, starts=None, max_new=None, lse=None, positions=None):
        """Hidden states ``x [tokens][hidden]`` (bf16) of the new tokens through all layers; the
        table has pages for them, and ``advance`` is the caller's.  ``positions``: where they are not
        the tokens' places."""
        n, HQ, H, d = x.shape[0], self.HQ, self.H, self.d
        if self._grouped != self.table.changes:
            self.regroup()
        table, lens, (groups, prefix) = self.table.dev, self.table.lens, self.groups
        for i, (W, cache) in enumerate(zip(self.layers, self.caches)):
            qkv = torch.matmul(x, W["Wqkv"]).view(n, HQ + 2 * H, d)
            q = cache.append(table, lens, qkv[:, :HQ], qkv[:, HQ:HQ + H], qkv[:, HQ + H:],
                             self.cos, self.sin, starts=starts, max_new=max_new, positions=positions)
            o, l = cache.attend(table, lens, q, starts=starts, max_new=max_new, out_dtype=torch.bfloat16, lse=lse,
                                want_lse=bool(self.mass), groups=groups, prefix=prefix)
            if self.mass:
                cache.weigh(table, lens, q, l, self.mass[i], starts=starts, max_new=max_new)
            x = x + torch.matmul(o.view(n, HQ * d), W["Wo"])
        return x

    def chunk(self, x, new):
        """``new[s]`` more tokens of every open place, their rows in ``x`` one place after the other
        (idle places have none)."""
        counts = self.table.counts(new)
        if x.shape[0] != sum(counts):
            raise ValueError(f"PagedStack.chunk: {x.shape[0]} rows for {sum(counts)} tokens of the open places")
        self.table.grow(new)
        kw = {"positions": self.table.positions(new)} if self.table.held != self.table.seen else {}   # (some were shed)
        y = self.forward(x, self.table.starts(new), max(counts), **kw)
        self.table.advance(new)
        return y

    def share(self, s: int, places, tokens: int) -> int:
        """Sequences at ``places`` that begin as the one at s does; what they share is read once from then on.
        Weights of shared positions start as what s's tokens have given them so far.  Returns the number of shared
        tokens (0 without places)."""
        n = 0
        for t in places:
            n = self.table.share(s, t, tokens)
            for mass in self.mass:
                mass[t, :, :n] = mass[s, :, :n]
        self.regroup()
        return n

    def _turns(self):
        """What turns the tokens of a step: not their places once tokens may be shed."""
        return self.table.pos if self.mass else None

    def regroup(self):
        """Groups of the sequences that share what they begin with, as the table is now (calls see to it when
        places have begun anew).  A captured step's stay where they are and become these, as far as there is room
        for them: the others' sequences read for themselves until the step is captured again."""
        self.groups, self._grouped = self.table.groups(), self.table.changes
        first, prefix = self._captured
        if first is None:
            return
        prefix.zero_()
        if self.groups[0] is not None:
            n = min(len(prefix), len(self.groups[1]))
            first[:n + 1] = self.groups[0][:n + 1]
            first[n + 1:] = self.groups[0][n]
            prefix[:n] = self.groups[1][:n]

    def shed(self, keep: int, sinks: int = 4, window: int = 64):
        """Every layer and KV head keeps the ``keep`` positions of every place that got most weight.  A step
        that was captured before stays good (there are no shared prefixes behind it)."""
        if not 0 <= sinks + window <= keep or min(sinks, window) < 0:
            raise ValueError(f"PagedStack.shed: {sinks} sinks and a window of {window} are not among {keep} tokens")
        to = self.table.shrink(keep)
        for cache, mass in zip(self.caches, self.mass):
            new = torch.zeros_like(mass)
            cache.evict(self.table.dev, self.table.lens, mass, to, keep, sinks=sinks, window=window, new_mass=new)
            mass.copy_(new)
        self.table.shrunk()
        self.regroup()

    def step(self, x):
        """One more token of every place (an idle one's row passes through the residual only)."""
        self.table.grow(1)
        y = self.forward(x, positions=self._turns())
        self.table.advance(1)
        return y

    def capture(self, x_in):
        """A step's layers as a CUDA graph on static ``x_in``; returns the hidden states it leaves.
        ``replay`` runs it."""
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        self._captured = (None, None)
        self.regroup()
        self._captured = self.groups                            # (a step captured earlier has its own)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream):
            torch.matmul(x_in, self.layers[0]["Wqkv"])          # cuBLAS sets itself up outside a capture only
            with torch.cuda.graph(self.graph, stream=stream):
                y = self.forward(x_in, positions=self._turns())
                self.table.advance_lens()
        torch.cuda.current_stream().wait_stream(stream)
        return y

    def replay(self):
        """The captured step: one more token of every open place, as ``step``."""
        if self._grouped != self.table.changes:
            self.regroup()
        self.table.grow(1)
        self.graph.replay()
        self.table.advance_held(1)

    def check(self):
        """Raises what a kernel recorded (bad tables, a wait that ran out)."""
        kvpop._ck(kvpop.kvpop_standalone_status(kvpop._stream()), "kvpop_standalone_status")


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("batch", 16), ("hidden", 4096), ("kv-heads", 8), ("q-per-kv", 4),
                        ("head-dim", 128), ("prompt", 2000), ("chunk", 512), ("steps", 64), ("shared", 0), ("keep", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    st = PagedStack(a.layers, a.batch, a.hidden, a.kv_heads, a.q_per_kv, a.head_dim, a.shared + a.prompt + a.steps + 2,
                    weights=a.keep > 0, keep=a.keep)
    g = torch.Generator(device="cuda").manual_seed(1)
    left = [max(1, a.prompt - 37 * s) for s in range(a.batch)]
    torch.cuda.synchronize()
    t0, tokens = time.perf_counter(), sum(left) + a.shared
    for s in range(a.batch):
        st.table.open(s)
    for at in range(0, a.shared, a.chunk):                     # the first place reads what all begin with
        n = min(a.chunk, a.shared - at)
        st.chunk(torch.randn((n, a.hidden), generator=g, device="cuda").bfloat16(), [n] + [0] * (a.batch - 1))
    if a.shared:
        st.share(0, range(1, a.batch), a.shared)
    while any(left):
        new = [min(a.chunk, k) for k in left]
        st.chunk(torch.randn((sum(new), a.hidden), generator=g, device="cuda").bfloat16(), new)
        left = [k - c for k, c in zip(left, new)]
    st.check()
    t1 = time.perf_counter()
    print(f"prompts: {tokens} tokens through {a.layers} layers in {1e3 * (t1 - t0):.1f} ms")
    if a.keep:
        st.shed(a.keep, window=max(0, min(64, a.keep // 2)), sinks=min(4, a.keep // 2))
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
