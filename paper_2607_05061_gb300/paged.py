"""Paged 8-bit key/value cache: layers that keep every token, beside the compressed ones.

``PagedCache`` is one attention layer's pages (e4m3 bytes with a power-of-two scale for each
block of 16 tokens and KV head) and the two calls on them, ``append`` (rotation and write) and
``attend``; both run in ``libkvpop.so`` and this module only checks and passes arguments.
``PageTable`` hands pages out to the sequences of a batch on the host; the layers of a model
share one table and one ``lens``, and each has its own pages.

One decode step of a batch::

    table.grow(new=1)                                   # pages for the coming tokens
    for layer, cache in ...:
        q = cache.append(table.dev, table.lens, q, k, v, cos, sin)
        o, _ = cache.attend(table.dev, table.lens, q)
    table.advance(new=1)                                # once, after the last layer
"""
from __future__ import annotations

import ctypes
import struct
from typing import List, Optional, Sequence

import numpy as np
import torch

from .kvpop import (KVPOP_BF16, KVPOP_F32, _ck, _ptr, _raw_stream, _stream, kvpop_paged_append, kvpop_paged_append_at,
                    kvpop_paged_attend, kvpop_paged_attend_shared, kvpop_paged_batch, kvpop_paged_evict,
                    kvpop_paged_pool, kvpop_paged_shared_bytes, kvpop_paged_weigh, kvpop_paged_workspace_bytes, kvpop_rows)

BLOCK = 16               # tokens that share a scale
_F8 = torch.float8_e4m3fn
_CODES = {torch.float32: KVPOP_F32, torch.bfloat16: KVPOP_BF16}
# the C structs kvpop_paged_batch and kvpop_rows as bytes: a call of a few tokens takes less time on
# the GPU than filling ctypes structures takes on the host
_batch_bytes, _rows_bytes = struct.Struct("PPPqiiii").pack, struct.Struct("Pqq").pack
assert struct.calcsize("PPPqiiii") == ctypes.sizeof(kvpop_paged_batch) and \
    struct.calcsize("Pqq") == ctypes.sizeof(kvpop_rows)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _want(what, name, t, dtype, shape):
    """Refuses a tensor that a call would read or write past its end or as another type."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: {name} is {t.dtype} {tuple(t.shape)} (strides {tuple(t.stride())}), not "
                         f"contiguous {dtype} {tuple(shape)}")


def _output(shape, dtype, device, stream):
    """A tensor of the stream that the call runs on: the current one's free memory may still be in use."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(_stream(stream), device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


class PagedCache:
    """One layer's pages.  ``k_pages, v_pages [n_pages][H][page][d]`` (float8_e4m3fn) and
    ``k_scale, v_scale [n_pages][H][page / 16]`` (fp32) stay the caller's; ``PagedCache.empty``
    makes them.  ``workspace``: another cache's, to share (some 90 MB).  Calls of ``attend`` and ``weigh``
    that use one workspace have to follow each other, on one stream or ordered by events, as those of a
    model's layers do; the class does not see to it.  That goes for one cache used on two streams."""

    def __init__(self, k_pages, v_pages, k_scale, v_scale, workspace: Optional[torch.Tensor] = None):
        n, H, page, d = k_pages.shape
        for name, t in (("k_pages", k_pages), ("v_pages", v_pages)):
            _want("PagedCache", name, t, _F8, (n, H, page, d))
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            _want("PagedCache", name, t, torch.float32, (n, H, page // BLOCK))
        if d not in (64, 128) or page < BLOCK or page > 1024 or page & (page - 1):
            raise ValueError(f"PagedCache: head size {d} (64 or 128), page {page} (a power of two, 16 to 1024)")
        self.device = k_pages.device
        for name, t in (("v_pages", v_pages), ("k_scale", k_scale), ("v_scale", v_scale)):
            if t.device != self.device:
                raise ValueError(f"PagedCache: {name} is on {t.device}, k_pages on {self.device}")
        self.k_pages, self.v_pages, self.k_scale, self.v_scale = k_pages, v_pages, k_scale, v_scale
        self.H, self.page, self.d = H, page, d
        self._pool = kvpop_paged_pool(_ptr(k_pages), _ptr(v_pages), _ptr(k_scale), _ptr(v_scale), n, H, d, page)
        if workspace is not None and (workspace.dtype is not torch.uint8 or workspace.device != self.device or
                                      not workspace.is_contiguous()):
            raise ValueError(f"PagedCache: workspace is {workspace.dtype} on {workspace.device}, not another cache's "
                             f"on {self.device}")
        if workspace is None and self.device.type == "cuda":
            with torch.cuda.device(self.device):
                workspace = torch.zeros(int(kvpop_paged_workspace_bytes()), dtype=torch.uint8, device=self.device)
                torch.cuda.current_stream().synchronize()      # zero for whatever stream comes first
        self.workspace = workspace
        self._index = k_pages.get_device()
        self._scratch = {}
        self._pool_ptr = ctypes.addressof(self._pool)
        self._work = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, page: int = 64, device="cuda",
              workspace: Optional[torch.Tensor] = None) -> "PagedCache":
        pages = [torch.zeros((n_pages, n_kv_heads, page, head_dim), dtype=torch.uint8, device=device).view(_F8)
                 for _ in range(2)]
        scales = [torch.ones((n_pages, n_kv_heads, page // BLOCK), device=device) for _ in range(2)]
        return cls(*pages, *scales, workspace=workspace)

    # ------------------------------------------------------------------ arguments
    def _elsewhere(self, what, *tensors):
        for t in tensors:
            if t is not None and t.get_device() != self._index:
                raise ValueError(f"{what}: a tensor is on {t.device}, the cache on {self.device}")

    def _on(self, what, stream):
        """The stream's handle, if the cache's device is the current one."""
        at = self._index
        if at < 0 or _current_device() != at:
            raise ValueError(f"{what}: the cache is on {self.device}, which is not the current CUDA device")
        return _raw_stream(at) if stream is None and _raw_stream is not None else _stream(stream)

    @staticmethod
    def _batch(what, table, lens, starts, n_tokens, max_new):
        shape = table.shape
        n, stride = shape[0], table.stride()
        if table.dtype is not torch.int32 or len(shape) != 2 or shape[1] < 1 or stride[1] != 1 or \
                (n > 1 and stride[0] < shape[1]):
            raise ValueError(f"{what}: table is {table.dtype} {tuple(shape)} (strides {tuple(stride)}), "
                             f"not {torch.int32} (sequences, pages) with neighbouring entries")
        _want(what, "lens", lens, torch.int32, (n,))
        if starts is None:
            if n_tokens != n:
                raise ValueError(f"{what}: {n_tokens} tokens of {n} sequences need starts")
            first, most = 0, 1
        else:
            _want(what, "starts", starts, torch.int32, (n + 1,))
            first, most = starts.data_ptr(), max(n_tokens if max_new is None else min(max_new, 0x7fffffff), 1)
        return _batch_bytes(table.data_ptr(), lens.data_ptr(), first, max(stride[0], shape[1]), shape[1], n, n_tokens,
                            most)

    def _rows(self, what, name, t, dtype, n_tokens, heads):
        shape, stride = t.shape, t.stride()
        if t.dtype is not dtype or len(shape) != 3 or shape[0] != n_tokens or shape[2] != self.d or \
                (shape[1] < 1 if heads is None else shape[1] != heads) or stride[2] != 1 or stride[0] < 0 or stride[1] < 0:
            raise ValueError(f"{what}: {name} is {t.dtype} {tuple(shape)} (strides {tuple(stride)}), not {dtype} "
                             f"({n_tokens}, {heads or 'heads'}, {self.d}) with contiguous rows")
        return _rows_bytes(t.data_ptr(), stride[0], stride[1])

    # ------------------------------------------------------------------ calls
    # (with a `stream`, outputs that are not given are that stream's)
    def append(self, table, lens, q, k, v, cos=None, sin=None, starts=None, max_new: Optional[int] = None,
               interleaved: bool = False, q_out=None, stream=None, positions=None, axes=None):
        """Rotates the new tokens' ``q [tokens][heads][d]`` and ``k [tokens][H][d]`` by the rows of
        ``cos, sin [positions][rot / 2]`` (none: no rotation) and writes k and ``v`` to the cache
        (q, k and v of one type, bf16 or fp32, any token and head strides of 16 bytes).  ``table
        [n][pages]`` int32, ``lens [n]`` int32 tokens held before (-1: idle), ``starts [n + 1]``
        int32 first token of each sequence (none: one each; rows past its last entry are nobody's and
        stay as they are in the outputs).  ``positions [tokens]`` or ``[tokens][up to 4 axes]`` int32:
        what turns the tokens, where that is not their place in the cache (none: ``lens`` onwards);
        ``axes``: the axis of each of the rot / 2 pairs (bytes, or numbers; with one axis not needed).
        Returns the rotated queries, bf16, in ``q_out`` if given (no memory of q, k or v)."""
        what, dtype, n_tokens = "PagedCache.append", k.dtype, k.shape[0]
        code = _CODES.get(dtype)
        if code is None:
            raise ValueError(f"{what}: k is {dtype}, not bf16 or fp32")
        kr = self._rows(what, "k", k, dtype, n_tokens, self.H)
        vr = self._rows(what, "v", v, dtype, n_tokens, self.H)
        qr, heads, to = None, 0, None
        if q is not None:
            qr, heads = self._rows(what, "q", q, dtype, n_tokens, None), q.shape[1]
            if q_out is None:
                q_out = _output((n_tokens, heads, self.d), torch.bfloat16, k.device, stream)
            _want(what, "q_out", q_out, torch.bfloat16, (n_tokens, heads, self.d))
            to = q_out.data_ptr()
        elif q_out is not None:
            raise ValueError(f"{what}: q_out without q")
        rot = rows = 0
        cos_ptr = sin_ptr = None
        if cos is not None and sin is not None:
            angles = cos.shape
            rows, rot = angles[0], 2 * angles[1]
            if rows < 1 or rot < 16 or rot > self.d or rot % 16:
                raise ValueError(f"{what}: cos is {tuple(cos.shape)}: 2 * {rot // 2} values of {self.d} cannot be "
                                 "rotated (a multiple of 16 can)")
            if cos.dtype is not torch.float32 or sin.dtype is not torch.float32 or sin.shape != angles or \
                    len(angles) != 2 or not cos.is_contiguous() or not sin.is_contiguous():
                _want(what, "cos", cos, torch.float32, (rows, rot // 2))
                _want(what, "sin", sin, torch.float32, (rows, rot // 2))
            cos_ptr, sin_ptr = cos.data_ptr(), sin.data_ptr()
        elif cos is not None or sin is not None:
            raise ValueError(f"{what}: cos and sin come together")
        if positions is not None:
            if cos is None:
                raise ValueError(f"{what}: positions without cos and sin")
            shape = positions.shape
            n_axes = shape[1] if len(shape) == 2 else 1
            if not 1 <= n_axes <= 4 or len(shape) > 2:
                raise ValueError(f"{what}: positions are {tuple(shape)}, not ({n_tokens}, up to 4)")
            _want(what, "positions", positions, torch.int32, (n_tokens,) if len(shape) < 2 else (n_tokens, n_axes))
            if positions.get_device() != self._index:
                self._elsewhere(what, positions)
            if axes is None:
                if n_axes > 1:
                    raise ValueError(f"{what}: positions on {n_axes} axes without axes")
            else:
                axes = bytes(axes)
                if len(axes) != rot // 2 or max(axes) >= n_axes:
                    raise ValueError(f"{what}: axes are {len(axes)} numbers up to {max(axes, default=0)}, not {rot // 2} "
                                     f"below {n_axes}")
        elif axes is not None:
            raise ValueError(f"{what}: axes without positions")
        batch = self._batch(what, table, lens, starts, n_tokens, max_new)
        at = self._index
        if not (table.get_device() == lens.get_device() == k.get_device() == v.get_device() == at and
                (q is None or q.get_device() == q_out.get_device() == at) and
                (cos is None or cos.get_device() == sin.get_device() == at) and
                (starts is None or starts.get_device() == at)):
            self._elsewhere(what, table, lens, starts, q, k, v, cos, sin, q_out)
        on = self._on(what, stream)
        if positions is None:
            status = kvpop_paged_append(self._pool_ptr, batch, qr, heads, kr, vr, code, cos_ptr, sin_ptr, rot, rows,
                                        1 if interleaved else 0, to, on)
        else:
            status = kvpop_paged_append_at(self._pool_ptr, batch, qr, heads, kr, vr, code, cos_ptr, sin_ptr, rot, rows,
                                           1 if interleaved else 0, positions.data_ptr(), n_axes, axes, to, on)
        if status != 0:
            _ck(status, "kvpop_paged_append" if positions is None else "kvpop_paged_append_at")
        return q_out

    def attend(self, table, lens, q, starts=None, max_new: Optional[int] = None, out=None, lse=None,
               out_dtype=torch.float32, want_lse: bool = False, stream=None, groups=None, prefix=None):
        """Attention of the new tokens' ``q [tokens][H * G][d]`` (bf16, rotated) over positions
        0 .. lens + i of their sequences; arguments as ``append``, with which the tokens' own keys
        came.  Sequences that share prefixes: ``groups [n + 1]`` int32, group g being the places groups[g]
        .. groups[g + 1] - 1, and ``prefix [n]`` int32 the positions that its sequences begin with in
        common (``PageTable.groups``); each is read once for all of them.  Returns (out fp32 or bf16 ``[tokens][H * G][d]``, natural-log normalisers
        ``[tokens][H * G]`` or None)."""
        what = "PagedCache.attend"
        n_tokens, heads = q.shape[0], q.shape[1]
        qr = self._rows(what, "q", q, torch.bfloat16, n_tokens, None)
        if heads % self.H:
            raise ValueError(f"{what}: {heads} query heads over {self.H} KV heads")
        if out is None:
            out = _output((n_tokens, heads, self.d), out_dtype, q.device, stream)
        code = _CODES.get(out.dtype)
        if code is None:
            raise ValueError(f"{what}: out is {out.dtype}, not fp32 or bf16")
        _want(what, "out", out, out.dtype, (n_tokens, heads, self.d))
        if lse is None and want_lse:
            lse = _output((n_tokens, heads), torch.float32, q.device, stream)
        if lse is not None:
            _want(what, "lse", lse, torch.float32, (n_tokens, heads))
        batch = self._batch(what, table, lens, starts, n_tokens, max_new)
        at = self._index
        if not (table.get_device() == lens.get_device() == q.get_device() == out.get_device() == at and
                (starts is None or starts.get_device() == at) and (lse is None or lse.get_device() == at)):
            self._elsewhere(what, table, lens, starts, q, out, lse)
        if groups is not None or prefix is not None:
            return self._attend_shared(what, batch, qr, heads, n_tokens, out, code, lse, groups, prefix, stream)
        on = self._on(what, stream)
        status = kvpop_paged_attend(self._pool_ptr, batch, qr, heads, out.data_ptr(), code,
                                    None if lse is None else lse.data_ptr(), *self._work, on)
        if status != 0:
            _ck(status, "kvpop_paged_attend")
        return out, lse


    def _attend_shared(self, what, batch, qr, heads, n_tokens, out, code, lse, groups, prefix, stream):
        if groups is None or prefix is None:
            raise ValueError(f"{what}: groups and prefix come together")
        n_groups = prefix.shape[0] if len(prefix.shape) else 0
        if n_groups < 1:
            raise ValueError(f"{what}: prefix is {tuple(prefix.shape)}, not one number for each group")
        _want(what, "prefix", prefix, torch.int32, (n_groups,))
        _want(what, "groups", groups, torch.int32, (n_groups + 1,))
        self._elsewhere(what, groups, prefix)
        on = self._on(what, stream)
        # (sizes decide: asked for once for each)
        sizes = (batch[24:], batch[16:24] == bytes(8), n_groups, heads)
        need = self._scratch.get(sizes)
        if need is None:
            need = kvpop_paged_shared_bytes(self._pool_ptr, batch, n_groups, heads)
            if len(self._scratch) >= 64:
                self._scratch.clear()
            self._scratch[sizes] = need
        scratch = _output((max(need, 1),), torch.uint8, out.device, stream)
        status = kvpop_paged_attend_shared(self._pool_ptr, batch, qr, heads, groups.data_ptr(), prefix.data_ptr(),
                                           n_groups, out.data_ptr(), code, None if lse is None else lse.data_ptr(),
                                           *self._work, scratch.data_ptr(), need, on)
        if status != 0:
            _ck(status, "kvpop_paged_attend_shared")
        return out, lse

    def _mass(self, what, name, mass, n, room):
        shape = mass.shape
        if mass.dtype is not torch.float32 or len(shape) != 3 or shape[0] != n or shape[1] != self.H or \
                shape[2] < room or not mass.is_contiguous():
            raise ValueError(f"{what}: {name} is {mass.dtype} {tuple(shape)} (strides {tuple(mass.stride())}), not "
                             f"contiguous {torch.float32} ({n}, {self.H}, {room} or more)")

    def weigh(self, table, lens, q, lse, mass, starts=None, max_new: Optional[int] = None, stream=None):
        """Adds the attention weights of the new tokens' ``q`` (as ``attend`` took it, with the ``lse``
        that it returned) to ``mass [n][H][positions]`` fp32, positions at least the table's pages times
        the page: over all query heads of a KV head, for each position of its sequence.  The new tokens'
        own positions start from nothing, so that a tensor kept along with the cache holds what each
        position has got so far.  Returns ``mass``."""
        what = "PagedCache.weigh"
        n_tokens, heads = q.shape[0], q.shape[1]
        qr = self._rows(what, "q", q, torch.bfloat16, n_tokens, None)
        if heads % self.H:
            raise ValueError(f"{what}: {heads} query heads over {self.H} KV heads")
        _want(what, "lse", lse, torch.float32, (n_tokens, heads))
        batch = self._batch(what, table, lens, starts, n_tokens, max_new)
        self._mass(what, "mass", mass, table.shape[0], table.shape[1] * self.page)
        self._elsewhere(what, table, lens, starts, q, lse, mass)
        on = self._on(what, stream)
        status = kvpop_paged_weigh(self._pool_ptr, batch, qr, heads, lse.data_ptr(), mass.data_ptr(), mass.shape[2],
                                   *self._work, on)
        if status != 0:
            _ck(status, "kvpop_paged_weigh")
        return mass

    def evict(self, table, lens, mass, to, keep: int, sinks: int = 0, window: int = 0, kept=None, new_mass=None,
              new_lens=None, stream=None):
        """Cuts sequences of more than ``keep`` tokens down to that, for each KV head by itself: the first
        ``sinks``, the last ``window``, and of the others those of largest ``mass`` (see ``weigh``; the
        lower position first among equals), in their order.  All sequences' tokens move to the pages of
        ``to [n][pages]`` int32, none of which the sequences hold (``PageTable.shrink`` hands them out);
        the old ones are not changed.  Returns (lengths ``[n]`` int32, the kept positions ``[n][H][keep]``
        int32, -1 behind them), in ``new_lens`` and ``kept`` if given; their weights go to ``new_mass
        [n][H][keep or more]`` if given.  What is appended next needs ``positions``: places are no longer
        those."""
        what = "PagedCache.evict"
        n = lens.shape[0] if len(lens.shape) else 0
        batch = self._batch(what, table, lens, None, n, None)
        keep, sinks, window = int(keep), int(sinks), int(window)
        shape, stride = to.shape, to.stride()
        if to.dtype is not torch.int32 or len(shape) != 2 or shape[0] != n or shape[1] < 1 or stride[1] != 1 or \
                (n > 1 and stride[0] < shape[1]):
            raise ValueError(f"{what}: to is {to.dtype} {tuple(shape)} (strides {tuple(stride)}), not {torch.int32} "
                             f"({n}, pages) with neighbouring entries")
        if not 1 <= keep <= min(shape[1] * self.page, 0x7fffffff) or sinks < 0 or window < 0 or sinks + window > keep:
            raise ValueError(f"{what}: keep {keep} of at most {shape[1] * self.page} places, {sinks} sinks and a window "
                             f"of {window}")
        self._mass(what, "mass", mass, n, table.shape[1] * self.page)
        if kept is None:
            kept = _output((n, self.H, keep), torch.int32, mass.device, stream)
        _want(what, "kept", kept, torch.int32, (n, self.H, keep))
        if new_lens is None:
            new_lens = _output((n,), torch.int32, mass.device, stream)
        _want(what, "new_lens", new_lens, torch.int32, (n,))
        if new_mass is not None:
            self._mass(what, "new_mass", new_mass, n, keep)
        self._elsewhere(what, table, lens, mass, to, kept, new_mass, new_lens)
        on = self._on(what, stream)
        status = kvpop_paged_evict(self._pool_ptr, batch, mass.data_ptr(), mass.shape[2], to.data_ptr(),
                                   max(stride[0], shape[1]), shape[1], keep, sinks, window, kept.data_ptr(),
                                   None if new_mass is None else new_mass.data_ptr(),
                                   0 if new_mass is None else new_mass.shape[2], new_lens.data_ptr(), on)
        if status != 0:
            _ck(status, "kvpop_paged_evict")
        return new_lens, kept


class PageTable:
    """Pages of a batch's sequences, handed out on the host: ``dev [n][max_pages]``, ``lens [n]``
    and ``pos [n]`` (int32, on the device; tokens held, and the position of the next one, which is the
    same until tokens are shed) are what the caches take.  A place of the batch is idle (length -1)
    until ``open``.  Sequences can share the pages that they begin with (``share``); a page is free
    again when the last of them has given it back."""

    def __init__(self, n_seq: int, max_pages: int, n_pages: int, page: int = 64, device="cuda"):
        self.page, self.max_pages = page, max_pages
        self.held: List[int] = [-1] * n_seq
        self.seen: List[int] = [-1] * n_seq                # tokens since open, shed ones among them
        self.pages: List[List[int]] = [[] for _ in range(n_seq)]
        self.users: List[int] = [0] * n_pages
        self.free: List[int] = list(range(n_pages - 1, -1, -1))
        self.dev = torch.full((n_seq, max_pages), -1, dtype=torch.int32, device=device)
        self.lens = torch.full((n_seq,), -1, dtype=torch.int32, device=device)
        self.pos = torch.full((n_seq,), -1, dtype=torch.int32, device=device)
        self._shrink: Optional[List[List[int]]] = None     # pages that ``shrink`` handed out
        self.changes = 0                                   # places that began anew on other pages: ``groups`` of before do not hold

    def counts(self, new) -> List[int]:
        """Tokens of every place (``new``: a number, or one for each place): none of idle ones, which
        have no rows among the tokens of a call with ``starts``."""
        n = len(self.held)
        counts = [int(new)] * n if isinstance(new, int) else [int(x) for x in new]
        if len(counts) != n or min(counts, default=0) < 0:
            raise ValueError(f"PageTable: {len(counts)} token counts for {n} places, none below 0")
        return [c if h >= 0 else 0 for c, h in zip(counts, self.held)]

    def _take(self) -> int:
        page = self.free.pop()
        self.users[page] = 1
        return page

    def _give(self, pages: Sequence[int]):
        for page in reversed(pages):
            self.users[page] -= 1
            if self.users[page] == 0:
                self.free.append(page)

    def _settled(self, what):
        if self._shrink is not None:
            raise ValueError(f"PageTable.{what}: tokens are being shed (shrink without shrunk)")

    def open(self, s: int):
        """A new sequence at place s."""
        self.close(s)
        self.changes += 1
        self.held[s] = self.seen[s] = 0
        self.lens[s] = 0
        self.pos[s] = 0

    def close(self, s: int):
        """Gives place s's pages back and leaves it idle."""
        self._settled("close")
        self._give(self.pages[s])
        self.pages[s] = []
        self.held[s] = self.seen[s] = -1
        self.lens[s] = -1
        self.pos[s] = -1
        self.dev[s] = -1

    def share(self, s: int, t: int, tokens: int) -> int:
        """A sequence at place t that begins with the first ``tokens`` tokens of the one at s, as far as they
        fill whole pages, which both then read.  Returns their number.  (Not of one that has shed tokens:
        its heads hold different ones.)"""
        self._settled("share")
        if s == t or self.held[s] < 0 or tokens < 0:
            raise ValueError(f"PageTable.share: {tokens} tokens of place {s} (holds {self.held[s]}) for place {t}")
        if self.held[s] != self.seen[s]:
            raise ValueError(f"PageTable.share: place {s} has shed {self.seen[s] - self.held[s]} of its tokens")
        self.close(t)
        self.changes += 1
        k = min(tokens, self.held[s]) // self.page
        self.pages[t] = self.pages[s][:k]
        for page in self.pages[t]:
            self.users[page] += 1
        self.held[t] = self.seen[t] = k * self.page
        if k:
            self.dev[t, :k] = self.dev[s, :k]
        self.lens[t] = k * self.page
        self.pos[t] = k * self.page
        return k * self.page

    def groups(self):
        """(groups, prefix) for ``PagedCache.attend``: runs of places whose sequences begin with the same
        pages.  (None, None) where none do.  They hold as long as ``changes`` stays what it is (more tokens and
        closed places do not matter).  Whether a group pays is not asked: it does from some 65000 positions that
        are not read again on, at 8 KV heads and d = 128, and calls of few sequences over short prefixes are faster
        without (4 over 512: 11 us, 15 with)."""
        live = [s for s, h in enumerate(self.held) if h >= 0]
        whole = [self.pages[s][:self.held[s] // self.page] for s in live]
        # (what neighbours have in common; a run has the least of it)
        common = [next((m for m, (x, y) in enumerate(zip(a, b)) if x != y), min(len(a), len(b)))
                  for a, b in zip(whole, whole[1:])]
        # the runs that save most reads of pages, the fewest of those that save alike: for the first k live places
        # what they are worth, pages saved before runs, and where the last run begins
        k_all = len(live)
        worth, begin = np.zeros(k_all + 1, np.int64), [0] * (k_all + 1)
        least, others = np.zeros(k_all, np.int64), np.arange(k_all, -1, -1)
        for k in range(1, k_all + 1):
            if k > 1:
                least[k - 2] = common[k - 2]
                np.minimum(least[:k - 2], common[k - 2], out=least[:k - 2])
            each = worth[:k] + others[k_all - k + 1:k_all + 1] * least[:k] * (k_all + 1)
            begin[k] = int(each.argmax())
            worth[k] = each[begin[k]] - 1
        cuts, k = [], len(live)
        while k > 0:
            cuts.append((begin[k], k))
            k = begin[k]
        runs, at, n = [], 0, len(self.held)
        for i, k in reversed(cuts):                        # (idle places within a run do not matter)
            first, end = live[i], live[k - 1] + 1
            if first > at:
                runs.append((at, first, 0))
            runs.append((first, end, min(common[i:k - 1]) * self.page if k - i > 1 else 0))
            at = end
        if at < n:
            runs.append((at, n, 0))
        if not any(p for _, _, p in runs):
            return None, None
        first, prefix = [0], []
        for k, (_, end, p) in enumerate(runs):
            if p == 0 and prefix and prefix[-1] == 0:
                first[-1] = end                            # (places that share nothing, together)
            else:
                first.append(end)
                prefix.append(p)
        dev = self.dev.device
        return torch.tensor(first, dtype=torch.int32, device=dev), torch.tensor(prefix, dtype=torch.int32, device=dev)

    def grow(self, new):
        """Pages for ``new`` more tokens of every sequence (a number, or one for each place); none
        are handed out when they do not suffice (MemoryError)."""
        self._settled("grow")
        counts = self.counts(new)
        need = [max(0, -(-(max(h, 0) + c) // self.page) - len(p)) for h, c, p in zip(self.held, counts, self.pages)]
        if any(len(p) + k > self.max_pages for p, k in zip(self.pages, need)):
            raise MemoryError(f"PageTable: a sequence needs more than {self.max_pages} pages")
        if sum(need) > len(self.free):
            raise MemoryError(f"PageTable: {sum(need)} pages wanted, {len(self.free)} free")
        where, ids = [], []
        for s, k in enumerate(need):
            for _ in range(k):
                where.append((s, len(self.pages[s])))
                ids.append(self._take())
                self.pages[s].append(ids[-1])
        if ids:
            at = torch.tensor(where, dtype=torch.int64, device=self.dev.device)
            self.dev[at[:, 0], at[:, 1]] = torch.tensor(ids, dtype=torch.int32, device=self.dev.device)

    def shrink(self, keep: int) -> torch.Tensor:
        """New pages for at most ``keep`` tokens of every open place, as the table that ``PagedCache.evict`` of
        every layer writes to; ``shrunk`` then makes it the table.  MemoryError when they do not suffice.  (Asked
        again before that, the earlier ones are given back.)"""
        if keep < 1:
            raise ValueError(f"PageTable.shrink: {keep} tokens")
        self._drop_shrink()
        need = [-(-min(max(h, 0), keep) // self.page) for h in self.held]
        if sum(need) > len(self.free):
            raise MemoryError(f"PageTable: {sum(need)} pages wanted, {len(self.free)} free")
        width = -(-keep // self.page)
        self._shrink = [[self._take() for _ in range(k)] for k in need]
        self._keep = keep
        rows = [p + [-1] * (width - len(p)) for p in self._shrink]
        return torch.tensor(rows, dtype=torch.int32, device=self.dev.device)

    def _drop_shrink(self):
        for pages in self._shrink or []:
            self._give(pages)
        self._shrink = None

    def shrunk(self):
        """Every layer has written its tokens to the pages of ``shrink``: the others are given back."""
        if self._shrink is None:
            raise ValueError("PageTable.shrunk: no shrink before it")
        new, self._shrink = self._shrink, None
        self.changes += 1
        for s, pages in enumerate(new):
            self._give(self.pages[s])
            self.pages[s] = pages
            self.held[s] = min(self.held[s], self._keep)
        rows = [p + [-1] * (self.max_pages - len(p)) for p in self.pages]
        self.dev.copy_(torch.tensor(rows, dtype=torch.int32))
        self.lens.copy_(torch.tensor(self.held, dtype=torch.int32))

    def advance_lens(self):
        """One more token of every open place, on the device alone: what a captured step ends with
        (``advance_held`` then tells the host at each replay)."""
        live = (self.lens >= 0).to(torch.int32)
        self.lens += live
        self.pos += live

    def advance_held(self, new):
        """The host's part of ``advance``, for tokens by which a replayed graph moved ``lens``."""
        counts = self.counts(new)
        self.held = [h + c if h >= 0 else h for h, c in zip(self.held, counts)]
        self.seen = [h + c if h >= 0 else h for h, c in zip(self.seen, counts)]

    def advance(self, new):
        """The new tokens are in every layer's cache."""
        self._settled("advance")
        counts = self.counts(new)
        self.advance_held(counts)
        if len(set(counts)) == 1 and min(self.held) >= 0:
            self.lens += counts[0]
            self.pos += counts[0]
        else:
            more = torch.tensor(counts, dtype=torch.int32, device=self.lens.device)
            self.lens += more
            self.pos += more

    def starts(self, new: Sequence[int]) -> torch.Tensor:
        """First token of every place, for the calls' ``starts``: the rows of the open places, one
        after the other (see ``counts``); the last entry is how many there are."""
        at = [0]
        for c in self.counts(new):
            at.append(at[-1] + c)
        return torch.tensor(at, dtype=torch.int32, device=self.dev.device)

    def positions(self, new: Sequence[int]) -> torch.Tensor:
        """Positions of the coming tokens, rows as those of ``starts`` (with one token of every place they
        are ``pos``)."""
        at = [h + i for h, c in zip(self.seen, self.counts(new)) for i in range(c)]
        return torch.tensor(at, dtype=torch.int32, device=self.dev.device)
