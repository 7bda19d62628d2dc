"""Operators of a serving layer over the paged 8-bit cache, as cases that can be measured.

Four kinds of pass over a cache that holds 8 bits a value (e4m3) with a power-of-two scale for
each block of 16 tokens and KV head:

- ``append``: rotate and write new tokens whose positions are given, on one axis (a cache that
  has shed tokens: a token's place is no longer its position) or several (time, height and width
  of image tokens among text) (``PagedCache.append`` with ``positions`` and ``axes``).
- ``shared``: grouped-query attention of a batch whose sequences share long prefixes, each of
  which is read once for all of them (``PagedCache.attend`` with ``groups`` and ``prefix``).
- ``weigh``: add up the attention weight that the new tokens give to every position of the cache
  (``PagedCache.weigh``).
- ``evict``: keep, for each sequence and KV head, the positions of the largest accumulated weight
  beside the first and the last ones, and write them to new pages (``PagedCache.evict``).

Keys and values are N(0, 1) with a few outlier key channels, as in this repository's workloads;
lengths follow from the case, every value from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 16               # tokens that share a scale
E_MIN = -96              # smallest scale exponent
LIMIT = 2.0 ** 108       # values from here on are stored as NaN


def _case(kind, name=None, **kw):
    c = {"kind": kind, "n_seq": 1, "kv_heads": 8, "q_per_kv": 4, "head_dim": 128, "page": 64,
         "lo": 4096, "hi": 4096, "new_lo": 1, "new_hi": 1, "chunks": 0, "idle": 0,
         "rot": 128, "interleaved": False, "dtype": "bf16", "images": False, "beyond": 0,
         "out": "f32", "groups": 0, "prefix_lo": 0, "prefix_hi": 0, "alone": 0,
         "keep": 0, "sinks": 0, "window": 0}
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a serving batch's next tokens after tokens were shed: places below 4200, positions far above
        _case("append", "append_beyond_b64", n_seq=64, lo=2048, hi=4200, beyond=60000),
        # prompts of text and images, three axes of positions
        _case("append", "append_images", n_seq=3, lo=3, hi=999, new_lo=2501, new_hi=6007, chunks=3, images=True),
        # a few drafts of one short question: the smallest, where latency counts
        _case("shared", "shared_b4_short", n_seq=4, groups=1, prefix_lo=512, prefix_hi=512, lo=40, hi=200),
        # one long document, 64 users asking about it
        _case("shared", "shared_b64", n_seq=64, groups=1, prefix_lo=32768, prefix_hi=32768, lo=100, hi=2000),
        # several system prompts, seven query heads to a KV head, users without one, idle places
        _case("shared", "shared_ragged", n_seq=70, kv_heads=4, q_per_kv=7, page=16, groups=3, prefix_lo=1000,
              prefix_hi=12000, lo=1, hi=3001, alone=5, idle=3, out="bf16"),
        # drafted tokens being verified for samples of two prompts, a d = 64 model
        _case("shared", "shared_verify_d64", n_seq=24, kv_heads=4, q_per_kv=2, head_dim=64, page=32, groups=2,
              prefix_lo=2000, prefix_hi=9000, lo=17, hi=700, new_lo=2, new_hi=6, chunks=24, out="bf16"),
        # one user's next token: the smallest, where latency counts
        _case("weigh", "weigh_b1", n_seq=1, lo=700, hi=700),
        # the serving batch: 64 sequences of 8192 tokens, one new token each
        _case("weigh", "weigh_b64", n_seq=64, lo=8191, hi=8191),
        # what the last tokens of prompts look at
        _case("weigh", "weigh_window", n_seq=3, lo=9001, hi=17011, new_lo=37, new_hi=64, chunks=3, page=128),
        # a whole prompt of odd length
        _case("weigh", "weigh_prompt", n_seq=1, lo=0, hi=0, new_lo=6001, new_hi=6001, chunks=1),
        # every 128 steps a serving batch goes back to its budget
        _case("evict", "evict_b64", n_seq=64, lo=4160, hi=4224, keep=4096, sinks=4, window=256),
        # long prompts are cut down once, odd numbers, a small d = 64 model
        _case("evict", "evict_prompts_d64", n_seq=5, kv_heads=4, q_per_kv=2, head_dim=64, page=16, lo=1001,
              hi=60013, keep=2003, sinks=3, window=129),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.7e12, w["flops"] / 1.9e15)


def draw(rng):
    most = max(map(_cost, listed()))
    while True:
        c = _draw(rng)
        held, new = _lengths(c)[:2]
        top = max(p + k for p, k in zip(held, new))
        # what the plain forms hold: keys of the whole batch, logits
        rows = c["n_seq"] * c["kv_heads"] * top * c["head_dim"]
        square = c["n_seq"] * c["kv_heads"] * c["q_per_kv"] * max(new) * top
        if _cost(c) <= most and rows <= 3e9 and square <= 2e9:
            return c


def _draw(rng):
    kind = rng.choice(["append_token", "append_images", "shared", "shared", "shared_few", "weigh", "weigh_rows", "evict",
                       "evict"])
    d = rng.choice([64, 128, 128])
    c = dict(kv_heads=rng.choice([1, 2, 3, 4, 8, 8]), q_per_kv=rng.choice([1, 2, 3, 4, 4, 5, 7, 8]), head_dim=d,
             page=rng.choice([16, 32, 64, 128]), out=rng.choice(["f32", "bf16"]))
    if kind.startswith("append"):
        c.update(rot=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.3, dtype=rng.choice(["bf16", "bf16", "f32"]))
        if kind == "append_token":
            n, lo = _log(rng, 1, 300), _log(rng, 1, 4000)
            return _case("append", n_seq=n, lo=lo, hi=lo + _log(rng, 1, 4000), beyond=_log(rng, 1, 90000), **c)
        n, lo = _log(rng, 1, 9), rng.randrange(0, 300)
        a = _log(rng, 2, 12000 // n)
        return _case("append", n_seq=n, lo=lo, hi=lo + _log(rng, 1, 500), new_lo=a,
                     new_hi=min(a + _log(rng, 1, 4000), 14000 // n), chunks=n, images=True, **c)
    if kind.startswith("shared"):
        g = rng.choice([1, 1, 2, 3, 4])
        n = g * _log(rng, 2, 64 // g)
        hi = _log(rng, 64, 40000)
        c.update(groups=g, prefix_lo=int(hi * rng.uniform(0.1, 1.0)), prefix_hi=hi, alone=rng.choice([0, 0, 1, 3]))
        if kind == "shared_few":
            lo = rng.randrange(2, 6)
            c.update(new_lo=lo, new_hi=lo + rng.randrange(0, 5), chunks=n + c["alone"])
        lo = _log(rng, 1, 1000)
        return _case("shared", n_seq=n + c["alone"], lo=lo, hi=lo + _log(rng, 1, 2000), idle=rng.choice([0, 0, n // 6]),
                     **c)
    if kind == "weigh":
        n, hi = _log(rng, 1, 100), _log(rng, 16, 100000)
        return _case("weigh", n_seq=n, lo=max(1, int(hi * rng.uniform(0.05, 1.0))), hi=hi,
                     idle=rng.choice([0, 0, n // 8]), **c)
    if kind == "weigh_rows":
        n, lo = _log(rng, 1, 8), rng.choice([0, _log(rng, 1, 9000)])
        a = _log(rng, 2, 5000 // n)
        return _case("weigh", n_seq=n, lo=lo, hi=int(lo * rng.uniform(1.0, 1.5)), new_lo=a,
                     new_hi=int(a * rng.uniform(1.0, 1.4)), chunks=n, **c)
    n, hi = _log(rng, 1, 64), _log(rng, 40, 60000)
    keep = max(16, int(hi * rng.uniform(0.05, 1.1)))
    window = rng.randrange(0, min(keep // 2, 300) + 1)
    return _case("evict", n_seq=n, lo=int(hi * rng.uniform(0.05, 1.0)), hi=hi, keep=keep, window=window,
                 sinks=rng.randrange(0, 5), idle=rng.choice([0, 0, n // 8]), **c)


# ------------------------------------------------------------------ lengths
def _lengths(case):
    """(tokens held, new tokens) of every sequence (-1 held: an idle place of the batch), and the
    groups' first sequences and shared tokens."""
    r = random.Random(case["n_seq"] * 7919 + case["hi"] * 31 + case["new_hi"] + case["prefix_hi"])
    n, page, groups = case["n_seq"], case["page"], case["groups"]
    held = [r.randint(case["lo"], case["hi"]) for _ in range(n)]
    new = [r.randint(case["new_lo"], case["new_hi"]) if s < case["chunks"] else 1 for s in range(n)]
    first, prefix = [0], []
    if groups:
        cuts = sorted(r.sample(range(2, n - case["alone"] - 1, 2), groups - 1)) if groups > 1 else []
        first += cuts + [n - case["alone"]]
        for g in range(groups):                      # whole pages are shared
            tokens = max(r.randint(case["prefix_lo"], case["prefix_hi"]) // page, 1) * page
            prefix.append(tokens)
            for s in range(first[g], first[g + 1]):
                held[s] += tokens
    for s in r.sample(range(n), case["idle"]):
        held[s] = -1
    return held, new, first, prefix


def work(case):
    held, new, first, prefix = _lengths(case)
    H, G, d = case["kv_heads"], case["q_per_kv"], case["head_dim"]
    live = [(p, n) for p, n in zip(held, new) if p >= 0]
    tokens = sum(n for _, n in live)
    ctx = sum(p + n for p, n in live)
    seen = sum(n * p + n * (n + 1) // 2 for p, n in live)
    if case["kind"] == "append":
        esz = 2 if case["dtype"] == "bf16" else 4
        blocks = sum((p + n - 1) // BLOCK - p // BLOCK + 1 for p, n in live)
        table = tokens * (case["rot"] * 4 + (12 if case["images"] else 4))
        return {"bytes": tokens * d * (2 * H * (esz + 1) + H * G * (esz + 2)) + blocks * H * 8 + table,
                "flops": tokens * H * (G + 1) * case["rot"] * 3}
    if case["kind"] == "shared":
        for g, tokens_shared in enumerate(prefix):   # once for all of a group
            members = sum(held[s] >= 0 for s in range(first[g], first[g + 1]))
            ctx -= max(members - 1, 0) * tokens_shared
        osz = 4 if case["out"] == "f32" else 2
        return {"bytes": ctx * H * (2 * d + 8 / BLOCK) + tokens * H * G * (d * (2 + osz) + 4),
                "flops": 4 * d * H * G * seen}
    if case["kind"] == "weigh":
        return {"bytes": ctx * H * (d + 4 / BLOCK + 4) + sum(p for p, _ in live) * H * 4 + tokens * H * G * (2 * d + 4),
                "flops": 2 * d * H * G * seen}
    kept = sum(min(p, case["keep"]) for p, _ in live)
    return {"bytes": sum(p for p, _ in live) * H * 4 + kept * H * (4 * d + 4 * 4 / BLOCK + 8),
            "flops": kept * H * d * 2}


# ------------------------------------------------------------------ inputs
def _exponent(amax):
    """Least e with amax <= 448 * 2^e, at least E_MIN (amax: finite, >= 0)."""
    m, k = torch.frexp(amax)
    return torch.where(amax > 0, k - 9 + (m > 0.875).to(k.dtype), torch.full_like(k, E_MIN)).clamp_min(E_MIN)


def _pow2(e, like):
    """2^e in the type of `like`, from its exponent's bits."""
    if like.dtype == torch.float64:
        return ((e.long() + 1023) << 52).view(torch.float64)
    return ((e.int() + 127) << 23).view(torch.float32)


def _tokens(g, shape, outliers):
    x = torch.randn(shape, generator=g, device="cuda")
    if outliers:
        x[..., 3::37] *= 10
    return x


def _pool(g, case, n_pages, outliers):
    """Pages full of tokens, as earlier calls left them."""
    H, d, page = case["kv_heads"], case["head_dim"], case["page"]
    x = _tokens(g, (n_pages, H, page // BLOCK, BLOCK, d), outliers)
    scale = _pow2(_exponent(x.abs().amax((3, 4))), x)
    return (x / scale[..., None, None]).to(torch.float8_e4m3fn).view(n_pages, H, page, d), scale


def _image_positions(r, n, base):
    """Positions (time, height, width) of n tokens: runs of text, and images of some rows and columns,
    after which text goes on behind the largest position."""
    at, out = base, []
    while len(out) < n:
        text = r.randint(1, 200)
        out += [(at + i,) * 3 for i in range(text)]
        at += text
        rows, cols = r.randint(2, 40), r.randint(2, 40)
        out += [(at, at + y, at + x) for y in range(rows) for x in range(cols)]
        at += max(rows, cols)
    return out[:n]


def _axes(case):
    """Axis of each rotated pair: a quarter of them turn with time, the others with height and width."""
    half = case["rot"] // 2
    a = half // 4
    b = (half - a) // 2
    return bytes([0] * a + [1] * b + [2] * (half - a - b))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H, G, d, page, kind = case["kv_heads"], case["q_per_kv"], case["head_dim"], case["page"], case["kind"]
    held, new, first, prefix = _lengths(case)
    n = case["n_seq"]
    extra = 0 if kind == "evict" else 1
    need = [(max(p, 0) + extra * k + page - 1) // page for p, k in zip(held, new)]
    shared = [0] * n                                 # pages of the group's prefix, at its first sequence's places
    for i, tokens in enumerate(prefix):
        shared[first[i]:first[i + 1]] = [tokens // page] * (first[i + 1] - first[i])
    to_pages = -(-case["keep"] // page)
    n_pages = sum(need) + n * to_pages + 3
    s = {"case": case, "max_new": max(new), "top": max(p + extra * k for p, k in zip(held, new))}
    s["k_pages"], s["k_scale"] = _pool(g, case, n_pages, True)
    s["v_pages"], s["v_scale"] = _pool(g, case, n_pages, False)
    table = torch.full((n, max(max(need), 1)), -1, dtype=torch.int32)
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).cpu()
    at, prefix_ids = 0, None
    for i, k in enumerate(need):
        if i in first[:len(prefix)]:
            prefix_ids = ids[at:at + shared[i]]
            at += shared[i]
        if held[i] >= 0:
            if shared[i]:
                table[i, :shared[i]] = prefix_ids
            table[i, shared[i]:k] = ids[at:at + k - shared[i]]
            at += k - shared[i]
    s["table"] = table.cuda()
    s["lens"] = torch.tensor(held, dtype=torch.int32, device="cuda")
    total = sum(new)
    starts = [0]
    for k in new:
        starts.append(starts[-1] + k)
    s["starts"] = None if max(new) == 1 else torch.tensor(starts, dtype=torch.int32, device="cuda")
    if kind == "append":
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        # q, k and v are columns of one projection's rows
        qkv = _tokens(g, (total, H * G + 2 * H, d), False)
        qkv[:, :H * G + H, 3::37] *= 10
        qkv = qkv.to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
        r = random.Random(seed)
        if case["images"]:
            rows = []
            for p, k in zip(held, new):
                rows += _image_positions(r, k, r.randint(0, max(p, 0)))
            s["positions"], s["axes"] = torch.tensor(rows, dtype=torch.int32, device="cuda"), _axes(case)
        else:
            rows = [max(p, 0) + r.randint(0, case["beyond"]) + i for p, k in zip(held, new) for i in range(k)]
            s["positions"], s["axes"] = torch.tensor(rows, dtype=torch.int32, device="cuda"), None
        half = case["rot"] // 2
        freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
        angle = torch.arange(s["top"] + case["beyond"] + 1, dtype=torch.float64)[:, None] * freq
        s["cos"], s["sin"] = angle.cos().float().cuda(), angle.sin().float().cuda()
        s["q_out"] = torch.zeros((total, H * G, d), dtype=torch.bfloat16, device="cuda")
    elif kind == "evict":
        to = torch.full((n, to_pages), -1, dtype=torch.int32)
        for i in range(n):
            if held[i] >= 0:
                to[i] = ids[at:at + to_pages]
                at += to_pages
        s["to"] = to.cuda()
        # sums of many softmax weights: many orders of magnitude, and some that no token looked at
        P = table.shape[1] * page
        mass = torch.randn((n, H, P), generator=g, device="cuda").mul_(2).exp_().mul_(1e-3)
        s["mass"] = mass * (torch.rand((n, H, P), generator=g, device="cuda") > 0.1)
        s["kept"] = torch.full((n, H, case["keep"]), -7, dtype=torch.int32, device="cuda")
        s["new_mass"] = torch.zeros((n, H, to_pages * page), device="cuda")
        s["new_lens"] = torch.zeros((n,), dtype=torch.int32, device="cuda")
    else:
        s["q"] = _tokens(g, (total, H * G, d), False).bfloat16()
        if kind == "shared":
            s["groups"] = torch.tensor(first, dtype=torch.int32, device="cuda")
            s["prefix"] = torch.tensor(prefix, dtype=torch.int32, device="cuda")
            s["out"] = torch.zeros((total, H * G, d), device="cuda",
                                   dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16)
            s["lse"] = torch.zeros((total, H * G), device="cuda")
        else:
            # the normalisers as the attention of the same tokens left them, and what earlier ones gave
            s["lse"] = _attention(s)[1]
            P = table.shape[1] * page
            s["mass"] = torch.randn((n, H, P), generator=g, device="cuda").exp_().mul_(1e-2)
    if own:
        from paper_2607_05061_gb300.paged import PagedCache
        s["cache"] = PagedCache(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"])
    return s


# ------------------------------------------------------------------ the plain forms
def _places(s):
    """Sequence, index among its new tokens and place of every new token."""
    total = s["q"].shape[0]
    dev = s["q"].device
    at = torch.arange(total, device=dev)
    if s["starts"] is None:
        seq, i = at, torch.zeros_like(at)
    else:
        seq = torch.searchsorted(s["starts"].long(), at, right=True) - 1
        i = at - s["starts"].long()[seq]
    return seq, i, s["lens"].long()[seq] + i


def _rotate(x, c, w, interleaved):
    """x [n][heads][d] in 32 bits, its first pairs rotated by c, w [n][1][pairs]."""
    half = c.shape[-1]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2] = a * c - b * w
        y[..., 1:2 * half:2] = b * c + a * w
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half] = a * c - b * w
        y[..., half:2 * half] = b * c + a * w
    return y


def _store(s, name, x, seq, i, pos):
    """Writes x [n][H][d] into the pages, with the scales of their blocks."""
    page = s["case"]["page"]
    pages, scale = s[name + "_pages"].view(torch.uint8), s[name + "_scale"]
    H, nb = x.shape[1], page // BLOCK
    at = s["table"].long()[seq, pos // page]
    block, row = pos % page // BLOCK, pos % page
    heads = torch.arange(H, device=x.device)
    fine = x.abs() < LIMIT
    need = _pow2(_exponent(torch.where(fine, x.abs(), 0.0).amax(-1)), x)
    # a block's scale so far: none where its first token is among the new ones
    first = pos % BLOCK == 0
    flat = (at[:, None] * H + heads) * nb + block[:, None]
    before = scale.view(-1)[flat]
    base = torch.where(first[:, None], 0.0, before)
    fresh = torch.zeros_like(scale.view(-1))
    fresh.scatter_reduce_(0, flat.view(-1), base.view(-1), "amin", include_self=False)
    fresh.scatter_reduce_(0, flat.view(-1), need.view(-1), "amax")
    after = fresh[flat]
    # tokens that share the block with a sequence's first new token, and came before it
    rows = torch.arange(BLOCK, device=x.device)
    lead = (i == 0)[:, None, None, None] & (rows < (pos % BLOCK)[:, None])[:, None, :, None]
    lead_at = (pos - pos % BLOCK) % page
    head = torch.arange(x.shape[0], device=x.device) if s["starts"] is None else s["starts"].long()[:-1]
    h_at, h_row = at[head], lead_at[head]
    old = pages.view(-1, H, nb, BLOCK, x.shape[2])[h_at, :, h_row // BLOCK]
    moved = (old.view(torch.float8_e4m3fn).float() * (before / after)[head][..., None, None])
    moved = moved.to(torch.float8_e4m3fn).view(torch.uint8)
    pages.view(-1, H, nb, BLOCK, x.shape[2])[h_at, :, h_row // BLOCK] = torch.where(lead[head], moved, old)
    scale.view(-1)[flat] = after
    code = torch.where(fine, x / after[..., None], float("nan")).to(torch.float8_e4m3fn)
    pages[at, :, row] = code.view(torch.uint8)


def _plain_append(s):
    seq, i, pos = _places(s)
    half = s["cos"].shape[1]
    pairs = torch.arange(half, device=pos.device)
    if s["axes"] is None:
        turn = s["positions"].long()[:, None].expand(-1, half)
    else:
        turn = s["positions"].long()[:, torch.tensor(list(s["axes"]), device=pos.device)]
    c, w = s["cos"][turn, pairs][:, None], s["sin"][turn, pairs][:, None]
    s["q_out"].copy_(_rotate(s["q"].float(), c, w, s["case"]["interleaved"]))
    _store(s, "k", _rotate(s["k"].float(), c, w, s["case"]["interleaved"]), seq, i, pos)
    _store(s, "v", s["v"].float(), seq, i, pos)


def _rows(s, pages, scale):
    """[n_seq][H][top][d] in 32 bits."""
    H, d, page = s["case"]["kv_heads"], s["case"]["head_dim"], s["case"]["page"]
    at = s["table"].long().clamp_min(0)
    x = pages[at].float().view(*at.shape, H, page // BLOCK, BLOCK, d) * scale[at][..., None, None]
    return x.view(*at.shape, H, page, d).transpose(1, 2).reshape(at.shape[0], H, -1, d)


def _logits(s):
    """Sequence and index of every token, and the logits [n][H][new][G][T] (-inf: not seen)."""
    c = s["case"]
    H, G, d = c["kv_heads"], c["q_per_kv"], c["head_dim"]
    seq, i, pos = _places(s)
    K = _rows(s, s["k_pages"], s["k_scale"])
    n, T, M = K.shape[0], K.shape[2], s["max_new"]
    q = torch.zeros((n, M, H, G, d), device=K.device)
    q[seq, i] = s["q"].float().view(-1, H, G, d)
    limit = torch.full((n, M), -1, dtype=torch.int64, device=K.device)
    limit[seq, i] = torch.where(s["lens"].long()[seq] >= 0, pos, -1)
    t = torch.arange(T, device=K.device)
    x = q.permute(0, 2, 1, 3, 4).reshape(n, H, M * G, d) @ K.transpose(2, 3) / math.sqrt(d)
    x = x.view(n, H, M, G, T).masked_fill_(t > limit[:, None, :, None, None], -math.inf)
    return seq, i, limit, x


def _attention(s, values=False):
    """Outputs (where asked for) and normalisers of the new tokens, [tokens][H * G] ..."""
    c = s["case"]
    H, G, d = c["kv_heads"], c["q_per_kv"], c["head_dim"]
    seq, i, limit, x = _logits(s)
    n, _, M, _, T = x.shape
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3)[seq, i].reshape(-1, H * G)
    if not values:
        return None, lse
    V = _rows(s, s["v_pages"], s["v_scale"])
    V = torch.where((torch.arange(T, device=x.device) <= limit.amax(1)[:, None])[:, None, :, None], V, 0.0)
    y = (p.view(n, H, M * G, T) @ V).view(n, H, M, G, d) / torch.where(total > 0, total, 1.0)
    return y.permute(0, 2, 1, 3, 4)[seq, i].reshape(-1, H * G, d), lse


def _plain_weigh(s):
    c = s["case"]
    H, G = c["kv_heads"], c["q_per_kv"]
    seq, i, limit, x = _logits(s)
    n, _, M, _, T = x.shape
    lse = torch.full((n, M, H, G), math.inf, device=x.device)
    lse[seq, i] = s["lse"].view(-1, H, G)
    p = torch.exp(x - lse.permute(0, 2, 1, 3)[..., None]).sum((2, 3))
    # positions of earlier tokens go on from what they had, the new tokens' own from nothing
    t = torch.arange(T, device=x.device)
    lens, last = s["lens"].long(), limit.amax(1)
    held = (t < lens[:, None])[:, None]
    here = (t <= last[:, None])[:, None]
    s["mass"].copy_(torch.where(here, torch.where(held, s["mass"], 0.0) + p, s["mass"]))


def _plain_evict(s):
    c = s["case"]
    H, d, page, keep = c["kv_heads"], c["head_dim"], c["page"], c["keep"]
    lens = s["lens"].long().clamp_min(0)
    P = s["mass"].shape[2]
    t = torch.arange(P, device=lens.device)
    count = lens.clamp_max(keep)
    always = (t < c["sinks"]) | (t >= lens[:, None] - c["window"])
    key = torch.where(always[:, None], math.inf, s["mass"])
    key = torch.where((t < lens[:, None])[:, None], key, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    order = torch.nn.functional.pad(order, (0, max(0, keep - P)))[..., :keep]
    j = torch.arange(keep, device=lens.device)
    there = (j < count[:, None])[:, None]
    kept = torch.sort(torch.where(there, order, P + j), dim=-1).values
    at = torch.where(there, kept, 0)
    s["kept"].copy_(torch.where(there, kept, -1))
    s["new_lens"].copy_(torch.where(s["lens"] >= 0, count.to(torch.int32), -1))
    room = s["new_mass"][..., :keep]
    room.copy_(torch.where(there, s["mass"].gather(2, at), room))
    seqs = torch.arange(lens.shape[0], device=lens.device)[:, None, None]
    heads = torch.arange(H, device=lens.device)[:, None]
    src = s["table"].long().clamp_min(0)[seqs, at // page]
    slots = s["to"].shape[1] * page
    full = torch.nn.functional.pad(there.expand(-1, H, -1), (0, slots - keep))
    blocks = full.view(*full.shape[:2], -1, BLOCK)
    dst = s["to"].long().clamp_min(0)
    for_block = dst.repeat_interleave(page // BLOCK, 1)[:, None]
    nb = torch.arange(slots // BLOCK, device=lens.device) % (page // BLOCK)
    some = blocks.any(-1)
    put = seqs.expand(-1, H, slots // BLOCK)[some]
    put_h = heads.expand(lens.shape[0], H, slots // BLOCK)[some]
    put_p = for_block.expand(-1, H, -1)[some]
    put_b = nb.expand(lens.shape[0], H, -1)[some]
    return _move(s, "k", src, heads, at, blocks, some, put_p, put_h, put_b) + \
        _move(s, "v", src, heads, at, blocks, some, put_p, put_h, put_b) + (put,)


def _move(s, name, src, heads, at, blocks, some, put_p, put_h, put_b):
    """The kept rows as blocks of 16 under scales of their own."""
    c = s["case"]
    d, page = c["head_dim"], c["page"]
    pages, scale = s[name + "_pages"], s[name + "_scale"]
    row = at % page
    x = pages.view(torch.uint8)[src, heads, row].view(torch.float8_e4m3fn).float() * scale[src, heads, row // BLOCK][..., None]
    x = torch.nn.functional.pad(x, (0, 0, 0, blocks.shape[2] * BLOCK - x.shape[2]))
    x = x.view(*blocks.shape, d)[some]
    there = blocks[some][..., None]
    held = there & ~torch.isnan(x)
    fresh = _pow2(_exponent(torch.where(held, x.abs(), 0.0).amax((1, 2))), x)
    code = (x / fresh[:, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    to = pages.view(torch.uint8).view(pages.shape[0], pages.shape[1], page // BLOCK, BLOCK, d)
    to[put_p, put_h, put_b] = torch.where(there, code, to[put_p, put_h, put_b])
    scale[put_p, put_h, put_b] = fresh
    return (code,)


def run(state):
    s = state
    c = s["case"]
    pages = {k: s[k] for k in ("k_pages", "v_pages", "k_scale", "v_scale")}
    if c["kind"] == "append":
        if own:
            s["cache"].append(s["table"], s["lens"], s["q"], s["k"], s["v"], s["cos"], s["sin"], starts=s["starts"],
                              max_new=s["max_new"], interleaved=c["interleaved"], q_out=s["q_out"],
                              positions=s["positions"], axes=s["axes"])
        else:
            _plain_append(s)
        return {"q": s["q_out"], **pages}
    if c["kind"] == "shared":
        if own:
            s["cache"].attend(s["table"], s["lens"], s["q"], starts=s["starts"], max_new=s["max_new"], out=s["out"],
                              lse=s["lse"], groups=s["groups"], prefix=s["prefix"])
        else:
            y, lse = _attention(s, True)
            s["out"].copy_(y)
            s["lse"].copy_(lse)
        return {"out": s["out"], "lse": s["lse"]}
    if c["kind"] == "weigh":
        if own:
            s["cache"].weigh(s["table"], s["lens"], s["q"], s["lse"], s["mass"], starts=s["starts"],
                             max_new=s["max_new"])
        else:
            _plain_weigh(s)
        return {"mass": s["mass"]}
    if own:
        s["cache"].evict(s["table"], s["lens"], s["mass"], s["to"], c["keep"], sinks=c["sinks"], window=c["window"],
                         kept=s["kept"], new_mass=s["new_mass"], new_lens=s["new_lens"])
    else:
        _plain_evict(s)
    return {"kept": s["kept"], "new_mass": s["new_mass"], "new_lens": s["new_lens"], **pages}


# ------------------------------------------------------------------ in 64 bits
def _round_e4m3(x):
    """Nearest e4m3 value, ties to even, of 64-bit x with |x| <= 448."""
    _, k = torch.frexp(x)
    step = _pow2((k - 4).clamp_min(-9), x)
    return torch.round(x / step) * step


def _exact_append(s, case, held, new):
    H, G, page = case["kv_heads"], case["q_per_kv"], case["page"]
    table = s["table"].cpu().tolist()
    q, at, half = s["q"].double(), 0, case["rot"] // 2
    out = {"q": torch.zeros(q.shape, dtype=torch.float64, device="cuda")}
    for name in ("k", "v"):
        out[name + "_pages"] = s[name + "_pages"].double()
        out[name + "_scale"] = s[name + "_scale"].double()

    def turn(x, a, n):
        pos = s["positions"][a:a + n].long()
        c, w = torch.zeros((2, n, 1, half), dtype=torch.float64, device="cuda")
        for j in range(half):
            p = pos if s["axes"] is None else pos[:, s["axes"][j]]
            c[:, 0, j], w[:, 0, j] = s["cos"][p, j].double(), s["sin"][p, j].double()
        if case["interleaved"]:
            z = torch.view_as_complex(x[..., :2 * half].reshape(n, -1, half, 2).contiguous())
            z = torch.view_as_real(z * torch.complex(c, w)).reshape(n, -1, 2 * half)
        else:
            z = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * torch.complex(c, w)
            z = torch.cat([z.real, z.imag], -1)
        return torch.cat([z, x[..., 2 * half:]], -1)

    for i in range(case["n_seq"]):
        p, n = held[i], new[i]
        if p >= 0:
            out["q"][at:at + n] = turn(q[at:at + n], at, n)
            ids = torch.tensor(table[i], device="cuda").clamp_min(0)
            b0, b1 = p // BLOCK, (p + n - 1) // BLOCK + 1
            for name, x in (("k", turn(s["k"][at:at + n].double(), at, n)), ("v", s["v"][at:at + n].double())):
                blk = torch.arange(b0, b1, device="cuda")
                pg, nb = ids[blk * BLOCK // page], blk % (page // BLOCK)
                codes, scales = out[name + "_pages"].view(-1, H, page // BLOCK, BLOCK, x.shape[2]), out[name + "_scale"]
                got, was = codes[pg, :, nb].clone(), scales[pg, :, nb].clone()
                lead = p - b0 * BLOCK
                vals = torch.zeros((b1 - b0) * BLOCK, H, x.shape[2], dtype=torch.float64, device="cuda")
                vals[lead:lead + n] = x
                vals = vals.view(b1 - b0, BLOCK, H, x.shape[2]).transpose(1, 2)
                fresh = _pow2(_exponent(vals.abs().amax((2, 3))), vals)
                if lead:
                    fresh[0] = torch.maximum(fresh[0], was[0])
                row = torch.arange((b1 - b0) * BLOCK, device="cuda").view(-1, 1, BLOCK, 1)
                code = _round_e4m3(vals / fresh[..., None, None])
                moved = _round_e4m3(got * (was / fresh)[..., None, None])
                got = torch.where(row < lead, moved, torch.where(row < lead + n, code, got))
                codes[pg, :, nb], scales[pg, :, nb] = got, fresh
        at += n
    return out


def _exact_rows(s, case, held, new):
    """Attention of each sequence and KV head by itself: outputs and normalisers, or the weights' sums."""
    H, G, d, page = case["kv_heads"], case["q_per_kv"], case["head_dim"], case["page"]
    table = s["table"].cpu().tolist()
    weigh = case["kind"] == "weigh"
    q, at = s["q"].double(), 0
    y = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if weigh else None
    for i in range(case["n_seq"]):
        p, n = held[i], new[i]
        if p >= 0:
            T = p + n
            ids = torch.tensor(table[i][:(T + page - 1) // page], device="cuda")
            if weigh:
                mass[i, :, p:T] = 0.0
            for h in range(H):
                k, v = ((s[m + "_pages"][ids, h].double().view(-1, BLOCK, d)
                         * s[m + "_scale"][ids, h].double().reshape(-1, 1, 1)).view(-1, d)[:T] for m in "kv")
                for j in range(0, n, 1024):
                    e = min(n, j + 1024)
                    qh = q[at + j:at + e, h * G:h * G + G].reshape(-1, d)
                    x = (qh @ k.T).view(e - j, G, T) / math.sqrt(d)
                    gone = torch.arange(T, device="cuda") > p + torch.arange(j, e, device="cuda")[:, None]
                    x = x.masked_fill(gone[:, None], -math.inf)
                    if weigh:
                        x = x - s["lse"][at + j:at + e, h * G:h * G + G].double()[..., None]
                        mass[i, h, :T] += x.exp().sum((0, 1))
                    else:
                        y[at + j:at + e, h * G:h * G + G] = torch.softmax(x, -1) @ v
                        lse[at + j:at + e, h * G:h * G + G] = torch.logsumexp(x, -1)
        at += n
    return {"mass": mass} if weigh else {"out": y, "lse": lse}


def _exact_evict(s, case, held):
    H, d, page, keep = case["kv_heads"], case["head_dim"], case["page"], case["keep"]
    out = {"kept": torch.full(s["kept"].shape, -1, dtype=torch.int64, device="cuda"),
           "new_mass": s["new_mass"].double(), "new_lens": torch.full((case["n_seq"],), -1, device="cuda")}
    for name in ("k", "v"):
        out[name + "_pages"] = s[name + "_pages"].double()
        out[name + "_scale"] = s[name + "_scale"].double()
    for i, L in enumerate(held):
        if L < 0:
            continue
        n = min(L, keep)
        out["new_lens"][i] = n
        ids, to = s["table"][i].long(), s["to"][i].long()
        for h in range(H):
            m = s["mass"][i, h, :L].double()
            if L > keep:
                a, b = case["sinks"], L - case["window"]
                middle = m[a:b]
                want = n - a - case["window"]
                # the want-th largest, all above it, and of its equals the first
                edge = middle.sort().values[middle.numel() - want] if want else torch.tensor(math.inf)
                above, equal = middle > edge, middle == edge
                chosen = above | (equal & (equal.cumsum(0) <= want - above.sum()))
                at = torch.cat([torch.arange(a, device="cuda"), a + chosen.nonzero().view(-1),
                                torch.arange(b, L, device="cuda")])
            else:
                at = torch.arange(L, device="cuda")
            out["kept"][i, h, :n] = at
            out["new_mass"][i, h, :n] = m[at]
            for name in ("k", "v"):
                codes, scales = s[name + "_pages"], s[name + "_scale"]
                x = codes.view(torch.uint8)[ids[at // page], h, at % page].view(torch.float8_e4m3fn).double()
                x = x * scales[ids[at // page], h, at % page // BLOCK].double()[:, None]
                x = torch.cat([x, torch.zeros((-n % BLOCK, d), dtype=torch.float64, device="cuda")]).view(-1, BLOCK, d)
                blk = torch.arange(x.shape[0], device="cuda")
                fresh = _pow2(_exponent(x.abs().amax((1, 2))), x)
                out[name + "_scale"][to[blk * BLOCK // page], h, blk % (page // BLOCK)] = fresh
                j = torch.arange(n, device="cuda")
                out[name + "_pages"][to[j // page], h, j % page] = _round_e4m3(x / fresh[:, None, None]).view(-1, d)[:n]
    return out


def exact(case, seed):
    global own
    saved, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = saved
    held, new = _lengths(case)[:2]
    if case["kind"] == "append":
        return _exact_append(s, case, held, new)
    if case["kind"] == "evict":
        return _exact_evict(s, case, held)
    return _exact_rows(s, case, held, new)
