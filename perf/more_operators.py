"""A cache in four bits and the pages it lives in, as cases that can be timed and compared.

perf/operators.py measures a serving round over pages of bf16 or e4m3.  This
file measures what lets more of it fit and move:

  attn     dart.PagedTreeAttention over pages of e2m1 (two codes a byte, an
           e4m3 scale for every 16 of them, an fp32 scale per token and head):
           single tokens and draft trees
  append   dart.KVCache.append into such pages and dart.KVCache.read, which
           gives the tokens of a cache back as bf16 rows
  fork     dart.PagePool.select and reserve, dart.KVCache.copy_pages: sequences
           become continuations of others, share their pages, get room for
           new rows and a copy of the page that both would write
  compact  dart.PagePool.trim and compact, dart.KVCache.copy_pages: pages of
           tokens that are no more are freed, the ones in use move to the front

Where `own` is false run() computes them from elementary torch operations in
32 bits (64 for angles and for what decides a rounding to few bits); exact()
computes them in 64 bits in another way.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEV = "cuda"
DH = 128
THETA = 1.0e6
E4M3 = torch.float8_e4m3fn
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # magnitudes of the codes 0 .. 7; 8 .. 15 are their negatives


def _attn(name, nseq, B, C, page, Hq=32, Hkv=8, L=16, W=16, fill=1.0):
    c = dict(op="attn", nseq=nseq, B=B, C=C, page=page, Hq=Hq, Hkv=Hkv, L=L, W=W, fill=fill)
    return dict(c, name=name) if name else c


def _append(name, nseq, R, C, page, path, Hq=32, Hkv=8):
    c = dict(op="append", nseq=nseq, R=R, C=C, page=page, path=path, Hq=Hq, Hkv=Hkv)
    return dict(c, name=name) if name else c


def _fork(name, n, kids, rows, C, page, fp8, Hkv=8):
    c = dict(op="fork", n=n, kids=kids, rows=rows, C=C, page=page, fp8=fp8, Hkv=Hkv)
    return dict(c, name=name) if name else c


def _compact(name, nseq, C, page, fp8, used, Hkv=8):
    c = dict(op="compact", nseq=nseq, C=C, page=page, fp8=fp8, used=used, Hkv=Hkv)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user, one token, a short chat: launches and latency
        _attn("decode-1", 1, 0, 500, 16),
        # many users, one token each, ragged lengths: the bytes of the cache
        _attn("decode-64", 64, 0, 8192, 64),
        # one user's small tree over a 2048-token context (the narrow benchmark shape)
        _attn("tree-64", 1, 64, 2048, 64, W=8),
        # eight users' large trees over ragged contexts: the tensor cores
        _attn("tree-8x512", 8, 512, 4096, 64, W=32),
        # one user's tree over a long document: a long axis and few rows
        _attn("tree-16-long", 1, 16, 131072, 128, L=8, W=4),
        # other heads, nothing a multiple of a tile, some tree rows unused
        _attn("tree-3x77", 3, 77, 1401, 16, Hq=16, Hkv=1, L=9, W=11, fill=0.8),
        # the rows that eight users' rounds kept: latency
        _append("commit-8", 8, 257, 2048, 64, True),
        # eight users' prompts: bandwidth
        _append("prompt-8x4096", 8, 4096, 0, 64, False),
        # one user's prompt continued in four ways: latency
        _fork("fork-1x4", 1, 4, 17, 700, 16, True),
        # many users' prompts, eight continuations each
        _fork("fork-32x8", 32, 8, 65, 4096, 64, False),
        # a small pool after a few chats have ended
        _compact("compact-4", 4, 500, 16, False, 0.5),
        # a large pool, half empty: bandwidth
        _compact("compact-64", 64, 8192, 64, True, 0.55),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "append", "fork", "compact"])
    page = rng.choice([16, 32, 64, 128])
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (16, 8), (8, 4), (32, 4), (16, 1)])
    if op == "attn":
        L, W = rng.randint(2, 16), _log(rng, 2, 64)
        B = 0 if rng.random() < 0.35 else min(L * W, _log(rng, 2, 512))
        nseq = _log(rng, 1, 64)
        C = _log(rng, 1, 131072)
        C = max(1, min(C, 64 * 8192 // nseq, 8 * 513 * 4096 // (nseq * (B + 1))))
        return _attn(None, nseq, B, C, page, Hq, Hkv, L, W, rng.choice([1.0, 0.8]))
    if op == "append":
        path = rng.random() < 0.4
        nseq = _log(rng, 1, 64)
        R = _log(rng, 2, 512) if path else max(1, min(_log(rng, 1, 32768), 32768 // nseq))
        return _append(None, nseq, R, _log(rng, 1, 20000) - 1, page, path, Hq, Hkv)
    fp8 = rng.random() < 0.5
    if op == "fork":
        n, kids = _log(rng, 1, 64), rng.randint(1, 8)
        C = max(2, min(_log(rng, 2, 16384), 32 * 8192 // n))
        return _fork(None, n, kids, _log(rng, 1, 65), C, page, fp8, Hkv)
    nseq = _log(rng, 1, 64)
    C = max(2, min(_log(rng, 2, 32768), 32 * 8192 // nseq))
    return _compact(None, nseq, C, page, fp8, rng.choice([0.3, 0.55, 0.9]), Hkv)


# ------------------------------------------------------------------ four bits

def _two(e):
    """2^e in 64 bits, exactly (a power function may be a unit off)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _to_grid(x, bits, low):
    """x >= 0 (64 bits) rounded to `bits` bits below the leading one, steps of
    at least 2^low, ties to even."""
    _, e = torch.frexp(x)  # x in [2^(e-1), 2^e)
    step = _two((e - 1 - bits).clamp(min=low))
    return torch.round(x / step) * step


def _quantise4(x):
    """Rows of 128 numbers (64 bits) as codes of e2m1 (0 .. 15), block scales
    on e4m3's grid and the row's scale: 2^-10 times the power of two at or below
    the row's largest magnitude, so that no block scale exceeds 342."""
    amax = x.abs().amax(-1)
    _, e = torch.frexp(amax)
    scale = torch.where(amax > 0, _two((e - 11).clamp(min=-120)), 1.0)
    y = (x / scale[..., None]).unflatten(-1, (8, 16))  # (by a power of two)
    top = y.abs().amax(-1)
    block = _to_grid(top / torch.full_like(top, 6.0), 3, -9)  # (a quotient: by a number it may be a product with 1 / 6)
    z = torch.where(block[..., None] > 0, y.abs() / block[..., None], 0.0)
    z = _to_grid(z, 1, -1).clamp(max=6.0)
    code = (z > 0.25).int() + (z > 0.75) + (z > 1.25) + (z > 1.75) + (z > 2.5) + (z > 3.5) + (z > 5.0)
    code = torch.where((y < 0) & (z > 0), code + 8, code)
    return code.flatten(-2).to(torch.uint8), block, scale


def _pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _unpack(byte, block, scale, dtype=torch.float32):
    """The numbers that packed codes with their scales stand for."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=dtype, device=DEV)
    v = torch.stack([table[(byte & 15).int()], table[(byte >> 4).int()]], -1).flatten(-2)
    return (v.unflatten(-1, (8, 16)) * block.to(dtype)[..., None]).flatten(-2) * scale.to(dtype)[..., None]


# ------------------------------------------------------------------ inputs

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (int(seed) + 1) + salt)
    return g


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _spread(n, top, low=0.0):
    """n whole numbers spread evenly over (low * top, top], the last one `top`."""
    return np.array([int(round(top * (low + (1.0 - low) * (i + 1) / n))) for i in range(n)], np.int32)


def _tree(B, L, W, n, g):
    """parents (-1: child of the last token, -2: unused) and depths (0:
    unused) of an n-node tree of at most W nodes a level, in level order."""
    parents, depths = np.full(B, -2, np.int32), np.zeros(B, np.int32)
    prev, i, dep = [-1], 0, 1
    while i < n:
        cnt = n - i if dep == L else min(W, n - i)
        for p in np.sort(g.integers(0, len(prev), size=cnt)):
            parents[i], depths[i] = prev[p], dep
            i += 1
        prev, dep = list(range(i - cnt, i)), dep + 1
    return parents, depths


def _trees(c, seed):
    g = np.random.default_rng([int(seed), 7])
    nseq, B, fill = c["nseq"], c["B"], c["fill"]
    depths, n_nodes = np.zeros((nseq, B), np.int32), np.zeros(nseq, np.int32)
    vis = np.zeros((nseq, B, B), bool)
    for s in range(nseq):
        n = B if fill == 1.0 else max(min(B, 1), int(round(fill * B)) - s % 3)
        parents, depths[s] = _tree(B, c["L"], c["W"], n, g)
        n_nodes[s] = n
        for i in range(n):
            if parents[i] >= 0:
                vis[s, i] = vis[s, parents[i]]
            vis[s, i, i] = True
    return depths, n_nodes, vis


def _words(vis):
    """Bit j of row i as 64-bit words."""
    nseq, B, _ = vis.shape
    nw = (B + 63) // 64
    bits = np.zeros((nseq, B, nw * 64), np.uint8)
    bits[:, :, :B] = vis
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int64).reshape(nseq, B, nw)


def _table(c, need, seed):
    """A page table for up to `need` tokens a sequence, its pages anywhere in the pool."""
    g = np.random.default_rng([int(seed), 11])
    most = max(1, -(-int(need) // c["page"]))
    pool = c["nseq"] * most
    return most, pool, g.permutation(pool).astype(np.int32).reshape(c["nseq"], most)


def _normal(g, shape, dtype):
    out = torch.empty(shape, dtype=dtype, device=DEV)
    step = max(1, (1 << 26) // max(1, math.prod(shape[1:])))
    for r in range(0, shape[0], step):
        n = min(step, shape[0] - r)
        out[r:r + n] = torch.randn((n,) + tuple(shape[1:]), generator=g, device=DEV)
    return out


def _empty4(pool, Hkv, page):
    """Pages of codes, block scales and scales, of keys or of values."""
    shape = (pool, Hkv, page)
    return (torch.zeros(shape + (DH // 2,), dtype=torch.uint8, device=DEV), torch.zeros(shape + (8,), device=DEV).to(E4M3),
            torch.zeros(shape, device=DEV))


def _pages4(c, pool, seed):
    """Such pages with numbers in them, rows of different magnitudes."""
    g, got = _gen(seed, 23), []
    for _ in range(2):
        code, block, scale = _empty4(pool, c["Hkv"], c["page"])
        step = max(1, (1 << 24) // (c["Hkv"] * c["page"] * DH))
        for r in range(0, pool, step):
            n = min(step, pool - r)
            x = torch.randn((n, c["Hkv"], c["page"], DH), generator=g, device=DEV)
            x = x * (0.5 + torch.rand((n, c["Hkv"], c["page"], 1), generator=g, device=DEV))
            a, b, d = _quantise4(x.double())
            code[r:r + n], block[r:r + n], scale[r:r + n] = _pack(a), b.to(E4M3), d
        got.append((code, block, scale))
    return got


def _attn_inputs(c, seed):
    nseq, B, Hq, Hkv = c["nseq"], c["B"], c["Hq"], c["Hkv"]
    order = np.random.default_rng([int(seed), 3]).permutation(nseq)
    lens = _spread(nseq, c["C"])[order]
    depths, n_nodes, vis = _trees(c, seed)
    most, pool, table = _table(c, lens.max(), seed)
    k, v = _pages4(c, pool, seed)
    qkv = _normal(_gen(seed, 31), (nseq, B + 1, Hq + 2 * Hkv, DH), torch.bfloat16)  # as a fused projection leaves them
    return SimpleNamespace(lens=lens, depths=depths, n_nodes=n_nodes, vis=vis, table=table, most=most, pk=k, pv=v,
                           q=qkv[:, :, :Hq], kt=qkv[:, :, Hq:Hq + Hkv], vt=qkv[:, :, Hq + Hkv:])


def _append_rows(c):
    """Tokens of each sequence: what a round kept, or a prompt's."""
    return np.maximum(_spread(c["nseq"], min(c["R"], 17)) if c["path"] else _spread(c["nseq"], c["R"], 0.75), 1)


def _append_inputs(c, seed):
    nseq, R, Hq, Hkv = c["nseq"], c["R"], c["Hq"], c["Hkv"]
    g = np.random.default_rng([int(seed), 5])
    lens = g.permutation(_spread(nseq, c["C"], 0.5))
    n_rows = g.permutation(_append_rows(c)).astype(np.int32)
    rows = np.full((nseq, R), -1, np.int32)
    for s in range(nseq):  # the last token's row, then the kept nodes' in ascending order
        rows[s, 0] = 0
        rows[s, 1:n_rows[s]] = np.sort(g.permutation(R - 1)[:n_rows[s] - 1] + 1)
    most, pool, table = _table(c, int(lens.max()) + int(n_rows.max()), seed)
    qkv = _normal(_gen(seed, 37), (nseq, R, Hq + 2 * Hkv, DH), torch.bfloat16)
    return SimpleNamespace(lens=lens, n_rows=n_rows, rows=rows if c["path"] else None, table=table, pool=pool,
                           k=qkv[:, :, Hq:Hq + Hkv], v=qkv[:, :, Hq + Hkv:])


def _pages(n, c, seed):
    """Pages of keys and of values (and their scales) with numbers in them."""
    g, shape = _gen(seed, 43), (n, c["Hkv"], c["page"], DH)
    k, v = (_normal(g, shape, E4M3 if c["fp8"] else torch.bfloat16) for _ in range(2))
    if not c["fp8"]:
        return [k, v]
    return [k, v] + [torch.rand(shape[:3], generator=g, device=DEV) for _ in range(2)]


def _fork_inputs(c, seed):
    """n sequences (a few of their first pages in common, as a system prompt's
    are) and kids times as many empty ones that are to continue them."""
    n, kids, page = c["n"], c["kids"], c["page"]
    g = np.random.default_rng([int(seed), 17])
    nseq = n * (kids + 1)
    lens = np.zeros(nseq, np.int32)
    lens[:n] = g.permutation(_spread(n, c["C"], 0.5))
    lens[:n] = np.maximum(lens[:n] - g.integers(0, page, n), 1)
    held = -(-lens // page)
    most = int(-(-(c["C"] + c["rows"]) // page))
    common = int(held[:n].min()) // 4
    pool = int((-(-_spread(n, c["C"], 0.5) // page)).sum()) * 5 // 4 + n * kids * (2 + c["rows"] // page) + 1
    order = g.permutation(pool).astype(np.int32)
    table, at = np.zeros((nseq, most), np.int32), common
    for s in range(n):
        table[s, :common] = order[:common]
        table[s, common:held[s]] = order[at:at + held[s] - common]
        at += held[s] - common
    parents = np.concatenate([np.arange(n), g.permutation(np.arange(n * kids) % n)]).astype(np.int32)
    n_rows = np.concatenate([np.zeros(n, np.int64), g.integers(1, c["rows"] + 1, n * kids)]).astype(np.int32)
    refs = np.bincount(np.concatenate([table[s, :held[s]] for s in range(nseq)]), minlength=pool).astype(np.int32)
    return SimpleNamespace(nseq=nseq, most=most, pool=pool, table=table, held=held.astype(np.int32), refs=refs, lens=lens,
                           parents=parents, n_rows=n_rows)


def _compact_inputs(c, seed):
    """Sequences whose pages lie anywhere in a pool that is partly empty; some
    have ended, some were rolled back by a few pages."""
    nseq, page = c["nseq"], c["page"]
    g = np.random.default_rng([int(seed), 19])
    old = g.permutation(_spread(nseq, c["C"]))
    held = np.maximum(-(-old // page), 1)
    most = int(held.max())
    pool = int(math.ceil(held.sum() / c["used"])) + 1
    order = g.permutation(pool).astype(np.int32)
    table, at = np.zeros((nseq, most), np.int32), 0
    for s in range(nseq):
        table[s, :held[s]] = order[at:at + held[s]]
        at += held[s]
    kind = g.random(nseq)
    lens = np.where(kind < 0.2, 0, np.where(kind < 0.5, np.maximum(old - g.integers(0, 4 * page, nseq), 1), old)).astype(np.int32)
    refs = np.bincount(order[:at], minlength=pool).astype(np.int32)
    return SimpleNamespace(nseq=nseq, most=most, pool=pool, table=table, held=held.astype(np.int32), refs=refs, lens=lens)


def prepare(case, seed):
    c = case
    if c["op"] == "attn":
        x = _attn_inputs(c, seed)
        tree = (None, None, None) if c["B"] == 0 else (_dev(x.depths), _dev(_words(x.vis)), _dev(x.n_nodes))
        s = SimpleNamespace(op="attn", c=c, pk=x.pk, pv=x.pv, q=x.q, kt=x.kt, vt=x.vt, table=_dev(x.table), lens=_dev(x.lens),
                            tree=tree, vis=_dev(x.vis))
    elif c["op"] == "append":
        x = _append_inputs(c, seed)
        pk, pv = (_empty4(x.pool, c["Hkv"], c["page"]) for _ in range(2))
        back = (c["nseq"], int(x.n_rows.max()), c["Hkv"], DH)
        s = SimpleNamespace(op="append", c=c, pk=pk, pv=pv, k=x.k, v=x.v, table=_dev(x.table), lens=_dev(x.lens),
                            n_rows=_dev(x.n_rows), rows=None if x.rows is None else _dev(x.rows),
                            back=tuple(torch.zeros(back, dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    else:
        x = _fork_inputs(c, seed) if c["op"] == "fork" else _compact_inputs(c, seed)
        s = SimpleNamespace(op=c["op"], c=c, pool=_pages(x.pool, c, seed), lens=_dev(x.lens))
        start = dict(refs=_dev(x.refs), table=_dev(x.table), held=_dev(x.held))
        if c["op"] == "fork":
            s.parents, s.n_rows = _dev(x.parents), _dev(x.n_rows)
        else:
            s.start = start
        if not own:
            s.pages = SimpleNamespace(pairs=torch.full((max(x.nseq, x.pool // 2), 2), -1, dtype=torch.int32, device=DEV),
                                      count=torch.zeros(1, dtype=torch.int32, device=DEV), **{m: t.clone() for m, t in start.items()})
    if own:
        from paper_2608_13524_gb300 import dart
        if c["op"] in ("attn", "append"):
            (k, kb, ks), (v, vb, vs) = s.pk, s.pv
            s.cache = dart.KVCache(k.view(torch.float4_e2m1fn_x2), v.view(torch.float4_e2m1fn_x2), ks, vs, kb, vb)
            if c["op"] == "attn":
                s.handle = dart.PagedTreeAttention(s.cache, c["nseq"], c["B"], x.most, c["Hq"], rope_theta=THETA)
        else:
            s.cache = dart.KVCache(*s.pool)
            s.pages = dart.PagePool(x.pool, c["page"], x.nseq, x.most)
            for m, t in start.items():
                getattr(s.pages, m).copy_(t)
    return s


# ------------------------------------------------------------ one pass

def _turn(x, pos, dtype=torch.float32):
    """Rotate-half RoPE of x [..., heads, dh] at positions pos [...]."""
    freq = THETA ** (-2.0 * torch.arange(DH // 2, dtype=torch.float64, device=DEV) / DH)
    a = pos.double()[..., None, None] * freq
    co, si = torch.cos(a).to(dtype), torch.sin(a).to(dtype)
    lo, hi = x.to(dtype).split(DH // 2, -1)
    return torch.cat([lo * co - hi * si, hi * co + lo * si], -1)


def _run_attn(s):
    c = s.c
    nseq, B, Hkv, G = c["nseq"], c["B"], c["Hkv"], c["Hq"] // c["Hkv"]
    at = s.table.long()

    def read(code, block, scale):
        y = _unpack(code[at], block.view(torch.uint8)[at].view(E4M3), scale[at])
        return y.transpose(2, 3).reshape(nseq, -1, Hkv, DH)

    depths, _, n_nodes = s.tree
    rows = torch.arange(B + 1, device=DEV)
    pos, live = s.lens[:, None].long(), torch.ones((nseq, 1), dtype=torch.bool, device=DEV)
    if B:
        pos = torch.cat([pos, pos + depths], 1)
        live = rows[None] <= n_nodes[:, None]
    q = _turn(s.q, pos).view(nseq, B + 1, Hkv, G, DH)
    kt, vt = _turn(s.kt, pos), torch.where(live[:, :, None, None], s.vt.float(), 0.0)
    kc, vc = read(*s.pk), read(*s.pv)
    inside = torch.arange(kc.shape[1], device=DEV)[None] < s.lens[:, None]  # keys of the context
    vc = torch.where(inside[:, :, None, None], vc, 0.0)
    seen = torch.zeros((nseq, B + 1, B + 1), dtype=torch.bool, device=DEV)
    seen[:, :, 0] = True
    seen[:, 1:, 1:] = s.vis
    seen = torch.cat([inside[:, None].expand(-1, B + 1, -1), seen], 2) & live[:, :, None]
    keys, vals = torch.cat([kc, kt], 1), torch.cat([vc, vt], 1)
    z = torch.einsum("sihgd,sjhd->shgij", q, keys) * DH ** -0.5
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    p = torch.where(seen[:, None, None], p / p.sum(-1, keepdim=True), 0.0)
    out = torch.einsum("shgij,sjhd->sihgd", p, vals)
    return out.reshape(nseq, B + 1, c["Hq"], DH).to(torch.bfloat16)


def _run_append(s):
    c = s.c
    nseq, R, page = c["nseq"], c["R"], c["page"]
    i = torch.arange(R, device=DEV)[None].expand(nseq, R)
    use = i < s.n_rows[:, None]
    src = i if s.rows is None else s.rows.long()
    at = torch.nonzero(use)
    seq, tok, row = at[:, 0], at[:, 1], src[use]
    pos = s.lens[seq].long() + tok
    page_of, slot = s.table[seq, pos // page].long(), pos % page
    # a code is decided by comparisons: the rotated keys in 64 bits
    for x, (code, block, scale) in ((_turn(s.k[seq, row], pos, torch.float64), s.pk), (s.v[seq, row].double(), s.pv)):
        q, b, d = _quantise4(x)
        code[page_of, :, slot] = _pack(q)
        block.view(torch.uint8)[page_of, :, slot] = b.to(E4M3).view(torch.uint8)
        scale[page_of, :, slot] = d.float()
    for (code, block, scale), out in zip((s.pk, s.pv), s.back):
        got = _unpack(code[page_of, :, slot], block.view(torch.uint8)[page_of, :, slot].view(E4M3), scale[page_of, :, slot])
        out[seq, tok] = got.to(torch.bfloat16)
    return s.back


def _copy_pages(pool, pairs, count):
    use = torch.arange(pairs.shape[0], device=DEV) < count
    src, dst = pairs[use].long().unbind(1)
    for x in pool:
        raw = x.view(torch.uint8)
        raw[dst] = raw[src]


def _plain_select(p, parents, lens, page):
    most = p.table.shape[1]
    i = torch.arange(most, device=DEV)[None]
    me = torch.arange(parents.shape[0], device=DEV)
    src = parents.clamp(min=0).long()
    other = parents != me
    gone = other[:, None] & (i < p.held[:, None])
    keep = torch.where(parents >= 0, torch.minimum(p.held[src], (lens[src] + page - 1) // page), 0)
    come = other[:, None] & (i < keep[:, None])
    theirs = p.table[src]
    p.refs.index_add_(0, p.table[gone].long(), torch.full_like(p.table[gone], -1))
    p.refs.index_add_(0, theirs[come].long(), torch.ones_like(theirs[come]))
    p.table.copy_(torch.where(come, theirs, p.table))
    p.held.copy_(torch.where(other, keep, p.held))
    lens.copy_(torch.where(other, torch.where(parents >= 0, lens[src], 0), lens))


def _plain_reserve(p, lens, n_rows, page):
    most = p.table.shape[1]
    i = torch.arange(most, device=DEV)[None]
    first = lens // page
    need = torch.where(n_rows > 0, (lens + n_rows + page - 1) // page, 0)
    have = i < p.held[:, None]
    at = torch.where(have, p.table, 0).long()
    shared = have & (p.refs[at] > 1)
    span = (i >= torch.minimum(first, p.held)[:, None]) & (i < need[:, None])
    fresh = span & (~have | shared) & (need <= most)[:, None]
    count = fresh.sum(1)
    free = p.refs == 0
    fresh &= (torch.cumsum(count, 0) <= free.sum())[:, None]
    number = torch.cumsum(fresh.flatten(), 0).view_as(fresh) - 1  # of the new pages, by sequence and place
    by_rank = torch.nonzero(free)[:, 0]
    page_of = by_rank[number[fresh]].int()
    old = fresh & shared
    pair = old & (i == first[:, None]) & (lens % page != 0)[:, None]
    table = p.table.clone()
    table[fresh] = page_of
    n = pair.sum()
    p.pairs[:p.pairs.shape[0]][torch.arange(p.pairs.shape[0], device=DEV) < n] = torch.stack([p.table[pair], table[pair]], 1)
    p.count.copy_(n[None])
    p.refs.index_add_(0, p.table[old].long(), torch.full_like(p.table[old], -1))
    p.refs.index_add_(0, page_of.long(), torch.ones_like(page_of))
    p.table.copy_(table)
    p.held.copy_(torch.maximum(p.held, torch.where(fresh.any(1), need, 0)))


def _plain_trim(p, lens, page):
    i = torch.arange(p.table.shape[1], device=DEV)[None]
    need = torch.minimum(p.held, (lens + page - 1) // page)
    gone = p.table[(i >= need[:, None]) & (i < p.held[:, None])]
    p.refs.index_add_(0, gone.long(), torch.full_like(gone, -1))
    p.held.copy_(need)


def _plain_compact(p):
    at = torch.arange(p.refs.shape[0], device=DEV)
    live = p.refs > 0
    n = live.sum()
    moved = at[live & (at >= n)]
    to = at[~live & (at < n)]
    new = at.clone()
    new[moved] = to
    have = torch.arange(p.table.shape[1], device=DEV)[None] < p.held[:, None]
    p.table.copy_(torch.where(have, new[torch.where(have, p.table, 0).long()].int(), p.table))
    refs = torch.zeros_like(p.refs)
    refs[new[live]] = p.refs[live]
    p.refs.copy_(refs)
    p.pairs[:moved.shape[0]] = torch.stack([moved, to], 1).int()
    p.count.fill_(moved.shape[0])


def run(state):
    s = state
    if s.op == "attn":
        if own:
            return s.handle(s.q, s.kt, s.vt, s.table, s.lens, *s.tree)
        return _run_attn(s)
    if s.op == "append":
        if not own:
            return _run_append(s)
        s.cache.append(s.k, s.v, s.table, s.lens, s.n_rows, rows=s.rows, rope_theta=THETA)
        s.cache.read(*s.back, s.table, s.lens, s.n_rows)
        return s.back
    p, page = s.pages, s.c["page"]
    if s.op == "fork":  # continuations of an earlier pass end here: every pass is the same
        if own:
            p.select(s.parents, s.lens)
            s.cache.copy_pages(*p.reserve(s.lens, s.n_rows))
        else:
            _plain_select(p, s.parents, s.lens, page)
            _plain_reserve(p, s.lens, s.n_rows, page)
            _copy_pages(s.pool, p.pairs, p.count)
        return dict(refs=p.refs, table=p.table, held=p.held, lens=s.lens, pairs=p.pairs, count=p.count, pool=s.pool)
    for m, t in s.start.items():  # a compact pool has nothing to move: as it was before
        getattr(p, m).copy_(t)
    if own:
        p.trim(s.lens)
        s.cache.copy_pages(*p.compact())
    else:
        _plain_trim(p, s.lens, page)
        _plain_compact(p)
        _copy_pages(s.pool, p.pairs, p.count)
    return dict(refs=p.refs, table=p.table, held=p.held, pairs=p.pairs, count=p.count, pool=s.pool)


def work(case):
    c = case
    if c["op"] in ("attn", "append"):
        Hq, Hkv = c["Hq"], c["Hkv"]
        per = 2 * Hkv * (DH // 2 + 8 + 4)  # a token's keys and values in the cache
    if c["op"] == "append":
        # rows in, pages out and in again, rows out
        n = int(_append_rows(c).sum())
        return {"bytes": n * (2 * 2 * Hkv * DH * 2 + 2 * per), "flops": n * Hkv * 9.0 * DH}
    if c["op"] == "attn":
        n, B = c["nseq"], c["B"]
        keys = int(_spread(n, c["C"]).sum())
        rows = 1 + B * c["fill"]
        io = n * (B + 1) * DH * (2 * Hq * 2 + 2 * Hkv * 2) + n * B * (4 + 8 * ((B + 63) // 64))
        return {"bytes": keys * per + io, "flops": 4.0 * DH * Hq * rows * (keys + n * (1 + min(c["L"], B) / 2))}
    size = 2 * c["Hkv"] * c["page"] * (DH + 4 if c["fp8"] else 2 * DH)  # of a page
    if c["op"] == "fork":
        x = _fork_inputs(c, 0)
        return {"bytes": 2 * size * x.nseq * c["kids"] / (c["kids"] + 1) + 4 * (2 * int(x.held.sum()) * c["kids"] + 2 * x.pool), "flops": 0}
    x = _compact_inputs(c, 0)
    live = int(np.minimum(x.held, -(-x.lens // c["page"])).sum())
    return {"bytes": 2 * size * live * (1.0 - live / x.pool) + 4 * (2 * int(x.held.sum()) + 3 * x.pool), "flops": 0}


# ------------------------------------------------------------- 64 bits

def _spin(x, pos):
    """The same rotation as a product of complex numbers, in 64 bits."""
    freq = torch.exp(-math.log(THETA) * 2.0 / DH * torch.arange(DH // 2, dtype=torch.float64, device=DEV))
    by = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos.double()[:, None] * freq)[:, None]
    y = torch.complex(x[..., :DH // 2].double(), x[..., DH // 2:].double()) * by
    return torch.cat([y.real, y.imag], -1)


def _nearest(grid, x):
    """Index of the value of an ascending grid next to x, the even one at a tie."""
    mid = (grid[1:] + grid[:-1]) / 2
    a, b = torch.searchsorted(mid, x.contiguous()), torch.searchsorted(mid, x.contiguous(), right=True)
    return torch.where(a % 2 == 0, a, b)


def _exact4(x):
    """What rows of 128 numbers are after a round trip through four bits."""
    e4m3 = torch.tensor([i * 2.0 ** -9 for i in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1],
                        dtype=torch.float64, device=DEV)
    e2m1 = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
    top = x.abs().amax(-1, keepdim=True)
    unit = (top / torch.frexp(top).mantissa * 2.0 ** -11).clamp(min=2.0 ** -120)
    unit = torch.where(top > 0, unit, 1.0)
    y = x.unflatten(-1, (8, 16))
    b = e4m3[_nearest(e4m3, y.abs().amax(-1) / (6 * unit))][..., None] * unit[..., None]
    z = e2m1[_nearest(e2m1, y.abs() / torch.where(b > 0, b, math.inf))]
    return (torch.sign(y) * z * b).flatten(-2)


def _exact_attn(c, seed):
    x = _attn_inputs(c, seed)
    nseq, B, Hq, Hkv, page = c["nseq"], c["B"], c["Hq"], c["Hkv"], c["page"]
    G = Hq // Hkv
    out = torch.zeros((nseq, B + 1, Hq, DH), dtype=torch.float64, device=DEV)
    values = torch.tensor([(v if h < 8 else -v) for h in range(16) for v in [E2M1[h % 8]]], dtype=torch.float64, device=DEV)
    for s in range(nseq):
        C, n = int(x.lens[s]), 1 + int(x.n_nodes[s])
        pos = C + _dev(np.concatenate([[0], x.depths[s, :n - 1]]))
        see = np.zeros((n, n), bool)
        see[:, 0] = True
        see[1:, 1:] = x.vis[s, :n - 1, :n - 1]
        hide = torch.cat([torch.zeros((n, C), dtype=torch.bool, device=DEV), ~_dev(see)], 1).repeat_interleave(G, 0)
        ids = _dev(x.table[s, :-(-C // page)]).long()
        q, kt = _spin(x.q[s, :n], pos), _spin(x.kt[s, :n], pos)

        def read(code, block, scale, h):
            byte = code[ids, h].reshape(-1, DH // 2)[:C].long()
            y = torch.empty((C, DH), dtype=torch.float64, device=DEV)
            y[:, 0::2], y[:, 1::2] = values[byte % 16], values[byte // 16]
            b = block.view(torch.uint8)[ids, h].view(E4M3).reshape(-1, 8)[:C].double() * scale[ids, h].reshape(-1, 1)[:C].double()
            return y * b.repeat_interleave(16, 1)

        for h in range(Hkv):
            keys = torch.cat([read(*x.pk, h), kt[:, h]])
            vals = torch.cat([read(*x.pv, h), x.vt[s, :n, h].double()])
            z = q[:, h * G:(h + 1) * G].reshape(n * G, DH) @ keys.T / math.sqrt(DH)
            w = torch.softmax(z.masked_fill_(hide, -math.inf), -1) @ vals
            out[s, :n, h * G:(h + 1) * G] = w.view(n, G, DH)
    return out


def _exact_append(c, seed):
    x = _append_inputs(c, seed)
    back = [torch.zeros((c["nseq"], int(x.n_rows.max()), c["Hkv"], DH), dtype=torch.float64, device=DEV) for _ in range(2)]
    for s in range(c["nseq"]):
        n = int(x.n_rows[s])
        rows = torch.arange(n, device=DEV) if x.rows is None else _dev(x.rows[s, :n]).long()
        pos = int(x.lens[s]) + torch.arange(n, device=DEV)
        back[0][s, :n], back[1][s, :n] = _exact4(_spin(x.k[s, rows], pos)), _exact4(x.v[s, rows].double())
    return tuple(back)


def _exact_moves(c, seed):
    """The pages after the copies, from sets and dicts."""
    page, moves = c["page"], {}
    if c["op"] == "fork":
        x = _fork_inputs(c, seed)
        free = iter([p for p in range(x.pool) if x.refs[p] == 0])
        users = x.refs.copy()
        for s in range(c["n"], x.nseq):
            p = int(x.parents[s])
            for j in range(int(x.held[p])):
                users[x.table[p, j]] += 1
        for s in range(c["n"], x.nseq):
            p = int(x.parents[s])
            for j in range(int(x.lens[p]) // page, -(-(int(x.lens[p]) + int(x.n_rows[s])) // page)):
                new = next(free)
                if j < x.held[p] and x.lens[p] % page:
                    moves[new] = int(x.table[p, j])
    else:
        x = _compact_inputs(c, seed)
        live = sorted(int(x.table[s, j]) for s in range(x.nseq) for j in range(min(int(x.held[s]), -(-int(x.lens[s]) // page))))
        taken = set(live)
        holes = iter([p for p in range(len(live)) if p not in taken])
        moves = {next(holes): p for p in live if p >= len(live)}
    pool = _pages(x.pool, c, seed)
    src, dst = (_dev(np.array(list(v), np.int64)) for v in (moves.values(), moves.keys()))
    got = []
    for t in pool:
        y = t.double()
        y[dst] = t.view(torch.uint8)[src].view(t.dtype).double()
        got.append(y)
    return got


def exact(case, seed):
    c = case
    if c["op"] == "attn":
        return _exact_attn(c, seed)
    if c["op"] == "append":
        return _exact_append(c, seed)
    whole = dict(refs=None, table=None, held=None, pairs=None, count=None, pool=_exact_moves(c, seed))
    return dict(whole, lens=None) if c["op"] == "fork" else whole
