"""The serving step around the draft tree, as cases that can be timed and compared.

A speculative-decoding round builds a draft tree (dart.Dart), runs the target
model over it, keeps the branch that the target agrees with and goes on from
there.  Three operators do what lies between the tree and the next round:

  attn    dart.PagedTreeAttention: the rows [last token ; tree nodes] of every
          sequence attend to a paged cache (bf16, or e4m3 with a scale per
          token and head) and to their own branch; no nodes is plain decoding
  append  dart.KVCache.append: keys and values of a prompt, or of the rows
          that a round kept, rotated, quantised and written into the pages
  verify  dart.TreeVerifier: which branch the target's probabilities keep and
          which token follows it, from given random numbers

Where `own` is false run() computes them from elementary torch operations in
32 bits (angles in 64); exact() computes them in 64 bits in another way.
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
FMAX = torch.finfo(torch.float32).max
E4M3 = torch.float8_e4m3fn


def _attn(name, nseq, B, C, page, fp8, Hq=32, Hkv=8, L=16, W=16, fill=1.0):
    c = dict(op="attn", nseq=nseq, B=B, C=C, page=page, fp8=fp8, Hq=Hq, Hkv=Hkv, L=L, W=W, fill=fill)
    return dict(c, name=name) if name else c


def _append(name, nseq, R, C, page, fp8, path, Hq=32, Hkv=8):
    c = dict(op="append", nseq=nseq, R=R, C=C, page=page, fp8=fp8, path=path, Hq=Hq, Hkv=Hkv)
    return dict(c, name=name) if name else c


def _verify(name, nseq, B, V, T, bf16, L=16, W=16):
    c = dict(op="verify", nseq=nseq, B=B, V=V, T=T, bf16=bf16, L=L, W=W)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user, one token, a short chat: launches and latency
        _attn("decode-1", 1, 0, 500, 16, False),
        # many users, one token each, ragged lengths, a quantised cache: the bytes of the cache
        _attn("decode-64-e4m3", 64, 0, 8192, 64, True),
        # one user's small tree over a 2048-token context (the narrow benchmark shape)
        _attn("tree-64", 1, 64, 2048, 64, False, W=8),
        # eight users' large trees over ragged contexts, a quantised cache: the tensor cores
        _attn("tree-8x512-e4m3", 8, 512, 4096, 64, True, W=32),
        # one user's tree over a long document: a long axis and few rows
        _attn("tree-16-long", 1, 16, 131072, 128, False, L=8, W=4),
        # other heads, nothing a multiple of a tile, some tree rows unused
        _attn("tree-3x77-e4m3", 3, 77, 1401, 16, True, Hq=16, Hkv=1, L=9, W=11, fill=0.8),
        # the rows that eight users' rounds kept: latency
        _append("commit-8", 8, 257, 2048, 64, True, True),
        # eight users' prompts into a quantised cache: bandwidth
        _append("prompt-8x4096-e4m3", 8, 4096, 0, 64, True, False),
        # a few chunks of prompts that have begun, odd lengths, a bf16 cache
        _append("chunk-5x700", 5, 700, 1300, 16, False, False, 16, 8),
        # the default benchmark's tree, sampling
        _verify("verify-1x256", 1, 256, 151936, 1.0, True),
        # eight users' large trees, sampling at another temperature
        _verify("verify-8x512", 8, 512, 151936, 0.7, True, W=32),
        # a small head's tree, greedy
        _verify("toy-greedy", 1, 16, 4096, 0.0, False, L=4, W=4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "append", "verify"])
    L, W = rng.randint(2, 16), _log(rng, 2, 64)
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (16, 8), (8, 8), (32, 4), (16, 1)])
    page, fp8 = rng.choice([16, 32, 64, 128]), rng.random() < 0.5
    if op == "attn":
        B = 0 if rng.random() < 0.35 else min(L * W, _log(rng, 2, 512))
        nseq = _log(rng, 1, 64)
        C = _log(rng, 1, 131072)
        C = max(1, min(C, 64 * 8192 // nseq, 8 * 513 * 4096 // (nseq * (B + 1))))
        return _attn(None, nseq, B, C, page, fp8, Hq, Hkv, L, W, rng.choice([1.0, 0.8]))
    if op == "append":
        path = rng.random() < 0.4
        nseq = _log(rng, 1, 64)
        R = _log(rng, 2, 512) if path else max(1, min(_log(rng, 1, 32768), 32768 // nseq))
        return _append(None, nseq, R, _log(rng, 1, 20000) - 1, page, fp8, path, Hq, Hkv)
    nseq, B = rng.randint(1, 8), max(2, min(L * W, _log(rng, 4, 512)))
    return _verify(None, nseq, B, _log(rng, 1000, 151936), rng.choice([0.0, 0.7, 1.0]), rng.random() < 0.7, L, W)


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
    nseq, B, fill = c["nseq"], c["B"], c.get("fill", 1.0)
    parents, depths = np.full((nseq, B), -2, np.int32), np.zeros((nseq, B), np.int32)
    n_nodes = np.zeros(nseq, np.int32)
    vis = np.zeros((nseq, B, B), bool)
    for s in range(nseq):
        n = B if fill == 1.0 else max(min(B, 1), int(round(fill * B)) - s % 3)
        parents[s], depths[s] = _tree(B, c["L"], c["W"], n, g)
        n_nodes[s] = n
        for i in range(n):
            if parents[s, i] >= 0:
                vis[s, i] = vis[s, parents[s, i]]
            vis[s, i, i] = True
    return parents, depths, n_nodes, vis


def _words(vis):
    """Bit j of row i as 64-bit words."""
    nseq, B, _ = vis.shape
    nw = (B + 63) // 64
    bits = np.zeros((nseq, B, nw * 64), np.uint8)
    bits[:, :, :B] = vis
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int64).reshape(nseq, B, nw)


def _pages(c, need, seed):
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


def _quantise(x):
    """e4m3 values and the scale of every row of the last axis."""
    amax = x.float().abs().amax(-1, keepdim=True)
    scale = torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))
    return (x.float() / scale).to(E4M3), scale[..., 0]


def _pool(c, pool, seed, filled):
    """The pages of the cache: k, v and (e4m3) their scales."""
    shape = (pool, c["Hkv"], c["page"], DH)
    dt = E4M3 if c["fp8"] else torch.bfloat16
    if not filled:
        k, v = torch.zeros(shape, dtype=dt, device=DEV), torch.zeros(shape, dtype=dt, device=DEV)
        ks = torch.zeros(shape[:3], device=DEV) if c["fp8"] else None
        return k, v, ks, None if ks is None else ks.clone()
    g = _gen(seed, 23)
    if not c["fp8"]:
        return _normal(g, shape, dt), _normal(g, shape, dt), None, None
    got = []
    for _ in range(2):
        q, sc = torch.empty(shape, dtype=dt, device=DEV), torch.empty(shape[:3], device=DEV)
        step = max(1, (1 << 26) // math.prod(shape[1:]))
        for r in range(0, pool, step):
            n = min(step, pool - r)
            q[r:r + n], sc[r:r + n] = _quantise(torch.randn((n,) + shape[1:], generator=g, device=DEV))
        got.append((q, sc))
    return got[0][0], got[1][0], got[0][1], got[1][1]


def _attn_inputs(c, seed):
    nseq, B, Hq, Hkv = c["nseq"], c["B"], c["Hq"], c["Hkv"]
    order = np.random.default_rng([int(seed), 3]).permutation(nseq)
    lens = _spread(nseq, c["C"])[order]
    parents, depths, n_nodes, vis = _trees(c, seed)
    most, pool, table = _pages(c, lens.max(), seed)
    k, v, ks, vs = _pool(c, pool, seed, True)
    qkv = _normal(_gen(seed, 31), (nseq, B + 1, Hq + 2 * Hkv, DH), torch.bfloat16)  # as a fused projection leaves them
    return SimpleNamespace(lens=lens, depths=depths, n_nodes=n_nodes, vis=vis, table=table, most=most, k=k, v=v, ks=ks, vs=vs,
                           q=qkv[:, :, :Hq], kt=qkv[:, :, Hq:Hq + Hkv], vt=qkv[:, :, Hq + Hkv:])


def _append_inputs(c, seed):
    nseq, R, Hq, Hkv = c["nseq"], c["R"], c["Hq"], c["Hkv"]
    g = np.random.default_rng([int(seed), 5])
    lens = g.permutation(_spread(nseq, c["C"], 0.5))
    n_rows = _spread(nseq, min(R, 17)) if c["path"] else _spread(nseq, R, 0.75)
    n_rows = g.permutation(np.maximum(n_rows, 1)).astype(np.int32)
    rows = np.full((nseq, R), -1, np.int32)
    for s in range(nseq):  # the last token's row, then the kept nodes' in ascending order
        rows[s, 0] = 0
        rows[s, 1:n_rows[s]] = np.sort(g.permutation(R - 1)[:n_rows[s] - 1] + 1)
    most, pool, table = _pages(c, int(lens.max()) + int(n_rows.max()), seed)
    qkv = _normal(_gen(seed, 37), (nseq, R, Hq + 2 * Hkv, DH), torch.bfloat16)
    return SimpleNamespace(lens=lens, n_rows=n_rows, rows=rows if c["path"] else None, table=table, pool=pool,
                           k=qkv[:, :, Hq:Hq + Hkv], v=qkv[:, :, Hq + Hkv:])


def _verify_inputs(c, seed):
    nseq, B, V, T = c["nseq"], c["B"], c["V"], c["T"]
    g, n = _gen(seed, 41), np.random.default_rng([int(seed), 13])
    parents, _, n_nodes, vis = _trees(c, seed)
    tokens = np.stack([n.permutation(V)[:B] for _ in range(nseq)]).astype(np.int32)
    logits = torch.empty((nseq, B + 1, V), dtype=torch.bfloat16 if c["bf16"] else torch.float32, device=DEV)
    unit = T if T > 0 else 1.0
    for s in range(nseq):
        z = torch.randn((B + 1, V), generator=g, device=DEV) * 2.0
        # the target mostly agrees with the drafter's best branch: the child
        # with the most descendants, or else some other token, stands out
        size = vis[s].sum(0)
        fav = np.full(B + 1, -1)
        for i in range(int(n_nodes[s])):
            p = parents[s, i] + 1
            if fav[p] < 0 or size[i] > size[fav[p]]:
                fav[p] = i
        other = n.integers(0, V, B + 1)
        child = np.where(fav >= 0, tokens[s][fav], other)
        high = math.log(V) + 2.0
        first = np.where(n.random(B + 1) < 0.8, child, other) if T == 0 else child
        rows = torch.arange(B + 1, device=DEV)
        z[rows, _dev(other)] = high + 0.3
        z[rows, _dev(first)] = high + 1.7
        logits[s] = z * unit
    u = torch.rand((nseq, B + 1), generator=g, device=DEV)
    noise = torch.empty((nseq, V), device=DEV).exponential_(generator=g)
    return SimpleNamespace(logits=logits, tokens=_dev(tokens), parents=_dev(parents), n_nodes=_dev(n_nodes),
                           u=u if T > 0 else None, noise=noise if T > 0 else None)


def prepare(case, seed):
    c = case
    if c["op"] == "verify":
        x = _verify_inputs(c, seed)
        s = SimpleNamespace(op="verify", c=c, **vars(x))
    elif c["op"] == "append":
        x = _append_inputs(c, seed)
        k, v, ks, vs = _pool(c, x.pool, seed, False)
        s = SimpleNamespace(op="append", c=c, pool=(k, v, ks, vs), k=x.k, v=x.v, table=_dev(x.table), lens=_dev(x.lens),
                            n_rows=_dev(x.n_rows), rows=None if x.rows is None else _dev(x.rows))
    else:
        x = _attn_inputs(c, seed)
        tree = (None, None, None) if c["B"] == 0 else (_dev(x.depths), _dev(_words(x.vis)), _dev(x.n_nodes))
        s = SimpleNamespace(op="attn", c=c, pool=(x.k, x.v, x.ks, x.vs), q=x.q, kt=x.kt, vt=x.vt, table=_dev(x.table),
                            lens=_dev(x.lens), tree=tree, vis=_dev(x.vis))
    if own:
        from paper_2608_13524_gb300 import dart
        if c["op"] == "verify":
            s.handle = dart.TreeVerifier(c["nseq"], c["B"], c["V"], c["T"])
        else:
            s.cache = dart.KVCache(*s.pool)
            if c["op"] == "attn":
                s.handle = dart.PagedTreeAttention(s.cache, c["nseq"], c["B"], x.most, c["Hq"], rope_theta=THETA)
    return s


# ------------------------------------------------------------ one pass

def _turn(x, pos):
    """Rotate-half RoPE of x [..., heads, dh] at positions pos [...]."""
    freq = THETA ** (-2.0 * torch.arange(DH // 2, dtype=torch.float64, device=DEV) / DH)
    a = pos.double()[..., None, None] * freq
    co, si = torch.cos(a).float(), torch.sin(a).float()
    lo, hi = x.float().split(DH // 2, -1)
    return torch.cat([lo * co - hi * si, hi * co + lo * si], -1)


def _run_attn(s):
    c = s.c
    nseq, B, Hkv, G, page = c["nseq"], c["B"], c["Hkv"], c["Hq"] // c["Hkv"], c["page"]
    k, v, ks, vs = s.pool
    at = s.table.long()

    def read(x, sc):
        y = x[at].float() if sc is None else x.view(torch.uint8)[at].view(E4M3).float() * sc[at][..., None]
        return y.transpose(2, 3).reshape(nseq, -1, Hkv, DH)

    depths, _, n_nodes = s.tree
    rows = torch.arange(B + 1, device=DEV)
    pos, live = s.lens[:, None].long(), torch.ones((nseq, 1), dtype=torch.bool, device=DEV)
    if B:
        pos = torch.cat([pos, pos + depths], 1)
        live = rows[None] <= n_nodes[:, None]
    q = _turn(s.q, pos).view(nseq, B + 1, Hkv, G, DH)
    kt, vt = _turn(s.kt, pos), torch.where(live[:, :, None, None], s.vt.float(), 0.0)
    kc, vc = read(k, ks), read(v, vs)
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
    seq, row = at[:, 0], src[use]
    pos = s.lens[seq].long() + at[:, 1]
    page_of, slot = s.table[seq, pos // page].long(), pos % page
    k, v, ks, vs = s.pool
    for x, pool, scale in ((_turn(s.k[seq, row], pos), k, ks), (s.v[seq, row].float(), v, vs)):
        if scale is None:
            pool[page_of, :, slot] = x.to(torch.bfloat16)
        else:
            val, sc = _quantise(x)
            pool.view(torch.uint8)[page_of, :, slot] = val.view(torch.uint8)
            scale[page_of, :, slot] = sc
    return [x for x in s.pool if x is not None]


def _run_verify(s):
    c = s.c
    nseq, B, V, T = c["nseq"], c["B"], c["V"], c["T"]
    unit = T if T > 0 else 1.0
    z = torch.nan_to_num(s.logits.float(), nan=-math.inf, posinf=FMAX, neginf=-math.inf)
    m = z.amax(-1)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    total = torch.exp((z - m[..., None]) / unit).sum(-1)
    i = torch.arange(B, device=DEV)
    seq = torch.arange(nseq, device=DEV)[:, None]
    live = (i[None] < s.n_nodes[:, None]) & (s.parents >= -1) & (s.tokens >= 0) & (s.tokens < V)
    up = (s.parents + 1).clamp(min=0).long()  # the parent's row
    tok = s.tokens.clamp(0, V - 1).long()
    sib = (up[:, :, None] == up[:, None]) & live[:, :, None] & live[:, None]  # [i][j]: children of one row
    before = sib & (i[None, :] < i[:, None])[None]
    again = (before & (tok[:, :, None] == tok[:, None])).any(-1)  # a token that an earlier sibling has
    zc, mc = z[seq, up, tok], m[seq, up]
    if T > 0:
        e = torch.where(live & ~again, torch.exp((zc - mc) / unit), 0.0)
        mass = (sib & (i[None, :] <= i[:, None])[None]).float() * e[:, None]
        hit = live & ((s.u[seq, up] * total[seq, up]) < mass.sum(-1))
        rest = (z > -math.inf).sum(-1)
        rest = rest.scatter_add(1, up, -(live & ~again & (zc > -math.inf)).long())
        some = (sib & hit[:, None]).any(-1)
        after = sib & (i[None, :] > i[:, None])[None]
        last = live & (e > 0) & ~(after & (e > 0)[:, None]).any(-1)
        take = (hit & ~(before & hit[:, None]).any(-1)) | (last & ~some & (rest[seq, up] == 0))
    else:
        ids = torch.arange(V, device=DEV)
        best = torch.where((z == m[..., None]) & (z > -math.inf), ids, V).amin(-1)
        take = live & ~again & (tok == best[seq, up])
    kept, ptr = take, torch.where(live, up, 0)
    kept = torch.cat([torch.ones((nseq, 1), dtype=torch.bool, device=DEV), kept], 1)  # by row: the last token's is kept
    ptr = torch.cat([torch.zeros((nseq, 1), dtype=torch.long, device=DEV), ptr], 1)
    for _ in range(max(1, B.bit_length())):  # a row is kept if all of its ancestors are
        kept, ptr = kept & torch.gather(kept, 1, ptr), torch.gather(ptr, 1, ptr)
    rows = torch.arange(B + 1, device=DEV)[None].expand(nseq, -1)
    rows = torch.where(kept, rows, B + 1).sort(1).values
    n_rows = kept.sum(1)
    stop = torch.gather(rows, 1, n_rows[:, None] - 1)
    zs, ms = z[seq, stop][:, 0], m[seq, stop]
    if T > 0:
        w = (zs - ms) / unit - torch.log(s.noise)
        mine = live & (up == stop)
        flat = torch.where(mine, tok + seq * V, nseq * V)
        w = torch.cat([w.reshape(-1), w.new_zeros(1)]).index_fill(0, flat.reshape(-1), -math.inf)[:-1].view(nseq, V)
        top = w.amax(1, keepdim=True)
        bonus = torch.where((w == top) & (w > -math.inf), torch.arange(V, device=DEV), V).amin(1)
    else:
        bonus = best[seq, stop][:, 0]
    bonus = torch.where(bonus == V, -1, bonus)
    used = rows <= B
    out_rows = torch.where(used, rows, -1)
    nxt = torch.cat([out_rows[:, 1:], out_rows.new_full((nseq, 1), -1)], 1)
    out_tok = torch.where(nxt > 0, torch.gather(tok, 1, (nxt - 1).clamp(min=0)), -1)
    out_tok.scatter_(1, n_rows[:, None] - 1, bonus[:, None])
    r = rows.clamp(max=B)
    lp = (z[seq, r, out_tok.clamp(min=0)] - m[seq, r]) / unit - torch.log(total[seq, r])
    return dict(n_rows=n_rows.int(), rows=out_rows.int(), tokens=out_tok.int(), logp=torch.where(out_tok >= 0, lp, 0.0))


def run(state):
    s = state
    if s.op == "attn":
        if own:
            return s.handle(s.q, s.kt, s.vt, s.table, s.lens, *s.tree)
        return _run_attn(s)
    if s.op == "append":
        if own:
            s.cache.append(s.k, s.v, s.table, s.lens, s.n_rows, rows=s.rows, rope_theta=THETA)
            return [x for x in s.pool if x is not None]
        return _run_append(s)
    if own:
        return s.handle(s.logits, s.tokens, s.parents, s.n_nodes, u=s.u, noise=s.noise)
    return _run_verify(s)


def work(case):
    c = case
    if c["op"] == "verify":
        # a branch goes on with about 0.75 of the steps: the rows it visits, one read of the noise, the tree and the answer
        n, B, V, size = c["nseq"], c["B"], c["V"], 2 if c["bf16"] else 4
        rows = n * sum(0.75 ** i for i in range(min(c["L"], B) + 1))
        return {"bytes": rows * V * size + (n * V * 4 if c["T"] > 0 else 0) + n * B * 8 + n * (B + 1) * 12, "flops": 3.0 * rows * V}
    Hq, Hkv, size = c["Hq"], c["Hkv"], 1 if c["fp8"] else 2
    per = 2 * Hkv * (DH * size + (4 if c["fp8"] else 0))  # a token's keys and values in the cache
    if c["op"] == "append":
        n = int(np.maximum(_spread(c["nseq"], min(c["R"], 17)) if c["path"] else _spread(c["nseq"], c["R"], 0.75), 1).sum())
        return {"bytes": n * (2 * Hkv * DH * 2 + per), "flops": n * Hkv * (3.0 * DH + (4.0 * DH if c["fp8"] else 0))}
    n, B = c["nseq"], c["B"]
    keys = int(_spread(n, c["C"]).sum())
    rows = 1 + B * c["fill"]
    io = n * (B + 1) * DH * (2 * Hq * 2 + 2 * Hkv * 2) + n * B * (4 + 8 * ((B + 63) // 64))
    return {"bytes": keys * per + io, "flops": 4.0 * DH * Hq * rows * (keys + n * (1 + min(c["L"], B) / 2))}


# ------------------------------------------------------------- 64 bits

def _spin(x, pos):
    """The same rotation as a product of complex numbers, in 64 bits."""
    freq = torch.exp(-math.log(THETA) * 2.0 / DH * torch.arange(DH // 2, dtype=torch.float64, device=DEV))
    by = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos.double()[:, None] * freq)[:, None]
    y = torch.complex(x[..., :DH // 2].double(), x[..., DH // 2:].double()) * by
    return torch.cat([y.real, y.imag], -1)


def _exact_attn(c, seed):
    x = _attn_inputs(c, seed)
    nseq, B, Hq, Hkv, page = c["nseq"], c["B"], c["Hq"], c["Hkv"], c["page"]
    G = Hq // Hkv
    out = torch.zeros((nseq, B + 1, Hq, DH), dtype=torch.float64, device=DEV)
    for s in range(nseq):
        C, n = int(x.lens[s]), 1 + int(x.n_nodes[s])
        pos = C + _dev(np.concatenate([[0], x.depths[s, :n - 1]]))
        see = np.zeros((n, n), bool)
        see[:, 0] = True
        see[1:, 1:] = x.vis[s, :n - 1, :n - 1]
        hide = torch.cat([torch.zeros((n, C), dtype=torch.bool, device=DEV), ~_dev(see)], 1).repeat_interleave(G, 0)
        ids = _dev(x.table[s, :-(-C // page)]).long()
        q, kt = _spin(x.q[s, :n], pos), _spin(x.kt[s, :n], pos)

        def read(pool, scale, h):
            if scale is None:
                return pool[ids, h].reshape(-1, DH)[:C].double()
            y = pool.view(torch.uint8)[ids, h].view(E4M3).reshape(-1, DH)[:C].double()
            return y * scale[ids, h].reshape(-1, 1)[:C].double()

        for h in range(Hkv):
            keys = torch.cat([read(x.k, x.ks, h), kt[:, h]])
            vals = torch.cat([read(x.v, x.vs, h), x.vt[s, :n, h].double()])
            z = q[:, h * G:(h + 1) * G].reshape(n * G, DH) @ keys.T / math.sqrt(DH)
            w = torch.softmax(z.masked_fill_(hide, -math.inf), -1) @ vals
            out[s, :n, h * G:(h + 1) * G] = w.view(n, G, DH)
    return out


def _exact_append(c, seed):
    x = _append_inputs(c, seed)
    shape = (x.pool, c["Hkv"], c["page"])
    k, v = (torch.zeros(shape + (DH,), dtype=torch.float64, device=DEV) for _ in range(2))
    ks, vs = (torch.zeros(shape, dtype=torch.float64, device=DEV) for _ in range(2))
    for s in range(c["nseq"]):
        n = int(x.n_rows[s])
        rows = torch.arange(n, device=DEV) if x.rows is None else _dev(x.rows[s, :n]).long()
        pos = int(x.lens[s]) + torch.arange(n, device=DEV)
        ids = _dev(x.table[s]).long()[pos // c["page"]]
        for y, pool, scale in ((_spin(x.k[s, rows], pos), k, ks), (x.v[s, rows].double(), v, vs)):
            if c["fp8"]:
                amax = y.abs().amax(-1)
                sc = torch.where(amax > 0, amax / 448.0, 1.0)
                y = (y / sc[..., None]).to(E4M3).double()
                scale[ids, :, pos % c["page"]] = sc
            pool[ids, :, pos % c["page"]] = y
    return [k, v, ks, vs] if c["fp8"] else [k, v]


def _exact_verify(c, seed):
    x = _verify_inputs(c, seed)
    nseq, B, T = c["nseq"], c["B"], c["T"]
    unit = T if T > 0 else 1.0
    logp = torch.zeros((nseq, B + 1), dtype=torch.float64, device=DEV)
    tokens, parents, n_nodes = x.tokens.cpu().numpy(), x.parents.cpu().numpy(), x.n_nodes.cpu().numpy()
    for s in range(nseq):
        row = 0
        for step in range(B + 1):
            lp = torch.log_softmax(x.logits[s, row].double() / unit, 0)
            kids = [i for i in range(n_nodes[s]) if parents[s, i] + 1 == row]
            nxt = None
            if T > 0:
                left = float(x.u[s, row])
                for i in kids:
                    left -= math.exp(float(lp[tokens[s, i]]))
                    if left < 0:
                        nxt = i
                        break
                w = lp - torch.log(x.noise[s].double())
                w[_dev(np.array([tokens[s, i] for i in kids], np.int64))] = -math.inf
            else:
                w = lp
            best = int(torch.argmax(w))
            if T == 0:
                best = int(torch.nonzero(w == w.max())[0])
                nxt = next((i for i in kids if tokens[s, i] == best), None)
            logp[s, step] = lp[best if nxt is None else int(tokens[s, nxt])]
            if nxt is None:
                break
            row = nxt + 1
    return dict(n_rows=None, rows=None, tokens=None, logp=logp)


def exact(case, seed):
    c = case
    return {"attn": _exact_attn, "append": _exact_append, "verify": _exact_verify}[c["op"]](c, seed)
