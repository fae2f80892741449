"""Inputs of the paged cache's tests: numpy arrays as the oracle takes them and
the same on the GPU.  Everything that a call must not use (slots past a
sequence's length, rows past its last node, mask bits of such rows) holds NaN
or garbage."""
from types import SimpleNamespace

import numpy as np
import torch

import canary

DH = 128
E4M3 = torch.float8_e4m3fn


def bf16(g, shape, scale=1.0):
    """Normal numbers that are bf16 values, as a float32 tensor."""
    return torch.from_numpy(g.standard_normal(shape).astype(np.float32) * scale).to(torch.bfloat16).float()


def random_tree(B, n, g, fanout=4):
    parents, depths = np.full(B, -2, np.int32), np.full(B, 12345, np.int32)
    for i in range(n):
        parents[i] = int(g.integers(max(-1, i - fanout * 2), i)) if i else -1
        depths[i] = 1 if parents[i] < 0 else depths[parents[i]] + 1
    return parents, depths


def mask_words(parents, n, B, g):
    """Ancestor bits as emitted, plus garbage bits of rows that are no node."""
    nw = (B + 63) // 64
    bits = np.zeros((B, nw * 64), np.uint8)
    bits[:, n:] = g.integers(0, 2, (B, nw * 64 - n))
    for i in range(n):
        j = i
        while j >= 0:
            bits[i, j] = 1
            j = parents[j]
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int64).reshape(B, nw)


def pool_of(tables, lens, page, Hkv, num_pages, fp8, g, scale=1.0):
    """A pool with the sequences' tokens in it and NaN in every other slot;
    returns the device tensors and ctx[s] = (keys, values) in fp64."""
    shape = (num_pages, Hkv, page, DH)
    if fp8:
        raw = [torch.full(shape, 0x7F, dtype=torch.uint8) for _ in range(2)]  # the NaN code
        scales = [torch.full(shape[:3], float("nan")) for _ in range(2)]
    else:
        raw = [torch.full(shape, float("nan"), dtype=torch.bfloat16) for _ in range(2)]
        scales = [None, None]
    ctx = []
    for s, n in enumerate(lens):
        pos = np.arange(n)
        at, slot = torch.from_numpy(tables[s][pos // page].astype(np.int64)), torch.from_numpy(pos % page)
        both = []
        for i in range(2):
            x = bf16(g, (n, Hkv, DH), scale)
            if fp8:
                sc = x.abs().amax(-1) / 448.0 * torch.from_numpy(g.uniform(1.0, 3.0, (n, Hkv)).astype(np.float32))
                sc = torch.clamp(sc, min=1e-30)
                code = (x / sc[..., None]).to(E4M3)
                raw[i][at, :, slot] = code.view(torch.uint8)
                scales[i][at, :, slot] = sc
                x = code.double() * sc[..., None].double()
            else:
                raw[i][at, :, slot] = x.to(torch.bfloat16)
            both.append(x.double().numpy())
        ctx.append(tuple(both))
    dev = [r.cuda().view(E4M3) if fp8 else r.cuda() for r in raw]
    return dev + [None if x is None else x.cuda() for x in scales], ctx


def attn_data(nseq, B, lens, page, fp8, Hq, Hkv, seed, fill=1.0, fused=True, q_scale=1.0, spare=3):
    g = np.random.default_rng(seed)
    R = B + 1
    max_pages = max(1, max(-(-n // page) for n in lens)) + 1
    num_pages = nseq * max_pages + spare
    tables = g.permutation(num_pages)[:nseq * max_pages].astype(np.int32).reshape(nseq, max_pages)
    for s, n in enumerate(lens):  # entries that no token needs are not page numbers
        tables[s, -(-n // page):] = 10 ** 9
    pool, ctx = pool_of(tables, lens, page, Hkv, num_pages, fp8, g)
    n_nodes = np.array([B if fill == 1.0 else int(round(fill * B)) * (s % 3 != 2) for s in range(nseq)], np.int32)
    parents, depths = np.full((nseq, B), -2, np.int32), np.zeros((nseq, B), np.int32)
    mask = np.zeros((nseq, B, (B + 63) // 64), np.int64)
    for s in range(nseq):
        if B:
            parents[s], depths[s] = random_tree(B, n_nodes[s], g)
            mask[s] = mask_words(parents[s], n_nodes[s], B, g)
    qkv = bf16(g, (nseq, R, Hq + 2 * Hkv, DH))
    qkv[:, :, :Hq] *= q_scale
    qkv = qkv.to(torch.bfloat16).float()
    for s in range(nseq):
        qkv[s, n_nodes[s] + 1:] = float("nan")
    parts = (qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:])
    if fused:
        d = qkv.to(torch.bfloat16).cuda()
        dev = (d[:, :, :Hq], d[:, :, Hq:Hq + Hkv], d[:, :, Hq + Hkv:])
    else:
        dev = tuple(x.contiguous().to(torch.bfloat16).cuda() for x in parts)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    return SimpleNamespace(q=parts[0].double().numpy(), kt=parts[1].double().numpy(), vt=parts[2].double().numpy(), ctx=ctx,
                           parents=parents, depths=depths, n_nodes=n_nodes, lens=np.array(lens, np.int32), B=B, Hq=Hq,
                           max_pages=max_pages, pool=pool, dev=dev, table=up(tables), d_lens=up(np.array(lens, np.int32)),
                           tree=(up(depths), up(mask), up(n_nodes)) if B else (None, None, None))


def guarded_cache(dart, pool):
    """The pool copied into guarded memory."""
    got = []
    for x in pool:
        if x is None:
            got.append(None)
            continue
        d = canary.empty(tuple(x.shape), dtype=x.dtype)
        d.view(torch.uint8).copy_(x.view(torch.uint8))
        got.append(d)
    return dart.KVCache(*got)
