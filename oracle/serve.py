"""The paged cache, the attention that reads it and the verification of the
tree, in plain fp64 numpy: loops over sequences, rows, heads and keys that
follow the definitions in include/dart_cache.h and include/dart_verify.h."""
from __future__ import annotations

import math

import numpy as np

from oracle.tree_attn import root_path, rope


def append(k, v, lens, n_rows, rows, theta):
    """{(sequence, position): (rotated keys, values) [Hkv][dh]} of the tokens
    that a call writes; k, v [nseq][R][Hkv][dh]."""
    got = {}
    for s in range(k.shape[0]):
        for i in range(int(n_rows[s])):
            src = i if rows is None else int(rows[s, i])
            pos = int(lens[s]) + i
            got[s, pos] = rope(k[s, src], pos, theta), v[s, src]
    return got


def attention(q, kt, vt, ctx, parents, depths, n_nodes, lens, theta, scale, rows=None):
    """out [nseq][B + 1][Hq][dh] and what its error bounds need: for every
    row and head the probability-weighted |values| [.., dh] and the largest
    scale * sum |q||k| over the cache's and over the tree's keys.
    ctx[s] = (keys, values) [len][Hkv][dh]; parents [nseq][B] (-1: a child of row 0)."""
    nseq, R, Hq, dh = q.shape
    Hkv = kt.shape[2]
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    grow = np.zeros((nseq, R, Hq, 2))
    for s, r in rows if rows is not None else [(s, r) for s in range(nseq) for r in range(R)]:
        if r > int(n_nodes[s]):
            continue
        at = lambda j: int(lens[s]) + (int(depths[s][j - 1]) if j else 0)  # noqa: E731
        seen = [0] + ([1 + i for i in root_path(parents[s], r - 1)] if r else [])
        kc, vc = ctx[s]
        for h in range(Hq):
            g = h // (Hq // Hkv)
            tree_k = np.stack([rope(kt[s, j, g], at(j), theta) for j in seen])
            keys = np.concatenate([kc[:, g], tree_k])
            vals = np.concatenate([vc[:, g], vt[s, seen, g]])
            x = rope(q[s, r, h], at(r), theta)
            z = scale * keys @ x
            w = np.exp(z - z.max())
            w /= w.sum()
            out[s, r, h], mag[s, r, h] = w @ vals, w @ np.abs(vals)
            a = scale * np.abs(keys) @ np.abs(x)
            grow[s, r, h] = a[:kc.shape[0]].max(initial=0.0), a[kc.shape[0]:].max()
    return out, mag, grow


def verify(logits, tokens, parents, n_nodes, T, u=None, noise=None):
    """Per sequence (rows kept, tokens after them, their log p)."""
    nseq, R, V = logits.shape
    got = []
    for s in range(nseq):
        rows, toks, logp, row = [], [], [], 0
        while True:
            z = np.nan_to_num(logits[s, row].astype(np.float64), nan=-np.inf, posinf=float(np.finfo(np.float32).max), neginf=-np.inf)
            top = z.max()
            dead = top == -np.inf
            e = np.zeros(V) if dead else np.exp((z - top) / (T or 1.0))
            kids, seen = [], set()
            for i in range(int(n_nodes[s])):
                p, t = int(parents[s, i]), int(tokens[s, i])
                if p + 1 == row and -1 <= p < i and 0 <= t < V and t not in seen:
                    kids.append(i)
                    seen.add(t)
            keep, nxt = None, -1
            if T == 0:
                nxt = -1 if dead else int(np.argmax(z))
                keep = next((i for i in kids if int(tokens[s, i]) == nxt), None)
            else:
                left = float(u[s, row]) * e.sum()
                for i in kids:
                    left -= e[int(tokens[s, i])]
                    if left < 0:
                        keep = i
                        break
                rest = z.copy()
                rest[list(seen)] = -np.inf
                rest[e < 2.0 ** -126] = -np.inf
                if keep is None and rest.max() == -np.inf:
                    keep = next((i for i in reversed(kids) if e[int(tokens[s, i])] > 0), None)
                if keep is None and rest.max() > -np.inf:
                    nxt = int(np.argmax((rest - top) / T - np.log(noise[s].astype(np.float64))))
            if keep is not None:
                nxt = int(tokens[s, keep])
            rows.append(row)
            toks.append(nxt)
            logp.append(0.0 if nxt < 0 else (z[nxt] - top) / (T or 1.0) - math.log(e.sum()))
            if keep is None:
                break
            row = keep + 1
        got.append((rows, toks, logp))
    return got
