"""Four-bit pages as a serving program uses them: what stands in a workspace
does not matter, and a captured step of writes, pages and attention gives what
eager calls give."""
import numpy as np
import pytest
import torch

import four_data as fd
import serve_data as sd

pytestmark = pytest.mark.gpu
THETA = 1.0e6


@pytest.fixture(scope="module")
def dart():
    from paper_2608_13524_gb300 import dart as d
    return d


def up(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("B,Hq,Hkv", [(0, 8, 2), (3, 16, 4), (16, 4, 4), (33, 8, 2), (100, 16, 1), (127, 4, 4), (300, 8, 2), (513, 4, 2)])
def test_a_workspace_of_anything(dart, kind, B, Hq, Hkv):
    """NaN, then zeros, in every byte of the workspace: the same bits.  Tails of
    0, 1, 27, 126 and 127 tokens, so that rows before, between and behind the
    tree rows of a tile are met."""
    lens = [0, 1, 127, 128, 155, 254, 641]
    data = fd.attn_data4 if kind == "e2m1" else lambda *a, **m: sd.attn_data(*a[:4], kind == "e4m3", *a[4:], **m)
    x = data(len(lens), B, lens, 32, Hq, Hkv, 9500 + B, fill=0.9)
    att = dart.PagedTreeAttention(dart.KVCache(*[t for t in x.pool if t is not None]), len(lens), B, x.max_pages, x.Hq, rope_theta=THETA)
    got = []
    for fill in (0xFF, 0x00, 0x7F):
        att.workspace.fill_(fill)
        got.append(att(*x.dev, x.table, x.d_lens, *x.tree).clone())
    assert torch.isfinite(got[0].float()).all()
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_a_captured_step(dart):
    """Room for new tokens, copies, writes and attention over them, captured once and
    replayed: three steps give what the same calls give one by one."""
    n, Hq, Hkv, page, R, most = 3, 8, 2, 16, 4, 12
    g = torch.Generator(device="cuda").manual_seed(7)
    rows = [torch.randn((3, n, R, h, 128), generator=g, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv)]
    prompt = [torch.randn((n, 40, Hkv, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]

    def start():
        cache = dart.KVCache.new(40, page, Hkv, dtype=torch.float4_e2m1fn_x2)
        pool = dart.PagePool(40, page, n, most)
        lens, add = up([0] * n), up([40, 0, 0])
        cache.copy_pages(*pool.reserve(lens, add))
        cache.append(*prompt, pool.table, lens, add)
        lens += add
        pool.select(up([0, 0, 0]), lens)  # three continuations of one prompt
        att = dart.PagedTreeAttention(cache, n, 0, most, Hq, rope_theta=THETA)
        one = torch.ones(n, dtype=torch.int32, device="cuda")
        return cache, pool, lens, att, one, [torch.empty((n, 1, h, 128), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv)]

    def step(cache, pool, lens, att, one, dev):
        q, k, v = dev
        cache.copy_pages(*pool.reserve(lens, one))
        out = att(q, k, v, pool.table, lens)
        cache.append(k, v, pool.table, lens, one, rope_theta=THETA)
        lens += one
        return out

    want, state = [], start()
    for i in range(3):
        for d, r in zip(state[5], rows):
            d.copy_(r[i, :, :1])
        want.append(step(*state).clone())
    after = [t.clone() for t in (state[1].refs, state[1].table, state[1].held, state[2], state[0].k.view(torch.uint8), state[0].v_scale)]

    state = start()
    torch.cuda.synchronize()
    keep = [t.clone() for t in (state[1].refs, state[1].table, state[1].held, state[2])]
    pages = [t.view(torch.uint8).clone() for t in (state[0].k, state[0].v, state[0].k_scale, state[0].v_scale, state[0].k_block, state[0].v_block)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*state)
    for t, k in zip((state[1].refs, state[1].table, state[1].held, state[2]), keep):
        t.copy_(k)
    for t, k in zip((state[0].k, state[0].v, state[0].k_scale, state[0].v_scale, state[0].k_block, state[0].v_block), pages):
        t.view(torch.uint8).copy_(k)
    for i in range(3):
        for d, r in zip(state[5], rows):
            d.copy_(r[i, :, :1])
        graph.replay()
        assert torch.equal(out, want[i]), i
    now = (state[1].refs, state[1].table, state[1].held, state[2], state[0].k.view(torch.uint8), state[0].v_scale)
    # (the pages in use: what stands in others may be of the step before the capture)
    for t, w in list(zip(now, after))[:4]:
        assert torch.equal(t, w)
    used = after[0] > 0
    for t, w in list(zip(now, after))[4:]:
        assert torch.equal(t[used], w[used])


def test_pages_behind_four_gigabytes(dart):
    """Writes, reads, copies and attention on the last pages of a pool whose codes
    take 4.6 GB a side: what the same calls give on a small pool."""
    n, Hq, Hkv, page, R = 2, 8, 2, 128, 300
    g = torch.Generator(device="cuda").manual_seed(11)
    kv = [torch.randn((n, R, Hkv, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    got = []
    for num in (8, 280_000):
        shape = (num, Hkv, page)
        k, v = (torch.empty(shape + (64,), dtype=torch.uint8, device="cuda").view(fd.F4) for _ in range(2))
        kb, vb = (torch.empty(shape + (8,), dtype=torch.uint8, device="cuda").view(sd.E4M3) for _ in range(2))
        ks, vs = (torch.empty(shape, device="cuda") for _ in range(2))
        cache = dart.KVCache(k, v, ks, vs, kb, vb)
        table = up(num - 1 - np.arange(6).reshape(n, 3))
        lens, rows = up([0] * n), up([R, R - 51])
        cache.append(*kv, table, lens, rows, rope_theta=THETA)
        pairs, count = up([[num - 1, num - 7], [num - 7, num - 8]]), up([1])
        cache.copy_pages(pairs, count)
        table[0, 0] = num - 7
        back = [torch.zeros_like(kv[0]) for _ in range(2)]
        cache.read(*back, table, lens, rows)
        got.append(back)
        for B in (0, 40, 300):
            h = torch.Generator(device="cuda").manual_seed(B)
            q, kt, vt = (torch.randn((n, B + 1, heads, 128), generator=h, device="cuda").to(torch.bfloat16) for heads in (Hq, Hkv, Hkv))
            tree = (None, None, None)
            if B:
                words = torch.zeros((n, B, (B + 63) // 64), dtype=torch.int64, device="cuda")
                for i in range(B):
                    words[:, i, i // 64] = 1 << (i % 64) if i % 64 < 63 else -(1 << 63)
                tree = (torch.ones((n, B), dtype=torch.int32, device="cuda"), words, up([B, B - 3]))
            att = dart.PagedTreeAttention(cache, n, B, 3, Hq, rope_theta=THETA)
            got[-1].append(att(q, kt, vt, table, rows, *tree).clone())
        torch.cuda.synchronize()
        del cache, k, v, kb, vb, ks, vs, att
    for a, b in zip(*got):
        assert torch.isfinite(a.float()).all() and torch.equal(a, b)
