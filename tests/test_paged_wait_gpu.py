"""A wait that gives up in one softmax warp alone, while its partner's does not:
both leave, also where the part's rows are no nodes' and the next part has some,
so the call ends and says so in its status.  In the -DDART_DEBUG build, whose
hook takes one wait for failed; nothing waits for longer than in a good run."""
import os
import subprocess
import sys

import pytest
import torch

import four_data as fd
import serve_data as sd
from test_paged_attn_gpu import dart  # noqa: F401

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_release_builds_have_no_hook(dart):  # noqa: F811
    if dart.dart_debug_build():
        pytest.skip("a debug build")
    dart.dart_test_paged_wait(-1, -1)
    with pytest.raises(dart.DartError):
        dart.dart_test_paged_wait(3, 0)


# B, Hq, Hkv: a full query tile and one of 36 rows, whose last two lane quarters have none; five tiles, laid out as f16 first
@pytest.mark.parametrize("B,Hq,Hkv", [(40, 16, 4), (150, 16, 4)])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
def test_one_warp_gives_up(dart, kind, B, Hq, Hkv):  # noqa: F811
    if not dart.dart_debug_build():
        pytest.skip("runs in the debug library's test process")
    lens = [300, 128, 1, 500] * 16
    data = fd.attn_data4 if kind == "e2m1" else lambda *a, **m: sd.attn_data(*a[:4], kind == "e4m3", *a[4:], **m)
    x = data(len(lens), B, lens, 32, Hq, Hkv, 9900 + B)
    att = dart.PagedTreeAttention(dart.KVCache(*[t for t in x.pool if t is not None]), len(lens), B, x.max_pages, x.Hq)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    good = att(*x.dev, x.table, x.d_lens, *x.tree, status=status).clone()
    assert int(status) == 0
    try:
        for warp in range(2, 10):
            for part in range(3):
                dart.dart_test_paged_wait(warp, part)
                status.zero_()
                att(*x.dev, x.table, x.d_lens, *x.tree, status=status)
                assert int(status) == 1, (warp, part)
    finally:
        dart.dart_test_paged_wait(-1, -1)
    status.zero_()
    assert torch.equal(att(*x.dev, x.table, x.d_lens, *x.tree, status=status), good) and int(status) == 0


def test_the_debug_build(dart):  # noqa: F811
    if os.environ.get("DART_TEST_LIBRARY"):
        pytest.skip("already the debug library's test process")
    from paper_2608_13524_gb300 import build
    env = dict(os.environ, DART_TEST_LIBRARY=build.build(debug=True))
    cmd = [sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_paged_wait_gpu.py::test_one_warp_gives_up"]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    tail = (r.stdout[-4000:] + "\n" + r.stderr[-2000:]).strip()
    assert r.returncode == 0, tail
    assert "6 passed" in r.stdout.strip().splitlines()[-1], tail
