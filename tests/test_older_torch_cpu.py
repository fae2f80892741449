"""A torch without four-bit tensors: the binding is there, with pages of bf16
and e4m3."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import torch
if hasattr(torch, "float4_e2m1fn_x2"):
    del torch.float4_e2m1fn_x2
torch.cuda.current_device = lambda: 0
from types import SimpleNamespace
from paper_2608_13524_gb300 import dart

def fake(shape, dtype):
    return SimpleNamespace(shape=torch.Size(shape), dtype=dtype, dim=lambda: len(shape), get_device=lambda: 0,
                           is_contiguous=lambda: True, data_ptr=lambda: 1 << 20, device="cuda:0")

b, e, s = fake((4, 2, 16, 128), torch.bfloat16), fake((4, 2, 16, 128), torch.float8_e4m3fn), fake((4, 2, 16), torch.float32)
assert dart.KVCache(b, b).c.dtype == dart.DART_KV_BF16
assert dart.KVCache(e, e, s, s).c.dtype == dart.DART_KV_E4M3
zeros = torch.zeros
torch.zeros = lambda *a, device=None, **kw: zeros(*a, **kw)
dart._expect = lambda t, *rest: t.data_ptr()
assert dart.KVCache.new(3, 16, 1).c.dtype == dart.DART_KV_BF16
assert dart.KVCache.new(3, 16, 1, dtype=torch.float8_e4m3fn).c.dtype == dart.DART_KV_E4M3
try:
    dart.KVCache(fake((4, 2, 16, 64), torch.uint8), fake((4, 2, 16, 64), torch.uint8))
except ValueError:
    print("fine")
"""


def test_the_binding_does_without():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "fine", r.stderr[-2000:]
