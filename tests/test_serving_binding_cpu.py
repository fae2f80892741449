"""The binding of the serving operators: two calls at once."""
import ctypes as C
from types import SimpleNamespace

import torch

from paper_2608_13524_gb300 import dart


def test_a_call_of_a_verifier_keeps_its_own_configuration(monkeypatch):
    """While one thread's call is inside the library (no interpreter lock is
    held there) another's, with logits of another type and stride, must not
    change what the first one reads."""
    seen, ver = [], None

    def library(ref, logits, *rest):
        cfg = C.cast(ref, C.POINTER(dart.DartVerifyConfig)).contents
        before = (cfg.dtype, cfg.ld)
        if not seen:  # the second call begins while this one is here
            seen.append(before)
            call(torch.zeros(1, 3, 12, dtype=torch.bfloat16)[..., :7])
            seen.append((cfg.dtype, cfg.ld))
        else:
            seen.append(before)
        return 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(dart, "_empty", lambda *a, **k: torch.empty(*a, dtype=k["dtype"]))
    monkeypatch.setattr(dart, "lib", lambda: SimpleNamespace(dart_verify_tree=library))
    ver = dart.TreeVerifier(1, 2, 7, 0.0)
    ints = torch.zeros(1, 2, dtype=torch.int32)

    def call(logits):
        ver(logits, ints, ints, torch.zeros(1, dtype=torch.int32), stream=5)

    call(torch.zeros(1, 3, 7))
    assert seen == [(dart.DART_F32, 7), (dart.DART_BF16, 12), (dart.DART_F32, 7)]


def test_the_stride_of_a_single_row_does_not_matter():
    """One row of one sequence: the strides of its dimensions of length 1 may be
    anything, and are no reason to refuse it."""
    flat = torch.zeros(4096, dtype=torch.bfloat16)
    for ss, sr in ((5, 1001), (1, 1), (0, 0), (1001, 3)):
        assert dart._rows(flat.as_strided((1, 1, 2, 128), (ss, sr, 128, 1)), "q", (1, 1, 2, 128), -1) == (flat.data_ptr(), 256)
    # one row each of several sequences: the stride between them; several rows of one: between these
    assert dart._rows(flat.as_strided((3, 1, 2, 128), (264, 7, 128, 1)), "q", (3, 1, 2, 128), -1)[1] == 264
    assert dart._rows(flat.as_strided((1, 3, 2, 128), (7, 264, 128, 1)), "q", (1, 3, 2, 128), -1)[1] == 264
