"""The bookkeeping of the decoding kernel's ring of stages (host code): when a
bounded wait runs out, the fills that are still on their way are those from the
failed one on, however many turns pass after it."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

DRIVER = r"""
#include <cstdio>
#include <cstdlib>
#include "dart_ring.h"
int main(int argc, char** argv) {  // turns, the turn whose wait runs out (-1: none)
    const int turns = atoi(argv[1]), bad = atoi(argv[2]);
    dart::StageRing<%d> ring;
    bool failed = false;
    while (ring.filled < turns && ring.room()) ring.filled++;
    for (int i = 0; i < turns; i++) {
        if (i == bad) failed = true;
        if (!failed && ring.used != i) return 1;
        ring.passed(failed);
        if (!failed && ring.filled < turns) ring.filled++;
    }
    for (int i = ring.used; i < ring.filled; i++) printf("%%d:%%d:%%u ", i, ring.stage(i), ring.parity(i));
    return 0;
}
"""


@pytest.mark.parametrize("stages", [2, 3])
def test_fills_on_their_way_when_a_wait_runs_out(tmp_path, stages):
    src, exe = tmp_path / "ring.cpp", tmp_path / "ring"
    src.write_text(DRIVER % stages)
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2608_13524_gb300", "csrc"), str(src), "-o", str(exe)], check=True)

    def left(turns, bad):
        r = subprocess.run([str(exe), str(turns), str(bad)], check=True, capture_output=True, text=True)
        return [tuple(int(x) for x in w.split(":")) for w in r.stdout.split()]

    for turns in (1, 2, 5, 9):
        assert left(turns, -1) == []
        for bad in range(turns):
            want = range(bad, min(turns, bad + stages))
            assert left(turns, bad) == [(i, i % stages, i // stages & 1) for i in want], (turns, bad)
