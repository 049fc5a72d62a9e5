"""The layer norm's kernels in the built library are those that some width reaches, no more: which lanes and pieces a lane rows of
a width take, as the dispatch's comment has it, against the kernels' names."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2301_02959_amd as fs

pytestmark = pytest.mark.skipif(not os.path.exists(fs.LIB_PATH) or shutil.which("nm") is None, reason="no built library, or no nm")

ALL = [(1, 4, 4, 1), (5, 8, 8, 1), (9, 16, 16, 1), (17, 32, 32, 1), (33, 64, 64, 1), (65, 128, 64, 2), (129, 256, 64, 4), (257, 512, 256, 2), (513, 1024, 256, 4)]
FORWARD = [(33, 48, 16, 3), (129, 192, 64, 3), (513, 768, 256, 3)]
BACKWARD = [(33, 48, 16, 3), (49, 64, 32, 2), (65, 96, 32, 3), (97, 128, 32, 4), (513, 768, 256, 3)]
BACKWARD_FEW = BACKWARD + [(9, 16, 8, 2), (17, 24, 8, 3), (25, 32, 16, 2)]        # rows of 16-bit types from their checkpoint


def reached(first):
    """(lanes, pieces a lane) of all widths; `first` goes before the rule for all."""
    got = set()
    for units in range(1, 1025):
        got.add(next((G, P) for lo, hi, G, P in first + ALL if lo <= units <= hi))
    return got


def instances(kernel):
    names = subprocess.run(["nm", "-C", "--defined-only", fs.LIB_PATH], capture_output=True, text=True, check=True).stdout
    found = {m.group(1) for m in re.finditer(r"\bfs::%s<([^>]*)>\(" % kernel, names)}
    assert found
    return {tuple(p.strip() for p in f.split(",")) for f in found}


def test_forward():
    want = {(str(dt), str(G), str(P), pack) for dt in range(3) for G, P in reached(FORWARD) for pack in ("true", "false")}
    assert {(dt, G, P, pack) for dt, G, P, U, pack in instances("norm_fwd_kernel")} == want


def test_backward():
    want = {(str(dt), str(G), str(P), packed, small) for dt in range(3) for packed in ("true", "false") for small in ("true", "false")
            for G, P in reached(BACKWARD_FEW if packed == "true" and dt > 0 else BACKWARD)}
    got = {(dt, G, P, packed, small) for dt, G, P, U, packed, small in instances("norm_bwd_kernel")}
    assert got - want == set(), "no width reaches these"
    assert want - got == set(), "the library lacks these"
