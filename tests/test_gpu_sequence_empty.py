"""The recurrence over batches in which most sequences have no rows: many of them inside a tile, in front of one, behind the last."""
import numpy as np
import pytest
import torch

import paper_2301_02959_amd as fs
from test_gpu_sequence import DEV, check_scan, offsets_of

pytestmark = pytest.mark.gpu


def gaps(k, length, count):
    return ([length] + [0] * k) * count


# a tile holds 64 to 1024 rows; its first 64 sequences, up to 8 rounds of 256 more, and past those each row's own are three paths
BATCHES = {"after 64": [1] * 64 + [0] * 3 + [5], "65 in a tile": gaps(64, 1, 3), "ones": [1] * 3000, "ones and none": [1, 0] * 2000,
           "one in ten": gaps(9, 7, 400), "one in a hundred": gaps(100, 3, 300), "gaps of a round": gaps(256, 9, 12),
           "gaps of rounds": gaps(1000, 30, 20), "either side of the rows' own": sum((gaps(k, 128, 3) for k in range(2106, 2118)), []) + [3],
           "gaps of many": gaps(20000, 37, 5), "long in front": [0] * 70000 + [5, 200], "long behind": [200, 5] + [0] * 70000,
           "long between": [100] + [0] * 70000 + [100], "one long over gaps": [0] * 20000 + [3000] + [0] * 20000 + [1]}


@pytest.mark.parametrize("name", list(BATCHES))
def test_batches_with_many_empty_sequences(name):
    lengths = BATCHES[name]
    check_scan(lengths, 8, torch.bfloat16, len(lengths), packed=(True,))
    check_scan(lengths, 64, torch.float32, len(lengths), packed=(False,))


@pytest.mark.parametrize("units", [1, 3, 8, 16, 17, 33])
def test_a_thousand_rows_in_many_sequences(units):
    rng = np.random.default_rng(units)
    lengths = np.bincount(rng.integers(0, 32768, 1000), minlength=32768).tolist()
    for dtype in (torch.float32, torch.float16):
        check_scan(lengths, units * (4 if dtype == torch.float32 else 8), dtype, units, carried=units % 2 == 1, packed=(False,))


@pytest.mark.parametrize("D", [8, 64])
def test_bad_offsets_of_many_sequences_stay_in_bounds(D):
    """Offsets in no order, past the rows, negative, on every path of the marks: reported, and nothing past the outputs is touched."""
    n, rng = 700, np.random.default_rng(D)
    x = torch.randn(n + 2, D, device=DEV)
    gate = torch.randn(n + 2, D, device=DEV)
    for S in (200, 3000, 40000):
        good = offsets_of(np.bincount(rng.integers(0, S, n), minlength=S))
        turned = good[::-1].copy()
        dealt = rng.permutation(good)
        wild = rng.integers(-(1 << 40), 1 << 40, S + 1)
        wild[0], wild[-1] = 0, n
        high = good.copy()
        high[S // 2:] += 5
        for bad in (turned, dealt, wild, high, np.full(S + 1, -3), np.full(S + 1, n)):
            off = torch.from_numpy(np.ascontiguousarray(bad)).to(DEV)
            st = torch.zeros(1, dtype=torch.int32, device=DEV)
            h, dx, dg = (torch.full((n + 2, D), 3.0, device=DEV) for _ in range(3))
            last, d0 = (torch.full((S + 2, D), 3.0, device=DEV) for _ in range(2))
            fs.fs_seq_scan_fwd(x[1:-1], gate[1:-1], off, 1, S, None, h[1:-1], last[1:-1], st)
            assert int(st.item()) == fs.FS_DEV_BAD_OFFSETS
            st.zero_()
            fs.fs_seq_scan_bwd(x[1:-1], None, x[1:-1], gate[1:-1], x[1:-1], off, 1, S, None, dx[1:-1], dg[1:-1], d0[1:-1], st)
            assert int(st.item()) == fs.FS_DEV_BAD_OFFSETS
            for t in (h, dx, dg, last, d0):
                assert (t[0] == 3).all() and (t[-1] == 3).all()


@pytest.mark.parametrize("dtype, D", [(torch.bfloat16, 8), (torch.float32, 64), (torch.float16, 136)])
def test_the_most_sequences_a_call_admits(dtype, D):
    """2^31 - 1 sequences, four of them with rows: the bits of a batch of those four."""
    S, at = (1 << 31) - 1, {0: 200, 7: 3, 1 << 30: 500, (1 << 31) - 2: 64}
    few = torch.from_numpy(offsets_of(list(at.values()))).to(DEV)
    n = int(few[-1])
    many = torch.empty(S + 1, dtype=torch.int64, device=DEV)
    edges = [0] + [s + 1 for s in at] + [S + 1]
    for i in range(len(edges) - 1):
        many[edges[i]:edges[i + 1]] = int(few[i])
    assert int(many[-1]) == n
    x, gate, dh = (torch.randn(n, D, device=DEV).to(dtype) for _ in range(3))
    got = []
    for off, T, B in ((few, 4, 1), (many, 1, S)):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        h, dx, dg = (torch.full_like(x, 7.0) for _ in range(3))
        fs.fs_seq_scan_fwd(x, gate, off, T, B, None, h, None, st)
        fs.fs_seq_scan_bwd(dh, None, x, gate, h, off, T, B, None, dx, dg, None, st)
        assert int(st.item()) == 0
        got.append((h, dx, dg))
    for a, b in zip(*got):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    del many
    torch.cuda.empty_cache()
