"""Rows with infinities and NaN: the layer norm's statistics are those of the formula, and only the row's own."""
import numpy as np
import pytest
import torch

import paper_2301_02959_amd as fs
from test_gpu_sequence import DEV, EPS, TYPES, generator, host, rows, same_bits, width

pytestmark = pytest.mark.gpu

# widths in 16-byte pieces whose rows lie in part of a wave, in a wave, in a workgroup, in no registers
UNITS = [1, 9, 16, 40, 65, 150, 300, 600, 1000, 1100]
BAD = {3: [("nan", 0)], 8: [("inf", -1)], 17: [("-inf", 1)], 40: [("inf", 0), ("-inf", -1)], 41: [("nan", 1), ("inf", 0)]}


def statistics(dtype, units, keep):
    """(x, mean, rstd, mean and rstd of the rows without their bad values) of 50 rows, BAD's with what it says in them"""
    D, n = width(units, dtype), 50
    gen = generator(units)
    x = rows(gen, n, D, dtype, 1.5, 0.3)
    gamma, beta = (torch.randn(D, generator=gen).to(DEV) for _ in range(2))
    mean, rstd, clean_mean, clean_rstd = (torch.full((n,), 7.0, device=DEV) for _ in range(4))
    y = torch.empty_like(x)
    kept = (torch.empty(n, D, dtype=torch.int8, device=DEV), torch.empty(n, -(-D // 32), dtype=torch.uint8, device=DEV)) if keep else ()
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y, clean_mean, clean_rstd, *kept)
    for row, values in BAD.items():
        for v, column in values:
            x[row, column] = float(v)
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y, mean, rstd, *kept)
    assert y[list(BAD)].isnan().all()
    return x, mean, rstd, clean_mean, clean_rstd


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("units", UNITS)
def test_rstd_of_a_bad_row_is_nan(dtype, units, keep):
    """(x - mean)^2 of a row with an infinity or a NaN holds a NaN, so 1 / sqrt(its mean + eps) is one."""
    x, mean, rstd, clean_mean, clean_rstd = statistics(dtype, units, keep)
    bad = torch.zeros(len(x), dtype=torch.bool, device=DEV)
    bad[list(BAD)] = True
    assert rstd[bad].isnan().all()
    assert same_bits(rstd[~bad], clean_rstd[~bad]) and same_bits(mean[~bad], clean_mean[~bad]) and rstd[~bad].isfinite().all()


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("units", UNITS)
def test_mean_of_a_row_with_an_infinity(dtype, units, keep):
    """The sum of a row with infinities of one sign is that infinity; with both, or a NaN, it is a NaN."""
    x, mean, *_ = statistics(dtype, units, keep)
    with np.errstate(invalid="ignore"):
        want = host(x).sum(1)[list(BAD)]
    assert np.isnan(want).any() and np.isposinf(want).any() and np.isneginf(want).any()
    got = host(mean)[list(BAD)]
    assert np.array_equal(got, want, equal_nan=True)
