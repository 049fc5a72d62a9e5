"""dgamma and dbeta of many rows, against bounds that count the additions in a column's longest chain; and gradients from a
checkpoint whose values pass fp16's range."""
import numpy as np
import pytest
import torch

import paper_2301_02959_amd as fs
from oracle import sequence as seq
from test_gpu_sequence import DEV, EPS, TYPES, generator, half_step, host, inside, norm_inputs, pack, width

pytestmark = pytest.mark.gpu


def layout(units, few):
    """Lanes of a row, pieces a lane, rows in flight of the backward pass, by the width; few: 16-bit rows from their checkpoint."""
    wide = [(768, 256, 4), (512, 256, 3), (256, 256, 2), (128, 64, 4), (96, 32, 4), (64, 32, 3), (48, 32, 2), (32, 16, 3)]
    narrow = [(24, 16, 2), (16, 8, 3), (8, 8, 2)] if few else [(16, 32, 1), (8, 16, 1)]
    G, P = next((G, P) for past, G, P in wide + narrow + [(4, 8, 1), (0, 4, 1)] if units > past)
    return G, P, 4 if P == 1 else 2 if G > 64 and P == 2 else 1


def additions(n, units, few):
    """A lane adds the rows that its group walks, a workgroup its groups, the second launch the workgroups' partial sums: 32 threads a
    share each, then those 32.  Up to 8 rounds of a workgroup are one workgroup's.  Rows past 1024 pieces go in 64 shares of rows."""
    if units > 1024:
        shares = min(n, 64)
        return -(-n // shares) + -(-shares // 32) + 32
    G, _, U = layout(units, few)
    groups = 256 // G
    rounds = -(-n // (groups * U))
    if n <= 8 * groups * U:
        return rounds * U + groups
    blocks = min(rounds, 512)
    return -(-rounds // blocks) * U + groups + -(-blocks // 32) + 32


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, units", [(100_003, 1), (60_001, 9), (30_011, 24), (20_011, 33), (20_011, 65), (9_001, 129), (5_003, 257), (4_001, 600), (2_003, 1000),
                                      (2_003, 1025), (300, 257), (31, 600), (700, 1), (700, 40)])
def test_sums_over_many_rows(dtype, n, units):
    D = width(units, dtype)
    x, dy, gamma, beta = norm_inputs(n, D, dtype, units + n)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y, mean, rstd)
    for packed in (False, True):
        dgamma, dbeta = torch.full((D,), 7.0, device=DEV), torch.full((D,), 7.0, device=DEV)
        if packed:
            codes, exps = pack(x)
            fs.fs_seq_norm_bwd_packed(dy, codes, exps, mean, rstd, gamma, dx, dgamma, dbeta)
            X = seq.unpack8(codes.cpu().numpy(), exps.cpu().numpy())
        else:
            fs.fs_seq_norm_bwd(dy, x, mean, rstd, gamma, dx, dgamma, dbeta)
            X = host(x)
        DY = host(dy)
        terms = DY * ((X - host(mean)[:, None]) * host(rstd)[:, None])
        # a term of dgamma: the difference and its product with rstd are rounded, the product with dy in the addition; one of dbeta is exact.
        # Second-order terms: less than (chain + 2)^2 2^-48, under 2^-10 of the bound for chains of up to 2^13.
        chain, more = additions(n, units, packed and dtype != torch.float32), 1 + 2.0 ** -10
        inside(dgamma, terms.sum(0), (chain + 2) * seq.U32 * more * np.abs(terms).sum(0))
        inside(dbeta, DY.sum(0), chain * seq.U32 * more * np.abs(DY).sum(0))


def test_a_checkpoint_past_fp16s_range():
    """65504 is 64 steps of 1024 in its block, 65536: the gradients are those of that value, not of the nearest fp16 number."""
    n, D = 6, 64
    x, dy, gamma, beta = norm_inputs(n, D, torch.float16, 3)
    x[2, 5], x[4, 40] = 65504.0, -65504.0
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    codes, exps = torch.empty(n, D, dtype=torch.int8, device=DEV), torch.empty(n, 2, dtype=torch.uint8, device=DEV)
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y, mean, rstd, codes, exps)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(D, device=DEV), torch.empty(D, device=DEV)
    fs.fs_seq_norm_bwd_packed(dy, codes, exps, mean, rstd, gamma, dx, dgamma, dbeta)
    V = seq.unpack8(codes.cpu().numpy(), exps.cpu().numpy())
    assert V[2, 5] == 65536 and V[4, 40] == -65536
    M, R, DY, G = host(mean), host(rstd), host(dy), host(gamma)
    wx, wg, wb = seq.norm_bwd(DY, V, M, R, G)
    u = np.abs((V - M[:, None]) * R[:, None])
    inside(dgamma, wg, (additions(n, 8, True) + 2) * seq.U32 * (1 + 2.0 ** -10) * (np.abs(DY) * u).sum(0))
    g = np.abs(DY * G)
    # 8 lanes of 8 values: chains of 8 additions, 3 steps over the lanes, one product; a few roundings of every term
    inside(dx, wx, half_step(torch.float16, wx) + 24 * seq.U32 * R[:, None] * (g + g.mean(1, keepdims=True) + u * (g * u).mean(1, keepdims=True)))
    back = torch.empty_like(x)
    fs.fs_seq_unpack8(codes, exps, back)
    assert back[2, 5] == 65504 and back[4, 40] == -65504
