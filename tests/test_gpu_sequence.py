"""The sequence operators on the GPU against oracle/sequence.py (64 bits).

Tolerances are counted in roundings.  An output is rounded once to its type (half a step: eps / 2 relative, below fp16's
normal numbers 2^-25).  Before that everything is fp32, each operation off by 2^-24 of its result; a sum of k terms in a chain of
c additions is off by c 2^-24 of the sum of the magnitudes.  The recurrence's bounds come with the oracle."""
import numpy as np
import pytest
import torch

import paper_2301_02959_amd as fs
from oracle import sequence as seq

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = [torch.float32, torch.float16, torch.bfloat16]
EPS = 1e-5


def half_step(dtype, v):
    """What the one rounding to `dtype` may take."""
    if dtype == torch.float32:
        return np.abs(v) * seq.U32
    return np.abs(v) * (torch.finfo(dtype).eps / 2) + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def rows(gen, n, D, dtype, std=1.0, mean=0.0):
    return (torch.randn(n, D, generator=gen) * std + mean).to(dtype).to(DEV)


def host(t):
    return t.detach().cpu().double().numpy()


def generator(seed):
    return torch.Generator().manual_seed(seed)


def inside(got, want, bound):
    got = host(got)
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got))
    over = np.abs(got - want)[fine] - bound[fine]
    assert got.shape == want.shape and (over.size == 0 or over.max() <= 0), f"{over.max():.3g} past the bound, {np.abs(got - want)[fine].max():.3g} off"


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def chain(D, dtype):
    """Additions in a row's longest chain: a lane's elements, then the lanes, the waves and a few products."""
    per = 4 if dtype == torch.float32 else 8
    units = -(-D // per)
    return per * (max(1, -(-units // 64)) if units <= 256 else -(-units // 256)) + 16


# widths in 16-byte pieces: one, few, odd ones, whole waves, two and four pieces a lane, past a lane's registers
UNITS = [1, 2, 3, 5, 9, 16, 17, 31, 32, 33, 64, 65, 100, 128, 129, 200, 256, 257, 600]


def width(units, dtype):
    return units * (4 if dtype == torch.float32 else 8)


# ---- checkpoints -----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, units", [(1, 1), (7, 9), (300, 17), (33, 64), (129, 5), (2, 600), (1000, 32)])
def test_pack_and_unpack(dtype, n, units):
    D = width(units, dtype)
    x = rows(generator(n + units), n, D, dtype) * torch.logspace(-4, 3, n).to(DEV)[:, None].to(dtype)
    codes = torch.full((n, D), 99, dtype=torch.int8, device=DEV)
    exps = torch.zeros(n, -(-D // 32), dtype=torch.uint8, device=DEV)
    back = torch.empty_like(x)
    fs.fs_seq_pack8(x, codes, exps)
    fs.fs_seq_unpack8(codes, exps, back)
    want_c, want_e = seq.pack8(host(x))
    assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(exps.cpu().numpy(), want_e)
    want = torch.from_numpy(seq.unpack8(want_c, want_e))
    if dtype == torch.float16:
        want = want.clamp(-65504, 65504)
    assert torch.equal(back.cpu(), want.to(dtype))        # exact before the one rounding (which only fp16's subnormals need)


@pytest.mark.parametrize("dtype", TYPES)
def test_pack_at_the_ends_of_the_range(dtype):
    info = torch.finfo(dtype)
    D = 64
    x = torch.zeros(12, D)
    x[0, :] = info.max
    x[1, 3] = -info.max
    x[2, :] = info.tiny
    x[3, 5] = info.smallest_normal * 2 ** -3               # subnormal in every type
    x[4, 31], x[4, 32] = float("nan"), 3.0
    x[5, 0], x[5, 1], x[5, 63] = float("inf"), -float("inf"), float("-inf")
    x[6, :] = torch.arange(64) - 31.5                       # ties
    x[7, :] = 1.9921875                                     # 127.5 steps: the next step
    x[8, :] = 1.9843750                                     # 127 steps
    x[9, 7] = -0.0
    x[10, :32] = info.smallest_normal * info.eps
    x[11, 0], x[11, 1] = info.max, 1.0
    x = x.to(dtype).to(DEV)
    codes, exps = torch.empty(12, D, dtype=torch.int8, device=DEV), torch.empty(12, 2, dtype=torch.uint8, device=DEV)
    back = torch.empty_like(x)
    fs.fs_seq_pack8(x, codes, exps)
    fs.fs_seq_unpack8(codes, exps, back)
    want_c, want_e = seq.pack8(host(x))
    assert np.array_equal(exps.cpu().numpy(), want_e)
    assert np.array_equal(codes.cpu().numpy(), want_c)
    want = torch.from_numpy(seq.unpack8(want_c, want_e))
    if dtype == torch.float16:
        want = torch.where(torch.isfinite(want), want.clamp(-65504, 65504), want)
    got = back.cpu()
    assert torch.equal(torch.nan_to_num(got, nan=7), torch.nan_to_num(want.to(dtype), nan=7)) and torch.equal(got.isnan(), want.isnan())


def test_unpack_takes_any_bytes():
    """Every pair of a code and an exponent, the ones that no checkpoint holds (code -128, exponent 0) among them."""
    c = torch.arange(-128, 128, dtype=torch.int16).to(torch.int8).repeat(256, 1)
    e = torch.arange(256, dtype=torch.int16).to(torch.uint8)[:, None].repeat(1, 8).contiguous()
    want = torch.from_numpy(seq.unpack8(c.numpy(), e.numpy()))
    for dtype in TYPES:
        back = torch.empty(256, 256, dtype=dtype, device=DEV)
        fs.fs_seq_unpack8(c.to(DEV), e.to(DEV), back)
        w = want
        if dtype == torch.float16:
            w = torch.where(torch.isfinite(w), w.clamp(-65504, 65504), w)
        elif dtype == torch.bfloat16 or dtype == torch.float32:
            w = w.float().double()                          # -128 steps of the largest exponent: past fp32, infinite there too
        got = back.cpu()
        assert torch.equal(got.isnan(), w.isnan())
        assert torch.equal(torch.nan_to_num(got, nan=7), torch.nan_to_num(w.to(dtype), nan=7))


# ---- layer norm ------------------------------------------------------------------------------------------------

def norm_inputs(n, D, dtype, seed, mean=0.3):
    gen = generator(seed)
    x, dy = rows(gen, n, D, dtype, 1.5, mean), rows(gen, n, D, dtype)
    gamma, beta = (torch.randn(D, generator=gen).to(DEV) for _ in range(2))
    return x, dy, gamma, beta


def check_norm(n, D, dtype, seed):
    x, dy, gamma, beta = norm_inputs(n, D, dtype, seed)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    codes, exps = torch.empty(n, D, dtype=torch.int8, device=DEV), torch.empty(n, -(-D // 32), dtype=torch.uint8, device=DEV)
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y, mean, rstd, codes, exps)
    X, G, Bt = host(x), host(gamma), host(beta)
    wy, wm, wr = seq.norm_fwd(X, G, Bt, EPS)
    c = chain(D, dtype) * seq.U32
    size = np.abs(X - wm[:, None])
    # the rounded mean: off by the chain's roundings of the row's magnitudes, twice over (the sum and its product with 1 / D);
    # y is taken about a mean that is corrected by what it is off, so there only the deviations' magnitudes count
    inside(mean, wm, 2 * c * np.abs(X).mean(1) + 1e-30)
    inside(rstd, wr, (c + 8 * seq.U32) * wr)
    inside(y, wy, half_step(dtype, wy) + (2 * c + 8 * seq.U32) * (np.abs(wy) + np.abs(Bt) + (size.mean(1) * wr)[:, None] * np.abs(G) + size * wr[:, None] * np.abs(G)))
    want_c, want_e = seq.pack8(X)
    assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(exps.cpu().numpy(), want_e)
    y2 = torch.empty_like(x)
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y2)              # serving: nothing kept, the same bits
    assert same_bits(y, y2)

    for packed in (False, True):
        dgamma, dbeta = torch.full((D,), 7.0, device=DEV), torch.full((D,), 7.0, device=DEV)
        if packed:
            fs.fs_seq_norm_bwd_packed(dy, codes, exps, mean, rstd, gamma, dx, dgamma, dbeta)
            V = seq.unpack8(want_c, want_e)
        else:
            fs.fs_seq_norm_bwd(dy, x, mean, rstd, gamma, dx, dgamma, dbeta)
            V = X
        M, R, DY = host(mean), host(rstd), host(dy)
        wx, wg, wb = seq.norm_bwd(DY, V, M, R, G)
        g, u = np.abs(DY * G), np.abs((V - M[:, None]) * R[:, None])
        terms = g + g.mean(1, keepdims=True) + u * (g * u).mean(1, keepdims=True)
        inside(dx, wx, half_step(dtype, wx) + (c + 8 * seq.U32) * R[:, None] * terms)
        # a column's chain: the rows a lane walks (of 1024 workgroups with 4 groups or more, 64 chunks of the widest rows), the groups
        # of a workgroup, the workgroups' partial sums; and a few roundings of every term
        per = 4 if dtype == torch.float32 else 8
        links = (160 + (n / 64 if D > 256 * per else n / 4096) + 4) * seq.U32
        inside(dgamma, wg, links * (np.abs(DY) * u).sum(0) + 1e-30)
        inside(dbeta, wb, links * np.abs(DY).sum(0) + 1e-30)
        again = torch.empty_like(dx), torch.empty_like(dgamma), torch.empty_like(dbeta)
        if packed:
            fs.fs_seq_norm_bwd_packed(dy, codes, exps, mean, rstd, gamma, *again)
        else:
            fs.fs_seq_norm_bwd(dy, x, mean, rstd, gamma, *again)
        assert all(same_bits(a, b) for a, b in zip(again, (dx, dgamma, dbeta)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("units", UNITS)
def test_norm_widths(dtype, units):
    check_norm(37, width(units, dtype), dtype, units)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 1000, 4099])
def test_norm_row_counts(n):
    check_norm(n, 64, torch.float32, n)
    check_norm(n, 72, torch.bfloat16, n)


def test_norm_many_rows():
    check_norm(70_001, 40, torch.float16, 5)                 # more rows than one round of the workgroups takes


def test_norm_without_rows():
    D = 64
    x = torch.empty(0, D, device=DEV)
    v, stat = torch.ones(D, device=DEV), torch.empty(0, device=DEV)
    dgamma, dbeta = torch.full((D,), 7.0, device=DEV), torch.full((D,), 7.0, device=DEV)
    fs.fs_seq_norm_fwd(x, v, v, EPS, x, stat, stat)
    fs.fs_seq_norm_bwd(x, x, stat, stat, v, x, dgamma, dbeta)
    assert not dgamma.any() and not dbeta.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("units", [3, 16, 65, 300])
def test_norm_of_equal_values_and_of_rows_far_from_zero(dtype, units):
    """A constant row has no deviations: zeros, so y = beta, whatever the constant.  A row far from zero keeps its deviations."""
    D = width(units, dtype)
    consts = torch.tensor([0.0, 1.0, -3.0, 1000.5, 61000.0, 1 / 3])
    x = consts[:, None].repeat(1, D).to(dtype).to(DEV)
    gamma, beta = torch.randn(D, generator=generator(1)).to(DEV), torch.randn(D, generator=generator(2)).to(DEV)
    y = torch.empty_like(x)
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y)
    want = host(beta)[None].repeat(len(consts), 0)
    # the corrected mean is off by its last rounding alone, 2^-24 of the constant's own rounding error: far below beta's
    # half step for deviations times 1 / sqrt(eps) = 316; allowed: 316 times 2^-40 of the constant
    inside(y, want, half_step(dtype, want) + 320 * 2.0 ** -40 * np.abs(host(x)) * np.abs(host(gamma)) + 2 * seq.U32 * np.abs(want))


def test_norm_keeps_bad_rows_to_themselves():
    D = 72
    x, dy, gamma, beta = norm_inputs(50, D, torch.bfloat16, 9)
    y0, y1 = torch.empty_like(x), torch.empty_like(x)
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y0)
    x[7, 3], x[20, 71], x[33, 0] = float("nan"), float("inf"), float("-inf")
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y1)
    bad = torch.zeros(50, dtype=torch.bool, device=DEV)
    bad[[7, 20, 33]] = True
    assert same_bits(y0[~bad], y1[~bad]) and y1[bad].isnan().all()


def test_norm_in_place_and_its_neighbours():
    """y may be x and dx may be dy; what lies before and behind the rows stays as it was."""
    D, n = 104, 77
    x, dy, gamma, beta = norm_inputs(n, D, torch.float16, 10)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    dx, dg, db = torch.empty_like(x), torch.empty(D, device=DEV), torch.empty(D, device=DEV)
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y, mean, rstd)
    fs.fs_seq_norm_bwd(dy, x, mean, rstd, gamma, dx, dg, db)
    big = torch.full((n + 2, D), 5.0, dtype=torch.float16, device=DEV)
    big[1:-1] = dy
    dg2, db2 = torch.empty_like(dg), torch.empty_like(db)
    fs.fs_seq_norm_bwd(big[1:-1], x, mean, rstd, gamma, big[1:-1], dg2, db2)
    assert same_bits(big[1:-1], dx) and same_bits(dg, dg2) and same_bits(db, db2) and (big[0] == 5).all() and (big[-1] == 5).all()
    big[1:-1] = x
    fs.fs_seq_norm_fwd(big[1:-1], gamma, beta, EPS, big[1:-1])
    assert same_bits(big[1:-1], y) and (big[0] == 5).all() and (big[-1] == 5).all()


# ---- recurrence ------------------------------------------------------------------------------------------------

def offsets_of(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


def scan_inputs(lengths, D, dtype, seed, bias=1.5):
    off = offsets_of(lengths)
    n, S = int(off[-1]), len(lengths)
    gen = generator(seed)
    x, dh, h = (rows(gen, n, D, dtype) for _ in range(3))
    gate = rows(gen, n, D, dtype, 2.0, bias)
    h0, dl = (torch.randn(S, D, generator=gen).to(DEV) for _ in range(2))
    return off, x, gate, h, dh, h0, dl


def pack(x):
    n, D = x.shape
    codes, exps = torch.empty(n, D, dtype=torch.int8, device=DEV), torch.empty(n, -(-D // 32), dtype=torch.uint8, device=DEV)
    fs.fs_seq_pack8(x, codes, exps)
    return codes, exps


def check_scan(lengths, D, dtype, seed, carried=True, bias=1.5, packed=(False, True)):
    off, x, gate, h_in, dh, h0, dl = scan_inputs(lengths, D, dtype, seed, bias)
    S, n = len(lengths), x.shape[0]
    if not carried:
        h0 = dl = None
    off_d = torch.from_numpy(off).to(DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    h = torch.full_like(x, 9.0)
    last = torch.full((S, D), 9.0, device=DEV)
    fs.fs_seq_scan_fwd(x, gate, off_d, 1, S, h0, h, last, st)
    hh = None if h0 is None else host(h0)
    wh, wl, bh, bl = seq.scan_fwd(host(x), host(gate), off, hh)
    inside(h, wh, half_step(dtype, wh) + bh)
    inside(last, wl, bl + seq.U32 * np.abs(wl))
    again = torch.empty_like(h)
    fs.fs_seq_scan_fwd(x, gate, off_d, 1, S, h0, again)
    assert same_bits(again, h)
    for p in packed:
        dx, dg, d0 = torch.full_like(x, 9.0), torch.full_like(x, 9.0), torch.full((S, D), 9.0, device=DEV)
        if p:
            parts = [pack(t) for t in (x, gate, h_in)]
            fs.fs_seq_scan_bwd_packed(dh, dl, *parts[0], *parts[1], *parts[2], off_d, 1, S, h0, dx, dg, d0, st)
            vx, vg, vh = (seq.unpack8(c.cpu().numpy(), e.cpu().numpy()) for c, e in parts)
        else:
            fs.fs_seq_scan_bwd(dh, dl, x, gate, h_in, off_d, 1, S, h0, dx, dg, d0, st)
            vx, vg, vh = host(x), host(gate), host(h_in)
        wx, wg, w0, bx, bg, b0 = seq.scan_bwd(host(dh), None if dl is None else host(dl), vx, vg, vh, off, hh)
        inside(dx, wx, half_step(dtype, wx) + bx)
        inside(dg, wg, half_step(dtype, wg) + bg)
        inside(d0, w0, b0 + seq.U32 * np.abs(w0))
    assert int(st.item()) == 0


RAGGED = [3, 0, 1, 17, 0, 0, 64, 5, 130, 2, 1, 1, 0, 255, 31, 33]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("units", [1, 2, 3, 9, 16, 17, 33, 64, 70])
def test_scan_widths(dtype, units):
    check_scan(RAGGED, width(units, dtype), dtype, units)


@pytest.mark.parametrize("carried", [False, True])
@pytest.mark.parametrize("lengths", [[1], [0], [0, 0, 0], [0, 1, 0], [2], [1] * 70, [1, 0] * 40, [127], [128], [129], [255, 1], [256], [257],
                                     [512, 512], [511, 513], [1, 1023], [1025], [0] * 300 + [5] + [0] * 300],
                         ids=lambda v: f"{len(v)}x{max(v)}")
def test_scan_lengths(lengths, carried):
    check_scan(lengths, 32, torch.float32, sum(lengths) + len(lengths), carried)
    check_scan(lengths, 72, torch.bfloat16, sum(lengths) + len(lengths), carried)


@pytest.mark.parametrize("dtype, D", [(torch.float32, 4), (torch.float16, 64), (torch.bfloat16, 256)])
def test_scan_one_long_sequence(dtype, D):
    check_scan([3, 9000, 0, 700], D, dtype, 3, bias=5.0)      # gates near one: what was long ago still counts


def test_scan_many_short_sequences():
    rng = np.random.default_rng(8)
    check_scan(rng.integers(0, 4, 4000).tolist(), 16, torch.float16, 8)


def test_scan_gates_at_the_ends():
    """A gate of -infinity forgets, one of +infinity keeps; the largest finite ones do the same up to what 32 bits hold."""
    off, x, gate, h_in, dh, h0, dl = scan_inputs([40, 3, 200], 64, torch.float32, 12)
    gate[5], gate[6], gate[60], gate[61] = float("-inf"), float("inf"), 3e38, -3e38
    gate[100:140] = float("inf")
    gate[150:153] = float("-inf")
    off_d = torch.from_numpy(off).to(DEV)
    h, last = torch.empty_like(x), torch.empty(3, 64, device=DEV)
    fs.fs_seq_scan_fwd(x, gate, off_d, 1, 3, h0, h, last)
    assert torch.equal(h[5], x[5]) and torch.equal(h[6], h[5]) and torch.equal(h[61], x[61])
    assert torch.equal(h[152], x[152])
    # rows 100 .. 139 keep row 99's state; bit for bit only where it reaches them row by row: a stretch of rows folded to v -> A v + B
    # first hands on another rounding of the same number.  Both lie within the recurrence's bound of the exact state (1 + 1 of them apart).
    wh, wl, bh, bl = seq.scan_fwd(host(x), np.clip(host(gate), -1000, 1000), off, host(h0))
    assert np.all(np.abs(host(h[139]) - host(h[99])) <= bh[139] + bh[99] + 2 * half_step(torch.float32, wh[99]))
    inside(h, wh, half_step(torch.float32, wh) + bh)
    dx, dg, d0 = torch.empty_like(x), torch.empty_like(x), torch.empty(3, 64, device=DEV)
    fs.fs_seq_scan_bwd(dh, dl, x, gate, h_in, off_d, 1, 3, h0, dx, dg, d0)
    wx, wg, w0, bx, bg, b0 = seq.scan_bwd(host(dh), host(dl), host(x), np.clip(host(gate), -1000, 1000), host(h_in), off, host(h0))
    inside(dx, wx, half_step(torch.float32, wx) + bx)
    inside(dg, wg, half_step(torch.float32, wg) + bg)
    inside(d0, w0, b0 + seq.U32 * np.abs(w0))
    assert not dx[6].any() and not dg[5].any()


@pytest.mark.parametrize("what", ["nan", "inf"])
def test_scan_keeps_bad_values_in_their_sequence(what):
    lengths = [10, 300, 7, 0, 90, 260]
    off, x, gate, h_in, dh, h0, dl = scan_inputs(lengths, 64, torch.bfloat16, 13)
    S = len(lengths)
    off_d = torch.from_numpy(off).to(DEV)

    def both():
        h, last = torch.empty_like(x), torch.empty(S, 64, device=DEV)
        dx, dg, d0 = torch.empty_like(x), torch.empty_like(x), torch.empty(S, 64, device=DEV)
        fs.fs_seq_scan_fwd(x, gate, off_d, 1, S, h0, h, last)
        fs.fs_seq_scan_bwd(dh, dl, x, gate, h_in, off_d, 1, S, h0, dx, dg, d0)
        return h, dx, dg, last, d0

    clean = both()
    v = float(what)
    x[off[1] + 3], dh[off[1] + 250], h0[2], dl[4], gate[off[5] + 5, 3] = v, v, v, v, float("nan")
    dirty = both()
    touched = torch.zeros(x.shape[0], dtype=torch.bool, device=DEV)
    for s in (1, 2, 4, 5):
        touched[off[s]:off[s + 1]] = True
    for a, b in zip(clean[:3], dirty[:3]):
        assert same_bits(a[~touched], b[~touched])
    for a, b in zip(clean[3:], dirty[3:]):
        assert same_bits(a[[0, 3]], b[[0, 3]])
    assert not dirty[0][off[1] + 10:off[2]].isfinite().any() and not dirty[3][1].isfinite().any()
    assert dirty[0][off[5] + 9, 3].isnan() and dirty[0][off[5] + 9, [0, 1, 2, 4]].isfinite().all()


def test_scan_bad_offsets_are_reported_and_stay_in_bounds():
    D, n = 64, 600
    x = torch.randn(n + 2, D, device=DEV)
    gate = torch.randn(n + 2, D, device=DEV)
    for bad in ([5, 100, 600], [0, 400, 300, 600], [0, 100, 599], [0, 700, 600], [-5, 100, 600], [0, 1 << 40, 600], [0, 100, -1],
                [0, 600, 0, 600], [0, 100, 700]):
        S = len(bad) - 1
        off = torch.tensor(bad, device=DEV)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        h = torch.full((n + 2, D), 3.0, device=DEV)
        last, d0 = torch.full((S + 2, D), 3.0, device=DEV), torch.full((S + 2, D), 3.0, device=DEV)
        dx, dg = torch.full_like(h, 3.0), torch.full_like(h, 3.0)
        fs.fs_seq_scan_fwd(x[1:-1], gate[1:-1], off, 1, S, None, h[1:-1], last[1:-1], st)
        assert int(st.item()) == fs.FS_DEV_BAD_OFFSETS, bad
        st.zero_()
        fs.fs_seq_scan_bwd(x[1:-1], None, x[1:-1], gate[1:-1], x[1:-1], off, 1, S, None, dx[1:-1], dg[1:-1], d0[1:-1], st)
        assert int(st.item()) == fs.FS_DEV_BAD_OFFSETS, bad
        for t in (h, dx, dg, last, d0):
            assert (t[0] == 3).all() and (t[-1] == 3).all(), bad


def test_scan_in_place_and_its_neighbours():
    lengths = [50, 0, 333, 1, 90]
    off, x, gate, h_in, dh, h0, dl = scan_inputs(lengths, 104, torch.float16, 14)
    S, n = len(lengths), x.shape[0]
    off_d = torch.from_numpy(off).to(DEV)
    h = torch.empty_like(x)
    fs.fs_seq_scan_fwd(x, gate, off_d, 1, S, h0, h)
    dx, dg = torch.empty_like(x), torch.empty_like(x)
    fs.fs_seq_scan_bwd(dh, dl, x, gate, h_in, off_d, 1, S, h0, dx, dg)
    big = torch.full((n + 2, 104), 5.0, dtype=torch.float16, device=DEV)
    mid = big[1:-1]
    mid.copy_(x)
    fs.fs_seq_scan_fwd(mid, gate, off_d, 1, S, h0, mid)
    assert same_bits(mid, h) and (big[0] == 5).all() and (big[-1] == 5).all()
    mid.copy_(dh)
    other = torch.empty_like(dg)
    fs.fs_seq_scan_bwd(mid, dl, x, gate, h_in, off_d, 1, S, h0, mid, other)
    assert same_bits(mid, dx) and same_bits(other, dg) and (big[0] == 5).all() and (big[-1] == 5).all()
    mid.copy_(dh)
    fs.fs_seq_scan_bwd(mid, dl, x, gate, h_in, off_d, 1, S, h0, other, mid)
    assert same_bits(mid, dg) and same_bits(other, dx) and (big[0] == 5).all() and (big[-1] == 5).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m, units", [(1, 1), (1, 16), (3, 17), (256, 16), (1000, 9)])
def test_step_is_one_row_of_the_scan(dtype, m, units):
    D = width(units, dtype)
    gen = generator(m + units)
    x, gate = rows(gen, m, D, dtype), rows(gen, m, D, dtype, 2.0, 1.5)
    state = torch.randn(m, D, generator=gen).to(DEV)
    out, h = torch.empty_like(state), torch.empty_like(x)
    fs.fs_seq_scan_step(x, gate, state, out, h)
    off = np.arange(m + 1)
    wh, wl, bh, bl = seq.scan_fwd(host(x), host(gate), off, host(state))
    inside(h, wh, half_step(dtype, wh) + bh)
    inside(out, wl, bl + seq.U32 * np.abs(wl))
    hs, last = torch.empty_like(x), torch.empty_like(state)
    fs.fs_seq_scan_fwd(x, gate, torch.from_numpy(off).to(DEV), 1, m, state, hs, last)
    assert same_bits(hs, h) and same_bits(last, out)
    fs.fs_seq_scan_step(x, gate, state, state, h)             # in place
    assert same_bits(state, out)


def test_prefill_then_steps_is_the_whole_scan():
    """A sequence taken whole, or its beginning and then token by token with the state carried: the same to the recurrence's bound."""
    D, L, cut = 64, 40, 33
    off, x, gate, _, _, h0, _ = scan_inputs([L], D, torch.bfloat16, 21)
    whole, last = torch.empty_like(x), torch.empty(1, D, device=DEV)
    fs.fs_seq_scan_fwd(x, gate, torch.tensor([0, L], device=DEV), 1, 1, h0, whole, last)
    state, part = torch.empty(1, D, device=DEV), torch.empty_like(x)
    fs.fs_seq_scan_fwd(x[:cut], gate[:cut], torch.tensor([0, cut], device=DEV), 1, 1, h0, part[:cut], state)
    for t in range(cut, L):
        fs.fs_seq_scan_step(x[t:t + 1], gate[t:t + 1], state, state, part[t:t + 1])
    wh, wl, bh, bl = seq.scan_fwd(host(x), host(gate), off, host(h0))
    inside(part, wh, half_step(torch.bfloat16, wh) + bh)
    inside(state, wl, bl)
    inside(last, wl, bl)
