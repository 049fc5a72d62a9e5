"""The sequence operators as a program uses them: a training step from the lookup to the optimizer, captured and replayed, on
several streams, with workspaces of exactly the size asked for, at sizes past 32 bits; and widths and lengths around the
tiles of the recurrence."""
import numpy as np
import pytest
import torch

import oracle
import paper_2301_02959_amd as fs
from helpers import random_jagged, random_placement
from oracle import sequence as seq
from test_gpu_sequence import (DEV, EPS, TYPES, chain, check_norm, check_scan, generator, half_step, host, inside, offsets_of, pack, rows, same_bits,
                               scan_inputs, width)

pytestmark = pytest.mark.gpu


class Step:
    """Lookup -> norm (rows kept in 8 bits) -> recurrence whose gates are a second lookup's rows -> gradients -> row gradients."""

    def __init__(self, seed, T=2, B=37, E=300, D=64, dtype=torch.bfloat16, max_len=70):
        rng = np.random.default_rng(seed)
        ids, off, base, n = random_jagged(rng, T, B, E, max_len)
        d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
        gen = generator(seed)
        self.T, self.B, self.R, self.D, self.n, self.dtype = T, B, T * E, D, n, dtype
        self.ids, self.off, self.base = d(ids), d(off), d(base)
        self.pl = d(random_placement(rng, T * E, 8, 4).view(np.int32))
        self.table, self.gates = rows(gen, self.R, D, dtype), rows(gen, self.R, D, dtype, 1.0, 1.0)
        self.gamma, self.beta = torch.randn(D, generator=gen).to(DEV), torch.randn(D, generator=gen).to(DEV)
        self.dh = rows(gen, n, D, dtype)
        like = lambda: torch.empty(n, D, dtype=dtype, device=DEV)  # noqa: E731
        codes = lambda: (torch.empty(n, D, dtype=torch.int8, device=DEV), torch.empty(n, -(-D // 32), dtype=torch.uint8, device=DEV))  # noqa: E731
        self.o = dict(bo=torch.zeros(9, dtype=torch.int64, device=DEV), rows=torch.zeros(n, dtype=torch.int64, device=DEV),
                      pos=torch.zeros(n, dtype=torch.int32, device=DEV), st=torch.zeros(1, dtype=torch.int32, device=DEV), x=like(), g=like(), y=like(),
                      h=like(), dy=like(), dg=like(), dx=like(), mean=torch.empty(n, device=DEV), rstd=torch.empty(n, device=DEV),
                      last=torch.empty(T * B, D, device=DEV), dgamma=torch.empty(D, device=DEV), dbeta=torch.empty(D, device=DEV),
                      uniq=torch.zeros(n, dtype=torch.int64, device=DEV), rg=torch.zeros(n, D, device=DEV), nu=torch.zeros(1, dtype=torch.int64, device=DEV),
                      x8=codes(), y8=codes(), g8=codes(), h8=codes())
        kind = {torch.float32: fs.FS_F32, torch.float16: fs.FS_F16, torch.bfloat16: fs.FS_BF16}[dtype]
        self.ws = {k: torch.empty(max(v, 256), dtype=torch.uint8, device=DEV) for k, v in dict(
            route=fs.route_workspace_bytes(T, B, n, 8, 4, 0), norm=fs.seq_norm_bwd_workspace_bytes(n, D, kind),
            fwd=fs.seq_scan_fwd_workspace_bytes(n, D, kind, T, B), bwd=fs.seq_scan_bwd_workspace_bytes(n, D, kind, T, B)).items()}
        # the sort's workspace has no size function of its own: more than it asks for at any size of these tests
        self.ws["grad"] = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)

    def run(self, o=None):
        o, ws, n = o or self.o, self.ws, self.n
        fs.fs_route_bucketize(self.ids, self.off, self.T, self.B, self.base, self.pl, n, 8, 4, 0, o["bo"], o["rows"], o["pos"], None, o["st"], workspace=ws["route"])
        fs.fs_seq_gather_fwd(self.table, o["rows"], o["pos"], 0, n, o["x"], o["st"])
        fs.fs_seq_gather_fwd(self.gates, o["rows"], o["pos"], 0, n, o["g"], o["st"])
        fs.fs_seq_norm_fwd(o["x"], self.gamma, self.beta, EPS, o["y"], o["mean"], o["rstd"], *o["x8"])
        fs.fs_seq_scan_fwd(o["y"], o["g"], self.off, self.T, self.B, None, o["h"], o["last"], o["st"], workspace=ws["fwd"])
        for k in "ygh":
            fs.fs_seq_pack8(o[k], *o[k + "8"])
        fs.fs_seq_scan_bwd_packed(self.dh, None, *o["y8"], *o["g8"], *o["h8"], self.off, self.T, self.B, None, o["dy"], o["dg"], None, o["st"], workspace=ws["bwd"])
        fs.fs_seq_norm_bwd_packed(o["dy"], *o["x8"], o["mean"], o["rstd"], self.gamma, o["dx"], o["dgamma"], o["dbeta"], workspace=ws["norm"])
        fs.fs_seq_grad_bwd(o["dx"], o["rows"], o["pos"], 0, n, self.R, 0, o["uniq"], o["rg"], n, o["nu"], o["st"], workspace=ws["grad"])
        return o

    def result(self, o):
        k = int(o["nu"].item())
        return [o[x].clone() for x in ("y", "h", "last", "dy", "dg", "dx", "dgamma", "dbeta", "mean", "rstd")] + [o["rg"][:k].clone(), o["uniq"][:k].clone()]


def equal(a, b):
    return len(a) == len(b) and all(same_bits(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_training_step_stage_by_stage(dtype):
    """Every stage against its definition in 64 bits on what the stage before it left."""
    s = Step(5, dtype=dtype)
    o = s.run()
    torch.cuda.synchronize()
    assert int(o["st"].item()) == 0
    off, G, Bt, D = s.off.cpu().numpy(), host(s.gamma), host(s.beta), s.D
    X = host(o["x"])
    wy, wm, wr = seq.norm_fwd(X, G, Bt, EPS)
    c = chain(D, dtype) * seq.U32
    size = np.abs(X - wm[:, None]) * wr[:, None] * np.abs(G)
    inside(o["y"], wy, half_step(dtype, wy) + (2 * c + 8 * seq.U32) * (np.abs(wy) + np.abs(Bt) + size + (np.abs(X - wm[:, None]).mean(1) * wr)[:, None] * np.abs(G)))
    wh, wl, bh, bl = seq.scan_fwd(host(o["y"]), host(o["g"]), off)
    inside(o["h"], wh, half_step(dtype, wh) + bh)
    inside(o["last"], wl, bl + seq.U32 * np.abs(wl))
    kept = {k: seq.unpack8(*(t.cpu().numpy() for t in o[k + "8"])) for k in "xygh"}
    for k in "xygh":
        assert np.array_equal(kept[k], seq.unpack8(*seq.pack8(host(o[k]))))
    wx, wg, _, bx, bg, _ = seq.scan_bwd(host(s.dh), None, kept["y"], kept["g"], kept["h"], off)
    inside(o["dy"], wx, half_step(dtype, wx) + bx)
    inside(o["dg"], wg, half_step(dtype, wg) + bg)
    M, R, DY = host(o["mean"]), host(o["rstd"]), host(o["dy"])
    wx, wga, wb = seq.norm_bwd(DY, kept["x"], M, R, G)
    g, u = np.abs(DY * G), np.abs((kept["x"] - M[:, None]) * R[:, None])
    inside(o["dx"], wx, half_step(dtype, wx) + (c + 8 * seq.U32) * R[:, None] * (g + g.mean(1, keepdims=True) + u * (g * u).mean(1, keepdims=True)))
    inside(o["dgamma"], wga, (165 + s.n / 4096) * seq.U32 * (np.abs(DY) * u).sum(0))
    inside(o["dbeta"], wb, (165 + s.n / 4096) * seq.U32 * np.abs(DY).sum(0))
    # the rows' gradients: the library's own summation order, bit for bit
    grad = o["dx"].float().cpu().numpy()
    rc, st, ou, og, _, onu = oracle.seq_grad_bwd(grad, o["rows"].cpu().numpy(), o["pos"].cpu().numpy(), 0, s.n, s.R)
    k = int(o["nu"].item())
    assert rc == 0 and st == 0 and k == onu and np.array_equal(o["uniq"][:k].cpu().numpy(), ou)
    assert np.array_equal(o["rg"][:k].cpu().numpy().view(np.uint32), og.view(np.uint32))


def test_captured_and_replayed():
    """One graph of the whole step; replays with the inputs changed in place, eager work and synchronisations between them."""
    s = Step(7, max_len=300)
    eager = s.result(s.run())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    first = s.table.clone()
    for i in range(4):
        for k, t in s.o.items():
            if isinstance(t, torch.Tensor) and t.is_floating_point():
                t.fill_(float("nan"))
        s.table.copy_(first if i % 2 == 0 else first.flip(0))
        graph.replay()
        got = s.result(s.o)
        torch.cuda.synchronize()
        want = s.result(s.run())
        assert equal(got, want), i
        if i % 2 == 0:
            assert equal(got, eager)
    assert int(s.o["st"].item()) == 0


def test_two_graphs_share_workspaces():
    """Two captured batches of different sizes that bring the same workspaces, replayed in turn."""
    a, b = Step(11, max_len=400), Step(12, T=3, B=11, D=136, max_len=90)
    for k in a.ws:
        a.ws[k] = b.ws[k] = a.ws[k] if a.ws[k].numel() >= b.ws[k].numel() else b.ws[k]
    want = [s.result(s.run()) for s in (a, b)]
    graphs = []
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            s.run()
        graphs.append(g)
    for _ in range(3):
        for s, g, w in zip((a, b), graphs, want):
            for k in ("y", "h", "dx", "rg"):
                s.o[k].fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert equal(s.result(s.o), w)


def test_side_by_side_on_two_streams():
    steps = [Step(21 + i, T=4, B=300, max_len=200) for i in range(2)]
    want = [s.result(s.run()) for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(3):
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                s.run()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert equal(s.result(s.o), w)


def test_another_device_is_refused(monkeypatch):
    x = torch.zeros(4, 8, device=DEV)
    v = torch.zeros(8, device=DEV)
    monkeypatch.setattr(fs, "_raw_device", lambda: 1)
    with pytest.raises(ValueError):
        fs.fs_seq_norm_fwd(x, v, v, EPS, x)
    with pytest.raises(ValueError):
        fs.fs_seq_scan_step(x, x, x, x, x)


def test_workspaces_of_the_size_asked_for():
    """Nothing is written past a workspace of exactly the size asked for; a byte less is refused."""
    lengths = [400, 0, 1, 777, 30]
    off, x, gate, h_in, dh, h0, dl = scan_inputs(lengths, 72, torch.float16, 31)
    off_d, S, n, D = torch.from_numpy(off).to(DEV), len(lengths), x.shape[0], 72
    mean, rstd = torch.zeros(n, device=DEV), torch.ones(n, device=DEV)
    v = [torch.empty(D, device=DEV) for _ in range(3)]
    h, dx, dg = (torch.empty_like(x) for _ in range(3))
    calls = [(fs.seq_scan_fwd_workspace_bytes(n, D, fs.FS_F16, 1, S), lambda w, **k: fs.fs_seq_scan_fwd(x, gate, off_d, 1, S, h0, h, workspace=w, **k)),
             (fs.seq_scan_bwd_workspace_bytes(n, D, fs.FS_F16, 1, S),
              lambda w, **k: fs.fs_seq_scan_bwd(dh, dl, x, gate, h_in, off_d, 1, S, h0, dx, dg, workspace=w, **k)),
             (fs.seq_norm_bwd_workspace_bytes(n, D, fs.FS_F16), lambda w, **k: fs.fs_seq_norm_bwd(dh, x, mean, rstd, v[0], dx, v[1], v[2], workspace=w, **k))]
    for size, call in calls:
        assert size > 0
        buf = torch.full((size + 4096,), 77, dtype=torch.uint8, device=DEV)
        call(buf[:size])
        torch.cuda.synchronize()
        assert (buf[size:] == 77).all()
        assert call(buf[:size - 1], raise_on_error=False) == 5
        with pytest.raises(fs.FlexShardError):
            call(buf[:size - 1])


def test_states_in_place():
    """h_last may be h0 and dh0 may be dh_last: a stream of batches needs one buffer of states."""
    lengths = [300, 0, 5, 700, 1, 128, 129, 0, 40]
    off, x, gate, h_in, dh, h0, dl = scan_inputs(lengths, 64, torch.float32, 33)
    off_d, S = torch.from_numpy(off).to(DEV), len(lengths)
    h, last = torch.empty_like(x), torch.empty_like(h0)
    dx, dg, d0 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(h0)
    fs.fs_seq_scan_fwd(x, gate, off_d, 1, S, h0, h, last)
    fs.fs_seq_scan_bwd(dh, dl, x, gate, h_in, off_d, 1, S, h0, dx, dg, d0)
    state, grad, h2, dx2, dg2 = h0.clone(), dl.clone(), torch.empty_like(h), torch.empty_like(dx), torch.empty_like(dg)
    fs.fs_seq_scan_fwd(x, gate, off_d, 1, S, state, h2, state)
    fs.fs_seq_scan_bwd(dh, grad, x, gate, h_in, off_d, 1, S, h0, dx2, dg2, grad)
    for a, b in ((state, last), (grad, d0), (h2, h), (dx2, dx), (dg2, dg)):
        assert same_bits(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("units", [4, 6, 7, 8, 12, 15, 24, 31, 32, 40, 48, 65])
def test_scan_more_widths(dtype, units):
    check_scan([200, 0, 1, 57, 300], width(units, dtype), dtype, units, packed=(units % 2 == 0,))


def test_scan_sequences_that_meet_the_tiles():
    """Tiles hold 128 rows of 256 bytes forward and 64 backward: sequences that begin and end with them, next to them, or span many."""
    for lengths in ([128] * 5, [64] * 9, [127, 1, 128, 129, 127], [63, 65, 64, 1, 63], [1] * 64 + [64], [640], [1, 640, 1], [127, 0, 0, 1, 0, 128]):
        check_scan(lengths, 128, torch.bfloat16, len(lengths), packed=(False,))


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_rows_past_a_waves_and_a_workgroups_registers(dtype):
    for units in (512, 513, 1024, 1025, 1400):
        check_norm(19, width(units, dtype), dtype, units)


@pytest.mark.parametrize("n", [255, 256, 257, 511, 512, 513])
def test_norm_around_one_launch(n):
    """Few rows go in one launch: 8 rounds of a workgroup."""
    check_norm(n, 128, torch.bfloat16, n)
    check_norm(n // 4, 600, torch.float32, n)


def test_scan_past_32_bits():
    """9 GB a tensor: offsets in bytes and in elements pass 2^32; the last sequences against 64 bits."""
    D, L = 256, 1000
    S = 9000
    n = S * L
    x = torch.empty(n, D, device=DEV)
    gate = torch.empty(n, D, device=DEV)
    for lo in range(0, n, 1 << 20):
        x[lo:lo + (1 << 20)].normal_()
        gate[lo:lo + (1 << 20)].normal_(1.0, 1.0)
    off = torch.arange(S + 1, device=DEV) * L
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    h, last = torch.empty_like(x), torch.empty(S, D, device=DEV)
    fs.fs_seq_scan_fwd(x, gate, off, S // 9, 9, None, h, last, st)
    dx, dg, d0 = torch.empty_like(x), torch.empty_like(x), torch.empty(S, D, device=DEV)
    fs.fs_seq_scan_bwd(x, None, x, gate, h, off, S // 9, 9, None, dx, dg, d0, st)
    assert int(st.item()) == 0
    for s in (0, S // 2, S - 2, S - 1):
        a, b = s * L, (s + 1) * L
        X, Gt, H = host(x[a:b]), host(gate[a:b]), host(h[a:b])
        wh, wl, bh, bl = seq.scan_fwd(X, Gt, [0, L])
        inside(h[a:b], wh, half_step(torch.float32, wh) + bh)
        inside(last[s:s + 1], wl, bl + seq.U32 * np.abs(wl))
        wx, wg, w0, bx, bg, b0 = seq.scan_bwd(X, None, X, Gt, H, [0, L])
        inside(dx[a:b], wx, half_step(torch.float32, wx) + bx)
        inside(dg[a:b], wg, half_step(torch.float32, wg) + bg)
        inside(d0[s:s + 1], w0, b0 + seq.U32 * np.abs(w0))
    del x, gate, h, dx, dg
    torch.cuda.empty_cache()


def test_the_most_rows_a_call_admits():
    """2^31 - 1 rows of one piece: norm, checkpoint and a single sequence; the last rows against 64 bits."""
    n, D, tail = (1 << 31) - 1, 8, 600
    x = torch.empty(n, D, dtype=torch.float16, device=DEV)
    for lo in range(0, n, 1 << 28):
        x[lo:lo + (1 << 28)].normal_()
    gamma, beta = torch.ones(D, device=DEV), torch.zeros(D, device=DEV)
    y = torch.empty_like(x)
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y)
    for at in (slice(0, 64), slice(n - 64, n)):
        part = torch.empty_like(y[at])
        fs.fs_seq_norm_fwd(x[at].clone(), gamma, beta, EPS, part)
        assert same_bits(y[at], part)
    # gates near 1/2: what is 200 rows back is gone from 32 bits
    off = torch.tensor([0, n], device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    fs.fs_seq_scan_fwd(x, x, off, 1, 1, None, y, None, st)
    X = host(x[n - tail:])
    wh, _, bh, _ = seq.scan_fwd(X, X, [0, tail])
    inside(y[n - tail + 400:], wh[400:], half_step(torch.float16, wh[400:]) + bh[400:] + 2.0 ** -60)
    assert int(st.item()) == 0
    codes = torch.empty(n, D, dtype=torch.int8, device=DEV)
    exps = torch.empty(n, 1, dtype=torch.uint8, device=DEV)
    fs.fs_seq_pack8(x, codes, exps)
    fs.fs_seq_unpack8(codes, exps, y)
    wc, we = seq.pack8(X)
    assert np.array_equal(codes[n - tail:].cpu().numpy(), wc) and np.array_equal(exps[n - tail:].cpu().numpy(), we)
    assert np.array_equal(host(y[n - tail:]), seq.unpack8(wc, we).astype(np.float16).astype(np.float64))
    del x, y, codes, exps
    torch.cuda.empty_cache()


@pytest.mark.parametrize("units", [1, 16, 65, 300, 1024, 1100])
@pytest.mark.parametrize("n", [3, 600])
def test_norm_gradients_in_place_at_every_width(units, n):
    """dx may be dy whatever kernels the width takes: the sums over dy have to be done with it first."""
    D = width(units, torch.bfloat16)
    gen = generator(units + n)
    x, dy = rows(gen, n, D, torch.bfloat16), rows(gen, n, D, torch.bfloat16)
    gamma, beta = torch.randn(D, generator=gen).to(DEV), torch.zeros(D, device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    codes, exps = torch.empty(n, D, dtype=torch.int8, device=DEV), torch.empty(n, -(-D // 32), dtype=torch.uint8, device=DEV)
    fs.fs_seq_norm_fwd(x, gamma, beta, EPS, y, mean, rstd, codes, exps)
    for packed in (False, True):
        got = []
        for in_place in (False, True):
            d = dy.clone()
            dx = d if in_place else torch.empty_like(d)
            dg, db = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
            if packed:
                fs.fs_seq_norm_bwd_packed(d, codes, exps, mean, rstd, gamma, dx, dg, db)
            else:
                fs.fs_seq_norm_bwd(d, x, mean, rstd, gamma, dx, dg, db)
            got.append((dx, dg, db))
        assert equal(*got)
    z = x.clone()
    fs.fs_seq_norm_fwd(z, gamma, beta, EPS, z)
    assert same_bits(z, y)


@pytest.mark.parametrize("dtype", TYPES)
def test_step_in_place(dtype):
    """h may be x and state_out may be state, both at once."""
    m, D = 300, width(9, dtype)
    gen = generator(3)
    x, gate, state = rows(gen, m, D, dtype), rows(gen, m, D, dtype, 2.0, 1.5), torch.randn(m, D, generator=gen).to(DEV)
    out, h = torch.empty_like(state), torch.empty_like(x)
    fs.fs_seq_scan_step(x, gate, state, out, h)
    fs.fs_seq_scan_step(x, gate, state, state, x)
    assert same_bits(x, h) and same_bits(state, out)


def test_the_binding_in_native_code_and_in_python():
    """The native look at the tensors and the one in Python give the same sizes and pointers, and refuse the same."""
    x = torch.zeros(6, 72, device=DEV, dtype=torch.bfloat16)
    good = dict(s=torch.empty_like(x), f=torch.empty(6, 72, device=DEV), c=torch.empty(72, device=DEV), r=torch.empty(6, device=DEV),
                p=torch.empty(6, 72, device=DEV, dtype=torch.int8), e=torch.empty(6, 3, device=DEV, dtype=torch.uint8),
                o=torch.zeros(4, device=DEV, dtype=torch.int64), t=torch.empty(3, 72, device=DEV))
    kinds = "".join(good)
    assert fs._fit is not None
    for tensors in (tuple(good.values()), (None,) * 8):
        assert fs._fit(kinds, 0, 3, x, *tensors) == fs._rows_checked("test", kinds, x, tensors, 3)

    class Sub(torch.Tensor):
        pass

    for k, t in good.items():
        bad = [t[1:], t.cpu(), t.to(torch.float64), t.unsqueeze(0), t.reshape(-1)[:-1], t[..., ::2]]
        if t.dim() > 1:
            bad += [t[:, 1:], t.t()]
        for b in bad:
            args = [b if k == j else None for j in good]
            assert fs._fit(kinds, 0, 3, x, *args) is None, (k, tuple(b.shape))
            with pytest.raises((ValueError, TypeError)):
                fs._rows_checked("test", kinds, x, tuple(args), 3)
    wide = torch.zeros(6, 144, device=DEV, dtype=torch.bfloat16)[:, :72]               # the right sizes, rows apart
    for args in ((x, wide), (wide, x)):
        assert fs._fit("s", 0, 0, *args) is None
        with pytest.raises(TypeError):
            fs._rows_checked("test", "s", args[0], args[1:], 0)
    assert fs._fit("s", 1, 0, x, x) is None and fs._fit("ss", 0, 0, x, x) is None and fs._fit("?", 0, 0, x, x) is None
    assert fs._fit("s", 0, 0, x, "text") is None and fs._fit("s", 0, 0, 7, x) is None and fs._fit() is None
    assert fs._fit("s", 0, 0, x.as_subclass(Sub), x) is None                            # Python's to look at
    assert fs._rows("test", "s", x.as_subclass(Sub), x) == fs._rows("test", "s", x, x)
    assert fs._rows("test", "s", torch.nn.Parameter(x), x)[3] == x.data_ptr()


@pytest.mark.parametrize("dtype", TYPES)
def test_the_longest_rows(dtype):
    """One 16-byte piece under 4 MB a row."""
    D = width((1 << 18) - 1, dtype)
    check_norm(2, D, dtype, 18)
    check_scan([1, 0, 2], D, dtype, 18)


def test_a_checkpoint_of_one_row_of_any_length():
    """A flat tensor as one row: the codes of the same values in many rows of whole blocks."""
    n, D = 1 << 12, 1 << 15
    x = torch.empty(n, D, dtype=torch.bfloat16, device=DEV).normal_()
    codes, exps = pack(x)
    flat, flat_exps = pack(x.view(1, -1))
    assert torch.equal(flat.view(n, D), codes) and torch.equal(flat_exps.view(n, -1), exps)
    back, flat_back = torch.empty_like(x), torch.empty_like(x)
    fs.fs_seq_unpack8(codes, exps, back)
    fs.fs_seq_unpack8(flat, flat_exps, flat_back.view(1, -1))
    assert same_bits(back, flat_back)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("units", [9, 13, 16, 17, 24, 25, 32, 40, 48, 49, 64, 65, 96, 97, 128, 150, 192, 193, 300, 512, 513, 768, 769])
def test_norm_either_side_of_every_layout(dtype, units):
    """Widths at which the lanes and pieces of a row change, in one launch and in two."""
    check_norm(5, width(units, dtype), dtype, units)
    check_norm(561, width(units, dtype), dtype, units)


def test_either_form_takes_the_others_workspace():
    """seq_norm_bwd_workspace_bytes holds for the packed form, whatever rows a workgroup of either takes at a time."""
    for dtype, kind in ((torch.float32, fs.FS_F32), (torch.float16, fs.FS_F16), (torch.bfloat16, fs.FS_BF16)):
        for units in (9, 24, 32, 40, 600, 1100):
            for n in (1, 100, 150, 3000):
                D = width(units, dtype)
                gen = generator(units + n)
                x, dy = rows(gen, n, D, dtype), rows(gen, n, D, dtype)
                gamma = torch.ones(D, device=DEV)
                mean, rstd = torch.zeros(n, device=DEV), torch.ones(n, device=DEV)
                codes, exps = pack(x)
                ws = torch.empty(fs.seq_norm_bwd_workspace_bytes(n, D, kind), dtype=torch.uint8, device=DEV)
                out = [torch.empty_like(x), torch.empty(D, device=DEV), torch.empty(D, device=DEV)]
                alone = [torch.empty_like(t) for t in out]
                fs.fs_seq_norm_bwd_packed(dy, codes, exps, mean, rstd, gamma, *out, workspace=ws)
                fs.fs_seq_norm_bwd_packed(dy, codes, exps, mean, rstd, gamma, *alone)
                assert all(same_bits(a, b) for a, b in zip(out, alone))
                fs.fs_seq_norm_bwd(dy, x, mean, rstd, gamma, *out, workspace=ws)
                # dbeta does not depend on x: n additions in either order
                assert torch.allclose(out[2], alone[2], rtol=0, atol=2 * n * 2.0 ** -24 * float(dy.float().abs().sum(0).max()))
