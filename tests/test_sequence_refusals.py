"""What the sequence operators refuse, on the host: wrong sizes, types, alignments and workspaces return their status before
anything is launched, and the binding raises for tensors that do not go together.  No GPU: the addresses are never read."""
import ctypes
import os

import pytest
import torch

import paper_2301_02959_amd as fs

pytestmark = pytest.mark.skipif(not os.path.exists(fs.LIB_PATH), reason="library not built (run __graft_entry__.build())")

NULL, SIZE, DTYPE, ALIGN, WORKSPACE, CONFIG = 1, 2, 3, 4, 5, 6
A = 1 << 20                     # an aligned address that nothing reads


def call(name, *args):
    return getattr(fs._typed(), name)(*args)


def size(v=1 << 40):
    return ctypes.byref(ctypes.c_size_t(v))


BASE = {
    "fs_seq_pack8": dict(x=A, n=5, D=64, dtype=0, codes=A, exps=A, stream=None),
    "fs_seq_unpack8": dict(codes=A, exps=A, n=5, D=64, dtype=0, x=A, stream=None),
    "fs_seq_norm_fwd": dict(x=A, n=5, D=64, dtype=0, gamma=A, beta=A, eps=1e-5, y=A, mean=A, rstd=A, codes=A, exps=A, stream=None),
    "fs_seq_norm_bwd": dict(dy=A, x=A, mean=A, rstd=A, n=5, D=64, dtype=0, gamma=A, dx=A, dgamma=A, dbeta=A, ws=A, size=1 << 40, stream=None),
    "fs_seq_norm_bwd_packed": dict(dy=A, codes=A, exps=A, mean=A, rstd=A, n=5, D=64, dtype=0, gamma=A, dx=A, dgamma=A, dbeta=A,
                                   ws=A, size=1 << 40, stream=None),
    "fs_seq_scan_fwd": dict(x=A, gate=A, n=5, D=64, dtype=0, offsets=A, T=2, B=3, h0=A, h=A, h_last=A, ws=A, size=1 << 40, stream=None,
                            status=None),
    "fs_seq_scan_bwd": dict(dh=A, dh_last=A, x=A, gate=A, h=A, n=5, D=64, dtype=0, offsets=A, T=2, B=3, h0=A, dx=A, dgate=A, dh0=A,
                            ws=A, size=1 << 40, stream=None, status=None),
    "fs_seq_scan_bwd_packed": dict(dh=A, dh_last=A, xc=A, xe=A, gc=A, ge=A, hc=A, he=A, n=5, D=64, dtype=0, offsets=A, T=2, B=3, h0=A,
                                   dx=A, dgate=A, dh0=A, ws=A, size=1 << 40, stream=None, status=None),
    "fs_seq_scan_step": dict(x=A, gate=A, n=5, D=64, dtype=0, state=A, state_out=A, h=A, stream=None),
}
OPTIONAL = {"mean", "rstd", "codes", "exps", "h0", "h_last", "dh_last", "dh0", "stream", "status", "ws", "size"}


def run(name, **change):
    args = dict(BASE[name], **change)
    assert set(args) == set(BASE[name])
    if "size" in args:
        args["size"] = size(args["size"]) if args["size"] is not None else None
    return call(name, *args.values())


@pytest.mark.parametrize("name", sorted(BASE))
def test_sizes_types_and_alignment(name):
    assert run(name, dtype=3) == DTYPE and run(name, dtype=-1) == DTYPE
    assert run(name, n=-1) == SIZE and run(name, n=1 << 31) == SIZE and run(name, D=0) == SIZE and run(name, D=-4) == SIZE
    assert run(name, D=66) == ALIGN and run(name, dtype=1, D=68) == ALIGN and run(name, dtype=2, D=4) == ALIGN
    for key in BASE[name]:
        if key in ("x", "y", "dy", "dx", "h", "dh", "dgate", "gate", "gamma", "beta", "h0", "h_last", "dh0", "dh_last", "state", "state_out"):
            assert run(name, **{key: A + 8}) == ALIGN, key
        if key in ("codes", "xc", "gc", "hc"):
            assert run(name, **{key: A + 2}) == ALIGN, key
            assert run(name, **{key: A + 4, "dtype": 1}) == ALIGN, key
        if key in ("mean", "rstd", "dgamma", "dbeta"):
            assert run(name, **{key: A + 2}) == ALIGN, key
        if key == "offsets":
            assert run(name, **{key: A + 4}) == ALIGN


@pytest.mark.parametrize("name", sorted(BASE))
def test_missing_pointers(name):
    must = [k for k, v in BASE[name].items() if v == A and (k not in OPTIONAL or (name.endswith("pack8") or "norm_bwd" in name))]
    for key in must:
        if key == "ws":
            continue
        assert run(name, **{key: None}) == NULL, key
    if "size" in BASE[name]:
        assert run(name, size=None) == NULL


def test_pairs_and_parameters():
    for one in ("mean", "rstd", "codes", "exps"):
        assert run("fs_seq_norm_fwd", **{one: None}) == NULL
    for eps in (0.0, -1.0, float("inf"), float("nan")):
        assert run("fs_seq_norm_fwd", eps=eps) == CONFIG
    for name in ("fs_seq_scan_fwd", "fs_seq_scan_bwd", "fs_seq_scan_bwd_packed"):
        assert run(name, T=0) == SIZE and run(name, B=0) == SIZE and run(name, T=1 << 16, B=1 << 15) == SIZE


@pytest.mark.parametrize("name", sorted(k for k in BASE if "size" in BASE[k]))
def test_workspaces(name):
    asked = ctypes.c_size_t(12345)
    args = dict(BASE[name], ws=None, size=ctypes.byref(asked))
    assert call(name, *args.values()) == 0
    assert run(name, ws=A + 128) == WORKSPACE
    if asked.value:
        assert run(name, size=asked.value - 1) == WORKSPACE
    # a larger batch needs no less
    more = ctypes.c_size_t(0)
    assert call(name, *dict(args, n=100_000, size=ctypes.byref(more)).values()) == 0
    assert more.value >= asked.value


def test_no_rows_need_no_pointers():
    for name in ("fs_seq_pack8", "fs_seq_unpack8", "fs_seq_scan_step"):
        assert run(name, **{k: None for k, v in BASE[name].items() if v == A}, n=0) == 0
    assert run("fs_seq_norm_fwd", **{k: None for k, v in BASE["fs_seq_norm_fwd"].items() if v == A}, n=0) == 0


def test_the_binding_compares_shapes():
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    x = z(4, 8)
    v, r = z(8), z(4)
    with pytest.raises(ValueError):
        fs.fs_seq_norm_fwd(x, v, z(4), 1e-5, z(4, 8))
    with pytest.raises(ValueError):
        fs.fs_seq_norm_fwd(x, v, v, 1e-5, z(3, 8))
    with pytest.raises(ValueError):
        fs.fs_seq_norm_fwd(x, v, v, 1e-5, z(4, 8, dtype=torch.float16))
    with pytest.raises(ValueError):
        fs.fs_seq_norm_fwd(x, v, v, 1e-5, z(4, 8), r, z(8))
    with pytest.raises(ValueError):
        fs.fs_seq_norm_fwd(z(8), v, v, 1e-5, z(8))
    with pytest.raises(TypeError):
        fs.fs_seq_norm_fwd(x.double(), v, v, 1e-5, x.double())
    with pytest.raises(ValueError):
        fs.fs_seq_pack8(x, z(4, 8, dtype=torch.int8), z(4, 2, dtype=torch.uint8))
    with pytest.raises(ValueError):
        fs.fs_seq_pack8(x, z(4, 8, dtype=torch.uint8), z(4, 1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        fs.fs_seq_norm_bwd(x, x, r, r, v, x, v, z(9))
    off = z(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        fs.fs_seq_scan_fwd(x, x, off, 1, 3, None, x)
    with pytest.raises(ValueError):
        fs.fs_seq_scan_fwd(x, x, off, 1, 2, z(3, 8), x)
    with pytest.raises(ValueError):
        fs.fs_seq_scan_step(x, x, z(4, 8, dtype=torch.float16), z(4, 8), x)
    with pytest.raises(TypeError):                       # all shapes fit, but this is host memory
        fs.fs_seq_scan_step(x, x, z(4, 8), z(4, 8), x)


@pytest.mark.parametrize("name", sorted(k for k in BASE if "size" in BASE[k]))
@pytest.mark.parametrize("n", [0, 1, 100])
def test_a_workspace_is_never_of_no_bytes(name, n):
    """A null workspace asks for the size, so a size of 0 would make a caller who allocates it ask again instead of running."""
    asked = ctypes.c_size_t(0)
    assert call(name, *dict(BASE[name], n=n, ws=None, size=ctypes.byref(asked)).values()) == 0
    assert asked.value >= 4


@pytest.mark.parametrize("name", sorted(k for k in BASE if "norm" in k or "scan_fwd" in k or "scan_bwd" in k))
def test_rows_of_four_megabytes_and_more(name):
    """Rows so long that a launch over their columns or an offset inside a tile would leave its range."""
    change = {"ws": None} if "size" in BASE[name] else {"n": 0}
    for dtype, D in ((0, 1 << 20), (1, 1 << 21), (2, 1 << 21), (0, 1 << 26), (2, (1 << 31) - 8)):
        assert run(name, dtype=dtype, D=D, **change) == SIZE
    for dtype, D in ((0, (1 << 20) - 4), (2, (1 << 21) - 8)):
        assert run(name, dtype=dtype, D=D, **change) == 0
