"""Sizes that do not fit the C entry points' 32-bit integers: the binding refuses them instead of handing on their low bits.  No
GPU: tensors without elements, whose pointers nothing reads."""
import ctypes
import os

import pytest
import torch

import paper_2301_02959_amd as fs

pytestmark = pytest.mark.skipif(not os.path.exists(fs.LIB_PATH), reason="library not built (run __graft_entry__.build())")

SIZE = 2
WIDE = [1 << 31, (1 << 32) + 8, (1 << 33) + 64]         # as an int32: negative, 8, 64


@pytest.fixture(autouse=True)
def host_pointers(monkeypatch):
    monkeypatch.setattr(fs, "_ptr", lambda t, dtypes=None: None if t is None else t.data_ptr())
    monkeypatch.setattr(fs, "_stream", lambda: None)
    monkeypatch.setattr(fs, "_raw_device", lambda: -1)       # what host tensors call their device


def refused(call, *args, **more):
    assert call(*args, raise_on_error=False, **more) == SIZE
    with pytest.raises(fs.FlexShardError):
        call(*args, **more)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", WIDE)
def test_rows_of_more_columns_than_an_int32_counts(D, dtype):
    """No rows, so nothing is allocated and nothing would be written; before rows are counted, D is refused."""
    x = torch.empty(0, D, dtype=dtype)
    f = torch.empty(0, D)
    codes, exps = torch.empty(0, D, dtype=torch.int8), torch.empty(0, -(-D // 32), dtype=torch.uint8)
    ws = torch.empty(256, dtype=torch.uint8)
    off, none = torch.zeros(2, dtype=torch.int64), torch.empty(0)
    refused(fs.fs_seq_pack8, x, codes, exps)
    refused(fs.fs_seq_unpack8, codes, exps, x)
    refused(fs.fs_seq_scan_step, x, x, f, f, x)
    refused(fs.fs_seq_norm_fwd, x, None, None, 1e-5, x)
    for more in ({}, {"workspace": ws}):
        refused(fs.fs_seq_norm_bwd, x, x, none, none, None, x, None, None, **more)
        refused(fs.fs_seq_norm_bwd_packed, x, codes, exps, none, none, None, x, None, None, **more)
        refused(fs.fs_seq_scan_fwd, x, x, off, 1, 1, None, x, **more)
        refused(fs.fs_seq_scan_bwd, x, None, x, x, x, off, 1, 1, None, x, x, **more)
        refused(fs.fs_seq_scan_bwd_packed, x, None, codes, exps, codes, exps, codes, exps, off, 1, 1, None, x, x, **more)


@pytest.mark.parametrize("big", WIDE + [(1 << 32) + 1])
def test_workspaces_of_sizes_past_an_int32(big):
    for size in (lambda: fs.seq_norm_bwd_workspace_bytes(5, big, 0), lambda: fs.seq_scan_fwd_workspace_bytes(5, big, 0, 1, 1),
                 lambda: fs.seq_scan_bwd_workspace_bytes(5, big, 0, 1, 1), lambda: fs.seq_scan_fwd_workspace_bytes(5, 64, 0, big, 1),
                 lambda: fs.seq_scan_fwd_workspace_bytes(5, 64, 0, 1, big), lambda: fs.seq_scan_bwd_workspace_bytes(5, 64, 0, big, 1),
                 lambda: fs.seq_scan_bwd_workspace_bytes(5, 64, 0, 1, big)):
        with pytest.raises(fs.FlexShardError) as e:
            size()
        assert e.value.code == SIZE


class Offsets(torch.Tensor):
    """Stands for the offsets of more sequences than this machine has memory for."""
    @staticmethod
    def __new__(cls, count):
        t = torch.Tensor._make_subclass(cls, torch.zeros(2, dtype=torch.int64))
        t.count = count
        return t

    shape = property(lambda self: torch.Size([self.count]))


@pytest.mark.parametrize("T, B", [((1 << 32) + 1, 1), (1, (1 << 32) + 1), (1 << 31, 1), (1 << 16, 1 << 15), ((1 << 32) + 2, 3)])
def test_more_sequences_than_an_int32_counts(T, B):
    x = torch.empty(0, 64)
    codes, exps = torch.empty(0, 64, dtype=torch.int8), torch.empty(0, 2, dtype=torch.uint8)
    off = Offsets(T * B + 1)
    ws = torch.empty(1 << 20, dtype=torch.uint8)
    for more in ({}, {"workspace": ws}):
        refused(fs.fs_seq_scan_fwd, x, x, off, T, B, None, x, **more)
        refused(fs.fs_seq_scan_bwd, x, None, x, x, x, off, T, B, None, x, x, **more)
        refused(fs.fs_seq_scan_bwd_packed, x, None, codes, exps, codes, exps, codes, exps, off, T, B, None, x, x, **more)


def test_the_c_calls_refuse_what_the_binding_hands_them():
    asked = ctypes.c_size_t(0)
    assert fs._typed().fs_seq_pack8(None, 0, 0, 0, None, None, None) == SIZE
    assert fs._typed().fs_seq_scan_fwd(None, None, 0, 64, 0, None, 0, 1, None, None, None, None, ctypes.byref(asked), None, None) == SIZE


def asked_for(name, n, D, dtype, S):
    """(status, bytes) of the recurrence's question for its workspace."""
    asked = ctypes.c_size_t(0)
    pointers = {"fs_seq_scan_fwd": ((None,) * 2, (None,) * 3), "fs_seq_scan_bwd": ((None,) * 5, (None,) * 4), "fs_seq_scan_bwd_packed": ((None,) * 8, (None,) * 4)}
    front, behind = pointers[name]
    code = getattr(fs._typed(), name)(*front, n, D, dtype, None, 1, S, *behind, None, ctypes.byref(asked), None, None)
    return code, asked.value


SCANS = ["fs_seq_scan_fwd", "fs_seq_scan_bwd", "fs_seq_scan_bwd_packed"]


@pytest.mark.parametrize("name", SCANS)
def test_wide_rows_in_many_sequences(name):
    """Few rows of many columns among more sequences than rows: the size of x decides, not the sequences times the columns."""
    for dtype, N in ((0, 4), (1, 8), (2, 8)):
        for units in ((1 << 18) - 1, (1 << 18) - 8, (1 << 17) + 8, 5000, 1):
            D = units * N
            for S in (1, 1 << 17, 1 << 18, 1 << 24, (1 << 31) - 1):
                for n in (0, 1, 5, 3000):
                    assert asked_for(name, n, D, dtype, S)[0] == 0, (n, D, dtype, S)


@pytest.mark.parametrize("name", SCANS)
def test_batches_too_large_for_one_launch(name):
    """2^24 workgroups of 256 threads are more than a launch takes.  No width reaches them below 200 GB in x."""
    for dtype, N in ((0, 4), (1, 8)):
        for units in (1, 2, 3, 9, 16, 17, 29, 31, 33, 65, 127, 1000, 4097, 99999, (1 << 18) - 1):
            n = min((1 << 31) - 1, 200 * 10 ** 9 // (16 * units))
            assert asked_for(name, n, units * N, dtype, 7)[0] == 0, (dtype, units)
        n = (1 << 31) - 1
        assert asked_for(name, n, 4096 * N, dtype, 7)[0] == SIZE and asked_for(name, n, ((1 << 18) - 1) * N, dtype, 7)[0] == SIZE


class Elsewhere(torch.Tensor):
    """A tensor of another device than the rows."""
    @staticmethod
    def __new__(cls, t):
        return torch.Tensor._make_subclass(cls, t)

    def get_device(self):
        return 1


def test_workspaces_and_status_words_of_another_device():
    """The kernels run on the current device; they would read and write the other one's memory."""
    x, off = torch.empty(0, 64), torch.zeros(2, dtype=torch.int64)
    codes, exps, none = torch.empty(0, 64, dtype=torch.int8), torch.empty(0, 2, dtype=torch.uint8), torch.empty(0)
    ws, st = torch.empty(1 << 16, dtype=torch.uint8), torch.zeros(1, dtype=torch.int32)
    scans = [lambda **more: fs.fs_seq_scan_fwd(x, x, off, 1, 1, None, x, **more),
             lambda **more: fs.fs_seq_scan_bwd(x, None, x, x, x, off, 1, 1, None, x, x, **more),
             lambda **more: fs.fs_seq_scan_bwd_packed(x, None, codes, exps, codes, exps, codes, exps, off, 1, 1, None, x, x, **more)]
    norms = [lambda **more: fs.fs_seq_norm_bwd(x, x, none, none, None, x, None, None, **more),
             lambda **more: fs.fs_seq_norm_bwd_packed(x, codes, exps, none, none, None, x, None, None, **more)]
    for call in scans + norms:
        with pytest.raises(ValueError):
            call(workspace=Elsewhere(ws))
    for call in scans:
        for more in ({}, {"workspace": ws}):
            with pytest.raises(ValueError):
                call(dev_status=Elsewhere(st), **more)


def test_a_workspace_without_bytes_is_too_small():
    """It has no address, and a call without one asks for the size instead of running."""
    x, off = torch.empty(0, 64), torch.zeros(2, dtype=torch.int64)
    codes, exps, none = torch.empty(0, 64, dtype=torch.int8), torch.empty(0, 2, dtype=torch.uint8), torch.empty(0)
    nothing = torch.empty(0, dtype=torch.uint8)
    assert nothing.data_ptr() == 0
    for call in (lambda **more: fs.fs_seq_scan_fwd(x, x, off, 1, 1, None, x, workspace=nothing, **more),
                 lambda **more: fs.fs_seq_scan_bwd(x, None, x, x, x, off, 1, 1, None, x, x, workspace=nothing, **more),
                 lambda **more: fs.fs_seq_scan_bwd_packed(x, None, codes, exps, codes, exps, codes, exps, off, 1, 1, None, x, x, workspace=nothing, **more),
                 lambda **more: fs.fs_seq_norm_bwd(x, x, none, none, None, x, None, None, workspace=nothing, **more),
                 lambda **more: fs.fs_seq_norm_bwd_packed(x, codes, exps, none, none, None, x, None, None, workspace=nothing, **more)):
        assert call(raise_on_error=False) == 5
        with pytest.raises(fs.FlexShardError):
            call()


@pytest.mark.parametrize("dtype, N, forward, backward", [(0, 4, 0.0375, 0.075), (1, 8, 0.075, 0.15), (2, 8, 0.075, 0.15)])
def test_the_recurrences_workspace_stays_under_what_the_header_says(dtype, N, forward, backward):
    """... of x, and 8 bytes a column and 1 KB: a caller may size a pool by it."""
    for units in list(range(1, 300)) + [449, 450, 1000, 1025, 4095, 4097, 65537, 99999, (1 << 18) - 1]:
        D = units * N
        for n in (0, 1, 31, 33, 65, 129, 257, 513, 1025, 4100, 100_000, 4_000_000):
            x = 16 * n * units
            if x > 200 * 10 ** 9:
                continue
            for size, share in ((fs.seq_scan_fwd_workspace_bytes, forward), (fs.seq_scan_bwd_workspace_bytes, backward)):
                for S in (1, 70_000):
                    assert size(n, D, dtype, 1, S) <= share * x + 8 * D + 1024, (n, D)
