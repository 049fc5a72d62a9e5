"""The native look at the tensors of a sequence operator and the one in Python refuse the same sizes."""
import pytest
import torch

import paper_2301_02959_amd as fs

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("D", [1 << 31, (1 << 32) + 8])
def test_more_columns_than_an_int32_counts(D):
    """No rows: nothing is allocated."""
    x = torch.empty(0, D, dtype=torch.float16, device=DEV)
    codes, exps = torch.empty(0, D, dtype=torch.int8, device=DEV), torch.empty(0, -(-D // 32), dtype=torch.uint8, device=DEV)
    assert fs._fit is not None and fs._fit("pe", 0, 0, x, codes, exps) is None
    for call in (lambda: fs.fs_seq_pack8(x, codes, exps), lambda: fs.fs_seq_unpack8(codes, exps, x), lambda: fs.fs_seq_norm_fwd(x, None, None, 1e-5, x)):
        with pytest.raises(fs.FlexShardError) as e:
            call()
        assert e.value.code == 2
    narrow = torch.empty(0, (1 << 31) - 8, dtype=torch.float16, device=DEV)
    assert fs._fit("", 0, 0, narrow)[:3] == (0, (1 << 31) - 8, fs.FS_F16)
