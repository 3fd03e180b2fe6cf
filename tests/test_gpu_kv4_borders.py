"""GPU: 4-bit keys whose exact values are as near to a border between two codes, or to 2^128, as 64 bits tell apart."""

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import specmemo as sm
from tests.kv4_ref import unpack
from tests.test_gpu_kv_rows import Rows

pytestmark = pytest.mark.gpu


def appended(x):
    """(codes, scale bytes) [tokens][d or d / 32] of the keys."""
    rows, kv = x.upload(), x.pool4()
    sm.kv4_append(x.dt, x.off, rows, kv, None)
    torch.cuda.synchronize()
    at = x.dest.cuda()
    return unpack(kv.k[0, at].cpu().numpy()), kv.k_scale[0, at].cpu().numpy()


def test_the_code_is_that_of_the_fp64_value():
    """a cos - b sin = 1/4 + 2^-k, the border between codes 0 and 1: a number of fp64 up to k = 54 (its steps there are 2^-54),
    nearest to 1/4 itself from k = 55 on (a tie, to the even of two neighbours), which is a tie between the codes too."""
    far = [20, 30, 45, 50, 53, 54, 55, 56, 60, 100]
    x = Rows("fp32", 0, 1, 128, [2 * len(far)], [0], n_pos=2 * len(far))
    x.k.zero_()
    x.k[:, :, 1] = 4.0                                             # the group's scale is one
    x.k[:, 0, 5], x.k[:, 0, 69] = 0.25, 1.0
    x.cos.fill_(1.0)
    x.sin.zero_()
    x.pos = torch.arange(2 * len(far), dtype=torch.int32)
    for i, k in enumerate(far):
        x.sin[2 * i, 5], x.sin[2 * i + 1, 5] = -2.0 ** -k, 2.0 ** -k
    code, scale = appended(x)
    assert (scale[:, 0] == 127).all() and (code[:, 1] == 6).all()
    assert [int(c) for c in code[0::2, 5]] == [int(k <= 54) for k in far]      # just above the border
    assert not code[1::2, 5].any()                                            # just below it


@pytest.mark.parametrize("above,byte", [(0.0, 252), (2.0 ** 100, 252), (2.0 ** 104, 255)])
def test_magnitudes_up_to_2_128(above, byte):
    """fp32's largest number, one between it and 2^128 and 2^128 itself."""
    x = Rows("fp32", 0, 1, 128, [1], [0])
    x.k.zero_()
    x.k[0, 0, 5], x.k[0, 0, 69] = torch.finfo(torch.float32).max, -2.0 ** 100
    x.cos.fill_(1.0)
    x.sin.zero_()
    x.sin[:, 5] = above / 2.0 ** 100
    code, scale = appended(x)
    assert scale[0, 0] == byte
    if byte != 255:
        assert code[0, 5] == 7 and not np.delete(code[0, :32], 5).any()
