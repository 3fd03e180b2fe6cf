"""GPU: columns of a query that are far smaller than the largest of their 32, where only they meet keys: the accuracy that
the header states for the 4-bit attention's queries."""

import numpy as np
import pytest

from tests.kv4_query_parts import Columns, stated

pytestmark = pytest.mark.gpu


def parity(dtype, x):
    exact, within, least = stated()[dtype]
    top = np.maximum(x.top, least)
    s, tol = x.scores()
    bound = np.where(np.abs(x.x) >= exact * top, 0, within * top) * x.scale + tol
    off = np.abs(s - x.x * x.scale)
    i = np.unravel_index((off / bound).argmax(), off.shape)
    assert (off <= bound).all(), f"{(off > bound).sum()} of {off.size} off, worst at {i}: {off[i]:.3g} against {bound[i]:.3g}"


# query rows of one KV head: up to 16, of 64-row blocks, of 128-row blocks
@pytest.mark.parametrize("far", [3, 8, 9, 11])
@pytest.mark.parametrize("T", [4, 16, 600])
def test_bf16(T, far):
    parity("bf16", Columns("bf16", T, 4, 4, 128, far, seed=far))


@pytest.mark.parametrize("far", [3, 8, 15, 18])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("T", [4, 50])
def test_fp32(T, d, far):
    parity("fp32", Columns("fp32", T, 3, 4, d, far, seed=far))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 96)])
@pytest.mark.parametrize("top", [120, 60, -60, -101, -104, -108, -112, -118])
@pytest.mark.parametrize("T", [4, 50])
def test_far_columns(dtype, d, top, T):
    """Columns of every magnitude, the scale to match."""
    parity(dtype, Columns(dtype, T, 4, 4, d, 6, top_exp=top, seed=T))
