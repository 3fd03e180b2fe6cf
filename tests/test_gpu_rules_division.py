"""GPU: the repetition penalty divides positive logits: fp32 results are the correctly rounded
quotient, and any positive penalty gives it, whose reciprocal fp32 cannot hold too."""

import numpy as np
import pytest

from paper_2506_01986_amd import specmemo as sm
from paper_2506_01986_amd import synth
from tests.test_gpu_logit_rules import Case

pytestmark = pytest.mark.gpu


def case(dtype, vocab, rep, tree=None, seed=1):
    x = Case(dtype, vocab, [tree or synth.t16()] * len(rep), seed=seed, hist=3 * vocab, penalties=("repetition",))
    x.pen["repetition"][:] = rep
    return x


@pytest.mark.parametrize("vocab", [1000, 1003])       # whole chunks, and single values at both ends of a row
def test_fp32_quotients_are_correctly_rounded(vocab):
    """One division or one product and nothing else: numpy's fp32 result, bit for bit."""
    x = case("fp32", vocab, [1.1, 1.3, 0.7, 3.0, 1.0])
    out = x.run().cpu().numpy()
    z = x.z.numpy()
    for b in range(x.B):
        rep = x.pen["repetition"][b]
        for u in range(x.ts[b].n):
            row, c = int(x.off[b]) + u, x.counts[b].copy()
            a = u
            while a >= 0:
                c[x.tok[int(x.off[b]) + a]] += 1
                a = int(x.ts[b].parent[a])
            want = np.where(c > 0, np.where(z[row] > 0, z[row] / rep, z[row] * rep), z[row])
            assert want.dtype == np.float32 and (c > 0).any()
            assert np.array_equal(out[row], want), (b, u)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rep", [1e-39, 2.0 ** -130, 2.0 ** -127, 3e38, 2.0 ** 127])
def test_penalties_without_a_normal_reciprocal(dtype, rep):
    """1 / rep overflows, or is subnormal; the logits are sized so that quotient and product are normal numbers."""
    x = case(dtype, 515, [rep, 1.25])
    z = x.z.double().numpy()
    r = np.float64(np.float32(rep))
    up = np.abs(z[:16]) * (2.0 ** 100 if rep > 1 else 2.0 ** -20)       # divided
    down = -np.abs(z[:16]) * (2.0 ** -20 if rep > 1 else 2.0 ** 30)     # multiplied
    x.z[:16] = x.z.new_tensor(np.where(z[:16] > 0, up, down))
    # a product with a subnormal penalty may be subnormal: a step of 2^-149 more (2^-133 in bf16)
    ref, tol = x.reference()
    out = x.run().double().cpu().numpy()
    assert np.isfinite(ref).all() and np.abs(ref[:16]).max() < 2.0 ** 127
    assert (np.abs(out - ref) <= tol + 2.0 ** (-149 if dtype == "fp32" else -133)).all()
    assert (np.abs(ref[:16]) > 0).any() and r > 0
