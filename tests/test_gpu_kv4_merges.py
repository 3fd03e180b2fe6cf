"""GPU: fp32 attention over 4-bit pools whose key ranges are cut and merged, for each count of 32-column groups."""

import pytest

from tests.kv4_forms import MERGES
from tests.kv4_ref import Batch4
from tests.test_gpu_kv4_attn import prompt_parity

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("name", list(MERGES))
def test_merged_parts(name, d):
    n_q, n_kv, n, L, P, shared = MERGES[name]
    prompt_parity(Batch4("fp32", n_q, n_kv, d, n, L, P, shared, seed=d))
