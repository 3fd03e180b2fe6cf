"""GPU: logit rules on batches whose blocks take several node rows, and on skewed batches,
against numpy in 64 bits."""

import numpy as np
import pytest

from paper_2506_01986_amd import synth
from tests.test_gpu_logit_rules import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,vocab,B", [("fp32", 1000, 513), ("bf16", 1001, 3899)])
def test_one_large_tree_among_single_nodes(dtype, vocab, B):
    """The row groups of the largest tree times the sequences would pass a launch's blocks in y."""
    r = np.random.default_rng(B)
    ts = [synth.chain_tree(1)] * B
    ts[B // 3] = synth.random_tree(r, 128)
    x = Case(dtype, vocab, ts, seed=B, bias=3, masks=4)
    x.check(x.run())
