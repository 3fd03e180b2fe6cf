"""GPU: logit rules on batches whose blocks take several node rows, and on skewed batches,
against numpy in 64 bits."""

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import synth
from tests.test_gpu_logit_rules import Case

pytestmark = pytest.mark.gpu

# nodes of the trees: fewer than a block's rows, than the places of a chunk a row may begin at, and not multiples of either
SIZES = [1, 3, 7, 8, 9, 17, 40, 63, 64, 100, 127, 128]
# type, vocabulary (rows that begin at one, two, four or eight places of a chunk), times the sizes -> node rows a block
# (tests/test_serving_plans.py looks)
CASES = [("bf16", 2055, 1, 2), ("bf16", 8263, 1, 4), ("bf16", 8262, 1, 4), ("bf16", 8260, 1, 4), ("bf16", 8263, 2, 8),
         ("bf16", 31999, 1, 8), ("bf16", 32000, 1, 8), ("fp32", 1029, 1, 2), ("fp32", 4099, 1, 4), ("fp32", 8263, 1, 8),
         ("fp32", 8262, 1, 8), ("fp32", 8264, 1, 8)]


def uneven(dtype, vocab, times):
    r = np.random.default_rng(vocab)
    return Case(dtype, vocab, [synth.random_tree(r, n) for n in SIZES * times], seed=vocab, hist=vocab // 4, bias=vocab // 20,
                masks=5)


@pytest.mark.parametrize("dtype,vocab,times", [c[:3] for c in CASES])
def test_several_rows_a_block(dtype, vocab, times):
    """Penalties, biases with repeated ids, masks; rows of one block that begin at different places of a chunk."""
    x = uneven(dtype, vocab, times)
    x.check(x.run())


@pytest.mark.parametrize("dtype,vocab,times", [CASES[4][:3], CASES[9][:3]])
def test_several_rows_a_block_in_place(dtype, vocab, times):
    x = uneven(dtype, vocab, times)
    want, z = x.run(), x.z.cuda()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(x.run(out=z, z=z).view(bits), want.view(bits))


@pytest.mark.parametrize("dtype,vocab,B", [("fp32", 1000, 513), ("bf16", 1001, 3899)])
def test_one_large_tree_among_single_nodes(dtype, vocab, B):
    """The row groups of the largest tree times the sequences would pass a launch's blocks in y."""
    r = np.random.default_rng(B)
    ts = [synth.chain_tree(1)] * B
    ts[B // 3] = synth.random_tree(r, 128)
    x = Case(dtype, vocab, ts, seed=B, bias=3, masks=4)
    x.check(x.run())
