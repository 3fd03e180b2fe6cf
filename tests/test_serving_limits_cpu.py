"""Limits of the prompt, shared-prefix and logit-rule calls that follow from their 32-bit
arithmetic and from a launch's size, on the host (fake device pointers: only where no GPU
is visible)."""

import pytest

from paper_2506_01986_amd import specmemo as sm
from paper_2506_01986_amd import synth
from tests.test_abi_cpu import FAKE, FakeTrees, cpu_only, expect


@cpu_only
@pytest.mark.parametrize("n", [2 ** 30, 2 ** 31 - 1])
def test_bias_entries(n):
    """A block steps through the entries 256 at a time: their indices plus a step stay within 32 bits."""
    rules = sm.LogitRules()
    rules.bias_off = rules.bias_id = rules.bias_val = FAKE
    rules.n_bias = n
    assert "n_bias" in expect("E_ARG", sm.logit_rules, sm.BF16, FakeTrees([synth.t16()]), 1000, FAKE, None, rules, FAKE * 2,
                              stream=0)
