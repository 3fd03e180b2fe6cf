"""Tensors that the append, 4-bit pool and 4-bit attention calls of the binding refuse: what the kernels would read or
write past their end, or as another type."""

import pytest
import torch

from paper_2506_01986_amd import specmemo as sm

bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)


@pytest.mark.parametrize("v", [bf(2, 29, 128), bf(1, 30, 128), bf(2, 31, 128), torch.zeros(2, 30, 128)])
def test_values_beside_keys(v):
    """A pool's V has K's rows and type: a shorter V would be written past its end."""
    kv = sm.KVPool(bf(2, 30, 128), v, i32(1), [0], [20], [3])
    x = sm.QKVRows(None, bf(5, 2, 128), bf(5, 2, 128))
    with pytest.raises(ValueError):
        sm.kv_append(sm.BF16, [0, 5], x, kv, None)
    kv.k = kv.v = bf(2, 29, 128)                  # cap_total says 30
    with pytest.raises(ValueError):
        sm.kv_append(sm.BF16, [0, 5], x, kv, None)
