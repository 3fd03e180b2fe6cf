"""The binding's LogitRules takes arrays of 32-bit values without gaps and refuses others: a mask
of truth values, for one, would be read four times past its end."""

import pytest
import torch

from paper_2506_01986_amd import specmemo as sm

I, F = dict(dtype=torch.int32), dict(dtype=torch.float32)


def test_masks():
    idx = torch.zeros(5, **I)
    for dtype in (torch.int32, torch.uint32):
        rules = sm.LogitRules()
        rules.set_mask(torch.zeros(3, 32, dtype=dtype), idx)
        assert (rules.n_masks, rules.mask_words) == (3, 32)
    for mask in (torch.zeros(3, 1000, dtype=torch.bool), torch.zeros(3, 32, dtype=torch.int64), torch.zeros(3, 32),
                 torch.zeros(3, 64, **I)[:, :32], torch.zeros(32, 3, **I).t(), torch.zeros(32, **I)):
        with pytest.raises(ValueError):
            sm.LogitRules().set_mask(mask, idx)
    with pytest.raises(ValueError):
        sm.LogitRules().set_mask(torch.zeros(3, 32, **I), idx.long())


def test_biases():
    off, ids, val = torch.tensor([0, 2, 3], **I), torch.zeros(3, **I), torch.zeros(3, **F)
    rules = sm.LogitRules()
    rules.set_bias(off, ids, val)
    assert rules.n_bias == 3
    for bad in ((off.long(), ids, val), (off, ids.long(), val), (off, ids, val.double()), (off, ids, val.bfloat16()),
                (off, torch.zeros(6, **I)[::2], val), (off, ids, val[:2])):
        with pytest.raises(ValueError):
            sm.LogitRules().set_bias(*bad)


def test_counts_and_penalties():
    counts, pen = torch.zeros(2, 50, **I), torch.ones(2, **F)
    sm.LogitRules(counts, pen, pen, pen)
    sm.LogitRules(None, None, None, pen)
    for bad in (dict(counts=counts.long()), dict(counts=torch.zeros(50, 2, **I).t()), dict(repetition=pen.double()),
                dict(presence=pen.bfloat16()), dict(frequency=torch.ones(4, **F)[::2])):
        with pytest.raises(ValueError):
            sm.LogitRules(**bad)
