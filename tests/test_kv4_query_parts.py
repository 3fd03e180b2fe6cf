"""The header's word on the queries' accuracy, against every bf16 magnitude through the three parts, and many fp32 ones
through the five."""

import os
import re

import numpy as np

from tests.kv4_query_parts import SHIFTS, rest, stated

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_01986_amd", "csrc")


def bf16_magnitudes(lo, hi):
    return np.concatenate([(128 + np.arange(128)) * 2.0 ** (e - 7) for e in range(lo, hi)])


def test_shifts_are_the_kernel_s():
    text = open(os.path.join(CSRC, "kv4_attn.hip")).read()
    assert re.search(r"bf16\s+3 parts, shifts 0, 4, 10", text) and re.search(r"fp32\s+5 parts, shifts 0, 4, 9, 14, 19", text)
    assert "return p == 0 ? 0 : F32 ? 5 * p - 1 : p == 1 ? 4 : 10;" in text


def test_bf16():
    exact, within, _ = stated()["bf16"]
    x = bf16_magnitudes(-30, 3)
    x = x[x <= 7.5]
    left = rest(x, SHIFTS["bf16"])
    worst = 0
    for top in x[x > 3.75]:
        m = x <= top
        worst = max(worst, (left[m] / top).max())
        assert (left[m & (x >= exact * top)] == 0).all(), top
        assert (left[m] <= within * top).all(), (top, np.log2(worst))
    assert worst > within / 1.1                       # not a looser bound than need be


def test_fp32():
    _, within, _ = stated()["fp32"]
    r = np.random.default_rng(0)
    x = (r.uniform(1, 2, 1 << 20) * 2.0 ** r.integers(-30, 3, 1 << 20)).astype(np.float32)
    x = x[x <= 7.5]
    left = rest(x, SHIFTS["fp32"])
    small = np.concatenate([x[x <= 3.75], np.float32([3.75])])
    assert (rest(small, SHIFTS["fp32"]) <= within * 3.75).all()          # any largest is above 3.75 units
    assert (left <= within * np.maximum(x, 3.75)).all()


def test_the_least_largest():
    """The kernel's least unit of the first part, 2^-103, is that of a largest just above 3.75 x 2^-103."""
    text = open(os.path.join(CSRC, "kv4_attn.hip")).read()
    assert "(u & 0x7FFFFFu) > 0x700000u), 24);" in text and 24 - 127 == -103
    for _, _, least in stated().values():
        assert 3.75 * 2.0 ** -103 <= least <= 4 * 2.0 ** -103
