"""The queries of the 4-bit attention as sums of six-bit parts: what include/specmemo.h says of their accuracy, the parts
in 64 bits, and attention calls whose results show one column of a query far more exactly than they are rounded."""

import os
import re

import numpy as np
import torch

from paper_2506_01986_amd import specmemo as sm
from tests.kv4_ref import pack, quantise

SHIFTS = {"bf16": (0, 4, 10), "fp32": (0, 4, 9, 14, 19)}
SIX_BITS = np.concatenate([np.arange(16) / 8, 2 + np.arange(8) / 4, 4 + np.arange(8) / 2])


def stated():
    """(columns from this much of the largest up are exact, others within this much of it, the least that it counts as)"""
    text = re.sub(r"\s+\*?\s*", " ", open(sm.HEADER).read())
    a, b = re.search(r"columns of magnitude below 2\^-([\d.]+) of the largest of their 32 are taken within 2\^-([\d.]+) of it", text).groups()
    c = re.search(r"fp32: columns are taken within 2\^-([\d.]+) of the largest of their 32", text).group(1)
    least = re.search(r"A largest under 2\^-([\d.]+) counts as 2\^-\1 in this", text)
    least = 2.0 ** -float(least.group(1)) if least else 0.0
    return {"bf16": (2.0 ** -float(a), 2.0 ** -float(b), least), "fp32": (np.inf, 2.0 ** -float(c), least)}


def rest(x, shifts):
    """What the parts leave of magnitudes x in units of 2^e, where the largest lies in (3.75, 7.5]."""
    x = np.asarray(x, np.float64)
    for s in shifts:
        y = np.abs(x) * 2.0 ** s
        i = np.clip(np.searchsorted(SIX_BITS, y), 1, 31)
        lo, hi = SIX_BITS[i - 1], SIX_BITS[i]
        up = (y - lo > hi - y) | ((y - lo == hi - y) & (i % 2 == 0))          # ties to the even code
        x = x - np.sign(x) * np.where(y > 7.5, 7.5, np.where(up, hi, lo)) * 2.0 ** -s
    return np.abs(x)


class Columns:
    """A prompt of one sequence behind two committed rows.  The first key has a 1 in one column of each KV head, all other
    keys are zero; the first value is 1, all others 0.  A query's score with the first key is that column times the scale,
    with the n others 0, and the result p = e^s / (e^s + n) gives s = ln p + ln n - ln(1 - p): a rounding of p is an
    absolute error of s, so that s around -40 shows the column to 2^-12 of itself in bf16, 2^-23 in fp32."""

    def __init__(self, dtype, T, n_kv, g, d, far, top_exp=0, seed=0, s_far=-60.0):
        """Columns are 2^-far .. 2^-far x 8 of the largest of their 32, whose exponent is top_exp."""
        r = np.random.default_rng(seed)
        self.dtype = torch.float32 if dtype == "fp32" else torch.bfloat16
        self.dt = sm.FP32 if dtype == "fp32" else sm.BF16
        self.T, self.n_q, self.n_kv, self.d = T, n_q, n_kv, d = T, n_kv * g, n_kv, d
        col = np.array([(5 + 37 * h) % d for h in range(n_kv)]).repeat(g)            # of each query head
        q = r.standard_normal((T, n_q, d)) * 2.0 ** r.integers(-20, 20, (T, n_q, d // 32)).repeat(32, 2)   # other groups: any scale
        top = r.uniform(1, 2, (T, n_q))
        top = np.where(r.random((T, n_q)) < 0.5, 1.875 * (1 + 2.0 ** -r.integers(5, 9, (T, n_q))), top)      # just above 3.75 units
        mine = (np.arange(d) // 32)[None, :] == (col // 32)[:, None]                                         # [n_q][d]
        for t in range(T):
            q[t][mine] = 0
        x = -top * 2.0 ** (3 * r.random((T, n_q)) - far)
        for h in range(n_q):
            lead = col[h] // 32 * 32
            for c in range(lead, lead + 32):
                q[:, h, c] = r.choice([-1, 1], T) * top[:, h] * r.random(T)
            q[:, h, lead + (col[h] + 7) % 32] = top[:, h] * r.choice([-1, 1], T)
            q[:, h, col[h]] = x[:, h]
        q *= np.where(mine, 2.0 ** top_exp, 1.0)
        self.q = torch.from_numpy(q).to(self.dtype)
        got = self.q.double().numpy()
        self.x = got[:, np.arange(n_q), col]
        self.top = np.abs(got * mine[None]).max(-1)
        self.scale = float(np.float32(s_far / self.x.min()))
        k = np.zeros((n_kv, 2 + T, d))
        k[np.arange(n_kv), 0, col[::g]] = 1
        v = np.zeros((n_kv, 2 + T, d))
        v[:, 0] = 1
        self.bytes = [(pack(c), s) for c, s in map(quantise, (k, v))]

    def scores(self):
        """(scores with the first key, a bound of what the rounding beside the queries' parts adds to them)"""
        (k, ks), (v, vs) = self.bytes
        kv = sm.KV4Pool(*(torch.from_numpy(x).cuda() for x in (k, v, ks, vs)), torch.tensor([2], dtype=torch.int32).cuda(), [0], [2 + self.T], [2])
        off = np.array([0, self.T], np.int32)
        out = torch.full_like(self.q, 777.0).cuda()
        n = sm.kv4_prompt_attn_bytes(self.dt, off, kv, self.n_q)
        ws = torch.full((max(16, n),), 255, dtype=torch.uint8, device="cuda")
        sm.kv4_prompt_attn(self.dt, off, kv, self.n_q, self.q.cuda(), out, scale=self.scale, ws=ws, ws_bytes=n)
        torch.cuda.synchronize()
        out = out.cpu().double().numpy()
        assert (out == out[..., :1]).all()
        p, others = out[..., 0], 2.0 + np.arange(self.T)[:, None]
        s = np.log(p) + np.log(others) - np.log1p(-p)
        # the score's sum, its product with the scale and the exponential's argument: eight roundings in 32 bits, of the
        # score (its log2 units are 1.45 times as many); the exponential, sums of weights and quotient: 2^-20 of the result.
        # bf16: the weight and the result are rounded once each, 2^-8 of them.
        tol = np.abs(self.x * self.scale) * 8 * 1.45 * 2.0 ** -24 + 2.0 ** -20
        return s, tol + (2 * 1.01 * 2.0 ** -8 if self.dt == sm.BF16 else 0)
