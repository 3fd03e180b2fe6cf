"""The 4-bit rows of the pool in 64 bits, and pools of such rows for the attention's tests."""

import numpy as np
import torch

from paper_2506_01986_amd import specmemo as sm
from tests.serving_ref import Batch

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantise(x):
    """(codes 0..15 [...][d], scale bytes [...][d / 32]) of x in 64 bits, by distance to the values of the format."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(g).max(-1)
    finite = np.isfinite(top) & (top <= np.finfo(np.float32).max)
    top = np.where(finite, top, 0)
    E = np.full(top.shape, -125)
    for e in range(-125, 125):                      # the least that holds the group
        E = np.where(top > 7 * 2.0 ** e, e + 1, E)
    u = np.abs(np.where(finite[..., None], g, 0)) * 2.0 ** -E[..., None].astype(np.float64)
    far = np.abs(u[..., None] - GRID)
    far[..., 1::2] = np.nextafter(far[..., 1::2], np.inf)        # of two equally near the even code
    code = far.argmin(-1) | np.where(np.signbit(g), 8, 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(finite, E + 127, 255).astype(np.uint8)


def values(code, scale):
    """The values of codes and scale bytes, in 64 bits."""
    v = np.where(code & 8, -1.0, 1.0) * GRID[code & 7]
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def pack(code):
    return (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)


def unpack(b):
    return np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], -1)


class Batch4(Batch):
    """A Batch whose pool is in 4 bits.  Rows that no call may read have NaN scales and codes of the largest values."""

    def __init__(self, *a, **k):
        super().__init__(*a, **k)
        self.bytes = []
        for name in ("k", "v"):
            x = getattr(self, name).double().numpy()
            code, scale = quantise(x)
            code[np.isnan(x)] = 7
            self.bytes.append((pack(code), scale))
            setattr(self, name, torch.from_numpy(values(code, scale)).to(self.dtype))      # exact in either type

    def upload(self):
        self.qd = self.q.cuda()
        self.out = torch.full_like(self.qd, 777.0)
        (k, ks), (v, vs) = self.bytes
        self.kv = sm.KV4Pool(*(torch.from_numpy(x).cuda() for x in (k, v, ks, vs)),
                             torch.tensor(self.L, dtype=torch.int32).cuda(), self.base, self.cap, self.L)
        self.px = sm.Prefix(self.pbase, self.plen) if any(self.plen) else None
        return self

    def tolerance(self, p, v, out, q, k, s, scale):
        """That of rows in 16 or 32 bits, and in bf16 the query's form: columns below 2^-8 of the largest of their 32 may be
        off by 2^-16 of it, a score by the sum of that over the keys' columns, a weight's numerator and sum by twice that.
        Codes of 0 let a result be made of far smaller weights alone: a weight under 2^-126 of the largest is no normal
        number and may count for nothing (2^-126 |v| each), nor is such a result (2^-126)."""
        tol = super().tolerance(p, v, out, q, k, s, scale)
        if self.dtype == torch.bfloat16:
            top = q.abs().unflatten(1, (-1, 32)).amax(-1).repeat_interleave(32, 1)
            off = torch.where(q.abs() < top * 2.0 ** -8, top * 2.0 ** -16, torch.zeros_like(q))
            tol = tol + 2 * scale * (off @ k.abs().t()).amax(1, keepdim=True) * (p @ v.abs()) + 2.0 ** -126 * (1 + v.abs().sum(0))
        return tol
