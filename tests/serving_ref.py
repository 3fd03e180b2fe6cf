"""Plain 64-bit forms of the prompt and shared-prefix attention, and the pools
their tests run on."""

import numpy as np
import torch

from paper_2506_01986_amd import specmemo as sm

NAN = float("nan")


class Batch:
    """A batch over one pool: prefixes first, then a slab per sequence with spare rows.  Every row that no call may
    read holds NaN."""

    def __init__(self, dtype, n_q, n_kv, d, n, L, P=None, shared=None, seed=0, slack=3, std=1.0):
        """n: query nodes, L: committed rows, P: prefix rows of each sequence; shared: which sequences use one prefix
        (a group number each; the prefix is as long as its first member says)."""
        g = torch.Generator().manual_seed(seed)
        B = len(n)
        P = [0] * B if P is None else list(P)
        shared = list(range(B)) if shared is None else shared
        self.n, self.L = list(n), list(L)
        self.dtype = torch.float32 if dtype == "fp32" else torch.bfloat16
        self.dt = sm.FP32 if dtype == "fp32" else sm.BF16
        self.n_q, self.n_kv, self.d, self.B = n_q, n_kv, d, B
        self.off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        at, self.pbase, self.plen, seen = 2, [], [], {}
        for b in range(B):
            if shared[b] not in seen:
                seen[shared[b]] = (at, P[b])
                at += P[b] + 1
            base, rows = seen[shared[b]]
            self.pbase.append(base)
            self.plen.append(rows)
        self.base, self.cap = [], []
        for b in range(B):
            self.base.append(at)
            self.cap.append(L[b] + n[b] + slack)
            at += self.cap[b] + 1
        self.k = torch.full((n_kv, at, d), NAN)
        self.v = torch.full((n_kv, at, d), NAN)
        for b in range(B):
            for s, m in ((self.pbase[b], self.plen[b]), (self.base[b], L[b] + n[b])):
                for x in (self.k, self.v):
                    x[:, s:s + m] = torch.randn(n_kv, m, d, generator=g) * std
        self.q = (torch.randn(int(self.off[-1]), n_q, d, generator=g) * std).to(self.dtype)
        self.k, self.v = self.k.to(self.dtype), self.v.to(self.dtype)

    def upload(self):
        self.qd, self.kd, self.vd = self.q.cuda(), self.k.cuda(), self.v.cuda()
        self.out = torch.full_like(self.qd, 777.0)
        self.kv = sm.KVPool(self.kd, self.vd, torch.tensor(self.L, dtype=torch.int32).cuda(), self.base, self.cap, self.L)
        self.px = sm.Prefix(self.pbase, self.plen) if any(self.plen) else None
        return self

    def rows(self, b):
        return np.concatenate([np.arange(self.plen[b]) + self.pbase[b], np.arange(self.L[b] + self.n[b]) + self.base[b]])

    def reference(self, sees, scale=None, device="cpu"):
        """(softmax(q k scale) v, tolerance) in 64 bits; sees(b): bool [n_b][n_b], which of the sequence's own nodes a
        node sees (committed and prefix rows all are)."""
        scale = self.d ** -0.5 if scale is None else scale
        out = torch.empty(self.q.shape, dtype=torch.float64)
        tol = torch.empty_like(out)
        g = self.n_q // self.n_kv
        for b in range(self.B):
            o, n, before = int(self.off[b]), self.n[b], self.plen[b] + self.L[b]
            if n == 0:
                continue
            rows = torch.from_numpy(self.rows(b))
            vis = torch.ones(n, before + n, dtype=torch.bool, device=device)
            vis[:, before:] = sees(b).to(device)
            for h in range(self.n_q):
                q = self.q[o:o + n, h].to(device).double()
                k, v = (x[h // g, rows].to(device).double() for x in (self.k, self.v))
                s = (q @ k.t() * scale).masked_fill(~vis, -np.inf)
                p = torch.softmax(s, 1)
                exact = p @ v
                out[o:o + n, h] = exact.cpu()
                tol[o:o + n, h] = self.tolerance(p, v, exact, q, k, s, scale).cpu()
        return out, tol

    def tolerance(self, p, v, out, q, k, s, scale):
        """A bound of the kernels' rounding.  With A = sum p |v|:
        bf16: each weight is rounded once (2^-8), in the numerator and in the sum of weights, and the result once:
        2^-8 (A + 2 |out|); the fp32 arithmetic beside it is far smaller (1e-4 A).
        fp32: a score's sum of d products is off by at most d 2^-24 sum |q k| scale, its exponent by 2^-22 |s|, the sums
        over the keys by 2^-24 each step; a weight's relative error is the score's error, in numerator and sum."""
        A = p @ v.abs()
        if self.dtype == torch.bfloat16:
            return 2.0 ** -8 * (A + 2 * out.abs()) + 1e-4 * A
        err = (q.abs() @ k.abs().t()).amax(1, keepdim=True) * scale * self.d * 2.0 ** -24
        span = s.masked_fill(s == -np.inf, 0).abs().amax(1, keepdim=True) * 2.0 ** -22
        return 2 * (err + span + (s.shape[1] + 16) * 2.0 ** -24) * A + 1e-30


def causal(n):
    return torch.ones(n, n, dtype=torch.bool).tril()


def root_paths(parent):
    n = len(parent)
    m = torch.zeros(n, n, dtype=torch.bool)
    for u in range(n):
        a = u
        while a >= 0:
            m[u, a] = True
            a = int(parent[a])
    return m


def check(got, ref, tol):
    err = (got.detach().cpu().double() - ref).abs()
    bad = ~(err <= tol)          # NaN counts
    if bad.any():
        i = int(torch.where(bad, err / tol, torch.zeros(())).nan_to_num(1e30).argmax())
        raise AssertionError(f"{int(bad.sum())} of {bad.numel()} values off; worst at {np.unravel_index(i, tuple(err.shape))}: "
                             f"{err.flatten()[i]:.3g} against {tol.flatten()[i]:.3g}")
