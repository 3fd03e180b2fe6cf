"""GPU: append of new rows (norm, rotation, pool of either type or of 4 bits), reading 4-bit rows back and their
compaction, against 64 bits."""

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import specmemo as sm
from paper_2506_01986_amd import synth
from tests.kv4_ref import GRID, pack, quantise, unpack, values
from tests.serving_ref import check

pytestmark = pytest.mark.gpu

EPS = 1e-5


class Rows:
    """A batch of new rows for slabs with room around them, and what every buffer has to hold afterwards."""

    def __init__(self, dtype, n_q, n_kv, d, n, L, rot=None, style="halves", norm=False, fused=False, seed=0, n_pos=500, std=1.0,
                 slack=2):
        g = torch.Generator().manual_seed(seed)
        self.dtype = torch.float32 if dtype == "fp32" else torch.bfloat16
        self.dt = sm.FP32 if dtype == "fp32" else sm.BF16
        self.n_q, self.n_kv, self.d, self.n, self.L = n_q, n_kv, d, list(n), list(L)
        self.rot, self.style = d if rot is None else rot, style
        self.off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        T = self.T = int(self.off[-1])
        rand = lambda *s: (torch.randn(*s, generator=g) * std).to(self.dtype)
        if fused:
            self.row = rand(T, n_q + 2 * n_kv, d)
            self.q, self.k, self.v = self.row[:, :n_q], self.row[:, n_q:n_q + n_kv], self.row[:, n_q + n_kv:]
        else:
            self.row, self.q, self.k, self.v = None, rand(T, n_q, d), rand(T, n_kv, d), rand(T, n_kv, d)
        self.q_norm, self.k_norm = ((1 + 0.3 * torch.randn(d, generator=g)).to(self.dtype) if norm else None for _ in range(2))
        self.pos = torch.randint(0, n_pos, (T,), generator=g, dtype=torch.int32)
        angle = torch.arange(n_pos).double()[:, None] * 10000.0 ** (-torch.arange(self.rot // 2).double() * 2 / max(self.rot, 1))
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        at, self.base, self.cap = 3, [], []
        for m, l in zip(n, L):
            self.base.append(at)
            self.cap.append(l + m + slack)
            at += self.cap[-1] + 1
        self.rows = at
        self.dest = torch.cat([torch.arange(m) + b + l for m, b, l in zip(self.n, self.base, self.L)] + [torch.zeros(0)]).long()

    def upload(self, **kw):
        up = lambda x: None if x is None else x.cuda()
        if self.row is not None:
            r = self.row.cuda()
            q, k, v = r[:, :self.n_q], r[:, self.n_q:self.n_q + self.n_kv], r[:, self.n_q + self.n_kv:]
        else:
            q, k, v = up(self.q), up(self.k), up(self.v)
        self.q_out = torch.full((self.T, self.n_q, self.d), 777.0, dtype=self.dtype, device="cuda")
        turn = {} if self.rot == 0 else dict(pos=up(self.pos), cos=up(self.cos), sin=up(self.sin))
        return sm.QKVRows(q if self.n_q else None, k, v, **turn, rot_dim=self.rot,
                          rot_style=sm.ROT_HALVES if self.style == "halves" else sm.ROT_PAIRS, q_norm=up(self.q_norm),
                          k_norm=up(self.k_norm), eps=EPS)

    def pool(self):
        k, v = (torch.full((self.n_kv, self.rows, self.d), 55.0, dtype=self.dtype, device="cuda") for _ in range(2))
        return sm.KVPool(k, v, torch.zeros(len(self.n), dtype=torch.int32, device="cuda"), self.base, self.cap, self.L)

    def pool4(self):
        mem = [torch.full((self.n_kv, self.rows, self.d // w), 171, dtype=torch.uint8, device="cuda") for w in (2, 2, 32, 32)]
        return sm.KV4Pool(*mem, torch.zeros(len(self.n), dtype=torch.int32, device="cuda"), self.base, self.cap, self.L)

    def turned(self, x, w):
        """(norm and rotation in 64 bits, a bound of their rounding in 32): the sum of d squares is off by (d + 2) 2^-24, its
        root by half that, six more operations by one rounding each, the rotation's by two of each product."""
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w.double()
        out, mag = x.clone(), x.abs()
        if self.rot:
            h = self.rot // 2
            a, b = (slice(0, h), slice(h, self.rot)) if self.style == "halves" else (slice(0, self.rot, 2), slice(1, self.rot, 2))
            c, s = (t[self.pos.long().clamp(0, len(t) - 1)].double()[:, None] for t in (self.cos, self.sin))
            out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
            mag[..., a] = (x[..., a] * c).abs() + (x[..., b] * s).abs()
            mag[..., b] = (x[..., b] * c).abs() + (x[..., a] * s).abs()
        half = torch.finfo(self.dtype).eps / 2
        return out, half * out.abs() + (self.d / 2 + 12) * 2.0 ** -24 * mag + 1e-38

    def check_pool(self, pool, want, tol=None):
        """The new rows hold `want` [tokens][n_kv][d]; every other row is as it was."""
        got = pool[:, self.dest.cuda()].transpose(0, 1)
        if tol is None:
            assert torch.equal(got.cpu(), want)
        else:
            check(got, want, tol)
        other = torch.ones(self.rows, dtype=torch.bool)
        other[self.dest] = False
        assert (pool[:, other.cuda()] == pool[0, 0, 0]).all() and pool[0, 0, 0] in (55.0, 171)


BATCHES = {
    # dtype, query heads, KV heads, head dim, new rows, committed rows, options
    "one": ("bf16", 1, 1, 128, [1], [0], {}),
    "tree_b3": ("bf16", 8, 2, 128, [16, 1, 64], [100, 0, 7], dict(norm=True)),
    "ragged": ("bf16", 5, 1, 128, [0, 3, 0, 0, 129, 1, 0], [5, 0, 1, 2, 60, 9, 3], dict(fused=True, norm=True)),
    "pairs": ("bf16", 4, 4, 128, [33, 2], [0, 20], dict(style="pairs", norm=True)),
    "part": ("bf16", 3, 2, 128, [7, 9], [1, 2], dict(rot=48, fused=True)),
    "part_pairs": ("bf16", 3, 2, 128, [7, 9], [1, 2], dict(rot=80, style="pairs")),
    "no_rotation": ("bf16", 4, 2, 128, [40], [3], dict(rot=0, norm=True)),
    "no_queries": ("bf16", 0, 8, 128, [40, 3], [3, 0], {}),
    "many": ("bf16", 2, 1, 128, [(i * 7) % 4 for i in range(700)], [i % 3 for i in range(700)], dict(norm=True)),
    "heads_7_of_3": ("bf16", 7, 3, 128, [50], [0], {}),
    "fp32": ("fp32", 4, 4, 64, [16], [128], {}),
    "fp32_norm": ("fp32", 6, 2, 96, [5, 0, 33], [1, 2, 3], dict(norm=True, fused=True)),
    "fp32_pairs": ("fp32", 2, 1, 32, [70, 1], [0, 1], dict(style="pairs", rot=24)),
    "fp32_128": ("fp32", 3, 3, 128, [9], [0], dict(rot=40, norm=True)),
}


@pytest.mark.parametrize("name", list(BATCHES))
def test_append(name):
    *a, opts = BATCHES[name]
    x = Rows(*a, seed=len(name), **opts)
    rows, kv = x.upload(), x.pool()
    sm.kv_append(x.dt, x.off, rows, kv, x.q_out)
    torch.cuda.synchronize()
    check(x.q_out, *x.turned(x.q, x.q_norm))
    x.check_pool(kv.k, *x.turned(x.k, x.k_norm))
    x.check_pool(kv.v, x.v)


@pytest.mark.parametrize("d,rot,style", [(4, 0, "halves"), (20, 16, "halves"), (36, 24, "pairs"), (100, 96, "halves"), (8, 8, "halves"),
                                         (124, 8, "pairs")])
def test_append_head_dims(d, rot, style):
    x = Rows("fp32", 3, 2, d, [5, 70], [0, 9], rot=rot, style=style, norm=True, seed=d)
    rows, kv = x.upload(), x.pool()
    sm.kv_append(x.dt, x.off, rows, kv, x.q_out)
    torch.cuda.synchronize()
    check(x.q_out, *x.turned(x.q, x.q_norm))
    x.check_pool(kv.k, *x.turned(x.k, x.k_norm))
    x.check_pool(kv.v, x.v)


@pytest.mark.parametrize("name", list(BATCHES))
def test_append4(name):
    *a, opts = BATCHES[name]
    x = Rows(*a, seed=len(name), **opts)
    rows, kv = x.upload(), x.pool4()
    sm.kv4_append(x.dt, x.off, rows, kv, x.q_out)
    ko, vo = (torch.full((x.T, x.n_kv, x.d), 777.0, dtype=x.dtype, device="cuda") for _ in range(2))
    sm.kv4_read(x.dt, x.off, kv, ko, vo)
    torch.cuda.synchronize()
    check(x.q_out, *x.turned(x.q, x.q_norm))
    for y, codes, scales, out in ((x.turned(x.k, x.k_norm)[0], kv.k, kv.k_scale, ko), (x.v.double(), kv.v, kv.v_scale, vo)):
        code, scale = quantise(y.numpy())
        x.check_pool(scales, torch.from_numpy(scale))
        x.check_pool(codes, torch.from_numpy(pack(code)))
        assert torch.equal(out.cpu().double(), torch.from_numpy(values(code, scale)))


# as many rows as let a slot have two heads or four, some slots with fewer (a block's 8 or 16 slots times twice or four
# times 512 blocks of rows)
LARGE = {
    "two_heads_7_of_3": ("bf16", 7, 3, 128, [800, 0, 1, 699], [3, 1, 0, 2], dict(norm=True)),
    "four_heads_7_of_3": ("bf16", 7, 3, 128, [1500, 0, 1, 1100], [3, 1, 0, 2], dict(norm=True, fused=True)),
    "four_heads_5_of_1": ("bf16", 5, 1, 128, [4999, 1], [0, 700], dict(rot=80, style="pairs")),
    "keys_alone": ("bf16", 0, 9, 128, [1900], [1], dict(norm=True)),
    "fp32_6_of_2": ("fp32", 6, 2, 96, [1000, 3, 700], [0, 5, 1], dict(norm=True, style="pairs", fused=True)),
    "fp32_9_of_9": ("fp32", 9, 9, 64, [1300], [7], dict(rot=40, norm=True)),
}


@pytest.mark.parametrize("name", list(LARGE))
def test_append_large(name):
    *a, opts = LARGE[name]
    x = Rows(*a, seed=len(name), **opts)
    rows, kv = x.upload(), x.pool()
    sm.kv_append(x.dt, x.off, rows, kv, x.q_out)
    torch.cuda.synchronize()
    check(x.q_out, *x.turned(x.q, x.q_norm))
    x.check_pool(kv.k, *x.turned(x.k, x.k_norm))
    x.check_pool(kv.v, x.v)


@pytest.mark.parametrize("name", list(LARGE))
def test_append4_large(name):
    *a, opts = LARGE[name]
    x = Rows(*a, seed=len(name), **opts)
    rows, kv = x.upload(), x.pool4()
    sm.kv4_append(x.dt, x.off, rows, kv, x.q_out)
    torch.cuda.synchronize()
    check(x.q_out, *x.turned(x.q, x.q_norm))
    for y, codes, scales in ((x.turned(x.k, x.k_norm)[0], kv.k, kv.k_scale), (x.v.double(), kv.v, kv.v_scale)):
        code, scale = quantise(y.numpy())
        x.check_pool(scales, torch.from_numpy(scale))
        x.check_pool(codes, torch.from_numpy(pack(code)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_codes(dtype):
    """Values on and beside every border between codes, at every scale; groups of zeros, of the smallest and largest numbers,
    with an infinity or a NaN."""
    d, T = 128, 251
    x = Rows(dtype, 0, 1, d, [T], [0], rot=0)
    r = np.random.default_rng(1)
    border = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7])
    v = np.zeros((T, 1, d))
    for t in range(T):
        y = r.choice(border, d) * r.choice([-1, 1], d)
        y = y * (1 + r.integers(-1, 2, d) * (2.0 ** -7 if dtype == "bf16" else 2.0 ** -23))
        y[::32] = r.choice([4, 5, 6.5, 7], 4)                    # the scale is that of the row's number
        y = np.clip(y, -7, 7)
        v[t, 0] = y * 2.0 ** (t - 125)
    v[3, 0, :32] = 0
    v[3, 0, 5] = -0.0
    v[4, 0, 40], v[5, 0, 70], v[6, 0, 100] = np.inf, np.nan, -np.inf
    v[7, 0, :32] = 1e-45                                         # fp32's smallest, nothing in bf16
    v[8, 0, :32] = np.where(np.arange(32) == 3, float(torch.finfo(x.dtype).max), 1.0)
    x.v = torch.from_numpy(v).to(x.dtype)
    x.k = x.v.flip(0).contiguous()
    rows, kv = x.upload(), x.pool4()
    sm.kv4_append(x.dt, x.off, rows, kv, None)
    ko, vo = (torch.empty(T, 1, d, dtype=x.dtype, device="cuda") for _ in range(2))
    sm.kv4_read(x.dt, x.off, kv, ko, vo)
    torch.cuda.synchronize()
    for y, codes, scales, out in ((x.k, kv.k, kv.k_scale, ko), (x.v, kv.v, kv.v_scale, vo)):
        code, scale = quantise(y.double().numpy())
        assert (scale == 255).sum() == 3
        x.check_pool(scales, torch.from_numpy(scale))
        got = unpack(codes[0, x.dest.cuda()].cpu().numpy())
        fine = np.repeat(scale[:, 0] != 255, 32, 1)
        assert np.array_equal(got[fine], code[:, 0][fine])
        assert np.array_equal(out.cpu().double().numpy(), values(code, scale), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_keys_of_an_infinite_norm(dtype):
    """A normed key with an infinity: its column and the one it turns with are NaN, all others x / inf = 0;
    a NaN takes the whole row.  No tolerance: zeros and NaN are exact in both forms."""
    x = Rows(dtype, 2, 1, 128, [4], [0], norm=True, rot=64, seed=4)
    x.k[1, 0, 5], x.k[2, 0, 100], x.k[3, 0, 64] = np.inf, -np.inf, np.nan
    rows, kv = x.upload(), x.pool4()
    sm.kv4_append(x.dt, x.off, rows, kv, x.q_out)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        want, _ = x.turned(x.k, x.k_norm)
    code, scale = quantise(want.numpy())
    assert (scale[1, 0] == 255).tolist() == [True, True, False, False]         # columns 5 and 37
    assert (scale[2, 0] == 255).tolist() == [False, False, False, True] and (scale[3, 0] == 255).all()
    got = kv.k_scale[:, x.dest.cuda()].transpose(0, 1).cpu().numpy()
    assert np.array_equal(got, scale)
    bits = unpack(kv.k[:, x.dest.cuda()].transpose(0, 1).cpu().numpy())
    held = np.repeat(scale != 255, 32, -1)
    held[0] = False                                                            # token 0 is as in test_append4
    assert np.array_equal(bits[held] & 7, code[held] & 7) and not (bits[held] & 7).any()
    # the same into a pool of the inputs' type
    rows, kv = x.upload(), x.pool()
    sm.kv_append(x.dt, x.off, rows, kv, x.q_out)
    torch.cuda.synchronize()
    got = kv.k[:, x.dest.cuda()].transpose(0, 1).cpu().double()
    assert torch.equal(got[1:].isnan(), want[1:].isnan())
    assert (got[1:][~want[1:].isnan()] == 0).all()


def test_keys_next_to_borders():
    """Rotated keys within 2^-40 of a border fall on its right side: y_a = a cos - b sin with a cos on a border and b sin of
    either sign and next to nothing."""
    d = 128
    x = Rows("fp32", 0, 1, d, [2 * 7], [0])
    border = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    x.k.zero_()
    x.k[:, :, 1] = 6.0                                           # the group's scale is one
    x.k[:, :, 65] = 2.0 ** -10
    x.cos, x.sin = torch.ones(2, 64), torch.full((2, 64), 2.0 ** -45)
    x.sin[:, 1] = 0
    x.sin[1] *= -1
    for i, b in enumerate(border):
        for sign in (0, 1):
            x.k[2 * i + sign, 0, 5], x.k[2 * i + sign, 0, 69] = b, 1.0
            x.pos[2 * i + sign] = sign
    rows, kv = x.upload(), x.pool4()
    sm.kv4_append(x.dt, x.off, rows, kv, None)
    torch.cuda.synchronize()
    code, scale = quantise(x.turned(x.k, None)[0].numpy())
    got = unpack(kv.k[0, x.dest.cuda()].cpu().numpy())
    assert np.array_equal(got & 7, code[:, 0] & 7)
    assert [int(c) for c in got[:, 5]] == [i + s for i in range(7) for s in (0, 1)]


def test_positions_out_of_range():
    """Tokens without a row of the table write nothing."""
    for four in (False, True):
        x = Rows("bf16", 4, 2, 128, [9, 5], [3, 0], seed=3)
        for i, p in ((0, -1), (4, 500), (8, 2 ** 31 - 1), (9, -2 ** 31), (13, 500)):
            x.pos[i] = p
        gone = torch.tensor([0, 4, 8, 9, 13])
        rows, kv = x.upload(), x.pool4() if four else x.pool()
        (sm.kv4_append if four else sm.kv_append)(x.dt, x.off, rows, kv, x.q_out)
        torch.cuda.synchronize()
        assert (x.q_out[gone.cuda()] == 777.0).all()
        keep = torch.ones(x.T, dtype=torch.bool)
        keep[gone] = False
        q, tol = x.turned(x.q, None)
        check(x.q_out[keep.cuda()], q[keep], tol[keep])
        was = 171 if four else 55.0
        assert all((p[:, x.dest[gone].cuda()] == was).all() for p in ((kv.k, kv.v, kv.k_scale, kv.v_scale) if four else (kv.k, kv.v)))


def test_in_place_and_strides():
    """q_out may be q itself; tokens may lie far apart."""
    x = Rows("bf16", 4, 2, 128, [40], [3], norm=True, seed=4)
    wide = torch.full((40, 1000), 3.0, dtype=torch.bfloat16)
    wide[:, 8:264] = x.k.reshape(40, 256)
    wide[:, 264:520] = x.v.reshape(40, 256)
    w = wide.cuda()
    q = x.q.cuda()
    rows = sm.QKVRows(q, w[:, 8:264].unflatten(1, (2, 128)), w[:, 264:520].unflatten(1, (2, 128)), x.pos.cuda(), x.cos.cuda(),
                      x.sin.cuda(), q_norm=x.q_norm.cuda(), k_norm=x.k_norm.cuda(), eps=EPS)
    kv = x.pool()
    sm.kv_append(x.dt, x.off, rows, kv, q)
    torch.cuda.synchronize()
    check(q, *x.turned(x.q, x.q_norm))
    x.check_pool(kv.k, *x.turned(x.k, x.k_norm))
    x.check_pool(kv.v, x.v)


def test_far_rows():
    """Slabs behind 2^32 bytes of rows, many more of them than a 32-bit offset covers."""
    x = Rows("bf16", 2, 2, 128, [3, 2], [1, 0], seed=5)
    x.base = [20_000_000, 30_000_000]
    x.rows = 30_000_010
    x.dest = torch.cat([torch.arange(3) + 20_000_001, torch.arange(2) + 30_000_000])
    rows, kv = x.upload(), x.pool()
    sm.kv_append(x.dt, x.off, rows, kv, x.q_out)
    torch.cuda.synchronize()
    x.check_pool(kv.k, *x.turned(x.k, None))
    x.check_pool(kv.v, x.v)
    del kv
    x.n_kv, kv4 = 2, None
    x.base = [70_000_000, 79_000_000]
    x.rows = 80_000_000
    x.dest = torch.cat([torch.arange(3) + 70_000_001, torch.arange(2) + 79_000_000])
    kv4 = x.pool4()
    sm.kv4_append(x.dt, x.off, rows, kv4, x.q_out)
    ko, vo = (torch.empty(5, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sm.kv4_read(x.dt, x.off, kv4, ko, vo)
    torch.cuda.synchronize()
    for y, codes, out in ((x.turned(x.k, None)[0], kv4.k, ko), (x.v.double(), kv4.v, vo)):
        code, scale = quantise(y.numpy())
        x.check_pool(codes, torch.from_numpy(pack(code)))
        assert torch.equal(out.cpu().double(), torch.from_numpy(values(code, scale)))


@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_compact(d):
    """Accepted rows move, codes and scales; everything else, and sequences with invalid paths, stay as they were."""
    r = np.random.default_rng(d)
    B, n_kv, stride = 300, 2, 6
    ts = [synth.random_tree(r, int(m), max_depth=4) for m in r.integers(1, 40, B)]
    off = np.concatenate([[0], np.cumsum([t.n for t in ts])])
    trees = sm.Trees(off, *(np.concatenate([getattr(t, f) for t in ts]) for f in ("parent", "depth", "rank")), device="cuda")
    L = r.integers(0, 30, B).astype(np.int32)
    cap = np.array([l + t.n + 1 for l, t in zip(L, ts)], np.int32)
    base = np.concatenate([[0], np.cumsum(cap)])[:-1].astype(np.int64)
    rows = int(cap.sum())
    mem = [torch.from_numpy(r.integers(0, 256, (n_kv, rows, d // w)).astype(np.uint8)) for w in (2, 2, 32, 32)]
    want = [m.clone() for m in mem]
    acc, path = np.zeros(B, np.int32), np.full((B, stride), -1, np.int32)
    seq_len = L.copy()
    for b, t in enumerate(ts):
        u, p = int(r.integers(0, t.n)), []
        while u >= 0:
            p.append(u)
            u = int(t.parent[u])
        p = p[::-1]
        acc[b], path[b, :len(p)] = len(p) - 1, p
        if b % 13 == 0:                                          # invalid, one way or another
            kind = b // 13 % 4
            if kind == 0:
                acc[b] = -1
            elif kind == 1:
                acc[b] = stride
            elif kind == 2:
                path[b, 0] = 1
            else:
                acc[b], path[b, 1] = 1, t.n
            continue
        seq_len[b] += len(p)
        for m, w in zip(mem, want):
            for j, node in enumerate(p):
                w[:, base[b] + L[b] + j] = m[:, base[b] + L[b] + node]
    dev = [m.cuda() for m in mem]
    kv = sm.KV4Pool(*dev, torch.from_numpy(L).cuda(), base, cap, L)
    sm.kv4_compact(trees, kv, torch.from_numpy(acc).cuda(), torch.from_numpy(path).cuda(), stride)
    torch.cuda.synchronize()
    for m, w in zip(dev, want):
        assert torch.equal(m.cpu(), w)
    assert np.array_equal(kv.seq_len.cpu().numpy(), seq_len)


def test_captured():
    """Append, compaction and reading back in a graph, replayed on new inputs."""
    x = Rows("bf16", 8, 2, 128, [16, 16], [100, 7], norm=True, seed=6)
    t = synth.t16()
    trees = sm.Trees([0, 16, 32], *(np.concatenate([getattr(t, f)] * 2) for f in ("parent", "depth", "rank")), device="cuda")
    rows, kv = x.upload(), x.pool4()
    leaf, p = 15, []
    while leaf >= 0:
        p.append(leaf)
        leaf = int(t.parent[leaf])
    p = p[::-1]
    acc = torch.tensor([len(p) - 1, 0], dtype=torch.int32, device="cuda")
    path = torch.full((2, 6), -1, dtype=torch.int32)
    path[0, :len(p)], path[1, 0] = torch.tensor(p, dtype=torch.int32), 0
    path = path.cuda()
    ko, vo = (torch.zeros(len(p) + 1, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            sm.kv4_append(x.dt, x.off, rows, kv, x.q_out)
            sm.kv4_compact(trees, kv, acc, path, 6)
            sm.kv4_read(x.dt, [0, len(p), len(p) + 1], kv, ko, vo)
        for i in range(3):
            x.k = torch.randn(x.k.shape, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16)
            rows.k.copy_(x.k)
            ko.zero_()
            g.replay()
            s.synchronize()
            kept = torch.tensor(p + [16])
            code, scale = quantise(x.turned(x.k, x.k_norm)[0][kept].numpy())
            assert torch.equal(ko.cpu().double(), torch.from_numpy(values(code, scale))), i
            code, scale = quantise(x.v.double()[kept].numpy())
            assert torch.equal(vo.cpu().double(), torch.from_numpy(values(code, scale))), i
            assert kv.seq_len.cpu().tolist() == [100 + len(p), 8]
