"""Refusals of the append, 4-bit pool and 4-bit attention calls, on the host, before any HIP call (fake device pointers:
only where no GPU is visible)."""

import ctypes as C

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import specmemo as sm
from paper_2506_01986_amd import synth
from tests.kv4_ref import quantise, values
from tests.test_abi_cpu import FAKE, FakeKV, FakeTrees, cpu_only, expect

FAR = 1 << 40            # of the other buffers


class FakeKV4(FakeKV):
    """Codes at FAR and 2 FAR, scales at 3 FAR and 4 FAR."""

    def __init__(self, *a, **k):
        super().__init__(*a, **k)
        self.k, self.v, self.k_scale, self.v_scale = FAR, 2 * FAR, 3 * FAR, 4 * FAR

    struct = sm.KV4Pool.struct


class FakeKVFar(FakeKV):
    def __init__(self, *a, **k):
        super().__init__(*a, **k)
        self.k, self.v = FAR, 2 * FAR


def rows(**kw):
    f = dict(q=FAKE, k=FAKE + (1 << 28), v=FAKE + (2 << 28), q_stride=512, k_stride=256, v_stride=256, q_norm=None, k_norm=None, eps=1e-5,
             cos=FAKE, sin=FAKE, pos=FAKE, n_pos=100, rot_dim=128, rot_style=0)
    f.update(kw)
    return sm._Rows(*(f[n] for n, _ in sm._Rows._fields_))


def append(off, kv, x, n_q=4, dt=sm.BF16, q_out=FAKE + (3 << 28), four=False):
    o = np.asarray(off, np.int32)
    fn = sm.load().specmemo_kv4_append if four else sm.load().specmemo_kv_append
    sm._check(fn(dt, len(o) - 1, o.ctypes.data, C.byref(x), n_q, C.byref(kv.struct()), q_out, None))


def pools(*a, **k):
    return (FakeKVFar(*a, **k), False), (FakeKV4(*a, **k), True)


@cpu_only
def test_append_arguments():
    for kv, four in pools([10, 0], [40, 40], [0, 50]):
        bad = lambda off=(0, 3, 5), code="E_ARG", kv=kv, x=None, **k: expect(code, append, off, kv, x or rows(), four=four, **k)
        bad(code="E_DTYPE", dt=7)
        bad(off=(1, 3, 5))
        bad(off=(0, 3, 2))
        bad(off=(0,))
        bad(n_q=-1)
        bad(n_q=1 << 20)
        bad(x=rows(q=None))
        bad(x=rows(k=FAKE + 8))
        bad(x=rows(v=None))
        assert "q_stride" in bad(x=rows(q_stride=504))          # less than the heads
        assert "k_stride" in bad(x=rows(k_stride=260))          # not whole 16 bytes
        assert "v_stride" in bad(x=rows(v_stride=(1 << 28) + 8))
        bad(q_out=None)
        bad(q_out=FAKE + (3 << 28) + 2)
        bad(x=rows(rot_dim=8))                                  # bf16: multiples of 16
        bad(x=rows(rot_dim=144))
        bad(x=rows(rot_dim=-16))
        bad(x=rows(rot_style=2))
        bad(x=rows(n_pos=0))
        bad(x=rows(cos=None))
        bad(x=rows(sin=FAKE + 4))
        bad(x=rows(pos=None))
        bad(x=rows(pos=FAKE + 2))
        bad(x=rows(q_norm=FAKE + 2))
        bad(x=rows(k_norm=FAKE, eps=-1.0))
        bad(x=rows(k_norm=FAKE, eps=float("nan")))
        assert "q_out overlaps q" in bad(q_out=FAKE + 1024)
        assert "q_out overlaps q" in bad(q_out=FAKE, x=rows(q_stride=1024))      # in place, but with gaps
        assert "q_out overlaps k" in bad(q_out=FAKE + (1 << 28))
        assert "overlaps the pool" in bad(x=rows(v=2 * FAR + 1024))
        assert "overlaps the pool" in bad(q_out=FAR - 1024)
        append((0, 0, 0), kv, rows(q=None, k=None, v=None, cos=None, sin=None, pos=None), q_out=None, four=four)   # no tokens


@cpu_only
def test_append_budget():
    for make, four in ((FakeKVFar, False), (FakeKV4, True)):
        bad = lambda off, kv, code="E_BUDGET": expect(code, append, off, kv, rows(), four=four)
        bad((0, 31, 31), make([10, 0], [40, 40], [0, 50]))             # 10 + 31 > 40
        bad((0, 1, 2), make([10, 0], [40, 40], [0, 39]))               # slabs overlap
        bad((0, 1, 2), make([10, 0], [40, 40], [0, 50], cap_total=89))
        bad((0, 1), make([-1], [40], [0]), "E_ARG")
        bad((0, 1), make([1], [40], [0], d=64), "E_DTYPE")
        bad((0, 1), make([1], [40], [0], cap_total=1 << 46), "E_ARG")


@cpu_only
def test_pool_of_4_bits():
    kv = FakeKV4([10, 0], [40, 40], [0, 50])
    for name in ("k", "v", "k_scale", "v_scale"):
        for at in (None, FAR + 8):
            x = FakeKV4([10, 0], [40, 40], [0, 50])
            setattr(x, name, at)
            expect("E_ARG", append, (0, 3, 5), x, rows(), four=True)
    x = FakeKV4([10, 0], [40, 40], [0, 50])
    x.v_scale = x.k + 64
    assert "overlap" in expect("E_ARG", append, (0, 3, 5), x, rows(), four=True)
    for d in (4, 48, 100, 160):
        expect("E_DTYPE", append, (0, 3, 5), FakeKV4([10, 0], [40, 40], [0, 50], d=d), rows(), dt=sm.FP32, four=True)
    for fn in ("specmemo_kv4_append", "specmemo_kv4_read"):
        o = np.array([0, 1], np.int32)
        args = (1, 1, o.ctypes.data, C.byref(rows()), 4, None, FAKE, None) if "append" in fn else (1, 1, o.ctypes.data, None, FAKE, FAKE, None)
        assert getattr(sm.load(), fn)(*args) == -1

    def read(off=(0, 3, 5), p=kv, k_out=FAKE, v_out=FAKE + (1 << 28), dt=sm.BF16):
        o = np.asarray(off, np.int32)
        sm._check(sm.load().specmemo_kv4_read(dt, len(o) - 1, o.ctypes.data, C.byref(p.struct()), k_out, v_out, None))

    expect("E_DTYPE", read, dt=2)
    expect("E_ARG", read, off=(0, 3, 2))
    expect("E_ARG", read, k_out=None)
    expect("E_ARG", read, v_out=FAKE + 8)
    assert "k_out overlaps v_out" in expect("E_ARG", read, v_out=FAKE + 64)
    assert "pool" in expect("E_ARG", read, k_out=3 * FAR)
    expect("E_BUDGET", read, off=(0, 31, 31))
    read(off=(0, 0, 0), k_out=None, v_out=None)


@cpu_only
def test_compact():
    t = FakeTrees([synth.t16(), synth.t16()])

    def call(trees=t, kv=None, acc=FAKE, path=FAKE, stride=6):
        kv = kv or FakeKV4([10, 0], [40, 40], [0, 50])
        sm._check(sm.load().specmemo_kv4_compact(C.byref(trees.struct()), C.byref(kv.struct()), acc, path, stride, None))

    expect("E_ARG", call, acc=None)
    expect("E_ARG", call, path=FAKE + 2)
    expect("E_ARG", call, stride=0)
    expect("E_BUDGET", call, kv=FakeKV4([30, 0], [40, 40], [0, 50]))
    expect("E_DTYPE", call, kv=FakeKV4([10, 0], [40, 40], [0, 50], d=48))
    expect("E_ARG", call, kv=FakeKV4([1], [40], [0], n_kv=1 << 17), trees=FakeTrees([synth.t16()]))
    x = FakeKV4([10, 0], [40, 40], [0, 50])
    x.seq_len = None
    expect("E_ARG", call, kv=x)
    bad = synth.t16()
    bad.parent[5] = 7
    expect("E_TREE", call, trees=FakeTrees([bad, synth.t16()]))


@cpu_only
def test_attention():
    kv = FakeKV4([5000, 0], [6000, 40], [0, 6000])

    def prompt(off=(0, 1, 3), p=kv, n_q=4, dt=sm.BF16, q=FAKE, out=FAKE * 2, ws=FAKE, ws_bytes=1 << 34, prefix=None, scale=0.0):
        sm.kv4_prompt_attn(dt, list(off), p, n_q, q, out, prefix=prefix, scale=scale, ws=ws, ws_bytes=ws_bytes, stream=0)

    need = sm.kv4_prompt_attn_bytes(sm.BF16, [0, 1, 3], kv, 4)
    assert need > 0
    assert sm.kv4_prompt_attn_bytes(sm.BF16, [0, 1, 3], kv, 3) == 0                    # invalid
    expect("E_WORKSPACE", prompt, ws_bytes=need - 1)
    expect("E_WORKSPACE", prompt, ws=None)
    expect("E_DTYPE", prompt, dt=5)
    expect("E_DTYPE", prompt, p=FakeKV4([10, 0], [40, 40], [0, 50], d=64))             # bf16: 128 alone
    expect("E_DTYPE", prompt, p=FakeKV4([10, 0], [40, 40], [0, 50], d=48), dt=sm.FP32)
    expect("E_ARG", prompt, n_q=3)
    expect("E_ARG", prompt, q=None)
    expect("E_ARG", prompt, out=FAKE)
    expect("E_ARG", prompt, scale=float("inf"))
    expect("E_BUDGET", prompt, off=(0, 1, 42))
    expect("E_BUDGET", prompt, prefix=sm.Prefix([0, 0], [5001, 0]))
    for dt in (sm.BF16, sm.FP32):                                                      # 32-bit offsets within a slab and a prefix
        expect("E_BUDGET", prompt, off=(0, 1), p=FakeKV4([10], [(1 << 23) + 1], [0]), dt=dt)
        big = FakeKV4([10, 0], [40, 40], [1 << 24, (1 << 24) + 50])
        expect("E_BUDGET", prompt, off=(0, 1, 2), p=big, dt=dt, prefix=sm.Prefix([0, 0], [(1 << 23) + 1] * 2))
    x = FakeKV4([5000, 0], [6000, 40], [0, 6000])
    x.k_scale = None
    expect("E_ARG", prompt, p=x)
    prompt(off=(0, 0, 0), q=None, out=None, ws=None, ws_bytes=0)

    t = FakeTrees([synth.t16(), synth.t16()])

    def tree(trees=t, p=kv, n_q=4, ws_bytes=1 << 34, prefix=None, dt=sm.BF16):
        sm.kv4_tree_attn(dt, trees, p, n_q, FAKE, FAKE * 2, prefix=prefix, ws=FAKE, ws_bytes=ws_bytes, stream=0)

    need = sm.kv4_tree_attn_bytes(sm.BF16, t, kv, 4)
    assert need > 0
    expect("E_WORKSPACE", tree, ws_bytes=need - 1)
    expect("E_ARG", tree, n_q=5)
    expect("E_BUDGET", tree, p=FakeKV4([30, 0], [40, 40], [0, 50]))
    expect("E_BUDGET", tree, prefix=sm.Prefix([0, 6010], [0, 1]))
    with pytest.raises(ValueError):
        tree(prefix=sm.Prefix([0], [5]))
    bad = synth.t16()
    bad.parent[5] = 7
    expect("E_TREE", tree, trees=FakeTrees([bad, synth.t16()]))


def test_binding_descriptors():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    k, pos, cos = bf(5, 2, 128), torch.zeros(5, dtype=torch.int32), torch.zeros(9, 64)
    ok = sm.QKVRows(bf(5, 4, 128), k, k, pos, cos, cos)
    assert (ok.n_q, ok.n_kv, ok.rot_dim, ok.n_pos, ok.dt) == (4, 2, 128, 9, sm.BF16)
    for a in (dict(q=bf(5, 4, 64)), dict(q=bf(4, 4, 128)), dict(q=torch.zeros(5, 4, 128)), dict(v=bf(5, 3, 128)), dict(k=None),
              dict(q=bf(5, 128, 4).transpose(1, 2)), dict(q=bf(4, 5, 128).transpose(0, 1)[:, ::2]), dict(cos=torch.zeros(9, 32)),
              dict(sin=None), dict(pos=pos.long()), dict(pos=pos[:4]), dict(q_norm=bf(64)), dict(k_norm=torch.zeros(128)),
              dict(cos=cos.double())):
        f = dict(q=bf(5, 4, 128), k=k, v=k, pos=pos, cos=cos, sin=cos)
        f.update(a)
        with pytest.raises(ValueError):
            sm.QKVRows(**f)
    half = torch.float16
    with pytest.raises(ValueError):
        sm.QKVRows(None, k.to(half), k.to(half))
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    mem = lambda: [u8(2, 30, 64), u8(2, 30, 64), u8(2, 30, 4), u8(2, 30, 4)]
    kv = sm.KV4Pool(*mem(), pos, [0], [20], [3])
    assert (kv.n_kv, kv.cap_total, kv.head_dim) == (2, 30, 128)
    for i, x in ((0, u8(2, 30, 128)[..., ::2]), (1, u8(2, 30, 32)), (2, u8(2, 30, 2)), (3, torch.zeros(2, 30, 4)), (2, u8(2, 29, 4))):
        m = mem()
        m[i] = x
        with pytest.raises(ValueError):
            sm.KV4Pool(*m, pos, [0], [20], [3])
    # what does not belong together
    for off, q_out in (([0, 4], bf(5, 4, 128)), ([0, 5], bf(5, 4, 64)), ([0, 5], torch.zeros(5, 4, 128)), ([0, 5], bf(5, 128, 4).transpose(1, 2)),
                       ([0, 2, 5], bf(5, 4, 128)), ([], bf(5, 4, 128)), ([0, 5], None)):
        with pytest.raises(ValueError):
            sm.kv4_append(sm.BF16, off, ok, kv, q_out)
    with pytest.raises(ValueError):
        sm.kv4_append(sm.FP32, [0, 5], ok, kv, bf(5, 4, 128))
    with pytest.raises(ValueError):
        sm.kv_append(sm.BF16, [0, 5], ok, sm.KVPool(torch.zeros(2, 30, 128), torch.zeros(2, 30, 128), pos, [0], [20], [3]), bf(5, 4, 128))
    with pytest.raises(ValueError):
        sm.kv4_read(sm.BF16, [0, 5], kv, bf(5, 2, 128), bf(4, 2, 128))
    with pytest.raises(ValueError):
        sm.kv4_read(sm.FP32, [0, 5], kv, bf(5, 2, 128), bf(5, 2, 128))


def test_memory():
    assert sm.mem_kv4_bytes(80, 10, 8, 128, 4096) == 2 * 80 * 10 * 8 * 4096 * 68
    assert sm.mem_kv4_bytes(1, 1, 1, 32, 0) == 0
    # 3.76 times the tokens of a bf16 pool in the same bytes
    assert sm.mem_kv_bytes(80, 10, 8, 128, 1700, 2) == sm.mem_kv4_bytes(80, 10, 8, 128, 6400)
    for a in ((80, 10, 8, 100, 1), (-1, 1, 1, 32, 1), (1, 1, 1, 32, -1), (1 << 30, 1 << 30, 1 << 30, 128, 1 << 40)):
        with pytest.raises(sm.SpecmemoError):
            sm.mem_kv4_bytes(*a)


def test_format():
    """The definition of the 4-bit rows: half a step at most, ties to even, the least scale that holds the group."""
    r = np.random.default_rng(0)
    x = r.standard_normal((200, 64)) * 2.0 ** r.integers(-20, 20, (200, 1))
    code, scale = quantise(x)
    v = values(code, scale)
    unit = np.repeat(2.0 ** (scale.astype(int) - 127), 32, 1)
    u = np.abs(x / unit)
    assert u.max() <= 7 and (u.reshape(200, 2, 32).max(-1) > 3.5).all()
    assert (np.abs(v - x) <= unit * np.where(u <= 2, 0.25, np.where(u <= 4, 0.5, 1.0))).all()
    t = np.zeros(32)
    t[:8] = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]
    assert list(values(*quantise(t))[:8]) == [6, 0, 1, 1, 2, 2, 4, 4]
    t[0] = np.nextafter(7, 8)
    assert quantise(t)[1][0] == 128
