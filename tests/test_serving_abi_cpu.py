"""Refusals of the prompt, shared-prefix and logit-rule calls, on the host, before any HIP call
(fake device pointers: only where no GPU is visible)."""

import numpy as np
import pytest

from paper_2506_01986_amd import specmemo as sm
from paper_2506_01986_amd import synth
from tests.test_abi_cpu import FAKE, FakeKV, FakeTrees, cpu_only, expect


def prompt(off, kv, n_q=4, dt=sm.BF16, q=FAKE, out=FAKE * 2, ws=FAKE, ws_bytes=1 << 34, prefix=None, scale=0.0):
    sm.prompt_attn(dt, off, kv, n_q, q, out, prefix=prefix, scale=scale, ws=ws, ws_bytes=ws_bytes, stream=0)


@cpu_only
def test_prompt_arguments():
    kv = FakeKV([10, 0], [40, 40], [0, 50])
    expect("E_DTYPE", prompt, [0, 3, 5], kv, dt=7)
    expect("E_DTYPE", prompt, [0, 3, 5], FakeKV([10, 0], [40, 40], [0, 50], d=64))
    expect("E_DTYPE", prompt, [0, 3, 5], FakeKV([10, 0], [40, 40], [0, 50], d=6), dt=sm.FP32)
    expect("E_ARG", prompt, [1, 3, 5], kv)
    expect("E_ARG", prompt, [0, 3, 2], kv)
    expect("E_ARG", prompt, [0], kv)                                    # no sequence
    expect("E_ARG", prompt, [0, 3, 5], kv, n_q=3)
    expect("E_ARG", prompt, [0, 3, 5], kv, n_q=0)
    expect("E_ARG", prompt, [0, 3, 5], kv, q=None)
    expect("E_ARG", prompt, [0, 3, 5], kv, out=FAKE * 2 + 8)
    assert "overlaps" in expect("E_ARG", prompt, [0, 3, 5], kv, out=FAKE + 4096)
    assert "overlaps" in expect("E_ARG", prompt, [0, 3, 5], kv, out=FAKE)
    expect("E_ARG", prompt, [0, 3, 5], kv, scale=float("inf"))
    expect("E_ARG", prompt, [0] * 4098, FakeKV([0] * 4097, [0] * 4097, [0] * 4097, cap_total=10))
    with pytest.raises(ValueError):
        prompt([0, 1, 2, 3], kv)                                        # more sequences than the pool describes
    prompt([0, 0, 0], kv, q=None, out=None, ws=None, ws_bytes=0)        # no tokens: nothing to do


@cpu_only
def test_prompt_budget():
    expect("E_BUDGET", prompt, [0, 31, 31], FakeKV([10, 0], [40, 40], [0, 50]))          # 10 + 31 > 40
    expect("E_BUDGET", prompt, [0, 1, 2], FakeKV([10, 0], [40, 40], [0, 39]))            # slabs overlap
    expect("E_BUDGET", prompt, [0, 1, 2], FakeKV([10, 0], [40, 40], [0, 50], cap_total=89))
    expect("E_BUDGET", prompt, [0, 1], FakeKV([10], [(1 << 23) + 1], [0]))
    expect("E_ARG", prompt, [0, 1], FakeKV([-1], [40], [0]))


@cpu_only
def test_prompt_launch_size():
    # 25.6 million work items of 256 threads: more threads than a launch's 32-bit count
    kv = FakeKV([0], [200000], [0], d=4, cap_total=200000, n_kv=4096)
    assert "work items" in expect("E_ARG", prompt, [0, 200000], kv, n_q=4096, dt=sm.FP32, out=1 << 45, ws_bytes=1 << 60)


@cpu_only
def test_prompt_workspace():
    kv = FakeKV([5000], [6000], [0])
    need = sm.prompt_attn_bytes(sm.BF16, [0, 1], kv, 4)
    assert need > 0
    expect("E_WORKSPACE", prompt, [0, 1], kv, ws_bytes=need - 1)
    expect("E_WORKSPACE", prompt, [0, 1], kv, ws=None)
    expect("E_WORKSPACE", prompt, [0, 1], kv, ws=FAKE + 4)
    assert sm.prompt_attn_bytes(sm.BF16, [0, 1], FakeKV([5], [60], [0]), 4) == 0         # one chunk
    assert sm.prompt_attn_bytes(sm.BF16, [0, 99], FakeKV([5], [60], [0]), 4) == 0        # invalid
    # more sets than the kernel arguments describe: the table is in the workspace
    many = FakeKV([5] * 90, [10] * 90, [10 * i for i in range(90)])
    assert sm.prompt_attn_bytes(sm.BF16, list(range(91)), many, 4) >= 90 * 52
    assert sm.prompt_attn_bytes(sm.BF16, list(range(77)), many, 4) == 0


@cpu_only
def test_plan_of_the_largest_prompt():
    # more row blocks than block slots by far: nothing to split, whatever the amount of work
    for n in (1 << 20, 1 << 28):
        assert sm.prompt_attn_bytes(sm.FP32, [0, n], FakeKV([0], [n], [0], d=4, n_kv=1), 1) == 0


@cpu_only
def test_prefix():
    kv = FakeKV([10, 0], [40, 40], [9000, 9050], cap_total=9100)
    ok = dict(ws=None, ws_bytes=0)                                      # a valid call would stop at its workspace
    bad = lambda base, n: expect("E_BUDGET", prompt, [0, 3, 5], kv, prefix=sm.Prefix(base, n))
    expect("E_WORKSPACE", prompt, [0, 1, 2], kv, prefix=sm.Prefix([0, 0], [9000, 9000]), **ok)
    expect("E_WORKSPACE", prompt, [0, 1, 2], kv, prefix=sm.Prefix([0, 0], [9010, 9010]), **ok)   # with committed rows of slab 0
    bad([0, 0], [9011, 9011])                                           # its eleventh row is not committed
    bad([0, 9050], [5, 1])                                              # slab 1 has none
    bad([0, 9095], [5, 6])                                              # past the pool
    bad([-1, 0], [5, 5])
    bad([2 ** 63 - 5, 0], [5, 5])
    expect("E_ARG", prompt, [0, 3, 5], kv, prefix=sm.Prefix([0, 0], [-1, 5]))
    big = FakeKV([10, 0], [40, 40], [1 << 24, (1 << 24) + 50])
    expect("E_BUDGET", prompt, [0, 3, 5], big, prefix=sm.Prefix([0, 0], [(1 << 23) + 1] * 2))
    huge = FakeKV([10], [40], [1 << 31], d=4, cap_total=1 << 32)
    expect("E_BUDGET", prompt, [0, 3], huge, dt=sm.FP32, prefix=sm.Prefix([0], [2 ** 31 - 1]))
    expect("E_ARG", prompt, [0, 3], FakeKV([10], [40], [0], cap_total=1 << 40))
    with pytest.raises(ValueError):
        prompt([0, 3, 5], kv, prefix=sm.Prefix([0], [5]))
    with pytest.raises(ValueError):
        sm.Prefix([0, 1], [5])


@cpu_only
def test_tree_prefix():
    t = FakeTrees([synth.t16(), synth.t16()])
    kv = FakeKV([10, 0], [40, 40], [9000, 9050], cap_total=9100)

    def call(trees=t, pool=kv, px=sm.Prefix([0, 0], [8000, 8000]), n_q=4, q=FAKE, ws=FAKE, ws_bytes=1 << 34, dt=sm.BF16):
        sm.tree_attn_prefix(dt, trees, pool, px, n_q, q, FAKE * 2, ws=ws, ws_bytes=ws_bytes, stream=0)

    need = sm.tree_attn_prefix_bytes(sm.BF16, t, kv, sm.Prefix([0, 0], [8000, 8000]), 4)
    assert need > 0
    expect("E_WORKSPACE", call, ws_bytes=need - 1)
    expect("E_ARG", call, px=None)
    expect("E_ARG", call, q=FAKE + 2)
    expect("E_ARG", call, n_q=5)
    expect("E_DTYPE", call, dt=3)
    expect("E_BUDGET", call, pool=FakeKV([30, 0], [40, 40], [9000, 9050], cap_total=9100))
    expect("E_BUDGET", call, px=sm.Prefix([0, 0], [8000, 9011]))
    bad = synth.t16()
    bad.parent[5] = 7
    expect("E_TREE", call, trees=FakeTrees([bad, synth.t16()]))
    assert sm.tree_attn_prefix_bytes(sm.BF16, t, kv, sm.Prefix([0, 0], [8000, 9011]), 4) == 0


def test_null_host_arrays():
    lib = sm.load()
    pool = FakeKV([10], [40], [0])
    kv = pool.struct()
    import ctypes as C
    off = np.array([0, 3], np.int32)
    px = sm._Prefix(None, None)
    assert lib.specmemo_prompt_attn(1, 1, None, C.byref(kv), None, 4, 0.0, FAKE, FAKE * 2, FAKE, 1 << 30, None) == -1
    assert lib.specmemo_prompt_attn(1, 1, off.ctypes.data, None, None, 4, 0.0, FAKE, FAKE * 2, FAKE, 1 << 30, None) == -1
    assert lib.specmemo_prompt_attn(1, 1, off.ctypes.data, C.byref(kv), C.byref(px), 4, 0.0, FAKE, FAKE * 2, FAKE, 1 << 30, None) == -1


@cpu_only
def test_rules():
    t = FakeTrees([synth.t16(), synth.t16()])

    def call(rules=None, trees=t, vocab=1000, dt=sm.BF16, z=FAKE, out=FAKE * 2, tok=FAKE):
        sm.logit_rules(dt, trees, vocab, z, tok, rules or sm.LogitRules(repetition=FAKE), out, stream=0)

    class Rules(sm.LogitRules):
        def __init__(self, **k):
            super().__init__()
            self.__dict__.update(k)

    expect("E_DTYPE", call, dt=9)
    expect("E_ARG", call, vocab=0)
    expect("E_ARG", call, vocab=(1 << 30) + 1)
    expect("E_ARG", call, z=None)
    expect("E_ARG", call, out=FAKE + 8)
    assert "overlap" in expect("E_ARG", call, out=FAKE + 64)
    expect("E_ARG", call, tok=None)
    expect("E_ARG", call, rules=Rules(counts=FAKE + 2))
    expect("E_ARG", call, rules=Rules(frequency=FAKE + 1))
    expect("E_ARG", call, rules=Rules(n_bias=3, bias_off=FAKE, bias_id=FAKE))
    expect("E_ARG", call, rules=Rules(n_bias=-1))
    expect("E_ARG", call, rules=Rules(n_masks=2, mask=FAKE, mask_idx=FAKE, mask_words=31))      # 32 needed
    expect("E_ARG", call, rules=Rules(n_masks=2, mask=FAKE, mask_words=32))
    bad = synth.t16()
    bad.parent[5] = 7
    expect("E_TREE", call, trees=FakeTrees([bad]))


@cpu_only
def test_counts():
    call = lambda off, vocab=10, dev=FAKE, tok=FAKE, counts=FAKE: sm.token_counts(vocab, off, dev, tok, counts, stream=0)
    expect("E_ARG", call, [0])
    expect("E_ARG", call, [1, 2])
    expect("E_ARG", call, [0, 3, 2])
    assert "tokens" in expect("E_ARG", call, [0, 2 ** 30])              # 32-bit positions
    expect("E_ARG", call, [0, 3], vocab=0)
    expect("E_ARG", call, [0, 3], dev=None)
    expect("E_ARG", call, [0, 3], tok=None)
    expect("E_ARG", call, [0, 3], counts=FAKE + 2)
    t = FakeTrees([synth.t16()])
    expect("E_ARG", sm.count_accepted, t, 10, FAKE, FAKE, None, 4, FAKE, stream=0)
    expect("E_ARG", sm.count_accepted, t, 10, FAKE, FAKE, FAKE, 0, FAKE, stream=0)
