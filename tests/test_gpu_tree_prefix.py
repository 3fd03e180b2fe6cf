"""GPU: tree attention over a shared prefix, against 64 bits and against tree
attention over slabs that hold the prefix themselves."""

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import specmemo as sm
from paper_2506_01986_amd import synth
from tests.serving_ref import Batch, check, root_paths

pytestmark = pytest.mark.gpu


def trees_of(kind, B, seed):
    rng = np.random.default_rng(seed)
    one = {"t64": synth.t64, "t16": synth.t16, "single": lambda: synth.chain_tree(1), "chain": lambda: synth.chain_tree(16)}
    if kind in one:
        return [one[kind]()] * B
    return [synth.random_tree(rng, int(n)) for n in rng.integers(1, 129, B)]


def make(dtype, kind, n_q, n_kv, d, L, P, shared, seed=0):
    ts = trees_of(kind, len(L), seed)
    x = Batch(dtype, n_q, n_kv, d, [t.n for t in ts], L, P, shared, seed=seed).upload()
    x.ts = ts
    x.trees = sm.Trees(x.off, *(np.concatenate([getattr(t, f) for t in ts]) for f in ("parent", "depth", "rank")), device="cuda")
    if x.px is None:
        x.px = sm.Prefix(x.pbase, x.plen)
    return x


def run(x):
    n = sm.tree_attn_prefix_bytes(x.dt, x.trees, x.kv, x.px, x.n_q)
    ws = torch.full((max(16, n),), 255, dtype=torch.uint8, device="cuda")
    sm.tree_attn_prefix(x.dt, x.trees, x.kv, x.px, x.n_q, x.qd, x.out, ws=ws, ws_bytes=n)
    torch.cuda.synchronize()
    return x.out


# trees, query heads, KV heads, committed rows, prefix rows, groups of one prefix
CASES = {
    "single_b1": ("single", 1, 1, [0], [1], None),
    "no_prefix": ("t64", 8, 2, [100, 0], [0, 0], None),
    "t64_gqa": ("t64", 16, 2, [70, 0, 129], [300] * 3, [0] * 3),
    "t64_mha": ("t64", 4, 4, [0, 64, 63, 5], [65] * 4, [0] * 4),
    "t16_mha": ("t16", 8, 8, [10, 0, 200, 64, 1, 90], [1000] * 6, [0] * 6),
    "chain": ("chain", 4, 2, [40, 1], [63, 63], [0, 0]),
    "random": ("random", 6, 2, [3, 500, 0, 64, 77], [128] * 5, [0] * 5),
    "single_gqa": ("single", 32, 4, [5, 0, 64, 700, 31, 1, 0, 90], [2000] * 8, [0] * 8),
    "two_groups": ("t16", 8, 1, [5, 9, 0, 64, 30, 2], [200, 200, 200, 77, 77, 77], [0, 0, 0, 1, 1, 1]),
    "apart": ("t16", 8, 2, [5, 9, 0, 64], [200, 64, 200, 64], [0, 1, 0, 1]),        # neighbours differ: nothing is packed
    "some_without": ("random", 5, 1, [5, 9, 0, 64, 20], [90, 90, 0, 90, 90], [0, 0, 1, 0, 0]),
    "many": ("t16", 4, 2, [int(v) for v in np.random.default_rng(6).integers(0, 60, 90)], [600] * 90, [i // 30 for i in range(90)]),
}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", list(CASES))
def test_parity(name, dtype):
    kind, n_q, n_kv, L, P, shared = CASES[name]
    x = make(dtype, kind, n_q, n_kv, 128 if dtype == "bf16" else 48, L, P, shared, seed=len(name))
    check(run(x), *x.reference(lambda b: root_paths(x.ts[b].parent)))


@pytest.mark.parametrize("name", ["t64_gqa", "t16_mha", "random"])
def test_against_slabs_with_the_prefix(name):
    """specmemo_tree_attn on slabs that start with a copy of the prefix: the same rows, two roundings apart."""
    kind, n_q, n_kv, L, P, shared = CASES[name]
    x = make("bf16", kind, n_q, n_kv, 128, L, P, shared, seed=2)
    got = run(x).clone()
    cap = [p + l + n + 1 for p, l, n in zip(x.plen, x.L, x.n)]
    base = np.concatenate([[0], np.cumsum(cap)])[:-1]
    k, v = (torch.zeros(n_kv, int(sum(cap)), 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for b in range(x.B):
        rows = torch.from_numpy(x.rows(b)).cuda()
        k[:, base[b]:base[b] + len(rows)] = x.kd[:, rows]
        v[:, base[b]:base[b] + len(rows)] = x.vd[:, rows]
    kv = sm.KVPool(k, v, x.kv.seq_len, base, cap, [p + l for p, l in zip(x.plen, x.L)])
    n = sm.workspace_bytes(sm.WS_ATTN, x.dt, x.trees, kv, n_q)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(x.qd)
    sm.tree_attn(x.dt, x.trees, kv, n_q, x.qd, out, ws=ws, ws_bytes=n)
    torch.cuda.synchronize()
    _, tol = x.reference(lambda b: root_paths(x.ts[b].parent))
    # the other kernel keeps its parts in bf16: one rounding more of each
    assert ((out.double() - got.double()).abs().cpu() <= 3 * tol).all()


def test_captured():
    kind, n_q, n_kv, L, P, shared = CASES["two_groups"]
    x = make("bf16", kind, n_q, n_kv, 128, L, P, shared, seed=3)
    want = run(x).clone()
    n = sm.tree_attn_prefix_bytes(x.dt, x.trees, x.kv, x.px, n_q)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            sm.tree_attn_prefix(x.dt, x.trees, x.kv, x.px, n_q, x.qd, x.out, ws=ws, ws_bytes=n)
        for i in range(3):
            x.out.zero_()
            ws.fill_(255)
            g.replay()
            s.synchronize()
            assert torch.equal(x.out.view(torch.int16), want.view(torch.int16)), i
