"""GPU: attention over a 4-bit pool, of prompts and of candidate trees, against 64 bits."""

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import specmemo as sm
from paper_2506_01986_amd import synth
from tests import serving_forms
from tests.kv4_ref import Batch4
from tests.serving_ref import causal, check, root_paths
from tests.test_gpu_prompt_attn import BF16 as PROMPTS
from tests.test_gpu_tree_prefix import CASES as TREES
from tests.test_gpu_tree_prefix import trees_of

pytestmark = pytest.mark.gpu


def scratch(n):
    return torch.full((max(16, n),), 255, dtype=torch.uint8, device="cuda")     # NaN in every unwritten part


def run_prompt(x, **kw):
    n = sm.kv4_prompt_attn_bytes(x.dt, x.off, x.kv, x.n_q, x.px)
    sm.kv4_prompt_attn(x.dt, x.off, x.kv, x.n_q, x.qd, x.out, prefix=x.px, ws=scratch(n), ws_bytes=n, **kw)
    torch.cuda.synchronize()
    return x.out


def prompt_parity(x, **kw):
    x.upload()
    ref, tol = x.reference(lambda b: causal(x.n[b]), scale=kw.get("scale"))
    check(run_prompt(x, **kw), ref, tol)


def with_trees(x, ts):
    x.upload()
    x.ts = ts
    x.trees = sm.Trees(x.off, *(np.concatenate([getattr(t, f) for t in ts]) for f in ("parent", "depth", "rank")), device="cuda")
    return x


def run_tree(x, **kw):
    n = sm.kv4_tree_attn_bytes(x.dt, x.trees, x.kv, x.n_q, x.px)
    sm.kv4_tree_attn(x.dt, x.trees, x.kv, x.n_q, x.qd, x.out, prefix=x.px, ws=scratch(n), ws_bytes=n, **kw)
    torch.cuda.synchronize()
    return x.out


@pytest.mark.parametrize("name", list(PROMPTS))
def test_prompt_bf16(name):
    n_q, n_kv, n, L, P, shared = PROMPTS[name]
    prompt_parity(Batch4("bf16", n_q, n_kv, 128, n, L, P, shared, seed=len(name)))


@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_prompt_fp32_head_dims(d):
    prompt_parity(Batch4("fp32", 6, 2, d, [1, 31, 32, 33, 70, 0], [0, 40, 1, 64, 100, 3], seed=d))


@pytest.mark.parametrize("name", ["decode", "one_long", "gqa_odd", "prefix_shared", "prefix_decode", "prefix_mixed", "many",
                                  "many_prefixes", "kv_heads_12"])
def test_prompt_fp32(name):
    n_q, n_kv, n, L, P, shared = PROMPTS[name]
    prompt_parity(Batch4("fp32", n_q, n_kv, 64, n, L, P, shared, seed=len(name)))


@pytest.mark.parametrize("name", list(serving_forms.PROMPTS))
def test_prompt_splits(name):
    n_q, n_kv, n, L, P, shared = serving_forms.PROMPTS[name]
    prompt_parity(Batch4("bf16", n_q, n_kv, 128, n, L, P, shared, seed=len(name)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", list(TREES))
def test_tree(name, dtype):
    kind, n_q, n_kv, L, P, shared = TREES[name]
    ts = trees_of(kind, len(L), len(name))
    x = with_trees(Batch4(dtype, n_q, n_kv, 128 if dtype == "bf16" else 64, [t.n for t in ts], L, P, shared, seed=len(name)), ts)
    check(run_tree(x), *x.reference(lambda b: root_paths(x.ts[b].parent)))


@pytest.mark.parametrize("name", list(serving_forms.TREES))
def test_tree_splits(name):
    kind, n_q, n_kv, L, P, shared = serving_forms.TREES[name]
    ts = serving_forms.trees_of(kind, len(L), len(name))
    x = with_trees(Batch4("bf16", n_q, n_kv, 128, [t.n for t in ts], L, P, shared, seed=len(name)), ts)
    check(run_tree(x), *x.reference(lambda b: root_paths(x.ts[b].parent)))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_scale_and_peaked_scores(dtype):
    """Scores of several hundred: one key takes almost all of a row, and the running maximum moves often."""
    prompt_parity(Batch4(dtype, 4, 2, 128 if dtype == "bf16" else 32, [90, 33], [200, 0], seed=3, std=3.0), scale=1.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_equal_scores(dtype):
    """Zero queries: the mean of the visible V rows."""
    x = Batch4(dtype, 2, 2, 128, [130], [70], seed=4)
    x.q.zero_()
    prompt_parity(x)


def test_queries_of_uneven_columns():
    """Columns of a query between 2^-30 and 2^10 of the others: each 32 of them have a scale of their own."""
    x = Batch4("bf16", 4, 2, 128, [70, 3], [200, 33], seed=5)
    g = torch.Generator().manual_seed(6)
    e = torch.randint(-30, 3, (x.q.shape[0], x.q.shape[1], 4), generator=g).repeat_interleave(32, 2)
    e = e + torch.where(torch.rand(x.q.shape, generator=g) < 0.1, -torch.randint(0, 20, x.q.shape, generator=g), torch.zeros(()).long())
    x.q = (x.q.double() * 2.0 ** e.double()).to(torch.bfloat16)
    prompt_parity(x)


@pytest.mark.parametrize("dtype,lift", [("bf16", 2.0 ** -60), ("bf16", 2.0 ** 40), ("fp32", 2.0 ** -40), ("fp32", 2.0 ** 30)])
def test_far_scales(dtype, lift):
    """Keys and values far from one, the queries to match."""
    x = Batch4(dtype, 4, 2, 64 if dtype == "fp32" else 128, [40, 3], [100, 33], seed=7)
    x.q = (x.q.double() / lift).to(x.dtype)
    shift = int(np.log2(lift))
    x.bytes = [(c, np.where(s == 255, 255, s.astype(int) + shift).astype(np.uint8)) for c, s in x.bytes]
    x.k, x.v = ((t.double() * lift).to(x.dtype) for t in (x.k, x.v))
    prompt_parity(x)


def test_captured():
    """A replayed graph, with other work between its replays."""
    n_q, n_kv, n, L, P, shared = PROMPTS["prefix_decode"]
    x = Batch4("bf16", n_q, n_kv, 128, n, L, P, shared, seed=2).upload()
    ref, tol = x.reference(lambda b: causal(x.n[b]))
    nb = sm.kv4_prompt_attn_bytes(x.dt, x.off, x.kv, n_q, x.px)
    ws = scratch(nb)
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            sm.kv4_prompt_attn(x.dt, x.off, x.kv, n_q, x.qd, x.out, prefix=x.px, ws=ws, ws_bytes=nb)
        for _ in range(3):
            x.out.fill_(777.0)
            ws.fill_(255)
            g.replay()
            s.synchronize()
            check(x.out, ref, tol)


def test_two_at_once():
    """Two calls on two streams, a workspace each."""
    xs = [Batch4("bf16", 16, 2, 128, [5, 1, 30], [3000, 200, 0], seed=s).upload() for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in xs]
    nb = [sm.kv4_prompt_attn_bytes(x.dt, x.off, x.kv, 16) for x in xs]
    ws = [scratch(n) for n in nb]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, s, w, n in zip(xs, streams, ws, nb):
            sm.kv4_prompt_attn(x.dt, x.off, x.kv, 16, x.qd, x.out, ws=w, ws_bytes=n, stream=s)
    torch.cuda.synchronize()
    for x in xs:
        check(x.out, *x.reference(lambda b: causal(x.n[b])))
