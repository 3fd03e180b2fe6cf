"""GPU: prompt and shared-prefix attention in each of the work splits that the timed batches take
(row blocks of 128 cut into chunks, packed prefixes of 128-row blocks, the table of sets in the
workspace): random batches against 64 bits, and batches in which every key weighs the same and
every value is 1 or -1, so that one key lost, doubled or given to another row shows in a row of
any length."""

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import specmemo as sm
from tests import serving_forms, test_gpu_prompt_attn, test_gpu_tree_prefix
from tests.serving_ref import Batch, causal, check, root_paths

pytestmark = pytest.mark.gpu

PROMPTS = {**test_gpu_prompt_attn.BF16, **serving_forms.PROMPTS}
TREES = {**test_gpu_tree_prefix.CASES, **serving_forms.TREES}


def prompt_batch(name, dtype, d):
    n_q, n_kv, n, L, P, shared = PROMPTS[name]
    x = Batch(dtype, n_q, n_kv, d, n, L, P, shared, seed=len(name))
    x.sees = lambda b: causal(x.n[b])
    return x, lambda: test_gpu_prompt_attn.run(x)


def tree_batch(name, dtype, d):
    kind, n_q, n_kv, L, P, shared = TREES[name]
    of = serving_forms.trees_of if name in serving_forms.TREES else test_gpu_tree_prefix.trees_of
    ts = of(kind, len(L), len(name))
    x = Batch(dtype, n_q, n_kv, d, [t.n for t in ts], L, P, shared, seed=len(name))
    x.sees = lambda b: root_paths(ts[b].parent)

    def run():
        x.trees = sm.Trees(x.off, *(np.concatenate([getattr(t, f) for t in ts]) for f in ("parent", "depth", "rank")), device="cuda")
        if x.px is None:
            x.px = sm.Prefix(x.pbase, x.plen)
        return test_gpu_tree_prefix.run(x)

    return x, run


def batch(name, dtype, d=None):
    return (prompt_batch if name in PROMPTS else tree_batch)(name, dtype, d or (128 if dtype == "bf16" else 48))


@pytest.mark.parametrize("name", list(serving_forms.WANT))
def test_bf16(name):
    x, run = batch(name, "bf16")
    x.upload()
    ref, tol = x.reference(x.sees, device="cuda")
    check(run(), ref, tol)


@pytest.mark.parametrize("name", ["split128_g5", "packed128", "packed128_table", "t16_packed128", "single_two_prefixes"])
def test_fp32(name):
    x, run = batch(name, "fp32", 20)
    x.upload()
    ref, tol = x.reference(x.sees, device="cuda")
    check(run(), ref, tol)


NAMES = list(PROMPTS) + [f"tree_{n}" if n in PROMPTS else n for n in TREES]
FP32 = [*serving_forms.WANT, "decode", "one_long", "gqa_odd", "many_packed", "tree_many", "single_gqa", "t64_gqa"]


@pytest.mark.parametrize("name,dtype", [(n, "bf16") for n in NAMES] + [(n, "fp32") for n in FP32])
def test_every_key_counts_once(name, dtype):
    """Queries of zero: every weight is exactly 1, sums of values 1 and -1 and the number of keys are exact in fp32, in
    any order and split.  What is left is 1 / l, the product with it (2^-24 each) and the result's rounding."""
    if name.startswith("tree_"):
        x, run = tree_batch(name[5:], dtype, 128 if dtype == "bf16" else 48)
    else:
        x, run = batch(name, dtype)
    x.q.zero_()
    x.v = torch.where(torch.isnan(x.v), x.v, torch.where(x.v > 0, 1.0, -1.0).to(x.dtype))
    x.upload()
    got = run().double().cpu()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    g = x.n_q // x.n_kv
    for b in range(x.B):
        if x.n[b] == 0:
            continue
        vis = torch.ones(x.n[b], x.plen[b] + x.L[b] + x.n[b], dtype=torch.float64)
        vis[:, x.plen[b] + x.L[b]:] = x.sees(b).double()
        v = x.v[:, torch.from_numpy(x.rows(b))].double()
        ref = torch.matmul(vis, v) / vis.sum(1)[None, :, None]                 # [n_kv][n][d]
        ref = ref.repeat_interleave(g, 0).transpose(0, 1)
        check(got[int(x.off[b]):int(x.off[b + 1])], ref, (half + 2.0 ** -22) * ref.abs())


@pytest.mark.parametrize("name", ["packed128_table", "split128_prefix", "t16_packed128", "single_table"])
def test_captured(name):
    """Replays between eager calls on other queries give the eager result, bit for bit."""
    x, run = batch(name, "bf16")
    x.upload()
    want = run().clone()
    if name in PROMPTS:
        n = sm.prompt_attn_bytes(x.dt, x.off, x.kv, x.n_q, x.px)
        call = lambda: sm.prompt_attn(x.dt, x.off, x.kv, x.n_q, x.qd, x.out, prefix=x.px, ws=ws, ws_bytes=n)
    else:
        n = sm.tree_attn_prefix_bytes(x.dt, x.trees, x.kv, x.px, x.n_q)
        call = lambda: sm.tree_attn_prefix(x.dt, x.trees, x.kv, x.px, x.n_q, x.qd, x.out, ws=ws, ws_bytes=n)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    side, graph, q0 = torch.cuda.Stream(), torch.cuda.CUDAGraph(), x.qd.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call()
        for i in range(3):
            x.out.fill_(555.0)
            ws.fill_(255)
            x.qd.copy_(q0)
            graph.replay()
            side.synchronize()
            assert torch.equal(x.out.view(torch.int16), want.view(torch.int16)), i
            x.qd.normal_()
            call()
            side.synchronize()
