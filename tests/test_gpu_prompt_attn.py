"""GPU: causal attention of prompt tokens over the pool, against 64 bits."""

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import specmemo as sm
from tests.serving_ref import Batch, causal, check

pytestmark = pytest.mark.gpu


def ws_for(x):
    n = sm.prompt_attn_bytes(x.dt, x.off, x.kv, x.n_q, x.px)
    return torch.full((max(16, n),), 255, dtype=torch.uint8, device="cuda"), n     # NaN in every unwritten part


def run(x, **kw):
    ws, n = ws_for(x)
    sm.prompt_attn(x.dt, x.off, x.kv, x.n_q, x.qd, x.out, prefix=x.px, ws=ws, ws_bytes=n, **kw)
    torch.cuda.synchronize()
    return x.out


def parity(x, **kw):
    x.upload()
    ref, tol = x.reference(lambda b: causal(x.n[b]), scale=kw.get("scale"))
    check(run(x, **kw), ref, tol)


def draw(seed, hi, n):
    return [int(v) for v in np.random.default_rng(seed).integers(0, hi, n)]


# query heads, KV heads, new tokens, committed rows, prefix rows, groups of one prefix
BF16 = {
    "one_token": (1, 1, [1], [0], None, None),
    "empty_and_single": (8, 2, [0, 1, 0, 3, 0], [5, 63, 0, 64, 7], None, None),
    "all_empty": (8, 2, [0, 0], [5, 0], None, None),
    "tile_edges": (4, 4, [63, 64, 65, 127, 128, 129], [0, 0, 0, 0, 0, 0], None, None),
    "after_committed": (4, 4, [63, 64, 65, 1, 2], [1, 64, 129, 300, 63], None, None),
    "one_long": (2, 2, [1000], [0], None, None),                       # split in chunks
    "one_long_gqa": (16, 2, [700], [333], None, None),
    "gqa_odd": (15, 3, [37, 150, 5], [20, 0, 400], None, None),        # five heads a KV head: rows end inside tokens
    "gqa_7": (7, 1, [130, 41], [0, 90], None, None),
    "mqa": (32, 1, [50, 3], [100, 17], None, None),                    # one KV head over all XCDs
    "kv_heads_12": (12, 12, [40, 200], [0, 10], None, None),
    "kv_heads_40": (40, 40, [33], [100], None, None),
    "decode": (64, 8, [1] * 9, [0, 1, 63, 64, 65, 1000, 3000, 127, 128], None, None),
    "decode_mha": (8, 8, [1] * 5, [2000, 100, 5, 0, 640], None, None),
    "few_tokens": (16, 2, [1, 7, 8, 9, 2], [500, 600, 2500, 0, 1], None, None),
    "prefix_shared": (8, 2, [20, 1, 64, 3], [0, 30, 7, 100], [150] * 4, [0, 0, 0, 0]),
    "prefix_decode": (32, 4, [1] * 12, draw(1, 90, 12), [700] * 12, [0] * 12),
    "prefix_mixed": (8, 8, [5, 90, 0, 4, 4, 1], [3, 0, 9, 64, 0, 12], [64, 64, 64, 0, 129, 129], [0, 0, 0, 1, 2, 2]),
    "prefix_long_prompts": (8, 1, [300, 200], [0, 70], [513, 513], [0, 0]),
    "most_in_arguments": (4, 2, draw(2, 30, 70) + [1] * 6, draw(3, 200, 76), None, None),
    "many": (4, 2, draw(2, 30, 90), draw(3, 200, 90), None, None),     # more sets than the arguments hold
    "many_prefixes": (4, 1, draw(4, 9, 100), draw(5, 60, 100), [40] * 100, [i // 2 for i in range(100)]),
    "many_packed": (4, 8 // 4, [1] * 90, draw(6, 60, 90), [800] * 90, [i // 30 for i in range(90)]),
}


@pytest.mark.parametrize("name", list(BF16))
def test_bf16(name):
    n_q, n_kv, n, L, P, shared = BF16[name]
    parity(Batch("bf16", n_q, n_kv, 128, n, L, P, shared, seed=len(name)))


@pytest.mark.parametrize("d", [4, 20, 32, 36, 64, 96, 100, 128])
def test_fp32_head_dims(d):
    parity(Batch("fp32", 6, 2, d, [1, 31, 32, 33, 70, 0], [0, 40, 1, 64, 100, 3], seed=d))


@pytest.mark.parametrize("name", ["decode", "one_long", "gqa_odd", "prefix_shared", "prefix_decode", "prefix_mixed", "many",
                                  "many_prefixes", "kv_heads_12"])
def test_fp32(name):
    n_q, n_kv, n, L, P, shared = BF16[name]
    parity(Batch("fp32", n_q, n_kv, 64, n, L, P, shared, seed=len(name)))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_scale_and_peaked_scores(dtype):
    """Scores of several hundred: one key takes almost all of a row, and the running maximum moves often."""
    parity(Batch(dtype, 4, 2, 128 if dtype == "bf16" else 36, [90, 33], [200, 0], seed=3, std=3.0), scale=1.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_equal_scores(dtype):
    """Zero queries: the mean of the visible V rows."""
    x = Batch(dtype, 2, 2, 128, [130], [70], seed=4)
    x.q.zero_()
    parity(x)


@pytest.mark.parametrize("n_q,n_kv,L,P", [(112, 112, 0, 0), (112, 112, 40, 70), (250, 50, 3, 0)])
def test_many_row_blocks(n_q, n_kv, L, P):
    """Thousands of row blocks, several rounds of them."""
    n = [257, 400, 1, 385, 128, 300, 270, 512, 129, 640, 333, 500, 3, 301, 257, 280, 450, 390, 260, 310]
    x = Batch("bf16", n_q, n_kv, 128, n if n_q == n_kv else n[:14], [L] * (20 if n_q == n_kv else 14),
              [P] * (20 if n_q == n_kv else 14), seed=P).upload()
    assert sm.prompt_attn_bytes(x.dt, x.off, x.kv, n_q, x.px) == 0          # nothing is split
    ref, tol = x.reference(lambda b: causal(x.n[b]), device="cuda")
    check(run(x), ref, tol)


def test_same_prompt_in_chunks():
    """A prompt in one call, and token ranges of it on their committed rows, agree within two roundings."""
    x = Batch("bf16", 8, 2, 128, [333], [0], seed=9).upload()
    whole = run(x).clone()
    for i0, i1 in ((0, 1), (1, 100), (100, 300), (300, 333)):
        kv = sm.KVPool(x.kd, x.vd, x.kv.seq_len, x.base, x.cap, [i0])
        out = torch.empty_like(x.qd[i0:i1])
        n = sm.prompt_attn_bytes(x.dt, [0, i1 - i0], kv, 8)
        ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
        sm.prompt_attn(x.dt, [0, i1 - i0], kv, 8, x.qd[i0:i1].contiguous(), out, ws=ws, ws_bytes=n)
        ref, tol = x.reference(lambda b: causal(333))
        check(out, ref[i0:i1], tol[i0:i1])
        assert (out.float() - whole[i0:i1].float()).abs().max() <= 2 * tol[i0:i1].max()


def test_prefix_in_committed_rows():
    """A prefix may be another sequence's committed rows."""
    x = Batch("bf16", 4, 2, 128, [9, 4], [200, 11], seed=5).upload()
    px = sm.Prefix([0, x.base[0]], [0, 120])
    n = sm.prompt_attn_bytes(x.dt, x.off, x.kv, 4, px)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    sm.prompt_attn(x.dt, x.off, x.kv, 4, x.qd, x.out, prefix=px, ws=ws, ws_bytes=n)
    torch.cuda.synchronize()
    x.pbase, x.plen = [0, x.base[0]], [0, 120]
    check(x.out, *x.reference(lambda b: causal(x.n[b])))


def test_nested_prefixes():
    """Prefixes of one base and different lengths."""
    x = Batch("bf16", 4, 2, 128, [9, 4, 30], [20, 11, 0], [100] * 3, [0] * 3, seed=6).upload()
    x.plen = [100, 60, 64]
    x.px = sm.Prefix(x.pbase, x.plen)
    check(run(x), *x.reference(lambda b: causal(x.n[b])))


@pytest.mark.parametrize("dtype,rows", [("bf16", 9_000_000), ("fp32", 5_000_000)])
def test_far_slabs(dtype, rows):
    """Slabs and prefix more than 2^32 bytes into the pool, in every KV head."""
    x = Batch(dtype, 4, 2, 128, [70, 1], [200, 500], [90, 90], [0, 0], seed=7).upload()
    small = [x.kd, x.vd]
    for name, t in (("kd", x.kd), ("vd", x.vd)):
        big = torch.empty(2, 2 * rows, 128, dtype=t.dtype, device="cuda")
        big[:, 2 * rows - t.shape[1]:] = t
        setattr(x, name, big)
    shift = 2 * rows - small[0].shape[1]
    assert shift * 128 * x.kd.element_size() > 2 ** 32
    x.kv = sm.KVPool(x.kd, x.vd, x.kv.seq_len, [b + shift for b in x.base], x.cap, x.L)
    x.px = sm.Prefix([b + shift for b in x.pbase], x.plen)
    check(run(x), *x.reference(lambda b: causal(x.n[b])))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 4)])
def test_largest_batch(dtype, d):
    """4096 sequences of one or two tokens and four packed prefixes: three rounds of the search for a block's set."""
    n = [1 + v for v in draw(11, 2, 4096)]
    parity(Batch(dtype, 2, 1, d, n, draw(12, 20, 4096), [600] * 4096, [i // 1024 for i in range(4096)], seed=13))


@pytest.mark.parametrize("name", ["gqa_odd", "prefix_decode", "one_long_gqa"])
def test_rows_past_the_batch(name):
    """A larger output than the batch: rows after the last token keep what they held."""
    n_q, n_kv, n, L, P, shared = BF16[name]
    x = Batch("bf16", n_q, n_kv, 128, n, L, P, shared, seed=10).upload()
    x.out = torch.full((x.qd.shape[0] + 300, n_q, 128), 777.0, dtype=x.dtype, device="cuda")
    run(x)
    assert (x.out[x.qd.shape[0]:] == 777.0).all()
    check(x.out[:x.qd.shape[0]], *x.reference(lambda b: causal(x.n[b])))


def test_two_calls_at_once():
    """Calls on two streams, each with a workspace of its own, one of them with its table of sets there."""
    xs = []
    for name in ("many", "prefix_decode"):
        n_q, n_kv, n, L, P, shared = BF16[name]
        xs.append(Batch("bf16", n_q, n_kv, 128, n, L, P, shared, seed=9).upload())
    want = [run(x).clone() for x in xs]
    ws = [ws_for(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    for x in xs:
        x.out.fill_(555.0)
    torch.cuda.synchronize()
    for _ in range(10):
        for x, (w, nb), s in zip(xs, ws, streams):
            with torch.cuda.stream(s):
                sm.prompt_attn(x.dt, x.off, x.kv, x.n_q, x.qd, x.out, prefix=x.px, ws=w, ws_bytes=nb)
    torch.cuda.synchronize()
    for x, w in zip(xs, want):
        assert torch.equal(x.out.view(torch.int16), w.view(torch.int16))


@pytest.mark.parametrize("name", ["prefix_mixed", "one_long_gqa", "many"])
def test_captured_and_on_another_stream(name):
    """A captured call, replayed between eager calls on other data, gives the eager result every time."""
    n_q, n_kv, n, L, P, shared = BF16[name]
    x = Batch("bf16", n_q, n_kv, 128, n, L, P, shared, seed=7).upload()
    want = run(x).clone()
    ws, nb = ws_for(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            sm.prompt_attn(x.dt, x.off, x.kv, x.n_q, x.qd, x.out, prefix=x.px, ws=ws, ws_bytes=nb)
        q0 = x.qd.clone()
        for i in range(3):
            x.out.fill_(555.0)
            x.qd.copy_(q0)
            graph.replay()
            side.synchronize()
            assert torch.equal(x.out.view(torch.int16), want.view(torch.int16)), i
            x.qd.normal_()                                   # an eager call on other queries in between
            sm.prompt_attn(x.dt, x.off, x.kv, x.n_q, x.qd, x.out, prefix=x.px, ws=ws, ws_bytes=nb)
            side.synchronize()


def test_repeats_bit_for_bit():
    n_q, n_kv, n, L, P, shared = BF16["prefix_decode"]
    x = Batch("bf16", n_q, n_kv, 128, n, L, P, shared, seed=8).upload()
    first = run(x).clone()
    for _ in range(3):
        assert torch.equal(run(x).view(torch.int16), first.view(torch.int16))
