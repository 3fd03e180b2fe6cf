"""GPU: the calls of a 4-bit cache together, as a chat server runs them: a system prompt appended once, prompts appended
and attended, then steps of append, tree attention, acceptance and compaction.  Every stage is compared on the buffers
that the stage before left on the GPU.  And the calls at their limits: pools past 2^32 bytes, the largest batches, more
tokens than a launch takes."""

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import specmemo as sm
from paper_2506_01986_amd import synth
from tests.kv4_ref import Batch4, pack, quantise, unpack, values
from tests.serving_ref import causal, check, root_paths
from tests.test_gpu_kv_rows import EPS, Rows

pytestmark = pytest.mark.gpu


def scratch(n):
    return torch.full((max(16, n),), 255, dtype=torch.uint8, device="cuda"), n


def view_of(kv, q, off, L, px, n_q, dtype):
    """What the attention's reference needs, from the pool's bytes as they are."""
    x = object.__new__(Batch4)
    x.dtype, x.dt = dtype, sm.FP32 if dtype == torch.float32 else sm.BF16
    x.n_q, x.n_kv, x.d, x.B = n_q, kv.n_kv, kv.head_dim, len(L)
    x.off, x.n, x.L = off, [int(b - a) for a, b in zip(off[:-1], off[1:])], [int(v) for v in L]
    x.base, (x.pbase, x.plen) = [int(v) for v in kv.seq_base_h], px
    x.q = q.cpu()
    x.k, x.v = (torch.from_numpy(values(unpack(c.cpu().numpy()), s.cpu().numpy())).to(dtype)
                for c, s in ((kv.k, kv.k_scale), (kv.v, kv.v_scale)))
    return x


def new_rows(r, dtype, T, n_q, n_kv, d, pos, cos, sin, norms):
    g = lambda h: torch.from_numpy(r.standard_normal((T, h, d))).to(dtype)
    q, k, v = g(max(n_q, 1)), g(n_kv), g(n_kv)
    rows = sm.QKVRows(q.cuda() if n_q else None, k.cuda(), v.cuda(), torch.from_numpy(pos.astype(np.int32)).cuda(), cos.cuda(), sin.cuda(),
                      q_norm=norms[0].cuda(), k_norm=norms[1].cuda(), eps=EPS)
    # the reference of the same rows
    x = object.__new__(Rows)
    x.dtype, x.d, x.rot, x.style, x.cos, x.sin, x.pos = dtype, d, d, "halves", cos, sin, torch.from_numpy(pos.astype(np.int64))
    return rows, x, q, k, v


@pytest.mark.parametrize("dtype,n_q,n_kv,d", [("bf16", 8, 2, 128), ("bf16", 3, 3, 128), ("fp32", 6, 2, 64)])
def test_prompt_then_steps(dtype, n_q, n_kv, d):
    r = np.random.default_rng(d + n_q)
    tdt = torch.float32 if dtype == "fp32" else torch.bfloat16
    dt = sm.FP32 if dtype == "fp32" else sm.BF16
    B, P, prompt, room = 4, 150, [70, 1, 130, 33], 60
    cap = np.array([n + room for n in prompt], np.int32)
    base = P + 1 + np.concatenate([[0], np.cumsum(cap + 1)])[:-1].astype(np.int64)
    total_rows = int(base[-1] + cap[-1] + 2)
    mem = [torch.full((n_kv, total_rows, d // w), 255, dtype=torch.uint8, device="cuda") for w in (2, 2, 32, 32)]
    seq_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    angle = torch.arange(600).double()[:, None] * 10000.0 ** (-torch.arange(d // 2).double() * 2 / d)
    cos, sin = angle.cos().float(), angle.sin().float()
    norms = [(1 + 0.2 * torch.from_numpy(r.standard_normal(d))).to(tdt) for _ in range(2)]
    pool = lambda L: sm.KV4Pool(*mem, seq_len, base, cap, L)

    def append(kv, off, pos, nq):
        rows, x, q, k, v = new_rows(r, tdt, len(pos), nq, n_kv, d, pos, cos, sin, norms)
        q_out = torch.empty(len(pos), nq, d, dtype=tdt, device="cuda") if nq else None
        sm.kv4_append(dt, off, rows, kv, q_out)
        ko, vo = (torch.empty(len(pos), n_kv, d, dtype=tdt, device="cuda") for _ in range(2))
        sm.kv4_read(dt, off, kv, ko, vo)
        torch.cuda.synchronize()
        if nq:
            check(q_out, *x.turned(q, norms[0]))
        assert torch.equal(ko.cpu().double(), torch.from_numpy(values(*quantise(x.turned(k, norms[1])[0].numpy()))))
        assert torch.equal(vo.cpu().double(), torch.from_numpy(values(*quantise(v.double().numpy()))))
        return q_out

    # 1. the system prompt, once, in rows of its own
    append(sm.KV4Pool(*mem, seq_len[:1].clone(), [0], [P], [0]), np.array([0, P]), np.arange(P), 0)
    px, pxh = sm.Prefix([0] * B, [P] * B), ([0] * B, [P] * B)
    # 2. the prompts
    off = np.concatenate([[0], np.cumsum(prompt)]).astype(np.int32)
    L = np.zeros(B, np.int32)
    q = append(pool(L), off, P + np.concatenate([np.arange(n) for n in prompt]), n_q)
    out = torch.empty_like(q)
    ws, n = scratch(sm.kv4_prompt_attn_bytes(dt, off, pool(L), n_q, px))
    sm.kv4_prompt_attn(dt, off, pool(L), n_q, q, out, prefix=px, ws=ws, ws_bytes=n)
    torch.cuda.synchronize()
    check(out, *view_of(pool(L), q, off, L, pxh, n_q, tdt).reference(lambda b: causal(prompt[b])))
    L = np.array(prompt, np.int32)
    # 3. steps
    for step in range(3):
        ts = [synth.random_tree(r, int(m), max_depth=4) for m in r.integers(1, 14, B)]
        noff = np.concatenate([[0], np.cumsum([t.n for t in ts])]).astype(np.int32)
        par, dep, rank = (np.concatenate([getattr(t, f) for t in ts]).astype(np.int32) for f in ("parent", "depth", "rank"))
        trees = sm.Trees(noff, par, dep, rank, device="cuda")
        kv = pool(L)
        q = append(kv, noff, P + np.repeat(L, [t.n for t in ts]) + dep, n_q)
        out = torch.empty_like(q)
        ws, n = scratch(sm.kv4_tree_attn_bytes(dt, trees, kv, n_q, px))
        sm.kv4_tree_attn(dt, trees, kv, n_q, q, out, prefix=px, ws=ws, ws_bytes=n)
        torch.cuda.synchronize()
        check(out, *view_of(kv, q, noff, L, pxh, n_q, tdt).reference(lambda b: root_paths(ts[b].parent)))
        # acceptance of random logits, and the accepted rows
        V = 64
        tok = torch.from_numpy(r.integers(0, V, int(noff[-1])).astype(np.int32)).cuda()
        logits = torch.from_numpy(r.standard_normal((int(noff[-1]), V))).to(tdt).cuda()
        for i in range(int(noff[-1])):                        # most nodes have their parent's approval
            b = int(np.searchsorted(noff, i, side="right") - 1)
            if par[i] >= 0 and r.random() < 0.7:
                logits[int(noff[b]) + int(par[i]), int(tok[i])] = 9.0
        acc, nxt = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
        path = torch.zeros(B, 5, dtype=torch.int32, device="cuda")
        aws, an = scratch(sm.workspace_bytes(sm.WS_ACCEPT, dt, trees, None, sm.GREEDY, V))
        sm.accept(dt, trees, V, sm.GREEDY, logits, tok, acc, path, 5, nxt, ws=aws, ws_bytes=an)
        before = [m.cpu().clone() for m in mem]
        sm.kv4_compact(trees, kv, acc, path, 5)
        torch.cuda.synchronize()
        a, p = acc.cpu().numpy(), path.cpu().numpy()
        for m, was in zip(mem, before):
            want = was.clone()
            for b in range(B):
                for j in range(int(a[b]) + 1):
                    want[:, base[b] + L[b] + j] = was[:, base[b] + L[b] + p[b, j]]
            assert torch.equal(m.cpu(), want)
        L = L + a + 1
        assert seq_len.cpu().tolist() == L.tolist()


def far_pool(x, shift):
    """x's batch with every slab and prefix `shift` rows further into the pool (new_rows of it on the GPU alone)."""
    rows = x.k.shape[1] + shift
    out = []
    for code, scale in x.bytes:
        for small in (code, scale):
            m = torch.empty(x.n_kv, rows, small.shape[2], dtype=torch.uint8, device="cuda")
            m[:, shift:] = torch.from_numpy(small).cuda()
            out.append(m)
    x.qd = x.q.cuda()
    x.out = torch.full_like(x.qd, 777.0)
    k, ks, v, vs = out
    x.kv = sm.KV4Pool(k, v, ks, vs, torch.tensor(x.L, dtype=torch.int32).cuda(), [b + shift for b in x.base], x.cap, x.L)
    x.px = sm.Prefix([b + shift for b in x.pbase], x.plen) if any(x.plen) else None


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 32)])
def test_attention_past_4_gib(dtype, d):
    """Rows whose bytes lie past 2^32, and the second KV head's past 2^33."""
    x = Batch4(dtype, 16 if dtype == "bf16" else 4, 2, d, [1, 70, 5], [300, 100, 0], [90, 90, 0], [0, 0, 1], seed=8)
    far_pool(x, 2 ** 32 // (d // 2) + 12345)
    n = sm.kv4_prompt_attn_bytes(x.dt, x.off, x.kv, x.n_q, x.px)
    ws, n = scratch(n)
    sm.kv4_prompt_attn(x.dt, x.off, x.kv, x.n_q, x.qd, x.out, prefix=x.px, ws=ws, ws_bytes=n)
    torch.cuda.synchronize()
    check(x.out, *x.reference(lambda b: causal(x.n[b])))


def test_long_context():
    """One token over 150000 keys: hundreds of chunks and parts."""
    x = Batch4("bf16", 8, 1, 128, [1], [150000], seed=9).upload()
    ws, n = scratch(sm.kv4_prompt_attn_bytes(x.dt, x.off, x.kv, 8))
    sm.kv4_prompt_attn(x.dt, x.off, x.kv, 8, x.qd, x.out, ws=ws, ws_bytes=n)
    torch.cuda.synchronize()
    check(x.out, *x.reference(lambda b: causal(1), device="cuda"))


def test_largest_batch():
    """4096 sequences: append, attention of their single tokens, compaction of single nodes."""
    B = 4096
    r = np.random.default_rng(3)
    L = [int(v) for v in r.integers(0, 40, B)]
    x = Rows("bf16", 2, 1, 128, [1] * B, L, seed=3)
    rows, kv = x.upload(), x.pool4()
    fill = Rows("bf16", 0, 1, 128, L, [0] * B, rot=0, seed=4, slack=3)      # the committed rows, in the same slabs
    assert fill.base == x.base
    sm.kv4_append(x.dt, fill.off, fill.upload(), sm.KV4Pool(kv.k, kv.v, kv.k_scale, kv.v_scale, kv.seq_len, x.base, x.cap, [0] * B), None)
    sm.kv4_append(x.dt, x.off, rows, kv, x.q_out)
    out = torch.empty_like(x.q_out)
    ws, n = scratch(sm.kv4_prompt_attn_bytes(x.dt, x.off, kv, 2))
    sm.kv4_prompt_attn(x.dt, x.off, kv, 2, x.q_out, out, ws=ws, ws_bytes=n)
    one = synth.chain_tree(1)
    trees = sm.Trees(np.arange(B + 1), *(np.concatenate([getattr(one, f)] * B) for f in ("parent", "depth", "rank")), device="cuda")
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    sm.kv4_compact(trees, kv, zero, zero, 1)
    torch.cuda.synchronize()
    check(out, *view_of(kv, x.q_out, x.off, L, ([0] * B, [0] * B), 2, torch.bfloat16).reference(lambda b: causal(1)))
    assert kv.seq_len.cpu().tolist() == [v + 1 for v in L]


@pytest.mark.parametrize("four", [False, True])
def test_more_tokens_than_a_launch(four):
    """65000 heads a token: 516 tokens a launch, a sequence on both sides of the cut."""
    d = 32 if four else 4
    n = [500, 3, 60, 0, 37]
    x = Rows("fp32", 65000 if not four else 66000, 1, d, n, [0, 1, 2, 0, 5], seed=2, rot=0 if not four else 16)
    rows, kv = x.upload(), x.pool4() if four else x.pool()
    (sm.kv4_append if four else sm.kv_append)(x.dt, x.off, rows, kv, x.q_out)
    torch.cuda.synchronize()
    if four:
        q, tol = x.turned(x.q, None)
        check(x.q_out, q, tol)
        code, scale = quantise(x.turned(x.k, None)[0].numpy())
        x.check_pool(kv.k, torch.from_numpy(pack(code)))
        x.check_pool(kv.k_scale, torch.from_numpy(scale))
    else:
        assert torch.equal(x.q_out.cpu(), x.q)
        x.check_pool(kv.k, x.k)
        x.check_pool(kv.v, x.v)


def test_other_stream():
    """The calls on a stream of the caller's, behind a copy on it."""
    x = Rows("bf16", 4, 2, 128, [30, 2], [3, 0], norm=True, seed=7)
    rows, kv = x.upload(), x.pool4()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    new = torch.randn(rows.k.shape, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    ko, vo = (torch.empty(32, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    with torch.cuda.stream(s):
        rows.k.copy_(new.pin_memory(), non_blocking=True)
    sm.kv4_append(x.dt, x.off, rows, kv, x.q_out, stream=s)
    sm.kv4_read(x.dt, x.off, kv, ko, vo, stream=s)
    s.synchronize()
    x.k = new
    assert torch.equal(ko.cpu().double(), torch.from_numpy(values(*quantise(x.turned(x.k, x.k_norm)[0].numpy()))))


def test_repeated_calls_agree():
    """The same call twice gives the same bits: nothing depends on an order that varies."""
    x = Batch4("bf16", 16, 2, 128, [1, 9, 64, 130], [3000, 500, 0, 40], seed=6).upload()
    outs = []
    for _ in range(4):
        ws, n = scratch(sm.kv4_prompt_attn_bytes(x.dt, x.off, x.kv, 16))
        x.out.fill_(777.0)
        sm.kv4_prompt_attn(x.dt, x.off, x.kv, 16, x.qd, x.out, ws=ws, ws_bytes=n)
        outs.append(x.out.clone())
    torch.cuda.synchronize()
    assert all(torch.equal(o.view(torch.int16), outs[0].view(torch.int16)) for o in outs)
