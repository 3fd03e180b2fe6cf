"""GPU: the serving operators together, as a chat server runs them: prompts after a shared
system prompt, then steps of tree attention over the prefix, logit rules, acceptance with
compaction, counts of the accepted tokens and a sampled next token.  Every stage is compared
on the buffers that the stage before left on the GPU."""

import numpy as np
import pytest
import torch

import oracle
from paper_2506_01986_amd import runner, synth
from paper_2506_01986_amd import specmemo as sm
from tests.serving_ref import Batch, causal, check, root_paths

pytestmark = pytest.mark.gpu

VOCAB, STEPS, T_SAMPLE = 1003, 3, 0.8


def ws_of(n):
    return torch.empty(max(16, n), dtype=torch.uint8, device="cuda"), n


@pytest.mark.parametrize("mode", [sm.GREEDY, sm.TYPICAL])
@pytest.mark.parametrize("dtype,n_q,n_kv,d", [("bf16", 8, 2, 128), ("fp32", 4, 2, 48)])
def test_prompt_then_steps(dtype, n_q, n_kv, d, mode):
    r = np.random.default_rng(d)
    prompt, room, P = [70, 1, 130, 33], 60, 200
    x = Batch(dtype, n_q, n_kv, d, prompt, [0] * 4, [P] * 4, [0] * 4, seed=d, slack=room).upload()
    B = x.B
    # 1. the prompts, after the system prompt
    ws, n = ws_of(sm.prompt_attn_bytes(x.dt, x.off, x.kv, n_q, x.px))
    sm.prompt_attn(x.dt, x.off, x.kv, n_q, x.qd, x.out, prefix=x.px, ws=ws, ws_bytes=n)
    torch.cuda.synchronize()
    check(x.out, *x.reference(lambda b: causal(prompt[b])))
    # 2. their tokens, the system prompt's among them
    hist = [r.integers(0, VOCAB, P + t) for t in prompt]
    off = np.concatenate([[0], np.cumsum([len(h) for h in hist])]).astype(np.int32)
    counts = torch.empty(B, VOCAB, dtype=torch.int32, device="cuda")
    sm.token_counts(VOCAB, off, torch.from_numpy(off).cuda(), torch.from_numpy(np.concatenate(hist).astype(np.int32)).cuda(), counts)
    want_counts = np.stack([np.bincount(h, minlength=VOCAB) for h in hist])
    assert np.array_equal(counts.cpu().numpy(), want_counts)

    lens = np.array(prompt, np.int32)
    rep, freq = r.uniform(1, 1.5, B).astype(np.float32), r.uniform(0, 0.5, B).astype(np.float32)
    words = (VOCAB + 31) // 32
    allowed = r.random((3, words * 32)) < np.array([[0.9], [0.4], [0.02]])
    allowed[:, :5] = True                                     # no state without a token
    mask = torch.from_numpy(np.packbits(allowed, axis=1, bitorder="little").view("<i4").reshape(3, words)).cuda()
    rules = sm.LogitRules(counts=counts, repetition=torch.from_numpy(rep).cuda(), frequency=torch.from_numpy(freq).cuda())
    tdt = torch.float32 if dtype == "fp32" else torch.bfloat16
    stride, moved = 5, 0
    for step in range(STEPS):
        ts = [synth.random_tree(r, int(m), max_depth=4) for m in r.integers(1, 12, B)]
        noff = np.concatenate([[0], np.cumsum([t.n for t in ts])]).astype(np.int32)
        par, dep, rank = (np.concatenate([getattr(t, f) for t in ts]).astype(np.int32) for f in ("parent", "depth", "rank"))
        trees = sm.Trees(noff, par, dep, rank, device="cuda")
        total = int(noff[-1])
        tok = np.zeros(total, np.int32)
        for b, t in enumerate(ts):                            # distinct tokens among siblings
            tok[noff[b]:noff[b + 1]] = r.choice(VOCAB, t.n, replace=False)
        # the base model's part: K/V rows and queries of the trees, logits
        for b, t in enumerate(ts):
            at = x.base[b] + int(lens[b])
            for pool in (x.kd, x.vd):
                pool[:, at:at + t.n] = torch.randn(n_kv, t.n, d, device="cuda").to(tdt)
        q = torch.randn(total, n_q, d, device="cuda").to(tdt)
        logits = torch.randn(total, VOCAB, device="cuda").to(tdt)
        for b, t in enumerate(ts):                            # some children follow
            for u in range(t.n):
                kids = synth.children(t, u)
                if kids and r.random() < 0.8:
                    logits[noff[b] + u, tok[noff[b] + int(r.choice(kids))]] = 16.0
        # 3. tree attention over the prefix
        dev_len = torch.from_numpy(lens.copy()).cuda()
        kv = sm.KVPool(x.kd, x.vd, dev_len, x.base, x.cap, lens)
        ws, n = ws_of(sm.tree_attn_prefix_bytes(x.dt, trees, kv, x.px, n_q))
        out = torch.empty_like(q)
        sm.tree_attn_prefix(x.dt, trees, kv, x.px, n_q, q, out, ws=ws, ws_bytes=n)
        torch.cuda.synchronize()
        y = Batch.__new__(Batch)
        y.__dict__.update(x.__dict__, n=[t.n for t in ts], L=[int(v) for v in lens], off=noff, q=q.cpu(), k=x.kd.cpu(), v=x.vd.cpu())
        check(out, *y.reference(lambda b: root_paths(ts[b].parent)))
        # 4. the rules
        idx = r.integers(-1, 3, total).astype(np.int32)
        rules.set_mask(mask, torch.from_numpy(idx).cuda())
        tok_d, ruled = torch.from_numpy(tok).cuda(), torch.empty_like(logits)
        sm.logit_rules(x.dt, trees, VOCAB, logits, tok_d, rules, ruled)
        hidden = (idx[:, None] >= 0) & ~allowed[idx][:, :VOCAB]
        got = ruled.double().cpu().numpy()
        assert np.array_equal(np.isneginf(got), hidden)
        z = logits.double().cpu().numpy()
        for b, t in enumerate(ts):
            for u in range(t.n):
                row, c = int(noff[b]) + u, want_counts[b].astype(np.float64).copy()
                a = u
                while a >= 0:
                    c[tok[noff[b] + a]] += 1
                    a = int(t.parent[a])
                ref = np.where(c > 0, np.where(z[row] > 0, z[row] / rep[b], z[row] * rep[b]) - freq[b] * c, z[row])
                size = np.abs(z[row]) * 1.5 + freq[b] * c
                tol = 5 * 2.0 ** -24 * size + (2.0 ** -24 if dtype == "fp32" else 2.0 ** -8) * np.abs(ref)
                assert (np.abs(got[row] - ref) <= tol)[~hidden[row]].all()
        # 5. acceptance and compaction on the ruled logits
        acc, nxt = (torch.empty(B, dtype=torch.int32, device="cuda") for _ in range(2))
        path = torch.empty(B, stride, dtype=torch.int32, device="cuda")
        ws, n = ws_of(sm.workspace_bytes(sm.WS_ACCEPT, x.dt, trees, None, mode))
        K, V = (runner.to_host_storage(t, dtype).copy() for t in (x.kd, x.vd))
        sm.accept_compact(x.dt, trees, kv, VOCAB, mode, ruled, tok_d, acc, path, stride, nxt, temperature=0.7, ws=ws, ws_bytes=n)
        torch.cuda.synchronize()
        # (the oracle sums p log p: hidden tokens as the lowest finite value instead of -inf)
        stored = runner.to_host_storage(torch.where(torch.isneginf(ruled), torch.finfo(tdt).min, ruled), dtype)
        if mode == sm.GREEDY:
            ra, rp, rn = oracle.accept_greedy(stored, tok, noff, par, dep, stride)
        else:
            ra, rp, rn = oracle.accept_typical(stored, tok, noff, par, dep, stride, 0.7, 0.09, 0.3)
        assert np.array_equal(acc.cpu().numpy(), ra) and np.array_equal(path.cpu().numpy(), rp)
        assert np.array_equal(nxt.cpu().numpy(), rn)
        new = oracle.kv_compact(K, V, np.array(x.base, np.int64), lens, ra, rp)
        assert np.array_equal(dev_len.cpu().numpy(), new)
        assert np.array_equal(runner.to_host_storage(x.kd, dtype).view(np.uint8), K.view(np.uint8))
        assert np.array_equal(runner.to_host_storage(x.vd, dtype).view(np.uint8), V.view(np.uint8))
        # 6. the committed tokens join the counts
        sm.count_accepted(trees, VOCAB, tok_d, acc, path, stride, counts)
        for b in range(B):
            for u in rp[b, :ra[b] + 1]:
                want_counts[b, tok[noff[b] + u]] += 1
        assert np.array_equal(counts.cpu().numpy(), want_counts)
        # 7. a sampled next token is one that the node's mask allows
        sm.sample_next(x.dt, trees, VOCAB, T_SAMPLE, 5, step, ruled, acc, path, stride, nxt)
        for b, t in enumerate(nxt.cpu().numpy()):
            assert not hidden[noff[b] + rp[b, ra[b]], t]
        moved += int(ra.sum())
        lens = new
    assert moved > 0
