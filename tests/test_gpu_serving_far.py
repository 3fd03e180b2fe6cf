"""GPU: queries, results and logits whose offsets pass 32 bits (attention over far slabs:
test_gpu_prompt_attn.py)."""

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import specmemo as sm
from paper_2506_01986_amd import synth

pytestmark = pytest.mark.gpu


def test_queries_past_4_gib():
    """4096 prompts of 66 tokens, 64 heads: zero queries and values of 1 and -1, so that sums and counts are exact."""
    B, T, n_q, n_kv, d = 4096, 66, 64, 8, 128
    q = torch.zeros(B * T, n_q, d, dtype=torch.bfloat16, device="cuda")
    assert q.numel() * 2 > 2 ** 32
    out = torch.full_like(q, 777.0)
    k = torch.randn(n_kv, B * T, d, device="cuda").bfloat16()
    v = torch.where(torch.rand(n_kv, B * T, d, device="cuda") < 0.5, 1.0, -1.0).bfloat16()
    lens = np.zeros(B, np.int32)
    kv = sm.KVPool(k, v, torch.from_numpy(lens).cuda(), np.arange(B) * T, np.full(B, T), lens)
    off = np.arange(B + 1, dtype=np.int32) * T
    n = sm.prompt_attn_bytes(sm.BF16, off, kv, n_q)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    sm.prompt_attn(sm.BF16, off, kv, n_q, q, out, ws=ws, ws_bytes=n)
    for h in range(n_q):
        ref = v[h * n_kv // n_q].float().view(B, T, d).cumsum(1) / torch.arange(1, T + 1, device="cuda")[None, :, None]
        err = (out[:, h].float().view(B, T, d) - ref).abs()
        assert (err <= (2.0 ** -8 + 2.0 ** -22) * ref.abs()).all(), h


def test_logits_past_2_31_values():
    """1060 trees of 64 nodes, in place: a bias and a mask of every sequence, and its token counts."""
    B, vocab, N = 1060, 32000, 64
    t = synth.t64()
    assert t.n == N and B * N * vocab > 2 ** 31
    trees = sm.Trees(np.arange(B + 1) * N, *(np.tile(getattr(t, f), B) for f in ("parent", "depth", "rank")), device="cuda")
    z = torch.empty(B, N, vocab, dtype=torch.bfloat16, device="cuda").normal_()
    b = torch.arange(B, device="cuda")
    seen, biased, hidden = 7 * b % vocab, (7 * b + 3) % vocab, (7 * b + 31000) % vocab     # three tokens of each sequence
    first, last = z[:2].clone(), z[-2:].clone()
    counts = torch.zeros(B, vocab, dtype=torch.int32, device="cuda")
    counts[b, seen] = 2
    rules = sm.LogitRules(counts=counts, frequency=torch.full((B,), 0.5, device="cuda"))
    i32 = torch.int32
    rules.set_bias(torch.arange(B + 1, dtype=i32, device="cuda"), biased.to(i32), torch.full((B,), 3.0, device="cuda"))
    words = np.full((B, vocab // 32), 0xFFFFFFFF, np.uint32)
    at = hidden.cpu().numpy()
    words[np.arange(B), at // 32] &= ~(np.uint32(1) << (at % 32).astype(np.uint32))
    rules.set_mask(torch.from_numpy(words.view(np.int32)).cuda(), b.repeat_interleave(N).to(i32))
    tok = torch.full((B * N,), -1, dtype=i32, device="cuda")                  # no path adds a count
    sm.logit_rules(sm.BF16, trees, vocab, z, tok, rules, z)
    for old, s in ((first, slice(0, 2)), (last, slice(B - 2, B))):
        want = old.clone()
        for j, i in enumerate(range(B)[s]):
            want[j, :, int(seen[i])] = (old[j, :, int(seen[i])].float() - 1.0).bfloat16()
            want[j, :, int(biased[i])] = (old[j, :, int(biased[i])].float() + 3.0).bfloat16()
            want[j, :, int(hidden[i])] = float("-inf")
        assert torch.equal(z[s], want)
    # every row of every sequence in between: its hidden token alone is -inf
    assert torch.isneginf(z.gather(2, hidden[:, None, None].expand(B, N, 1))).all()
    total = sum(int(torch.isneginf(z[i:i + 100]).sum()) for i in range(0, B, 100))
    assert total == B * N
