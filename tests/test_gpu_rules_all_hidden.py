"""GPU: a row whose mask allows no token is all -inf, and greedy acceptance takes token 0 there."""

import numpy as np
import pytest
import torch

from paper_2506_01986_amd import specmemo as sm
from paper_2506_01986_amd import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [1, 40, 1003, 32000])
def test_greedy_takes_token_0(dtype, vocab):
    """Chains of three nodes whose rows are all hidden: node 1 is accepted where it holds token 0, node 2 where both do."""
    tdt, dt = (torch.bfloat16, sm.BF16) if dtype == "bf16" else (torch.float32, sm.FP32)
    other = min(1, vocab - 1)
    toks = [[other, 0, 0], [other, 0, other], [other, other, 0]]
    want = [2, 1 if other else 2, 0 if other else 2]
    B, stride = len(toks), 4
    t = synth.chain_tree(3)
    trees = sm.Trees(np.arange(B + 1) * 3, *(np.tile(getattr(t, f), B) for f in ("parent", "depth", "rank")), device="cuda")
    tok = torch.tensor(sum(toks, []), dtype=torch.int32).cuda()
    logits = torch.randn(3 * B, vocab, device="cuda").to(tdt)
    rules = sm.LogitRules(repetition=torch.full((B,), 1.3, device="cuda"))
    rules.set_mask(torch.zeros(1, (vocab + 31) // 32, dtype=torch.int32, device="cuda"),
                   torch.zeros(3 * B, dtype=torch.int32, device="cuda"))
    out = torch.empty_like(logits)
    sm.logit_rules(dt, trees, vocab, logits, tok, rules, out)
    assert torch.isneginf(out).all()
    acc, nxt = (torch.full((B,), 9, dtype=torch.int32, device="cuda") for _ in range(2))
    path = torch.empty(B, stride, dtype=torch.int32, device="cuda")
    n = sm.workspace_bytes(sm.WS_ACCEPT, dt, trees, None, sm.GREEDY)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    sm.accept(dt, trees, vocab, sm.GREEDY, out, tok, acc, path, stride, nxt, ws=ws, ws_bytes=n)
    assert acc.tolist() == want and nxt.tolist() == [0] * B
