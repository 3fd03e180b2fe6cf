"""Tensors that the append, 4-bit pool and 4-bit attention calls of the binding refuse: what the kernels would read or
write past their end, or as another type."""

import pytest
import torch

from paper_2506_01986_amd import specmemo as sm

bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)


@pytest.mark.parametrize("v", [bf(2, 29, 128), bf(1, 30, 128), bf(2, 31, 128), torch.zeros(2, 30, 128)])
def test_values_beside_keys(v):
    """A pool's V has K's rows and type: a shorter V would be written past its end."""
    kv = sm.KVPool(bf(2, 30, 128), v, i32(1), [0], [20], [3])
    x = sm.QKVRows(None, bf(5, 2, 128), bf(5, 2, 128))
    with pytest.raises(ValueError):
        sm.kv_append(sm.BF16, [0, 5], x, kv, None)
    kv.k = kv.v = bf(2, 29, 128)                  # cap_total says 30
    with pytest.raises(ValueError):
        sm.kv_append(sm.BF16, [0, 5], x, kv, None)


def pool4(n=1):
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    return sm.KV4Pool(u8(2, 30, 64), u8(2, 30, 64), u8(2, 30, 4), u8(2, 30, 4), i32(n), [0] * n, [20] * n, [3] * n)


FUSED = bf(5, 4 + 2 + 2, 128)
BAD = [torch.zeros(5, 4, 128), bf(4, 4, 128), FUSED[:, :4], bf(4, 5, 128).transpose(0, 1), bf(5, 128, 4).transpose(1, 2)]
TREES = sm.Trees([0, 5], [-1, 0, 0, 1, 1], [0, 1, 1, 2, 2], [0, 0, 1, 0, 1], dev_arrays=[i32(5)] * 4)
CALLS = {"prompt": lambda q, out: sm.kv4_prompt_attn(sm.BF16, [0, 5], pool4(), 4, q, out),
         "tree": lambda q, out: sm.kv4_tree_attn(sm.BF16, TREES, pool4(), 4, q, out)}


@pytest.mark.parametrize("bad", range(len(BAD)))
@pytest.mark.parametrize("call", list(CALLS))
def test_attention_tensors(call, bad):
    """Queries and outputs of another type, too few, or with gaps (queries as a slice of a fused row)."""
    with pytest.raises(ValueError):
        CALLS[call](BAD[bad], bf(5, 4, 128))
    with pytest.raises(ValueError):
        CALLS[call](bf(5, 4, 128), BAD[bad])


@pytest.mark.parametrize("name,bad", [("accept_len", i32(1)), ("accept_len", torch.zeros(2, dtype=torch.int64)), ("accept_len", i32(4)[::2]),
                                      ("path", i32(11)), ("path", torch.zeros(2, 6, dtype=torch.int64)), ("path", i32(6, 2).t()),
                                      ("path", i32(2, 8)[:, :6]), ("seq_len", i32(1))])
def test_compaction_tensors(name, bad):
    """Accepted lengths, paths and the pool's lengths: 32-bit integers, as many as the call reads or writes."""
    trees = sm.Trees([0, 2, 4], [-1, 0] * 2, [0, 1] * 2, [0, 0] * 2, dev_arrays=[i32(4)] * 4)
    kv = pool4(2)
    kv.seq_base_h[1] = 10
    kv.seq_cap_h[:] = 10
    f = dict(accept_len=i32(2), path=i32(2, 6), seq_len=i32(2))
    f[name] = bad
    kv.seq_len = f["seq_len"]
    with pytest.raises(ValueError):
        sm.kv4_compact(trees, kv, f["accept_len"], f["path"], 6)


def test_type_of_a_pool_s_lengths():
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    for bad in (torch.zeros(1), torch.zeros(1, dtype=torch.int64), i32(4)[::2]):
        with pytest.raises(ValueError):
            sm.KV4Pool(u8(2, 30, 64), u8(2, 30, 64), u8(2, 30, 4), u8(2, 30, 4), bad, [0], [20], [3])


@pytest.mark.parametrize("short", ["seq_base_h", "seq_cap_h", "seq_len_h"])
def test_more_trees_than_sequences(short):
    """The pool's host arrays have an entry for every tree."""
    trees = sm.Trees([0, 2, 4], [-1, 0] * 2, [0, 1] * 2, [0, 0] * 2, dev_arrays=[i32(4)] * 4)
    kv = pool4(2)
    setattr(kv, short, getattr(kv, short)[:1])
    with pytest.raises(ValueError):
        sm.kv4_tree_attn_bytes(sm.BF16, trees, kv, 4)
    with pytest.raises(ValueError):
        sm.kv4_tree_attn(sm.BF16, trees, kv, 4, bf(4, 4, 128), bf(4, 4, 128))
    with pytest.raises(ValueError):
        sm.kv4_compact(trees, kv, i32(2), i32(2, 6), 6)
