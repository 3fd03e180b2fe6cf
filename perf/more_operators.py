"""Timed cases of the cache's write and of the cache in 4 bits.

Operators: norm, position rotation and append of new rows to the KV pool
(``append``, in the pool's own type or in 4 bits), the rows that a verify step
commits to a 4-bit pool (``commit``: append, compaction, reading back), and
attention over a 4-bit pool, of candidate trees (``tree4``) and of prompts, chunks
and single tokens (``prompt4``).  ``run`` computes them with elementary torch
operations, or, where ``own`` is true, through the library's binding.  Lengths,
trees and accepted paths follow from a case's ``shape`` number alone; all values
follow from the seed.

4 bits: groups of 32 columns of a row, each value a sign and one of 0, 1/2, 1, 3/2,
2, 3, 4, 6, times the group's 2^E with E the least in [-125, 125] for which no
magnitude passes 7 x 2^E (the nearest value, ties to the even code).  Values are
compared with the borders between codes in 64 bits.
"""

import math

import numpy as np
import torch

own = False

NEG_INF = float("-inf")
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-5

# query heads, KV heads, head dim (the shapes of the repository's workloads)
TINY = dict(dtype="fp32", n_q=4, n_kv=4, head_dim=64)
M7B = dict(dtype="bf16", n_q=32, n_kv=32, head_dim=128)
M13B = dict(M7B, n_q=40, n_kv=40)
M70B = dict(M7B, n_q=64, n_kv=8)


def _case(kind, m, B, tree, dist, lo, hi, past_lo=0, past_hi=0, prefix=0, groups=1, shape=1, bits=4, norm=False,
          style="halves", rot=0, fused=False, far=0):
    """tree: "" (lo .. hi new tokens a sequence) or the trees' kind; past: committed rows of the slabs; rot: rotated
    columns (0: all); fused: q, k and v of a token in one row; far: position of the first row."""
    return dict(kind=kind, dtype=m["dtype"], n_q=m["n_q"], n_kv=m["n_kv"], head_dim=m["head_dim"], B=B, tree=tree, dist=dist,
                lo=lo, hi=hi, past_lo=past_lo, past_hi=past_hi, prefix=prefix, groups=groups, shape=shape, bits=bits,
                norm=norm, style=style, rot=rot or m["head_dim"], fused=fused, far=far)


def listed():
    return [
        # one tree's rows into an fp32 pool: latency of one call
        dict(_case("append", TINY, 1, "T16", "", 0, 0, 128, 128, bits=32), name="append_tiny_fp32"),
        # one user's prompt on a 7B-shaped model into a bf16 pool, queries and keys normed
        dict(_case("append", M7B, 1, "", "fixed", 1024, 1024, bits=16, norm=True), name="append_7b_prompt"),
        # one new token of each of 32 users into a 4-bit pool, far along their texts
        dict(_case("append", M70B, 32, "", "fixed", 1, 1, 256, 16384, shape=4, fused=True, far=60000), name="append4_single_70b_b32"),
        # the prompts of the 70B-shaped serving batch into a 4-bit pool, q, k and v of a token in one row
        dict(_case("append", M70B, 10, "", "uniform", 512, 4096, shape=3, norm=True, fused=True), name="append4_70b_b10"),
        # the rows of a 7B-shaped step: tree rows in, the accepted path kept and read back
        dict(_case("commit", M7B, 1, "T64", "", 0, 0, 1024, 1024), name="commit_7b_b1"),
        # the same of 32 uneven trees on a 70B-shaped model, adjacent pairs rotated
        dict(_case("commit", M70B, 32, "random", "", 0, 0, 256, 4096, shape=4, norm=True, style="pairs"), name="commit_70b_b32"),
        # the smallest tree step over a 4-bit cache: latency
        dict(_case("tree4", TINY, 1, "T16", "", 0, 0, 128, 128), name="tree4_tiny_fp32"),
        # the 70B-shaped tree step
        dict(_case("tree4", M70B, 10, "T64", "", 0, 0, 512, 4096, shape=3), name="tree4_70b_b10"),
        # uneven trees over uneven long contexts
        dict(_case("tree4", M70B, 32, "random", "", 0, 0, 256, 16384, shape=4), name="tree4_stress_b32"),
        # prompts on a 7B-shaped model, a KV head for each query head, behind a shared instruction
        dict(_case("prompt4", M7B, 4, "", "uniform", 200, 1000, prefix=700, shape=2), name="prompt4_7b_b4"),
        # a batch without drafts: one token a sequence over uneven long contexts
        dict(_case("prompt4", M70B, 32, "", "fixed", 1, 1, 256, 16384, shape=4), name="prompt4_single_70b_b32"),
        # the second half of a long document's prompt over the first
        dict(_case("prompt4", M70B, 1, "", "fixed", 8192, 8192, 8192, 8192), name="prompt4_chunk_70b"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """A case of the ranges above that costs no more than the largest listed one."""
    while True:
        case = _draw(rng)
        w = work(case)
        if w["bytes"] <= 8e8 and w["flops"] <= 3e12 and _plain_scores(case) <= 5e9:
            return case


def _draw(rng):
    kind = rng.choice(["append", "append", "commit", "tree4", "tree4", "prompt4", "prompt4"])
    shape = rng.randrange(1 << 20)
    if rng.random() < 0.3:
        n_kv = rng.choice([1, 2, 4])
        bits = 32 if kind == "append" and rng.random() < 0.5 else 4
        d = 32 * rng.randint(1, 4) if bits == 4 else 8 * rng.randint(2, 16)
        m = dict(dtype="fp32", n_kv=n_kv, n_q=n_kv * rng.choice([1, 2, 3, 4]), head_dim=d)
    else:
        m = rng.choice([M7B, M13B, M70B, dict(M70B, n_q=32), dict(M70B, n_q=16, n_kv=2), dict(M70B, n_q=5, n_kv=1)])
        bits = 16 if kind == "append" and rng.random() < 0.4 else 4
    fp32 = m["dtype"] == "fp32"
    more = dict(shape=shape, bits=bits)
    if kind in ("append", "commit"):
        rot = m["head_dim"] if rng.random() < 0.7 else rng.choice([r for r in range(16, m["head_dim"] + 1, 16)])
        more.update(norm=rng.random() < 0.5, style=rng.choice(["halves", "pairs"]), rot=rot, fused=rng.random() < 0.5,
                    far=rng.choice([0, 0, _log_int(rng, 1, 100000)]))
    B = _log_int(rng, 1, 8 if fp32 else 48)
    trees = ["T64", "T16", "random", "single"]
    if kind == "append" and rng.random() < 0.7 or kind == "prompt4":
        if rng.random() < 0.3:          # single tokens, or a few, over the cache
            t = _log_int(rng, 1, 8)
            past = _log_int(rng, 8, 2048 if fp32 else 16384)
            return _case(kind, m, B, "", "uniform", 1, t, past // rng.choice([1, 2, 8]), past, **more)
        hi = _log_int(rng, 8, 1024 if fp32 else 8192)
        past = rng.choice([0, 0, rng.randint(1, hi)])
        prefix = rng.choice([0, 0, rng.randint(1, 1500)]) if kind == "prompt4" else 0
        return _case(kind, m, B, "", rng.choice(["uniform", "loguniform"]), max(1, hi // rng.choice([1, 3, 16])), hi, past // 3,
                     past, prefix=prefix, groups=min(B, rng.choice([1, 1, 2])), **more)
    past = _log_int(rng, 8, 1024 if fp32 else 16384)
    prefix = rng.choice([0, 0, rng.randint(1, 4096)]) if kind == "tree4" and not fp32 else 0
    return _case(kind, m, B, rng.choice(trees[1:2] if fp32 else trees), "", 0, 0, past // rng.choice([1, 4, 16]), past,
                 prefix=prefix, groups=min(B, rng.choice([1, 1, 2, 3])), **more)


# ---- what follows from the case alone --------------------------------------------

def _lens(r, dist, lo, hi, n):
    if dist == "loguniform":
        return np.clip(np.rint(np.exp(r.uniform(math.log(lo), math.log(hi), n))), lo, hi).astype(np.int32)
    return r.integers(lo, hi + 1, n).astype(np.int32)


def _random_tree(r, n):
    """Parents of a tree of n nodes in breadth-first order, depth <= 4, at most ten children a node."""
    while True:
        parent, depth, u = [-1], [0], 0
        while u < len(parent) < n:
            if depth[u] < 4:
                kids = min(int(r.integers(0, 11)), n - len(parent))
                parent += [u] * kids
                depth += [depth[u] + 1] * kids
            u += 1
        if len(parent) == n:
            return parent


def _parents(case, r):
    T16 = [-1, 0, 0, 0, 0, 1, 1, 2, 2, 3, 3, 5, 5, 6, 7, 8]
    T64 = [-1] + [0] * 10 + [1 + i // 3 for i in range(23)] + [11 + i // 2 for i in range(23)] + [34 + 2 * i for i in range(7)]
    kinds = {"T16": T16, "T64": T64, "single": [-1]}
    if case["tree"] in kinds:
        return [kinds[case["tree"]]] * case["B"]
    return [_random_tree(r, int(r.choice([8, 16, 32, 64, 128]))) for _ in range(case["B"])]


class _Shape:
    """Lengths, trees, prefixes, slabs, positions and accepted paths of a case."""

    def __init__(self, case):
        r = np.random.default_rng(case["shape"])
        B = case["B"]
        if case["tree"]:
            self.parents = _parents(case, r)
            self.n = np.array([len(p) for p in self.parents], np.int32)
            self._trees()
        else:
            self.n = _lens(r, case["dist"], case["lo"], case["hi"], B)
            self.depth = np.concatenate([np.arange(n) for n in self.n]).astype(np.int32)
        lo, hi = case["past_lo"], case["past_hi"]
        self.L = _lens(r, "loguniform" if lo > 0 and hi > 4 * lo else "uniform", lo, hi, B)
        self.off = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32)
        self.total = int(self.off[-1])
        self.seq = np.repeat(np.arange(B), self.n)
        # one prefix a group, first in the pool; a group's sequences are neighbours
        G = case["groups"]
        group = np.arange(B) * G // B
        plen = [max(0, case["prefix"] - 37 * i) for i in range(G)]
        pbase = np.concatenate([[0], np.cumsum(plen)]).astype(np.int64)
        self.plen = np.array([plen[g] for g in group], np.int32)
        self.pbase = np.array([pbase[g] for g in group], np.int64)
        live = self.L.astype(np.int64) + self.n
        self.cap = (live + live // 10 + 1).astype(np.int32)
        self.base = pbase[-1] + np.concatenate([[0], np.cumsum(self.cap.astype(np.int64))])[:-1]
        self.cap_total = int(pbase[-1] + self.cap.astype(np.int64).sum())
        self.group_rows = int(sum(plen))
        # position in the text and pool row of every new row
        self.pos = (case["far"] + (self.plen + self.L)[self.seq] + self.depth).astype(np.int32)
        self.n_pos = int(self.pos.max()) + 1
        self.dest = (self.base + self.L - self.off[:-1])[self.seq] + np.arange(self.total)
        if case["kind"] == "commit":
            paths = [t[int(r.integers(0, len(t)))] for t in self.paths]
            self.acc = np.array([len(p) - 1 for p in paths], np.int32)
            self.path = np.full((B, int(self.depth.max()) + 1), -1, np.int32)
            for b, p in enumerate(paths):
                self.path[b, :len(p)] = p
            self.acc_off = np.concatenate([[0], np.cumsum(self.acc + 1)]).astype(np.int32)
            self.kept = np.concatenate([int(o) + np.array(p) for o, p in zip(self.off, paths)])

    def _trees(self):
        par, dep, rank = [], [], []
        for p in self.parents:
            d, k, seen = [0], [0], {}
            for u in p[1:]:
                d.append(d[u] + 1)
                k.append(seen.get(u, 0))
                seen[u] = seen.get(u, 0) + 1
            par.append(p), dep.append(d), rank.append(k)
        self.parent, self.depth, self.rank = (np.concatenate([np.asarray(a) for a in x]).astype(np.int32) for x in (par, dep, rank))
        self.paths = [[self._path(p, u) for u in range(len(p))] for p in self.parents]

    @staticmethod
    def _path(p, u):
        out = []
        while u >= 0:
            out.append(u)
            u = p[u]
        return out[::-1]


def _plain_scores(case):
    """Scores of a KV head in the padded plain form."""
    if case["kind"] not in ("tree4", "prompt4"):
        return 0
    sh = _Shape(case)
    return case["B"] * int(sh.n.max()) * (case["n_q"] // case["n_kv"]) * int((sh.plen + sh.L + sh.n).max())


def work(case):
    sh = _Shape(case)
    e = 4 if case["dtype"] == "fp32" else 2
    d, n_q, n_kv = case["head_dim"], case["n_q"], case["n_kv"]
    row4 = d / 2 + d / 32                     # a row of a head in 4 bits
    if case["kind"] in ("append", "commit"):
        by = sh.total * (2 * n_q + 2 * n_kv) * d * e + len(np.unique(sh.pos)) * case["rot"] * 4 + 4 * sh.total
        by += 2 * sh.total * n_kv * (row4 if case["bits"] == 4 else d * e)
        fl = sh.total * (n_q + n_kv) * (3 * case["rot"] + (4 * d if case["norm"] else 0))
        if case["bits"] == 4:
            rows = sh.total if case["kind"] == "append" else int(sh.acc_off[-1])
            by += 2 * rows * n_kv * (row4 + d * e)                      # read back
            by += 4 * rows * n_kv * row4 if case["kind"] == "commit" else 0
            fl += 4 * sh.total * n_kv * d
        return {"bytes": int(by), "flops": int(fl)}
    n, L, P = (x.astype(np.int64) for x in (sh.n, sh.L, sh.plen))
    if case["kind"] == "prompt4":
        pairs = int((n * (P + L) + n * (n + 1) // 2).sum())
    else:
        pairs = int((n * (P + L)).sum()) + sum(len(p) for t in sh.paths for p in t)
    rows = int((L + n).sum()) + sh.group_rows
    return {"bytes": int(2 * rows * n_kv * row4 + 2 * sh.total * n_q * d * e), "flops": int(4 * d * n_q * pairs)}


# ---- prepare ----------------------------------------------------------------------

class _State:
    pass


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _normal(case, seed, salt):
    dtype = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + salt)
    return dtype, g, lambda *shape: torch.empty(*shape, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g)


def _rows_inputs(case, seed):
    """New rows of q, k and v, norm weights, the rotation's table, and for pools in the inputs' type what they hold."""
    sh = _Shape(case)
    dtype, _, normal = _normal(case, seed, 37)
    d, n_q, n_kv = case["head_dim"], case["n_q"], case["n_kv"]
    # some columns are larger than others, in keys the most
    x = dict(sh=sh)
    q = normal(sh.total, n_q, d) * torch.exp(0.3 * normal(d))
    k = normal(sh.total, n_kv, d) * torch.exp(0.7 * normal(d))
    v = normal(sh.total, n_kv, d) * torch.exp(0.3 * normal(d))
    x["q_norm"], x["k_norm"] = ((1 + 0.2 * normal(d)).to(dtype) if case["norm"] else None for _ in range(2))
    if case["fused"]:
        row = torch.cat([q, k, v], 1).to(dtype)
        x["q"], x["k"], x["v"] = row[:, :n_q], row[:, n_q:n_q + n_kv], row[:, n_q + n_kv:]
    else:
        x["q"], x["k"], x["v"] = q.to(dtype), k.to(dtype), v.to(dtype)
    freq = 10000.0 ** (-torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda") * 2 / case["rot"])
    angle = torch.arange(sh.n_pos, dtype=torch.float64, device="cuda")[:, None] * freq
    x["cos"], x["sin"] = angle.cos().float(), angle.sin().float()
    if case["bits"] != 4:
        x["pool_k"], x["pool_v"] = (normal(n_kv, sh.cap_total, d).to(dtype) for _ in range(2))
    return x


def _cache_inputs(case, seed):
    """Queries, and codes and scales of the pool's rows: values of either sign whose magnitudes spread as a normal's do."""
    sh = _Shape(case)
    dtype, g, normal = _normal(case, seed, 41)
    d, n_kv = case["head_dim"], case["n_kv"]
    x = dict(sh=sh, q=normal(sh.total, case["n_q"], d).to(dtype))
    for name in ("k", "v"):
        codes, scales = [], []
        for _ in range(n_kv):                 # a head at a time: the values take eight times their codes' bytes
            c, s = _quantise(normal(sh.cap_total, d))
            codes.append(c[:, 0::2] | c[:, 1::2] << 4)
            scales.append(s)
        x[name], x[name + "_scale"] = torch.stack(codes), torch.stack(scales)
    return x


def prepare(case, seed):
    s = _State()
    s.case = case
    attn = case["kind"] in ("tree4", "prompt4")
    x = _cache_inputs(case, seed) if attn else _rows_inputs(case, seed)
    sh = s.sh = x["sh"]
    dtype = x["q"].dtype
    d, n_q, n_kv, B = case["head_dim"], case["n_q"], case["n_kv"], case["B"]
    s.q, s.k, s.v = x["q"], x["k"], x["v"]
    s.seq_len = _dev(sh.L)
    if attn:
        s.k_scale, s.v_scale = x["k_scale"], x["v_scale"]
        s.out = torch.empty_like(s.q)
        _attn_indices(s, case, sh)
    else:
        for name in ("q_norm", "k_norm", "cos", "sin"):
            setattr(s, name, x[name])
        s.pos, s.dest = _dev(sh.pos), _dev(sh.dest.astype(np.int64))
        s.q_out = torch.empty(sh.total, n_q, d, dtype=dtype, device="cuda")
        if case["bits"] == 4:
            rows = int(sh.acc_off[-1]) if case["kind"] == "commit" else sh.total
            s.k_out, s.v_out = (torch.empty(rows, n_kv, d, dtype=dtype, device="cuda") for _ in range(2))
        else:
            s.pool_k, s.pool_v = x["pool_k"], x["pool_v"]
        if case["kind"] == "commit":
            s.acc, s.path, s.kept = _dev(sh.acc), _dev(sh.path), _dev(sh.kept.astype(np.int64))
            s.L = _dev(sh.L)
    if own:
        from paper_2506_01986_amd import specmemo as sm
        s.sm, s.dt = sm, sm.FP32 if case["dtype"] == "fp32" else sm.BF16
        if not attn:
            s.rows = sm.QKVRows(s.q, s.k, s.v, s.pos, s.cos, s.sin, rot_dim=case["rot"],
                                rot_style=sm.ROT_HALVES if case["style"] == "halves" else sm.ROT_PAIRS,
                                q_norm=s.q_norm, k_norm=s.k_norm, eps=EPS)
        if case["bits"] != 4:
            s.kv = sm.KVPool(s.pool_k, s.pool_v, s.seq_len, sh.base, sh.cap, sh.L)
        else:
            if not attn:
                mem = [torch.empty(n_kv, sh.cap_total, d // w, dtype=torch.uint8, device="cuda") for w in (2, 2, 32, 32)]
            else:
                mem = [s.k, s.v, s.k_scale, s.v_scale]
            s.kv = sm.KV4Pool(*mem, s.seq_len, sh.base, sh.cap, sh.L)
        if case["tree"]:
            s.trees = sm.Trees(sh.off, sh.parent, sh.depth, sh.rank, device="cuda")
        if attn:
            s.px = sm.Prefix(sh.pbase, sh.plen) if sh.group_rows else None
            if case["tree"]:
                s.ws_bytes = sm.kv4_tree_attn_bytes(s.dt, s.trees, s.kv, n_q, s.px)
            else:
                s.ws_bytes = sm.kv4_prompt_attn_bytes(s.dt, sh.off, s.kv, n_q, s.px)
            s.ws = torch.empty(max(16, s.ws_bytes), dtype=torch.uint8, device="cuda")
    return s


def _attn_indices(s, case, sh):
    """The batch as a padded one: pool row of every key, query row of every node, and which nodes a tree's node sees."""
    B, n, before = case["B"], sh.n.astype(np.int64), (sh.plen + sh.L).astype(np.int64)
    j = np.arange(int((before + n).max()))[None, :]
    P = sh.plen[:, None]
    rows = np.where(j < P, sh.pbase[:, None] + j, sh.base[:, None] + j - P)
    s.rows_of = _dev(np.minimum(rows, (sh.base + sh.L + n - 1)[:, None] * (j >= P) + rows * (j < P)))
    i = np.arange(int(n.max()))[None, :]
    s.nodes_of = _dev(sh.off[:-1, None] + np.minimum(i, n[:, None] - 1))
    s.node_at = _dev(sh.seq * i.shape[1] + np.arange(sh.total) - sh.off[:-1][sh.seq])
    s.before, s.n = _dev(before), _dev(n)
    if case["tree"]:
        sees = np.zeros((B, i.shape[1], i.shape[1]), bool)
        for b, t in enumerate(sh.paths):
            for u, p in enumerate(t):
                sees[b, u, p] = True
        s.sees = _dev(sees)


# ---- run --------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)[s.case["kind"]](s)


def _own_append(s):
    if s.case["bits"] != 4:
        s.sm.kv_append(s.dt, s.sh.off, s.rows, s.kv, s.q_out)
        return s.q_out, s.pool_k, s.pool_v
    s.sm.kv4_append(s.dt, s.sh.off, s.rows, s.kv, s.q_out)
    s.sm.kv4_read(s.dt, s.sh.off, s.kv, s.k_out, s.v_out)
    return s.q_out, s.k_out, s.v_out


def _own_commit(s):
    s.sm.kv4_append(s.dt, s.sh.off, s.rows, s.kv, s.q_out)
    s.sm.kv4_compact(s.trees, s.kv, s.acc, s.path, s.path.shape[1])
    s.sm.kv4_read(s.dt, s.sh.acc_off, s.kv, s.k_out, s.v_out)
    return s.q_out, s.k_out, s.v_out, s.seq_len


def _own_tree4(s):
    s.sm.kv4_tree_attn(s.dt, s.trees, s.kv, s.case["n_q"], s.q, s.out, prefix=s.px, ws=s.ws, ws_bytes=s.ws_bytes)
    return s.out


def _own_prompt4(s):
    s.sm.kv4_prompt_attn(s.dt, s.sh.off, s.kv, s.case["n_q"], s.q, s.out, prefix=s.px, ws=s.ws, ws_bytes=s.ws_bytes)
    return s.out


def _turn(s, x, w, wide):
    """Norm (where there is a weight) and rotation of [rows][heads][d], in `wide`."""
    x = x.to(wide)
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.to(wide)
    r, pos = s.case["rot"], s.pos.long()
    c, t = s.cos[pos].to(wide)[:, None], s.sin[pos].to(wide)[:, None]
    if s.case["style"] == "halves":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * c - b * t, b * c + a * t], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * c - b * t, b * c + a * t], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _quantise(x):
    """Codes [...][d] (sign in bit 3) and scale bytes [...][d / 32] of x."""
    g = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(g.abs().amax(-1))
    E = torch.where(m <= 0.875, e - 3, e - 2).clamp(-125, 125)
    E = torch.where(m == 0, -125, E)
    y = torch.ldexp(g, -E[..., None])
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    for border, closed in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += a >= border if closed else a > border
    return (code | (y < 0).to(torch.uint8) << 3).flatten(-2), (E + 127).to(torch.uint8)


def _values(code, scale):
    """The values that codes [...][d] of groups with these scale bytes stand for, in 32 bits."""
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=code.device)
    return (grid[code.long()].unflatten(-1, (-1, 32)) * torch.exp2(scale.float() - 127)[..., None]).flatten(-2)


def _unpacked(codes, scale):
    return _values(torch.stack([codes & 15, codes >> 4], -1).flatten(-2), scale)


def _plain_append(s):
    dtype, four = s.q.dtype, s.case["bits"] == 4
    q = _turn(s, s.q, s.q_norm, torch.float32).to(dtype)
    k = _turn(s, s.k, s.k_norm, torch.float64 if four else torch.float32)
    if four:
        return q, _values(*_quantise(k)).to(dtype), _values(*_quantise(s.v.double())).to(dtype)
    s.pool_k.index_copy_(1, s.dest, k.to(dtype).transpose(0, 1))
    s.pool_v.index_copy_(1, s.dest, s.v.transpose(0, 1))
    return q, s.pool_k, s.pool_v


def _plain_commit(s):
    q, k, v = _plain_append(s)
    return q, k[s.kept], v[s.kept], s.L + s.acc + 1


def _plain_attn(s):
    """softmax(q k^T / sqrt(d)) v in 32 bits over the padded batch, as many KV heads at once as 2^30 scores are."""
    n_q, n_kv, d = s.case["n_q"], s.case["n_kv"], s.case["head_dim"]
    (B, keys), nodes, g = s.rows_of.shape, s.nodes_of.shape[1], n_q // n_kv
    at = torch.arange(keys, device="cuda")[None, None, :] - s.before[:, None, None]      # key's place among the new rows
    if s.case["tree"]:
        rel = at.clamp(0, nodes - 1).expand(B, nodes, keys)
        hidden = (at >= 0) & ~(s.sees.gather(2, rel) & (at < s.n[:, None, None]))
    else:
        hidden = at > torch.arange(nodes, device="cuda")[None, :, None]
    q = (s.q.float() * (1.0 / math.sqrt(d)))[s.nodes_of].view(B, nodes, n_kv, g, d).permute(2, 0, 1, 3, 4)
    step = max(1, min(n_kv, (1 << 30) // (B * nodes * g * keys)))
    parts = []
    for h in range(0, n_kv, step):
        kf, vf = (_unpacked(c[h:h + step], e[h:h + step])[:, s.rows_of].view(-1, keys, d)
                  for c, e in ((s.k, s.k_scale), (s.v, s.v_scale)))
        z = torch.bmm(q[h:h + step].reshape(-1, nodes * g, d), kf.transpose(1, 2).contiguous()).view(-1, B, nodes, g, keys)
        z.masked_fill_(hidden[None, :, :, None, :], NEG_INF)
        z -= z.amax(-1, keepdim=True)
        z.exp_()
        tot = z.sum(-1, keepdim=True)
        parts.append(torch.bmm(z.view(-1, nodes * g, keys), vf).view(-1, B, nodes, g, d) / tot)
    out = torch.cat(parts).permute(1, 2, 0, 3, 4).reshape(B * nodes, n_q, d)
    return out[s.node_at].to(s.q.dtype)


_own = dict(append=_own_append, commit=_own_commit, tree4=_own_tree4, prompt4=_own_prompt4)
_plain = dict(append=_plain_append, commit=_plain_commit, tree4=_plain_attn, prompt4=_plain_attn)


# ---- the definition in 64 bits -----------------------------------------------------

def exact(case, seed):
    if case["kind"] in ("append", "commit"):
        return _exact_rows(case, seed)
    return _exact_attn(case, seed)


def _nearest(x):
    """x [rows][heads][d] in 4 bits, as values: the nearest of the grid by distance, of two equally near the even code."""
    g = x.view(*x.shape[:2], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    E = torch.full_like(top, -125.0)
    for e in range(-125, 125):                # the least exponent that holds the group
        E = torch.where(top > 7 * 2.0 ** e, e + 1.0, E)
        if bool((top <= 7 * 2.0 ** e).all()):
            break
    u = (g * torch.exp2(-E)).abs()
    best, value = torch.full_like(u, float("inf")), torch.zeros_like(u)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):        # even codes first: an odd one has to be nearer
        far = (u - GRID[i]).abs()
        value = torch.where(far < best, GRID[i], value)
        best = torch.minimum(best, far)
    return (torch.sign(g) * value * torch.exp2(E)).view(x.shape)


def _exact_rows(case, seed):
    x = _rows_inputs(case, seed)
    sh, r = x["sh"], case["rot"]
    pos = _dev(sh.pos).long()
    first = torch.arange(r // 2, device="cuda") * (1 if case["style"] == "halves" else 2)
    second = first + (r // 2 if case["style"] == "halves" else 1)
    c, t = x["cos"].double()[pos].unsqueeze(1), x["sin"].double()[pos].unsqueeze(1)

    def turned(y, w):
        y = y.double()
        if w is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / case["head_dim"] + EPS) * w.double()
        out = y.clone()
        out[..., first] = y[..., first] * c - y[..., second] * t
        out[..., second] = y[..., first] * t + y[..., second] * c
        return out

    q, k, v = turned(x["q"], x["q_norm"]), turned(x["k"], x["k_norm"]), x["v"].double()
    if case["bits"] != 4:
        pool_k, pool_v = x["pool_k"].double(), x["pool_v"].double()
        dest = _dev(sh.dest.astype(np.int64))
        pool_k[:, dest], pool_v[:, dest] = k.transpose(0, 1), v.transpose(0, 1)
        return q, pool_k, pool_v
    k, v = _nearest(k), _nearest(v)
    if case["kind"] == "append":
        return q, k, v
    kept = _dev(sh.kept.astype(np.int64))
    return q, k[kept], v[kept], _dev((sh.L + sh.acc + 1).astype(np.int32))


def _exact_attn(case, seed):
    x = _cache_inputs(case, seed)
    sh, q = x["sh"], x["q"]
    n_q, d = case["n_q"], case["head_dim"]
    out = torch.empty(sh.total, n_q, d, dtype=torch.float64, device="cuda")
    grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")

    def head(name, kv, rows):
        byte = x[name][kv, rows].long()
        y = torch.empty(len(rows), d, dtype=torch.float64, device="cuda")
        for odd in (0, 1):
            nib = byte // 16 if odd else byte % 16
            y[:, odd::2] = grid[nib % 8] * (1 - 2 * (nib // 8))
        return y * torch.exp2(x[name + "_scale"][kv, rows].double() - 127).repeat_interleave(32, 1)

    for b in range(case["B"]):
        o, n, L, P = int(sh.off[b]), int(sh.n[b]), int(sh.L[b]), int(sh.plen[b])
        rows = _dev(np.concatenate([np.arange(P) + int(sh.pbase[b]), np.arange(L + n) + int(sh.base[b])]).astype(np.int64))
        if case["tree"]:
            bar = np.ones((n, n), bool)
            for u in range(n):
                bar[u, sh.paths[b][u]] = False
            bar = _dev(bar)
        for kv in range(case["n_kv"]):
            kd, vd = head("k", kv, rows), head("v", kv, rows)
            for h in range(kv * n_q // case["n_kv"], (kv + 1) * n_q // case["n_kv"]):
                for i0 in range(0, n, 4096):
                    i1 = min(n, i0 + 4096)
                    z = q[o + i0:o + i1, h].double() @ kd.t().contiguous() / math.sqrt(d)
                    if case["tree"]:
                        z[:, P + L:] = z[:, P + L:].masked_fill(bar, NEG_INF)
                    else:
                        z = z.masked_fill(torch.ones_like(z, dtype=torch.bool).triu_(P + L + i0 + 1), NEG_INF)
                    out[o + i0:o + i1, h] = torch.exp(z - torch.logsumexp(z, 1, keepdim=True)) @ vd
    return out
