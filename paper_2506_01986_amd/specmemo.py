"""ctypes binding of libspecmemo (include/specmemo.h).

Argument marshalling only: torch tensors provide device memory and the stream,
numpy arrays the host mirrors; every stage runs in the library's HIP kernels.
The library is loaded on first use; if it has not been built, ``load()``
raises instead of falling back to anything else.
"""

from __future__ import annotations

import ctypes as C
import os
import re
from typing import Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "_build", "libspecmemo.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "specmemo.h")

FP32, BF16 = 0, 1
GREEDY, TYPICAL = 0, 1
HEADS_ROWMAJOR, HEADS_PACKED, HEADS_INPUT_PER_HEAD = 0, 1, 2
WS_TOPK, WS_ATTN, WS_ACCEPT, WS_PAD, WS_SAMPLE = 0, 1, 2, 3, 4
ROT_HALVES, ROT_PAIRS = 0, 1

STATUS = {0: "OK", -1: "E_ARG", -2: "E_DTYPE", -3: "E_TREE", -4: "E_BUDGET", -5: "E_WORKSPACE", -6: "E_HIP"}


class SpecmemoError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code
        self.name = STATUS.get(code, str(code))


class _Trees(C.Structure):
    _fields_ = [("B", C.c_int32), ("node_off", C.c_void_p), ("parent", C.c_void_p), ("depth", C.c_void_p),
                ("rank", C.c_void_p), ("node_off_h", C.c_void_p), ("parent_h", C.c_void_p),
                ("depth_h", C.c_void_p), ("rank_h", C.c_void_p)]


class _KV(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("cap_total", C.c_int64), ("n_kv", C.c_int32),
                ("head_dim", C.c_int32), ("seq_len", C.c_void_p), ("seq_base_h", C.c_void_p),
                ("seq_cap_h", C.c_void_p), ("seq_len_h", C.c_void_p)]


class _Prefix(C.Structure):
    _fields_ = [("base_h", C.c_void_p), ("len_h", C.c_void_p)]


class _Rows(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64),
                ("v_stride", C.c_int64), ("q_norm", C.c_void_p), ("k_norm", C.c_void_p), ("eps", C.c_float),
                ("cos", C.c_void_p), ("sin", C.c_void_p), ("pos", C.c_void_p), ("n_pos", C.c_int32),
                ("rot_dim", C.c_int32), ("rot_style", C.c_int32)]


class _KV4(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("cap_total", C.c_int64), ("n_kv", C.c_int32), ("head_dim", C.c_int32), ("seq_len", C.c_void_p),
                ("seq_base_h", C.c_void_p), ("seq_cap_h", C.c_void_p), ("seq_len_h", C.c_void_p)]


class _Rules(C.Structure):
    _fields_ = [("counts", C.c_void_p), ("repetition", C.c_void_p), ("presence", C.c_void_p), ("frequency", C.c_void_p),
                ("bias_off", C.c_void_p), ("bias_id", C.c_void_p), ("bias_val", C.c_void_p), ("n_bias", C.c_int32),
                ("mask", C.c_void_p), ("mask_idx", C.c_void_p), ("n_masks", C.c_int32), ("mask_words", C.c_int32)]


class _Budget(C.Structure):
    _fields_ = [("max_memory", C.c_int64), ("base_model_bytes", C.c_int64), ("head_bytes", C.c_int64),
                ("layers", C.c_int32), ("n_kv", C.c_int32), ("head_dim", C.c_int32), ("vocab", C.c_int32),
                ("elem_bytes", C.c_int32), ("batch", C.c_int32), ("query_count", C.c_int32),
                ("query_length", C.c_int32), ("default_heads", C.c_int32)]


class _BudgetPlan(C.Structure):
    _fields_ = [("kind", C.c_int32), ("heads", C.c_int32), ("nodes", C.c_int32), ("leaves", C.c_int32),
                ("kv_bytes", C.c_int64), ("total_bytes", C.c_int64)]


PLAN_DEFAULT, PLAN_PRUNED, PLAN_FEWER_HEADS, PLAN_NONE = 0, 1, 2, -1

_lib = None


def load():
    """Load libspecmemo.so; raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libspecmemo is not built ({LIB_PATH}); run __graft_entry__.build()")
        lib = C.CDLL(LIB_PATH)
        vp, i32, sz, f32 = C.c_void_p, C.c_int32, C.c_size_t, C.c_float
        PT, PK = C.POINTER(_Trees), C.POINTER(_KV)
        lib.specmemo_medusa_topk.argtypes = [i32, PT, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.specmemo_pack_heads.argtypes = [i32, i32, i32, i32, vp, vp, vp]
        lib.specmemo_pack_heads.restype = C.c_int
        lib.specmemo_packed_heads_bytes.argtypes = [i32, i32, i32, i32]
        lib.specmemo_packed_heads_bytes.restype = C.c_size_t
        lib.specmemo_tree_attn.argtypes = [i32, PT, PK, i32, f32, vp, vp, vp, sz, vp]
        lib.specmemo_tree_attn_noalloc.argtypes = [i32, PT, PK, i32, f32, vp, vp, vp]
        lib.specmemo_accept.argtypes = [i32, PT, i32, i32, f32, f32, f32, vp, vp, vp, vp, i32, vp, vp, sz, vp]
        lib.specmemo_kv_compact.argtypes = [i32, PT, PK, vp, vp, i32, vp]
        lib.specmemo_accept_compact.argtypes = [i32, PT, PK, i32, i32, f32, f32, f32, vp, vp, vp, vp, i32, vp, vp, sz, vp]
        lib.specmemo_workspace_bytes.argtypes = [i32, i32, PT, PK, i32, i32]
        lib.specmemo_workspace_bytes.restype = C.c_size_t
        lib.specmemo_last_error.restype = C.c_char_p
        lib.specmemo_abi_version.restype = C.c_int32
        for f in ("specmemo_medusa_topk", "specmemo_tree_attn", "specmemo_accept", "specmemo_kv_compact",
                  "specmemo_accept_compact", "specmemo_tree_attn_noalloc"):
            getattr(lib, f).restype = C.c_int
        i64 = C.c_int64
        u64 = C.c_uint64
        lib.specmemo_head_logits.argtypes = [i32, i32, i32, i32, i32, vp, vp, i32, vp, vp]
        lib.specmemo_head_logits.restype = C.c_int
        lib.specmemo_medusa_resblock.argtypes = [i32, i32, i32, i32, vp, vp, i32, vp, vp, vp]
        lib.specmemo_medusa_resblock.restype = C.c_int
        lib.specmemo_sample_next.argtypes = [i32, PT, i32, f32, u64, u64, vp, vp, vp, i32, vp, vp, sz, vp]
        lib.specmemo_sample_next.restype = C.c_int
        lib.specmemo_key_mask_words.argtypes = [i64]
        lib.specmemo_key_mask_words.restype = i64
        lib.specmemo_tree_attn_padded.argtypes = [i32, PT, PK, vp, i64, i32, f32, vp, vp, vp, sz, vp]
        lib.specmemo_tree_attn_padded.restype = C.c_int
        lib.specmemo_kv_pad_update.argtypes = [i32, PT, PK, vp, vp, i32, vp, i64, vp, vp, sz, vp]
        lib.specmemo_kv_pad_update.restype = C.c_int
        PP = C.POINTER(_Prefix)
        lib.specmemo_prompt_attn.argtypes = [i32, i32, vp, PK, PP, i32, f32, vp, vp, vp, sz, vp]
        lib.specmemo_prompt_attn.restype = C.c_int
        lib.specmemo_prompt_attn_bytes.argtypes = [i32, i32, vp, PK, PP, i32]
        lib.specmemo_prompt_attn_bytes.restype = sz
        lib.specmemo_tree_attn_prefix.argtypes = [i32, PT, PK, PP, i32, f32, vp, vp, vp, sz, vp]
        lib.specmemo_tree_attn_prefix.restype = C.c_int
        lib.specmemo_tree_attn_prefix_bytes.argtypes = [i32, PT, PK, PP, i32]
        lib.specmemo_tree_attn_prefix_bytes.restype = sz
        PR, P4 = C.POINTER(_Rows), C.POINTER(_KV4)
        lib.specmemo_kv_append.argtypes = [i32, i32, vp, PR, i32, PK, vp, vp]
        lib.specmemo_kv4_append.argtypes = [i32, i32, vp, PR, i32, P4, vp, vp]
        lib.specmemo_kv4_read.argtypes = [i32, i32, vp, P4, vp, vp, vp]
        lib.specmemo_kv4_prompt_attn.argtypes = [i32, i32, vp, P4, PP, i32, f32, vp, vp, vp, sz, vp]
        lib.specmemo_kv4_prompt_attn_bytes.argtypes = [i32, i32, vp, P4, PP, i32]
        lib.specmemo_kv4_tree_attn.argtypes = [i32, PT, P4, PP, i32, f32, vp, vp, vp, sz, vp]
        lib.specmemo_kv4_tree_attn_bytes.argtypes = [i32, PT, P4, PP, i32]
        lib.specmemo_kv4_compact.argtypes = [PT, P4, vp, vp, i32, vp]
        for f in ("specmemo_kv_append", "specmemo_kv4_append", "specmemo_kv4_read", "specmemo_kv4_prompt_attn",
                  "specmemo_kv4_tree_attn", "specmemo_kv4_compact"):
            getattr(lib, f).restype = C.c_int
        for f in ("specmemo_kv4_prompt_attn_bytes", "specmemo_kv4_tree_attn_bytes"):
            getattr(lib, f).restype = sz
        lib.specmemo_mem_kv4_bytes.argtypes = [i32, i32, i32, i32, i64]
        lib.specmemo_mem_kv4_bytes.restype = i64
        lib.specmemo_logit_rules.argtypes = [i32, PT, i32, C.POINTER(_Rules), vp, vp, vp, vp]
        lib.specmemo_token_counts.argtypes = [i32, i32, vp, vp, vp, vp, i32, vp]
        lib.specmemo_count_accepted.argtypes = [PT, i32, vp, vp, vp, i32, vp, vp]
        for f in ("specmemo_logit_rules", "specmemo_token_counts", "specmemo_count_accepted"):
            getattr(lib, f).restype = C.c_int
        lib.specmemo_mem_kv_bytes.argtypes = [i32, i32, i32, i32, i64, i32]
        lib.specmemo_mem_buffer_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
        lib.specmemo_mem_total_bytes.argtypes = [i64, i64, i32, i64, i64]
        lib.specmemo_tree_full_nodes.argtypes = [i32, i32]
        for f in ("specmemo_mem_kv_bytes", "specmemo_mem_buffer_bytes", "specmemo_mem_total_bytes",
                  "specmemo_tree_full_nodes"):
            getattr(lib, f).restype = i64
        lib.specmemo_tree_build.argtypes = [i32, i32, i32, i32, vp, vp, vp]
        lib.specmemo_tree_build.restype = C.c_int
        lib.specmemo_tree_leaves.argtypes = [i32, vp, vp, vp]
        lib.specmemo_tree_leaves.restype = i32
        lib.specmemo_tree_prune.argtypes = [i32, vp, vp, vp, i32, vp, vp, vp, vp, vp]
        lib.specmemo_tree_prune.restype = C.c_int
        lib.specmemo_plan_budget.argtypes = [C.POINTER(_Budget), i32, vp, vp, vp, C.POINTER(_BudgetPlan)]
        lib.specmemo_plan_budget.restype = C.c_int
        lib.specmemo_plan_tree_sizes.argtypes = [i32, vp, vp, i32, vp]
        lib.specmemo_plan_tree_sizes.restype = C.c_int
        _lib = lib
    return _lib


def declared_functions() -> list:
    """Names of the functions include/specmemo.h declares."""
    text = open(HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(specmemo_\w+)\s*\(", text)))


def _check(rc: int):
    if rc != 0:
        raise SpecmemoError(rc, load().specmemo_last_error().decode())


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    try:
        return x.data_ptr()      # tensors first: a step passes about 35 of them (0.1 us each, 0.3 after type checks)
    except AttributeError:
        if isinstance(x, int):
            return x
        if isinstance(x, np.ndarray):
            return x.ctypes.data
        raise


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        # asking whether a GPU is available, and for a stream object, takes 3.6 us of a call: once CUDA is in use the
        # current stream's handle alone is asked for
        if torch.cuda.is_initialized():
            return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
        if not torch.cuda.is_available():
            return None
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _i32(x) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(x, dtype=np.int32))


_addressof, _from_buffer, _ndarray = C.addressof, C.c_char.from_buffer, np.ndarray


def _host_addr(a) -> int:
    """Address of a numpy array, asked for on every call (an array may be
    resized in place).  The buffer protocol answers in 0.25 us; ``ctypes.data``,
    which also serves what it does not take (read-only, strided and empty
    arrays), in 1.15 us."""
    if type(a) is _ndarray:
        try:
            return _addressof(_from_buffer(a))
        except (TypeError, ValueError, BufferError):
            pass
    return a.ctypes.data


class Trees:
    """Ragged batch of candidate trees: device arrays plus host mirrors."""

    _MIRRORS = ("node_off_h", "parent_h", "depth_h", "rank_h")

    def __init__(self, node_off, parent, depth, rank, device=None, dev_arrays=None):
        self.node_off_h, self.parent_h = _i32(node_off), _i32(parent)
        self.depth_h, self.rank_h = _i32(depth), _i32(rank)
        self.B = len(self.node_off_h) - 1
        if dev_arrays is not None:
            self.dev = dev_arrays
        else:
            import torch
            self.dev = [torch.from_numpy(a.copy()).to(device) for a in
                        (self.node_off_h, self.parent_h, self.depth_h, self.rank_h)]

    @property
    def total_nodes(self) -> int:
        return int(self.node_off_h[-1])

    @property
    def max_depth(self) -> int:
        return int(self.depth_h.max())

    def _addresses(self) -> tuple:
        return (_host_addr(self.node_off_h), _host_addr(self.parent_h), _host_addr(self.depth_h), _host_addr(self.rank_h))

    def struct(self) -> _Trees:
        w, x, y, z = self.node_off_h, self.parent_h, self.depth_h, self.rank_h
        if type(w) is type(x) is type(y) is type(z) is _ndarray:
            try:       # tensors and plain arrays without a call for each (2.1 us, 2.9 through the general form)
                a, b, c, d = self.dev
                return _Trees(self.B, a.data_ptr(), b.data_ptr(), c.data_ptr(), d.data_ptr(), _addressof(_from_buffer(w)),
                              _addressof(_from_buffer(x)), _addressof(_from_buffer(y)), _addressof(_from_buffer(z)))
            except (AttributeError, TypeError, ValueError, BufferError):
                pass
        return _Trees(self.B, *[_ptr(t) for t in self.dev], *self._addresses())


class KVPool:
    """One layer's budget-capped KV pool: device K, V and seq_len, host mirrors."""

    _MIRRORS = ("seq_base_h", "seq_cap_h", "seq_len_h")

    def __init__(self, k, v, seq_len_dev, seq_base, seq_cap, seq_len):
        self.k, self.v, self.seq_len = k, v, seq_len_dev
        self.seq_base_h = np.ascontiguousarray(seq_base, dtype=np.int64)
        self.seq_cap_h = _i32(seq_cap)
        self.seq_len_h = _i32(seq_len)
        self.n_kv, self.cap_total, self.head_dim = (int(s) for s in k.shape)

    def _addresses(self) -> tuple:
        return _host_addr(self.seq_base_h), _host_addr(self.seq_cap_h), _host_addr(self.seq_len_h)

    def struct(self) -> _KV:
        x, y, z = self.seq_base_h, self.seq_cap_h, self.seq_len_h
        if type(x) is type(y) is type(z) is _ndarray:
            try:
                return _KV(self.k.data_ptr(), self.v.data_ptr(), self.cap_total, self.n_kv, self.head_dim,
                           self.seq_len.data_ptr(), _addressof(_from_buffer(x)), _addressof(_from_buffer(y)),
                           _addressof(_from_buffer(z)))
            except (AttributeError, TypeError, ValueError, BufferError):
                pass
        return _KV(_ptr(self.k), _ptr(self.v), self.cap_total, self.n_kv, self.head_dim,
                   _ptr(self.seq_len), *self._addresses())


def abi_version() -> int:
    return load().specmemo_abi_version()


def workspace_bytes(which: int, dt: int, trees: Trees, kv: Optional[KVPool], n_q_or_heads: int, vocab: int = 0) -> int:
    ts = trees.struct()
    ks = kv.struct() if kv is not None else None
    return load().specmemo_workspace_bytes(which, dt, C.byref(ts), C.byref(ks) if ks is not None else None,
                                           n_q_or_heads, vocab)


def medusa_topk(dt: int, trees: Trees, hidden: int, vocab: int, n_heads: int, topk: Sequence[int], h, head_w,
                root_tok, topk_ids, node_tok, logits_out=None, topk_vals=None, ws=None, ws_bytes: int = 0,
                stream=None, head_layout: int = HEADS_ROWMAJOR):
    ts = trees.struct()
    tk = _i32(topk)
    _check(load().specmemo_medusa_topk(dt, C.byref(ts), hidden, vocab, n_heads, tk.ctypes.data, _ptr(h),
                                       _ptr(head_w), head_layout, _ptr(root_tok), _ptr(logits_out),
                                       _ptr(topk_ids), _ptr(topk_vals), _ptr(node_tok), _ptr(ws), ws_bytes,
                                       _stream(stream)))


def head_logits(dt: int, B: int, hidden: int, vocab: int, n_heads: int, h, head_w, logits_out,
                head_layout: int = HEADS_ROWMAJOR, stream=None):
    _check(load().specmemo_head_logits(dt, B, hidden, vocab, n_heads, _ptr(h), _ptr(head_w), head_layout,
                                       _ptr(logits_out), _stream(stream)))


def medusa_resblock(dt: int, B: int, hidden: int, n_heads: int, h, w1, b1, out, w1_layout: int = HEADS_PACKED,
                    stream=None):
    _check(load().specmemo_medusa_resblock(dt, B, hidden, n_heads, _ptr(h), _ptr(w1), w1_layout, _ptr(b1),
                                           _ptr(out), _stream(stream)))


def sample_next(dt: int, trees: Trees, vocab: int, temperature: float, seed: int, offset: int, base_logits,
                accept_len, path, path_stride: int, next_tok, ws=None, ws_bytes: int = 0, stream=None):
    ts = trees.struct()
    _check(load().specmemo_sample_next(dt, C.byref(ts), vocab, temperature, seed, offset, _ptr(base_logits),
                                       _ptr(accept_len), _ptr(path), path_stride, _ptr(next_tok), _ptr(ws),
                                       ws_bytes, _stream(stream)))


def packed_heads_bytes(dt: int, n_heads: int, vocab: int, hidden: int) -> int:
    return int(load().specmemo_packed_heads_bytes(dt, n_heads, vocab, hidden))


def pack_heads(dt: int, n_heads: int, vocab: int, hidden: int, src, dst, stream=None):
    _check(load().specmemo_pack_heads(dt, n_heads, vocab, hidden, _ptr(src), _ptr(dst), _stream(stream)))


def tree_attn(dt: int, trees: Trees, kv: KVPool, n_q: int, q, out, scale: float = 0.0, ws=None,
              ws_bytes: int = 0, stream=None):
    ts, ks = trees.struct(), kv.struct()
    _check(load().specmemo_tree_attn(dt, C.byref(ts), C.byref(ks), n_q, scale, _ptr(q), _ptr(out), _ptr(ws),
                                     ws_bytes, _stream(stream)))


STATIC_SCRATCH_BYTES = 32 << 20


def tree_attn_noalloc(dt: int, trees: Trees, kv: KVPool, n_q: int, q, out, scale: float = 0.0, stream=None):
    ts, ks = trees.struct(), kv.struct()
    _check(load().specmemo_tree_attn_noalloc(dt, C.byref(ts), C.byref(ks), n_q, scale, _ptr(q), _ptr(out),
                                             _stream(stream)))


def accept(dt: int, trees: Trees, vocab: int, mode: int, base_logits, node_tok, accept_len, path, path_stride: int,
           next_tok, temperature: float = 1.0, eps: float = 0.09, delta: float = 0.3, ws=None, ws_bytes: int = 0,
           stream=None):
    ts = trees.struct()
    _check(load().specmemo_accept(dt, C.byref(ts), vocab, mode, temperature, eps, delta, _ptr(base_logits),
                                  _ptr(node_tok), _ptr(accept_len), _ptr(path), path_stride, _ptr(next_tok),
                                  _ptr(ws), ws_bytes, _stream(stream)))


def accept_compact(dt: int, trees: Trees, kv: KVPool, vocab: int, mode: int, base_logits, node_tok, accept_len, path,
                   path_stride: int, next_tok, temperature: float = 1.0, eps: float = 0.09, delta: float = 0.3,
                   ws=None, ws_bytes: int = 0, stream=None):
    ts, ks = trees.struct(), kv.struct()
    _check(load().specmemo_accept_compact(dt, C.byref(ts), C.byref(ks), vocab, mode, temperature, eps, delta,
                                          _ptr(base_logits), _ptr(node_tok), _ptr(accept_len), _ptr(path),
                                          path_stride, _ptr(next_tok), _ptr(ws), ws_bytes, _stream(stream)))


def kv_compact(dt: int, trees: Trees, kv: KVPool, accept_len, path, path_stride: int, stream=None):
    ts, ks = trees.struct(), kv.struct()
    _check(load().specmemo_kv_compact(dt, C.byref(ts), C.byref(ks), _ptr(accept_len), _ptr(path), path_stride,
                                      _stream(stream)))


# ---- padded batching -------------------------------------------------------------

def key_mask_words(cap_total: int) -> int:
    return int(load().specmemo_key_mask_words(cap_total))


def pack_key_valid(flags) -> np.ndarray:
    """Per-row flags (nonzero = token, 0 = pad) -> the library's uint32 words
    (bit r % 32 of word r / 32), padded to key_mask_words(len(flags))."""
    f = np.asarray(flags) != 0
    words = np.zeros(key_mask_words(len(f)), np.uint32)
    packed = np.packbits(f, bitorder="little")
    packed = np.concatenate([packed, np.zeros((-len(packed)) % 4, np.uint8)])
    words[:len(packed) // 4] = packed.view("<u4")
    return words


def unpack_key_valid(words, cap_total: int) -> np.ndarray:
    """Inverse of pack_key_valid: uint8 flags [cap_total]."""
    w = np.ascontiguousarray(np.asarray(words, dtype=np.uint32))
    return np.unpackbits(w.view(np.uint8), bitorder="little")[:cap_total]


def _words(key_valid, words):
    if words is not None:
        return words
    return int(key_valid.numel()) if hasattr(key_valid, "numel") else len(key_valid)


def tree_attn_padded(dt: int, trees: Trees, kv: KVPool, key_valid, n_q: int, q, out, scale: float = 0.0, ws=None,
                     ws_bytes: int = 0, stream=None, key_valid_words=None):
    ts, ks = trees.struct(), kv.struct()
    _check(load().specmemo_tree_attn_padded(dt, C.byref(ts), C.byref(ks), _ptr(key_valid),
                                            _words(key_valid, key_valid_words), n_q, scale, _ptr(q), _ptr(out),
                                            _ptr(ws), ws_bytes, _stream(stream)))


def kv_pad_update(dt: int, trees: Trees, kv: KVPool, accept_len, path, path_stride: int, key_valid, pos, ws=None,
                  ws_bytes: int = 0, stream=None, key_valid_words=None):
    ts, ks = trees.struct(), kv.struct()
    _check(load().specmemo_kv_pad_update(dt, C.byref(ts), C.byref(ks), _ptr(accept_len), _ptr(path), path_stride,
                                         _ptr(key_valid), _words(key_valid, key_valid_words), _ptr(pos), _ptr(ws),
                                         ws_bytes, _stream(stream)))


# ---- prompts and shared prefixes ----------------------------------------------------

class Prefix:
    """Rows of the pool that a sequence sees before its own slab rows: first row and length per sequence (host arrays)."""

    def __init__(self, base, length):
        self.base_h = np.ascontiguousarray(base, dtype=np.int64)
        self.len_h = _i32(length)
        if self.base_h.shape != self.len_h.shape or self.base_h.ndim != 1:
            raise ValueError("one base and one length per sequence")

    def struct(self) -> _Prefix:
        return _Prefix(_host_addr(self.base_h), _host_addr(self.len_h))


def _prefix_ref(prefix: Optional[Prefix], B: int):
    if prefix is None:
        return None
    if len(prefix.base_h) != B or len(prefix.len_h) != B:
        raise ValueError(f"prefix of {len(prefix.base_h)} sequences for a batch of {B}")
    return C.byref(prefix.struct())


def _new_off(new_off, kv: KVPool) -> np.ndarray:
    off = _offsets(new_off)
    if off.ndim != 1 or len(off) < 1 or min(len(kv.seq_base_h), len(kv.seq_cap_h), len(kv.seq_len_h)) < len(off) - 1:
        raise ValueError(f"new_off of {off.shape} for a pool of {len(kv.seq_base_h)} sequences")
    return off


def prompt_attn_bytes(dt: int, new_off, kv: KVPool, n_q: int, prefix: Optional[Prefix] = None) -> int:
    off, ks = _new_off(new_off, kv), kv.struct()
    return int(load().specmemo_prompt_attn_bytes(dt, len(off) - 1, _host_addr(off), C.byref(ks),
                                                 _prefix_ref(prefix, len(off) - 1), n_q))


def prompt_attn(dt: int, new_off, kv: KVPool, n_q: int, q, out, prefix: Optional[Prefix] = None, scale: float = 0.0,
                ws=None, ws_bytes: int = 0, stream=None):
    off, ks = _new_off(new_off, kv), kv.struct()
    _check(load().specmemo_prompt_attn(dt, len(off) - 1, _host_addr(off), C.byref(ks), _prefix_ref(prefix, len(off) - 1),
                                       n_q, scale, _ptr(q), _ptr(out), _ptr(ws), ws_bytes, _stream(stream)))


def tree_attn_prefix_bytes(dt: int, trees: Trees, kv: KVPool, prefix: Prefix, n_q: int) -> int:
    ts, ks = trees.struct(), kv.struct()
    return int(load().specmemo_tree_attn_prefix_bytes(dt, C.byref(ts), C.byref(ks), _prefix_ref(prefix, trees.B), n_q))


def tree_attn_prefix(dt: int, trees: Trees, kv: KVPool, prefix: Prefix, n_q: int, q, out, scale: float = 0.0, ws=None,
                     ws_bytes: int = 0, stream=None):
    ts, ks = trees.struct(), kv.struct()
    _check(load().specmemo_tree_attn_prefix(dt, C.byref(ts), C.byref(ks), _prefix_ref(prefix, trees.B), n_q, scale,
                                            _ptr(q), _ptr(out), _ptr(ws), ws_bytes, _stream(stream)))


# ---- new rows of the pool, and the pool in 4 bits -------------------------------------

class KV4Pool:
    """One layer's pool in 4 bits: codes [n_kv][rows][head_dim / 2] and scale bytes [n_kv][rows][head_dim / 32] of K and V
    (uint8 tensors), device seq_len, host mirrors."""

    def __init__(self, k, v, k_scale, v_scale, seq_len_dev, seq_base, seq_cap, seq_len):
        self.n_kv, self.cap_total, half = (int(s) for s in k.shape)
        self.head_dim = 2 * half
        for name, x, w in (("k", k, half), ("v", v, half), ("k_scale", k_scale, half // 16), ("v_scale", v_scale, half // 16)):
            _check_tensor(name, x, ("torch.uint8",))
            if tuple(x.shape) != (self.n_kv, self.cap_total, w):
                raise ValueError(f"{name}: shape {tuple(x.shape)}, expected {(self.n_kv, self.cap_total, w)}")
        _check_tensor("seq_len", seq_len_dev, _INT32)
        self.k, self.v, self.k_scale, self.v_scale, self.seq_len = k, v, k_scale, v_scale, seq_len_dev
        self.seq_base_h = np.ascontiguousarray(seq_base, dtype=np.int64)
        self.seq_cap_h = _i32(seq_cap)
        self.seq_len_h = _i32(seq_len)

    def struct(self) -> _KV4:
        x, y, z = self.seq_base_h, self.seq_cap_h, self.seq_len_h
        if type(x) is type(y) is type(z) is _ndarray:
            try:       # as KVPool (1.6 us, 2.6 through the general form)
                return _KV4(self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(),
                            self.cap_total, self.n_kv, self.head_dim, self.seq_len.data_ptr(), _addressof(_from_buffer(x)),
                            _addressof(_from_buffer(y)), _addressof(_from_buffer(z)))
            except (AttributeError, TypeError, ValueError, BufferError):
                pass
        return _KV4(_ptr(self.k), _ptr(self.v), _ptr(self.k_scale), _ptr(self.v_scale), self.cap_total, self.n_kv,
                    self.head_dim, _ptr(self.seq_len), _host_addr(x), _host_addr(y), _host_addr(z))


_VALUES = ("torch.float32", "torch.bfloat16")
_TYPES = {}        # torch types seen -> the library's, or _INT32


class QKVRows:
    """New tokens' q, k and v [tokens][heads][head_dim], the norm and the rotation (include/specmemo.h, specmemo_rows).

    The three may be slices of one buffer: a token's heads lie together, tokens at one stride.  q: None for keys and
    values alone.  cos, sin: fp32 [positions][rot_dim / 2]; pos: int32 [tokens]; rot_dim None: cos's columns twice, 0: no
    rotation."""

    def __init__(self, q, k, v, pos=None, cos=None, sin=None, rot_dim: Optional[int] = None, rot_style: int = ROT_HALVES,
                 q_norm=None, k_norm=None, eps: float = 1e-5):
        if k is None or v is None or k.dim() != 3:
            raise ValueError("keys and values [tokens][heads][head_dim] are needed")
        d = int(k.shape[2])
        for name, x in (("q", q), ("k", k), ("v", v)):
            if x is None:
                continue
            if x.dim() != 3 or int(x.shape[0]) != int(k.shape[0]) or int(x.shape[2]) != d or x.dtype != k.dtype or str(x.dtype) not in _VALUES:
                raise ValueError(f"{name}: {tuple(x.shape)} of {x.dtype} beside keys {tuple(k.shape)} of {k.dtype}")
            if x.stride(2) != 1 or (x.shape[1] > 1 and x.stride(1) != d):
                raise ValueError(f"{name}: a token's heads must lie together, got strides {x.stride()}")
        if v.shape != k.shape:
            raise ValueError(f"values {tuple(v.shape)} beside keys {tuple(k.shape)}")
        for name, w in (("q_norm", q_norm), ("k_norm", k_norm)):
            _check_tensor(name, w, (str(k.dtype),))
            if w is not None and w.numel() != d:
                raise ValueError(f"{name}: {w.numel()} weights for heads of {d}")
        if rot_dim is None:
            rot_dim = 0 if cos is None else 2 * int(cos.shape[1])
        n_pos = 0
        if rot_dim:
            if cos is None or sin is None or pos is None:
                raise ValueError("a rotation needs cos, sin and pos")
            _check_tensor("cos", cos, _FLOAT32)
            _check_tensor("sin", sin, _FLOAT32)
            _check_tensor("pos", pos, _INT32)
            n_pos = int(cos.shape[0])
            if tuple(cos.shape) != (n_pos, rot_dim // 2) or cos.shape != sin.shape:
                raise ValueError(f"cos {tuple(cos.shape)}, sin {tuple(sin.shape)} for {rot_dim} rotated columns")
            if int(pos.numel()) != int(k.shape[0]):
                raise ValueError(f"{pos.numel()} positions for {k.shape[0]} tokens")
        self.q, self.k, self.v, self.pos, self.cos, self.sin = q, k, v, pos, cos, sin
        self.q_norm, self.k_norm, self.eps = q_norm, k_norm, eps
        self.tokens, self.n_q, self.n_kv, self.head_dim = int(k.shape[0]), 0 if q is None else int(q.shape[1]), int(k.shape[1]), d
        self.rot_dim, self.rot_style, self.n_pos, self.dt = rot_dim, rot_style, n_pos, _VALUES.index(str(k.dtype))
        stride = lambda x: 0 if x is None else int(x.stride(0)) if self.tokens > 1 else int(x.shape[1]) * d
        self._layout = stride(q), stride(k), stride(v)

    def struct(self) -> _Rows:
        at = lambda x: None if x is None else x.data_ptr()
        return _Rows(at(self.q), self.k.data_ptr(), self.v.data_ptr(), *self._layout, at(self.q_norm), at(self.k_norm),
                     self.eps, at(self.cos), at(self.sin), at(self.pos), self.n_pos, self.rot_dim, self.rot_style)


def _offsets(new_off) -> np.ndarray:
    """Host offsets as an int32 array (arrays of that kind as they are: 0.1 us, 0.5 through numpy's conversions)."""
    if type(new_off) is _ndarray and new_off.dtype is _I32 and new_off.ndim == 1 and new_off.flags.c_contiguous:
        return new_off
    return _i32(new_off)


_I32 = np.dtype(np.int32)


def _out_tensor(name: str, x, dtype, values: int):
    if x.dtype is not dtype or x.numel() != values or not x.is_contiguous():
        raise ValueError(f"{name}: {values} values of {dtype} without gaps expected, got {tuple(x.shape)} of {x.dtype}")


def _q_and_out(dt: int, q, out, values: int) -> tuple:
    """Addresses of queries and outputs.  Tensors are read and written as they lie: at least `values` of the call's type
    (rows past a batch are left alone), without gaps; addresses are taken as they are.  (0.6 us of a call.)"""
    try:
        if (_TYPES[q.dtype] == _TYPES[out.dtype] == dt and q.numel() >= values and out.numel() >= values and q.is_contiguous()
                and out.is_contiguous()):
            return q.data_ptr(), out.data_ptr()
    except (AttributeError, KeyError):
        pass
    for name, x in (("q", q), ("out", out)):
        if hasattr(x, "is_contiguous"):
            if str(x.dtype) in _VALUES:
                _TYPES[x.dtype] = _VALUES.index(str(x.dtype))
            if _TYPES.get(x.dtype) != dt or x.numel() < values or not x.is_contiguous():
                raise ValueError(f"{name}: {values} values of type {dt} without gaps expected, got {tuple(x.shape)} of {x.dtype}, "
                                 f"strides {x.stride()}")
    return _ptr(q), _ptr(out)


def _append(fn, dt: int, new_off, rows: QKVRows, kv, q_out, stream):
    off = _offsets(new_off)
    B, tokens = len(off) - 1, rows.tokens
    if B < 0 or len(kv.seq_len_h) < B or len(kv.seq_base_h) < B or len(kv.seq_cap_h) < B:
        raise ValueError(f"new_off of {off.shape} for a pool of {len(kv.seq_base_h)} sequences")
    if off[B] != tokens or rows.n_kv != kv.n_kv or rows.head_dim != kv.head_dim or rows.dt != dt:
        raise ValueError(f"{tokens} tokens of {rows.n_kv} KV heads of {rows.head_dim}, type {rows.dt}, for {off[B]} tokens and a "
                         f"pool of {kv.n_kv} heads of {kv.head_dim}, type {dt}")
    if q_out is None:
        if rows.n_q and tokens:
            raise ValueError("q_out is missing")
    else:
        _out_tensor("q_out", q_out, rows.k.dtype, tokens * rows.n_q * rows.head_dim)
    _check(fn(dt, B, _host_addr(off), C.byref(rows.struct()), rows.n_q, C.byref(kv.struct()),
              None if q_out is None else q_out.data_ptr(), _stream(stream)))


def kv_append(dt: int, new_off, rows: QKVRows, kv: KVPool, q_out, stream=None):
    values = kv.n_kv * kv.cap_total * kv.head_dim
    for x in (kv.k, kv.v):      # written in the rows' type, as they lie, up to the last row
        if x.dtype is not rows.k.dtype or not x.is_contiguous() or x.numel() != values:
            raise ValueError(f"a pool of {values} values of {rows.k.dtype} without gaps expected, got {tuple(x.shape)} of {x.dtype}, "
                             f"strides {x.stride()}")
    _append(load().specmemo_kv_append, dt, new_off, rows, kv, q_out, stream)


def kv4_append(dt: int, new_off, rows: QKVRows, kv: KV4Pool, q_out, stream=None):
    _append(load().specmemo_kv4_append, dt, new_off, rows, kv, q_out, stream)


def kv4_read(dt: int, new_off, kv: KV4Pool, k_out, v_out, stream=None):
    off = _offsets(new_off)
    B = len(off) - 1
    if B < 0 or len(kv.seq_len_h) < B or len(kv.seq_base_h) < B or len(kv.seq_cap_h) < B:
        raise ValueError(f"new_off of {off.shape} for a pool of {len(kv.seq_base_h)} sequences")
    if str(k_out.dtype) != _VALUES[dt]:
        raise ValueError(f"outputs of {k_out.dtype} for type {dt}")
    values = int(off[B]) * kv.n_kv * kv.head_dim
    _out_tensor("k_out", k_out, k_out.dtype, values)
    _out_tensor("v_out", v_out, k_out.dtype, values)
    _check(load().specmemo_kv4_read(dt, B, _host_addr(off), C.byref(kv.struct()), k_out.data_ptr(), v_out.data_ptr(),
                                    _stream(stream)))


def kv4_prompt_attn_bytes(dt: int, new_off, kv: KV4Pool, n_q: int, prefix: Optional[Prefix] = None) -> int:
    off, ks = _new_off(new_off, kv), kv.struct()
    return int(load().specmemo_kv4_prompt_attn_bytes(dt, len(off) - 1, _host_addr(off), C.byref(ks),
                                                     _prefix_ref(prefix, len(off) - 1), n_q))


def kv4_prompt_attn(dt: int, new_off, kv: KV4Pool, n_q: int, q, out, prefix: Optional[Prefix] = None, scale: float = 0.0,
                    ws=None, ws_bytes: int = 0, stream=None):
    off, ks = _new_off(new_off, kv), kv.struct()
    q_at, out_at = _q_and_out(dt, q, out, off.item(-1) * n_q * kv.head_dim)
    _check(load().specmemo_kv4_prompt_attn(dt, len(off) - 1, _host_addr(off), C.byref(ks), _prefix_ref(prefix, len(off) - 1),
                                           n_q, scale, q_at, out_at, _ptr(ws), ws_bytes, _stream(stream)))


def _check_sequences(trees: Trees, kv: KV4Pool):
    if trees.B > len(kv.seq_base_h) or trees.B > len(kv.seq_cap_h) or trees.B > len(kv.seq_len_h):
        raise ValueError(f"{trees.B} trees for a pool of {min(len(kv.seq_base_h), len(kv.seq_cap_h), len(kv.seq_len_h))} sequences")


def kv4_tree_attn_bytes(dt: int, trees: Trees, kv: KV4Pool, n_q: int, prefix: Optional[Prefix] = None) -> int:
    _check_sequences(trees, kv)
    ts, ks = trees.struct(), kv.struct()
    return int(load().specmemo_kv4_tree_attn_bytes(dt, C.byref(ts), C.byref(ks), _prefix_ref(prefix, trees.B), n_q))


def kv4_tree_attn(dt: int, trees: Trees, kv: KV4Pool, n_q: int, q, out, prefix: Optional[Prefix] = None, scale: float = 0.0,
                  ws=None, ws_bytes: int = 0, stream=None):
    _check_sequences(trees, kv)
    ts, ks = trees.struct(), kv.struct()
    q_at, out_at = _q_and_out(dt, q, out, trees.node_off_h.item(-1) * n_q * kv.head_dim)
    _check(load().specmemo_kv4_tree_attn(dt, C.byref(ts), C.byref(ks), _prefix_ref(prefix, trees.B), n_q, scale, q_at, out_at,
                                         _ptr(ws), ws_bytes, _stream(stream)))


def _compact_integers(B: int, seq_len, accept_len, path, path_stride: int):
    """Lengths and paths are read and written as they lie: 32-bit integers, as many as the batch has, without gaps (0.8 us of
    a call); addresses are taken as they are."""
    try:
        if (_TYPES[accept_len.dtype] == _TYPES[path.dtype] == _INT32 and accept_len.numel() >= B and path.numel() >= B * path_stride
                and seq_len.numel() >= B and accept_len.is_contiguous() and path.is_contiguous()):
            return
    except (AttributeError, KeyError):
        pass
    for name, x, values in (("seq_len", seq_len, B), ("accept_len", accept_len, B), ("path", path, B * path_stride)):
        if not hasattr(x, "is_contiguous"):
            continue
        _check_tensor(name, x, _INT32)
        _TYPES[x.dtype] = _INT32
        if x.numel() < values:
            raise ValueError(f"{name}: {values} values expected, got {x.numel()}")


def kv4_compact(trees: Trees, kv: KV4Pool, accept_len, path, path_stride: int, stream=None):
    _check_sequences(trees, kv)
    ts, ks = trees.struct(), kv.struct()
    _compact_integers(trees.B, kv.seq_len, accept_len, path, path_stride)
    _check(load().specmemo_kv4_compact(C.byref(ts), C.byref(ks), _ptr(accept_len), _ptr(path), path_stride, _stream(stream)))


# ---- rules on logits ----------------------------------------------------------------

_INT32, _FLOAT32 = ("torch.int32",), ("torch.float32",)


def _check_tensor(name: str, x, dtypes: tuple):
    """Tensors are read as they lie: of one of these types, without gaps (addresses are taken as they are)."""
    if hasattr(x, "is_contiguous") and (str(x.dtype) not in dtypes or not x.is_contiguous()):
        raise ValueError(f"{name}: a contiguous tensor of {' or '.join(dtypes)} expected, got {x.dtype} of strides {x.stride()}")


class LogitRules:
    """Device arrays of the penalties, biases and masks (include/specmemo.h, specmemo_rules); None leaves a rule out."""

    def __init__(self, counts=None, repetition=None, presence=None, frequency=None):
        _check_tensor("counts", counts, _INT32)
        for name, x in (("repetition", repetition), ("presence", presence), ("frequency", frequency)):
            _check_tensor(name, x, _FLOAT32)
        self.counts, self.repetition, self.presence, self.frequency = counts, repetition, presence, frequency
        self.bias_off = self.bias_id = self.bias_val = self.mask = self.mask_idx = None
        self.n_bias = self.n_masks = self.mask_words = 0

    def set_bias(self, off, ids, values):
        """Sequence b's biases are entries off[b] .. off[b+1] - 1 of ids and values."""
        if ids.numel() != values.numel():
            raise ValueError(f"{ids.numel()} bias ids, {values.numel()} values")
        _check_tensor("bias offsets", off, _INT32)
        _check_tensor("bias ids", ids, _INT32)
        _check_tensor("bias values", values, _FLOAT32)
        self.bias_off, self.bias_id, self.bias_val, self.n_bias = off, ids, values, int(ids.numel())

    def set_mask(self, mask, idx):
        """mask: [masks][words] 32-bit words (bit v % 32 of word v / 32: token v is allowed); idx: mask of each node, -1 for none."""
        _check_tensor("masks", mask, _INT32 + ("torch.uint32",))
        _check_tensor("mask indices", idx, _INT32)
        n, words = (int(s) for s in mask.shape)
        self.mask, self.mask_idx, self.n_masks, self.mask_words = mask, idx, n, words

    def struct(self) -> _Rules:
        return _Rules(_ptr(self.counts), _ptr(self.repetition), _ptr(self.presence), _ptr(self.frequency),
                      _ptr(self.bias_off), _ptr(self.bias_id), _ptr(self.bias_val), self.n_bias, _ptr(self.mask),
                      _ptr(self.mask_idx), self.n_masks, self.mask_words)


def logit_rules(dt: int, trees: Trees, vocab: int, logits, node_tok, rules: LogitRules, out, stream=None):
    ts, rs = trees.struct(), rules.struct()
    _check(load().specmemo_logit_rules(dt, C.byref(ts), vocab, C.byref(rs), _ptr(node_tok), _ptr(logits), _ptr(out),
                                       _stream(stream)))


def token_counts(vocab: int, tok_off_h, tok_off, tokens, counts, accumulate: bool = False, stream=None):
    """tok_off_h: host offsets [B+1]; tok_off: the same on the device."""
    off = _i32(tok_off_h)
    _check(load().specmemo_token_counts(len(off) - 1, vocab, _host_addr(off), _ptr(tok_off), _ptr(tokens), _ptr(counts),
                                        int(accumulate), _stream(stream)))


def count_accepted(trees: Trees, vocab: int, node_tok, accept_len, path, path_stride: int, counts, stream=None):
    ts = trees.struct()
    _check(load().specmemo_count_accepted(C.byref(ts), vocab, _ptr(node_tok), _ptr(accept_len), _ptr(path), path_stride,
                                          _ptr(counts), _stream(stream)))


# ---- memory budget and tree construction (host) ------------------------------

def _bytes(v: int) -> int:
    if v < 0:
        raise SpecmemoError(-1, load().specmemo_last_error().decode())
    return int(v)


def mem_kv_bytes(layers: int, batch: int, n_kv: int, head_dim: int, tokens: int, elem_bytes: int) -> int:
    return _bytes(load().specmemo_mem_kv_bytes(layers, batch, n_kv, head_dim, tokens, elem_bytes))


def mem_kv4_bytes(layers: int, batch: int, n_kv: int, head_dim: int, tokens: int) -> int:
    return _bytes(load().specmemo_mem_kv4_bytes(layers, batch, n_kv, head_dim, tokens))


def mem_buffer_bytes(batch: int, nodes: int, seqs: int, levels: int, vocab: int, elem_bytes: int) -> int:
    return _bytes(load().specmemo_mem_buffer_bytes(batch, nodes, seqs, levels, vocab, elem_bytes))


def mem_total_bytes(base_model_bytes: int, head_bytes: int, heads: int, kv: int, buffers: int) -> int:
    return _bytes(load().specmemo_mem_total_bytes(base_model_bytes, head_bytes, heads, kv, buffers))


def tree_full_nodes(arity: int, levels: int) -> int:
    return _bytes(load().specmemo_tree_full_nodes(arity, levels))


def tree_build(nodes: int, leaves: int, max_depth: int, arity: int):
    """(parent, depth, rank) int32 arrays of the built tree."""
    out = [np.zeros(max(nodes, 1), np.int32) for _ in range(3)]
    _check(load().specmemo_tree_build(nodes, leaves, max_depth, arity, *(a.ctypes.data for a in out)))
    return tuple(out)


def tree_leaves(parent, depth, rank) -> int:
    p, d, r = _i32(parent), _i32(depth), _i32(rank)
    s = load().specmemo_tree_leaves(len(p), p.ctypes.data, d.ctypes.data, r.ctypes.data)
    if s < 0:
        raise SpecmemoError(-3, load().specmemo_last_error().decode())
    return int(s)


def tree_prune(parent, depth, rank, keep: Sequence[int]):
    """Right-to-left pruning with per-level keep counts; (parent, depth, rank) of the kept nodes."""
    p, d, r, k = _i32(parent), _i32(depth), _i32(rank), _i32(keep)
    n = len(p)
    out = [np.zeros(max(n, 1), np.int32) for _ in range(3)]
    m = C.c_int32(0)
    _check(load().specmemo_tree_prune(n, p.ctypes.data, d.ctypes.data, r.ctypes.data, len(k),
                                      k.ctypes.data if len(k) else None, C.addressof(m),
                                      *(a.ctypes.data for a in out)))
    return tuple(a[:m.value].copy() for a in out)


def plan_budget(max_memory: int, base_model_bytes: int, head_bytes: int, layers: int, n_kv: int, head_dim: int,
                vocab: int, elem_bytes: int, batch: int, query_count: int, query_length: int, default_heads: int,
                default_tree) -> dict:
    """Alg. 1 without quantisation: dict(kind, heads, nodes, leaves, kv_bytes, total_bytes)."""
    parent, depth, rank = (_i32(a) for a in default_tree)
    m = _Budget(max_memory, base_model_bytes, head_bytes, layers, n_kv, head_dim, vocab, elem_bytes, batch,
                query_count, query_length, default_heads)
    out = _BudgetPlan()
    _check(load().specmemo_plan_budget(C.byref(m), len(parent), parent.ctypes.data, depth.ctypes.data,
                                       rank.ctypes.data, C.byref(out)))
    return {f: int(getattr(out, f)) for f, _ in _BudgetPlan._fields_}


def plan_tree_sizes(seq_len, seq_cap, default_nodes: int) -> np.ndarray:
    ln, cp = _i32(seq_len), _i32(seq_cap)
    out = np.zeros(max(len(ln), 1), np.int32)
    _check(load().specmemo_plan_tree_sizes(len(ln), ln.ctypes.data, cp.ctypes.data, default_nodes, out.ctypes.data))
    return out[:len(ln)]
