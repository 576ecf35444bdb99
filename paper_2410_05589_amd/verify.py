"""ctypes binding of the entry points around a verification (include/ps_verify.h): tree construction, acceptance walk, the
target's 8-bit cache, tree attention over it, its distributions.  Same names as the C ABI, argument marshalling only; the
work runs in the HIP library."""
import ctypes

import numpy as np

from . import binding as B

PS_TREE_MAX_NODES = 64
PS_CACHE_BLOCK = 32
PS_CACHE_MAX_BATCH = 64
EXPORTED_SYMBOLS = ("ps_tree_tokens", "ps_verify_walk", "ps_verify_workspace_bytes", "ps_verify_walk_static",
                    "ps_cache_write", "ps_cache_read", "ps_tree_attention", "ps_tree_attention_workspace_bytes",
                    "ps_target_probs", "ps_target_probs_workspace_bytes")


class ps_tree_shape(ctypes.Structure):
    _fields_ = [("n_nodes", ctypes.c_int32), ("parent", ctypes.POINTER(ctypes.c_int32)),
                ("rank", ctypes.POINTER(ctypes.c_int32))]


class ps_verify_args(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("rows", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("tokens", ctypes.c_void_p), ("q", ctypes.c_void_p), ("p", ctypes.c_void_p), ("r", ctypes.c_void_p),
                ("n_accepted", ctypes.c_void_p), ("path", ctypes.c_void_p),
                ("out_tokens", ctypes.c_void_p), ("top_ids", ctypes.c_void_p), ("topk", ctypes.c_int32),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class ps_cache(ctypes.Structure):
    _fields_ = [("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("kv_offsets", ctypes.POINTER(ctypes.c_int64))]


class ps_cache_write_args(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("rows", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("cache", ctypes.POINTER(ps_cache)), ("k_rows", ctypes.c_void_p), ("v_rows", ctypes.c_void_p),
                ("row_stride", ctypes.c_int64), ("kv_len", ctypes.POINTER(ctypes.c_int32)), ("kv_len_dev", ctypes.c_void_p),
                ("n_seq", ctypes.POINTER(ctypes.c_int32)), ("n_accepted", ctypes.c_void_p), ("path", ctypes.c_void_p),
                ("path_rows", ctypes.c_int32), ("len_out", ctypes.c_void_p)]


class ps_cache_read_args(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("rows", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("cache", ctypes.POINTER(ps_cache)), ("k_rows", ctypes.c_void_p), ("v_rows", ctypes.c_void_p),
                ("row_stride", ctypes.c_int64), ("start", ctypes.POINTER(ctypes.c_int32)),
                ("n_seq", ctypes.POINTER(ctypes.c_int32))]


class ps_tree_attn_args(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("cache", ctypes.POINTER(ps_cache)), ("q", ctypes.c_void_p), ("k_rows", ctypes.c_void_p),
                ("v_rows", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("kv_stride", ctypes.c_int64),
                ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("kv_len", ctypes.POINTER(ctypes.c_int32)),
                ("kv_len_dev", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class ps_target_probs_args(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("logits", ctypes.c_void_p), ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p),
                ("top_p", ctypes.c_void_p), ("min_p", ctypes.c_void_p), ("r", ctypes.c_void_p), ("probs", ctypes.c_void_p),
                ("ids", ctypes.c_void_p), ("id_probs", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


_ready = False


def _lib():
    global _ready
    lib = B.load_library()
    if not _ready:
        lib.ps_tree_tokens.restype = ctypes.c_int
        lib.ps_tree_tokens.argtypes = [ctypes.POINTER(ps_tree_shape), ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        lib.ps_verify_walk.restype = ctypes.c_int
        lib.ps_verify_walk.argtypes = [ctypes.POINTER(ps_tree_shape), ctypes.POINTER(ps_verify_args), ctypes.c_void_p]
        lib.ps_verify_walk_static.restype = ctypes.c_int
        lib.ps_verify_walk_static.argtypes = lib.ps_verify_walk.argtypes
        lib.ps_verify_workspace_bytes.restype = ctypes.c_size_t
        lib.ps_verify_workspace_bytes.argtypes = [ctypes.c_int32, ctypes.c_int32]
        for name, args in (("ps_cache_write", ps_cache_write_args), ("ps_cache_read", ps_cache_read_args),
                           ("ps_target_probs", ps_target_probs_args)):
            call = getattr(lib, name)
            call.restype = ctypes.c_int
            call.argtypes = [ctypes.POINTER(args), ctypes.c_void_p]
        lib.ps_tree_attention.restype = ctypes.c_int
        lib.ps_tree_attention.argtypes = [ctypes.POINTER(ps_tree_shape), ctypes.POINTER(ps_tree_attn_args), ctypes.c_void_p]
        lib.ps_tree_attention_workspace_bytes.restype = ctypes.c_size_t
        lib.ps_tree_attention_workspace_bytes.argtypes = [ctypes.POINTER(ps_tree_shape), ctypes.POINTER(ps_tree_attn_args)]
        lib.ps_target_probs_workspace_bytes.restype = ctypes.c_size_t
        lib.ps_target_probs_workspace_bytes.argtypes = [ctypes.POINTER(ps_target_probs_args)]
        _ready = True
    return lib


def make_tree(parent, rank=None):
    """ps_tree_shape over host arrays (kept alive by the returned object)."""
    parent = np.ascontiguousarray(parent, dtype=np.int32)
    t = ps_tree_shape()
    t.n_nodes = len(parent)
    t._parent = parent
    t.parent = parent.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    if rank is not None:
        rank = np.ascontiguousarray(rank, dtype=np.int32)
        assert len(rank) == len(parent)
        t._rank = rank
        t.rank = rank.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    return t


def ps_tree_tokens(tree, batch, rows, topk, top_ids_ptr, tokens_ptr, stream_ptr):
    return _lib().ps_tree_tokens(ctypes.byref(tree) if tree is not None else None, batch, rows, topk,
                                 top_ids_ptr, tokens_ptr, stream_ptr)


def ps_verify_walk(tree, args, stream_ptr):
    return _lib().ps_verify_walk(ctypes.byref(tree) if tree is not None else None,
                                 ctypes.byref(args) if args is not None else None, stream_ptr)


def ps_verify_walk_static(tree, args, stream_ptr):
    return _lib().ps_verify_walk_static(ctypes.byref(tree) if tree is not None else None,
                                        ctypes.byref(args) if args is not None else None, stream_ptr)


def ps_verify_workspace_bytes(batch, vocab):
    return int(_lib().ps_verify_workspace_bytes(batch, vocab))


def _ints(values, kind=ctypes.c_int32):
    """A host array (kept alive by the structure that it is assigned to), or None."""
    return None if values is None else (kind * len(values))(*[int(v) for v in values])


def _ref(args):
    return ctypes.byref(args) if args is not None else None


def _dtype(dtype):
    return {"bf16": B.PS_BF16, "f32": B.PS_F32}.get(dtype, dtype)


def make_cache(n_kv_heads, head_dim, k_codes_ptr, v_codes_ptr, k_scale_ptr, v_scale_ptr, kv_offsets):
    """ps_cache over device pointers and a copy of the host's kv_offsets."""
    c = ps_cache()
    c.n_kv_heads, c.head_dim = n_kv_heads, head_dim
    c.k_codes, c.v_codes, c.k_scale, c.v_scale = k_codes_ptr, v_codes_ptr, k_scale_ptr, v_scale_ptr
    c.kv_offsets = _ints(kv_offsets, ctypes.c_int64)
    c._batch = len(kv_offsets) - 1
    return c


def _on_cache(a, cache, dtype):
    a.batch, a.dtype, a.cache = cache._batch, _dtype(dtype), ctypes.pointer(cache)
    return a


def make_cache_write_args(cache, rows, dtype, kv_len, n_seq=None):
    """Sizes and host arrays; the caller sets the device pointers."""
    a = _on_cache(ps_cache_write_args(), cache, dtype)
    a.rows, a.kv_len, a.n_seq = rows, _ints(kv_len), _ints(n_seq)
    return a


def make_cache_read_args(cache, rows, dtype, start=None, n_seq=None):
    a = _on_cache(ps_cache_read_args(), cache, dtype)
    a.rows, a.start, a.n_seq = rows, _ints(start), _ints(n_seq)
    return a


def make_tree_attn_args(cache, n_heads, dtype, kv_len):
    a = _on_cache(ps_tree_attn_args(), cache, dtype)
    a.n_heads, a.kv_len = n_heads, _ints(kv_len)
    return a


def ps_cache_write(args, stream_ptr):
    return _lib().ps_cache_write(_ref(args), stream_ptr)


def ps_cache_read(args, stream_ptr):
    return _lib().ps_cache_read(_ref(args), stream_ptr)


def ps_tree_attention(tree, args, stream_ptr):
    return _lib().ps_tree_attention(_ref(tree), _ref(args), stream_ptr)


def ps_tree_attention_workspace_bytes(tree, args):
    return int(_lib().ps_tree_attention_workspace_bytes(_ref(tree), _ref(args)))


def ps_target_probs(args, stream_ptr):
    return _lib().ps_target_probs(_ref(args), stream_ptr)


def ps_target_probs_workspace_bytes(args):
    return int(_lib().ps_target_probs_workspace_bytes(_ref(args)))
