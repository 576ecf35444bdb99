"""ctypes binding of group-wise parallel training (include/ps_train.h: embeddings, attention, loss and their gradients): same
names as the C ABI, argument marshalling only; the work runs in the HIP library."""
import ctypes

from . import binding as B

EXPORTED_SYMBOLS = ("ps_group_attention_workspace_bytes", "ps_group_attention", "ps_group_attention_lse",
                    "ps_group_attention_grad_workspace_bytes", "ps_group_attention_grad", "ps_group_embed",
                    "ps_group_embed_grad_workspace_bytes", "ps_group_embed_grad", "ps_vocab_loss_workspace_bytes", "ps_vocab_loss")


class ps_group_attn_args(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int32), ("tokens", ctypes.c_int32), ("k", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("rope_base", ctypes.c_float),
                ("q", ctypes.c_void_p), ("k_", ctypes.c_void_p), ("v", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class ps_group_attn_grad_args(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int32), ("tokens", ctypes.c_int32), ("k", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("rope_base", ctypes.c_float),
                ("q", ctypes.c_void_p), ("k_", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("d_out", ctypes.c_void_p),
                ("d_q", ctypes.c_void_p), ("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class ps_group_embed_args(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int32), ("tokens", ctypes.c_int32), ("k", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("token_ids", ctypes.c_void_p), ("embed", ctypes.c_void_p), ("mask_emb", ctypes.c_void_p), ("x", ctypes.c_void_p)]


class ps_group_embed_grad_args(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int32), ("tokens", ctypes.c_int32), ("k", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("token_ids", ctypes.c_void_p), ("d_x", ctypes.c_void_p), ("d_embed", ctypes.c_void_p), ("d_mask", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class ps_vocab_loss_args(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("hidden", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("h", ctypes.c_void_p), ("w_lm", ctypes.c_void_p), ("targets", ctypes.c_void_p), ("weights", ctypes.c_void_p),
                ("loss", ctypes.c_void_p), ("d_hidden", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


_ready = False


def _lib():
    global _ready
    lib = B.load_library()
    if not _ready:
        for name, args in (("ps_group_attention", ps_group_attn_args), ("ps_group_attention_grad", ps_group_attn_grad_args),
                           ("ps_group_embed", ps_group_embed_args), ("ps_group_embed_grad", ps_group_embed_grad_args),
                           ("ps_vocab_loss", ps_vocab_loss_args)):
            call = getattr(lib, name)
            call.restype = ctypes.c_int
            call.argtypes = [ctypes.POINTER(args), ctypes.c_void_p]
            if name != "ps_group_embed":                      # (the one that needs no workspace)
                need = getattr(lib, name + "_workspace_bytes")
                need.restype = ctypes.c_size_t
                need.argtypes = [ctypes.POINTER(args)]
        lib.ps_group_attention_lse.restype = ctypes.c_int
        lib.ps_group_attention_lse.argtypes = [ctypes.POINTER(ps_group_attn_args), ctypes.c_void_p, ctypes.c_void_p]
        _ready = True
    return lib


def _dtype(dtype):
    return B.PS_BF16 if dtype == "bf16" else B.PS_F32


def _ref(args):
    return ctypes.byref(args) if args is not None else None


def _attention_args(a, seqs, tokens, k, n_heads, n_kv_heads, head_dim, dtype, rope_base):
    a.seqs, a.tokens, a.k = seqs, tokens, k
    a.n_heads, a.n_kv_heads, a.head_dim = n_heads, n_kv_heads, head_dim
    a.dtype = _dtype(dtype)
    a.rope_base = rope_base
    return a


def make_args(seqs, tokens, k, n_heads, n_kv_heads, head_dim, dtype, rope_base):
    return _attention_args(ps_group_attn_args(), seqs, tokens, k, n_heads, n_kv_heads, head_dim, dtype, rope_base)


def make_grad_args(seqs, tokens, k, n_heads, n_kv_heads, head_dim, dtype, rope_base):
    return _attention_args(ps_group_attn_grad_args(), seqs, tokens, k, n_heads, n_kv_heads, head_dim, dtype, rope_base)


def _embed_args(a, seqs, tokens, k, hidden, vocab, dtype, scale):
    a.seqs, a.tokens, a.k = seqs, tokens, k
    a.hidden, a.vocab = hidden, vocab
    a.dtype = _dtype(dtype)
    a.scale = scale
    return a


def make_embed_args(seqs, tokens, k, hidden, vocab, dtype, scale=1.0):
    return _embed_args(ps_group_embed_args(), seqs, tokens, k, hidden, vocab, dtype, scale)


def make_embed_grad_args(seqs, tokens, k, hidden, vocab, dtype, scale=1.0):
    return _embed_args(ps_group_embed_grad_args(), seqs, tokens, k, hidden, vocab, dtype, scale)


def make_loss_args(rows, hidden, vocab, dtype):
    a = ps_vocab_loss_args()
    a.rows, a.hidden, a.vocab = rows, hidden, vocab
    a.dtype = _dtype(dtype)
    return a


def ps_group_attention_workspace_bytes(args):
    return int(_lib().ps_group_attention_workspace_bytes(_ref(args)))


def ps_group_attention(args, stream_ptr):
    return _lib().ps_group_attention(_ref(args), stream_ptr)


def ps_group_attention_lse(args, lse_ptr, stream_ptr):
    return _lib().ps_group_attention_lse(_ref(args), lse_ptr, stream_ptr)


def ps_group_attention_grad_workspace_bytes(args):
    return int(_lib().ps_group_attention_grad_workspace_bytes(_ref(args)))


def ps_group_attention_grad(args, stream_ptr):
    return _lib().ps_group_attention_grad(_ref(args), stream_ptr)


def ps_group_embed(args, stream_ptr):
    return _lib().ps_group_embed(_ref(args), stream_ptr)


def ps_group_embed_grad_workspace_bytes(args):
    return int(_lib().ps_group_embed_grad_workspace_bytes(_ref(args)))


def ps_group_embed_grad(args, stream_ptr):
    return _lib().ps_group_embed_grad(_ref(args), stream_ptr)


def ps_vocab_loss_workspace_bytes(args):
    return int(_lib().ps_vocab_loss_workspace_bytes(_ref(args)))


def ps_vocab_loss(args, stream_ptr):
    return _lib().ps_vocab_loss(_ref(args), stream_ptr)
