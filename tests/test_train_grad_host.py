"""CPU tests of the entry points of the training layout's embeddings, gradients and loss: struct layouts, refusals on the host, sizes of
workspaces."""
import os
import re

import pytest

from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import train as TR

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2410_05589_amd.build import build_library
        build_library(verbose=False)
    return B.load_library()


@pytest.mark.parametrize("name", ["ps_group_attn_grad_args", "ps_group_embed_args", "ps_group_embed_grad_args", "ps_vocab_loss_args"])
def test_struct_layouts_match_the_header(name):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ps_train.h")).read(), flags=re.S)
    body = text[text.index("typedef struct %s {" % name):text.index("} %s;" % name)]
    names = [n for line in re.findall(r"[^;{]+;", body) for n in re.findall(r"\*?\s*([a-z_]+)\s*[,;]", line)]
    assert names == [f[0] for f in getattr(TR, name)._fields_]


def _filled(a, **kw):
    for n, t in a._fields_:
        if t is TR.ctypes.c_void_p:
            setattr(a, n, 0x100000)
    if hasattr(a, "workspace_bytes"):
        a.workspace_bytes = 1 << 40
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def _attn(**kw):
    return _filled(TR.make_grad_args(1, 64, 4, 8, 8, 64, "bf16", 10000.0), **kw)


def _embed(**kw):
    return _filled(TR.make_embed_args(2, 30, 4, 64, 100, "bf16", 1.0), **kw)


def _embed_grad(**kw):
    return _filled(TR.make_embed_grad_args(2, 30, 4, 64, 100, "bf16", 1.0), **kw)


def _loss(**kw):
    return _filled(TR.make_loss_args(30, 64, 100, "bf16"), **kw)


CALLS = [
    (_attn, TR.ps_group_attention_grad, TR.ps_group_attention_grad_workspace_bytes, ("q", "k_", "v", "out", "lse", "d_out", "d_q", "d_k", "d_v", "workspace")),
    (_embed, TR.ps_group_embed, None, ("token_ids", "embed", "mask_emb", "x")),
    (_embed_grad, TR.ps_group_embed_grad, TR.ps_group_embed_grad_workspace_bytes, ("token_ids", "d_x", "workspace")),
    (_loss, TR.ps_vocab_loss, TR.ps_vocab_loss_workspace_bytes, ("h", "w_lm", "targets", "loss", "workspace")),
]
REFUSED = {
    _attn: (B.PS_ERR_SHAPE, [dict(seqs=0), dict(tokens=0), dict(k=-1), dict(n_kv_heads=3), dict(n_heads=0), dict(dtype=5), dict(rope_base=0.0), dict(rope_base=float("nan"))],
            [dict(head_dim=96), dict(k=16), dict(tokens=1 << 20), dict(seqs=65536)]),
    _embed: (B.PS_ERR_SHAPE, [dict(seqs=0), dict(tokens=-3), dict(k=-1), dict(hidden=0), dict(vocab=0), dict(dtype=2), dict(scale=float("inf")), dict(scale=float("nan"))],
             [dict(hidden=48), dict(hidden=1 << 17), dict(k=16), dict(seqs=1 << 12, tokens=1025), dict(vocab=(1 << 23) + 1), dict(x=0x100002), dict(embed=0x100001),
              dict(token_ids=0x100002)]),
    _embed_grad: (B.PS_ERR_SHAPE, [dict(seqs=0), dict(tokens=0), dict(k=-1), dict(hidden=0), dict(vocab=-1), dict(dtype=2), dict(scale=float("nan"))],
                  [dict(hidden=48), dict(k=16), dict(seqs=1 << 16, tokens=1 << 16), dict(vocab=1 << 24), dict(d_x=0x100002), dict(d_mask=0x100002)]),
    _loss: (B.PS_ERR_SHAPE, [dict(rows=0), dict(hidden=0), dict(vocab=0), dict(rows=-1), dict(dtype=-1)],
            [dict(hidden=48), dict(hidden=1 << 17), dict(vocab=(1 << 23) + 1), dict(rows=(1 << 22) + 1), dict(h=0x100008), dict(w_lm=0x100004), dict(d_hidden=0x100008),
             dict(loss=0x100002), dict(targets=0x100002), dict(weights=0x100001)]),
}


@pytest.mark.parametrize("make,call,need,pointers", CALLS)
def test_refusals(lib, make, call, need, pointers):
    assert call(None, None) == B.PS_ERR_NULL
    shape, sizes, unsupported = REFUSED[make]
    for kw in sizes:
        assert call(make(**kw), None) == shape, kw
    for kw in unsupported:
        assert call(make(**kw), None) == B.PS_ERR_UNSUPPORTED, kw
    for n in pointers:
        assert call(make(**{n: None}), None) == B.PS_ERR_NULL, n
    if need is None:
        return
    assert need(None) == 0
    for kw in sizes:
        assert need(make(**kw)) == 0, kw
    total = need(make())
    assert total > 0 and total % 256 == 0
    assert call(make(workspace_bytes=total - 1), None) == B.PS_ERR_WORKSPACE
    assert call(make(workspace=0x100080), None) == B.PS_ERR_WORKSPACE


def test_outputs_that_are_not_wanted(lib):
    assert TR.ps_group_embed_grad(_embed_grad(d_embed=None, d_mask=None), None) == B.PS_ERR_NULL
    assert TR.ps_group_embed_grad(_embed_grad(d_embed=None, k=0), None) == B.PS_ERR_NULL
    with_grad, without = (TR.ps_vocab_loss_workspace_bytes(_loss(rows=5000, hidden=4096, vocab=32000, d_hidden=d)) for d in (0x100000, None))
    assert 0 < without < with_grad


def test_forward_pass_for_training(lib):
    a = _filled(TR.make_args(1, 64, 4, 8, 8, 64, "bf16", 10000.0))
    assert TR.ps_group_attention_lse(None, 0x100000, None) == B.PS_ERR_NULL
    assert TR.ps_group_attention_lse(a, None, None) == B.PS_ERR_NULL
    a.k = 16
    assert TR.ps_group_attention_lse(a, 0x100000, None) == B.PS_ERR_UNSUPPORTED


def test_workspaces_stay_small_beside_what_they_work_on(lib):
    """The loss keeps a piece of the vocabulary's exponentials, not the logits; the attention's gradient nothing of rows x rows."""
    logits = 40960 * 128256 * 4
    assert TR.ps_vocab_loss_workspace_bytes(_loss(rows=40960, hidden=4096, vocab=128256)) < logits // 20
    q = 32 * 128 * 2
    for T in (2048, 65536):
        a = _attn(tokens=T, n_heads=32, n_kv_heads=32, head_dim=128)
        assert TR.ps_group_attention_grad_workspace_bytes(a) < 4 * T * 5 * q


def test_attention_gradient_launches_fit_the_grid(lib):
    """Threads along a side of a grid are counted in 32 bits: the largest layouts are taken, larger ones refused before anything is launched."""
    most = dict(tokens=(1 << 20) - 15, k=15, n_kv_heads=1, head_dim=64)
    assert TR.ps_group_attention_grad_workspace_bytes(_attn(n_heads=64, **most)) > 1 << 36
    few = dict(tokens=1, k=4, head_dim=64)
    assert TR.ps_group_attention_grad_workspace_bytes(_attn(seqs=65535, n_heads=32, n_kv_heads=32, **few)) > 0
    for kw in (dict(n_heads=160, **most), dict(seqs=65535, n_heads=128, n_kv_heads=128, **few), dict(seqs=65535, n_heads=65535, n_kv_heads=65535, **few)):
        assert TR.ps_group_attention_grad_workspace_bytes(_attn(**kw)) == 0
        assert TR.ps_group_attention_grad(_attn(**kw), None) == B.PS_ERR_UNSUPPORTED


@pytest.mark.parametrize("grad", [None, 0x100000])
def test_loss_launches_fit_the_grid(lib, grad):
    """The threads of a launch are counted in 32 bits, 512 for a tile of 256 x 256: the sizes that are taken stay within."""
    from paper_2410_05589_amd import debug as DBG
    for rows in (1, 97, 65536, 1 << 22):
        for hidden in (32, 256, 288, 4096, 1 << 16):
            for vocab in (1, 32000, 128256, (1 << 23) - 300, 1 << 23):
                st, plan = DBG.ps_train_debug_loss_plan(_loss(rows=rows, hidden=hidden, vocab=vocab, d_hidden=grad))
                assert st == B.PS_OK
                if plan["tile"] == 256:
                    assert plan["workgroups"] * 512 < 1 << 32, (rows, hidden, vocab, plan)
    assert DBG.ps_train_debug_loss_plan(_loss(vocab=(1 << 23) + 1))[0] == B.PS_ERR_UNSUPPORTED
