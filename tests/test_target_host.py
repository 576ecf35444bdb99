"""CPU tests of the target's cache, tree attention and distributions: struct layouts match the header, and bad arguments are reported
before anything touches a device."""
import os
import re

import pytest

from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import verify as VF

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "ps_verify.h")


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2410_05589_amd.build import build_library
        build_library(verbose=False)
    return B.load_library()


@pytest.mark.parametrize("name", ["ps_cache", "ps_cache_write_args", "ps_cache_read_args", "ps_tree_attn_args", "ps_target_probs_args"])
def test_struct_layouts_match_header(name):
    code = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = code[code.index("typedef struct %s {" % name) + len("typedef struct %s {" % name):code.index("} %s;" % name)]
    names = [n for line in re.findall(r"[^;{]+;", body) for n in re.findall(r"\*?\s*([a-z_]+)\s*[,;]", line)]
    assert names == [f[0] for f in getattr(VF, name)._fields_]
    for macro in ("PS_CACHE_BLOCK", "PS_CACHE_MAX_BATCH"):
        assert int(re.search(r"#define %s (\d+)" % macro, code).group(1)) == getattr(VF, macro)


def _cache(offsets=(0, 64, 160), heads=2, d=64, **kw):
    c = VF.make_cache(heads, d, 0x10000, 0x20000, 0x30000, 0x40000, offsets)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _set(a, pointers, kw):
    for n in pointers:
        setattr(a, n, 0x100000)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _write(cache=None, rows=5, kv_len=(0, 40), n_seq=None, dtype="bf16", **kw):
    return _set(VF.make_cache_write_args(cache or _cache(), rows, dtype, kv_len, n_seq), ("k_rows", "v_rows"), kw)


def _read(cache=None, rows=5, start=(0, 40), n_seq=None, dtype="bf16", **kw):
    return _set(VF.make_cache_read_args(cache or _cache(), rows, dtype, start, n_seq), ("k_rows", "v_rows"), kw)


def _attn(cache=None, n_heads=4, kv_len=(64, 70), dtype="bf16", **kw):
    return _set(VF.make_tree_attn_args(cache or _cache(), n_heads, dtype, kv_len), ("q", "k_rows", "v_rows", "out", "workspace"), kw)


TREE = VF.make_tree([-1, 0, 0, 1])

BAD_CACHES = [
    (B.PS_ERR_NULL, dict(k_codes=None)), (B.PS_ERR_NULL, dict(v_codes=None)), (B.PS_ERR_NULL, dict(k_scale=None)),
    (B.PS_ERR_NULL, dict(v_scale=None)), (B.PS_ERR_NULL, dict(kv_offsets=None)),
    (B.PS_ERR_SHAPE, dict(heads=0)), (B.PS_ERR_SHAPE, dict(d=0)), (B.PS_ERR_UNSUPPORTED, dict(d=32)), (B.PS_ERR_UNSUPPORTED, dict(d=96)),
    (B.PS_ERR_UNSUPPORTED, dict(d=256)), (B.PS_ERR_OFFSETS, dict(offsets=(0, 64, 161))), (B.PS_ERR_OFFSETS, dict(offsets=(16, 64, 160))),
    (B.PS_ERR_OFFSETS, dict(offsets=(0, 160, 64))), (B.PS_ERR_OFFSETS, dict(offsets=(-32, 64, 160))),
    (B.PS_ERR_UNSUPPORTED, dict(offsets=(0, 64, 1 << 37))), (B.PS_ERR_UNSUPPORTED, dict(k_codes=0x10008)),
    (B.PS_ERR_UNSUPPORTED, dict(v_scale=0x40002)), (B.PS_ERR_UNSUPPORTED, dict(heads=2048)),
]


@pytest.mark.parametrize("status,kw", BAD_CACHES)
def test_bad_caches_are_refused(status, kw):
    assert VF.ps_cache_write(_write(_cache(**kw)), None) == status
    assert VF.ps_cache_read(_read(_cache(**kw)), None) == status
    n_heads = 4 * kw.get("heads", 1) if kw.get("heads", 1) < 64 else 4096
    assert VF.ps_tree_attention(TREE, _attn(_cache(**kw), n_heads=max(n_heads, 4)), None) == status


def test_a_batch_beyond_the_limit_is_refused():
    many = _cache(offsets=[32 * i for i in range(66)])
    assert VF.ps_cache_write(_write(many, kv_len=[0] * 65, rows=1), None) == B.PS_ERR_UNSUPPORTED
    assert VF.ps_cache_read(_read(many, start=[0] * 65, rows=1), None) == B.PS_ERR_UNSUPPORTED
    assert VF.ps_tree_attention(TREE, _attn(many, kv_len=[0] * 65), None) == B.PS_ERR_UNSUPPORTED
    a = _write()
    a.batch = 0
    assert VF.ps_cache_write(a, None) == B.PS_ERR_SHAPE


@pytest.mark.parametrize("status,kw", [
    (B.PS_ERR_NULL, dict(k_rows=None)), (B.PS_ERR_NULL, dict(v_rows=None)), (B.PS_ERR_NULL, dict(kv_len=None)),
    (B.PS_ERR_NULL, dict(n_accepted=0x1000, path_rows=3)), (B.PS_ERR_NULL, dict(path=0x1000, path_rows=3)),
    (B.PS_ERR_SHAPE, dict(rows=0)), (B.PS_ERR_SHAPE, dict(dtype=7)), (B.PS_ERR_SHAPE, dict(kv_len=(-1, 0))),
    (B.PS_ERR_SHAPE, dict(n_seq=(5, 6))), (B.PS_ERR_SHAPE, dict(n_seq=(-1, 5))),
    (B.PS_ERR_SHAPE, dict(n_accepted=0x1000, path=0x1000, path_rows=0)), (B.PS_ERR_SHAPE, dict(n_accepted=0x1000, path=0x1000, path_rows=64)),
    (B.PS_ERR_SHAPE, dict(n_accepted=0x1000, path=0x1000, path_rows=3, n_seq=(1, 1))),
    (B.PS_ERR_SHAPE, dict(row_stride=127)), (B.PS_ERR_UNSUPPORTED, dict(row_stride=129)), (B.PS_ERR_UNSUPPORTED, dict(k_rows=0x100002)),
    (B.PS_ERR_UNSUPPORTED, dict(kv_len_dev=0x1001)), (B.PS_ERR_UNSUPPORTED, dict(len_out=0x1002)),
    (B.PS_ERR_KV_CAPACITY, dict(kv_len=(60, 40))), (B.PS_ERR_KV_CAPACITY, dict(kv_len=(0, 92))),
    (B.PS_ERR_KV_CAPACITY, dict(kv_len=(0, 2 ** 31 - 1))), (B.PS_ERR_KV_CAPACITY, dict(kv_len=(61, 0), n_accepted=0x1000, path=0x1000, path_rows=3)),
])
def test_bad_writes_are_refused(status, kw):
    assert VF.ps_cache_write(None, None) == B.PS_ERR_NULL
    if kw.get("kv_len", 0) is None:
        a = _write()
        a.kv_len = None
    else:
        a = _write(**kw)
    assert VF.ps_cache_write(a, None) == status


@pytest.mark.parametrize("status,kw", [
    (B.PS_ERR_NULL, dict(k_rows=None, v_rows=None)), (B.PS_ERR_SHAPE, dict(rows=0)), (B.PS_ERR_SHAPE, dict(start=(-1, 0))),
    (B.PS_ERR_SHAPE, dict(n_seq=(1, 6))), (B.PS_ERR_SHAPE, dict(dtype=-1)), (B.PS_ERR_SHAPE, dict(row_stride=64)),
    (B.PS_ERR_KV_CAPACITY, dict(start=(60, 0))), (B.PS_ERR_KV_CAPACITY, dict(start=(0, 2 ** 31 - 1))), (B.PS_ERR_UNSUPPORTED, dict(v_rows=0x100001)),
])
def test_bad_reads_are_refused(status, kw):
    assert VF.ps_cache_read(None, None) == B.PS_ERR_NULL
    assert VF.ps_cache_read(_read(**kw), None) == status


@pytest.mark.parametrize("status,kw", [
    (B.PS_ERR_NULL, dict(q=None)), (B.PS_ERR_NULL, dict(out=None)), (B.PS_ERR_NULL, dict(k_rows=None)), (B.PS_ERR_NULL, dict(v_rows=None)),
    (B.PS_ERR_SHAPE, dict(n_heads=3)), (B.PS_ERR_SHAPE, dict(n_heads=0)), (B.PS_ERR_SHAPE, dict(dtype=2)), (B.PS_ERR_SHAPE, dict(scale=-1.0)),
    (B.PS_ERR_SHAPE, dict(scale=float("nan"))), (B.PS_ERR_SHAPE, dict(scale=float("inf"))), (B.PS_ERR_SHAPE, dict(kv_len=(-1, 0))),
    (B.PS_ERR_SHAPE, dict(q_stride=255)), (B.PS_ERR_SHAPE, dict(kv_stride=127)), (B.PS_ERR_UNSUPPORTED, dict(q_stride=257)),
    (B.PS_ERR_UNSUPPORTED, dict(n_heads=2048)), (B.PS_ERR_UNSUPPORTED, dict(scale=2.0 ** -21)), (B.PS_ERR_UNSUPPORTED, dict(scale=2.0 ** 21)), (B.PS_ERR_UNSUPPORTED, dict(out=0x100002)), (B.PS_ERR_UNSUPPORTED, dict(lse=0x100001)),
    (B.PS_ERR_KV_CAPACITY, dict(kv_len=(65, 0))), (B.PS_ERR_KV_CAPACITY, dict(kv_len=(0, 97))),
])
def test_bad_attention_calls_are_refused(status, kw):
    assert VF.ps_tree_attention(TREE, None, None) == B.PS_ERR_NULL
    assert VF.ps_tree_attention(None, _attn(), None) == B.PS_ERR_NULL
    assert VF.ps_tree_attention(TREE, _attn(**kw), None) == status


def test_bad_trees_are_refused():
    for parent in ([0, 0], [-1, 1], [-1, -1], [-1, 0, 3], [-1] + [0] * 64, []):
        assert VF.ps_tree_attention(VF.make_tree(parent), _attn(), None) == B.PS_ERR_SHAPE, parent
        assert VF.ps_tree_attention_workspace_bytes(VF.make_tree(parent), _attn()) == 0


def test_attention_workspace():
    long = _cache(offsets=(0, 32768, 65536), heads=8, d=128)
    a = _attn(long, n_heads=32, kv_len=(32768, 100))
    need = VF.ps_tree_attention_workspace_bytes(TREE, a)
    assert need > 0 and need % 256 == 0
    a.workspace_bytes = need - 1
    assert VF.ps_tree_attention(TREE, a, None) == B.PS_ERR_WORKSPACE
    a.workspace_bytes, a.workspace = need, 0x100010
    assert VF.ps_tree_attention(TREE, a, None) == B.PS_ERR_WORKSPACE
    a.workspace = None
    assert VF.ps_tree_attention(TREE, a, None) == B.PS_ERR_NULL
    # what it needs grows with the lengths that a call may have, not with what lies in device memory
    assert VF.ps_tree_attention_workspace_bytes(TREE, _attn(long, n_heads=32, kv_len=(0, 0))) == 0


def _probs(batch=2, rows=3, vocab=100, dtype=B.PS_F32, **kw):
    a = VF.ps_target_probs_args()
    a.batch, a.rows, a.vocab, a.dtype = batch, rows, vocab, dtype
    return _set(a, ("logits", "probs", "ids", "r"), kw)


def test_distribution_workspace():
    need = VF.ps_target_probs_workspace_bytes(_probs(batch=8, rows=1, vocab=128256))
    assert need > 0 and need % 256 == 0                      # (several workgroups per row)
    assert VF.ps_target_probs_workspace_bytes(_probs(batch=8, rows=61, vocab=128256)) == 0 == VF.ps_target_probs_workspace_bytes(_probs(vocab=32000))
    assert VF.ps_target_probs_workspace_bytes(_probs(vocab=0)) == 0
    a = _probs(batch=8, rows=1, vocab=128256, workspace=0x100000, workspace_bytes=need - 1)
    assert VF.ps_target_probs(a, None) == B.PS_ERR_WORKSPACE
    a.workspace_bytes, a.workspace = need, 0x100080
    assert VF.ps_target_probs(a, None) == B.PS_ERR_WORKSPACE
    a.workspace = None
    assert VF.ps_target_probs(a, None) == B.PS_ERR_NULL


@pytest.mark.parametrize("status,kw", [
    (B.PS_ERR_NULL, dict(logits=None)), (B.PS_ERR_NULL, dict(probs=None, ids=None)), (B.PS_ERR_NULL, dict(r=None)),
    (B.PS_ERR_NULL, dict(ids=None, id_probs=0x1000)), (B.PS_ERR_SHAPE, dict(batch=0)), (B.PS_ERR_SHAPE, dict(rows=0)), (B.PS_ERR_SHAPE, dict(vocab=0)),
    (B.PS_ERR_SHAPE, dict(dtype=3)), (B.PS_ERR_UNSUPPORTED, dict(vocab=(1 << 20) + 1)), (B.PS_ERR_UNSUPPORTED, dict(batch=1 << 12, rows=1 << 9)),
    (B.PS_ERR_UNSUPPORTED, dict(logits=0x100002)), (B.PS_ERR_UNSUPPORTED, dict(logits=0x100001, dtype=B.PS_BF16)),
    (B.PS_ERR_UNSUPPORTED, dict(probs=0x100002)), (B.PS_ERR_UNSUPPORTED, dict(top_k=0x1001)), (B.PS_ERR_UNSUPPORTED, dict(id_probs=0x1003)),
])
def test_bad_distribution_calls_are_refused(status, kw):
    assert VF.ps_target_probs(None, None) == B.PS_ERR_NULL
    assert VF.ps_target_probs(_probs(**kw), None) == status
