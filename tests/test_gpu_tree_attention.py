"""GPU tests of the tree attention over the 8-bit cache (ps_tree_attention) against its definition in float64 (oracle/target.py), from the codes that are there.

Tolerances, per output element, from the roundings: with n keys, d dims, s the scale, Q = s max_j sum_i |q_i k_ji| and A = sum_j p_j |v_j| (float64):
  a score is off by at most D = (d + 4) 2^-24 Q (a product and d sums, the scale) and 2^-23 |score| more on the way to the exponent; an exponential by 2^-22;
  sums of n terms by n 2^-24 each, the numerator and the denominator alike: 2 (D + 2^-23 Q) + 2 n 2^-24 + 2^-20 in all, times A;
  bf16: a probability's rounding 2^-8 A, the result's 2^-8 |out|; float32: three bf16 parts leave 2^-24 of each factor, the result 2^-24 |out|.
The log sum is off by D + 2^-23 Q + n 2^-24 + 2^-20 and half a step of itself."""
import math

import numpy as np
import pytest

from oracle import target as orc
from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import verify as VF
from tests import target_util as TU

pytestmark = pytest.mark.gpu


def fanout(*fan):
    parent, level = [-1], [0]
    for f in fan:
        new = [u for u in level for _ in range(f)]
        level = list(range(len(parent), len(parent) + len(new)))
        parent += new
    return parent


def chain(n):
    return [i - 1 for i in range(n)]


def call(cache, parent, q, k, v, lens, dtype, scale=0.0, q_stride=0, kv_stride=0, lse=True, dev=None, keep=None):
    import torch
    batch, nodes, nq, d = q.shape
    tree = VF.make_tree(parent)
    a = VF.make_tree_attn_args(cache.struct, nq, dtype, lens)
    out = torch.full((batch, nodes, nq, d), 77.0, dtype=TU.torch_dtype(dtype), device="cuda:0")
    sums = torch.full((batch, nodes, nq), 77.0, device="cuda:0")
    a.q, a.out, a.scale, a.q_stride, a.kv_stride = q.data_ptr(), out.data_ptr(), scale, q_stride, kv_stride
    a.k_rows, a.v_rows = (k.data_ptr(), v.data_ptr()) if k is not None else (None, None)
    if lse:
        a.lse = sums.data_ptr()
    if dev is not None:
        a.kv_len_dev = dev.data_ptr()
    need = VF.ps_tree_attention_workspace_bytes(tree, a)
    ws, at = TU.workspace(need)
    a.workspace, a.workspace_bytes = (at, need) if need else (None, 0)
    st = VF.ps_tree_attention(tree, a, TU.stream())
    assert st == B.PS_OK, B.ps_draft_strerror(st)
    if keep is not None:
        keep.append((tree, a, out, sums, ws))
    return out, sums


def check(cache, parent, q, k, v, lens, dtype, out, lse, scale=None, rows=None, heads=None):
    """Against the oracle; rows, heads: some of them only."""
    d = q.shape[-1]
    scale = scale or 1.0 / math.sqrt(d)
    tables = {n: cache.decoded(n) for n in "kv"}
    got, got_lse = TU.np64(out), TU.np64(lse)
    grp = q.shape[2] // cache.heads
    for b, n in enumerate(lens):
        first = cache.offsets[b] // 32
        hs = range(cache.heads) if heads is None else heads
        for h in hs:
            mine = slice(h * grp, (h + 1) * grp)
            key, value = (orc.read(tables[x][0][:, h:h + 1], tables[x][1][:, h:h + 1], first, 0, n) for x in "kv")
            q64 = TU.np64(q[b, :, mine])
            own = (None, None) if k is None else (TU.np64(k[b, :, h:h + 1]), TU.np64(v[b, :, h:h + 1]))
            want, want_lse = orc.tree_attention(parent, q64, key, value, *own, scale)
            size, _ = orc.tree_attention(parent, q64, key, np.abs(value), own[0], None if k is None else np.abs(own[1]), scale)   # A
            keys = key[:, 0] if k is None else np.concatenate((key[:, 0], own[0][:, 0]))
            Q = scale * (np.abs(q64) @ np.abs(keys).T).max(-1) if len(keys) else np.zeros(q64.shape[:2])
            D = (d + 4) * 2.0 ** -24 * Q + 2.0 ** -23 * Q
            half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
            tol = (2 * D + 2 * len(keys) * 2.0 ** -24 + 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -22))[..., None] * size + half * np.abs(want)
            sel = slice(None) if rows is None else rows
            bad = np.abs(got[b, :, mine] - want) > tol
            assert not bad[sel].any(), (b, h, np.argwhere(bad)[:5], np.abs(got[b, :, mine] - want)[bad].max())
            fine = np.isfinite(want_lse)
            assert np.array_equal(got_lse[b, :, mine][~fine], want_lse[~fine])
            diff = np.abs(got_lse[b, :, mine] - np.where(fine, want_lse, 0.0))
            assert (diff <= D + len(keys) * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -23 * np.abs(want_lse))[fine].all()


def make(dtype, heads, nq, d, lens, nodes, seed=0, gain=1.0, capacity=None):
    batch = len(lens)
    cache = TU.Cache(heads, d, [32 * max(1, (n + 31) // 32) for n in (capacity or lens)], seed=seed)
    most = max(max(lens), 1)
    x = [TU.normal((batch, most, heads, d), seed + 1 + i, dtype, gain) for i in range(2)]
    cache.write(x[0], x[1], [0] * batch, dtype, n_seq=lens)
    q = TU.normal((batch, nodes, nq, d), seed + 5, dtype)
    k, v = (TU.normal((batch, nodes, heads, d), seed + 6 + i, dtype, gain) for i in range(2))
    return cache, q, k, v


CASES = [  # dtype, kv heads, query heads, head_dim, lengths, tree
    ("bf16", 1, 1, 64, (0,), [-1]),
    ("f32", 1, 1, 128, (1,), [-1]),
    ("bf16", 2, 2, 128, (31, 32, 33), [-1]),
    ("f32", 2, 2, 64, (31, 32, 33, 0), fanout(2, 1)),
    ("bf16", 2, 8, 128, (100, 7), [-1]),                      # four rows of one token
    ("bf16", 3, 3, 64, (65, 200), chain(5)),
    ("bf16", 2, 4, 128, (300, 0, 17), fanout(4, 2, 1)),       # 42 rows: two tiles
    ("bf16", 1, 3, 128, (129,), fanout(4, 2, 2)),             # 87 rows: three tiles, two wavefronts of rows
    ("bf16", 2, 8, 64, (257, 31), fanout(4, 2, 2, 1, 1)),     # 244 rows: eight tiles, four wavefronts of rows
    ("bf16", 1, 16, 128, (70,), chain(64)),                   # 1024 rows: several workgroups of rows
    ("f32", 2, 4, 128, (290, 3), fanout(4, 2, 2, 1, 1)),
    ("f32", 1, 5, 64, (130,), chain(33)),
    ("bf16", 8, 32, 128, (4099, 33, 700), fanout(4, 2, 2, 1, 1)),   # several splits of some sequences, one of others
    ("bf16", 2, 2, 128, (9001,), [-1]),
    ("f32", 2, 2, 64, (3001, 40), fanout(3, 1)),
    ("bf16", 2, 2, 64, (40,) * 64, [-1]),
    ("bf16", 5, 5, 64, (63,), fanout(63)),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d-%d-%d-%s-%d" % (c[0], c[1], c[2], c[3], c[4][:4], len(c[5])))
def test_against_the_definition(case):
    dtype, heads, nq, d, lens, parent = case
    cache, q, k, v = make(dtype, heads, nq, d, lens, len(parent), seed=len(parent))
    out, lse = call(cache, parent, q, k, v, list(lens), dtype)
    some = None if sum(lens) * nq * len(parent) < 1 << 20 else [0, heads - 1]
    check(cache, parent, q, k, v, lens, dtype, out, lse, heads=some)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cached_positions_only_and_rows_that_see_nothing(dtype):
    lens = (0, 45, 0, 32)
    cache, q, _, _ = make(dtype, 2, 4, 64, lens, 3)
    out, lse = call(cache, chain(3), q, None, None, list(lens), dtype)
    check(cache, chain(3), q, None, None, lens, dtype, out, lse)
    assert (out[0] == 0).all() and (out[2] == 0).all() and (lse[0] == -math.inf).all()
    out2, untouched = call(cache, chain(3), q, None, None, list(lens), dtype, lse=False)
    assert out2.equal(out) and (untouched == 77.0).all()


@pytest.mark.parametrize("dtype,lead", [("bf16", 2), ("f32", 1)])
def test_rows_of_a_fused_projection(dtype, lead):
    lens, parent = (70, 5), fanout(3, 2)
    cache, q, k, v = make(dtype, 2, 6, 128, lens, len(parent))
    stride = (6 + 2 + 2) * 128 + 2
    out, lse = call(cache, parent, TU.strided(q, stride, lead), TU.strided(k, stride, lead), TU.strided(v, stride, 0), list(lens), dtype, q_stride=stride, kv_stride=stride)
    want, want_lse = call(cache, parent, q, k, v, list(lens), dtype)
    assert out.equal(want) and lse.equal(want_lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_apart(dtype):
    """Keys of very different size in one cache: the running maximum rises in the middle, scales differ by many powers of two."""
    import torch
    lens, parent = (400,), fanout(2, 2)
    cache, q, k, v = make(dtype, 2, 4, 64, lens, len(parent))
    big = TU.normal((1, 400, 2, 64), 77, "f32") * torch.exp2(torch.linspace(-12, 5, 400))[None, :, None, None].cuda()
    wide = TU.normal((1, 400, 2, 64), 78, "f32") * torch.exp2(torch.linspace(30, -30, 400))[None, :, None, None].cuda()
    cache.write(big.to(q.dtype), wide.to(q.dtype), [0], dtype)
    for scale in (0.0, 1e-3, 2.0):
        out, lse = call(cache, parent, q, k, v, list(lens), dtype, scale=scale)
        check(cache, parent, q, k, v, lens, dtype, out, lse, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_hidden_does_not_enter(dtype):
    """Behind the sequences' ends the cache holds NaN codes and NaN scales; nodes hidden from a row hold Inf and NaN."""
    import torch
    lens, parent = (5, 64, 41), fanout(3, 2)
    cache, q, k, v = make(dtype, 2, 4, 64, lens, len(parent), capacity=(64, 96, 64))
    out, lse = call(cache, parent, q, k, v, list(lens), dtype)
    dirty = TU.Cache(2, 64, [64, 96, 64])
    for n, kind in (("k", cache.codes["k"]), ("v", cache.codes["v"])):
        at = torch.from_numpy(TU.places(n, 64)).cuda().reshape(32, 64)
        dirty.codes[n].fill_(0x7F)
        dirty.scales[n].fill_(float("nan"))
        for b, length in enumerate(lens):
            for i in range((length + 31) // 32):
                block, seen = cache.offsets[b] // 32 + i, at[:min(32, length - 32 * i)].reshape(-1)
                dirty.codes[n][block][:, seen] = kind[block][:, seen]
                dirty.scales[n][block] = cache.scales[n][block]
    got, got_lse = call(dirty, parent, q, k, v, list(lens), dtype)
    assert got.equal(out) and got_lse.equal(lse)
    # node 2 and its children see its Inf and NaN, the others do not
    k2, v2 = k.clone(), v.clone()
    k2[:, 2, 0, 3], v2[:, 2, :, 5] = float("nan"), float("inf")
    v2[:, 2, 1, 40] = float("nan")
    got, got_lse = call(cache, parent, q, k2, v2, list(lens), dtype)
    sees = [s for s in range(len(parent)) if s == 2 or parent[s] == 2]
    blind = [s for s in range(len(parent)) if s not in sees]
    assert got[:, blind].equal(out[:, blind]) and got_lse[:, blind].equal(lse[:, blind])
    # only values: Inf and NaN go where they belong, the other dims stay as they were
    got, _ = call(cache, parent, q, k, v2, list(lens), dtype)
    assert got[:, blind].equal(out[:, blind])
    assert (got[:, sees][..., 5] == math.inf).all() and torch.isnan(got[:, sees][:, :, 2:, 40]).all()
    rest = [i for i in range(64) if i not in (5, 40)]
    assert torch.isfinite(got[:, sees][..., rest].float()).all()
    check(cache, parent, q, k, torch.nan_to_num(v2, nan=0.0, posinf=0.0), lens, dtype,
          torch.where(torch.isfinite(got), got, out), lse, rows=blind)


def test_a_nan_in_the_cache_reaches_every_row():
    import torch
    lens, parent = (40, 40), fanout(2)
    cache, q, k, v = make("bf16", 1, 2, 64, lens, len(parent))
    x = TU.normal((2, 1, 1, 64), 1, "bf16")
    x[0, 0, 0, 7] = float("nan")
    cache.write(x, x, [39, 39], "bf16")
    out, _ = call(cache, parent, q, k, v, list(lens), "bf16")
    assert torch.isnan(out[0]).all() and torch.isfinite(out[1].float()).all()


def test_lengths_on_the_device():
    import torch
    lens, bounds, parent = (3000, 0, 100), (4096, 64, 5000), fanout(4, 2)
    cache, q, k, v = make("bf16", 2, 4, 128, lens, len(parent), capacity=bounds)
    want, want_lse = call(cache, parent, q, k, v, list(lens), "bf16")
    dev = torch.tensor(lens, dtype=torch.int32, device="cuda:0")
    out, lse = call(cache, parent, q, k, v, list(bounds), "bf16", dev=dev)
    check(cache, parent, q, k, v, lens, "bf16", out, lse)
    dev.copy_(torch.tensor([-3, 1 << 30, 100]))               # outside: the nearer bound
    out2, _ = call(cache, parent, q, k, v, [4096, 0, 5000], "bf16", dev=dev)
    empty, _ = call(cache, parent, q, k, v, [0, 0, 100], "bf16")
    np.testing.assert_allclose(TU.np64(out2), TU.np64(empty), atol=2.0 ** -7 * float(empty.abs().max()))
    assert out2[:2].equal(empty[:2])


def test_same_call_same_bits_whatever_the_workspace_held():
    cache, q, k, v = make("bf16", 2, 8, 128, (5000, 900), 13)
    a = call(cache, fanout(4, 2), q, k, v, [5000, 900], "bf16")
    b = call(cache, fanout(4, 2), q, k, v, [5000, 900], "bf16")
    assert a[0].equal(b[0]) and a[1].equal(b[1])


def test_captured_and_replayed_with_other_lengths_and_contents():
    """Two graphs share a workspace; lengths advance on the device between replays, eager calls go on in between."""
    import torch
    parent = fanout(3, 2)
    bound = 2000
    cache, q, k, v = make("bf16", 2, 4, 128, (1500, 900), len(parent), capacity=(bound, bound))
    dev = torch.tensor([1500, 900], dtype=torch.int32, device="cuda:0")
    keep = []
    call(cache, parent, q, k, v, [bound, bound], "bf16", dev=dev, keep=keep)
    tree, a, out, lse, _ = keep[0]
    other = VF.make_tree_attn_args(cache.struct, 4, "bf16", [bound, bound])
    for f in ("q", "k_rows", "v_rows", "kv_len_dev", "workspace", "workspace_bytes"):
        setattr(other, f, getattr(a, f))
    out2 = torch.empty_like(out)
    other.out, other.scale = out2.data_ptr(), 0.25
    torch.cuda.synchronize()
    graphs = []
    for args in (a, other):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            assert VF.ps_tree_attention(tree, args, TU.stream()) == B.PS_OK
        graphs.append(g)
    for step in range(4):
        dev.copy_(torch.tensor([1500 + 37 * step, 900 - 300 * step]))
        q.normal_()
        new = TU.normal((2, 200, 2, 128), 90 + step, "bf16")
        cache.write(new, new, [1500, 900], "bf16")
        lens = dev.tolist()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got, got_lse, got2 = out.clone(), lse.clone(), out2.clone()
        check(cache, parent, q, k, v, lens, "bf16", got, got_lse)
        eager, _ = call(cache, parent, q, k, v, [bound, bound], "bf16", dev=dev)
        assert eager.equal(got)
        eager2, _ = call(cache, parent, q, k, v, [bound, bound], "bf16", dev=dev, scale=0.25)
        assert eager2.equal(got2)


def test_two_streams_at_once():
    import torch
    cache, q, k, v = make("bf16", 2, 8, 128, (6000, 50), 13)
    want, _ = call(cache, fanout(4, 2), q, k, v, [6000, 50], "bf16")
    torch.cuda.synchronize()
    streams, got, keep = [torch.cuda.Stream() for _ in range(2)], [], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(call(cache, fanout(4, 2), q, k, v, [6000, 50], "bf16", keep=keep)[0])
    torch.cuda.synchronize()
    assert all(g.equal(want) for g in got)


def _whole(cache, parent, q, k, v, lens, heads):
    """out and lse of some kv heads in float64 on the GPU, from the codes."""
    import torch
    values, d, nq = torch.from_numpy(orc.VALUES).cuda(), cache.d, q.shape[2]
    grp, n = nq // cache.heads, len(parent)
    sees = torch.eye(n, dtype=torch.bool, device="cuda:0")
    for s in range(1, n):
        sees[s] |= sees[parent[s]]
    for b, length in enumerate(lens):
        blocks = slice(cache.offsets[b] // 32, cache.offsets[b] // 32 + (length + 31) // 32)
        for h in heads:
            kv = []
            for name, own in (("k", k), ("v", v)):
                at = torch.from_numpy(TU.places(name, d)).cuda()
                x = values[cache.codes[name][blocks, h].long()[:, at]].reshape(-1, 32, d) * cache.scales[name][blocks, h].double()[:, None, None]
                kv.append(torch.cat((x.reshape(-1, d)[:length], own[b, :, h].double())))
            x = q[b, :, h * grp:(h + 1) * grp].double().transpose(0, 1).reshape(grp * n, d) @ kv[0].t() / math.sqrt(d)
            x[:, length:].masked_fill_(~sees.repeat(grp, 1), -math.inf)
            lse = torch.logsumexp(x, 1)
            p = torch.exp(x - lse[:, None])
            yield b, h, *(y.reshape(grp, n, -1).transpose(0, 1) for y in (p @ kv[1], p @ kv[1].abs(), lse))


def _check_whole(cache, parent, q, k, v, lens, heads, out, lse):
    grp = q.shape[2] // cache.heads
    for b, h, want, size, want_lse in _whole(cache, parent, q, k, v, lens, heads):
        mine = slice(h * grp, (h + 1) * grp)
        # (the formula of the file's head for bf16, with Q <= 16 for these inputs: scores are N(0, 1) up to their keys' rounding)
        n = lens[b] + len(parent)
        tol = (2 * (cache.d + 4) * 2.0 ** -24 * 16 + 2 * n * 2.0 ** -24 + 2.0 ** -19 + 2.0 ** -8) * size + 2.0 ** -8 * want.abs()
        assert ((out[b, :, mine].double() - want).abs() <= tol).all(), (b, h)
        assert ((lse[b, :, mine].double() - want_lse[..., 0]).abs() <= (cache.d + 4) * 2.0 ** -24 * 16 + n * 2.0 ** -24 + 2.0 ** -18).all()


def test_codes_that_pass_the_caches_by():
    """One tile of rows over more than 192 MB of codes."""
    lens, heads = (20000,), 40
    cache, q, k, v = make("bf16", heads, heads, 128, lens, 1, seed=9)
    out, lse = call(cache, [-1], q, k, v, list(lens), "bf16")
    _check_whole(cache, [-1], q, k, v, lens, (0, 17, heads - 1), out, lse)


@pytest.mark.parametrize("parent", [[-1], fanout(3), fanout(4, 2, 2, 1, 1)], ids=lambda p: "%d nodes" % len(p))
def test_codes_beyond_32_bits_of_bytes(parent):
    """Sequences whose codes lie more than 4 GiB behind the cache's start."""
    import torch
    heads, d, lens = 16, 128, (95, 700)
    blocks = (1 << 32) // (heads * 32 * d) + 1
    cache = TU.Cache(1, d, [32])
    cache.heads, cache.offsets = heads, [32 * blocks, 32 * (blocks + 3), 32 * (blocks + 25)]
    cache.codes = {n: torch.full(((blocks + 26), heads, 32 * d), 0x7F, dtype=torch.uint8, device="cuda:0") for n in "kv"}
    cache.scales = {n: torch.full((blocks + 26, heads), float("nan"), device="cuda:0") for n in "kv"}
    cache.struct = VF.make_cache(heads, d, cache.codes["k"].data_ptr(), cache.codes["v"].data_ptr(), cache.scales["k"].data_ptr(), cache.scales["v"].data_ptr(), cache.offsets)
    x = [TU.normal((2, 700, heads, d), i, "bf16") for i in range(2)]
    cache.write(x[0], x[1], [0, 0], "bf16", n_seq=lens)
    q = TU.normal((2, len(parent), 2 * heads, d), 5, "bf16")
    k, v = (TU.normal((2, len(parent), heads, d), 6 + i, "bf16") for i in range(2))
    out, lse = call(cache, parent, q, k, v, list(lens), "bf16")
    _check_whole(cache, parent, q, k, v, lens, (0, heads - 1), out, lse)


# Batches whose workgroups take four tiles of rows (blocks by way of LDS; float32: one wavefront per tile): many sequences or many blocks, three tiles and more
MANY = tuple(37 * i % 211 for i in range(64))


@pytest.mark.parametrize("dtype,heads,nq,d,parent", [("bf16", 4, 16, 128, fanout(4, 2, 2, 1, 1)), ("bf16", 4, 16, 64, fanout(4, 2, 2, 1, 1)),
                                                    ("f32", 4, 16, 128, fanout(4, 2, 2, 1, 1)), ("f32", 4, 16, 64, fanout(4, 2, 2, 1, 1)),
                                                    ("bf16", 8, 24, 64, chain(29)), ("bf16", 8, 24, 128, fanout(4, 2, 1, 1))])   # 87 rows: a wavefront without any
def test_four_tiles(dtype, heads, nq, d, parent):
    cache, q, k, v = make(dtype, heads, nq, d, MANY, len(parent), seed=3)
    out, lse = call(cache, parent, q, k, v, list(MANY), dtype)
    check(cache, parent, q, k, v, MANY, dtype, out, lse, heads=[0, heads - 1])
    # the cached positions only
    out, lse = call(cache, parent, q, None, None, list(MANY), dtype)
    check(cache, parent, q, None, None, MANY, dtype, out, lse, heads=[1])


@pytest.mark.parametrize("heads,nq,d,lens,splits", [(2, 16, 128, (9000, 4099, 12001, 5000, 7001, 8000, 31, 6000), 32), (4, 64, 64, (9000, 4099, 12001, 5000), 16)])
def test_four_tiles_in_splits(heads, nq, d, lens, splits):
    parent = fanout(4, 2, 2, 1, 1)
    a = VF.make_tree_attn_args(TU.Cache(heads, d, [32 * ((n + 31) // 32) for n in lens]).struct, nq, "bf16", list(lens))
    assert VF.ps_tree_attention_workspace_bytes(VF.make_tree(parent), a) == splits * heads * 61 * (nq // heads) * (d + 4) * 4   # (two tiles: other splits)
    cache, q, k, v = make("bf16", heads, nq, d, lens, 61, seed=4)
    out, lse = call(cache, parent, q, k, v, list(lens), "bf16")
    _check_whole(cache, parent, q, k, v, lens, (0, heads - 1), out, lse)


@pytest.mark.parametrize("d", [64, 128])
def test_four_tiles_what_is_hidden_does_not_enter(d):
    import torch
    parent, heads, nq = fanout(4, 2, 2, 1, 1), 4, 16
    cache, q, k, v = make("bf16", heads, nq, d, MANY, 61, seed=5, capacity=[n + 32 for n in MANY])
    out, lse = call(cache, parent, q, k, v, list(MANY), "bf16")
    dirty = TU.Cache(heads, d, [32 * ((n + 63) // 32) for n in MANY])
    for n, kind in (("k", cache.codes["k"]), ("v", cache.codes["v"])):
        at = torch.from_numpy(TU.places(n, d)).cuda().reshape(32, d)
        dirty.codes[n].fill_(0x7F)
        dirty.scales[n].fill_(float("nan"))
        for b, length in enumerate(MANY):
            for i in range((length + 31) // 32):
                block, seen = cache.offsets[b] // 32 + i, at[:min(32, length - 32 * i)].reshape(-1)
                dirty.codes[n][block][:, seen] = kind[block][:, seen]
                dirty.scales[n][block] = cache.scales[n][block]
    got, got_lse = call(dirty, parent, q, k, v, list(MANY), "bf16")
    assert got.equal(out) and got_lse.equal(lse)
    # a node's Inf and NaN, and the rows that do not see it
    v2 = v.clone()
    v2[:, 2, :, 5], v2[:, 2, :, 40] = float("inf"), float("nan")
    got, got_lse = call(cache, parent, q, k, v2, list(MANY), "bf16")
    sees = [s for s in range(61) if any(t == 2 for t in _line(parent, s))]
    blind = [s for s in range(61) if s not in sees]
    assert got[:, blind].equal(out[:, blind]) and got_lse.equal(lse)
    assert (got[:, sees][..., 5] == math.inf).all() and torch.isnan(got[:, sees][..., 40]).all()
    rest = [i for i in range(d) if i not in (5, 40)]
    # (the node's other values are what they were; a probability that met Inf is no less exact than before)
    assert got[:, sees][..., rest].equal(out[:, sees][..., rest])


def _line(parent, s):
    while s >= 0:
        yield s
        s = parent[s]


def test_four_tiles_captured_and_replayed_with_other_lengths():
    import torch
    parent = fanout(4, 2, 2, 1, 1)
    cache, q, k, v = make("bf16", 4, 16, 64, MANY, 61, seed=6)
    dev = torch.tensor(MANY, dtype=torch.int32, device="cuda:0")
    keep, s = [], torch.cuda.Stream()
    call(cache, parent, q, k, v, list(MANY), "bf16", dev=dev)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out, lse = call(cache, parent, q, k, v, list(MANY), "bf16", dev=dev, keep=keep)
    for turn in range(4):
        lens = [n if turn == 0 else n * turn // 4 for n in MANY]
        dev.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        want, want_lse = call(cache, parent, q, k, v, list(MANY), "bf16", dev=dev)
        assert out.equal(want) and lse.equal(want_lse)
        check(cache, parent, q, k, v, lens, "bf16", out, lse, heads=[2])


def test_four_tiles_beyond_32_bits_of_bytes():
    import torch
    heads, d, parent = 16, 128, fanout(4, 2, 2, 1, 1)
    base = (1 << 32) // (heads * 32 * d) + 1
    cache = TU.Cache(1, d, [32])
    need = [(n + 31) // 32 for n in MANY]
    cache.heads, cache.offsets = heads, [32 * (base + sum(need[:b])) for b in range(len(MANY) + 1)]
    cache.codes = {n: torch.full((base + sum(need), heads, 32 * d), 0x7F, dtype=torch.uint8, device="cuda:0") for n in "kv"}
    cache.scales = {n: torch.full((base + sum(need), heads), float("nan"), device="cuda:0") for n in "kv"}
    cache.struct = VF.make_cache(heads, d, cache.codes["k"].data_ptr(), cache.codes["v"].data_ptr(), cache.scales["k"].data_ptr(), cache.scales["v"].data_ptr(), cache.offsets)
    x = [TU.normal((len(MANY), max(MANY), heads, d), i, "bf16") for i in range(2)]
    cache.write(x[0], x[1], [0] * len(MANY), "bf16", n_seq=MANY)
    q = TU.normal((len(MANY), 61, 2 * heads, d), 5, "bf16")
    k, v = (TU.normal((len(MANY), 61, heads, d), 6 + i, "bf16") for i in range(2))
    out, lse = call(cache, parent, q, k, v, list(MANY), "bf16")
    _check_whole(cache, parent, q, k, v, MANY, (0, heads - 1), out, lse)
