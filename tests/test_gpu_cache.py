"""GPU tests of the target's 8-bit cache (ps_cache_write, ps_cache_read) against oracle/target.py.  Scales are powers of two and every rounding is one to the
nearest e4m3 value, so codes and scales have to be the oracle's exactly, and what is read back is code * scale, exact in both types."""
import numpy as np
import pytest

from oracle import target as orc
from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import verify as VF
from tests import target_util as TU

pytestmark = pytest.mark.gpu


def _check(cache, before, writes):
    """The cache's contents against the oracle's after `writes` (kind -> [(sequence's first block, length, rows)]); blocks untouched as they were."""
    for n in "kv":
        values, scales = before[n]
        for first, length, rows in writes[n]:
            orc.write(values, scales, first, length, rows)
        got, got_scales = cache.decoded(n)
        assert np.array_equal(got_scales, scales), n
        assert np.array_equal(got, values, equal_nan=True), n
        assert np.array_equal(np.signbit(got), np.signbit(values)) or np.isnan(values).any(), n


CASES = [  # dtype, heads, d, lengths, rows, rows per sequence, gain
    ("bf16", 1, 64, (0,), 1, None, 1.0),
    ("f32", 1, 128, (0,), 1, None, 1.0),
    ("bf16", 3, 128, (31, 32, 33), 1, None, 4.0),
    ("f32", 2, 64, (0, 5, 64, 95), 70, None, 3.0),
    ("bf16", 5, 128, (1, 30, 0), 33, (33, 2, 0), 9.0),
    ("f32", 3, 128, (7, 63), 200, (199, 1), 0.01),
    ("bf16", 8, 64, (17,) * 9, 40, tuple(range(9)), 1.0),
    ("bf16", 40, 128, (100, 3), 65, None, 20.0),
    ("f32", 2, 128, (3,) * 64, 2, None, 2.0),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_write_and_read(case):
    import torch
    dtype, heads, d, lens, rows, n_seq, gain = case
    batch = len(lens)
    cache = TU.Cache(heads, d, [32 * ((n + rows + 31) // 32 + 1) for n in lens], seed=3)
    # what is there already: written by the call itself, with a smaller range so that scales grow
    old = {n: TU.normal((batch, max(max(lens), 1), heads, d), 10 + i, dtype) for i, n in enumerate("kv")}
    cache.write(old["k"], old["v"], [0] * batch, dtype, n_seq=lens)
    before = {n: cache.decoded(n) for n in "kv"}
    new = {n: TU.normal((batch, rows, heads, d), 20 + i, dtype, gain) for i, n in enumerate("kv")}
    cache.write(new["k"], new["v"], lens, dtype, n_seq=n_seq)
    counts = n_seq or (rows,) * batch
    first = [o // 32 for o in cache.offsets]
    _check(cache, before, {n: [(first[b], lens[b], TU.np64(new[n][b, :counts[b]])) for b in range(batch)] for n in "kv"})
    # and back: from the start of the new rows, from the start of all, and one of the two only
    got = {n: torch.full((batch, rows, heads, d), -7.0, dtype=TU.torch_dtype(dtype), device="cuda:0") for n in "kv"}
    cache.read(got["k"], got["v"], lens, dtype, n_seq=counts)
    for n in "kv":
        values, scales = cache.decoded(n)
        for b in range(batch):
            assert np.array_equal(TU.np64(got[n][b, :counts[b]]), orc.read(values, scales, first[b], lens[b], counts[b]))
            assert (got[n][b, counts[b]:] == -7.0).all()
    total = [n + c for n, c in zip(lens, counts)]
    whole = torch.full((batch, max(max(total), 1), heads, d), -7.0, dtype=TU.torch_dtype(dtype), device="cuda:0")
    cache.read(None, whole, None, dtype, n_seq=total)
    values, scales = cache.decoded("v")
    for b in range(batch):
        assert np.array_equal(TU.np64(whole[b, :total[b]]), orc.read(values, scales, first[b], 0, total[b]))
        assert (whole[b, total[b]:] == -7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_first_write_of_a_block_needs_nothing_of_it(dtype):
    """Codes and scales are random bytes (among them NaN) before: nothing of them is left in blocks that begin with the write."""
    cache = TU.Cache(2, 64, [96, 64], seed=8)
    before = {n: cache.decoded(n) for n in "kv"}
    x = TU.normal((2, 40, 2, 64), 1, dtype)
    cache.write(x, x, [0, 0], dtype, n_seq=[40, 32])
    first = [o // 32 for o in cache.offsets]
    _check(cache, before, {n: [(first[b], 0, TU.np64(x[b, :m])) for b, m in ((0, 40), (1, 32))] for n in "kv"})


@pytest.mark.parametrize("dtype,lead,gap", [("bf16", 0, 64), ("bf16", 2, 2), ("f32", 1, 7), ("f32", 3, 128)])
def test_rows_of_a_fused_projection(dtype, lead, gap):
    """Rows further apart than they are long, aligned to 4 bytes only; what lies between them is NaN and is neither read nor written."""
    import torch
    heads, d, lens, rows = 3, 64, (9, 40), 35
    cache, same = (TU.Cache(heads, d, [96, 96], seed=4) for _ in range(2))
    stride = heads * d + gap
    x = [TU.normal((2, rows, heads, d), 30 + i, dtype) for i in range(2)]
    for c, wide in ((cache, True), (same, False)):
        c.write(x[0], x[1], [0, 0], dtype, n_seq=lens if max(lens) <= rows else [9, 35])
        k, v = (TU.strided(y, stride, lead) for y in x) if wide else x
        c.write(k, v, lens, dtype, stride=stride if wide else 0)
    for n in "kv":
        assert torch.equal(cache.codes[n], same.codes[n]) and torch.equal(cache.scales[n].view(torch.int32), same.scales[n].view(torch.int32))
    flat = torch.full((lead + 2 * rows * stride,), 5.0, dtype=TU.torch_dtype(dtype), device="cuda:0")
    out = flat[lead:].as_strided((2, rows, heads, d), (rows * stride, stride, d, 1))
    dense = torch.empty((2, rows, heads, d), dtype=flat.dtype, device="cuda:0")
    cache.read(out, None, lens, dtype, stride=stride)
    cache.read(dense, None, lens, dtype)
    assert torch.equal(out, dense)
    outside = torch.ones_like(flat, dtype=torch.bool)
    outside[lead:].as_strided((2, rows, heads, d), (rows * stride, stride, d, 1)).fill_(False)
    assert (flat[outside] == 5.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_accepted_path_is_committed(dtype):
    """What a walk leaves: different numbers of accepted nodes, a given-up walk (-2), entries that are no nodes; lengths on the device, in place or not."""
    import torch
    heads, d, nodes, depth = 4, 128, 21, 6
    lens = [0, 31, 64, 30, 5, 29, 77, 12]
    acc = [0, 6, 3, -2, 4, 2, 6, 9]
    paths = [[1, 2, 3, 4, 5, 6]] * 2 + [[20, 19, 3, 0, 0, 0]] + [[1] * 6] + [[4, 7, 21, 9, -1, -1]] + [[-1, 5, -1, -1, -1, -1]] + [[2, 2, 2, 20, 20, 1], [3, 5, 8, 9, 11, 14]]
    batch = len(lens)
    tree = {n: TU.normal((batch, nodes, heads, d), 50 + i, dtype, 3.0) for i, n in enumerate("kv")}
    old = TU.normal((batch, 80, heads, d), 60, dtype)
    n_acc, path = (torch.tensor(x, dtype=torch.int32, device="cuda:0") for x in (acc, paths))
    taken = [orc.path_rows(a, p, nodes) for a, p in zip(acc, paths)]
    for in_place in (False, True):
        cache = TU.Cache(heads, d, [128] * batch, seed=6)
        cache.write(old, old, [0] * batch, dtype, n_seq=lens)
        before = {n: cache.decoded(n) for n in "kv"}
        dev = torch.tensor(lens, dtype=torch.int32, device="cuda:0")
        out = dev if in_place else torch.full((batch,), -9, dtype=torch.int32, device="cuda:0")
        cache.write(tree["k"], tree["v"], [121] * batch, dtype, n_accepted=n_acc, path=path, path_rows=depth, kv_len_dev=dev, len_out=out)
        assert out.tolist() == [n + len(t) for n, t in zip(lens, taken)]
        if not in_place:
            assert dev.tolist() == lens
        first = [o // 32 for o in cache.offsets]
        _check(cache, before, {n: [(first[b], lens[b], TU.np64(tree[n][b])[taken[b]]) for b in range(batch)] for n in "kv"})


def test_lengths_outside_their_bounds_count_as_the_bounds():
    import torch
    x = TU.normal((3, 4, 2, 64), 1, "f32")
    a, b = (TU.Cache(2, 64, [64] * 3, seed=2, scales=1.0) for _ in range(2))
    dev = torch.tensor([-5, 1 << 30, 20], dtype=torch.int32, device="cuda:0")
    out = torch.empty_like(dev)
    a.write(x, x, [30, 30, 30], "f32", kv_len_dev=dev, len_out=out)
    b.write(x, x, [0, 30, 20], "f32")
    assert out.tolist() == [4, 34, 24]
    assert torch.equal(a.codes["k"], b.codes["k"]) and torch.equal(a.codes["v"], b.codes["v"])


def test_numbers_at_the_ends_of_the_range():
    """Zeros, denormal numbers, the largest floats, numbers on a rounding border, Inf and NaN."""
    import torch
    d = 64
    rows = torch.zeros((1, 9, 1, d))
    rows[0, 0, 0, :8] = torch.tensor([0.0, -0.0, 1e-40, -1e-45, 2.0 ** -126, 2.0 ** -110, -(2.0 ** -111), 2.0 ** -109])
    rows[0, 1, 0, :4] = torch.tensor([3.4028234663852886e38, -1e38, 1.0, -3e36])
    rows[0, 2, 0, :5] = torch.tensor([float("inf"), -float("inf"), float("nan"), 448.0, -17.0])
    rows[0, 3, 0, :4] = torch.tensor([448.0, 17.0, -19.0, 2.0 ** -10])
    rows[0, 4, 0, :4] = torch.tensor([449.0, 17.0, -18.0, 3 * 2.0 ** -10])
    rows[0, 5, 0, :2] = torch.tensor([1.75 * 2.0 ** 20, 1.0])
    rows[0, 6, 0, :2] = torch.tensor([1.7500001 * 2.0 ** 20, 1.0])
    rows[0, 7, 0, :] = float("nan")
    rows = rows.cuda()
    for i in range(9):                                        # each as the only row of a block, then all of them in one
        cache = TU.Cache(1, d, [64], seed=i)
        before = {n: cache.decoded(n) for n in "kv"}
        cache.write(rows[:, i:i + 1].contiguous(), rows[:, i:i + 1].contiguous(), [0], "f32")
        _check(cache, before, {n: [(1, 0, TU.np64(rows[0, i:i + 1]))] for n in "kv"})
    cache = TU.Cache(1, d, [64], seed=11)
    before = {n: cache.decoded(n) for n in "kv"}
    for i in range(9):
        cache.write(rows[:, i:i + 1].contiguous(), rows[:, i:i + 1].contiguous(), [i], "f32")
    _check(cache, before, {n: [(1, i, TU.np64(rows[0, i:i + 1])) for i in range(9)] for n in "kv"})
    for dtype in ("f32", "bf16"):
        back = torch.empty((1, 9, 1, d), dtype=TU.torch_dtype(dtype), device="cuda:0")
        cache.read(back, None, [0], dtype)
        values, scales = cache.decoded("k")
        # (the largest float is nearest to 256 * 2^120, which is 2^128 and beyond both types: Inf)
        want = torch.from_numpy(orc.read(values, scales, 1, 0, 9)).to(back.dtype)
        assert np.array_equal(TU.np64(back[0]), TU.np64(want), equal_nan=True)


def test_blocks_beyond_32_bits_of_bytes():
    """A sequence whose codes lie more than 4 GiB behind the cache's start."""
    import torch
    heads, d = 16, 128
    blocks = (1 << 32) // (heads * 32 * d) + 3
    codes = [torch.empty(blocks * heads * 32 * d, dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    scales = [torch.empty((blocks, heads), device="cuda:0") for _ in range(2)]
    for c in codes:
        c[:1 << 20] = 0x55
    struct = VF.make_cache(heads, d, codes[0].data_ptr(), codes[1].data_ptr(), scales[0].data_ptr(), scales[1].data_ptr(), [32 * (blocks - 2), 32 * blocks])
    x = TU.normal((1, 40, heads, d), 1, "bf16")
    a = VF.make_cache_write_args(struct, 40, "bf16", [3])
    a.k_rows = a.v_rows = x.data_ptr()
    b = VF.make_cache_write_args(struct, 3, "bf16", [0])
    b.k_rows = b.v_rows = x.data_ptr()
    assert VF.ps_cache_write(b, TU.stream()) == B.PS_OK and VF.ps_cache_write(a, TU.stream()) == B.PS_OK
    back = torch.empty_like(x)
    r = VF.make_cache_read_args(struct, 40, "bf16", [3])
    r.k_rows = back.data_ptr()
    assert VF.ps_cache_read(r, TU.stream()) == B.PS_OK
    assert ((back.float() - x.float()).abs() <= x.float().abs() * 2.0 ** -4 + 2.0 ** -16).all()
    assert all((c[:1 << 20] == 0x55).all() for c in codes)
