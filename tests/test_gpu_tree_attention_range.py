"""GPU tests of the tree attention (ps_tree_attention) with values of very different size: what has no weight in the results' numerator still has its part of the sum.

All keys and values are numbers that the cache holds exactly, scores are powers of two in exponent (scale = log 2, or q in proportion), so results have closed forms."""
import math

import numpy as np
import pytest

from paper_2410_05589_amd import verify as VF
from tests import target_util as TU
from tests.test_gpu_tree_attention import call, chain

pytestmark = pytest.mark.gpu

# how rows are cut: one, two and four tiles of 32 rows per workgroup (17 nodes of 4 query heads per kv head are 68 rows); dtype, query heads per kv head, tree, wavefronts that
# divide a tile's blocks
SHAPES = [("bf16", 1, [-1], 8), ("f32", 1, [-1], 4), ("bf16", 2, chain(17), 4), ("f32", 2, chain(17), 2), ("bf16", 4, chain(17), 1), ("f32", 4, chain(17), 1)]


def _filled(heads, d, k, v):
    """A cache of one sequence with the rows k, v [n, d] of all heads (made on the device)."""
    import torch
    n = k.shape[0]
    cache = TU.Cache(1, d, [32])
    cache.heads, cache.offsets = heads, [0, (n + 31) // 32 * 32]
    blocks = (n + 31) // 32
    cache.codes = {x: torch.empty((blocks, heads, 32 * d), dtype=torch.uint8, device="cuda:0") for x in "kv"}
    cache.scales = {x: torch.empty((blocks, heads), device="cuda:0") for x in "kv"}
    cache.struct = VF.make_cache(heads, d, cache.codes["k"].data_ptr(), cache.codes["v"].data_ptr(), cache.scales["k"].data_ptr(), cache.scales["v"].data_ptr(), cache.offsets)
    for at in range(0, n, 4096):
        kk, vv = (x[None, at:at + 4096, None].expand(1, -1, heads, d).to(torch.bfloat16).contiguous() for x in (k, v))
        cache.write(kk, vv, [at], "bf16")
    return cache


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%s-%d-%d" % (s[0], s[1], len(s[2])))
def test_probabilities_of_values_that_are_zero_are_in_the_sum(shape, d):
    """32768 positions whose score is 2^-27 of the first one's and whose values are all zero (their blocks' scale is the least there is): together 2^-12 of the sum.
    256 kv heads, so that a workgroup has a whole sequence.  Tolerance: sums of positive terms, per wavefront 16 terms of a block and then block by block, then a
    few joins, each addition off by 2^-24 of the sum; exponentials and the logarithm 2^-20."""
    import torch
    dtype, grp, parent, wk = shape
    n, heads = 32768, 256
    k = torch.zeros((n, d), device="cuda:0")
    k[1:, 0], k[1:, 1] = -13.0, -14.0
    v = torch.zeros((n, d), device="cuda:0")
    v[0] = 1.0
    cache = _filled(heads, d, k, v)
    assert float(cache.scales["v"][1:].max()) == 2.0 ** -100
    q = torch.zeros((1, len(parent), heads * grp, d), dtype=TU.torch_dtype(dtype), device="cuda:0")
    q[..., 0] = q[..., 1] = 1.0
    out, lse = call(cache, parent, q, None, None, [n], dtype, scale=math.log(2))
    total = 1.0 + (n - 1) * 2.0 ** -27
    tol = (n / 32 / wk + 64) * 2.0 ** -24 + 2.0 ** -20
    assert tol < 0.75 * (n / wk) * 2.0 ** -27                 # (what one wavefront's positions add is seen)
    assert np.abs(TU.np64(lse) - math.log(total)).max() <= tol
    assert np.abs(TU.np64(out) * total - 1.0).max() <= tol + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -22)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%s-%d-%d" % (s[0], s[1], len(s[2])))
@pytest.mark.parametrize("size", [2.0 ** 125, 2.0 ** 60, 2.0 ** -60, 2.0 ** -90])
def test_values_at_the_ends_of_the_range(shape, d, size):
    """Values near the largest and the smallest numbers, block by block with a score that is 1.75 powers of two higher than in the one before, so that the maximum that
    exponentials are taken against is behind for some blocks."""
    import torch
    dtype, grp, parent, _ = shape
    n, heads = 32 * 40, 64
    block = torch.arange(n, device="cuda:0") // 32
    k = torch.zeros((n, d), device="cuda:0")
    score = 1.75 * block
    k[:, 0] = torch.where(torch.arange(n, device="cuda:0") % 32 == 5, (block / 4).floor(), -1.0)    # (e4m3: whole numbers up to 16)
    k[:, 1] = torch.where(torch.arange(n, device="cuda:0") % 32 == 5, block % 4, -64.0)
    v = torch.zeros((n, d), device="cuda:0")
    v[:] = (1.0 + (block % 4)[:, None] / 4) * size / 2
    v[:, 1::2] *= -1
    cache = _filled(heads, d, k, v)
    q = torch.zeros((1, len(parent), heads * grp, d), dtype=TU.torch_dtype(dtype), device="cuda:0")
    q[..., 0], q[..., 1] = 7.0, 1.75
    out, lse = call(cache, parent, q, None, None, [n], dtype, scale=math.log(2))
    s = np.where(np.arange(n) % 32 == 5, TU.np64(score.float()), -7.0 - 112.0)
    p = np.exp2(s - s.max())
    want = (p[:, None] * TU.np64(v)).sum(0) / p.sum()
    # (a score of up to 70 is off by 2^-23 of itself, the rest as in the test before; bf16: probabilities and results by 2^-8 each)
    tol = 70 * 2.0 ** -22 + 104 * 2.0 ** -24 + 2.0 ** -20 + (2.0 ** -7 if dtype == "bf16" else 0.0)
    assert np.abs(TU.np64(out) / want - 1.0).max() <= tol
    assert np.abs(TU.np64(lse) - (s.max() * math.log(2) + math.log(p.sum()))).max() <= 70 * 2.0 ** -22 + 104 * 2.0 ** -24 + 2.0 ** -20


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%s-%d-%d" % (s[0], s[1], len(s[2])))
def test_queries_of_zero_over_the_largest_keys(shape):
    """All scores are zero, whatever the keys and the scale are: the mean of the values."""
    import torch
    dtype, grp, parent, _ = shape
    n, heads, d = 75, 2, 64
    k = torch.full((n, d), 2.0 ** 125, device="cuda:0")
    v = (torch.arange(n, device="cuda:0") % 8).float()[:, None].expand(n, d).contiguous()
    cache = _filled(heads, d, k, v)
    q = torch.zeros((1, len(parent), heads * grp, d), dtype=TU.torch_dtype(dtype), device="cuda:0")
    out, lse = call(cache, parent, q, None, None, [n], dtype, scale=2.0 ** 20)
    want = float(v[:, 0].double().mean())
    assert np.abs(TU.np64(out) - want).max() <= want * (2.0 ** -7 if dtype == "bf16" else 2.0 ** -18)
    assert np.abs(TU.np64(lse) - math.log(n)).max() <= 2.0 ** -18
