"""Pins of oracle/target.py: e4m3 against torch's conversion, scales, block layout, attention and distributions against other formulations."""
import math

import numpy as np
import pytest
import torch

from oracle import target as orc


def test_codes_stand_for_what_torch_says():
    ours = orc.e4m3_values()
    theirs = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ours, theirs, equal_nan=True)


def test_rounding_is_to_nearest_even():
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(4000, generator=g) * s for s in (1e-3, 0.1, 3.0, 100.0)]).clamp(-448, 448)
    grid = torch.from_numpy(orc.VALUES[:127])
    x = torch.cat([x.double(), grid, (grid[1:] + grid[:-1]) / 2, -(grid[1:] + grid[:-1]) / 2])      # values and the places between them
    assert np.array_equal(orc.e4m3_round(x.numpy()), x.float().to(torch.float8_e4m3fn).double().numpy())


def test_scale_is_the_least_power_of_two():
    for x in (448.0, 448.0001, 1.0, 1.75, 1.7500001, 3e38, 2.0 ** -92, 1e-40, 0.0):
        s = orc.scale_of(np.array([0.5 * x, -x]))
        assert math.log2(s) == int(math.log2(s)) and x <= 448 * s
        assert s == 2.0 ** -100 or x > 448 * s / 2
    assert orc.scale_of(np.array([math.nan, math.inf, 3.0])) == orc.scale_of(np.array([3.0]))


@pytest.mark.parametrize("kind", ["k", "v"])
@pytest.mark.parametrize("d", [64, 128])
def test_layout_places_every_byte_once(kind, d):
    t, j = np.meshgrid(np.arange(32), np.arange(d), indexing="ij")
    assert sorted(orc.place(kind, t, j).reshape(-1)) == list(range(32 * d))


def test_rows_written_at_once_or_one_by_one_differ_by_the_second_rounding_only():
    rng = np.random.default_rng(5)
    rows = rng.standard_normal((50, 2, 64)) * np.exp(rng.standard_normal((50, 1, 1)))
    one = [np.zeros((3, 2, 32, 64)), np.zeros((3, 2))]
    many = [np.zeros((3, 2, 32, 64)), np.zeros((3, 2))]
    orc.write(*one, 0, 0, rows)
    for i in range(50):
        orc.write(*many, 0, i, rows[i:i + 1])
    assert np.array_equal(one[1][:2], many[1][:2])
    a, b = orc.read(*one, 0, 0, 50), orc.read(*many, 0, 0, 50)
    # where the scale grew, codes below 2^-6 lose bits once more: half a step of 2^-9
    scale = np.repeat(one[1][:2].T, 32, axis=1).T[:50][:, :, None]
    assert (np.abs(a - b) <= 2.0 ** -9 * scale).all()
    assert np.abs(a - rows).max() <= (np.abs(rows) * 2.0 ** -4 + 2.0 ** -10 * scale).max()


def test_attention_is_softmax_under_the_tree_mask():
    rng = np.random.default_rng(2)
    parent = [-1, 0, 0, 1, 3, 2]
    q, k, v = rng.standard_normal((6, 4, 8)), rng.standard_normal((9 + 6, 2, 8)), rng.standard_normal((9 + 6, 2, 8))
    out, lse = orc.tree_attention(parent, q, k[:9], v[:9], k[9:], v[9:], 0.3)
    mask = torch.zeros(6, 15, dtype=torch.bool)
    mask[:, :9] = True
    for s in range(6):
        u = s
        while u >= 0:
            mask[s, 9 + u] = True
            u = parent[u]
    kk, vv = (torch.from_numpy(x).repeat_interleave(2, 1).transpose(0, 1) for x in (k, v))
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(0, 1), kk, vv, attn_mask=mask, scale=0.3)
    np.testing.assert_allclose(out, want.transpose(0, 1).numpy(), atol=1e-12)
    logits = (torch.from_numpy(q).transpose(0, 1) @ kk.transpose(1, 2) * 0.3).masked_fill(~mask, -math.inf)
    np.testing.assert_allclose(lse, torch.logsumexp(logits, -1).t().numpy(), atol=1e-12)


def test_distribution_keeps_what_it_says():
    x = np.array([1.0, 3.0, 2.0, 3.0, -math.inf, 0.0])
    e = np.exp(x - 3.0)
    p, _ = orc.distribution(x)
    np.testing.assert_allclose(p, e / e.sum())
    assert orc.distribution(x, temperature=0.0)[0].tolist() == [0, 1, 0, 0, 0, 0]
    assert (orc.distribution(x, top_k=1)[0] > 0).tolist() == [False, True, False, False, False, False]
    assert (orc.distribution(x, top_k=3)[0] > 0).tolist() == [False, True, True, True, False, False]
    # the two largest have 2 / 2.5532 = 0.783 of the mass
    assert (orc.distribution(x, top_p=0.78)[0] > 0).sum() == 2 and (orc.distribution(x, top_p=0.79)[0] > 0).sum() == 3
    assert (orc.distribution(x, top_p=0.0)[0] > 0).tolist() == [False, True, False, False, False, False]
    assert (orc.distribution(x, min_p=0.36)[0] > 0).sum() == 3 and (orc.distribution(x, min_p=0.37)[0] > 0).sum() == 2
    assert (orc.distribution(x, min_p=1.0)[0] > 0).sum() == 2 == (orc.distribution(x, min_p=7.0)[0] > 0).sum()
    assert (orc.distribution(np.full(3, -math.inf))[0] == 0).all() and np.isnan(orc.distribution(np.array([1.0, math.inf]))[0]).all()


def test_draws_follow_the_distribution():
    rng = np.random.default_rng(3)
    p, _ = orc.distribution(rng.standard_normal(7) * 2)
    r = (np.arange(20000) + 0.5) / 20000
    got = np.bincount([orc.draw(p, x)[0] for x in r], minlength=7) / 20000
    np.testing.assert_allclose(got, p, atol=1e-4)
    assert orc.draw(np.array([0.0, 1.0, 0.0]), 0.0)[0] == 1 == orc.draw(np.array([0.0, 1.0, 0.0]), 1 - 2.0 ** -24)[0]


def test_a_path_ends_before_what_is_no_row():
    assert orc.path_rows(-2, [1, 2], 5) == [] and orc.path_rows(0, [1, 2], 5) == [0]
    assert orc.path_rows(2, [3, 4], 5) == [0, 3, 4] and orc.path_rows(2, [3, 5], 5) == [0, 3] and orc.path_rows(2, [-1, 4], 5) == [0]
