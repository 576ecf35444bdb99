"""GPU tests of what Inf and NaN do in the training attention's backward pass where the mask lets them through: a value enters the sums that the formulas
have it in, whether the two rows meet in a tile that the mask cuts or in one that is seen whole, and no other sum.

  d_v[j, c] = sum_i P_ij d_out[i, c]      d_out[i, c] reaches column c of every key that row i sees, and that column only
  d_q[i]    = sum_j dS_ij k~_j            k~_j (columns c and c + d / 2) reaches every row that sees key j: dS_ij times Inf is Inf, or NaN where dS_ij = 0
  d_k[j]    = sum_i dS_ij q~_i            likewise
  v enters dP and delta, not P: d_v stays what it is.

Every comparison is of bits, or for not being finite."""
import math

import pytest

from tests.test_gpu_group_attention_grad import backward, forward, make

pytestmark = pytest.mark.gpu

# dtype, seqs, T, k, heads, kv heads, head_dim: tiles cut by the mask and whole ones, [MASK] keys, shared heads; the last three have 256 blocks of query rows
CASES = [("bf16", 1, 70, 4, 2, 1, 128), ("f32", 1, 70, 4, 2, 2, 64), ("bf16", 1, 150, 2, 2, 1, 64), ("f32", 1, 45, 15, 2, 1, 128), ("bf16", 1, 200, 0, 2, 2, 128),
         ("bf16", 4, 37, 4, 32, 8, 128), ("f32", 4, 50, 2, 32, 16, 64), ("bf16", 4, 70, 2, 32, 32, 64)]
VALUES = [float("nan"), float("inf"), -float("inf")]
COL = 5


def _places(T, k):
    """(group, slot) of the row that is hit: the first and the last, a real token and a [MASK] token in between."""
    return sorted({(0, 0), (T // 2, 0), (T // 3, min(k, 2)), (T - 1, k)})


def _sees(T, k):
    import torch
    row = torch.arange(T * (k + 1), device="cuda:0")
    group, slot = row // (k + 1), row % (k + 1)
    return (row[:, None] >= row[None, :]) & ((slot[None, :] == 0) | (group[:, None] == group[None, :]))


def _odd(t):
    import torch
    return ~torch.isfinite(t.float())


@pytest.mark.parametrize("case", CASES)
def test_a_gradient_reaches_the_values_that_its_row_sees(case):
    import torch
    dtype, seqs, T, k, nq, nkv, d = case
    x = make(seqs, T, k, nq, nkv, d, dtype, 21)
    out, lse = forward(x, T, k)
    want = backward(x, out, lse, T, k)
    sees, b, h, hk = _sees(T, k), seqs - 1, nq - 1, nkv - 1
    for g, s in _places(T, k):
        bad = g * (k + 1) + s
        keys = sees[bad]
        for value in VALUES:
            print("case d_out", case, g, s, value, flush=True)
            y = dict(x, d_out=x["d_out"].clone())
            y["d_out"][b, bad, h, COL] = value
            got = backward(y, out, lse, T, k)
            hit = got["d_v"][b, keys, hk, COL].float()
            assert bool((torch.isnan(hit) if math.isnan(value) else torch.isnan(hit) | (hit == value)).all()), int((~_odd(hit)).sum())
            rest = got["d_v"].clone()
            rest[b, keys, hk, COL] = want["d_v"][b, keys, hk, COL]
            assert torch.equal(rest, want["d_v"])
            assert bool(_odd(got["d_q"][b, bad, h]).all()) and bool(_odd(got["d_k"][b, keys, hk]).all())
            got["d_q"][b, bad, h] = want["d_q"][b, bad, h]
            got["d_k"][b, keys, hk] = want["d_k"][b, keys, hk]
            assert torch.equal(got["d_q"], want["d_q"]) and torch.equal(got["d_k"], want["d_k"])


@pytest.mark.parametrize("case", CASES)
def test_a_key_reaches_the_queries_that_see_it_and_a_query_the_keys_that_it_sees(case):
    import torch
    dtype, seqs, T, k, nq, nkv, d = case
    x = make(seqs, T, k, nq, nkv, d, dtype, 22)
    sees, b, hk, group = _sees(T, k), seqs - 1, nkv - 1, nq // nkv
    columns = [COL, COL + d // 2]
    for g, s in _places(T, k):
        bad = g * (k + 1) + s
        for value in VALUES:
            print("case key, query", case, g, s, value, flush=True)
            y = dict(x, k=x["k"].clone())
            y["k"][b, bad, hk, COL] = value
            out, lse = forward(y, T, k)
            got = backward(y, out, lse, T, k)["d_q"][b, sees[:, bad], hk * group:]
            assert bool(_odd(got[..., columns]).all()), int((~_odd(got[..., columns])).sum())
            y = dict(x, q=x["q"].clone())
            y["q"][b, bad, nq - 1, COL] = value
            out, lse = forward(y, T, k)
            got = backward(y, out, lse, T, k)["d_k"][b, sees[bad], hk]
            assert bool(_odd(got[..., columns]).all()), int((~_odd(got[..., columns])).sum())


@pytest.mark.parametrize("case", CASES)
def test_a_value_does_not_reach_the_gradients_of_values(case):
    import torch
    dtype, seqs, T, k, nq, nkv, d = case
    x = make(seqs, T, k, nq, nkv, d, dtype, 23)
    out, lse = forward(x, T, k)
    want = backward(x, out, lse, T, k)["d_v"]
    for g, s in _places(T, k):
        for value in VALUES:
            print("case value", case, g, s, value, flush=True)
            y = dict(x, v=x["v"].clone())
            y["v"][seqs - 1, g * (k + 1) + s, nkv - 1, COL] = value
            out, lse = forward(y, T, k)
            assert torch.equal(backward(y, out, lse, T, k)["d_v"], want)
