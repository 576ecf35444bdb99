"""GPU tests of the training attention's backward pass (ps_group_attention_lse, ps_group_attention_grad) against its
formulas in float64.

Tolerances, element by element.  With S_dv = sum_i P_ij |d_out_i|, S_dk = sum_i |dS_ij| |q~_i|, S_dq = sum_j |dS_ij| |k~_j| (over sqrt(d)) and T_dk, T_dq the
same with P (|dP| + |delta|) in the place of |dS|:
  float32: a score and a dP are sums of d products (errors of about sqrt(d) 2^-24 of |q||k|), so e = 2^-18 (1 + |q||k| / sqrt(d)) of S and T;
  bf16: P and dS are rounded once, half a step 2^-8 each, so 2^-8 of S more; a rotated key's element that lies on a rounding boundary may
  fall to the other side and move by a step, 2^-7 of its value, which moves a score by up to e_s = 2^-7 max|q~| max|k~| / sqrt(d), and a
  probability by that factor: e_s of S and T more; half a step of the result.
A probability below the smallest normal float32, 2^-126, may be taken for zero: 2^-126 in the place of P more in each sum.
As a whole (2-norms): float32 2e-6 plus what the scores' length adds; bf16 2^-8, which is twice what two independent roundings leave."""
import math

import numpy as np
import pytest

from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import train as TR

pytestmark = pytest.mark.gpu

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def _tdtype(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def make(seqs, T, k, nq, nkv, d, dtype, seed, length=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    rows = T * (k + 1)

    def normal(heads, std=1.0):
        return (torch.randn((seqs, rows, heads, d), generator=g) * std).to(_tdtype(dtype)).cuda()
    return {"q": normal(nq, length), "k": normal(nkv), "v": normal(nkv), "d_out": normal(nq)}


def _workspace(need):
    import torch
    ws = torch.full((need + 512,), 0xFF, dtype=torch.uint8, device="cuda:0")
    at = (ws.data_ptr() + 255) & ~255
    return ws, at


def forward(x, T, k, base=10000.0, lse=True):
    import torch
    seqs, rows, nq, d = x["q"].shape
    dtype = "bf16" if x["q"].dtype == torch.bfloat16 else "f32"
    a = TR.make_args(seqs, T, k, nq, x["k"].shape[2], d, dtype, base)
    need = TR.ps_group_attention_workspace_bytes(a)
    ws, a.workspace = _workspace(need)
    a.workspace_bytes = need
    out = torch.full((seqs, rows, nq, d), 77.0, device="cuda:0")
    sums = torch.full((seqs, rows, nq), 77.0, device="cuda:0")
    a.q, a.k_, a.v, a.out = x["q"].data_ptr(), x["k"].data_ptr(), x["v"].data_ptr(), out.data_ptr()
    st = TR.ps_group_attention_lse(a, sums.data_ptr(), _stream()) if lse else TR.ps_group_attention(a, _stream())
    assert st == B.PS_OK
    torch.cuda.synchronize()
    return out, sums


def grad_args(x, out, lse, T, k, base=10000.0):
    import torch
    seqs, rows, nq, d = x["q"].shape
    dtype = "bf16" if x["q"].dtype == torch.bfloat16 else "f32"
    a = TR.make_grad_args(seqs, T, k, nq, x["k"].shape[2], d, dtype, base)
    need = TR.ps_group_attention_grad_workspace_bytes(a)
    ws, a.workspace = _workspace(need)
    a.workspace_bytes = need
    got = {n: torch.full_like(x[n[2:]], 77.0) for n in ("d_q", "d_k", "d_v")}
    a.q, a.k_, a.v, a.d_out = x["q"].data_ptr(), x["k"].data_ptr(), x["v"].data_ptr(), x["d_out"].data_ptr()
    a.out, a.lse = out.data_ptr(), lse.data_ptr()
    a.d_q, a.d_k, a.d_v = (got[n].data_ptr() for n in ("d_q", "d_k", "d_v"))
    return a, got, ws


def backward(x, out, lse, T, k, base=10000.0):
    import torch
    a, got, ws = grad_args(x, out, lse, T, k, base)
    assert TR.ps_group_attention_grad(a, _stream()) == B.PS_OK
    torch.cuda.synchronize()
    end = a.workspace - ws.data_ptr() + a.workspace_bytes
    assert bool((ws[end:] == 0xFF).all())
    return got


def _turn(x, pos, base, sign):
    import torch
    d = x.shape[-1]
    angle = pos.double()[:, None] * base ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
    a, b = x[..., :d // 2], x[..., d // 2:]
    cos, sin = angle.cos(), sign * angle.sin()
    return torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)


def reference(x, T, k, base=10000.0):
    """The formulas in float64, sequence by sequence and head by head over the whole layout; (gradient, tolerance) of each."""
    import torch
    seqs, rows, nq, d = x["q"].shape
    nkv, dtype = x["k"].shape[2], "bf16" if x["q"].dtype == torch.bfloat16 else "f32"
    row = torch.arange(rows, device="cuda:0")
    g, slot = row // (k + 1), row % (k + 1)
    sees = (row[:, None] >= row[None, :]) & ((slot[None, :] == 0) | (g[:, None] == g[None, :]))
    want = {n: torch.zeros(x[n[2:]].shape, dtype=torch.float64, device="cuda:0") for n in ("d_q", "d_k", "d_v")}
    tol = {n: torch.zeros_like(w) for n, w in want.items()}
    out, lse = torch.zeros((seqs, rows, nq, d), dtype=torch.float64, device="cuda:0"), torch.zeros((seqs, rows, nq), dtype=torch.float64, device="cuda:0")
    for b in range(seqs):
        for h in range(nq):
            hk = h // (nq // nkv)
            q = _turn(x["q"][b, :, h].double(), g + slot, base, 1.0)
            kr = _turn(x["k"][b, :, hk].double(), g + slot, base, 1.0).to(x["k"].dtype).double()
            v, do = x["v"][b, :, hk].double(), x["d_out"][b, :, h].double()
            s = (q @ kr.t() / math.sqrt(d)).masked_fill(~sees, -math.inf)
            lse[b, :, h] = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[b, :, h][:, None])
            out[b, :, h] = p @ v
            dp, delta = do @ v.t(), (do * out[b, :, h]).sum(1, keepdim=True)
            ds, most = p * (dp - delta), p * (dp.abs() + delta.abs())
            dq, dk = ds @ kr / math.sqrt(d), ds.t() @ q / math.sqrt(d)
            reach = float(q.norm(dim=1).max() * kr.norm(dim=1).max()) / math.sqrt(d)
            e = 2.0 ** -18 * (1 + reach)
            if dtype == "bf16":
                e += 2.0 ** -7 * float(q.abs().max() * kr.abs().max()) / math.sqrt(d)
            half = 2.0 ** -8 if dtype == "bf16" else 0.0
            tiny = torch.where(sees, 2.0 ** -126, 0.0)
            both = half * ds.abs() + e * (ds.abs() + most) + tiny * (dp.abs() + delta.abs())
            turned = lambda z: z + torch.cat((z[:, d // 2:], z[:, :d // 2]), 1)   # (a rotation mixes the two of a pair)
            want["d_q"][b, :, h] += _turn(dq, g + slot, base, -1.0)
            want["d_k"][b, :, hk] += _turn(dk, g + slot, base, -1.0)
            want["d_v"][b, :, hk] += p.t() @ do
            tol["d_q"][b, :, h] += turned(both @ kr.abs()) / math.sqrt(d)
            tol["d_k"][b, :, hk] += turned(both.t() @ q.abs()) / math.sqrt(d)
            tol["d_v"][b, :, hk] += (p * (half + e) + tiny).t() @ do.abs()
    for n in want:
        tol[n] += want[n].abs() * HALF_STEP[dtype] * 1.01
    return want, tol, out, lse, reach


def check(x, got, want, tol, reach, dtype):
    for n in ("d_q", "d_k", "d_v"):
        err = (got[n].double() - want[n]).abs()
        assert bool((err <= tol[n]).all()), (n, float((err / tol[n].clamp(min=1e-300)).max()))
        norm = float(want[n].norm())
        rel = float(err.norm()) / norm if norm > 1e-12 * want[n].numel() ** 0.5 else 0.0
        print("    %s relative error %.2g" % (n, rel), flush=True)
        assert rel <= (2e-6 + 2.0 ** -22 * reach if dtype == "f32" else 2.0 ** -8), (n, rel)


CASES = [  # dtype, seqs, T, k, heads, kv heads, head_dim
    ("bf16", 1, 1, 0, 1, 1, 64), ("f32", 1, 1, 0, 1, 1, 128), ("bf16", 1, 1, 4, 2, 1, 64), ("f32", 2, 1, 15, 2, 2, 64),
    ("f32", 2, 37, 4, 4, 2, 64), ("bf16", 2, 37, 4, 4, 2, 64),             # blocks that end inside a group, a ragged last block, shared heads
    ("f32", 1, 50, 2, 2, 2, 128), ("bf16", 1, 50, 2, 2, 2, 128),
    ("bf16", 1, 21, 7, 2, 1, 64), ("bf16", 1, 32, 3, 2, 1, 128),           # groups that divide the tiles
    ("f32", 1, 9, 15, 2, 2, 64), ("bf16", 1, 40, 15, 8, 2, 128),           # the longest groups
    ("f32", 1, 70, 0, 4, 4, 64), ("bf16", 1, 300, 0, 4, 1, 128),           # k = 0: ordinary causal attention
    ("bf16", 1, 129, 8, 8, 2, 128), ("bf16", 3, 128, 5, 2, 2, 64), ("bf16", 1, 127, 1, 2, 2, 128),
    ("f32", 1, 260, 3, 2, 1, 64), ("f32", 1, 140, 6, 2, 2, 128), ("bf16", 1, 520, 4, 2, 1, 128), ("bf16", 1, 700, 2, 3, 3, 64),
]


@pytest.mark.parametrize("dtype,seqs,T,k,nq,nkv,d", CASES)
def test_gradients(dtype, seqs, T, k, nq, nkv, d):
    import torch
    print("case grad", dtype, seqs, T, k, nq, nkv, d, flush=True)
    x = make(seqs, T, k, nq, nkv, d, dtype, T + k)
    out, lse = forward(x, T, k)
    plain, _ = forward(x, T, k, lse=False)
    assert torch.equal(out, plain)                           # the forward pass for training: the same bits
    want, tol, out64, lse64, reach = reference(x, T, k)
    flip = 2.0 ** -7 * 25.0 / math.sqrt(d) if dtype == "bf16" else 0.0   # (see the module's text: e_s with |q~|, |k~| up to 5)
    assert float((lse - lse64).abs().max()) <= 2.0 ** -18 * (1 + reach) + flip
    got = backward(x, out, lse, T, k)
    check(x, got, want, tol, reach, dtype)
    again = backward(x, out, lse, T, k)
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("dtype,d,length", [("f32", 64, 20.0), ("bf16", 128, 20.0), ("f32", 64, 1000.0)])
def test_scores_that_lie_far_apart(dtype, d, length):
    """Queries 20 and 1000 times as long: probabilities that are 0 and 1, scores in the thousands."""
    x = make(1, 90, 3, 2, 1, d, dtype, 5, length)
    print("case far apart", dtype, d, length, flush=True)
    out, lse = forward(x, 90, 3)
    want, tol, _, _, reach = reference(x, 90, 3)
    got = backward(x, out, lse, 90, 3)
    for n in got:
        assert bool(((got[n].double() - want[n]).abs() <= tol[n]).all()), n


@pytest.mark.parametrize("base", [2.0, 500000.0])
def test_other_rotary_bases(base):
    x = make(1, 150, 3, 2, 1, 64, "f32", 6)
    print("case base", base, flush=True)
    out, lse = forward(x, 150, 3, base)
    want, tol, _, _, reach = reference(x, 150, 3, base)
    check(x, backward(x, out, lse, 150, 3, base), want, tol, reach, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_addresses_that_are_multiples_of_4_only(dtype):
    import torch
    T, k = 45, 2
    x = make(1, T, k, 2, 1, 64, dtype, 7)
    out, lse = forward(x, T, k)
    want = backward(x, out, lse, T, k)

    def moved(t):
        n = 4 // t.element_size()
        y = torch.empty(t.numel() + n, dtype=t.dtype, device="cuda:0")[n:]
        return y.copy_(t.reshape(-1)).reshape(t.shape)
    print("case moved", dtype, flush=True)
    y = {n: moved(t) for n, t in x.items()}
    out2, lse2 = moved(out), moved(lse)
    a, got, ws = grad_args(y, out2, lse2, T, k)
    got = {n: moved(t) for n, t in got.items()}
    a.d_q, a.d_k, a.d_v = (got[n].data_ptr() for n in ("d_q", "d_k", "d_v"))
    assert TR.ps_group_attention_grad(a, _stream()) == B.PS_OK
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in got)


@pytest.mark.parametrize("dtype,T,k,d", [("bf16", 70, 4, 128), ("f32", 70, 4, 64), ("bf16", 150, 2, 64), ("bf16", 200, 0, 128)])
@pytest.mark.parametrize("what", ["k", "v", "q", "d_out"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(dtype, T, k, d, what, value):
    """Row (g, s) of one input holds Inf or NaN.  As a key or value it reaches the rows that see it, as a query or gradient
    its own row; those rows reach the keys that they see.  Everything else is what it is without them, bit for bit."""
    import torch
    x = make(1, T, k, 2, 2, d, dtype, 8)
    g, s = T - 9, min(k, 2)                                  # (k = 0: a real token)
    bad = g * (k + 1) + s
    rows = T * (k + 1)
    row = torch.arange(rows, device="cuda:0")
    grp, slot = row // (k + 1), row % (k + 1)
    sees = (row[:, None] >= row[None, :]) & ((slot[None, :] == 0) | (grp[:, None] == grp[None, :]))
    hit_rows = sees[:, bad] if what in ("k", "v") else row == bad
    hit_keys = sees[hit_rows].any(0)
    print("case not finite", dtype, T, k, d, what, value, flush=True)
    out, lse = forward(x, T, k)
    y = {n: t.clone() for n, t in x.items()}
    y[what][0, bad, 0, 5] = value
    out2, lse2 = forward(y, T, k)
    got = backward(y, out2, lse2, T, k)
    # (the forward pass works rows near such a value out by themselves, in another order: both calls get the same outputs for them)
    keep = ~hit_rows
    out[0, keep], lse[0, keep] = out2[0, keep], lse2[0, keep]
    want = backward(x, out, lse, T, k)
    assert torch.equal(got["d_q"][0, :, 1], want["d_q"][0, :, 1])           # the other head
    assert torch.equal(got["d_q"][0, ~hit_rows, 0], want["d_q"][0, ~hit_rows, 0])
    for n in ("d_k", "d_v"):
        assert torch.equal(got[n][0, :, 1], want[n][0, :, 1])
        assert torch.equal(got[n][0, ~hit_keys, 0], want[n][0, ~hit_keys, 0]), n
    if math.isnan(value):
        assert bool(torch.isnan(got["d_q"][0, hit_rows, 0]).all())
        if what in ("q", "k"):
            assert bool(torch.isnan(got["d_k"][0, hit_keys, 0]).all())


def test_gradients_against_differences():
    import torch
    T, k = 7, 2
    x = make(1, T, k, 2, 1, 64, "f32", 9)
    out, lse = forward(x, T, k)
    got = backward(x, out, lse, T, k)

    def total(y):
        _, _, o, _, _ = reference(y, T, k)
        return float((o * x["d_out"].double()).sum())
    for n, at in (("q", (0, 20, 1, 3)), ("k", (0, 9, 0, 40)), ("k", (0, 10, 0, 7)), ("v", (0, 0, 0, 63)), ("v", (0, 17, 0, 1))):
        up, down = ({m: t.double() if m != "d_out" else t for m, t in x.items()} for _ in range(2))
        up[n], down[n] = up[n].clone(), down[n].clone()
        up[n][at] += 1e-5
        down[n][at] -= 1e-5
        slope = (total(up) - total(down)) / 2e-5
        assert abs(slope - float(got["d_" + n][at])) <= 1e-5 * (1 + abs(slope)), (n, at)


def test_a_captured_call_replayed():
    """Forward and backward pass recorded into a graph, replayed with other inputs in the same buffers, eager work in between."""
    import torch
    T, k = 60, 3
    x, z = (make(1, T, k, 4, 2, 64, "bf16", s) for s in (10, 11))
    want = []
    for y in (x, z):
        out, lse = forward(y, T, k)
        want.append(backward(y, out, lse, T, k))
    buf = {n: t.clone() for n, t in x.items()}
    out, lse = torch.zeros_like(out), torch.zeros_like(lse)
    f = TR.make_args(1, T, k, 4, 2, 64, "bf16", 10000.0)
    need = TR.ps_group_attention_workspace_bytes(f)
    fws, f.workspace = _workspace(need)
    f.workspace_bytes = need
    f.q, f.k_, f.v, f.out = buf["q"].data_ptr(), buf["k"].data_ptr(), buf["v"].data_ptr(), out.data_ptr()
    a, got, ws = grad_args(buf, out, lse, T, k)
    print("case captured", flush=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert TR.ps_group_attention_lse(f, lse.data_ptr(), _stream()) == B.PS_OK
        assert TR.ps_group_attention_grad(a, _stream()) == B.PS_OK
    for turn in range(4):
        y = (x, z)[turn & 1]
        for n in buf:
            buf[n].copy_(y[n])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[turn & 1][n]) for n in got), turn


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_behind_a_shorter_sequence(dtype):
    """A padded batch: tokens behind a sequence's end with finite values and a gradient of zeros change nothing in front of them."""
    import torch
    T, k, n = 90, 3, 53
    x = make(2, T, k, 2, 1, 64, dtype, 12)
    x["d_out"][0, n * (k + 1):] = 0
    out, lse = forward(x, T, k)
    got = backward(x, out, lse, T, k)
    y = {m: t[:1, :n * (k + 1)].contiguous() for m, t in x.items()}
    want, tol, _, _, reach = reference(y, n, k)
    check(y, {m: t[:1, :n * (k + 1)] for m, t in got.items()}, want, tol, reach, dtype)
    assert all(bool((got[m][0, n * (k + 1):] == 0).all()) for m in got)
