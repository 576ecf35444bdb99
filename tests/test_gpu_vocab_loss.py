"""GPU tests of the cross entropy against the LM head and its gradient (ps_vocab_loss) against their definition in float64.

Tolerances.  A logit is a float32 sum of H products (of exact bf16 or float32 values): off by at most H 2^-24 sum |h W| in the worst
case, and by about sqrt(H) 2^-24 |h||W| in fact; tests use |logit error| <= e_l = 4 sqrt(H) 2^-24 |h| max |W_v|, and add 2^-23 of the
logit for each of the roundings on its way into the exponential.  loss: 2 e_l + 2^-20 (sums, logarithm).
d_hidden: exponentials off by a factor 1 + 2 e_l + 2^-20 (bf16: and by half a step, 2^-8, each, independently), then half a step of the
result: |error| <= w ((2 e_l + 2^-20 + 2^-24 sqrt(V)) sum_v p_v |W_v| + half steps) where bf16's half steps add up to at most
2^-8 sum_{v != t} p_v |W_v|.  The exponentials are held as exp(l_v - l_t) / 2^64, and what is below the smallest normal number 2^-126 may be
taken for zero: so a probability may be off by 2^-62 of the target's, and a gradient by w 2^-62 (sum_v |W_v| + V |W_t|)."""
import numpy as np
import pytest

from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import train as TR

pytestmark = pytest.mark.gpu

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _make(rows, H, V, dtype, seed, lean=20.0, std=0.05):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    w = (torch.randn((V, H), generator=g) * std).to(dt)
    t = torch.randint(0, V, (rows,), generator=g)
    toward = w[t].float()
    toward *= (torch.rand(rows, generator=g) * 2 - 1).clamp(min=0)[:, None] * lean / toward.square().sum(1, keepdim=True).clamp(min=1e-12)
    h = (torch.randn((rows, H), generator=g) + toward).to(dt)
    weights = torch.rand(rows, generator=g) + 0.1
    return h.cuda(), w.cuda(), t.to(torch.int32).cuda(), weights.cuda()


def _call(h, w, t, weights, dtype, grad=True, stream=None):
    import torch
    rows, H = h.shape
    loss = torch.full((rows + 8,), 77.0, device="cuda:0")
    d = torch.full((rows + 1, H), 77.0, dtype=h.dtype, device="cuda:0")
    a = TR.make_loss_args(rows, H, w.shape[0], dtype)
    a.h, a.w_lm, a.targets, a.weights = h.data_ptr(), w.data_ptr(), t.data_ptr(), weights.data_ptr() if weights is not None else None
    a.loss, a.d_hidden = loss.data_ptr(), d.data_ptr() if grad else None
    need = TR.ps_vocab_loss_workspace_bytes(a)
    ws = torch.full((need + 512,), 0xFF, dtype=torch.uint8, device="cuda:0")
    a.workspace, a.workspace_bytes = (ws.data_ptr() + 255) & ~255, need
    assert TR.ps_vocab_loss(a, torch.cuda.current_stream().cuda_stream if stream is None else stream) == B.PS_OK
    torch.cuda.synchronize()
    end = a.workspace - ws.data_ptr() + need
    assert bool((ws[end:] == 0xFF).all()) and bool((loss[rows:] == 77.0).all()) and bool((d[rows:] == 77.0).all())
    return loss[:rows], d[:rows]


def _check(h, w, t, weights, dtype, loss, d, grad=True):
    import torch
    H, V = h.shape[1], w.shape[0]
    h64, w64 = h.double(), w.double()
    logits = h64 @ w64.t()
    at = t.long()
    counts = (at >= 0) & (at < V)
    wt = (weights.double() if weights is not None else torch.ones(len(at), dtype=torch.float64, device="cuda:0")).clone()
    wt[~counts] = 0.0
    at = at.clamp(0, V - 1)
    lse = torch.logsumexp(logits, 1)
    lt = logits.gather(1, at[:, None])[:, 0]
    want = wt * (lse - lt)
    top = logits.abs().amax(1)
    e_l = 4 * H ** 0.5 * 2.0 ** -24 * h64.norm(dim=1) * w64.norm(dim=1).max() + top * 2.0 ** -22
    live = wt != 0
    assert bool((loss[~live] == 0).all())
    err = (loss.double() - want).abs()
    assert bool((err <= wt.abs() * (2 * e_l + 2.0 ** -20 * (1 + (lse - lt).abs())))[live].all()), float(err[live].max())
    print("    loss error", float(err.max()), flush=True)
    if not grad:
        return
    assert bool((d[~live] == 0).all())
    p = torch.exp(logits - lse[:, None])
    others = p.clone()
    others.scatter_(1, at[:, None], 0.0)
    want = wt[:, None] * (others @ w64 - others.sum(1, keepdim=True) * w64[at])
    size = others @ w64.abs() + others.sum(1, keepdim=True) * w64[at].abs()
    step = HALF_STEP[dtype] if dtype == "bf16" else 0.0
    tol = wt.abs()[:, None] * size * ((2 * e_l + 2.0 ** -20)[:, None] + 2.0 ** -24 * V ** 0.5 + step) + want.abs() * HALF_STEP[dtype] * 1.01
    tol += wt.abs()[:, None] * 2.0 ** -62 * (w64.abs().sum(0)[None, :] + V * w64[at].abs())
    err = (d.double() - want).abs()
    assert bool((err <= tol)[live].all()), float((err / tol.clamp(min=1e-300))[live].max())
    rel = float((d.double() - want).norm() / want.norm().clamp(min=1e-300))
    print("    d_hidden relative error", rel, flush=True)
    assert rel <= (1e-5 if dtype == "f32" else 2.0 ** -8)


CASES = [  # dtype, rows, hidden, vocab
    ("f32", 1, 16, 1), ("bf16", 1, 32, 1), ("bf16", 1, 32, 2), ("f32", 3, 48, 129),
    ("f32", 130, 256, 1024), ("bf16", 5, 512, 2064), ("bf16", 127, 96, 127), ("bf16", 129, 160, 1000), ("bf16", 257, 288, 4099),
    ("f32", 300, 80, 513), ("bf16", 1218, 1056, 3001), ("bf16", 64, 4096, 32000), ("bf16", 700, 512, 20000), ("f32", 33, 512, 2064),
    # one row and one token more and less than a tile, half a stage at the end, one stage, several chunks of rows (tiles of 64); the last: tiles
    # of 256, two pieces, many parts (those whose gradients leave the product at once: tests/test_gpu_train_paths.py)
    ("bf16", 513, 64, 257), ("bf16", 511, 32, 255), ("bf16", 300, 2080, 770), ("bf16", 1030, 4096, 1000), ("bf16", 4200, 4096, 600),
    ("bf16", 2500, 8192, 700), ("bf16", 1400, 256, 128256),
    # tiles of 128: a row more than 64, an odd number of tokens (the third: tiles of 256 with few rows and many tokens; the last: of 64, float32)
    ("bf16", 65, 96, 26001), ("bf16", 90, 128, 40001), ("bf16", 3, 64, 102400), ("bf16", 200, 160, 30100), ("f32", 65, 64, 20001)]


@pytest.mark.parametrize("dtype,rows,hidden,vocab", CASES)
def test_loss_and_gradient(dtype, rows, hidden, vocab):
    print("case loss", dtype, rows, hidden, vocab, flush=True)
    h, w, t, weights = _make(rows, hidden, vocab, dtype, rows + vocab)
    loss, d = _call(h, w, t, weights, dtype)
    _check(h, w, t, weights, dtype, loss, d)
    only, untouched = _call(h, w, t, weights, dtype, grad=False)
    assert bool((untouched == 77.0).all())
    _check(h, w, t, weights, dtype, only, None, grad=False)
    import torch
    again = _call(h, w, t, weights, dtype)                   # the same bits, whatever the workspace held
    assert torch.equal(again[0], loss) and torch.equal(again[1], d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ignored_rows_whatever_they_hold(dtype):
    h, w, t, weights = _make(40, 64, 300, dtype, 3)
    t[::3] = -100
    t[1], t[2] = 300, -1
    weights[4] = 0.0
    weights[5] = -2.5                                        # (a weight may have any sign)
    h[0], h[3], h[4] = float("nan"), float("inf"), float("nan")
    print("case ignored rows", dtype, flush=True)
    loss, d = _call(h, w, t, weights, dtype)
    h[0], h[3], h[4] = 0.0, 0.0, 0.0
    _check(h, w, t, weights, dtype, loss, d)
    import torch
    t2 = torch.full_like(t, -100)                            # nothing counts
    loss, d = _call(h, w, t2, None, dtype)
    assert bool((loss == 0).all()) and bool((d == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_whose_values_are_not_finite(dtype):
    """Inf and NaN in a row make that row's loss and gradient what they are and no other's."""
    import torch
    h, w, t, weights = _make(20, 64, 300, dtype, 4)
    h[7, 3], h[11, 5] = float("nan"), float("inf")
    print("case not finite", dtype, flush=True)
    loss, d = _call(h, w, t, weights, dtype)
    keep = torch.ones(20, dtype=torch.bool)
    keep[[7, 11]] = False
    assert bool(torch.isnan(loss[7])) and bool(torch.isnan(d[7]).all()) and not bool(torch.isfinite(loss[11]))
    _check(h[keep].contiguous(), w, t[keep].contiguous(), weights[keep].contiguous(), dtype, loss[keep], d[keep])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length", [4.0, 30.0, 300.0])
def test_logits_that_lie_far_apart(dtype, length):
    """Rows so long that logits spread over hundreds and thousands: losses from 0 to far beyond the range of exp."""
    h, w, t, weights = _make(70, 256, 700, dtype, 5, std=0.1)
    h = (h.float() * length).to(h.dtype)
    print("case far apart", dtype, length, flush=True)
    loss, d = _call(h, w, t, weights, dtype)
    print("    largest loss", float((loss / weights).max()), flush=True)
    _check(h, w, t, weights, dtype, loss, d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_are_sure_of_their_target(dtype):
    """The target's logit leads by 15 to 60: the gradient is that of the small rest, to its own relative accuracy."""
    h, w, t, weights = _make(50, 256, 500, dtype, 6, lean=0.0, std=0.02)
    toward = w[t.long()].float()
    toward = toward / toward.square().sum(1, keepdim=True)
    import torch
    lead = torch.linspace(15.0, 60.0, 50, device="cuda:0")
    h = (h.float() + toward * lead[:, None]).to(h.dtype)
    print("case sure", dtype, flush=True)
    loss, d = _call(h, w, t, weights, dtype)
    _check(h, w, t, weights, dtype, loss, d)
    want = torch.logsumexp(h.double() @ w.double().t(), 1) - (h.double() * w.double()[t.long()]).sum(1)
    sure = want > 1e-13                                      # (float64's own limit)
    assert bool(((loss / weights).double()[sure] > 0.5 * want[sure]).all()) and int(sure.sum()) > 20


def test_gradient_against_differences():
    import torch
    h, w, t, weights = _make(6, 32, 90, "f32", 9)
    _, d = _call(h, w, t, weights, "f32")
    h64, w64 = h.double(), w.double()

    def total(x):
        logits = x @ w64.t()
        return (weights.double() * (torch.logsumexp(logits, 1) - logits.gather(1, t.long()[:, None])[:, 0])).sum()
    for i, j in ((0, 0), (3, 17), (5, 31)):
        step = torch.zeros_like(h64)
        step[i, j] = 1e-4
        slope = float((total(h64 + step) - total(h64 - step)) / 2e-4)
        assert abs(slope - float(d[i, j])) <= 1e-6 + 1e-5 * abs(slope)


@pytest.mark.parametrize("rows,hidden,vocab", [(300, 512, 32000), (40, 256, 3000)])
def test_a_captured_call_replayed(rows, hidden, vocab):
    """One graph, two inputs in turn in the same buffers, an eager call and a synchronisation between replays."""
    import torch
    both = [_make(rows, hidden, vocab, "bf16", s) for s in (21, 22)]
    want = [[t.clone() for t in _call(*x, "bf16")] for x in both]
    buf = [t.clone() for t in both[0]]
    loss, d = torch.zeros(rows, device="cuda:0"), torch.zeros_like(buf[0])
    a = TR.make_loss_args(rows, hidden, vocab, "bf16")
    a.h, a.w_lm, a.targets, a.weights, a.loss, a.d_hidden = (t.data_ptr() for t in (*buf, loss, d))
    need = TR.ps_vocab_loss_workspace_bytes(a)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda:0")
    a.workspace, a.workspace_bytes = (ws.data_ptr() + 255) & ~255, need
    print("case captured loss", rows, hidden, vocab, flush=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert TR.ps_vocab_loss(a, torch.cuda.current_stream().cuda_stream) == B.PS_OK
    for turn in range(4):
        for to, x in zip(buf, both[turn & 1]):
            to.copy_(x)
        graph.replay()
        eager = _call(*both[1 - (turn & 1)], "bf16")
        torch.cuda.synchronize()
        assert torch.equal(loss, want[turn & 1][0]) and torch.equal(d, want[turn & 1][1]), turn
        assert torch.equal(eager[0], want[1 - (turn & 1)][0]) and torch.equal(eager[1], want[1 - (turn & 1)][1]), turn
