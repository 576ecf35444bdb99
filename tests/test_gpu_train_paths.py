"""GPU tests of the training operators' kernels that large calls take: every case says how its call is cut, as the library itself plans it, so that a
change of the rules cannot leave a kernel without a test.  References and tolerances are those of the operators' own tests.

Attention's gradients: one wavefront for 32 query rows (kw 1, from 256 blocks of query rows on), 128 keys of head_dim 64 in a workgroup, one and several
parts of a key tile's rows.  Loss: tiles of 256 whose gradients leave the last product at once (one part), with one and several pieces of the vocabulary,
several chunks of rows, a last tile of few rows and columns."""
import pytest

import tests.test_gpu_group_attention_grad as AG
import tests.test_gpu_vocab_loss as VL
from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import debug as DBG
from paper_2410_05589_amd import train as TR

pytestmark = pytest.mark.gpu


def _attention_plan(dtype, seqs, T, k, nq, nkv, d):
    st, plan = DBG.ps_train_debug_grad_plan(TR.make_grad_args(seqs, T, k, nq, nkv, d, dtype, 10000.0))
    assert st == B.PS_OK
    return plan["kw"], plan["keys"], plan["parts"]


GRADIENTS = [  # dtype, seqs, T, k, heads, kv heads, head_dim; (kw, keys, parts)
    (("bf16", 4, 37, 4, 32, 8, 128), (1, 128, 3)), (("f32", 4, 50, 2, 32, 16, 64), (1, 64, 3)), (("f32", 2, 45, 6, 44, 11, 128), (1, 64, 10)),
    (("bf16", 2, 203, 2, 26, 26, 64), (1, 64, 2)), (("bf16", 4, 520, 1, 8, 4, 128), (1, 128, 3)), (("bf16", 1, 1000, 0, 32, 4, 128), (1, 128, 8)),
    (("bf16", 4, 140, 1, 32, 32, 64), (1, 128, 1)), (("f32", 4, 140, 1, 32, 32, 64), (1, 128, 1)), (("bf16", 2, 300, 3, 64, 16, 128), (1, 128, 2)),
    (("f32", 2, 261, 2, 24, 24, 128), (1, 64, 1)),
    (("bf16", 16, 130, 15, 32, 8, 64), (1, 128, 2)),
]


@pytest.mark.parametrize("case,plan", GRADIENTS)
def test_gradients_of_large_calls(case, plan):
    import torch
    dtype, seqs, T, k, nq, nkv, d = case
    assert _attention_plan(*case) == plan
    print("case grad", case, plan, flush=True)
    x = AG.make(seqs, T, k, nq, nkv, d, dtype, T + k)
    out, lse = AG.forward(x, T, k)
    want, tol, _, lse64, reach = AG.reference(x, T, k)
    flip = 2.0 ** -7 * 25.0 / d ** 0.5 if dtype == "bf16" else 0.0   # (as in the gradients' own tests)
    assert float((lse - lse64).abs().max()) <= 2.0 ** -18 * (1 + reach) + flip
    got = AG.backward(x, out, lse, T, k)
    AG.check(x, got, want, tol, reach, dtype)
    again = AG.backward(x, out, lse, T, k)
    assert all(torch.equal(got[n], again[n]) for n in got)


HIDDEN = [("bf16", 3300, 4, 128, (1, 128, 4)), ("f32", 3300, 4, 64, (1, 64, 4)), ("bf16", 5500, 2, 64, (1, 64, 4))]   # two heads, one sequence


@pytest.mark.parametrize("dtype,T,k,d,plan", HIDDEN)
@pytest.mark.parametrize("what", ["k", "v", "q", "d_out"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_values_that_are_not_finite_in_large_calls(dtype, T, k, d, plan, what, value):
    assert _attention_plan(dtype, 1, T, k, 2, 2, d) == plan
    AG.test_values_that_are_not_finite_stay_with_the_rows_that_see_them(dtype, T, k, d, what, value)


@pytest.mark.parametrize("case,plan", [GRADIENTS[0], GRADIENTS[1], GRADIENTS[6]])
def test_addresses_that_are_multiples_of_4_only_in_large_calls(case, plan):
    import torch
    dtype, seqs, T, k, nq, nkv, d = case
    assert _attention_plan(*case) == plan
    print("case moved", case, flush=True)
    x = AG.make(seqs, T, k, nq, nkv, d, dtype, 17)
    out, lse = AG.forward(x, T, k)
    want = AG.backward(x, out, lse, T, k)

    def moved(t):
        n = 4 // t.element_size()
        y = torch.empty(t.numel() + n, dtype=t.dtype, device="cuda:0")[n:]
        return y.copy_(t.reshape(-1)).reshape(t.shape)
    y, out, lse = {n: moved(t) for n, t in x.items()}, moved(out), moved(lse)
    a, got, _ws = AG.grad_args(y, out, lse, T, k)
    got = {n: moved(t) for n, t in got.items()}
    a.d_q, a.d_k, a.d_v = (got[n].data_ptr() for n in ("d_q", "d_k", "d_v"))
    assert TR.ps_group_attention_grad(a, AG._stream()) == B.PS_OK
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in got)


LOSSES = [  # rows, hidden, vocab; (rows of a chunk, tokens of a piece, parts, of the last chunk)
    ((4096, 4096, 2064), (4096, 2304, 1, 1)),                # whole tiles, one chunk
    ((7780, 4128, 2064), (3840, 2304, 1, 3)),                # three chunks, the last one in parts; a column tile of 32
    ((33000, 288, 4700), (32768, 2560, 1, 5)),               # two pieces; a column tile of 32
    ((65400, 32, 2400), (65400, 1280, 1, 1)),                # two pieces, one stage of the contraction, a row tile of 120
]


def _loss_plan(rows, hidden, vocab):
    a = TR.make_loss_args(rows, hidden, vocab, "bf16")
    a.d_hidden = 0x100000
    st, plan = DBG.ps_train_debug_loss_plan(a)
    assert st == B.PS_OK and plan["tile"] == 256
    return plan["rows"], plan["piece"], plan["parts"], plan["last_parts"]


@pytest.mark.parametrize("case,plan", LOSSES)
def test_loss_whose_gradients_leave_the_product_at_once(case, plan):
    import torch
    rows, hidden, vocab = case
    assert _loss_plan(*case) == plan
    print("case loss", case, plan, flush=True)
    x = VL._make(rows, hidden, vocab, "bf16", rows + vocab)
    loss, d = VL._call(*x, "bf16")
    VL._check(*x, "bf16", loss, d)
    only, untouched = VL._call(*x, "bf16", grad=False)
    assert bool((untouched == 77.0).all())
    VL._check(*x, "bf16", only, None, grad=False)
    again = VL._call(*x, "bf16")
    assert torch.equal(again[0], loss) and torch.equal(again[1], d)


@pytest.mark.parametrize("case,plan", LOSSES)
def test_rows_of_every_kind_side_by_side(case, plan):
    """Ignored rows whatever they hold, weights of zero, rows whose logits lie far apart (alone, four in a row, across a chunk's end), Inf and NaN."""
    import torch
    rows, hidden, vocab = case
    assert _loss_plan(*case) == plan
    print("case kinds", case, flush=True)
    h, w, t, weights = VL._make(rows, hidden, vocab, "bf16", 5, lean=0.0)
    at = torch.arange(rows, device="cuda:0")
    far = torch.tensor(sorted({0, 9, 256, 257, 258, 259, 511, plan[0] - 1, plan[0] % rows, rows - 2}), device="cuda:0")
    h[far] = (h[far].float() * 3000.0 / hidden ** 0.5 / 0.05).to(h.dtype)
    none = (at % 7 == 3) & ~torch.isin(at, far)
    t[none] = torch.tensor([-100, -1, vocab, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda:0")[at[none] % 5]
    zero = (at % 11 == 5) & ~torch.isin(at, far)
    weights[zero] = 0.0
    weights[at % 13 == 1] *= -1.0
    h[(at % 25 == 4) & ~torch.isin(at, far)] = float("nan")  # (rows without a target among them, and others)
    h[(at % 77 == 5) & zero] = float("inf")
    odd = ~torch.isfinite(h.float()).all(1)
    ignored = none | zero
    loss, d = VL._call(h, w, t, weights, "bf16")
    bad = odd & ~ignored
    assert bool(torch.isnan(loss[bad]).all()) and bool(torch.isnan(d[bad]).all()) and int(bad.sum()) > 0
    h[odd] = 0.0
    keep = ~bad
    logits = h[far].double() @ w.double().t()
    apart = logits.amax(1) - logits.gather(1, t[far].long().clamp(0, vocab - 1)[:, None])[:, 0]
    assert int((apart > 110).sum()) >= 5
    VL._check(h[keep], w, t[keep], weights[keep], "bf16", loss[keep], d[keep])
    only, _ = VL._call(h, w, t, weights, "bf16", grad=False)
    VL._check(h, w, t, weights, "bf16", only, None, grad=False)


def test_a_captured_call_of_large_tiles_replayed():
    assert _loss_plan(4100, 4096, 2064)[2:] == (1, 4)
    VL.test_a_captured_call_replayed(4100, 4096, 2064)


@pytest.mark.parametrize("rows,hidden,vocab,plan", [(5000, 1024, 20001, (64, 4096, 10048, 1, 4))])
def test_loss_of_float32_in_pieces(rows, hidden, vocab, plan):
    """Products that go on from what the pieces before have left, in two chunks of rows, the second one's in parts."""
    a = TR.make_loss_args(rows, hidden, vocab, "f32")
    a.d_hidden = 0x100000
    st, got = DBG.ps_train_debug_loss_plan(a)
    assert st == B.PS_OK and (got["tile"], got["rows"], got["piece"], got["parts"], got["last_parts"]) == plan, got
    print("case loss f32", rows, hidden, vocab, plan, flush=True)
    x = VL._make(rows, hidden, vocab, "f32", 31)
    loss, d = VL._call(*x, "f32")
    VL._check(*x, "f32", loss, d)


def test_losses_of_the_largest_vocabulary():
    """More tiles than one launch takes: losses only, 2^16 rows against 2^23 tokens, in two pieces.  Some rows are checked."""
    import torch
    rows, hidden, vocab = 1 << 16, 32, 1 << 23
    a = TR.make_loss_args(rows, hidden, vocab, "bf16")
    st, plan = DBG.ps_train_debug_loss_plan(a)
    assert st == B.PS_OK and (plan["tile"], plan["rows"], plan["piece"]) == (256, rows, vocab // 2)
    print("case largest vocabulary", flush=True)
    g = torch.Generator(device="cuda:0").manual_seed(41)
    w = (torch.randn((vocab, hidden), generator=g, device="cuda:0") * 0.05).to(torch.bfloat16)
    h = torch.randn((rows, hidden), generator=g, device="cuda:0").to(torch.bfloat16)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda:0").to(torch.int32)
    t[0], t[1], t[rows - 1] = vocab - 1, vocab // 2, 0
    loss, _ = VL._call(h, w, t, None, "bf16", grad=False)
    assert bool(torch.isfinite(loss).all())
    some = torch.tensor([0, 1, 255, 256, 4097, 65279, rows - 1], device="cuda:0")
    VL._check(h[some], w, t[some], None, "bf16", loss[some], None, grad=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,hidden,vocab", [(70, 64, 1), (70, 64, 2), (300, 64, 900), (4200, 4096, 2064)])
def test_targets_whose_logit_is_not_finite(dtype, rows, hidden, vocab):
    """log(sum exp) - l_t where l_t is Inf or NaN: NaN, unless every other logit is finite or Inf and l_t -Inf (Inf); never a loss of zero."""
    import torch
    h, w, t, _ = VL._make(rows, hidden, vocab, dtype, 51)
    w[:, 7] = w[:, 7].float().clamp(max=-1e-3).to(w.dtype)   # (the row's others: -Inf, so that nothing but the target's logit shows it)
    t[:] = vocab - 1
    w[vocab - 1, 7] = 0.03
    print("case target not finite", dtype, rows, hidden, vocab, flush=True)
    want, want_d = VL._call(h, w, t, None, dtype)
    h[rows // 2, 7], h[rows - 1, 7] = float("inf"), float("nan")
    for grad in (True, False):
        loss, d = VL._call(h, w, t, None, dtype, grad=grad)
        hit = torch.zeros(rows, dtype=torch.bool, device="cuda:0")
        hit[[rows // 2, rows - 1]] = True
        assert bool(torch.isnan(loss[hit]).all()), loss[hit]
        assert torch.equal(loss[~hit], want[~hit])
        if grad:
            assert bool(torch.isnan(d[hit]).all()) and torch.equal(d[~hit], want_d[~hit])


FORWARD = [  # dtype, seqs, T, k, heads, kv heads, head_dim; kernel, as ps_train_debug_launch numbers it
    (("bf16", 1, 1, 4, 2, 1, 128), 1), (("bf16", 1, 5, 4, 2, 1, 128), 1), (("bf16", 1, 3, 4, 4, 2, 64), 1), (("bf16", 2, 16, 8, 4, 2, 64), 1), (("bf16", 2, 16, 8, 4, 2, 128), 1),
    (("bf16", 1, 70, 0, 2, 1, 128), 2), (("f32", 1, 1000, 3, 8, 8, 64), 3), (("f32", 1, 700, 3, 8, 4, 64), 4), (("f32", 1, 400, 4, 8, 4, 128), 0),
]


@pytest.mark.parametrize("length", [1.0, 30.0])
@pytest.mark.parametrize("case,kernel", FORWARD)
def test_log_sums_of_every_forward_kernel(case, kernel, length):
    """Also of queries 30 times as long (log sums up to hundreds): float32 leaves 2^-18 (1 + reach), a rotated bf16 key e_s (see the gradients' tests)."""
    import torch
    dtype, seqs, T, k, nq, nkv, d = case
    st, launch = DBG.ps_train_debug_launch(TR.make_args(seqs, T, k, nq, nkv, d, dtype, 10000.0))
    assert st == B.PS_OK and launch["kernel"] == kernel
    print("case log sums", case, length, flush=True)
    x = AG.make(seqs, T, k, nq, nkv, d, dtype, 61, length)
    out, lse = AG.forward(x, T, k)
    plain, _ = AG.forward(x, T, k, lse=False)
    assert torch.equal(out, plain)
    _, _, out64, lse64, reach = AG.reference(x, T, k)
    flip = 2.0 ** -7 * 25.0 * length / d ** 0.5 if dtype == "bf16" else 0.0
    assert float((lse - lse64).abs().max()) <= 2.0 ** -18 * (1 + reach) + flip
