"""GPU tests of the target's distributions and draws (ps_target_probs) against oracle/target.py.

Which tokens are kept and which one is drawn has to be the oracle's wherever its decisions are no closer than 1e-9 of the mass (both sides carry more than 40 bits;
cases built on a border are exact: sums of equal exponentials).  A probability is an exponential from a float32 argument in [-1/2, 1/2] (2^-25 of rounding),
1 ulp of the instruction, one factor and its own rounding: 8 half steps are allowed, 2^-21."""
import math

import numpy as np
import pytest

from oracle import target as orc
from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import verify as VF
from tests import target_util as TU

pytestmark = pytest.mark.gpu

RTOL = 2.0 ** -21


def call(logits, settings=None, r=None, probs=True, keep=None):
    """logits [batch, rows, vocab] on the GPU; settings: name -> list.  Returns probs, ids, id_probs."""
    import torch
    batch, rows, vocab = logits.shape
    a = VF.ps_target_probs_args()
    a.batch, a.rows, a.vocab, a.dtype = batch, rows, vocab, B.PS_BF16 if logits.dtype == torch.bfloat16 else B.PS_F32
    held = [torch.tensor(x, dtype=torch.int32 if n == "top_k" else torch.float32, device="cuda:0") for n, x in (settings or {}).items()]
    for n, x in zip(settings or {}, held):
        setattr(a, n, x.data_ptr())
    out = torch.full((batch, rows, vocab), -3.0, device="cuda:0") if probs else None
    ids = torch.full((batch, rows), -9, dtype=torch.int32, device="cuda:0") if r is not None else None
    id_p = torch.full((batch, rows), -3.0, device="cuda:0") if r is not None else None
    a.logits = logits.data_ptr()
    if probs:
        a.probs = out.data_ptr()
    if r is not None:
        a.r, a.ids, a.id_probs = r.data_ptr(), ids.data_ptr(), id_p.data_ptr()
    need = VF.ps_target_probs_workspace_bytes(a)
    ws, at = TU.workspace(need)
    a.workspace, a.workspace_bytes = (at, need) if need else (None, 0)
    st = VF.ps_target_probs(a, TU.stream())
    assert st == B.PS_OK, B.ps_draft_strerror(st)
    if keep is not None:
        keep.append((a, held, out, ids, id_p, ws))
    return out, ids, id_p


def check(logits, settings, r, out, ids, id_p, at=None):
    batch, rows, _ = logits.shape
    x = TU.np64(logits)
    settings = {n: np.asarray(s, dtype=np.float32 if n != "top_k" else np.int64).astype(np.float64 if n != "top_k" else np.int64) for n, s in (settings or {}).items()}
    for b in range(batch):
        for i in range(rows) if at is None else at:
            p, margin = orc.distribution(x[b, i], **{n: s[b] for n, s in settings.items()})
            assert margin > 1e-9 or margin == 0.0, "a case on a border"
            if out is not None:
                got = TU.np64(out[b, i])
                assert np.array_equal(np.isnan(got), np.isnan(p))
                assert np.array_equal(got > 2.0 ** -60, p > 2.0 ** -60), (b, i, np.nonzero((got > 0) != (p > 0))[0][:5])
                np.testing.assert_allclose(got, p, rtol=RTOL, atol=2.0 ** -60)
            if ids is not None:
                want, distance = orc.draw(p, float(r[b, i]))
                assert distance > 1e-9 or distance == 0.0
                assert int(ids[b, i]) == want, (b, i)
                np.testing.assert_allclose(float(id_p[b, i]), p[want] if want >= 0 else p[0], rtol=RTOL)


def language(batch, rows, vocab, dtype, seed):
    """Logits with a few tokens that stand out."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((batch, rows, vocab), generator=g) * 2.0
    at = torch.randint(0, vocab, (batch, rows, min(24, vocab)), generator=g)
    x.scatter_add_(2, at, torch.rand(at.shape, generator=g) * 9.0)
    return x.to(TU.torch_dtype(dtype)).cuda(), torch.rand((batch, rows), generator=g).cuda()


SETTINGS = [
    None,
    dict(temperature=[0.7, 1.3, 0.0]),
    dict(top_k=[1, 5, 0]),
    dict(top_k=[50, 3000, -1], temperature=[1.0, 0.5, 2.0]),
    dict(top_p=[0.1, 0.9, 0.999]),
    dict(min_p=[0.02, 0.5, 0.0]),
    dict(temperature=[0.8, 1.0, 1.7], top_k=[40, 7, 600], top_p=[0.95, 0.5, 0.8], min_p=[0.0, 0.1, 0.01]),
    dict(top_p=[0.0, 1.0, -1.0], min_p=[1.0, 2.0, -1.0]),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 1000, 5003])
@pytest.mark.parametrize("i", range(len(SETTINGS)))
def test_settings(dtype, vocab, i):
    logits, r = language(3, 2, vocab, dtype, 100 * i + vocab)
    out, ids, id_p = call(logits, SETTINGS[i], r)
    check(logits, SETTINGS[i], r, out, ids, id_p)
    alone, _, _ = call(logits, SETTINGS[i])
    assert alone.equal(out)
    _, ids2, id_p2 = call(logits, SETTINGS[i], r, probs=False)
    assert ids2.equal(ids) and id_p2.equal(id_p)


@pytest.mark.parametrize("dtype,vocab,rows", [("f32", 32000, 3), ("bf16", 32001, 3), ("f32", 128256, 2), ("bf16", 128256, 3), ("f32", 70001, 2), ("bf16", 300000, 1), ("f32", 1 << 20, 1)])
def test_large_vocabularies(dtype, vocab, rows):
    settings = dict(temperature=[0.9, 1.0, 1.0, 1.2], top_k=[0, 60, 0, 5000], top_p=[0.9, 0.95, 1.0, 0.7], min_p=[0.0, 0.0, 0.05, 0.0])
    logits, r = language(4, rows, vocab, dtype, vocab)
    out, ids, id_p = call(logits, settings, r)
    check(logits, settings, r, out, ids, id_p, at=range(min(rows, 2)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 9000, 70000])
def test_equal_logits_go_to_the_lowest_ids(dtype, vocab):
    """Everything equal, or two values only: thousands of tokens at one place of the order.  The sums of equal exponentials are exact, so borders are too."""
    import torch
    same = torch.full((4, 1, vocab), 1.5, dtype=TU.torch_dtype(dtype), device="cuda:0")
    r = torch.tensor([[0.0], [0.5], [0.25], [1.0 - 2.0 ** -24]], device="cuda:0")
    settings = dict(top_k=[vocab // 2, 0, 17, vocab - 1], top_p=[1.0, 0.25, 0.5, 0.75])
    out, ids, _ = call(same, settings, r)
    kept = [vocab // 2, math.ceil(0.25 * vocab), math.ceil(0.5 * 17), math.ceil(0.75 * (vocab - 1))]
    for b, n in enumerate(kept):
        assert (out[b, 0, :n] > 0).all() and (out[b, 0, n:] == 0).all(), b
        np.testing.assert_allclose(TU.np64(out[b, 0, :n]), 1.0 / n, rtol=RTOL)
        assert int(ids[b, 0]) == min(int(float(r[b, 0]) * n), n - 1)
    two = same.clone()
    two[:, :, 1::2] = -0.5
    out, _, _ = call(two, dict(top_k=[vocab // 2 + 3] * 4, min_p=[0.0, 0.2, 0.0, 0.0]), None)
    want = torch.zeros(vocab, dtype=torch.bool, device="cuda:0")
    want[0::2] = True
    full = want.clone()
    more = vocab // 2 + 3 - (vocab + 1) // 2
    full[1:2 * more:2] = True
    assert torch.equal(out[0, 0] > 0, full) and torch.equal(out[1, 0] > 0, want)


def test_zeros_of_either_sign_are_equal():
    import torch
    x = torch.tensor([[[-0.0, 0.0, -0.0, -1.0, 0.0]]], device="cuda:0")
    for k, want in ((1, [0]), (2, [0, 1]), (3, [0, 1, 2])):
        out, _, _ = call(x, dict(top_k=[k]))
        assert out[0, 0].nonzero()[:, 0].tolist() == want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_and_broken_rows(dtype):
    """Tokens at -Inf, at the type's lowest value, rows with nothing left, rows with NaN or +Inf; settings that are no numbers."""
    import torch
    x, r = language(1, 9, 777, dtype, 4)
    x[0, 0, ::3] = -math.inf
    x[0, 1, 1:] = -math.inf
    x[0, 2] = -math.inf
    x[0, 3, 776] = math.nan
    x[0, 4, 0] = math.inf
    x[0, 5, 5:] = torch.finfo(x.dtype).min
    x[0, 6] = torch.finfo(x.dtype).min
    x[0, 7, :700] = -math.inf
    for settings in (None, dict(top_k=[100], top_p=[0.9]), dict(top_p=[0.99], min_p=[0.01]), dict(top_k=[760])):
        out, ids, id_p = call(x, settings, r)
        check(x, settings, r, out, ids, id_p)
    odd = dict(temperature=[math.nan], top_p=[math.nan], min_p=[math.nan])
    out, ids, id_p = call(x, odd, r)
    check(x, dict(temperature=[0.0]), r, out, ids, id_p)
    out, ids, id_p = call(x, dict(top_p=[math.nan], min_p=[math.nan]), r)
    check(x, None, r, out, ids, id_p)
    # an infinite temperature: all that is left is equal; a tiny one: the largest
    out, _, _ = call(x, dict(temperature=[math.inf]), r)
    np.testing.assert_allclose(TU.np64(out[0, 0]), np.where(np.arange(777) % 3 == 0, 0.0, 1 / 518), rtol=RTOL)
    assert (out[0, 2] == 0).all() and torch.isnan(out[0, 3]).all()
    out, _, _ = call(x, dict(temperature=[1e-42], top_p=[0.99]), r)
    assert int((out[0, 8] > 0).sum()) == int((x[0, 8] == x[0, 8].max()).sum())


def test_rows_that_start_anywhere():
    """Odd vocabularies: rows start at any multiple of an element; what lies behind the last row stays as it was."""
    import torch
    for dtype in ("bf16", "f32"):
        for vocab in (1021, 5, 4099):
            mem = torch.randn(3 * vocab + 9, generator=torch.Generator().manual_seed(vocab)).to(TU.torch_dtype(dtype)).cuda()
            x = mem[1:1 + 3 * vocab].reshape(1, 3, vocab)
            out = torch.full((3 * vocab + 8,), -5.0, device="cuda:0")
            a = VF.ps_target_probs_args()
            a.batch, a.rows, a.vocab, a.dtype = 1, 3, vocab, B.PS_BF16 if dtype == "bf16" else B.PS_F32
            a.logits, a.probs = x.data_ptr(), out[3:].data_ptr()
            assert VF.ps_target_probs(a, TU.stream()) == B.PS_OK
            check(x, None, None, out[3:3 + 3 * vocab].reshape(1, 3, vocab), None, None)
            assert (out[:3] == -5.0).all() and (out[3 + 3 * vocab:] == -5.0).all()


def test_uniform_numbers_at_their_ends():
    import torch
    x, _ = language(1, 4, 3001, "f32", 9)
    x = x[:, :1].expand(1, 4, 3001).contiguous()
    x[0, :, :10] = -math.inf
    x[0, :, -10:] = -math.inf
    r = torch.tensor([[0.0, 1.0 - 2.0 ** -24, 1.0, math.nan]], device="cuda:0")
    _, ids, id_p = call(x, None, r)
    assert ids[0].tolist()[:1] == [10] and 10 <= int(ids[0, 1]) < 2991 and int(ids[0, 2]) == 2990 and int(ids[0, 3]) == 10
    assert (id_p > 0).all()


def test_draws_follow_the_distribution():
    import torch
    n = 1 << 14
    x, _ = language(1, 1, 50, "f32", 12)
    x = (x * 0.3).expand(1, n, 50).contiguous()
    r = ((torch.arange(n) + 0.5) / n).reshape(1, n).cuda()
    out, ids, _ = call(x, dict(top_p=[0.9]), r)
    got = torch.bincount(ids[0].long(), minlength=50).double().cpu().numpy() / n
    np.testing.assert_allclose(got, TU.np64(out[0, 0]), atol=2.0 / n)


def test_captured_and_replayed_with_other_inputs():
    import torch
    x, r = language(2, 5, 32000, "bf16", 1)
    keep = []
    call(x, dict(temperature=[0.8, 1.0], top_k=[50, 0], top_p=[0.9, 0.8], min_p=[0.0, 0.05]), r, keep=keep)
    a, held, out, ids, id_p, _ = keep[0]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert VF.ps_target_probs(a, TU.stream()) == B.PS_OK
    for step in range(4):
        new, new_r = language(2, 5, 32000, "bf16", 20 + step)
        x.copy_(new)
        r.copy_(new_r)
        settings = dict(temperature=[0.6 + 0.2 * step, 1.0], top_k=[20 * step, 100], top_p=[0.9, 1.0 - 0.1 * step], min_p=[0.0, 0.02])
        for (n, s), t in zip(settings.items(), held):
            t.copy_(torch.tensor(s))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, ids, id_p)]
        check(x, settings, r, *got, at=[0, 4])
        eager = call(x, settings, r)
        assert all(p.equal(q) for p, q in zip(eager, got))


def test_two_streams_at_once():
    import torch
    x, r = language(4, 3, 128256, "f32", 3)
    settings = dict(top_p=[0.9, 1.0, 0.5, 0.99])
    want = call(x, settings, r)
    torch.cuda.synchronize()
    got, keep = [], []
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(call(x, settings, r, keep=keep))
    torch.cuda.synchronize()
    assert all(p.equal(q) for g in got for p, q in zip(g, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_and_broken_rows_of_a_large_vocabulary(dtype):
    """The same where several workgroups share a row: what one of them sees decides for all."""
    import torch
    V = 65536 + 11
    x, r = language(1, 8, V, dtype, 5)
    x[0, 0, ::3] = -math.inf
    x[0, 1] = -math.inf
    x[0, 1, V - 1] = -2.0
    x[0, 2] = -math.inf
    x[0, 3, V - 1] = math.nan
    x[0, 4, 20000] = math.inf
    x[0, 5, 5:] = torch.finfo(x.dtype).min
    x[0, 6] = 0.25
    x[0, 7, :V - 300] = -math.inf
    odd = [1, 2, 3, 4, 5, 7]
    for settings in (None, dict(top_k=[100], top_p=[0.9]), dict(top_p=[0.99], min_p=[0.01]), dict(top_k=[40000]), dict(temperature=[0.0])):
        out, ids, id_p = call(x, settings, r)
        check(x, settings, r, out, ids, id_p, at=[0] + odd)
        _, ids2, id_p2 = call(x, settings, r, probs=False)
        assert ids2.equal(ids) and torch.equal(id_p2.nan_to_num(7.0), id_p.nan_to_num(7.0))
        alone, _, _ = call(x, settings)
        assert torch.equal(alone.nan_to_num(7.0), out.nan_to_num(7.0))
    out, ids, _ = call(x, dict(top_k=[70000], top_p=[0.5]), r)
    n = math.ceil(V / 2)
    assert (out[0, 6, :n] > 0).all() and (out[0, 6, n:] == 0).all() and int(ids[0, 6]) == min(int(float(r[0, 6]) * n), n - 1)


def test_a_row_is_the_same_alone_and_among_others():
    """One workgroup per row (many rows) or several: the same bits."""
    import torch
    x, r = language(1, 300, 70000, "bf16", 6)
    settings = dict(temperature=[0.9], top_p=[0.9])
    out, ids, id_p = call(x, settings, r)
    one, one_id, one_p = call(x[:, :100].contiguous(), settings, r[:, :100].contiguous())
    assert one.equal(out[:, :100]) and one_id.equal(ids[:, :100]) and one_p.equal(id_p[:, :100])
    few, few_id, few_p = call(x[:, 7:9].contiguous(), settings, r[:, 7:9].contiguous())
    assert few.equal(out[:, 7:9]) and few_id.equal(ids[:, 7:9]) and few_p.equal(id_p[:, 7:9])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,batch,rows", [(128256, 2, 2), (70001, 1, 64), (1 << 20, 1, 1)])
def test_greedy_ties_in_and_across_the_parts_of_a_large_row(dtype, vocab, batch, rows):
    """The largest logit at several places: the row's own lowest id, whichever workgroup had it; the settings given or not, with others or not."""
    import torch
    g = torch.Generator().manual_seed(5)
    x = (torch.rand((batch, rows, vocab), generator=g) * 4 - 8).to(TU.torch_dtype(dtype))
    first = torch.randint(0, vocab - 40000, (batch, rows), generator=g)
    for b in range(batch):
        for i in range(rows):
            at = int(first[b, i])
            x[b, i, [at, at + 1, at + 9000, at + 39000, vocab - 1]] = 1.5 - i   # (the largest of the first six rows, in bf16 of more; the others have one by chance)
    want = (x == x.amax(-1, keepdim=True)).int().argmax(-1).int().cuda()
    assert want[0, 0] == first[0, 0]
    x = x.cuda()
    r = torch.rand((batch, rows), generator=g).cuda()
    for settings in (dict(temperature=[0.0] * batch), dict(top_k=[1] * batch), dict(temperature=[0.0] * batch, top_k=[50] * batch, top_p=[0.9] * batch, min_p=[0.5] * batch)):
        out, ids, id_p = call(x, settings, r)
        assert ids.equal(want) and (id_p == 1.0).all()
        assert out.sum(-1).equal(torch.ones_like(id_p)) and out.gather(2, want[..., None].long()).eq(1.0).all()
        _, ids, _ = call(x, settings, r, probs=False)
        assert ids.equal(want)
    # all equal ones are kept where nothing filters but min_p, and the draw is among them
    out, ids, _ = call(x, dict(min_p=[0.999] * batch), r)
    kept = x.double() >= x.double().amax(-1, keepdim=True) + math.log(0.999)
    assert (out > 0).equal(kept) and (kept[0, 0].sum() == 5) and kept.gather(2, ids[..., None].long()).all()


@pytest.mark.parametrize("rows", [16, 17, 64, 65])
def test_rows_up_to_which_a_large_row_is_cut_up(rows):
    logits, r = language(1, rows, 66000, "bf16", rows)
    for settings in (dict(top_k=[40]), dict(top_p=[0.9]), dict(top_k=[40], top_p=[0.9], temperature=[0.7])):
        out, ids, id_p = call(logits, settings, r)
        check(logits, settings, r, out, ids, id_p, at=[0, 7, rows - 1])
