"""GPU tests of the target's distributions (ps_target_probs) on crowded rows: more tokens at or near the bound than the kernels' lists hold (2048)."""
import math

import pytest

from tests import target_util as TU
from tests.test_gpu_target_probs import call, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,batch,vocab", [("f32", 4, 5000), ("bf16", 4, 32000), ("f32", 3, 128256), ("bf16", 300, 9000)])
def test_a_small_top_k_among_thousands_of_equal_tokens(dtype, batch, vocab):
    """top_k up to 512 first lists what some threads' maxima reach; here that is the whole row, and the bound is found over all of it.  Every row of the call takes that
    way, with numbers of its own."""
    import torch
    g = torch.Generator().manual_seed(vocab)
    x = torch.full((batch, 1, vocab), 1.5)
    if dtype == "f32":                                       # different numbers in one step of the histogram: 4096 of them, each for many tokens
        x[::2] += torch.randint(0, 4096, ((batch + 1) // 2, 1, vocab), generator=g) * 2.0 ** -20
    x = x.to(TU.torch_dtype(dtype)).cuda()
    r = torch.rand((batch, 1), generator=g).cuda()
    for least in (2, 17, 300):
        settings = dict(top_k=[min(512, least + 7 * b) for b in range(batch)], temperature=[1.0 + 0.25 * (b % 3) for b in range(batch)])
        for _ in range(4):
            out, ids, id_p = call(x, settings, r)
            for b in range(batch) if batch < 10 else (0, 1, 2, batch // 2, batch - 1):
                check(x[b:b + 1], {n: s[b:b + 1] for n, s in settings.items()}, r[b:b + 1], out[b:b + 1], ids[b:b + 1], id_p[b:b + 1])
            if dtype == "bf16":
                k = torch.tensor(settings["top_k"]).cuda()
                kept = (torch.arange(vocab).cuda()[None] < k[:, None])[:, None]
                assert (out > 0).equal(kept)
                assert ids.equal((r.double() * k[:, None]).floor().int())


def _crowded(vocab, seed):
    """float32 rows whose crowded step lies across a border of the numbers' exponents, with tokens of steps before it on one side."""
    import torch
    g = torch.Generator().manual_seed(seed)
    rows = []
    x = torch.full((vocab,), -9.0)                           # across 8: 10 tokens in front of the step's 1500 and 1500
    at = torch.randperm(vocab, generator=g)
    x[at[:10]], x[at[10:1510]], x[at[1510:3010]] = 8.03, 8.001, 7.999
    rows.append(x)
    x = torch.full((vocab,), -9.0)                           # across 2, every number another one
    x[at[:3500]] = 2.0 + (torch.rand(3500, generator=g) - 0.5) * 0.012
    x[at[3500:4400]] = 2.03 + torch.rand(900, generator=g) * 0.08
    x[at[4400]] = 2.0 + 5.5 * math.log(2) / 32               # (a step is 1/32 of a power of two)
    rows.append(x)
    x = torch.full((vocab,), -9.0)                           # across 0
    x[at[:4000]] = torch.randn(4000, generator=g) * 0.003
    x[at[4000:4600]] = 0.02 + torch.rand(600, generator=g) * 0.03
    rows.append(x)
    rows.append(torch.randn(vocab, generator=g) * 2.0)       # with a high temperature
    return torch.stack(rows)[:, None].contiguous(), torch.rand((4, 1), generator=g)


CROWDED = [                                                  # (the fourth row's: a temperature and a top_k for 128256 tokens, in proportion for fewer)
    dict(top_k=[700, 2000, 2500, 20000], temperature=[1.0, 1.0, 1.0, 8.0]),
    dict(top_k=[1511, 3000, 1500, 30000], temperature=[1.0, 1.0, 1.0, 16.0]),
    dict(top_p=[0.3, 0.4, 0.5, 0.3], temperature=[1.0, 1.0, 1.0, 16.0]),
    dict(top_k=[2900, 4300, 4500, 60000], top_p=[0.4, 0.6, 0.7, 0.8], temperature=[1.0, 1.0, 1.0, 20.0]),
]


def _settings(vocab, i):
    s = {n: list(x) for n, x in CROWDED[i].items()}
    s["temperature"][3] *= 128256 / vocab
    if "top_k" in s:
        s["top_k"][3] = s["top_k"][3] * vocab // 128256
    return s


@pytest.mark.parametrize("i", range(len(CROWDED)))
@pytest.mark.parametrize("vocab,copies", [(9000, 1), (40000, 1), (70000, 1), (128256, 1), (70000, 17), (9000, 70)])
def test_a_crowded_step_across_a_border_of_exponents(vocab, copies, i):
    """One workgroup per row, several, and one of 512 threads (more than 256 rows); rows behind the first are copies and have to come out as it did."""
    import torch
    x, r = _crowded(vocab, 3 * vocab + i)
    x, r = x.expand(4, copies, vocab).contiguous().cuda(), r.expand(4, copies).contiguous().cuda()
    settings = _settings(vocab, i)
    out, ids, id_p = call(x, settings, r)
    check(x, settings, r, out, ids, id_p, at=[0])
    assert out.equal(out[:, :1].expand_as(out)) and ids.equal(ids[:, :1].expand_as(ids)) and id_p.equal(id_p[:, :1].expand_as(id_p))
    again, ids2, id_p2 = call(x, settings, r)
    assert again.equal(out) and ids2.equal(ids) and id_p2.equal(id_p)


def test_top_k_of_a_flat_row():
    """20000 of 128256 tokens at a temperature of 8: a step of several hundred tokens' logits in a bucket with 20000 others, whole and cut up."""
    import torch
    x = (torch.randn((1, 1, 128256), generator=torch.Generator().manual_seed(2)) * 2.0).cuda()
    for settings in (dict(top_k=[20000], temperature=[8.0]), dict(top_k=[20000], temperature=[8.0], top_p=[1.0])):
        out, _, _ = call(x, settings)
        check(x, settings, None, out, None, None)
        assert int((out > 0).sum()) == 20000


@pytest.mark.parametrize("vocab,rows", [(50, 1), (70000, 1), (70000, 65)])
@pytest.mark.parametrize("other", [{}, dict(top_p=[1.0]), dict(top_k=[40]), dict(top_k=[1500])])
def test_a_min_p_of_almost_nothing(vocab, rows, other):
    """min_p below 2^-80, which whole masses do not resolve: kept are the e that reach it all the same, and those below have probability zero."""
    import torch
    x = torch.full((1, rows, vocab), -math.inf)
    logits = [0.0, -40.0, -55.0, -57.0, -60.0, -69.0, -69.2, -80.0, -85.0, -87.0]
    x[:, :, 3:3 + len(logits)] = torch.tensor(logits)
    r = torch.full((1, rows), 0.5)
    for min_p in (2.0 ** -79.0, 2.0 ** -80.0, 2.0 ** -80.5, 1e-25, 1e-30, 1e-35, 1e-37, 2.0 ** -126):
        out, ids, _ = call(x.cuda(), dict(min_p=[min_p], **other), r.cuda())
        least = float(torch.tensor(min_p))
        p = [math.exp(l) if math.exp(l) >= least else 0.0 for l in x[0, 0, 3:3 + len(logits)].tolist()]   # (the float32 numbers: -69.2 is none)
        want = torch.zeros(vocab, dtype=torch.float64)
        want[3:3 + len(logits)] = torch.tensor(p, dtype=torch.float64) / math.fsum(p)
        got = out[0, -1].double().cpu()
        assert (got > 0).equal(want > 0), (min_p, got[:14])
        assert ((got - want).abs() <= want * 2.0 ** -20).all()
        assert (ids == 3).all()
