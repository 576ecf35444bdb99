"""GPU tests of the target's distributions (ps_target_probs) on crowded rows: more tokens at or near the bound than the kernels' lists hold (2048)."""
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
