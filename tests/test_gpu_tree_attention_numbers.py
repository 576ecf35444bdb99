"""GPU tests of the tree attention: its results are numbers wherever the definition's are (a comparison by `difference > tolerance` does not see a NaN), in every way that
calls are cut, for fused rows, device lengths and replays."""
import pytest

from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import verify as VF
from tests import target_util as TU
from tests import test_gpu_tree_attention as TA

pytestmark = pytest.mark.gpu


def finite(x):
    import torch
    return bool(torch.isfinite(x.float()).all())


@pytest.mark.parametrize("case", TA.CASES, ids=lambda c: "%s-%d-%d-%d-%s-%d" % (c[0], c[1], c[2], c[3], c[4][:4], len(c[5])))
def test_results_are_numbers(case):
    dtype, heads, nq, d, lens, parent = case
    cache, q, k, v = TA.make(dtype, heads, nq, d, lens, len(parent), seed=len(parent))
    out, lse = TA.call(cache, parent, q, k, v, list(lens), dtype)
    assert finite(out) and finite(lse)                       # (every row sees itself)
    out, lse = TA.call(cache, parent, q, None, None, list(lens), dtype)
    assert finite(out)
    for b, n in enumerate(lens):
        assert finite(lse[b]) if n else bool((lse[b] == -float("inf")).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("parent", [[-1], TA.fanout(3, 2), TA.fanout(4, 2, 2, 1, 1)], ids=len)
def test_fused_rows_device_lengths_and_replays(dtype, d, parent):
    import torch
    lens, stride = list(TA.MANY), (16 + 4 + 4) * d + 2
    cache, q, k, v = TA.make(dtype, 4, 16, d, lens, len(parent), seed=7)
    want, want_lse = TA.call(cache, parent, q, k, v, lens, dtype)
    assert finite(want) and finite(want_lse)
    fused = [TU.strided(x, stride, 2) for x in (q, k, v)]
    dev = torch.tensor(lens, dtype=torch.int32, device="cuda:0")
    keep = []
    out, lse = TA.call(cache, parent, *fused, lens, dtype, q_stride=stride, kv_stride=stride, dev=dev, keep=keep)
    assert out.equal(want) and lse.equal(want_lse)
    tree, a = keep[0][:2]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert VF.ps_tree_attention(tree, a, TU.stream()) == B.PS_OK
    for turn in range(3):
        now = [n * (3 - turn) // 3 for n in lens]
        dev.copy_(torch.tensor(now, dtype=torch.int32))
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert finite(out) and finite(lse)
        TA.check(cache, parent, q, k, v, now, dtype, out, lse, heads=[1])
