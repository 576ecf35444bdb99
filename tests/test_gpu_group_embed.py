"""GPU tests of the parallel-group layout's embeddings and their gradients (ps_group_embed, ps_group_embed_grad) against
their definition in float64.

Tolerances.  x is one float32 product, rounded once: where the product is exact in float64 too, x is that value to half a step of
its type.  A gradient is a float32 sum of n terms and one product, rounded once: its error is at most (n + 1) 2^-24 of the sum of the
terms' magnitudes (any order of adding), and half a step of the result."""
import numpy as np
import pytest

from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import train as TR

pytestmark = pytest.mark.gpu

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _torch_dtype(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def _ids(seqs, T, vocab, g, kind):
    import torch
    if kind == "same":
        ids = torch.full((seqs, T), vocab - 1)
    elif kind == "zipf":
        ids = torch.exp(torch.rand((seqs, T), generator=g, dtype=torch.float64) * np.log(vocab)).long().clamp(max=vocab) - 1
    else:
        ids = torch.randint(0, vocab, (seqs, T), generator=g)
    if kind == "padded":                                     # ids that are none: a padded batch's
        ids[:, T - T // 3:] = -1
        ids[0, 0] = vocab
        ids[-1, T // 2] = -100
    return ids.to(torch.int32).cuda()


def _offset(x, elements):
    """The same values `elements` behind the start of an allocation."""
    import torch
    y = torch.empty(x.numel() + elements, dtype=x.dtype, device=x.device)[elements:]
    y.copy_(x.reshape(-1))
    return y.reshape(x.shape)


CASES = [  # dtype, seqs, T, k, hidden, vocab, scale, ids
    ("f32", 1, 1, 0, 16, 1, 1.0, "same"),
    ("bf16", 1, 1, 15, 32, 7, 2.0, "zipf"),
    ("f32", 3, 21, 4, 256, 1024, 16.0, "zipf"),
    ("bf16", 2, 37, 2, 96, 50, 0.37, "padded"),
    ("bf16", 1, 203, 5, 5120, 32000, 1.0, "zipf"),
    ("bf16", 4, 300, 3, 512, 2064, 22.627417, "zipf"),
    ("f32", 2, 129, 1, 1040, 300, -1.5, "same"),             # one range of several windows, more pieces than threads
    ("f32", 1, 64, 0, 64, 9, 1.0, "padded"),                 # exactly one window
    ("bf16", 1, 65, 0, 64, 2, 1.0, "any"),
    ("bf16", 2, 2500, 1, 128, 40, 1.0, "any"),               # a chunk of more than 4096 positions
    ("f32", 5, 4000, 2, 64, 1000, 3.0, "zipf"),              # more than one chunk
    ("bf16", 3, 16384, 1, 32, 5, 1.0, "any"),                # whole chunks, long ranges
    ("f32", 1, 1000, 2, 8208, 17, 1.0, "padded"),            # more 16-byte pieces than a workgroup has threads
]


@pytest.mark.parametrize("dtype,seqs,T,k,hidden,vocab,scale,kind", CASES)
@pytest.mark.parametrize("shift", [0, 4])
def test_embed(dtype, seqs, T, k, hidden, vocab, scale, kind, shift):
    import torch
    print("case embed", dtype, seqs, T, k, hidden, vocab, kind, flush=True)
    g = torch.Generator().manual_seed(7)
    dt = _torch_dtype(dtype)
    ids = _ids(seqs, T, vocab, g, kind)
    n = shift // (2 if dtype == "bf16" else 4)               # pointers are aligned to 4 bytes only
    embed = _offset(torch.randn((vocab, hidden), generator=g).to(dt).cuda(), n)
    mask = _offset(torch.randn((max(k, 1), hidden), generator=g).to(dt).cuda(), n)
    x = _offset(torch.full((seqs, T * (k + 1), hidden), 77.0, dtype=dt, device="cuda:0"), n)
    a = TR.make_embed_args(seqs, T, k, hidden, vocab, dtype, scale)
    a.token_ids, a.embed, a.mask_emb, a.x = ids.data_ptr(), embed.data_ptr(), mask.data_ptr() if k else None, x.data_ptr()
    assert TR.ps_group_embed(a, _stream()) == B.PS_OK
    torch.cuda.synchronize()
    known = (ids >= 0) & (ids < vocab)
    want = torch.zeros((seqs, T, k + 1, hidden), dtype=torch.float64, device="cuda:0")
    s = float(np.float32(scale))
    want[:, :, 0] = torch.where(known[:, :, None], embed.double()[ids.long().clamp(0, vocab - 1)] * s, 0.0)
    want[:, :, 1:] = mask.double()[:k] * s
    got = x.reshape(want.shape).double()
    assert bool(((got - want).abs() <= want.abs() * (HALF_STEP[dtype] + 2.0 ** -24)).all())


@pytest.mark.parametrize("dtype,seqs,T,k,hidden,vocab,scale,kind", CASES)
def test_embed_grad(dtype, seqs, T, k, hidden, vocab, scale, kind):
    import torch
    print("case embed_grad", dtype, seqs, T, k, hidden, vocab, kind, flush=True)
    g = torch.Generator().manual_seed(8)
    dt = _torch_dtype(dtype)
    ids = _ids(seqs, T, vocab, g, kind)
    n = 4 // (2 if dtype == "bf16" else 4)
    dx = _offset(torch.randn((seqs, T * (k + 1), hidden), generator=g).to(dt).cuda(), n)
    a = TR.make_embed_grad_args(seqs, T, k, hidden, vocab, dtype, scale)
    need = TR.ps_group_embed_grad_workspace_bytes(a)

    def call(table, mask):
        d_embed = _offset(torch.full((vocab, hidden), 77.0, dtype=dt, device="cuda:0"), n)
        d_mask = _offset(torch.full((max(k, 1), hidden), 77.0, dtype=dt, device="cuda:0"), n)
        ws = torch.full((need + 512,), 0xA5, dtype=torch.uint8, device="cuda:0")
        a.token_ids, a.d_x = ids.data_ptr(), dx.data_ptr()
        a.d_embed, a.d_mask = d_embed.data_ptr() if table else None, d_mask.data_ptr() if mask else None
        a.workspace, a.workspace_bytes = (ws.data_ptr() + 255) & ~255, need
        assert TR.ps_group_embed_grad(a, _stream()) == B.PS_OK
        torch.cuda.synchronize()
        end = a.workspace - ws.data_ptr() + need
        assert bool((ws[end:] == 0xA5).all()) and bool((ws[:end - need] == 0xA5).all())
        return d_embed, d_mask[:k]

    d_embed, d_mask = call(True, k > 0)
    rows = dx.double().reshape(seqs * T, k + 1, hidden)
    flat, s = ids.long().reshape(-1), float(np.float32(scale))
    known = (flat >= 0) & (flat < vocab)
    want, size = (torch.zeros((vocab, hidden), dtype=torch.float64, device="cuda:0") for _ in range(2))
    want.index_add_(0, flat[known], rows[known, 0] * s)
    size.index_add_(0, flat[known], rows[known, 0].abs() * abs(s))
    count = torch.bincount(flat[known], minlength=vocab)[:, None]
    assert bool(((d_embed.double() - want).abs() <= size * (count + 1) * 2.0 ** -24 + want.abs() * HALF_STEP[dtype] * 1.01).all())
    assert bool((d_embed[count[:, 0] == 0] == 0).all())
    if k:
        want, size = rows[:, 1:].sum(0) * s, rows[:, 1:].abs().sum(0) * abs(s)
        assert bool(((d_mask.double() - want).abs() <= size * (seqs * T + 1) * 2.0 ** -24 + want.abs() * HALF_STEP[dtype] * 1.01).all())
        alone = call(False, True)                            # one output without the other: the same bits
        assert torch.equal(alone[1], d_mask) and bool((alone[0] == 77.0).all())
    again = call(True, False)
    assert torch.equal(again[0], d_embed)


def test_captured_calls_replayed():
    """Embeddings and their gradients in one graph (three chunks of positions), two inputs in turn, the eager calls in between."""
    import torch
    seqs, T, k, hidden, vocab = 5, 8000, 1, 64, 700
    both = []
    for seed in (31, 32):
        g = torch.Generator().manual_seed(seed)
        both.append((_ids(seqs, T, vocab, g, "zipf"), torch.randn((vocab, hidden), generator=g).cuda(), torch.randn((k, hidden), generator=g).cuda(),
                     torch.randn((seqs, T * (k + 1), hidden), generator=g).cuda()))

    def calls(ids, embed, mask, dx):
        out = [torch.full_like(t, 77.0) for t in (dx, embed, mask)]
        e, b = TR.make_embed_args(seqs, T, k, hidden, vocab, "f32", 3.0), TR.make_embed_grad_args(seqs, T, k, hidden, vocab, "f32", 3.0)
        e.token_ids, e.embed, e.mask_emb, e.x = ids.data_ptr(), embed.data_ptr(), mask.data_ptr(), out[0].data_ptr()
        b.token_ids, b.d_x, b.d_embed, b.d_mask = ids.data_ptr(), dx.data_ptr(), out[1].data_ptr(), out[2].data_ptr()
        need = TR.ps_group_embed_grad_workspace_bytes(b)
        ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda:0")
        b.workspace, b.workspace_bytes = (ws.data_ptr() + 255) & ~255, need

        def run():
            assert TR.ps_group_embed(e, _stream()) == B.PS_OK
            assert TR.ps_group_embed_grad(b, _stream()) == B.PS_OK
        return run, out, ws

    want = []
    for x in both:
        run, out, _ws = calls(*x)
        run()
        torch.cuda.synchronize()
        want.append(out)
    buf = [t.clone() for t in both[0]]
    run, out, _ws = calls(*buf)
    print("case captured embeddings", flush=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for turn in range(4):
        for to, x in zip(buf, both[turn & 1]):
            to.copy_(x)
        graph.replay()
        eager, got, _w = calls(*both[1 - (turn & 1)])
        eager()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[turn & 1])), turn
        assert all(torch.equal(a, b) for a, b in zip(got, want[1 - (turn & 1)])), turn
