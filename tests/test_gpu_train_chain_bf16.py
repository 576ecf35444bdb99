"""GPU test of the training operators in bf16 as a training step uses them together, at sizes that take the kernels of large calls: token ids -> rows of the
parallel layout -> attention -> cross entropy against the frozen LM head -> the attention's gradients -> the tables' gradients, with plain projections in
between.  Each operator's outputs are compared with its definition in float64 on what the step itself had in its buffers, to the tolerances of the
operator's own tests; the step is captured and replayed, and gives the same bits as when it runs eagerly."""
import pytest

import tests.test_gpu_group_attention_grad as AG
import tests.test_gpu_vocab_loss as VL
from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import debug as DBG
from paper_2410_05589_amd import train as TR

pytestmark = pytest.mark.gpu

SEQS, T, K, HEADS, KV, D, VOCAB, SCALE = 4, 70, 4, 32, 8, 64, 8001, 3.0
H, ROWS = HEADS * D, T * (K + 1)
N = SEQS * ROWS


def _params(seed):
    import torch
    g = torch.Generator().manual_seed(seed)

    def n(*shape, std):
        return (torch.randn(shape, generator=g) * std).to(torch.bfloat16).cuda()
    p = {"embed": n(VOCAB, H, std=0.3), "mask": n(K, H, std=0.3), "wq": n(H, HEADS * D, std=0.02), "wk": n(H, KV * D, std=0.02),
         "wv": n(H, KV * D, std=0.02), "wo": n(HEADS * D, H, std=0.02), "lm": n(VOCAB, H, std=0.02)}
    ids = torch.randint(0, VOCAB, (SEQS, T), generator=g).to(torch.int32)
    ids[0, T - 9:] = -1                                      # a padded sequence
    group, slot = torch.arange(ROWS) // (K + 1), torch.arange(ROWS) % (K + 1)
    at = group + slot + 1
    targets = torch.where(at < T, ids[:, at.clamp(max=T - 1)].long(), -100)
    targets[ids[:, group] < 0] = -100
    weights = (0.8 ** slot.double()).float().repeat(SEQS)
    return p, ids.cuda(), targets.reshape(-1).to(torch.int32).cuda(), weights.cuda()


class Step:
    """Every buffer of a step and the calls on it, on the current stream; one workspace for all of them."""

    def __init__(self, p, ids, targets, weights):
        import torch
        self.p, self.ids, self.targets, self.weights = p, ids, targets, weights

        def new(*shape, dtype=torch.bfloat16):
            return torch.full(shape, 77.0, dtype=dtype, device="cuda:0")
        f32 = torch.float32
        self.x, self.h, self.d_h, self.d_x = (new(N, H) for _ in range(4))
        self.out, self.lse, self.loss = new(SEQS, ROWS, HEADS, D, dtype=f32), new(SEQS, ROWS, HEADS, dtype=f32), new(N, dtype=f32)
        self.q, self.d_q, self.d_out, self.out16 = (new(N, HEADS * D) for _ in range(4))
        self.k, self.v, self.d_k, self.d_v = (new(N, KV * D) for _ in range(4))
        self.d_embed, self.d_mask = new(VOCAB, H), new(K, H)
        e = TR.make_embed_args(SEQS, T, K, H, VOCAB, "bf16", SCALE)
        e.token_ids, e.embed, e.mask_emb, e.x = ids.data_ptr(), p["embed"].data_ptr(), p["mask"].data_ptr(), self.x.data_ptr()
        a = TR.make_args(SEQS, T, K, HEADS, KV, D, "bf16", 10000.0)
        a.q, a.k_, a.v, a.out = self.q.data_ptr(), self.k.data_ptr(), self.v.data_ptr(), self.out.data_ptr()
        c = TR.make_loss_args(N, H, VOCAB, "bf16")
        c.h, c.w_lm, c.targets, c.weights = self.h.data_ptr(), p["lm"].data_ptr(), targets.data_ptr(), weights.data_ptr()
        c.loss, c.d_hidden = self.loss.data_ptr(), self.d_h.data_ptr()
        b = TR.make_grad_args(SEQS, T, K, HEADS, KV, D, "bf16", 10000.0)
        b.q, b.k_, b.v, b.out, b.lse, b.d_out = (t.data_ptr() for t in (self.q, self.k, self.v, self.out, self.lse, self.d_out))
        b.d_q, b.d_k, b.d_v = self.d_q.data_ptr(), self.d_k.data_ptr(), self.d_v.data_ptr()
        f = TR.make_embed_grad_args(SEQS, T, K, H, VOCAB, "bf16", SCALE)
        f.token_ids, f.d_x, f.d_embed, f.d_mask = ids.data_ptr(), self.d_x.data_ptr(), self.d_embed.data_ptr(), self.d_mask.data_ptr()
        needs = (TR.ps_group_attention_workspace_bytes(a), TR.ps_vocab_loss_workspace_bytes(c), TR.ps_group_attention_grad_workspace_bytes(b),
                 TR.ps_group_embed_grad_workspace_bytes(f))
        self.ws = torch.full((max(needs) + 256,), 0xFF, dtype=torch.uint8, device="cuda:0")
        for args, need in zip((a, c, b, f), needs):
            args.workspace, args.workspace_bytes = (self.ws.data_ptr() + 255) & ~255, need
        self.args = e, a, c, b, f

    def run(self):
        import torch
        p, (e, a, c, b, f) = self.p, self.args
        s = torch.cuda.current_stream().cuda_stream
        assert TR.ps_group_embed(e, s) == B.PS_OK
        for w, t in (("wq", self.q), ("wk", self.k), ("wv", self.v)):
            torch.mm(self.x, p[w], out=t)
        assert TR.ps_group_attention_lse(a, self.lse.data_ptr(), s) == B.PS_OK
        self.out16.copy_(self.out.view(N, -1))
        torch.addmm(self.x, self.out16, p["wo"], out=self.h)
        assert TR.ps_vocab_loss(c, s) == B.PS_OK
        torch.mm(self.d_h, p["wo"].t(), out=self.d_out)
        assert TR.ps_group_attention_grad(b, s) == B.PS_OK
        self.d_x.copy_(self.d_h)
        for w, t in (("wq", self.d_q), ("wk", self.d_k), ("wv", self.d_v)):
            self.d_x.addmm_(t, p[w].t())
        assert TR.ps_group_embed_grad(f, s) == B.PS_OK

    def results(self):
        return {n: getattr(self, n).clone() for n in ("x", "out", "lse", "loss", "d_h", "d_q", "d_k", "d_v", "d_x", "d_embed", "d_mask")}


def test_every_operator_of_a_step_against_its_definition():
    import torch
    st, plan = DBG.ps_train_debug_grad_plan(TR.make_grad_args(SEQS, T, K, HEADS, KV, D, "bf16", 10000.0))
    assert st == B.PS_OK and plan["kw"] == 1
    step = Step(*_params(3))
    print("case step bf16", flush=True)
    step.run()
    torch.cuda.synchronize()
    p, ids = step.p, step.ids.long().reshape(-1)
    known = ids >= 0
    # embeddings: one product, one rounding
    want = torch.cat((torch.where(known[:, None], p["embed"].double()[ids.clamp(min=0)], 0.0)[:, None], p["mask"].double().expand(SEQS * T, K, H)), 1) * SCALE
    assert bool(((step.x.double() - want.reshape(N, H)).abs() <= want.reshape(N, H).abs() * (2.0 ** -8 + 2.0 ** -24)).all())
    # attention and its gradients
    x = {"q": step.q.view(SEQS, ROWS, HEADS, D), "k": step.k.view(SEQS, ROWS, KV, D), "v": step.v.view(SEQS, ROWS, KV, D),
         "d_out": step.d_out.view(SEQS, ROWS, HEADS, D)}
    want, tol, _, _, reach = AG.reference(x, T, K)
    AG.check(x, {n: getattr(step, n).view(want[n].shape) for n in want}, want, tol, reach, "bf16")
    # loss
    VL._check(step.h, p["lm"], step.targets, step.weights, "bf16", step.loss, step.d_h)
    # the tables' gradients: float32 sums, rounded once
    d = step.d_x.double().view(SEQS * T, K + 1, H) * SCALE
    want, size = (torch.zeros((VOCAB, H), dtype=torch.float64, device="cuda:0") for _ in range(2))
    want.index_add_(0, ids[known], d[known, 0])
    size.index_add_(0, ids[known], d[known, 0].abs())
    count = torch.bincount(ids[known], minlength=VOCAB)[:, None]
    assert bool(((step.d_embed.double() - want).abs() <= size * (count + 1) * 2.0 ** -24 + want.abs() * 2.0 ** -8 * 1.01).all())
    want, size = d[:, 1:].sum(0), d[:, 1:].abs().sum(0)
    assert bool(((step.d_mask.double() - want).abs() <= size * (SEQS * T + 1) * 2.0 ** -24 + want.abs() * 2.0 ** -8 * 1.01).all())


def test_a_step_captured_and_replayed():
    import torch
    one, two = _params(4), _params(5)
    want = []
    for y in (one, two):
        step = Step(*y)
        step.run()
        torch.cuda.synchronize()
        want.append(step.results())
    buf = tuple({n: t.clone() for n, t in x.items()} if isinstance(x, dict) else x.clone() for x in one)
    step = Step(*buf)
    print("case captured step bf16", flush=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()                                           # (the library's own products set up what they need)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    for turn in range(4):
        y, w = ((two, want[1]), (one, want[0]))[turn & 1]
        for n in buf[0]:
            buf[0][n].copy_(y[0][n])
        for to, t in zip(buf[1:], y[1:]):
            to.copy_(t)
        graph.replay()
        eager = Step(*y)
        eager.run()
        torch.cuda.synchronize()
        got, eager = step.results(), eager.results()
        assert all(torch.equal(got[n], w[n]) and torch.equal(eager[n], w[n]) for n in w), turn
