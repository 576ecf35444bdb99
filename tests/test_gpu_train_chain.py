"""GPU tests of the training operators as a training step uses them together: token ids -> rows of the parallel layout (ps_group_embed) -> attention
(ps_group_attention_lse) -> cross entropy against the frozen LM head (ps_vocab_loss) -> the attention's gradients -> the tables' gradients
(ps_group_embed_grad), with a plain projection in between; the whole against float64 automatic differentiation, in one captured graph, and on
another stream.

Tolerances (float32, 2-norms relative to the gradient's).  Each operator adds at most 2e-6 (its own tests) and each of the six small
products with H = 64 terms at most sqrt(64) 2^-24 = 5e-7; errors are carried on by factors of the size of the products themselves.  Of the
ten operations on the way to the tables a factor of at most 4 each on the relative error leaves 4 (4 2e-6 + 6 5e-7) = 4.4e-5; tested 1e-4 for
gradients and 1e-5 for the loss (a mean of logarithms of sums, 64 products)."""
import math

import pytest

from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import train as TR

pytestmark = pytest.mark.gpu

SEQS, T, K, HEADS, KV, D, VOCAB = 2, 41, 3, 4, 2, 64, 503
H, ROWS = HEADS * D, T * (K + 1)


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def _ws(need):
    import torch
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda:0")
    return ws, (ws.data_ptr() + 255) & ~255


def _params(seed):
    import torch
    g = torch.Generator().manual_seed(seed)

    def n(*shape, std):
        return (torch.randn(shape, generator=g) * std).cuda()
    p = {"embed": n(VOCAB, H, std=0.05), "mask": n(K, H, std=0.05), "wq": n(H, HEADS * D, std=0.2), "wk": n(H, KV * D, std=0.2),
         "wv": n(H, KV * D, std=0.2), "wo": n(HEADS * D, H, std=0.2), "lm": n(VOCAB, H, std=0.1)}
    ids = torch.randint(0, VOCAB, (SEQS, T), generator=g).to(torch.int32)
    ids[0, T - 9:] = -1                                      # a padded sequence
    group, slot = torch.arange(ROWS) // (K + 1), torch.arange(ROWS) % (K + 1)
    at = group + slot + 1
    targets = torch.where(at < T, ids[:, at.clamp(max=T - 1)].long(), -100)
    targets[(ids[:, group] < 0)] = -100                      # rows of tokens that are none
    targets[targets < 0] = -100
    weights = (0.8 ** slot.double() / (targets >= 0).sum()).float().repeat(SEQS)
    return p, ids.cuda(), targets.reshape(-1).to(torch.int32).cuda(), weights.cuda()


class Step:
    """Every buffer of a step and the calls on it, on the current stream."""

    def __init__(self, p, ids, targets, weights):
        import torch
        self.p, n = p, SEQS * ROWS

        def new(*shape):
            return torch.full(shape, 77.0, device="cuda:0")
        self.x, self.out, self.lse, self.loss = new(SEQS, ROWS, H), new(SEQS, ROWS, HEADS, D), new(SEQS, ROWS, HEADS), new(n)
        self.q, self.kk, self.v = new(n, HEADS * D), new(n, KV * D), new(n, KV * D)
        self.h, self.d_h, self.d_out, self.d_x = new(n, H), new(n, H), new(n, HEADS * D), new(n, H)
        self.d_q, self.d_k, self.d_v = new(n, HEADS * D), new(n, KV * D), new(n, KV * D)
        self.d_embed, self.d_mask = new(VOCAB, H), new(K, H)
        self.keep = [ids, targets, weights]
        e = TR.make_embed_args(SEQS, T, K, H, VOCAB, "f32", 2.0)
        e.token_ids, e.embed, e.mask_emb, e.x = ids.data_ptr(), p["embed"].data_ptr(), p["mask"].data_ptr(), self.x.data_ptr()
        a = TR.make_args(SEQS, T, K, HEADS, KV, D, "f32", 10000.0)
        a.q, a.k_, a.v, a.out = self.q.data_ptr(), self.kk.data_ptr(), self.v.data_ptr(), self.out.data_ptr()
        c = TR.make_loss_args(n, H, VOCAB, "f32")
        c.h, c.w_lm, c.targets, c.weights = self.h.data_ptr(), p["lm"].data_ptr(), targets.data_ptr(), weights.data_ptr()
        c.loss, c.d_hidden = self.loss.data_ptr(), self.d_h.data_ptr()
        b = TR.make_grad_args(SEQS, T, K, HEADS, KV, D, "f32", 10000.0)
        b.q, b.k_, b.v, b.out, b.lse, b.d_out = (t.data_ptr() for t in (self.q, self.kk, self.v, self.out, self.lse, self.d_out))
        b.d_q, b.d_k, b.d_v = self.d_q.data_ptr(), self.d_k.data_ptr(), self.d_v.data_ptr()
        f = TR.make_embed_grad_args(SEQS, T, K, H, VOCAB, "f32", 2.0)
        f.token_ids, f.d_x, f.d_embed, f.d_mask = ids.data_ptr(), self.d_x.data_ptr(), self.d_embed.data_ptr(), self.d_mask.data_ptr()
        needs = (TR.ps_group_attention_workspace_bytes(a), TR.ps_vocab_loss_workspace_bytes(c), TR.ps_group_attention_grad_workspace_bytes(b),
                 TR.ps_group_embed_grad_workspace_bytes(f))
        ws, at = _ws(max(needs))                             # one workspace: the calls follow each other on a stream
        self.keep.append(ws)
        for args, need in zip((a, c, b, f), needs):
            args.workspace, args.workspace_bytes = at, need
        self.args = e, a, c, b, f

    def run(self):
        import torch
        p, (e, a, c, b, f) = self.p, self.args
        flat, s = self.x.view(-1, H), _stream()
        assert TR.ps_group_embed(e, s) == B.PS_OK
        for w, t in (("wq", self.q), ("wk", self.kk), ("wv", self.v)):
            torch.mm(flat, p[w], out=t)
        assert TR.ps_group_attention_lse(a, self.lse.data_ptr(), s) == B.PS_OK
        torch.addmm(flat, self.out.view(-1, HEADS * D), p["wo"], out=self.h)
        assert TR.ps_vocab_loss(c, s) == B.PS_OK
        torch.mm(self.d_h, p["wo"].t(), out=self.d_out)
        assert TR.ps_group_attention_grad(b, s) == B.PS_OK
        self.d_x.copy_(self.d_h)
        for w, t in (("wq", self.d_q), ("wk", self.d_k), ("wv", self.d_v)):
            self.d_x.addmm_(t, p[w].t())
        assert TR.ps_group_embed_grad(f, s) == B.PS_OK

    def results(self):
        return {n: getattr(self, n).clone() for n in ("loss", "d_h", "d_q", "d_k", "d_v", "d_x", "d_embed", "d_mask")}


def _reference(p, ids, targets, weights):
    import torch
    q = {n: t.double().requires_grad_(n in ("embed", "mask")) for n, t in p.items()}
    ids = ids.long()
    real = torch.where((ids >= 0)[..., None], q["embed"][ids.clamp(min=0)], torch.zeros((), dtype=torch.float64, device="cuda:0"))
    x = torch.cat((real[:, :, None], q["mask"].expand(SEQS, T, K, H)), 2).reshape(SEQS, ROWS, H) * 2.0
    row = torch.arange(ROWS, device="cuda:0")
    g, slot = row // (K + 1), row % (K + 1)
    sees = (row[:, None] >= row[None, :]) & ((slot[None, :] == 0) | (g[:, None] == g[None, :]))
    angle = (g + slot).double()[:, None] * 10000.0 ** (-2.0 * torch.arange(D // 2, device="cuda:0", dtype=torch.float64) / D)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def turn(y):
        u, w = y[..., :D // 2], y[..., D // 2:]
        return torch.cat((u * cos - w * sin, w * cos + u * sin), -1)
    outs = []
    for b in range(SEQS):
        qq, kk = turn((x[b] @ q["wq"]).view(ROWS, HEADS, D)), turn((x[b] @ q["wk"]).view(ROWS, KV, D))
        vv, heads = (x[b] @ q["wv"]).view(ROWS, KV, D), []
        for h in range(HEADS):
            hk = h // (HEADS // KV)
            s = (qq[:, h] @ kk[:, hk].t() / math.sqrt(D)).masked_fill(~sees, -math.inf)
            heads.append(torch.softmax(s, 1) @ vv[:, hk])
        outs.append(torch.cat(heads, 1))
    hidden = x + torch.stack(outs) @ q["wo"]
    logits = hidden.reshape(-1, H) @ q["lm"].t()
    t = targets.long()
    nll = torch.logsumexp(logits, 1) - logits.gather(1, t.clamp(min=0)[:, None])[:, 0]
    loss = torch.where(t >= 0, nll * weights.double(), torch.zeros((), dtype=torch.float64, device="cuda:0"))
    loss.sum().backward()
    return loss.detach(), q["embed"].grad, q["mask"].grad


def test_a_training_step_against_automatic_differentiation():
    import torch
    inputs = _params(3)
    step = Step(*inputs)
    print("case step", flush=True)
    step.run()
    torch.cuda.synchronize()
    loss, d_embed, d_mask = _reference(*inputs)
    assert float((step.loss.double() - loss).norm() / loss.norm()) <= 1e-5
    for got, want in ((step.d_embed, d_embed), (step.d_mask, d_mask)):
        assert float((got.double() - want).norm() / want.norm()) <= 1e-4
    unused = torch.ones(VOCAB, dtype=torch.bool, device="cuda:0")
    unused[inputs[1].long().clamp(min=0).reshape(-1)] = False
    assert bool((step.d_embed[unused] == 0).all())


def test_a_training_step_captured_and_replayed():
    """One graph with every operator and one workspace, replayed with other ids and tables in the same buffers, the eager step in between."""
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
    print("case captured step", flush=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()                                           # (the library's own products set up what they need)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    for turn in range(4):
        y = (two, one)[turn & 1]
        for n in buf[0]:
            buf[0][n].copy_(y[0][n])
        for to, x in zip(buf[1:], y[1:]):
            to.copy_(x)
        graph.replay()
        eager = Step(*y)
        eager.run()
        torch.cuda.synchronize()
        got, eager = step.results(), eager.results()
        assert all(torch.equal(eager[n], want[1 - (turn & 1)][n]) for n in got), turn
        assert all(torch.equal(got[n], want[1 - (turn & 1)][n]) for n in got), turn


def test_two_steps_on_two_streams_at_once():
    import torch
    inputs = [_params(6), _params(7)]
    want = []
    for y in inputs:
        step = Step(*y)
        step.run()
        torch.cuda.synchronize()
        want.append(step.results())
    steps, streams = [Step(*y) for y in inputs], [torch.cuda.Stream() for _ in inputs]
    torch.cuda.synchronize()
    for _ in range(3):
        for step, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                step.run()
    torch.cuda.synchronize()
    for step, w in zip(steps, want):
        got = step.results()
        assert all(torch.equal(got[n], w[n]) for n in got)
