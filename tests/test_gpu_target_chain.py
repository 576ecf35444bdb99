"""GPU tests of the target's operators together, as a program uses them in rounds of speculative decoding: the prompt's keys and values into the
cache, then per round the attention of the draft tree's rows, their distributions from logits, the walk over them, and the accepted path into the
cache, lengths advancing on the device.  The target model between attention and logits is a fixed matrix; its keys and values are given.

Each operator is checked against its definition on what the chain handed to it (tolerances: the operators' own tests); the walk's inputs are the kernels' probabilities,
so its outputs have to be the oracle's wherever its decisions are no closer than 1e-9."""
import numpy as np
import pytest

from oracle import target as orc
from oracle import verify_walk as vw
from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import inputs
from paper_2410_05589_amd import verify as VF
from tests import target_util as TU
from tests.test_gpu_target_probs import check as check_probs
from tests.test_gpu_tree_attention import check as check_attention

pytestmark = pytest.mark.gpu

BATCH, HEADS, NQ, D, VOCAB, TOPK = 3, 2, 4, 64, 1000, 8
FANOUT = [3, 2, 1]
ROWS = len(FANOUT) + 1
CAPACITY = 256


class Round:
    """The calls of one round, on buffers that stay."""

    def __init__(self, dtype, seed):
        import torch
        dev = "cuda:0"
        self.dtype, dt = dtype, TU.torch_dtype(dtype)
        self.parent, self.rank = inputs.draft_tree(FANOUT)
        self.nodes = len(self.parent)
        self.tree = VF.make_tree(self.parent, self.rank)
        self.cache = TU.Cache(HEADS, D, [CAPACITY] * BATCH, seed=seed)
        self.len = torch.zeros(BATCH, dtype=torch.int32, device=dev)
        self.q = torch.empty((BATCH, self.nodes, NQ, D), dtype=dt, device=dev)
        self.k, self.v = (torch.empty((BATCH, self.nodes, HEADS, D), dtype=dt, device=dev) for _ in range(2))
        self.out = torch.empty_like(self.q)
        self.lse = torch.empty((BATCH, self.nodes, NQ), device=dev)
        self.head = TU.normal((NQ * D, VOCAB), seed + 9, "f32", 0.3)
        self.logits = torch.empty((BATCH, self.nodes, VOCAB), device=dev)
        self.p = torch.empty((BATCH, self.nodes, VOCAB), device=dev)
        self.settings = dict(temperature=[0.8, 1.0, 1.2], top_k=[0, 40, 0], top_p=[0.9, 1.0, 0.95], min_p=[0.0, 0.0, 0.02])
        self.set_dev = {n: torch.tensor(s, dtype=torch.int32 if n == "top_k" else torch.float32, device=dev) for n, s in self.settings.items()}
        self.draft = torch.empty((BATCH, ROWS, VOCAB), device=dev)
        self.top_ids = torch.empty((BATCH, ROWS, TOPK), dtype=torch.int32, device=dev)
        self.r = torch.empty((BATCH, self.nodes), device=dev)
        self.n_acc = torch.empty(BATCH, dtype=torch.int32, device=dev)
        self.path = torch.empty((BATCH, ROWS), dtype=torch.int32, device=dev)
        self.tokens = torch.empty((BATCH, ROWS + 1), dtype=torch.int32, device=dev)
        bound = [CAPACITY - ROWS - 1] * BATCH

        a = VF.make_tree_attn_args(self.cache.struct, NQ, dtype, bound)
        a.q, a.k_rows, a.v_rows, a.out, a.lse = (x.data_ptr() for x in (self.q, self.k, self.v, self.out, self.lse))
        a.kv_len_dev = self.len.data_ptr()
        need = VF.ps_tree_attention_workspace_bytes(self.tree, a)
        self.ws, at = TU.workspace(need)
        a.workspace, a.workspace_bytes = (at, need) if need else (None, 0)
        d = VF.ps_target_probs_args()
        d.batch, d.rows, d.vocab, d.dtype, d.logits, d.probs = BATCH, self.nodes, VOCAB, B.PS_F32, self.logits.data_ptr(), self.p.data_ptr()
        for n, x in self.set_dev.items():
            setattr(d, n, x.data_ptr())
        w = VF.ps_verify_args()
        w.batch, w.rows, w.vocab, w.topk, w.top_ids = BATCH, ROWS, VOCAB, TOPK, self.top_ids.data_ptr()
        w.q, w.p, w.r = self.draft.data_ptr(), self.p.data_ptr(), self.r.data_ptr()
        w.n_accepted, w.path, w.out_tokens = self.n_acc.data_ptr(), self.path.data_ptr(), self.tokens.data_ptr()
        c = self.cache.write_args(self.k, self.v, bound, dtype)
        c.kv_len_dev = c.len_out = self.len.data_ptr()
        c.n_accepted, c.path, c.path_rows = self.n_acc.data_ptr(), self.path.data_ptr(), ROWS
        self.calls = (a, d, w, c)

    def new_inputs(self, seed):
        import torch
        g = torch.Generator().manual_seed(seed)
        for x in (self.q, self.k, self.v):
            x.copy_(torch.randn(x.shape, generator=g))
        draft = torch.softmax(torch.randn(self.draft.shape, generator=g) * 2.5, -1)
        self.draft.copy_(draft)
        self.top_ids.copy_(draft.topk(TOPK).indices.to(torch.int32))
        self.r.copy_(torch.rand(self.r.shape, generator=g))

    def run(self):
        import torch
        a, d, w, c = self.calls
        assert VF.ps_tree_attention(self.tree, a, TU.stream()) == B.PS_OK
        torch.matmul(self.out.float().reshape(BATCH * self.nodes, NQ * D), self.head, out=self.logits.view(BATCH * self.nodes, VOCAB))
        self.logits[:, :, :].add_(torch.log(self.draft[:, :1] + 1e-4))          # (a target that agrees with its drafter now and then)
        assert VF.ps_target_probs(d, TU.stream()) == B.PS_OK
        assert VF.ps_verify_walk(self.tree, w, TU.stream()) == B.PS_OK
        assert VF.ps_cache_write(c, TU.stream()) == B.PS_OK

    def check(self, before, lens):
        """What the round left against the definitions; before: the cache's contents, lens: the lengths before it."""
        after = {n: self.cache.decoded(n) for n in "kv"}
        n_acc, path, tokens = (x.cpu().numpy() for x in (self.n_acc, self.path, self.tokens))
        for b in range(BATCH):
            tok = vw.tree_tokens(self.top_ids[b].cpu().numpy(), self.parent, self.rank)
            ref = vw.acceptance_walk(self.parent, tok, TU.np64(self.draft[b]), TU.np64(self.p[b]), TU.np64(self.r[b]))
            assert ref["accept_margin"] > 1e-9 and ref["cdf_margin"] > 1e-9
            assert n_acc[b] == ref["n_accepted"] and tokens[b, :n_acc[b] + 1].tolist() == ref["tokens"]
            rows = orc.path_rows(n_acc[b], path[b], self.nodes)
            for n, x in (("k", self.k), ("v", self.v)):
                orc.write(*before[n], self.cache.offsets[b] // 32, lens[b], TU.np64(x[b])[rows])
            assert int(self.len[b]) == lens[b] + 1 + n_acc[b]
        for n in "kv":
            assert np.array_equal(after[n][0], before[n][0], equal_nan=True) and np.array_equal(after[n][1], before[n][1])
        check_probs(self.logits, self.settings, None, self.p, None, None)
        return n_acc


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rounds_from_a_prompt_on(dtype):
    import torch
    R = Round(dtype, 3)
    prompt = [40, 1, 97]
    k, v = (TU.normal((BATCH, max(prompt), HEADS, D), 70 + i, dtype) for i in range(2))
    R.cache.write(k, v, [0] * BATCH, dtype, n_seq=prompt, len_out=R.len)
    assert R.len.tolist() == prompt
    accepted = 0
    for i in range(6):
        R.new_inputs(100 + i)
        lens, before = R.len.tolist(), {n: R.cache.decoded(n) for n in "kv"}
        frozen = TU.Cache(HEADS, D, [CAPACITY] * BATCH)                          # (the cache as the attention saw it)
        for n in "kv":
            frozen.codes[n].copy_(R.cache.codes[n])
            frozen.scales[n].copy_(R.cache.scales[n])
        R.run()
        check_attention(frozen, R.parent, R.q, R.k, R.v, lens, dtype, R.out, R.lse)
        accepted += int(R.check(before, lens).sum())
    assert accepted > 0
    # what has been committed reads back
    lens = R.len.tolist()
    back = torch.zeros((BATCH, max(lens), HEADS, D), dtype=TU.torch_dtype(dtype), device="cuda:0")
    R.cache.read(back, None, None, dtype, n_seq=lens)
    for b, n in enumerate(prompt):
        assert ((back[b, :n].float() - k[b, :n].float()).abs() <= k[b, :n].float().abs() * 2.0 ** -3 + 2.0 ** -7).all()


def test_a_captured_round_replayed():
    """The whole round in one graph, replayed with new inputs and eager rounds of another decoder in between; every replay against the definitions."""
    import torch
    R, other = Round("bf16", 5), Round("bf16", 6)
    prompt = [33, 64, 5]
    k, v = (TU.normal((BATCH, max(prompt), HEADS, D), 80 + i, "bf16") for i in range(2))
    for x in (R, other):
        x.cache.write(k, v, [0] * BATCH, "bf16", n_seq=prompt, len_out=x.len)
        x.new_inputs(1)
    other.run()                                              # (the walk's and the libraries' first calls)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        R.run()
    for i in range(5):
        R.new_inputs(200 + i)
        lens, before = R.len.tolist(), {n: R.cache.decoded(n) for n in "kv"}
        g.replay()
        torch.cuda.synchronize()
        R.check(before, lens)
        other.new_inputs(300 + i)
        other.run()
        torch.cuda.synchronize()
