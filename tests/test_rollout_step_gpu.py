"""One block of a drafted rollout step as it is run: qkv projection in 4 bit, rotation into the paged cache, attention over it, output
projection, residual stream, head, verification; eager, on a stream of its own, and captured in a graph that follows the sequences
while they grow.  Each operator is held to its definition elsewhere; here the run is held to the same run in 64 bits, from the
values that every operator was given."""
import pytest
import torch

import paged_formulas as formulas
from operator_formulas import join

pytestmark = pytest.mark.gpu

HALF_BF = 2.0 ** -8
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Block:
    """A small block of 16 query and 2 kv heads of 64 channels, with its caches, for B sequences of up to 4 tokens a step."""

    def __init__(self, B=5, seed=0):
        import paper_2607_26515_b200 as m
        self.m, self.B = m, B
        g = self.g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s, std=1.0: (torch.randn(s, generator=g, device="cuda") * std).to(BF)
        K, Hq, Hkv, D, V = 1024, 16, 2, 64, 1500
        self.K, self.Hq, self.Hkv, self.D, self.V = K, Hq, Hkv, D, V
        self.wqkv, self.wo, self.head = (m.pack_weight(rand(n, K, std=0.03)) for n in ((Hq + 2 * Hkv) * D, K, V))
        self.bias, self.gamma = rand((Hq + 2 * Hkv) * D, std=0.3), (1 + rand(K, std=0.1)).to(BF)
        self.inv_freq = 1e4 ** (-torch.arange(D // 2, dtype=torch.float64, device="cuda") / (D // 2))
        self.k, self.v = (rand(60, 16, Hkv, D) for _ in range(2))
        self.table = torch.randperm(60, generator=g, device="cuda")[:B * 12].view(B, 12).to(I32)
        self.n = [4, 1, 3, 4, 2][:B]
        starts = [0]
        for n in self.n:
            starts.append(starts[-1] + n)
        self.T = starts[-1]
        self.q_start, self.kv_len = torch.tensor(starts, dtype=I32, device="cuda"), torch.tensor([n + 20 * b for b, n in enumerate(self.n)], dtype=I32, device="cuda")
        self.work = m.alloc_workspace(max(m.resq_workspace_bytes(self.T, (Hq + 2 * Hkv) * D, K, m.S_2_4), m.resq_workspace_bytes(self.T, K, K, m.S_2_4)))
        self.attn_work = m.alloc_workspace(m.paged_attention_workspace_bytes(self.T, B, Hq, Hkv, D, 4))
        self.inputs()

    def inputs(self):
        rand = lambda *s, std=1.0: torch.randn(s, generator=self.g, device="cuda") * std
        if not hasattr(self, "h"):
            self.h, self.drafts = torch.empty((self.T, self.K), dtype=F32, device="cuda"), torch.empty(self.T, dtype=torch.int64, device="cuda")
            self.u, self.noise = torch.empty(self.T, device="cuda"), torch.empty((self.B, 1504), device="cuda")[:, :self.V]
        self.h.copy_(rand(self.T, self.K))
        self.drafts.copy_(torch.randint(0, self.V, (self.T,), generator=self.g, device="cuda"))
        self.u.copy_(torch.rand(self.T, generator=self.g, device="cuda") * 1e-3)  # small: some drafts are kept
        self.noise.copy_(torch.empty((self.B, self.V), device="cuda").exponential_(generator=self.g).clamp_min(1e-30))

    def step(self):
        m = self.m
        seqs = (self.q_start, self.kv_len, self.table)
        x = torch.empty((self.T, self.K), dtype=BF, device="cuda").copy_(self.h)
        qkv = m.resq_linear(x, *self.wqkv, m.S_2_4, workspace=self.work)
        q = m.rope_append(qkv, self.k, self.v, *seqs, self.inv_freq, bias=self.bias)
        o, lse = m.paged_attention(q, self.k, self.v, *seqs, max_new=4, lse=True, workspace=self.attn_work)
        b = m.resq_linear(o, *self.wo, m.S_2_4, workspace=self.work)
        h, y = m.block_join(self.h, b, self.gamma)
        logits = m.w4a16_gemv(y, *self.head, "hif4", out_dtype=F32)
        out = m.verify_drafts(logits, self.q_start, self.drafts, self.u, self.noise)
        return dict(qkv=qkv, q=q, o=o, lse=lse, b=b, h=h, y=y, logits=logits, **out)

    def hold(self, r, before):
        start, kv = self.q_start.tolist(), self.kv_len.tolist()
        want = formulas.rope_append(r["qkv"], self.bias, *before, start, kv, self.table, self.inv_freq, False)
        size = 2 * float((r["qkv"].double() + self.bias.double()).abs().max())
        for got, w in ((r["q"], want[0]), (self.k, want[1]), (self.v, want[2])):
            assert ((got.double() - w).abs() <= HALF_BF * w.abs() + 16 * 2.0 ** -24 * size).all()
        o, lse, mag, _ = formulas.attention(r["q"], self.k, self.v, start, kv, self.table, self.D ** -0.5)
        assert ((r["o"].double() - o).abs() <= (HALF_BF + 1e-3) * mag + HALF_BF * o.abs()).all()
        assert ((r["lse"].double() - lse).abs() <= 1e-4).all()
        h, y = join(self.h.double(), r["b"].double(), self.gamma.double(), None, None, "linear", 1.0, 1e-6)
        assert ((r["y"].double() - y).abs() <= HALF_BF * y.abs() + 1e-4).all()
        accepted, tokens, logp = formulas.verify(r["logits"], start, self.drafts, self.u, self.noise, None, None, None, 1.0)
        assert r["accepted"].tolist() == accepted and r["tokens"].tolist() == tokens
        assert all(abs(a - b) <= 1e-5 for a, b in zip(r["logp"].tolist(), logp))
        assert self.m.check(self.work) == 0 and self.m.check(self.attn_work) == 0


def test_rollout_step_eager_and_on_a_stream():
    b = Block()
    before = (b.k.clone(), b.v.clone())
    first = b.step()
    b.hold(first, before)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = b.step()
    torch.cuda.current_stream().wait_stream(s)
    for name in first:
        assert torch.equal(first[name], again[name]), name


def test_rollout_step_captured_follows_the_sequences():
    b = Block(seed=1)
    b.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = b.step()
    kept = 0
    for i in range(5):
        b.inputs()
        before = (b.k.clone(), b.v.clone())
        graph.replay()
        torch.cuda.synchronize()
        b.hold(r, before)
        # what was kept, and the token behind it, stay in the cache; the other drafts' slots are written again
        kept += int(r["accepted"].sum())
        b.kv_len += r["accepted"] + 1
    assert kept > 0
