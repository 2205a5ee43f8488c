"""Verification of drafted tokens on the GPU, against its definition in 64 bits (paged_formulas.py).

Which tokens are kept and drawn is a matter of whole numbers: it has to be the same, unless a real number lies so near its border
that fp32 sums decide: the seeds below keep every decision further than 1e-5 of its border away (asserted).  A
log-probability is off by 2^-20 of 1 and by 4 u of its magnitude: the argument of an exponential (x - peak) / T is within
2 u |x - peak| / T, log_sum within 2^-20 of sums of up to 2^18 terms."""
import pytest
import torch

import paged_formulas as formulas

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
INF, NAN = float("inf"), float("nan")


def rq():
    import paper_2607_26515_b200 as m
    return m


def rows(M, K, dtype, pad=0):
    return torch.full((M, (K + 7) // 8 * 8 + pad), NAN, dtype=dtype, device="cuda")[:, :K]


def problem(counts, V, dtype, kind, seed=0, T=1.0, pad=0, likely=(2.0, 12.0)):
    g = torch.Generator(device="cuda").manual_seed(seed)
    R, B = sum(counts), len(counts)
    x = rows(R, V, dtype, pad)
    x.copy_(torch.randn((R, V), generator=g, device="cuda") * 2)
    drafts = torch.randint(0, V, (R,), generator=g, device="cuda")
    at = torch.arange(R, device="cuda")
    x[at, drafts] += (likely[0] + (likely[1] - likely[0]) * torch.rand(R, generator=g, device="cuda")).to(dtype)
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    a = dict(logits=x, row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), drafts=drafts, temperature=T)
    if kind == "greedy":
        return {**a, "temperature": 0.0}
    a["u"] = torch.rand(R, generator=g, device="cuda")
    e = rows(B, V, F32, pad)
    e.copy_(torch.empty((B, V), device="cuda").exponential_(generator=g).clamp_min(1e-30))
    a["noise"] = e
    if kind == "logits":
        d = rows(R, V, dtype, pad)
        d.copy_(x.float() + torch.randn((R, V), generator=g, device="cuda"))
        z = d.double() / T
        a["draft_logits"], a["draft_peak"] = d, d.amax(-1).float()
        a["draft_log_sum"] = (z - z.amax(-1, keepdim=True)).exp().sum(-1).log().float()
    return a


def hold(a, got=None):
    got = rq().verify_drafts(**a) if got is None else got
    want = formulas.verify(a["logits"], a["row_start"].tolist(), a["drafts"], a.get("u"), a.get("noise"), a.get("draft_logits"),
                           a.get("draft_peak"), a.get("draft_log_sum"), a["temperature"])
    assert got["accepted"].tolist() == want[0]
    tokens, logp = got["tokens"].tolist(), got["logp"].double().tolist()
    for r, (t, lp) in enumerate(zip(want[1], want[2])):
        if t is None:
            continue
        assert tokens[r] == t, r
        assert abs(logp[r] - lp) <= 2.0 ** -20 + 4 * U * abs(lp) + 4 * U * (30 / (a["temperature"] or 1)), (r, logp[r], lp)
    return got, want


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kind", ["logits", "sure", "greedy"])
@pytest.mark.parametrize("counts, V", [([1], 1), ([2], 3), ([5], 131072), ([1, 4, 2, 8, 1, 3], 50001), ([3] * 40, 999), ([2, 70, 1, 33, 34], 77),
                                       ([5] * 20, 20000), ([6] * 300, 64), ([2], 262144)])
def test_verify(counts, V, kind, dtype):
    hold(problem(counts, V, dtype, kind, seed=V + len(counts)))


@pytest.mark.parametrize("T", [0.3, 0.7, 1.7])
@pytest.mark.parametrize("kind", ["logits", "sure"])
def test_verify_temperature(kind, T):
    hold(problem([4] * 12, 5001, F32, kind, seed=int(T * 10), T=T, pad=8))


def test_verify_keeps_and_refuses():
    """Both happen, at every place of a sequence."""
    got, want = hold(problem([5] * 60, 300, F32, "sure", seed=9, likely=(5.0, 9.0)))
    assert set(want[0]) == {0, 1, 2, 3, 4}
    got, want = hold(problem([5] * 60, 300, F32, "logits", seed=9, likely=(1.0, 5.0)))
    assert set(want[0]) == {0, 1, 2, 3, 4}
    got, want = hold(problem([4] * 60, 300, F32, "greedy", seed=9, likely=(3.0, 9.0)))
    assert set(want[0]) == {0, 1, 2, 3}


@pytest.mark.parametrize("kind", ["logits", "sure", "greedy"])
def test_verify_drafts_that_name_no_token(kind):
    a = problem([4] * 6, 500, BF, kind, seed=4, likely=(20.0, 21.0))
    a["drafts"][1] = -1          # the proposals of sequence 0 end behind one
    a["drafts"][4] = 500         # those of sequence 1 at once
    a["drafts"][10] = 2 ** 40
    a["drafts"][15] = -7         # a last row's is not read
    got, want = hold(a)
    assert want[0][0] <= 1 and want[0][1] == 0 and want[0][2] <= 2


@pytest.mark.parametrize("kind", ["logits", "sure", "greedy"])
def test_verify_masked_logits(kind):
    a = problem([3] * 8, 3000, F32, kind, seed=6)
    keep = a["drafts"]
    mask = torch.rand(a["logits"].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) < 0.7
    mask[torch.arange(len(keep)), keep] = False
    mask[3, keep[3]] = True     # a draft of probability 0
    if kind != "logits":
        mask[6] = True          # a row of nothing at all
    a["logits"].masked_fill_(mask, -INF)
    if kind == "logits":        # the draft may still offer what the target masks
        a["draft_logits"][9:12].masked_fill_(mask[9:12], -INF)
        z = a["draft_logits"].double()
        a["draft_peak"] = z.amax(-1).float()
        a["draft_log_sum"] = (z - z.amax(-1, keepdim=True)).exp().sum(-1).log().float()
    got, want = hold(a)
    assert want[0][1] == 0


@pytest.mark.parametrize("kind", ["sure", "greedy"])
@pytest.mark.parametrize("value", [NAN, INF])
def test_verify_rows_that_are_no_distribution(kind, value):
    a = problem([3] * 5, 700, BF, kind, seed=8, likely=(25.0, 26.0))
    a["logits"][4, 650] = value
    got, want = hold(a)
    assert want[0][1] <= 1 and (want[1][4] == -1 if want[0][1] == 1 else True)


def test_verify_equal_logits_go_to_the_lowest():
    a = problem([2] * 4, 64, F32, "greedy", seed=1)
    a["logits"].fill_(1.0)
    a["drafts"][:] = torch.tensor([0, 5, 1, 5, 0, 0, 63, 0], device="cuda")
    got, want = hold(a)
    assert want[0] == [1, 0, 1, 0] and want[1] == [0, 0, 0, -1, 0, 0, 0, -1]
    a = problem([1] * 3, 64, F32, "sure", seed=1)
    a["logits"].fill_(1.0)
    a["noise"].fill_(0.5)
    got, want = hold(a)
    assert want[1] == [0, 0, 0]


def test_verify_near_a_border_decides_in_64_bits():
    """u within a few steps of fp32 of p / q, and two ratios that differ by less than fp32 resolves."""
    a = problem([2] * 64, 40, F32, "sure", seed=2, likely=(1.0, 3.0))
    z = a["logits"].double()
    lp = torch.log_softmax(z, -1)[torch.arange(128), a["drafts"]]
    near = lp.exp().float()
    step = torch.where(torch.arange(128, device="cuda") % 4 < 2, 1 + 3e-6, 1 - 3e-6)
    a["u"] = (near.double() * step).float()
    hold(a)
    # the last row's drawing: tokens 3 and 7 of nearly the same ratio, 7 larger by 2e-6
    a = problem([1] * 32, 40, F32, "sure", seed=3)
    p = torch.softmax(a["logits"].double(), -1)
    big = (p / a["noise"].double()).amax(-1)
    for j, f in ((3, 4.0), (7, 4.0 * (1 + 2e-6))):
        a["noise"][:, j] = (p[:, j] / (big * f)).float()
    got, want = hold(a)
    assert want[1] == [7] * 32


@pytest.mark.parametrize("V", [200, 1000])
def test_verify_draws_where_the_draft_is_close_to_the_target(V):
    """p - q keeps less than a hundredth of p, so the ratios lose digits: thousands of draws, each the one that 64 bits make from the
    same fp32 peaks and log_sums.  (Their own error in 64 bits is 1e-15 of p, far below the asserted distance of the two largest.)"""
    B = 4096
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (torch.randn((2 * B, V), generator=g, device="cuda") * 2)
    d = x + 0.005 * torch.randn((2 * B, V), generator=g, device="cuda")
    noise = torch.empty((B, V), device="cuda").exponential_(generator=g).clamp_min(1e-30)
    none = torch.full((2 * B,), -1, dtype=torch.int64, device="cuda")
    of_x, of_d = rq().token_logprobs(x, none), rq().token_logprobs(d, none)
    p = ((x.double() - of_x["peak"].double()[:, None]) - of_x["log_sum"].double()[:, None]).exp()
    q = ((d.double() - of_d["peak"].double()[:, None]) - of_d["log_sum"].double()[:, None]).exp()
    drafts = (q / p).argmax(-1)  # refused: u is next to 1
    got = rq().verify_drafts(x, torch.arange(0, 2 * B + 1, 2, dtype=torch.int32, device="cuda"), drafts,
                             torch.full((2 * B,), 1 - 2.0 ** -20, device="cuda"), noise, d, of_d["peak"], of_d["log_sum"])
    assert not got["accepted"].any()
    ratio = (p - q).clamp_min(0)[::2] / noise.double()
    two = ratio.topk(2, dim=-1)
    assert (two.values[:, 0] > two.values[:, 1] * (1 + 1e-10)).all()
    assert torch.equal(got["tokens"][::2], two.indices[:, 0])


@pytest.mark.parametrize("T", [1e-3, 1e-4, 1e-5])
def test_verify_far_drafts_by_64_bits(T):
    """log p and log q of -1000 and below, where fp32 keeps too few digits of their difference: u next to the ratio."""
    V = 64
    for seed in range(32):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = torch.randn((2, V), generator=g, device="cuda") * 2
        d = torch.randn((2, V), generator=g, device="cuda") * 2
        none = torch.full((2,), -1, dtype=torch.int64, device="cuda")
        of_d, of_x = rq().token_logprobs(d, none, T), rq().token_logprobs(x, none, T)
        x[0, 5] = of_x["peak"][0] - 1.5
        d[0, 5] = x[0, 5] - of_x["peak"][0] + of_d["peak"][0] + 0.4 * T
        lp = (x[0, 5].double() - of_x["peak"][0].double()) / T - of_x["log_sum"][0].double()
        lq = (d[0, 5].double() - of_d["peak"][0].double()) / T - of_d["log_sum"][0].double()
        ratio = float((lp - lq).exp())
        for step, kept in ((-2e-6, 1), (2e-6, 0)):
            u = torch.full((2,), ratio * (1 + step), device="cuda")
            if float(u[0]) >= 1:
                continue
            got = rq().verify_drafts(x, torch.tensor([0, 2], dtype=torch.int32, device="cuda"), torch.full((2,), 5, device="cuda"), u,
                                     torch.ones((1, V), device="cuda"), d, of_d["peak"], of_d["log_sum"], T)
            assert got["accepted"].tolist() == [kept]


def test_verify_draws_from_the_target():
    """Kept and drawn first tokens together follow p: 40000 sequences of one draft over 12 tokens; each share within 5 of its
    standard deviations sqrt(p (1 - p) / n)."""
    g = torch.Generator(device="cuda").manual_seed(0)
    B, V = 4000, 12
    z, zq = torch.randn(V, generator=g, device="cuda"), torch.randn(V, generator=g, device="cuda")
    p, counts = torch.softmax(z.double(), 0), torch.zeros(V, dtype=F64, device="cuda")
    for kind in ("logits", "sure"):
        counts.zero_()
        for i in range(10):
            logits = rows(2 * B, V, F32)
            logits.copy_(z.expand(2 * B, V))
            a = dict(logits=logits, row_start=torch.arange(0, 2 * B + 1, 2, dtype=torch.int32, device="cuda"), u=torch.rand(2 * B, generator=g, device="cuda"))
            q = torch.softmax(zq, 0)
            a["drafts"] = torch.multinomial(q, 2 * B, replacement=True, generator=g) if kind == "logits" else torch.full((2 * B,), 4, device="cuda")
            e = rows(B, V, F32)
            e.copy_(torch.empty((B, V), device="cuda").exponential_(generator=g).clamp_min(1e-30))
            a["noise"] = e
            if kind == "logits":
                d = rows(2 * B, V, F32)
                d.copy_(zq.expand(2 * B, V))
                a["draft_logits"], a["draft_peak"] = d, zq.max().expand(2 * B).contiguous()
                a["draft_log_sum"] = (zq - zq.max()).exp().sum().log().expand(2 * B).contiguous()
            tokens = rq().verify_drafts(**a)["tokens"]
            counts += torch.bincount(tokens[0::2], minlength=V)
        n = 10 * B
        assert ((counts / n - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all(), kind


@pytest.mark.parametrize("kind", ["logits", "sure", "greedy"])
def test_verify_wild_starts_and_rows_of_no_sequence(kind):
    a = problem([3] * 6, 200, BF, kind, seed=5)
    out = {"accepted": torch.full((6,), -9, dtype=torch.int32, device="cuda"), "tokens": torch.full((18,), -9, device="cuda"),
           "logp": torch.full((18,), -9.0, device="cuda")}
    a["row_start"] = torch.tensor([2, 5, 5, 4, 9, 12, 14], dtype=torch.int32, device="cuda")  # an empty one, one that ends before it starts
    a["row_start"][3] = 5
    got, _ = hold(a, rq().verify_drafts(**a, out=out))
    assert got is out and out["tokens"][:2].tolist() == [-9, -9] and (out["tokens"][14:] == -9).all() and (out["logp"][14:] == -9).all()
    assert out["accepted"][1] == 0
    a["row_start"] = torch.tensor([-5, 2, 4, 10 ** 9, 3, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    got = rq().verify_drafts(**a)
    torch.cuda.synchronize()
    assert got["accepted"][3] == 0 and got["accepted"][5] == 0


def test_verify_captured_and_on_another_stream():
    m = rq()
    a = problem([4] * 9, 9000, BF, "logits", seed=3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = m.verify_drafts(**a, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    hold(a, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = m.verify_drafts(**a)
    for seed in (11, 12):
        b = problem([4] * 9, 9000, BF, "logits", seed=seed)
        for name in ("logits", "drafts", "u", "noise", "draft_logits", "draft_peak", "draft_log_sum"):
            a[name].copy_(b[name])
        graph.replay()
        torch.cuda.synchronize()
        hold(a, got)


def test_verify_takes_what_token_logprobs_gives():
    """A draft's peak and log_sum as the framework computes them; drafts equal to the target are all kept."""
    m = rq()
    a = problem([6] * 10, 4000, BF, "sure", seed=7, T=0.8)
    a["draft_logits"] = rows(60, 4000, BF)
    a["draft_logits"].copy_(a["logits"])
    d = m.token_logprobs(a["draft_logits"], a["drafts"], temperature=0.8)
    a["draft_peak"], a["draft_log_sum"] = d["peak"], d["log_sum"]
    a["u"].mul_(0.999)
    got = m.verify_drafts(**a)
    assert got["accepted"].tolist() == [5] * 10
    lp = m.token_logprobs(a["logits"], got["tokens"], temperature=0.8)["logp"]
    assert torch.allclose(lp, got["logp"], rtol=1e-6, atol=1e-6)
