"""Verification of drafted tokens where 32 bits do not decide, against the definition in 64 bits."""
import pytest
import torch

import paged_formulas as formulas
from test_verify_gpu import BF, F32, F64, INF, NAN, problem, rows, rq

pytestmark = pytest.mark.gpu


def refused(x, d, seed, T=1.0):
    """A sequence of one refused draft per pair of rows: (the call's arguments, p, q in 64 bits from the fp32 peaks and log_sums)."""
    R, V = x.shape
    g = torch.Generator(device="cuda").manual_seed(seed)
    noise = rows(R // 2, V, F32)
    noise.copy_(torch.empty((R // 2, V), device="cuda").exponential_(generator=g).clamp_min(1e-30))
    none = torch.full((R,), -1, dtype=torch.int64, device="cuda")
    of_x, of_d = rq().token_logprobs(x, none, T), rq().token_logprobs(d, none, T)
    p = ((x[::2].double() - of_x["peak"][::2].double()[:, None]) / T - of_x["log_sum"][::2].double()[:, None]).exp()
    q = ((d[::2].double() - of_d["peak"][::2].double()[:, None]) / T - of_d["log_sum"][::2].double()[:, None]).exp()
    drafts = torch.zeros(R, dtype=torch.int64, device="cuda")
    drafts[::2] = (q / p).argmax(-1)
    a = dict(logits=x, row_start=torch.arange(0, R + 1, 2, dtype=torch.int32, device="cuda"), drafts=drafts,
             u=torch.full((R,), 1 - 2.0 ** -24, device="cuda"), noise=noise, draft_logits=d, draft_peak=of_d["peak"],
             draft_log_sum=of_d["log_sum"], temperature=T)
    return a, p, q


def hold_drawn(a, p, q, least):
    """Each refused row's token is the one that 64 bits draw.  p and q are 64-bit exponentials, off by 2^-52 of themselves or so: rows
    whose two largest ratios lie nearer than that leaves room for are asserted to be few and are not compared."""
    got = rq().verify_drafts(**a)
    x = a["drafts"][::2]
    ratio = (p / q).gather(1, x[:, None])[:, 0]
    went = ratio <= a["u"][::2].double()  # refused (others differ from the draft by nothing that u can tell)
    assert torch.equal(got["accepted"] == 0, went) and int(went.sum()) >= least
    w = (p - q).clamp_min(0)
    left = w.amax(-1) > 0
    s = torch.where(left[:, None], w, p) / a["noise"].double()
    two = s.topk(2, dim=-1)
    at = two.indices[:, :1]
    slack = 2.0 ** -48 * torch.where(left[:, None], p.gather(1, at) / w.gather(1, at).clamp_min(1e-300), torch.ones_like(at, dtype=F64))[:, 0]
    clear = went & (two.values[:, 0] > two.values[:, 1] * (1 + slack))
    assert int((went & ~clear).sum()) <= 0.01 * int(went.sum())
    wrong = clear & (got["tokens"][::2] != at[:, 0])
    assert not wrong.any(), f"{int(wrong.sum())} of {int(clear.sum())} tokens are others"


@pytest.mark.parametrize("V, B", [(200, 4096), (1000, 4096), (20000, 512)])
@pytest.mark.parametrize("std", [5e-3, 5e-4, 5e-5, 5e-6])
def test_verify_draws_where_hardly_anything_is_left(V, B, std):
    """p - q of 1e-3 of p down to 1e-6: fp32 exponentials leave it few digits, or none."""
    g = torch.Generator(device="cuda").manual_seed(V)
    x, d = rows(2 * B, V, F32), rows(2 * B, V, F32)
    x.copy_(torch.randn((2 * B, V), generator=g, device="cuda") * 2)
    d.copy_(x + std * torch.randn((2 * B, V), generator=g, device="cuda"))
    hold_drawn(*refused(x, d, V), least=B // 2)


@pytest.mark.parametrize("V, B", [(1000, 2048), (20000, 512), (131072, 64)])
@pytest.mark.parametrize("up", [True, False])
def test_verify_draws_where_one_logit_differs(V, B, up):
    """The target's and the draft's logits differ in one place by one step of bf16: what is left is that place, or all others."""
    g = torch.Generator(device="cuda").manual_seed(V + up)
    x, d = rows(2 * B, V, BF), rows(2 * B, V, BF)
    x.copy_(torch.randn((2 * B, V), generator=g, device="cuda") * 2)
    d.copy_(x)
    row = torch.arange(2 * B, device="cuda")
    at = x.float().topk(40, dim=-1).indices[row, torch.randint(0, 40, (2 * B,), generator=g, device="cuda")]
    v = x[row, at]
    assert (v > 0).all()
    step = (v.view(torch.int16) + (1 if up else -1)).view(BF)
    x[row, at] = step
    hold_drawn(*refused(x, d, V), least=B // 4)


def test_verify_draws_where_the_draft_is_the_target():
    """Nothing is left of p - q: drawn from p."""
    B, V = 64, 5000
    g = torch.Generator(device="cuda").manual_seed(0)
    x = rows(2 * B, V, F32)
    x.copy_(torch.randn((2 * B, V), generator=g, device="cuda") * 2)
    a, p, q = refused(x, x.clone(memory_format=torch.preserve_format), 1)
    a["draft_logits"] = x
    a["u"].fill_(1.0)  # from outside of [0, 1): refuses what u < 1 would keep
    hold_drawn(a, p, q, least=B)


@pytest.mark.parametrize("T", [0.05, 0.7])
def test_verify_draws_where_hardly_anything_is_left_at_other_temperatures(T):
    g = torch.Generator(device="cuda").manual_seed(3)
    B, V = 2048, 500
    x, d = rows(2 * B, V, F32), rows(2 * B, V, F32)
    x.copy_(torch.randn((2 * B, V), generator=g, device="cuda") * 2)
    d.copy_(x + 5e-5 * T * torch.randn((2 * B, V), generator=g, device="cuda"))
    hold_drawn(*refused(x, d, V, T), least=B // 2)


@pytest.mark.parametrize("T", [1e-50, -1e-50, 9e-7, -1.0, 1.1e6, NAN, INF])
def test_verify_refuses_temperatures_that_are_none(T):
    """Numbers too small for fp32 among them: they are not temperature 0."""
    a = problem([2, 3], 40, F32, "sure", seed=1)
    with pytest.raises(ValueError, match="temperature"):
        rq().verify_drafts(**{**a, "temperature": T})


# ------------------------------------------------------------------------------------------------ borders of the other tests' problems

def distance(a):
    """How near the decisions of a call are to their borders: the smallest |u q - p| / p of the drafts that are looked at, and the
    smallest relative distance of the two largest ratios of the places that are drawn."""
    x, T, V = a["logits"].double(), a["temperature"], a["logits"].shape[1]
    start, drafts = a["row_start"].tolist(), a["drafts"].tolist()
    accepted = formulas.verify(a["logits"], start, a["drafts"], a["u"], a["noise"], a.get("draft_logits"), a.get("draft_peak"),
                               a.get("draft_log_sum"), T)[0]
    near, tie = INF, INF
    for b, kept in enumerate(accepted):
        n = start[b + 1] - start[b]
        for i in range(min(kept + 1, n)):
            r = start[b] + i
            p = torch.softmax(x[r] / T, 0)
            if "draft_logits" in a:
                q = torch.exp((a["draft_logits"][r].double() - a["draft_peak"][r].double()) / T - a["draft_log_sum"][r].double())
            else:
                q = torch.zeros_like(p)
                q[drafts[r]] = 1.0
            if i < n - 1:
                near = min(near, abs(float(a["u"][r]) * float(q[drafts[r]] / p[drafts[r]]) - 1))
            if i == kept:
                w = torch.relu(p - q) if i < n - 1 else p
                s = w / a["noise"][b].double()
                if V > 1 and float(s.max()) > 0:
                    two = s.topk(2).values
                    tie = min(tie, float(1 - two[1] / two[0]))
    return near, tie


@pytest.mark.parametrize("kind", ["logits", "sure"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("counts, V", [([1], 1), ([2], 3), ([5], 131072), ([1, 4, 2, 8, 1, 3], 50001), ([3] * 40, 999), ([2, 70, 1, 33, 34], 77),
                                       ([5] * 20, 20000), ([6] * 300, 64), ([2], 262144)])
def test_verify_problems_are_clear(counts, V, kind, dtype):
    """Every decision of the problems that test_verify compares whole numbers of is further than 1e-5 from its border."""
    near, tie = distance(problem(counts, V, dtype, kind, seed=V + len(counts)))
    assert near > 1e-5 and tie > 1e-5, (near, tie)


@pytest.mark.parametrize("kind", ["logits", "sure"])
def test_verify_other_problems_are_clear(kind):
    for T in (0.3, 0.7, 1.7):
        near, tie = distance(problem([4] * 12, 5001, F32, kind, seed=int(T * 10), T=T, pad=8))
        assert near > 1e-5 and tie > 1e-5, (T, near, tie)
    near, tie = distance(problem([5] * 60, 300, F32, kind, seed=9, likely=(5.0, 9.0) if kind == "sure" else (1.0, 5.0)))
    assert near > 1e-5 and tie > 1e-5, (near, tie)
