"""What the operators on a paged cache do at their edges, against their definitions in 64 bits (paged_formulas.py; tolerances of
attention as in test_paged_gpu.py)."""
import math
from fractions import Fraction

import pytest
import torch

import paged_formulas as formulas
from test_paged_gpu import BF, F32, F64, HALF_BF, I32, NAN, U, Paged, freqs, gen, hold, ints, rq

pytestmark = pytest.mark.gpu

INF = float("inf")


# ------------------------------------------------------------------------------------------------ shares that weigh nothing

def far_scores(n, keys, high, D=128, g=4):
    """One sequence whose scores are 0 but for key `high`, which scores 100 (2^-144 of its weight is left to the others)."""
    p = Paged([(n, keys - n)], 2, D, 16, seed=n)
    q = torch.zeros((n, 2 * g * D), dtype=BF, device="cuda")
    q.view(n, 2 * g, D)[:, :, 0] = 8
    for j in range(keys):
        page, row = int(p.table[0, j // 16]), j % 16
        p.k[page, row] = 0
        if j == high:
            p.k[page, row, :, 0] = 12.5
    return p, q


# keys of one CTA's share and of several; query rows per kv head of each kernel
FAR = [(1, 64, 20), (1, 5000, 4000), (6, 128, 60), (6, 5000, 4000), (12, 200, 150), (12, 5000, 4000), (100, 600, 400), (100, 6000, 4000)]


@pytest.mark.parametrize("n, keys, high", FAR)
def test_attention_a_score_of_nan_is_never_lost(n, keys, high):
    p, q = far_scores(n, keys, high)
    p.k[int(p.table[0, 0]), 3, 0, 1] = NAN  # key 3 of the first kv head; seen by all
    for hint in (n, None):
        out, lse = rq().paged_attention(q, *p.args(), scale=1.0, max_new=hint, lse=True)
        assert torch.isnan(lse[:, :4]).all() and torch.isnan(out[:, :4 * 128]).all(), hint
        assert torch.isfinite(lse[:, 4:]).all() and torch.isfinite(out[:, 4 * 128:]).all(), hint


@pytest.mark.parametrize("n, keys, high", FAR)
@pytest.mark.parametrize("value", [INF, NAN])
def test_attention_a_visible_strange_value_is_never_lost(n, keys, high, value):
    p, q = far_scores(n, keys, high)
    p.v[int(p.table[0, 0]), 3, 0, 5] = value
    for hint in (n, None):
        out, lse = rq().paged_attention(q, *p.args(), scale=1.0, max_new=hint, lse=True)
        strange = ~torch.isfinite(out.view(n, 8, 128))
        assert strange[:, :4, 5].all() and int(strange.sum()) == 4 * n, hint
        assert torch.isfinite(lse).all()


# ------------------------------------------------------------------------------------------------ values near the ends of their type

@pytest.mark.parametrize("size", [1e34, 1e-25])
@pytest.mark.parametrize("n, keys", [(1, 3000), (12, 3000), (100, 1000), (300, 5000)])
def test_attention_values_of_any_size(n, keys, size):
    """Scores that rise by 13 (19 in the exponent of 2) behind the first keys; sums of weights up to 1 times these values are within
    fp32, of weights up to 2^19 they would not be."""
    p, q = far_scores(n, keys, keys - n - 40)
    p.k.mul_(0.13)
    p.v.nan_to_num_(0.0).mul_(size)
    for hint in (n, None):
        out, lse = rq().paged_attention(q, *p.args(), scale=1.0, max_new=hint, lse=True)
        hold(out, lse, q, p, 1.0, f"hint {hint}")


# ------------------------------------------------------------------------------------------------ starts out of order

def backwards(n):
    """n sequences of two rows from the last to the first, and between them n - 1 without rows."""
    return [x for i in range(n - 1, -1, -1) for x in (2 * i, 2 * i + 2)]


@pytest.mark.parametrize("starts, T", [([4, 9, 2, 4], 12), ([20, 3, 3, 0, 2, -4], 12), ([50, 60, 0, 9, 10, 40, 44], 70), ([5, 2 ** 31 - 1, -3, 2, 1, -2 ** 31], 9),
                                       (backwards(64), 140), (backwards(65), 130), (backwards(700), 1409)])
def test_append_starts_out_of_order(starts, T):
    """Every sequence has the rows from its start to its end, wherever the others lie; the lists give each row to one sequence at most."""
    B = len(starts) - 1
    p = Paged([(2, 30)] * B, 2, 64, 8)
    p.table = torch.cat([p.table, p.table.new_full((B, 10), -1)], 1)
    p.k.nan_to_num_(0.5)
    p.v.nan_to_num_(0.25)
    qkv = torch.randn((T, 8 * 64), generator=p.g, device="cuda").to(BF)
    q_start = ints(starts)
    want = formulas.rope_append(qkv, None, p.k, p.v, starts, p.kv, p.table, freqs(64), False)
    owned = sum(max(min(max(b, 0), T) - min(max(a, 0), T), 0) for a, b in zip(starts, starts[1:]))
    there = ~torch.isnan(want[0])
    assert int(there[:, 0].sum()) == owned > 0
    q = torch.full((T, 4 * 64), 3.0, dtype=BF, device="cuda")
    rq().rope_append(qkv, p.k, p.v, q_start, p.kv_len, p.table, freqs(64), q=q)
    tol = lambda w: HALF_BF * w.abs() + 16 * U * 2 * float(qkv.abs().max())
    assert ((q.double() - want[0]).abs() <= tol(want[0]))[there].all() and (q[~there] == 3).all()
    assert ((p.k.double() - want[1]).abs() <= tol(want[1])).all() and ((p.v.double() - want[2]).abs() <= tol(want[2])).all()


@pytest.mark.parametrize("B", [1, 40, 128, 129, 300, 4096])
def test_append_rows_behind_many_sequences(B):
    """Rows of no sequence are looked for in all of them, and stay as they were."""
    p = Paged([(i % 2, 3) for i in range(B)] if B > 1 else [(1, 3)], 1, 64, 8)
    T = p.T + 21
    qkv = torch.randn((T, 4 * 64), generator=p.g, device="cuda").to(BF)
    q = torch.full((T, 2 * 64), 3.0, dtype=BF, device="cuda")
    rq().rope_append(qkv, *p.args(), freqs(64), q=q)
    want = formulas.rope_append(qkv, None, p.k, p.v, p.starts, p.kv, p.table, freqs(64), False)[0]
    assert (q[p.T:] == 3).all()
    assert ((q.double() - want).abs()[:p.T] <= HALF_BF * want[:p.T].abs() + 16 * U * 2 * float(qkv.abs().max())).all()


# ------------------------------------------------------------------------------------------------ angles

# 1 / (2 pi) to 84 digits
INV_2PI = Fraction(159154943091895335768883763372514362034459645740456448747667344058896797634226535090, 10 ** 84)


def test_append_angles_of_any_position_and_frequency():
    """A pair (sin, cos) of its own angle turns into (0, 1): what is left in the first place is the error of the angle, of its sine and
    cosine.  Tolerance: the angle 2 pi (2^-32 + 2^-26) (fixed point; fp32 number of half turns), sine and cosine one unit in the last
    place each (2^-24 (|sin| + |cos|) <= 1.42 * 2^-24), a rounded product 2^-25 and the output's rounding."""
    g = gen(0)
    f = torch.cat([freqs(128)[:20], torch.rand(14, generator=g, dtype=F64, device="cuda"), torch.rand(10, generator=g, dtype=F64, device="cuda") * 100,
                   -torch.rand(10, generator=g, dtype=F64, device="cuda"), -torch.rand(4, generator=g, dtype=F64, device="cuda") * 50,
                   torch.rand(3, generator=g, dtype=F64, device="cuda") * 1e-9, -torch.rand(3, generator=g, dtype=F64, device="cuda") * 1e-9])
    pos = [0, 1, -1, 2, 77, 8191, 131071, 900001, 2 ** 24 + 1, 2 ** 30 - 1, -2 ** 30 - 5, 2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1]
    pos += torch.randint(-2 ** 31, 2 ** 31, (40,), generator=g, device="cuda").tolist()
    T, tau = len(pos), 6.283185307179586476925
    exact = [Fraction(x) * INV_2PI for x in f.tolist()]
    turn = torch.tensor([[float((p * e + Fraction(1, 2)) % 1 - Fraction(1, 2)) for e in exact] for p in pos], dtype=F64, device="cuda")
    s, c = (turn * tau).sin(), (turn * tau).cos()
    qkv = torch.zeros((T, 3 * 128), dtype=F32, device="cuda")
    qkv[:, :64], qkv[:, 64:128] = s, c
    a, b = qkv[:, :64].double(), qkv[:, 64:128].double()
    p = Paged([(T, 0)], 1, 128, 8)
    q = rq().rope_append(qkv, *p.args(), f, positions=ints(pos)).double()
    want = a * c - b * s
    err = (q[:, :64] - want).abs()
    tol = tau * (2.0 ** -32 + 2.0 ** -26) + 1.42 * 2.0 ** -24 + 2.0 ** -25 + HALF_BF * want.abs()
    assert (err <= tol).all(), f"{int((err > tol).sum())} of {err.numel()} off, worst {float((err / tol).max())} of the tolerance"
    assert ((q[:, 64:] - 1).abs() <= HALF_BF + 1e-6).all()


# ------------------------------------------------------------------------------------------------ waits

TIMEOUT = 7


@pytest.mark.parametrize("lens, Hq, Hkv, D", [([(100, 900), (300, 40)], 4, 2, 128), ([(40, 700)], 8, 2, 64), ([(1, 9000)], 128, 1, 64),
                                              ([(17, 30)] * 60, 16, 2, 128), ([(2000, 0)], 8, 2, 128), ([(3, 129)], 100, 1, 128)])
def test_attention_bounded_waits_expire_and_the_context_stays_usable(lens, Hq, Hkv, D):
    """The test hook makes the repairs of value tiles wait for a barrier that nothing arrives at: they give up after 4096 polls, the
    other roles find no tile and give up behind them, copies and products under way are waited for, tensor memory is freed
    (the next call would not get it otherwise), the status is recorded, and the next call on the same workspace is an ordinary one."""
    m = rq()
    p = Paged(lens, Hkv, D, 16)
    q = p.queries(Hq)
    ws = m.alloc_workspace(m.paged_attention_workspace_bytes(p.T, len(lens), Hq, Hkv, D, 0))
    around = torch.full((p.T + 2, Hq * D), 3.0, dtype=BF, device="cuda")
    for i in range(4):
        m.debug_expire_next_wait(True, attention=True)
        m.paged_attention(q, *p.args(), workspace=ws, out=around[1:p.T + 1])
        assert m.check(ws) == TIMEOUT and "gave up" in m.last_error()
        torch.cuda.synchronize()
        assert (around[0] == 3).all() and (around[-1] == 3).all()
        out, lse = m.paged_attention(q, *p.args(), workspace=ws, lse=True)
        assert m.check(ws) == 0, m.last_error()
        hold(out, lse, q, p, D ** -0.5)


def test_attention_requests_to_expire_are_their_own():
    """A request for attention is not taken by calls of few rows or by other kernels, and can be withdrawn."""
    m = rq()
    p = Paged([(1, 90), (1, 5)], 2, 128, 16)
    q = p.queries(4)
    ws = m.alloc_workspace(m.paged_attention_workspace_bytes(2, 2, 4, 2, 128, 1))
    m.debug_expire_next_wait(True, attention=True)
    m.paged_attention(q, *p.args(), workspace=ws, max_new=1)
    assert m.check(ws) == 0
    m.debug_expire_next_wait(False)
    p = Paged([(90, 90)], 2, 128, 16)
    q = p.queries(4)
    ws = m.alloc_workspace(m.paged_attention_workspace_bytes(90, 1, 4, 2, 128, 0))
    out, lse = m.paged_attention(q, *p.args(), workspace=ws, lse=True)
    assert m.check(ws) == 0
    hold(out, lse, q, p, 128 ** -0.5)


def test_attention_waits_as_long_as_the_keys_take():
    """Nearly 2^31 keys (one page, over and over): each CTA goes through its share for most of a second, at whose end a repair is
    due.  Scores of 0 and values of powers of 2 make every sum exact: 2^-20 times up to 2^26 keys, in steps of 16 at least."""
    m = rq()
    page, pages, Hkv, D = 8192, 262135, 8, 64
    k = torch.zeros((1, page, Hkv, D), dtype=BF, device="cuda")
    value = 2.0 ** (torch.arange(Hkv * D, device="cuda") % 7 - 3.0) * (1 - 2 * (torch.arange(Hkv * D, device="cuda") % 2))
    v = value.view(1, 1, Hkv, D).expand(1, page, Hkv, D).to(BF).contiguous()
    q = torch.ones((1, 128 * Hkv * D), dtype=BF, device="cuda")
    ws = m.alloc_workspace(m.paged_attention_workspace_bytes(1, 1, 128 * Hkv, Hkv, D, 1))
    out, lse = m.paged_attention(q, k, v, ints([0, 1]), ints([page * pages]), torch.zeros((1, pages), dtype=I32, device="cuda"), lse=True, max_new=1,
                                 workspace=ws)
    assert m.check(ws) == 0, m.last_error()
    assert torch.equal(out.view(Hkv, 128, D), value.view(Hkv, 1, D).expand(Hkv, 128, D).to(BF))
    assert ((lse - math.log(page * pages)).abs() <= 64 * U * math.log(page * pages)).all()
