"""Rotation into a paged cache and attention over it on the GPU, against their definitions in 64 bits (paged_formulas.py).

Tolerances.  u = 2^-24 is half a step of fp32, and a rounding to bf16 is off by at most 2^-8 of the value.
  rotation   bias, two products and their sum are 4 roundings of terms of at most |x| + |y|; the angle is within 2^-32 of a turn
             (2 pi 2^-32 = 1.5e-9 rad), a sine or cosine of an fp32 number of half turns within pi 2^-25 + 2 u: together below 16 u of
             |x| + |y|, and then the output's own rounding.
  attention  a score is a sum of D <= 128 products that are exact in fp32: off by at most 2 u D times the sum of their
             magnitudes (2 u: tensor cores cut), so with a = max scale sum |q k| by 256 u a; the exponential's argument by 8 u a more, and
             the fast exponential by 2^-21.  Each weight is off by d = 264 u a + 2^-21 relative to the row, and by 2^-8 from its
             rounding to bf16; sum and products add their chain of at most keys / 8 + 256 additions.  So out is within
             (2^-8 + 2 d + 2 u chain) sum p |v| + 2^-8 |out|, lse within d + u (chain + 2 |lse|)."""
import pytest
import torch

import paged_formulas as formulas

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_BF = 2.0 ** -8
BF, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
NAN = float("nan")


def rq():
    import paper_2607_26515_b200 as m
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ints(v):
    return torch.tensor(v, dtype=I32, device="cuda")


class Paged:
    """Sequences of (new, past) tokens over a cache whose pages are dealt out at random; free pages and the rows of a page behind a
    sequence's keys hold NaN."""

    def __init__(self, lens, Hkv, D, page, seed=0, layout="token", spare=2, extra_pages=1, std=1.0):
        g = self.g = gen(seed)
        self.lens, self.Hkv, self.D, self.page = lens, Hkv, D, page
        used = [(n + p + page - 1) // page for n, p in lens]
        P = sum(used) + spare
        order = torch.randperm(P, generator=g, device="cuda").to(I32)
        self.table = torch.full((len(lens), max(used + [0]) + extra_pages), -7, dtype=I32, device="cuda")
        if layout == "head":
            both = torch.full((P, 2, Hkv, page, D), NAN, dtype=BF, device="cuda").transpose(2, 3)
            self.k, self.v = both[:, 0], both[:, 1]
        else:
            self.k, self.v = (torch.full((P, page, Hkv, D), NAN, dtype=BF, device="cuda") for _ in range(2))
        at = 0
        for b, (n, p) in enumerate(lens):
            ids = order[at:at + used[b]]
            at += used[b]
            self.table[b, :used[b]] = ids
            for c in (self.k, self.v):
                rows = torch.full((used[b] * page, Hkv, D), NAN, dtype=BF, device="cuda")
                rows[:n + p] = (torch.randn((n + p, Hkv, D), generator=g, device="cuda") * std).to(BF)
                if used[b]:
                    c[ids.long()] = rows.view(used[b], page, Hkv, D)
        self.starts = [0]
        for n, _ in lens:
            self.starts.append(self.starts[-1] + n)
        self.T = self.starts[-1]
        self.kv = [n + p for n, p in lens]
        self.q_start, self.kv_len = ints(self.starts), ints(self.kv)

    def queries(self, Hq, T=None, std=2.0, pad=0):
        T = self.T if T is None else T
        buf = torch.full((T, Hq * self.D + pad), NAN, dtype=BF, device="cuda")
        q = buf[:, :Hq * self.D]
        q.copy_(torch.randn((T, Hq * self.D), generator=self.g, device="cuda") * std)
        return q

    def args(self):
        return self.k, self.v, self.q_start, self.kv_len, self.table


def hold(got, lse, q, p, scale, what=""):
    """Asserts the call's results against the formulas."""
    want, want_lse, size, terms = formulas.attention(q, p.k, p.v, p.q_start.tolist(), p.kv_len.tolist(), p.table, scale)
    T, Hq = want_lse.shape
    row = torch.isfinite(want_lse) | (want_lse == float("-inf"))  # rows of a sequence
    chain = max(p.kv_len.tolist() + [0]) / 8 + 256
    d = 264 * U * terms + 2.0 ** -21
    el = row.repeat_interleave(p.D, 1)
    dd = d.repeat_interleave(p.D, 1)
    tol = (HALF_BF + 2 * dd + 2 * U * chain) * size + HALF_BF * want.abs()
    err = (got.double() - want).abs()
    bad = el & ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / tol.clamp_min(1e-30))[bad].nan_to_num(9e9).max()):.3g} of the tolerance"
    if lse is not None:
        none = want_lse == float("-inf")
        assert (lse[none] == float("-inf")).all(), what
        some = row & ~none
        e = (lse.double() - want_lse).abs()[some]
        t = (d + U * (chain + 2 * want_lse.abs()))[some]
        assert (e <= t).all(), f"{what}: lse off by {float((e / t).max())} of its tolerance"


def check(lens, Hq, Hkv, D, page, seed=0, layout="token", max_new="right", pad=0, **kw):
    p = Paged(lens, Hkv, D, page, seed, layout, **kw)
    q = p.queries(Hq, pad=pad)
    hint = {"right": max(n for n, _ in lens), "none": None, "small": 1}[max_new]
    out, lse = rq().paged_attention(q, *p.args(), max_new=hint, lse=True)
    hold(out, lse, q, p, D ** -0.5, f"{lens} {Hq}/{Hkv}x{D} pages of {page}")
    return p, q, out, lse


HEADS = [(16, 2, 128), (28, 4, 128), (14, 2, 64), (4, 4, 128), (6, 6, 64), (32, 1, 64), (9, 3, 128)]


@pytest.mark.parametrize("Hq, Hkv, D", HEADS)
@pytest.mark.parametrize("page", [8, 16, 24, 64, 256])
def test_attention_single_tokens(Hq, Hkv, D, page):
    check([(1, 0), (1, 6), (1, 7), (1, 62), (1, 63), (1, 64), (1, 127), (1, 128), (1, 1000), (1, 3)], Hq, Hkv, D, page, seed=page + Hq)


@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("past", [0, 1, 15, 16, 63, 200, 5000, 40001])
def test_attention_one_sequence(past, layout):
    check([(1, past)], 16, 2, 128, 16, seed=past, layout=layout)
    check([(1, past)], 7, 1, 64, 40, seed=past + 1, layout=layout)


@pytest.mark.parametrize("Hq, Hkv, D", HEADS)
@pytest.mark.parametrize("n", [2, 3, 5, 8])
def test_attention_drafts(n, Hq, Hkv, D):
    check([(n, 0), (n, 50), (1, 120), (max(1, n - 1), 700), (n, 64 - n), (n, 65 - n)], Hq, Hkv, D, 16, seed=n, layout="head")


@pytest.mark.parametrize("Hq, Hkv, D", HEADS)
@pytest.mark.parametrize("page", [8, 24, 128])
def test_attention_chunks(page, Hq, Hkv, D):
    check([(17, 0), (33, 5), (64, 64), (100, 300), (1, 77), (127, 1), (129, 0), (255, 700), (0, 9), (3, 0)], Hq, Hkv, D, page, seed=page)


@pytest.mark.parametrize("max_new", ["none", "small"])
def test_attention_does_not_depend_on_the_hint(max_new):
    check([(17, 0), (33, 5), (1, 300), (130, 64), (2, 1)], 16, 2, 128, 16, max_new=max_new)


@pytest.mark.parametrize("n, past", [(1024, 0), (1000, 3000), (300, 9000), (2, 20000), (777, 1)])
def test_attention_long(n, past):
    check([(n, past)], 8, 2, 128, 64, seed=n)
    check([(n, past), (1, past)], 3, 1, 64, 16, seed=n, layout="head")


def test_attention_many_sequences():
    lens = [((i * 7) % 5, (i * 131) % 400) for i in range(700)]
    check(lens, 4, 2, 64, 16, seed=3)
    check([(1, (i * 37) % 90) for i in range(4096)], 2, 1, 64, 8, seed=4)


@pytest.mark.parametrize("lens", [[(1, 100)], [(1, 0)], [(1, 300), (1, 5), (1, 1000)], [(2, 129), (1, 0)], [(40, 77)]])
@pytest.mark.parametrize("Hq, Hkv, D", [(128, 1, 64), (100, 1, 128), (130, 2, 64)])
def test_attention_large_groups(lens, Hq, Hkv, D):
    """More than 64 query heads per kv head: a single token fills half a tile."""
    check(lens, Hq, Hkv, D, 16, seed=Hq)


@pytest.mark.parametrize("n", [1, 12, 200])
def test_attention_heads_that_share_their_keys_in_memory(n):
    """A stride of 0, which tensor maps do not take."""
    p = Paged([(n, 70), (n, 3)], 1, 64, 16)
    wide = [c.expand(-1, -1, 3, -1) for c in (p.k, p.v)]
    q = p.queries(9)
    out = rq().paged_attention(q, *wide, p.q_start, p.kv_len, p.table)
    p.k, p.v = wide
    hold(out, None, q, p, 64 ** -0.5)


@pytest.mark.parametrize("page", [40, 48, 136, 512])
def test_attention_other_pages(page):
    check([(3, 500), (70, 300), (130, 137)], 8, 2, 128, page, seed=page)


def test_attention_strided_rows():
    check([(5, 100), (1, 30)], 6, 2, 128, 16, pad=4 * 128)
    p = Paged([(5, 100), (40, 30)], 2, 128, 16)
    q = p.queries(6)
    buf = torch.full((p.T + 1, 6 * 128 + 8), 5.0, dtype=BF, device="cuda")
    out = buf[:p.T, :6 * 128]
    assert rq().paged_attention(q, *p.args(), out=out, scale=0.05) is out
    hold(out, None, q, p, 0.05)
    assert (buf[p.T:] == 5).all() and (buf[:, 6 * 128:] == 5).all()


@pytest.mark.parametrize("max_new", [1, None])
def test_attention_rows_that_see_nothing(max_new):
    """No keys at all, fewer keys than new tokens, no new tokens; rows of no sequence stay as they were."""
    p = Paged([(2, 30), (3, 0), (5, 0), (1, 0), (0, 0), (40, 20)], 2, 128, 16)
    p.kv_len = ints([32, 0, 2, 1, 0, 60])
    q = p.queries(4, T=p.T + 9)
    out = torch.full_like(q, 3.0)
    _, lse = rq().paged_attention(q, *p.args(), lse=True, out=out, max_new=max_new)
    assert (out[p.T:] == 3).all()
    hold(out, lse, q, p, 128 ** -0.5)
    assert (out[2:5] == 0).all() and (lse[2:5] == float("-inf")).all()
    assert (out[5:8] == 0).all() and torch.isfinite(lse[8:10]).all()


@pytest.mark.parametrize("n", [1, 4, 50])
def test_attention_wild_arrays(n):
    """Starts out of order and out of range, lengths and pages out of range: no access leaves the tensors, and what is cut reads as
    the header says."""
    p = Paged([(n, 90), (n, 20), (n, 60), (n, 33)], 2, 64, 8)
    q = p.queries(4)
    p.kv_len = ints([10 ** 9, -5, p.kv[2], p.kv[3]])
    p.table[0, 12:] = 10 ** 6
    p.table[2, 1] = -1
    p.table[3, 0] = p.k.shape[0]
    p.k.nan_to_num_(0.5)
    p.v.nan_to_num_(0.25)
    out, lse = rq().paged_attention(q, *p.args(), lse=True)
    hold(out, lse, q, p, 64 ** -0.5)
    p.q_start = ints([-3, n, n + 1, 2 ** 31 - 1, -2 ** 31])
    out = torch.zeros_like(q)
    rq().paged_attention(q, *p.args(), out=out)
    hold(out, None, q, p, 64 ** -0.5)


@pytest.mark.parametrize("n, past", [(4, 100), (3, 61), (8, 120), (16, 100), (21, 50), (60, 40), (200, 500), (300, 0)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_strange_values_behind_a_token(n, past, D):
    """NaN and infinities in the keys and values of later tokens of the same chunk do not reach the earlier ones."""
    p = Paged([(n, past), (n, past + 3)], 2, D, 16)
    q = p.queries(6)
    bad = past + n // 2
    page, row = int(p.table[0, bad // 16]), bad % 16
    p.v[page, row, 0, 5] = NAN
    p.v[page, row, 1, 7] = float("inf")
    p.k[page, row, 1, 3] = float("-inf")
    page, row = int(p.table[1, (past + n + 2) // 16]), (past + n + 2) % 16
    p.v[page, row, 1] = float("inf")
    out, lse = rq().paged_attention(q, *p.args(), lse=True)
    want, want_lse, _, _ = formulas.attention(q, p.k, p.v, p.starts, p.kv, p.table, D ** -0.5)
    clean = torch.isfinite(want)
    assert torch.equal(torch.isfinite(out), clean)
    assert ((out.double() - want).abs()[clean] <= 0.05).all()
    # beyond the strange key only the columns that hold its values are strange
    assert clean[n // 2, 6 * D // 2 - 1] and not clean[n // 2, 5]


def test_attention_scores_of_all_sizes():
    """Scores up to the thousands, equal scores, and a key far above the others late in the sequence."""
    for std in (0.0, 1e-3, 8.0, 100.0):
        p = Paged([(3, 500), (70, 100)], 2, 128, 16, seed=5)
        q = p.queries(4, std=std)
        out, lse = rq().paged_attention(q, *p.args(), lse=True)
        hold(out, lse, q, p, 128 ** -0.5, f"std {std}")


def test_attention_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes and 2^31 elements, its last pages in use."""
    P, page, Hkv, D = 70000, 64, 4, 128
    k, v = (torch.empty((P, page, Hkv, D), dtype=BF, device="cuda") for _ in range(2))
    p = Paged([(1, 300), (2, 500), (60, 30)], Hkv, D, page)
    for c, small in ((k, p.k), (v, p.v)):
        c[P - small.shape[0]:] = small
    p.table = torch.where(p.table >= 0, p.table + (P - p.k.shape[0]), p.table)
    p.k, p.v = k, v
    q = p.queries(8)
    for hint in (2, None):
        out, lse = rq().paged_attention(q, *p.args(), lse=True, max_new=hint)
        hold(out, lse, q, p, D ** -0.5)


@pytest.mark.parametrize("Hq, Hkv, D", [(14, 2, 64), (16, 2, 128), (4, 4, 128)])
def test_attention_many_short_chunks_one_after_the_other(Hq, Hkv, D):
    """CTAs that go through several items of one tile or a few, with rows for one half of a tile or both: their parts hand buffers
    and barriers on from item to item.  Every run has to end in time and with the same bits."""
    m = rq()
    g = torch.Generator().manual_seed(D + Hq)
    n = torch.randint(1, 20, (300,), generator=g).tolist()
    past = torch.randint(0, 600, (300,), generator=g).tolist()
    past = [p if i % 3 else p * 5 for i, p in enumerate(past)]
    p = Paged([(a if i % 7 else 2 * a, b) for i, (a, b) in enumerate(zip(n, past))], Hkv, D, 16, seed=D)
    q = p.queries(Hq)
    ws = m.alloc_workspace(m.paged_attention_workspace_bytes(p.T, 300, Hq, Hkv, D, 0))
    first, lse = m.paged_attention(q, *p.args(), lse=True, workspace=ws)
    hold(first, lse, q, p, D ** -0.5)
    for _ in range(100):
        out = m.paged_attention(q, *p.args(), workspace=ws)
        assert m.check(ws) == 0, m.last_error()
        assert torch.equal(out, first)


def test_attention_is_the_same_from_run_to_run():
    p = Paged([(1, 5000), (5, 300), (90, 800)], 2, 128, 16)
    q = p.queries(16)
    first = rq().paged_attention(q, *p.args(), lse=True)
    for _ in range(3):
        again = rq().paged_attention(q, *p.args(), lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ------------------------------------------------------------------------------------------------ rotation and append

def freqs(rot, base=1e6):
    return base ** (-2.0 * torch.arange(rot // 2, dtype=F64, device="cuda") / max(rot, 1))


def check_append(lens, Hq, Hkv, D, page, rot, dtype=BF, bias=True, pairs=False, positions=False, layout="token", pad=0, T=None, kv=None, table=None,
                 in_place=False, seed=0):
    p = Paged(lens, Hkv, D, page, seed, layout)
    if kv is not None:
        p.kv_len = ints(kv)
    if table is not None:
        table(p)
    p.k.nan_to_num_(0.5)
    p.v.nan_to_num_(0.25)
    T = p.T if T is None else T
    W = (Hq + 2 * Hkv) * D
    buf = torch.full((T, W + pad), NAN, dtype=dtype, device="cuda")
    qkv = buf[:, :W]
    qkv.copy_(torch.randn((T, W), generator=p.g, device="cuda"))
    b = torch.randn(W, generator=p.g, device="cuda").to(BF) if bias else None
    pos = torch.randint(-2 ** 31, 2 ** 31, (T,), generator=p.g, device="cuda").to(I32) if positions else None
    want = formulas.rope_append(qkv.clone(), b, p.k, p.v, p.q_start.tolist(), p.kv_len.tolist(), p.table, freqs(rot), pairs, pos)
    # the sum of the magnitudes that meet in an element
    x = (qkv.double() + (0 if b is None else b.double())).abs()
    size = float(x.max()) * 2
    q = qkv[:, :Hq * D] if in_place else torch.full((T, Hq * D), 3.0, dtype=BF, device="cuda")
    before = (p.k.clone(), p.v.clone())
    got = rq().rope_append(qkv, *p.args(), freqs(rot), bias=b, positions=pos, pairs=pairs, q=q)
    assert got is q
    for name, g, w, old in (("q", q, want[0], None), ("k", p.k, want[1], before[0]), ("v", p.v, want[2], before[1])):
        there = ~torch.isnan(w)
        err = (g.double() - w).abs()
        tol = HALF_BF * w.abs() + 16 * U * size
        assert not (there & ~(err <= tol)).any(), f"{name}: {int((there & ~(err <= tol)).sum())} off, worst {float((err / tol)[there].max())}"
        if old is not None:  # what no token owns is as it was
            same = w == old.double()
            assert torch.equal(g[same], old[same])
    if not in_place:
        assert (q[torch.isnan(want[0])] == 3).all()
    return p, q


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("Hq, Hkv, D, rot", [(16, 2, 128, 128), (28, 4, 128, 64), (14, 2, 64, 64), (3, 3, 64, 16), (2, 1, 128, 0), (5, 1, 128, 96)])
def test_append(Hq, Hkv, D, rot, pairs, dtype):
    check_append([(1, 0), (3, 14), (9, 100), (1, 15), (17, 3), (0, 5), (2, 16)], Hq, Hkv, D, 16, rot, dtype, pairs=pairs, seed=rot)


@pytest.mark.parametrize("page", [8, 24, 256])
@pytest.mark.parametrize("layout", ["token", "head"])
def test_append_pages(page, layout):
    check_append([(30, 7), (1, 300)], 6, 2, 128, page, 128, layout=layout, pad=64, bias=False)


@pytest.mark.parametrize("T", [1, 591, 1183, 1184, 2400])
def test_append_rows_per_block(T):
    check_append([(T - T // 3, 5), (T // 3, 77)], 2, 1, 64, 16, 64, seed=T)


def test_append_many_sequences():
    check_append([((i * 5) % 3, (i * 13) % 40) for i in range(1100)], 2, 1, 64, 8, 64, seed=2)


def test_append_positions_of_any_size():
    check_append([(40, 3)], 4, 2, 128, 16, 128, positions=True)
    check_append([(40, 3)], 4, 2, 64, 16, 32, positions=True, pairs=True, dtype=F32)


def test_append_far_into_a_sequence():
    """Angles of positions near 2^30 (64-bit sums of turns; in fp32 they would be off by whole radians)."""
    p = Paged([(6, 10)], 2, 128, 16)
    pos = torch.arange(2 ** 30, 2 ** 30 + 6, device="cuda").to(I32)
    qkv = torch.randn((6, 8 * 128), generator=p.g, device="cuda").to(BF)
    want = formulas.rope_append(qkv, None, p.k, p.v, p.starts, p.kv, p.table, freqs(128), False, pos)[0]
    got = rq().rope_append(qkv, *p.args(), freqs(128), positions=pos)
    assert ((got.double() - want).abs() <= HALF_BF * want.abs() + 16 * U * 2 * float(qkv.abs().max())).all()


def test_append_in_place_of_the_queries():
    check_append([(5, 3), (70, 9)], 6, 2, 128, 16, 128, in_place=True, pad=8)


def test_append_rows_of_no_sequence_and_places_of_none():
    def table(p):
        p.table[0, 0] = -1
        p.table[1, 1] = p.k.shape[0]
    check_append([(20, 0), (3, 20), (6, 0), (2, 2)], 3, 1, 64, 8, 64, T=40, kv=[20, 23, 4, -9], table=table)


def test_append_on_another_stream_and_captured():
    m = rq()
    p = Paged([(1, 30), (1, 90)], 2, 128, 16)
    qkv = torch.randn((2, 8 * 128), generator=p.g, device="cuda").to(BF)
    want = m.rope_append(qkv, *p.args(), freqs(128)).clone()
    out = m.paged_attention(want, *p.args())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    q2 = m.rope_append(qkv, *p.args(), freqs(128), stream=s)
    out2 = m.paged_attention(q2, *p.args(), stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(q2, want) and torch.equal(out, out2)
    # captured once, replayed while the sequences grow
    static, inv = qkv.clone(), freqs(128)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q3 = m.rope_append(static, *p.args(), inv)
        out3, lse3 = m.paged_attention(q3, *p.args(), lse=True, max_new=1)
    for step in range(3):
        p.kv_len += 1
        static.copy_(torch.randn((2, 8 * 128), generator=p.g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = formulas.rope_append(static, None, p.k, p.v, p.starts, p.kv_len.tolist(), p.table, inv, False)
        assert ((q3.double() - want[0]).abs() <= HALF_BF * want[0].abs() + 16 * U * 2 * float(static.abs().max())).all()
        hold(out3, lse3, q3, p, 128 ** -0.5, f"step {step}")


# ------------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("Hq, Hkv, D", [(16, 2, 128), (14, 2, 64)])
def test_prompt_in_pieces_is_the_prompt_at_once(Hq, Hkv, D):
    """A prompt appended and attended to at once, in chunks, and token by token gives the same rows up to the roundings."""
    m, n, page = rq(), 150, 16
    g = gen(1)
    qkv = torch.randn((n, (Hq + 2 * Hkv) * D), generator=g, device="cuda").to(BF)
    results = []
    for cuts in ([150], [70, 50, 30], [140] + [1] * 10):
        k, v = (torch.full((10, page, Hkv, D), NAN, dtype=BF, device="cuda") for _ in range(2))
        table = torch.arange(10, dtype=I32, device="cuda")[None].flip(1).contiguous()
        rows, at = [], 0
        for c in cuts:
            seq = (ints([0, c]), ints([at + c]), table)
            q = m.rope_append(qkv[at:at + c], k, v, *seq, freqs(D))
            rows.append(m.paged_attention(q, k, v, *seq))
            at += c
        results.append((torch.cat(rows), k, v))
    for out, k, v in results[1:]:
        assert torch.equal(k.view(torch.int16), results[0][1].view(torch.int16)) and torch.equal(v.view(torch.int16), results[0][2].view(torch.int16))
        # each is within 2^-8 of its weights and 2^-8 of its value; values here are below 6 in magnitude
        assert ((out.double() - results[0][0].double()).abs() <= 4 * HALF_BF * 6).all()
