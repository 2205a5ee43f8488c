"""The few-token 4-bit product, the residual-stream join and the token log-probabilities on the GPU, against their definitions
in 64 bits (operator_formulas.py and a decoder of the packed formats written here).

Tolerances.  u = 2^-24 is half a step of fp32, and a rounding to bf16 is off by at most 2^-8 of the value.
  product    products of decoded weights and bf16 activations are exact in fp32; a sum of n terms along a chain of d additions is
             off by at most 2 d u sum |terms| (2 u: the tensor cores cut instead of rounding); d <= K / 32 + 64.
  join       every elementary step is within a few u of its value, a sum along d <= 64 additions within d u of its terms'
             magnitudes: 2^-16 = 256 u of the magnitudes of the terms covers all of them together.
  logprobs   exp((x - max) / T): the argument y is within 2 u |y|, so the term within (2 |y| + 4) u of its value; the sums add
             d u with d <= V / 256 + 64 additions in a chain.  E |y| under the row's distribution weighs the first part."""
import pytest
import torch

from operator_formulas import join, join_gradient_sizes, join_gradients, log_softmax, logprobs, logprobs_gradient

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def rq():
    import paper_2607_26515_b200 as m
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rows(M, K, dtype, pad=0, fill=float("nan")):
    """A view [M, K] of a buffer with a pitch that is a multiple of 8, and the buffer."""
    buf = torch.full((M, (K + 7) // 8 * 8 + pad), fill, dtype=dtype, device="cuda")
    return buf[:, :K], buf


def randn(M, K, dtype, g, std=1.0, pad=0):
    t, _ = rows(M, K, dtype, pad)
    t.copy_(torch.randn((M, K), generator=g, device="cuda") * std)
    return t


def close(got, want, tol, what=""):
    err = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all(), what
    bad = err > tol
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / tol.clamp_min(1e-300)).max()):.3g} of the tolerance"


# ------------------------------------------------------------------------------------------------ few-token product

def decode(codes, side, fmt):
    """The packed weights in 64 bits, from the layout that the header states."""
    N, K = codes.shape[0], codes.shape[1] * 2
    c = codes.long()
    code = torch.stack((c & 15, c >> 4), -1).view(N, K)
    sign = 1.0 - 2.0 * (code >> 3).double()
    k = torch.arange(K, device=codes.device)
    if fmt == "hif4":
        m = (side.long() & 0xFFFFFFFF)[:, k // 64]
        e = ((m >> 2) & 63) - 48 + ((m >> (8 + k % 64 // 8)) & 1) + ((m >> (16 + k % 64 // 4)) & 1)
        return sign * (code & 7) / 4 * (1 + (m & 3).double() / 4) * torch.pow(2.0, e.double())
    mag = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=F64, device=codes.device)[code & 7]
    return sign * mag * torch.pow(2.0, (side.long()[:, k // 32] - 127).double())


def gemv_tol(x, w, y, out):
    return 2 * U * (x.shape[1] / 32 + 64) * (x.abs() @ w.abs().T) + (HALF[out] * y.abs() if out == BF else 0)


def check_gemv(x, codes, side, fmt, out):
    y = rq().w4a16_gemv(x, codes, side, fmt, out_dtype=out)
    w, x8 = decode(codes, side, fmt), x.double()
    want = x8 @ w.T
    assert y.dtype == out and y.shape == want.shape
    close(y, want, gemv_tol(x8, w, want, out), f"{fmt} {tuple(x.shape)} {codes.shape[0]}")
    return y


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("fmt", ["hif4", "mxfp4"])
@pytest.mark.parametrize("M, N, K", [(1, 1, 64), (1, 16, 128), (2, 17, 192), (3, 130, 320), (5, 77, 2048), (8, 250, 704), (9, 33, 448),
                                     (16, 129, 1152), (1, 2048, 2048), (4, 3584, 1088), (7, 1000, 4160), (16, 64, 18944), (6, 2, 11008),
                                     (16, 40, 32768), (11, 33, 49152), (8, 16, 49152), (1, 700, 49152)])
def test_gemv_parity(M, N, K, fmt, out):
    m, g = rq(), gen(M * 1000 + N + K)
    codes, side = m.pack_weight(randn(N, K, BF, g, 0.02), fmt)
    x = randn(M, K, BF, g, pad=16)
    x[:, ::97] *= 50
    check_gemv(x, codes, side, fmt, out)


@pytest.mark.parametrize("K", [32, 96, 160, 224, 288, 2080])
def test_gemv_mxfp4_odd_numbers_of_blocks(K):
    """K / 32 odd: rows of scales that start on odd bytes, a last unit of one to three blocks."""
    m, g = rq(), gen(K)
    codes, side = m.pack_weight(randn(35, K, BF, g), "mxfp4")
    check_gemv(randn(3, K, BF, g), codes, side, "mxfp4", F32)


@pytest.mark.parametrize("fmt", ["hif4", "mxfp4"])
def test_gemv_every_code_and_scale(fmt):
    """Random codes and side words: every nibble in every place, every micro-exponent, scales over the whole range that
    leaves the product finite."""
    g = gen(5)
    N, K = 256, 512
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
    if fmt == "hif4":
        side = torch.randint(-2 ** 31, 2 ** 31, (N, K // 64), generator=g, device="cuda").to(torch.int32)
        side[:, 0] = (side[:, 0] & ~255) | torch.arange(N, device="cuda", dtype=torch.int32)
    else:
        # one scale code for each row, 0 to 254; rows of large and small weights apart
        side = torch.arange(N, device="cuda").clamp_max(254).to(torch.uint8)[:, None].expand(N, K // 32).contiguous()
    x = randn(2, K, BF, g, 2.0 ** -20)
    if fmt == "mxfp4":
        x *= 2.0 ** -2
    y = rq().w4a16_gemv(x, codes, side, fmt, out_dtype=F32)
    w, x8 = decode(codes, side, fmt), x.double()
    want = x8 @ w.T
    # below 2^-126 a product of the tensor cores may be cut to the subnormal grid (or to 0): K terms of at most 2^-126
    tol = gemv_tol(x8, w, want, F32) + K * 2.0 ** -126
    # the two largest MXFP4 scales, 2^126 and 2^127, take the elements 4 and 6 past the range of bf16 and fp32 (4 * 2^126 =
    # 2^128): those weights are infinite, here as in the library's decoder, and the row is not finite
    fits = (w.abs().amax(-1) < 2.0 ** 128)
    assert fits.all() if fmt == "hif4" else (~fits).sum() == 3
    assert torch.isinf(rq().dequantize(codes, side, fmt)).any(-1).equal(~fits)
    close(y[:, fits], want[:, fits], tol[:, fits], fmt)
    assert not y[:, ~fits].isfinite().any()


@pytest.mark.parametrize("fmt", ["hif4", "mxfp4"])
def test_gemv_rows_are_independent(fmt):
    """NaN and infinity stay in their token's row; each row has the bits that it has alone among the same number of rows."""
    m, g = rq(), gen(11)
    codes, side = m.pack_weight(randn(70, 256, BF, g), fmt)
    x = randn(6, 256, BF, g)
    clean = m.w4a16_gemv(x, codes, side, fmt, out_dtype=F32)
    x[2, 7], x[4, 0] = float("nan"), float("inf")
    y = m.w4a16_gemv(x, codes, side, fmt, out_dtype=F32)
    for i in (0, 1, 3, 5):
        assert torch.equal(y[i], clean[i])
    assert y[2].isnan().all()
    assert not y[4].isfinite().any()


def test_gemv_leaves_the_padding_alone():
    m, g = rq(), gen(12)
    codes, side = m.pack_weight(randn(21, 128, BF, g))
    x = randn(3, 128, BF, g)
    for out in (BF, F32):
        y, buf = rows(3, 21, out, pad=8, fill=7.0)
        assert m.w4a16_gemv(x, codes, side, Y=y) is y
        assert (buf[:, 21:] == 7).all() and torch.equal(y, m.w4a16_gemv(x, codes, side, out_dtype=out))


def test_gemv_agrees_with_the_linear_call_and_repeats_itself():
    m, g = rq(), gen(13)
    codes, side = m.pack_weight(randn(2560, 2048, BF, g, 0.02))
    x = randn(4, 2048, BF, g)
    y = m.w4a16_gemv(x, codes, side, out_dtype=F32)
    assert torch.equal(y, m.w4a16_gemv(x, codes, side, out_dtype=F32))
    w, x8 = decode(codes, side, "hif4"), x.double()
    tol = gemv_tol(x8, w, None, F32) + 1e-5 * (x8.abs() @ w.abs().T) + 2e-3 * (x8 @ w.T).abs()
    close(y, m.w4a16_linear(x, codes, side, out_dtype=F32).double(), tol)


def test_gemv_behind_four_gigabytes():
    """Row offsets beyond 2^32 bytes of codes and 2^31 of metadata words' bytes."""
    m, g = rq(), gen(14)
    K = 18944
    N = 2 ** 32 // (K // 2) + 40
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    side = torch.full((N, K // 64), 150, dtype=torch.int32, device="cuda")
    x = randn(2, K, BF, g)
    y = m.w4a16_gemv(x, codes, side, out_dtype=F32)
    for at in (slice(0, 20), slice(N - 40, N)):
        w, x8 = decode(codes[at], side[at], "hif4"), x.double()
        want = x8 @ w.T
        close(y[:, at], want, gemv_tol(x8, w, want, F32))


def test_gemv_refuses_in_the_binding():
    m, g = rq(), gen(15)
    codes, side = m.pack_weight(randn(16, 128, BF, g))
    x = randn(2, 128, BF, g)
    for bad in (lambda: m.w4a16_gemv(randn(2, 64, BF, g), codes, side), lambda: m.w4a16_gemv(x.float(), codes, side),
                lambda: m.w4a16_gemv(x, codes[:, ::2], side), lambda: m.w4a16_gemv(x, codes, side[:, :1]),
                lambda: m.w4a16_gemv(x, codes, side, "mxfp4"), lambda: m.w4a16_gemv(x, codes.cpu(), side),
                lambda: m.w4a16_gemv(x, codes, side, out_dtype=torch.float16), lambda: m.w4a16_gemv(x.t(), codes, side),
                lambda: m.w4a16_gemv(x, codes, side, Y=torch.empty((2, 15), device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(m.ResqError) as e:
        m.w4a16_gemv(randn(17, 128, BF, g), codes, side)
    assert e.value.status == 2


# ------------------------------------------------------------------------------------------------ residual stream

def join_case(M, K, stream, post, gate, seed, pad=0):
    g = gen(seed)
    v = {"H": randn(M, K, stream, g, 2.0, pad), "B": randn(M, K, BF, g, 0.5, pad),
         "gamma_pre": (1 + 0.2 * torch.randn(K, generator=g, device="cuda")).to(BF),
         "gamma_post": (1 + 0.2 * torch.randn(K, generator=g, device="cuda")).to(BF) if post else None, "gate": None}
    if gate == "channel":
        v["gate"] = torch.randn(K, generator=g, device="cuda").to(BF)
    elif gate == "full":
        v["gate"] = randn(M, K, BF, g, pad=pad)
    return v


def wide(v):
    return [None if t is None else t.double() for t in v]


SHAPES = [(1, 1), (1, 8), (3, 5), (2, 64), (5, 257), (4, 1000), (300, 96), (2, 2048), (33, 3584), (3, 5003), (2, 8200), (7, 5130), (2, 18944), (3, 24577), (3, 26000), (1, 32768)]
FORMS = [(BF, False, "none", "linear"), (F32, True, "channel", "linear"), (BF, True, "full", "sigmoid"), (F32, False, "channel", "sigmoid"),
         (BF, True, "none", "linear"), (F32, False, "full", "linear")]


@pytest.mark.parametrize("stream, post, gate, act", FORMS)
@pytest.mark.parametrize("M, K", SHAPES)
def test_join_parity(M, K, stream, post, gate, act):
    v = join_case(M, K, stream, post, gate, M + K, pad=8)
    alpha, eps = 0.7, 1e-5
    H, X = rq().block_join(**v, act=act, alpha=alpha, eps=eps)
    w = {n: None if t is None else t.double() for n, t in v.items()}
    h, x = join(w["H"], w["B"], w["gamma_pre"], w["gamma_post"], w["gate"], act, alpha, eps)
    assert H.dtype == stream and X.dtype == BF
    size = w["H"].abs() + (h - w["H"]).abs()
    close(H, h, 2.0 ** -16 * size + HALF[stream] * h.abs(), "H")
    r = 1 / torch.sqrt(h.square().mean(-1, keepdim=True) + eps)
    close(X, x, 2.0 ** -16 * (size * r * w["gamma_pre"].abs() + x.abs()) + HALF[BF] * x.abs(), "X")


@pytest.mark.parametrize("stream, post, gate, act", FORMS)
@pytest.mark.parametrize("M, K", SHAPES + [(2500, 64), (1500, 1030)])
def test_join_backward_parity(M, K, stream, post, gate, act):
    v = join_case(M, K, stream, post, gate, M + 2 * K, pad=8)
    g = gen(3)
    dHo, dX = randn(M, K, stream, g, 0.5, 8), randn(M, K, BF, g, 0.5, 8)
    alpha, eps = -1.3, 1e-5
    got = rq().block_join_backward(dHo, dX, v["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], act, alpha, eps)
    args = wide([dHo, dX, v["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"]]) + [act, alpha, eps]
    want, size = join_gradients(*args), join_gradient_sizes(*args)
    assert sorted(got) == sorted(want)
    for name in want:
        half = HALF[got[name].dtype] * want[name].abs()
        # column sums: a chain of M / 148 + 300 additions at the very most
        chain = U * (M / 148 + 300) if want[name].dim() == 1 else 0.0
        close(got[name], want[name], (2.0 ** -16 + chain) * size[name] + half, name)


def test_join_one_gradient_missing():
    v = join_case(37, 520, F32, True, "full", 1)
    g = gen(4)
    dHo, dX = randn(37, 520, F32, g), randn(37, 520, BF, g)
    for a, b in ((dHo, None), (None, dX)):
        got = rq().block_join_backward(a, b, v["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], "sigmoid", 0.5, 1e-6)
        args = wide([a, b, v["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"]]) + ["sigmoid", 0.5, 1e-6]
        want, size = join_gradients(*args), join_gradient_sizes(*args)
        assert sorted(got) == sorted(want) and ("dgamma_pre" in got) == (b is not None)
        for name in want:
            close(got[name], want[name], 2.0 ** -15 * size[name] + HALF[got[name].dtype] * want[name].abs(), name)


def test_join_without_the_next_norm():
    v = join_case(9, 300, BF, True, "none", 2)
    v["gamma_pre"] = None
    H, X = rq().block_join(**v, alpha=2.0, eps=1e-6)
    h, _ = join(v["H"].double(), v["B"].double(), None, v["gamma_post"].double(), None, "linear", 2.0, 1e-6)
    assert X is None
    close(H, h, 2.0 ** -16 * (v["H"].double().abs() + (h - v["H"].double()).abs()) + HALF[BF] * h.abs())


def test_join_rows_of_zeros_and_large_values():
    """A row of zeros has the norm 1 / sqrt(eps) of nothing: zeros, and finite gradients; eps = 0 there is 0 * inf."""
    m = rq()
    v = join_case(4, 264, BF, True, "full", 3)
    v["H"][1], v["B"][1] = 0, 0
    v["gate"][2], v["gate"][3] = -200, 200
    H, X = m.block_join(**v, act="sigmoid", alpha=1.0, eps=1e-6)
    assert not H[1].any() and not X[1].any()
    assert torch.equal(H[2], v["H"][2])  # a closed gate adds nothing
    g = m.block_join_backward(H, X, H, v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], "sigmoid", 1.0, 1e-6)
    assert all(t.isfinite().all() for t in g.values())
    assert not g["dgate"][2].any()
    v["H"][0, 5] = float("nan")
    H2, X2 = m.block_join(**v, act="sigmoid", alpha=1.0, eps=1e-6)
    assert X2[0].isnan().all() and torch.equal(H2[1:], H[1:]) and torch.equal(X2[1:], X[1:])


@pytest.mark.parametrize("K", [64, 1003, 5003])
@pytest.mark.parametrize("stream", [BF, F32])
def test_join_in_place_and_padding(K, stream):
    m = rq()
    v = join_case(21, K, stream, True, "full", K)
    want_h, want_x = m.block_join(**v, alpha=0.5)
    h, hbuf = rows(21, K, stream, pad=8, fill=3.0)
    x, xbuf = rows(21, K, BF, pad=8, fill=4.0)
    h.copy_(v["H"])
    got_h, got_x = m.block_join(**{**v, "H": h}, alpha=0.5, H_out=h, X=x)
    assert got_h is h and got_x is x and torch.equal(h, want_h) and torch.equal(x, want_x)
    assert (hbuf[:, K:] == 3).all() and (xbuf[:, K:] == 4).all()
    g = gen(9)
    dHo, dX = randn(21, K, stream, g), randn(21, K, BF, g)
    args = (v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], "linear", 0.5)
    want = m.block_join_backward(dHo, dX, want_h, *args)
    d, dbuf = rows(21, K, stream, pad=16, fill=5.0)
    d.copy_(dHo)
    got = m.block_join_backward(d, dX, want_h, *args, dH=d)
    assert (dbuf[:, K:] == 5).all() and all(torch.equal(got[n], want[n]) for n in want)


def test_join_backward_repeats_itself_bit_for_bit():
    m = rq()
    v = join_case(4000, 520, F32, True, "channel", 5)
    g = gen(6)
    dHo, dX = randn(4000, 520, F32, g), randn(4000, 520, BF, g)
    run = lambda: m.block_join_backward(dHo, dX, v["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"])
    a, b = run(), run()
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_join_refuses_in_the_binding():
    m = rq()
    v = join_case(4, 64, BF, True, "full", 6)
    H = v["H"]
    for bad in (dict(B=v["B"].float()), dict(B=v["B"][:, :56]), dict(gamma_pre=v["gamma_pre"][:32]), dict(gate=v["gate"][:2]),
                dict(gate=v["gate"][:1].expand(4, 64)), dict(act="tanh"), dict(H=H.half()), dict(gamma_post=v["gamma_post"].float()),
                dict(H=H.t()), dict(B=v["B"].cpu()), dict(X=torch.empty((4, 64), device="cuda")), dict(H_out=torch.empty((4, 64), device="cuda"))):
        with pytest.raises(ValueError):
            m.block_join(**{**v, **bad})
    with pytest.raises(m.ResqError):
        m.block_join(**v, eps=-1.0)
    with pytest.raises(ValueError):
        m.block_join_backward(None, None, H, v["B"], v["gamma_pre"])
    with pytest.raises(ValueError):
        m.block_join_backward(None, v["B"], H, v["B"])
    with pytest.raises(m.ResqError):
        m.block_join_backward(H, None, H, v["B"], workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


# ------------------------------------------------------------------------------------------------ log-probabilities

def check_logprobs(x, tok, T=1.0, top=0):
    got = rq().token_logprobs(x, tok, temperature=T, top=top)
    x8, V = x.double(), x.shape[1]
    want = logprobs(x8, tok, T, top)
    z = x8 / T
    far = (z - z.amax(-1, keepdim=True)).abs()
    lp = log_softmax(z)
    spread = (lp.exp() * far.clamp_max(1e30)).sum(-1)
    base = U * (8 + 4 * spread + V / 256 + 64)          # absolute error of log s
    there = (tok >= 0) & (tok < V)
    ft = far.gather(1, torch.where(there, tok, torch.zeros_like(tok))[:, None])[:, 0]
    fin = want["logp"].isfinite()
    assert torch.equal(got["logp"].isfinite(), fin) and torch.equal(got["logp"][~fin].double(), want["logp"][~fin])
    close(got["logp"][fin], want["logp"][fin], (base + 4 * U * ft + 2 * U * want["logp"].abs())[fin] + 1e-30, "logp")
    assert torch.equal(got["peak"].double(), want["peak"])
    close(got["log_sum"], want["log_sum"], base + 2 * U * want["log_sum"], "log_sum")
    # entropy: sum of p |log p|, each term within (4 + 4 y) u of itself, y up to the row's spread where p counts
    second = (lp.exp() * far.clamp_max(1e30).square()).sum(-1)
    close(got["entropy"], want["entropy"], base * (2 + spread) + 8 * U * (second + spread), "entropy")
    if top:
        assert torch.equal(got["top_ids"], want["top_ids"])
        tf = far.gather(1, want["top_ids"].long())
        ok = want["top_logp"].isfinite()
        assert torch.equal(got["top_logp"].isfinite(), ok)
        close(got["top_logp"][ok], want["top_logp"][ok], (base[:, None] + 4 * U * tf + 2 * U * want["top_logp"].abs())[ok], "top_logp")
    return got


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M, V, top", [(1, 1, 1), (3, 2, 2), (2, 7, 5), (5, 31, 31), (4, 100, 32), (7, 1000, 20), (300, 257, 3), (2, 4099, 8),
                                       (1, 50001, 20), (17, 50001, 32), (3, 131072, 5), (1, 200003, 32), (600, 9001, 0), (200, 20011, 1)])
def test_logprobs_parity(M, V, top, dtype):
    g = gen(M + V)
    x = randn(M, V, dtype, g, 2.5, pad=8)
    tok = torch.randint(0, V, (M,), generator=g, device="cuda")
    tok[::3] = x[::3].double().argmax(-1)
    check_logprobs(x, tok, 1.0, top)
    check_logprobs(x, tok, 0.6, top)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [40, 3000, 70001])
def test_logprobs_ties_go_to_the_lowest_id(V, dtype):
    """Whole rows of one value, few values, -0 among 0, rising and falling rows, and the largest in every kind of place."""
    g = gen(V)
    few = torch.randint(-2, 3, (5, V), generator=g, device="cuda").float()
    zeros = torch.zeros((1, V), device="cuda")
    zeros[0, ::2] = -0.0
    ramp = torch.arange(V, device="cuda").float()[None] / V * 8
    spikes = torch.zeros((1, V), device="cuda")
    spikes[0, -1] = spikes[0, 0] = spikes[0, V // 2] = 3
    block = torch.zeros((1, V), device="cuda")
    block[0, V // 2:V // 2 + 40] = 1 + torch.arange(min(40, V - V // 2), device="cuda").float() / 64
    x, _ = rows(10, V, dtype, 8)
    x.copy_(torch.cat([few, zeros, ramp, -ramp, spikes, block]))
    tok = torch.randint(0, V, (10,), generator=g, device="cuda")
    for top in (1, 7, 32):
        check_logprobs(x, tok, 1.0, top)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [50, 5000, 60001])
def test_logprobs_masked_rows(V, dtype):
    g = gen(V + 1)
    x = randn(7, V, dtype, g, 3.0)
    inf = float("inf")
    x[6] = torch.where(torch.rand(V, generator=g, device="cuda") < 0.9, torch.finfo(dtype).min, x[6].float()).to(dtype)
    x[6, 7] = 1.0
    x[1] = torch.where(torch.rand(V, generator=g, device="cuda") < 0.9, -inf, x[1].float()).to(dtype)
    x[1, 3] = 0.5
    x[2] = -inf
    x[2, V - 1] = -4.0                       # one place left
    x[3] = -inf                              # none left
    x[4] = torch.finfo(dtype).min            # the lowest value is a value
    tok = torch.tensor([0, 3, 0, 1, 5, -7, 7], device="cuda")
    m = rq()
    got = m.token_logprobs(x, tok, top=32)
    live = [0, 1, 2, 4, 5, 6]
    for top in (1, 20):
        check_logprobs(randn(6, V, dtype, g).copy_(x[live]), tok[live], 1.0, top)
    assert got["logp"][2] == -inf and got["entropy"][2] == 0 and got["peak"][2] == -4 and got["log_sum"][2] == 0
    assert got["top_ids"][2].tolist() == [V - 1] + list(range(31)) and got["top_logp"][2, 0] == 0 and (got["top_logp"][2, 1:] == -inf).all()
    assert got["logp"][3] == -inf and got["entropy"][3] == 0 and got["peak"][3] == -inf and got["log_sum"][3] == 0
    assert got["top_ids"][3].tolist() == list(range(32)) and (got["top_logp"][3] == -inf).all()
    assert got["logp"][5] == 0               # no token named
    one = torch.ones(7, device="cuda")
    d = m.token_logprobs_backward(x, tok, got["logp"], got["peak"], got["log_sum"], got["entropy"], one, one)
    assert d.isfinite().all() and not d[3].any() and not d[1][x[1] == -inf].any()
    # a row of the type's lowest value: every p is 1 / V, and log p + entropy = 0 to (8 + 4 log V + V / 256 + 64) u
    flat = torch.full((V,), -1.0 / V, dtype=F64, device="cuda")
    flat[5] += 1
    close(d[4], flat, (HALF[dtype] + U * (100 + V / 128)) * flat.abs() + U * (100 + V / 128) / V, "lowest")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_logprobs_best_in_few_lanes(dtype):
    """The largest logits where a division of the row into strides puts them together: more of them than the selection keeps
    at hand, and whole groups of neighbours; with NaN and +inf among the logits their order is defined too."""
    m, g = rq(), gen(77)
    V = 160000
    for stride in (8 * 256, 8 * 1024, 8 * 32, 16 * 256, 1):
        x = randn(3, V, dtype, g, 1.0)
        at = (torch.arange(0, 2000, device="cuda")[:, None] * stride + torch.arange(8, device="cuda")).flatten() % V
        x[0, at] = (20 + torch.rand(at.numel(), generator=g, device="cuda")).to(dtype)
        x[1, at] = 20
        x[2] = torch.arange(V, device="cuda").to(dtype)
        check_logprobs(x, torch.tensor([5, 6, 7], device="cuda"), 1.0, 32)
    x = randn(2, 5000, dtype, g, 1.0)
    x[0, 0] = x[0, 4999] = x[1, 3] = float("nan")
    x[0, 9] = x[1, 2] = float("inf")
    ids = m.token_logprobs(x, torch.zeros(2, dtype=torch.int64, device="cuda"), top=3)["top_ids"].tolist()
    assert ids[0] == [0, 4999, 9] and ids[1][:2] == [3, 2]


def test_logprobs_infinity_and_nan_spoil_their_row_only():
    m, g = rq(), gen(21)
    for dtype in (BF, F32):
        x = randn(4, 3001, dtype, g, 2.0)
        tok = torch.tensor([5, 6, 7, 8], device="cuda")
        clean = m.token_logprobs(x, tok, top=4)
        x[1, 2900], x[2, 17] = float("inf"), float("nan")
        got = m.token_logprobs(x, tok, top=4)
        for n in clean:
            assert torch.equal(got[n][[0, 3]], clean[n][[0, 3]])
        assert all(got[n][1:3].isnan().all() for n in ("logp", "entropy", "peak", "log_sum", "top_logp"))
        assert got["top_ids"][1, 0] == 2900 and got["top_ids"][2, 0] == 17


def test_logprobs_near_certainty():
    """A token that holds nearly all of the probability: -logp is the sum of the others, to 2^-18 of itself (V / 256 + 64
    additions and the arguments' |y| <= 20: under 200 u)."""
    for V in (1000, 131072):
        x = torch.zeros((1, V), dtype=F32, device="cuda")
        x[0, 77] = 30.0
        tok = torch.tensor([77], device="cuda")
        got, want = rq().token_logprobs(x, tok), logprobs(x.double(), tok, 1.0)
        assert abs(float(got["logp"] / want["logp"]) - 1) < 2.0 ** -14
        assert abs(float(got["entropy"] / want["entropy"]) - 1) < 2.0 ** -14
        one = torch.ones(1, device="cuda")
        d = rq().token_logprobs_backward(x, tok, got["logp"], got["peak"], got["log_sum"], None, one)
        ref = logprobs_gradient(x.double(), tok, one.double(), None, 1.0)
        assert abs(float(d[0, 77].double() / ref[0, 77]) - 1) < 2.0 ** -14


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M, V, T, entropy", [(1, 1, 1.0, True), (2, 9, 0.5, True), (5, 1000, 1.0, False), (3, 4099, 1.7, True), (40, 50001, 1.0, True),
                                              (2, 131072, 0.7, False), (700, 130, 1.0, True)])
def test_logprobs_backward_parity(M, V, T, entropy, dtype):
    m, g = rq(), gen(M * V)
    x = randn(M, V, dtype, g, 2.5, pad=8)
    tok = torch.randint(-1, V, (M,), generator=g, device="cuda")
    tok[0] = V + 3 if M > 1 else 0
    fwd = m.token_logprobs(x, tok, temperature=T)
    dlogp = torch.randn(M, generator=g, device="cuda")
    dent = torch.randn(M, generator=g, device="cuda") if entropy else None
    got = m.token_logprobs_backward(x, tok, fwd["logp"], fwd["peak"], fwd["log_sum"], fwd["entropy"], dlogp, dent, temperature=T)
    x8 = x.double()
    want = logprobs_gradient(x8, tok, dlogp.double(), None if dent is None else dent.double(), T)
    z = x8 / T
    lp = log_softmax(z)
    p = lp.exp()
    hot = torch.zeros_like(p)
    there = (tok >= 0) & (tok < V)
    hot[torch.arange(M, device="cuda")[there], tok[there]] = 1
    H = -(p * lp).sum(-1, keepdim=True)
    # p is off by the error of log p (the sums of the forward call and the roundings of z - max); 1 - p like p
    dz = U * (80 + V / 256 + 8 * (z.amax(-1, keepdim=True) - z) + 8 * (lp.abs() + H))
    size = (dlogp.double().abs()[:, None] * p) + (0 if dent is None else dent.double().abs()[:, None] * p * (1 + lp.abs() + H))
    close(got, want, dz * size / T + 4 * U * want.abs() + HALF[dtype] * want.abs() + 1e-38, "dlogits")


def test_logprobs_backward_in_place_and_padding():
    m, g = rq(), gen(31)
    for dtype in (BF, F32):
        x, buf = rows(9, 1003, dtype, pad=8, fill=6.0)
        x.copy_(randn(9, 1003, dtype, g, 2.0))
        tok = torch.randint(0, 1003, (9,), generator=g, device="cuda")
        f = m.token_logprobs(x, tok)
        d = torch.randn(9, generator=g, device="cuda")
        want = m.token_logprobs_backward(x, tok, f["logp"], f["peak"], f["log_sum"], f["entropy"], d, d)
        got = m.token_logprobs_backward(x, tok, f["logp"], f["peak"], f["log_sum"], f["entropy"], d, d, dlogits=x)
        assert got is x and torch.equal(x, want) and (buf[:, 1003:] == 6).all()


def test_logprobs_behind_two_to_the_31_elements():
    m, g = rq(), gen(32)
    V = 131072
    M = 2 ** 31 // V + 3
    x = torch.empty((M, V), dtype=BF, device="cuda").normal_(generator=g)
    tok = torch.randint(0, V, (M,), generator=g, device="cuda")
    got = m.token_logprobs(x, tok, top=2)
    want = logprobs(x[-4:].double(), tok[-4:], 1.0, 2)
    assert torch.equal(got["top_ids"][-4:], want["top_ids"])
    assert torch.allclose(got["logp"][-4:].double(), want["logp"], rtol=0, atol=1e-4)
    one = torch.ones(M, device="cuda")
    d = m.token_logprobs_backward(x, tok, got["logp"], got["peak"], got["log_sum"], None, one, dlogits=x[:, :V])
    ref = torch.zeros(4, device="cuda")
    assert torch.allclose(d[-4:].float().sum(-1), ref, atol=2e-2)  # V / 2 roundings of at most 2^-8 p each: 2^-8


def test_logprobs_refuses_in_the_binding():
    m, g = rq(), gen(33)
    x = randn(3, 64, BF, g)
    tok = torch.zeros(3, dtype=torch.int64, device="cuda")
    v = torch.zeros(3, device="cuda")
    for bad in (lambda: m.token_logprobs(x.half(), tok), lambda: m.token_logprobs(x, tok.int()), lambda: m.token_logprobs(x, tok[:2]),
                lambda: m.token_logprobs(x, tok.cpu()), lambda: m.token_logprobs(x[0], tok), lambda: m.token_logprobs(x.t(), tok),
                lambda: m.token_logprobs_backward(x, tok, v, v.double(), v, v, v), lambda: m.token_logprobs_backward(x, tok, v, v, v, None, v, v),
                lambda: m.token_logprobs_backward(x, tok, v, v, v, v, v, dlogits=x.float()), lambda: m.token_logprobs_backward(x, tok, v, v, v, v, None)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: m.token_logprobs(x, tok, top=33), lambda: m.token_logprobs(x, tok, temperature=0.0),
                lambda: m.token_logprobs(x[:, :4], tok, top=5)):
        with pytest.raises(m.ResqError):
            bad()


# ------------------------------------------------------------------------------------------------ together

def step(m, v, head, head_t, tok, dlogp, dent, dHo):
    """A token's way from a block's output to its log-probability, and the gradient's way back."""
    H, X = m.block_join(v["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], act="sigmoid", alpha=0.5)
    logits = m.w4a16_gemv(X, *head)
    lp = m.token_logprobs(logits, tok, temperature=0.8, top=4)
    dlogits = m.token_logprobs_backward(logits, tok, lp["logp"], lp["peak"], lp["log_sum"], lp["entropy"], dlogp, dent, temperature=0.8)
    dX = m.dgrad_linear(dlogits, *head_t)
    grads = m.block_join_backward(dHo, dX, H, v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], "sigmoid", 0.5)
    return {"H": H, "X": X, "logits": logits, **lp, "dlogits": dlogits, "dX": dX, **grads}


def together(seed):
    m, g = rq(), gen(seed)
    M, K, V = 8, 512, 1024
    v = join_case(M, K, F32, True, "full", seed)
    W = randn(V, K, BF, g, 0.1)
    head, head_t = m.pack_weight(W), m.pack_weight_transposed(W)
    tok = torch.randint(-1, V, (M,), generator=g, device="cuda")
    return v, head, head_t, tok, torch.randn(M, generator=g, device="cuda"), torch.randn(M, generator=g, device="cuda") * 0.01, randn(M, K, F32, g, 0.1)


def test_a_run_of_the_operators_together():
    m = rq()
    v, head, head_t, tok, dlogp, dent, dHo = args = together(41)
    got = step(m, *args)
    w = {n: t.double() for n, t in v.items()}
    h, x = join(w["H"], w["B"], w["gamma_pre"], w["gamma_post"], w["gate"], "sigmoid", 0.5, 1e-6)
    close(got["H"], h, 2.0 ** -16 * (w["H"].abs() + h.abs() + 1))
    x = got["X"].double()                      # each stage against its definition on the stage before
    wd = decode(*head, "hif4")
    close(got["logits"], x @ wd.T, gemv_tol(x, wd, x @ wd.T, BF))
    lp = logprobs(got["logits"].double(), tok, 0.8, 4)
    assert torch.equal(got["top_ids"], lp["top_ids"])
    for n in ("logp", "entropy", "peak", "log_sum", "top_logp"):
        assert torch.allclose(got[n].double(), lp[n], rtol=1e-5, atol=1e-5), n
    d = logprobs_gradient(got["logits"].double(), tok, dlogp.double(), dent.double(), 0.8)
    assert torch.allclose(got["dlogits"].double(), d, rtol=2.0 ** -8 * 1.1, atol=1e-7)
    back = [dHo, got["dX"], got["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"]]
    want, size = (f(*wide(back), "sigmoid", 0.5, 1e-6) for f in (join_gradients, join_gradient_sizes))
    for n in want:
        close(got[n], want[n], 2.0 ** -15 * size[n] + HALF[got[n].dtype] * want[n].abs(), n)


def test_on_a_stream_of_its_own():
    """Inputs made on the current stream, the calls on another one (named, as an object and as a handle), results read back
    after one event; temporaries of the calls belong to that stream."""
    m = rq()
    args = together(42)
    want = step(m, *args)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (s, s.cuda_stream):
        v = args[0]
        for _ in range(3):
            H, X = m.block_join(v["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], act="sigmoid", alpha=0.5, stream=stream)
            logits = m.w4a16_gemv(X, *args[1], stream=stream)
            lp = m.token_logprobs(logits, args[3], temperature=0.8, top=4, stream=stream)
            dl = m.token_logprobs_backward(logits, args[3], lp["logp"], lp["peak"], lp["log_sum"], lp["entropy"], args[4], args[5], temperature=0.8, stream=stream)
            gr = m.block_join_backward(args[6], want["dX"], H, v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], "sigmoid", 0.5, stream=stream)
        torch.cuda.current_stream().wait_stream(s)
        got = {"H": H, "X": X, "logits": logits, **lp, "dlogits": dl, **gr}
        assert all(torch.equal(got[n], want[n]) for n in got)
    with torch.cuda.stream(s):
        got = step(m, *args)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(got[n], want[n]) for n in got)


def test_captured_and_replayed_with_new_inputs():
    """Two graphs of the same calls, each with its own memory, replayed in turn on changed inputs."""
    m = rq()
    sets = [together(43), together(44)]
    want = [{n: t.clone() for n, t in step(m, *a).items()} for a in sets]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for a in sets:
            step(m, *a)
    torch.cuda.current_stream().wait_stream(s)
    graphs, outs = [], []
    for a in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(m, *a))
        graphs.append(graph)
    for _ in range(2):
        for graph, o, w in zip(graphs, outs, want):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o[n], w[n]) for n in w)
    for n, t in sets[0][0].items():
        t.copy_(sets[1][0][n])
    sets[0][3].copy_(sets[1][3])
    changed = step(m, *sets[0])
    graphs[0].replay()
    graphs[1].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(outs[0][n], changed[n]) for n in changed) and all(torch.equal(outs[1][n], want[1][n]) for n in want[1])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [19, 150, 300, 512, 520, 1000, 2050, 8200, 131072])
def test_logprobs_alternatives_that_share_a_lane(V, dtype):
    """Large logits a fixed distance apart, for the distances at which a division of the row among threads gives several of
    them to one thread, in one vector, in neighbouring vectors and far apart; rows with fewer vectors than alternatives."""
    g = gen(V + 9)
    base = randn(1, V, dtype, g).float()[0]
    steps = [s for s in (1, 3, 8, 16, 256, 512, 1024, 2048, 4096, 8192) if s < V]
    x, _ = rows(len(steps) + 1, V, dtype, 8)
    for i, s in enumerate(steps):
        row = base.clone()
        at = torch.arange(i, V, s, device="cuda")[:40]
        row[at] = 6 + torch.randperm(len(at), generator=g, device="cuda").float() / 64
        x[i].copy_(row)
    x[-1].copy_(base)
    tok = torch.randint(0, V, (len(steps) + 1,), generator=g, device="cuda")
    for top in (1, 5, 19, 32):
        if top <= V:
            check_logprobs(x, tok, 1.0, top)


@pytest.mark.parametrize("stream, post, gate, act", [(BF, True, "full", "sigmoid"), (F32, True, "channel", "linear"), (F32, False, "none", "linear")])
@pytest.mark.parametrize("M, K", [(1, 4099), (160, 4104), (33, 5120), (300, 5121), (700, 250), (2000, 500), (3000, 200), (1100, 1000)])
def test_join_backward_at_the_bounds_of_its_splits(M, K, stream, post, gate, act):
    """Row lengths on both sides of the thread counts, and every way to add the partial column sums."""
    test_join_backward_parity(M, K, stream, post, gate, act)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M", [310, 600, 800, 1100, 1300])
def test_logprobs_every_number_of_rows_per_multiprocessor(M, dtype):
    """Numbers of rows at which the threads of a row change, rows long enough to have use for all of them."""
    g = gen(M)
    x = randn(M, 6007, dtype, g, 2.5, pad=8)
    tok = torch.randint(0, 6007, (M,), generator=g, device="cuda")
    for top in (0, 32):
        check_logprobs(x, tok, 1.0, top)


@pytest.mark.parametrize("stream", [BF, F32])
@pytest.mark.parametrize("K", [9, 64, 250, 256, 264])
def test_join_backward_rows_do_not_depend_on_the_rows_before(K, stream):
    """Rows of one or two warps, a dozen of them through the buffers of each block, chunks of which are copied by other lanes than
    those that read them: each row has the bits that it has in a call in which it is a block's only row."""
    m = rq()
    M, part = 30000, 1000
    v = join_case(M, K, stream, True, "full", K)
    g = gen(K + 1)
    dHo, dX = randn(M, K, stream, g, 0.5), randn(M, K, BF, g, 0.5)
    rest = (v["gamma_pre"], v["gamma_post"])
    whole = m.block_join_backward(dHo, dX, v["H"], v["B"], *rest, v["gate"], "sigmoid", 0.5)
    for r in range(0, M, part):
        at = slice(r, r + part)
        alone = m.block_join_backward(dHo[at], dX[at], v["H"][at], v["B"][at], *rest, v["gate"][at], "sigmoid", 0.5)
        for name in ("dH", "dB", "dgate"):
            assert torch.equal(whole[name][at], alone[name]), (name, r)


@pytest.mark.parametrize("M", [1, 5, 400])
@pytest.mark.parametrize("gate", ["channel", "full"])
@pytest.mark.parametrize("stream, post", [(BF, True), (F32, False)])
def test_join_gradient_of_open_and_closed_gates(stream, post, gate, M):
    """Sigmoid gates from -20 to 20: the slope s (1 - s) keeps its digits on both sides.  Formed from e = exp(-g) it is off by
    the argument's rounding, 2 |g| u, and a dozen roundings: 52 u of itself at 20, which the 2^-16 = 256 u of every term covers.
    (In 64 bits 1 - s at 20 is off by 2^-54 / 2^-29, half of u.)"""
    K = 481
    v = join_case(M, K, stream, post, gate, M + 7)
    v["gate"].copy_(torch.linspace(-20, 20, K, device="cuda").expand(v["gate"].shape))
    g = gen(M + 8)
    dHo, dX = randn(M, K, stream, g, 0.5), randn(M, K, BF, g, 0.5)
    back = lambda: rq().block_join_backward(dHo, dX, v["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], "sigmoid", 0.5, 1e-5)
    got = back()
    args = wide([dHo, dX, v["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"]]) + ["sigmoid", 0.5, 1e-5]
    want, size = join_gradients(*args), join_gradient_sizes(*args)
    for name in want:
        chain = U * (M / 148 + 300) if want[name].dim() == 1 else 0.0
        close(got[name], want[name], (2.0 ** -16 + chain) * size[name] + HALF[got[name].dtype] * want[name].abs(), name)
    # gates so far out that the slope is 0 in 32 bits, and infinite ones: no gradient, and none of 0 * inf
    far = torch.tensor([-float("inf"), -3e38, -200.0, 200.0, 3e38, float("inf")], device="cuda", dtype=BF)
    v["gate"][..., :6] = far
    got = back()
    assert all(t.isfinite().all() for t in got.values())
    assert not got["dgate"][..., :6].any()


@pytest.mark.parametrize("top", [33, 10 ** 9, 2 ** 31, 2 ** 32, 2 ** 32 + 5, -1, -2 ** 32])
def test_logprobs_refuses_numbers_of_alternatives_out_of_range(top):
    """Those beyond 32 bits too: no call with what their low bits say, and no memory is asked for."""
    m = rq()
    x, tok = randn(3, 64, BF, gen(34)), torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(m.ResqError) as e:
        m.token_logprobs(x, tok, top=top)
    assert e.value.status == 2


@pytest.mark.parametrize("stream", [BF, F32])
def test_join_rows_of_zeros_without_eps(stream):
    """eps = 0: a row of zeros is 0 / 0, NaN in its own rows and in the column sums, and no other row knows of it."""
    m = rq()
    v = join_case(4, 264, stream, True, "full", 11)
    clean = m.block_join(**v, act="sigmoid", eps=0.0)
    v["H"][1], v["B"][1] = 0, 0
    H, X = m.block_join(**v, act="sigmoid", eps=0.0)
    others = [0, 2, 3]
    assert H[1].isnan().all() and X[1].isnan().all()
    assert torch.equal(H[others], clean[0][others]) and torch.equal(X[others], clean[1][others])
    H[1] = 0
    g = m.block_join_backward(clean[0], X, H, v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], "sigmoid", 1.0, 0.0)
    alone = m.block_join_backward(clean[0][2:], X[2:], H[2:], v["B"][2:], v["gamma_pre"], v["gamma_post"], v["gate"][2:], "sigmoid", 1.0, 0.0)
    for name in ("dH", "dB", "dgate"):
        assert g[name][1].isnan().all() and torch.equal(g[name][2:], alone[name])
    assert g["dgamma_pre"].isnan().all() and g["dgamma_post"].isnan().all()


@pytest.mark.parametrize("scale_h, scale_b", [(1e15, 1e12), (1e12, 1e15), (1e-12, 1e-12), (1e15, 1e-12)])
@pytest.mark.parametrize("stream, post, gate, act", FORMS)
def test_join_rows_of_large_and_small_values(stream, post, gate, act, scale_h, scale_b):
    """Squares from 1e-24 to 1e30 a term, next to rows of ordinary values (eps is small against none of the norms)."""
    M, K, alpha, eps = 6, 264, 0.7, 1e-30
    v = join_case(M, K, stream, post, gate, 12)
    v["H"][::2] *= scale_h
    v["B"][::2] *= scale_b
    H, X = rq().block_join(**v, act=act, alpha=alpha, eps=eps)
    w = {n: None if t is None else t.double() for n, t in v.items()}
    h, x = join(w["H"], w["B"], w["gamma_pre"], w["gamma_post"], w["gate"], act, alpha, eps)
    size = w["H"].abs() + (h - w["H"]).abs()
    close(H, h, 2.0 ** -16 * size + HALF[stream] * h.abs(), "H")
    r = 1 / torch.sqrt(h.square().mean(-1, keepdim=True) + eps)
    close(X, x, 2.0 ** -16 * (size * r * w["gamma_pre"].abs() + x.abs()) + HALF[BF] * x.abs(), "X")
    g = gen(13)
    dHo, dX = randn(M, K, stream, g, 0.5), randn(M, K, BF, g, 0.5)
    dHo[::2] /= scale_h  # of the size of the norm's own gradient
    got = rq().block_join_backward(dHo, dX, H, v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], act, alpha, eps)
    args = wide([dHo, dX, H, v["B"], v["gamma_pre"], v["gamma_post"], v["gate"]]) + [act, alpha, eps]
    want, size = join_gradients(*args), join_gradient_sizes(*args)
    for name in want:
        half = HALF[got[name].dtype] * want[name].abs()
        chain = U * (M / 148 + 300) if want[name].dim() == 1 else 0.0
        close(got[name], want[name], (2.0 ** -16 + chain) * size[name] + half, name)


def test_join_squares_beyond_the_range():
    """A row whose sum of squares is infinite has r = 0, as the header says: X is 0, and the other rows are as they were."""
    m = rq()
    v = join_case(3, 264, F32, False, "none", 14)
    want = m.block_join(**v)
    v["H"][1] = 3e19
    H, X = m.block_join(**v)
    assert (H[1] == 3e19).all() and not X[1].any()
    assert torch.equal(H[::2], want[0][::2]) and torch.equal(X[::2], want[1][::2])
