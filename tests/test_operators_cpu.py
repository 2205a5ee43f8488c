"""Host-side refusals of the few-token product, the residual-stream join and the token log-probabilities (no device work),
and the formulas that the GPU tests hold the gradients to, checked against differences."""
import ctypes
import os

import pytest
import torch

from operator_formulas import join, join_gradients, logprobs, logprobs_gradient

OK, NULL, SHAPE, ALIGN, WORKSPACE, PATTERN = 0, 1, 2, 3, 4, 5
P = 0x100000  # an aligned address that no call below gets far enough to use


@pytest.fixture(scope="module")
def lib():
    from paper_2607_26515_b200 import binding, build
    build.build()
    return binding.lib()


def call(fn, args, **changes):
    """fn with `args` (an ordered dict), some of them changed."""
    assert set(changes) <= set(args), changes
    return fn(*{**args, **changes}.values())


GEMV = dict(X=P, M=4, K=256, ldx=256, codes=P, side=P, N=100, Y=P, out=0, ldy=104, stream=None)
GEMV_BAD = [
    (NULL, dict(X=None)), (NULL, dict(codes=None)), (NULL, dict(side=None)), (NULL, dict(Y=None)),
    (SHAPE, dict(M=0)), (SHAPE, dict(M=17)), (SHAPE, dict(M=-1)), (SHAPE, dict(N=0)), (SHAPE, dict(K=0)), (SHAPE, dict(K=16)),
    (SHAPE, dict(N=2 ** 31)), (SHAPE, dict(K=49152 + 64, ldx=49152 + 64)), (PATTERN, dict(out=2)), (PATTERN, dict(out=-1)),
    (ALIGN, dict(X=P + 8)), (ALIGN, dict(ldx=248)), (ALIGN, dict(ldx=260)), (ALIGN, dict(codes=P + 4)), (ALIGN, dict(side=P + 4)),
    (ALIGN, dict(Y=P + 4)), (ALIGN, dict(ldy=96)), (ALIGN, dict(ldy=100)), (ALIGN, dict(out=1, ldy=102)),
]


@pytest.mark.parametrize("name", ["hif4_w4a16_gemv", "mxfp4_w4a16_gemv"])
@pytest.mark.parametrize("status, changes", GEMV_BAD)
def test_gemv_refuses(lib, name, status, changes):
    assert call(getattr(lib, name), GEMV, **changes) == status
    assert lib.resq_last_error()


def test_gemv_block_size_of_the_format(lib):
    assert call(lib.hif4_w4a16_gemv, GEMV, K=96, ldx=96) == SHAPE
    assert b"multiple of 64" in lib.resq_last_error()
    assert call(lib.mxfp4_w4a16_gemv, GEMV, K=80, ldx=80) == SHAPE
    assert b"multiple of 32" in lib.resq_last_error()


JOIN = dict(H=P, dtype=0, B=P, M=4, K=100, ldh=104, ldb=104, gate=P, ldg=104, act=0, gamma_post=P, gamma_pre=P, alpha=1.0, eps=1e-6,
            H_out=P, ldho=104, X=P, ldx=104, stream=None)
JOIN_BAD = [
    (NULL, dict(H=None)), (NULL, dict(B=None)), (NULL, dict(H_out=None)), (NULL, dict(gamma_pre=None)),
    (SHAPE, dict(M=0)), (SHAPE, dict(K=0)), (SHAPE, dict(K=32769, ldh=32776, ldb=32776, ldg=32776, ldho=32776, ldx=32776)),
    (SHAPE, dict(M=2 ** 31)), (SHAPE, dict(eps=-1.0)), (SHAPE, dict(eps=float("nan"))), (SHAPE, dict(eps=float("inf"))),
    (SHAPE, dict(alpha=float("nan"))), (SHAPE, dict(alpha=float("inf"))), (PATTERN, dict(dtype=2)), (PATTERN, dict(act=2)), (PATTERN, dict(act=-1)),
    (ALIGN, dict(H=P + 2)), (ALIGN, dict(B=P + 8)), (ALIGN, dict(gate=P + 2)), (ALIGN, dict(gamma_post=P + 4)), (ALIGN, dict(gamma_pre=P + 4)),
    (ALIGN, dict(H_out=P + 4)), (ALIGN, dict(X=P + 4)), (ALIGN, dict(ldh=96)), (ALIGN, dict(ldb=100)), (ALIGN, dict(ldg=8)),
    (ALIGN, dict(ldho=108)), (ALIGN, dict(ldx=0)), (ALIGN, dict(dtype=1, ldh=102)), (ALIGN, dict(gate=P + 8, ldg=0)),
]


@pytest.mark.parametrize("status, changes", JOIN_BAD)
def test_block_join_refuses(lib, status, changes):
    assert call(lib.resq_block_join, JOIN, **changes) == status


JOIN_BWD = dict(dH_out=P, dX=P, H_out=P, dtype=0, B=P, M=4, K=100, lddho=104, lddx=104, ldho=104, ldb=104, gate=P, ldg=104, act=0,
                gamma_post=P, gamma_pre=P, alpha=1.0, eps=1e-6, dH=P, lddh=104, dB=P, lddb=104, dgate=P, lddg=104, dgamma_post=P,
                dgamma_pre=P, ws=P, ws_bytes=1 << 30, stream=None)
JOIN_BWD_BAD = [
    (NULL, dict(dH_out=None, dX=None)), (NULL, dict(H_out=None)), (NULL, dict(B=None)), (NULL, dict(dH=None)), (NULL, dict(dB=None)),
    (NULL, dict(gamma_pre=None)), (NULL, dict(dgamma_pre=None)), (NULL, dict(dgamma_post=None)), (NULL, dict(dgate=None)),
    (SHAPE, dict(M=0)), (SHAPE, dict(K=-8)), (SHAPE, dict(lddx=2 ** 31)), (SHAPE, dict(lddg=2 ** 32 + 104)), (SHAPE, dict(eps=-1e-9)), (SHAPE, dict(alpha=float("inf"))),
    (PATTERN, dict(dtype=7)), (PATTERN, dict(act=9)),
    (ALIGN, dict(dH_out=P + 2)), (ALIGN, dict(dX=P + 2)), (ALIGN, dict(dH=P + 8)), (ALIGN, dict(dB=P + 8)), (ALIGN, dict(dgate=P + 8)),
    (ALIGN, dict(lddho=96)), (ALIGN, dict(lddx=99)), (ALIGN, dict(lddh=100)), (ALIGN, dict(lddb=0)), (ALIGN, dict(lddg=0)),
    (ALIGN, dict(dgamma_pre=P + 2)), (ALIGN, dict(dgamma_post=P + 1)), (ALIGN, dict(ldg=0, dgate=P + 2)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws=P + 128)), (WORKSPACE, dict(ws_bytes=100)),
]


@pytest.mark.parametrize("status, changes", JOIN_BWD_BAD)
def test_block_join_backward_refuses(lib, status, changes):
    assert call(lib.resq_block_join_backward, JOIN_BWD, **changes) == status


def test_block_join_backward_workspace(lib):
    q = lib.resq_block_join_backward_workspace_bytes
    assert q(0, 64) == q(4, 0) == q(4, 32769) == 0
    assert q(1, 1) >= 3 * 8 * 4 and q(1, 1) % 256 == 0
    assert q(4, 100) >= 4 * 3 * 100 * 4
    assert q(10 ** 6, 2048) == q(10 ** 9, 2048)  # the partial sums stop growing once the device is full
    need = q(4, 100)
    assert call(lib.resq_block_join_backward, JOIN_BWD, ws_bytes=need - 1) == WORKSPACE


LP = dict(x=P, dtype=0, M=4, V=100, ld=104, tokens=P, T=1.0, top=5, logp=P, entropy=P, peak=P, log_sum=P, ids=P, tlogp=P, stream=None)
LP_BAD = [
    (NULL, dict(x=None)), (NULL, dict(tokens=None)), (NULL, dict(ids=None)), (NULL, dict(tlogp=None)),
    (NULL, dict(logp=None, entropy=None, peak=None, log_sum=None, top=0)),
    (SHAPE, dict(M=0)), (SHAPE, dict(V=0)), (SHAPE, dict(V=(1 << 28) + 1, ld=(1 << 28) + 8)), (SHAPE, dict(M=2 ** 31)), (SHAPE, dict(top=33)),
    (SHAPE, dict(top=-1)), (SHAPE, dict(V=4, top=5)), (SHAPE, dict(T=0.0)), (SHAPE, dict(T=-1.0)), (SHAPE, dict(T=float("nan"))),
    (SHAPE, dict(T=1e7)), (PATTERN, dict(dtype=2)), (ALIGN, dict(x=P + 2)), (ALIGN, dict(ld=96)), (ALIGN, dict(ld=100)),
    (ALIGN, dict(dtype=1, ld=101)), (ALIGN, dict(tokens=P + 4)), (ALIGN, dict(logp=P + 2)), (ALIGN, dict(ids=P + 1)),
]


@pytest.mark.parametrize("status, changes", LP_BAD)
def test_token_logprobs_refuses(lib, status, changes):
    assert call(lib.resq_token_logprobs, LP, **changes) == status


LP_BWD = dict(x=P, dtype=0, M=4, V=100, ld=104, tokens=P, T=1.0, logp=P, peak=P, log_sum=P, entropy=P, dlogp=P, dentropy=P, dx=P, ldd=104, stream=None)
LP_BWD_BAD = [
    (NULL, dict(x=None)), (NULL, dict(tokens=None)), (NULL, dict(logp=None)), (NULL, dict(peak=None)), (NULL, dict(log_sum=None)), (NULL, dict(dlogp=None)),
    (NULL, dict(dx=None)), (NULL, dict(entropy=None)), (SHAPE, dict(M=-1)), (SHAPE, dict(V=0)), (SHAPE, dict(T=0.0)),
    (PATTERN, dict(dtype=5)), (ALIGN, dict(dx=P + 4)), (ALIGN, dict(ldd=96)), (ALIGN, dict(ldd=100)), (ALIGN, dict(peak=P + 2)), (ALIGN, dict(log_sum=P + 2)),
]


@pytest.mark.parametrize("status, changes", LP_BWD_BAD)
def test_token_logprobs_backward_refuses(lib, status, changes):
    assert call(lib.resq_token_logprobs_backward, LP_BWD, **changes) == status


def test_binding_refuses_what_the_library_cannot_see():
    """Types, devices and strides are the binding's to check: CPU tensors never reach the library."""
    import paper_2607_26515_b200 as rq
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        rq.w4a16_gemv(x, torch.zeros((8, 32), dtype=torch.uint8), torch.zeros((8, 1), dtype=torch.int32))
    with pytest.raises(ValueError):
        rq.block_join(x, x)
    with pytest.raises(ValueError):
        rq.block_join_backward(x, None, x, x)
    with pytest.raises(ValueError):
        rq.token_logprobs(x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        rq.token_logprobs_backward(x, torch.zeros(2, dtype=torch.int64), *[torch.zeros(2)] * 5)


# ---------------------------------------------------------------- the formulas against differences

def directional(f, inputs, i, v, step=1e-5):
    """Derivative of f along v in its i-th input, by central differences in 64 bits."""
    at = lambda s: f(*[x + s * v if j == i else x for j, x in enumerate(inputs)])
    return (at(step) - at(-step)) / (2 * step)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate, act", [("none", "linear"), ("channel", "linear"), ("channel", "sigmoid"), ("full", "linear"), ("full", "sigmoid")])
def test_join_gradients_against_differences(post, gate, act):
    g = torch.Generator().manual_seed(7)
    rand = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    M, K, alpha, eps = 3, 11, 0.7, 1e-3
    H, B, wpre = rand(M, K), rand(M, K), rand(K)
    wpost = rand(K) if post else None
    G = {"none": None, "channel": rand(K), "full": rand(M, K)}[gate]
    dHo, dX = rand(M, K), rand(M, K)
    names = ["H", "B", "gamma_pre"] + ["gamma_post"] * post + ["gate"] * (G is not None)
    full = {"H": H, "B": B, "gamma_pre": wpre, "gamma_post": wpost, "gate": G}

    def loss(*values):
        v = {**full, **dict(zip(names, values))}
        h, x = join(v["H"], v["B"], v["gamma_pre"], v["gamma_post"], v["gate"], act, alpha, eps)
        return (h * dHo).sum() + (x * dX).sum()

    h, _ = join(H, B, wpre, wpost, G, act, alpha, eps)
    got = join_gradients(dHo, dX, h, B, wpre, wpost, G, act, alpha, eps)
    for i, name in enumerate(names):
        v = torch.randn(full[name].shape, generator=g, dtype=torch.float64)
        want = directional(loss, [full[n] for n in names], i, v)
        assert torch.allclose((got["d" + name] * v).sum(), want, rtol=1e-7, atol=1e-8), name


def test_logprobs_gradient_against_differences():
    g = torch.Generator().manual_seed(8)
    x = 2 * torch.randn((4, 9), generator=g, dtype=torch.float64)
    tok = torch.tensor([0, 8, -1, 4])
    dlogp, dent = torch.randn(4, generator=g, dtype=torch.float64), torch.randn(4, generator=g, dtype=torch.float64)
    for T in (0.5, 1.0, 2.5):
        def loss(y):
            r = logprobs(y, tok, T)
            return (r["logp"] * dlogp).sum() + (r["entropy"] * dent).sum()
        got = logprobs_gradient(x, tok, dlogp, dent, T)
        for _ in range(3):
            v = torch.randn(x.shape, generator=g, dtype=torch.float64)
            assert torch.allclose((got * v).sum(), directional(loss, [x], 0, v), rtol=1e-7, atol=1e-8)
