"""Measured cases of the operators that a rollout or a training step calls beside the 4-bit linear layers.

gemv       Y = X deq(W)^T for a few tokens on HiF4 / MXFP4 packed weights
join       H' = H + alpha g(G) norm(B),  X = norm(H') of the residual stream between two blocks, and its gradients
logprobs   log-probabilities of given tokens with entropy and the top alternatives, and the gradient of the logits

`run` computes the plain form in elementary torch operations, or, where `own` is true, calls the library.
"""
import math

import torch

own = False

_DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one token through an output projection: launch and memory latency
        {"name": "gemv hif4 1 token o", "op": "gemv", "fmt": "hif4", "M": 1, "N": 2048, "K": 2048, "out": "bf16"},
        # one token through gate and up of the larger block: the plain streaming size
        {"name": "gemv hif4 1 token gate_up", "op": "gemv", "fmt": "hif4", "M": 1, "N": 37888, "K": 3584, "out": "bf16"},
        # a small batch through a down projection: long rows, few of them
        {"name": "gemv mxfp4 4 tokens down", "op": "gemv", "fmt": "mxfp4", "M": 4, "N": 2048, "K": 11008, "out": "f32"},
        # a batch through a head with an odd number of rows, logits in 32 bits
        {"name": "gemv hif4 11 tokens head", "op": "gemv", "fmt": "hif4", "M": 11, "N": 100003, "K": 3584, "out": "f32"},
        # one decoded token between two blocks
        {"name": "join 1 token", "op": "join", "M": 1, "K": 2048, "post": False, "gate": "none", "act": "linear", "stream": "bf16"},
        # a prefill with norms on both sides of the block and a gate of its own for each token
        {"name": "join prefill, gated", "op": "join", "M": 16384, "K": 3584, "post": True, "gate": "full", "act": "sigmoid", "stream": "bf16"},
        # a training step: residual stream in 32 bits, one learned gate for each channel
        {"name": "join backward, channel gate", "op": "join_bwd", "M": 8192, "K": 2048, "post": True, "gate": "channel", "act": "linear", "stream": "f32"},
        # a ragged batch, gated token by token, odd width
        {"name": "join backward, odd width", "op": "join_bwd", "M": 1021, "K": 5003, "post": True, "gate": "full", "act": "sigmoid", "stream": "bf16"},
        # one decoded token: its log-probability and the alternatives shown beside it
        {"name": "logprobs 1 token top 20", "op": "logprobs", "M": 1, "V": 131072, "dtype": "bf16", "top": 20, "temp": 0.7},
        # decoded tokens of a batch, logits in 32 bits, odd vocabulary
        {"name": "logprobs 333 tokens top 5", "op": "logprobs", "M": 333, "V": 50001, "dtype": "f32", "top": 5, "temp": 1.0},
        # the policy's pass over finished rollouts
        {"name": "logprobs 4096 tokens", "op": "logprobs", "M": 4096, "V": 131072, "dtype": "bf16", "top": 0, "temp": 1.0},
        # the gradient of a policy loss with an entropy bonus
        {"name": "logprobs backward", "op": "logprobs_bwd", "M": 2048, "V": 131072, "dtype": "bf16", "entropy": True, "temp": 1.0},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["gemv", "gemv", "join", "join_bwd", "logprobs", "logprobs_bwd"])
    if op == "gemv":
        fmt = rng.choice(["hif4", "mxfp4"])
        unit = 64 if fmt == "hif4" else 32
        K = unit * _log_uniform(rng, 2, 18944 // unit)
        N = _log_uniform(rng, 16, min(100003, 300_000_000 // K))
        return {"op": op, "fmt": fmt, "M": _log_uniform(rng, 1, 16), "N": N, "K": K, "out": rng.choice(["bf16", "f32"])}
    if op in ("join", "join_bwd"):
        K = _log_uniform(rng, 64, 18944)
        M = _log_uniform(rng, 1, min(16384, 58_000_000 // K))
        return {"op": op, "M": M, "K": K, "post": rng.random() < 0.5, "gate": rng.choice(["none", "channel", "full"]),
                "act": rng.choice(["linear", "sigmoid"]), "stream": rng.choice(["bf16", "f32"])}
    V = _log_uniform(rng, 100, 200000)
    M = _log_uniform(rng, 1, min(4096, 250_000_000 // V))
    case = {"op": op, "M": M, "V": V, "dtype": rng.choice(["bf16", "f32"]), "temp": rng.choice([0.6, 1.0, 1.3])}
    if op == "logprobs":
        return {**case, "top": rng.choice([0, 1, 5, 20, 32])}
    return {**case, "entropy": rng.random() < 0.5}


def work(case):
    op = case["op"]
    if op == "gemv":
        M, N, K = case["M"], case["N"], case["K"]
        side = K // 64 * 4 if case["fmt"] == "hif4" else K // 32
        return {"bytes": N * (K // 2 + side) + 2 * M * K + M * N * (2 if case["out"] == "bf16" else 4), "flops": 2 * M * N * K}
    if op in ("join", "join_bwd"):
        M, K = case["M"], case["K"]
        s = 2 if case["stream"] == "bf16" else 4
        gate_in = {"none": 0, "channel": 2 * K, "full": 2 * M * K}[case["gate"]]
        weights = 2 * K * (2 if case["post"] else 1)
        if op == "join":
            return {"bytes": M * K * (2 * s + 4) + gate_in + weights, "flops": 12 * M * K}
        gate_out = {"none": 0, "channel": 4 * K, "full": 2 * M * K}[case["gate"]]
        return {"bytes": M * K * (3 * s + 6) + gate_in + gate_out + 3 * weights, "flops": 30 * M * K}
    M, V, b = case["M"], case["V"], 2 if case["dtype"] == "bf16" else 4
    if op == "logprobs":
        return {"bytes": M * V * b + M * (8 + 16 + 8 * case["top"]), "flops": 6 * M * V}
    return {"bytes": 2 * M * V * b + M * 28, "flops": 8 * M * V}


# ------------------------------------------------------------------------------------------------ inputs

def _rows(M, K, dtype):
    """[M, K] whose rows start on 16-byte boundaries."""
    return torch.empty((M, (K + 7) // 8 * 8), dtype=dtype, device=_DEV)[:, :K]


def _normal(g, M, K, dtype, std=1.0):
    out = _rows(M, K, dtype)
    for r in range(0, M, 1024):
        n = min(1024, M - r)
        out[r:r + n] = torch.randn((n, K), generator=g, device=_DEV) * std
    return out


def _with_outliers(x, g, scale=50.0):
    K = x.shape[1]
    ch = torch.randperm(K, generator=g, device=_DEV)[:max(1, K // 200)]
    x[:, ch] = (x[:, ch].float() * scale).to(x.dtype)
    return x


def _pack_hif4(w):
    """Rows of w as HiF4 codes and metadata: the smallest scales that do not clip."""
    N, K = w.shape
    b = w.view(N, K // 64, 64)
    t = b.abs().amax(-1).clamp_min(2.0 ** -47) / 7
    m, e = torch.frexp(t)
    m4 = torch.ceil((2 * m - 1) * 4)
    e = (e - 1 + 48 + (m4 == 4)).to(torch.int64).clamp(0, 63)
    m4 = torch.where(m4 == 4, torch.zeros_like(m4), m4).to(torch.int64)
    s1 = (1 + m4 / 4) * torch.exp2((e - 48).float())
    e2 = b.view(N, K // 64, 8, 8).abs().amax(-1) > 3.5 * s1[..., None]
    top = (1.75 * s1[..., None] * torch.exp2(e2.float())).repeat_interleave(2, -1)
    e3 = b.view(N, K // 64, 16, 4).abs().amax(-1) > top
    step = (s1[..., None] * torch.exp2(e2.float().repeat_interleave(2, -1) + e3.float()) / 4).repeat_interleave(4, -1)
    q = torch.round(b / step).clamp(-7, 7)
    c = (q.abs() + 8 * (q < 0)).to(torch.uint8).view(N, K // 2, 2)
    meta = e * 4 + m4 + (e2.to(torch.int64) << torch.arange(8, 16, device=_DEV)).sum(-1)
    meta = meta + (e3.to(torch.int64) << torch.arange(16, 32, device=_DEV)).sum(-1)
    meta = torch.where(meta >= 2 ** 31, meta - 2 ** 32, meta)
    return c[..., 0] | c[..., 1] << 4, meta.to(torch.int32)


def _pack_mxfp4(w):
    N, K = w.shape
    b = w.view(N, K // 32, 32)
    _, e = torch.frexp(b.abs().amax(-1).clamp_min(2.0 ** -100))
    e = e - 1 - 2
    v = (b / torch.exp2(e.float())[..., None]).abs()
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=_DEV)
    c = (torch.bucketize(v, edges) + 8 * (b < 0)).to(torch.uint8).view(N, K // 2, 2)
    return c[..., 0] | c[..., 1] << 4, (e + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device=_DEV).manual_seed(seed)
    op = case["op"]
    st = {"case": case}
    if op == "gemv":
        M, N, K = case["M"], case["N"], case["K"]
        st["X"] = _with_outliers(_normal(g, M, K, torch.bfloat16), g)
        st["codes"] = torch.empty((N, K // 2), dtype=torch.uint8, device=_DEV)
        hif4 = case["fmt"] == "hif4"
        st["side"] = torch.empty((N, K // 64), dtype=torch.int32, device=_DEV) if hif4 else torch.empty((N, K // 32), dtype=torch.uint8, device=_DEV)
        step = max(1, 40_000_000 // K)
        for r in range(0, N, step):
            n = min(step, N - r)
            w = torch.randn((n, K), generator=g, device=_DEV) * 0.02
            st["codes"][r:r + n], st["side"][r:r + n] = _pack_hif4(w) if hif4 else _pack_mxfp4(w)
        st["out"] = torch.bfloat16 if case["out"] == "bf16" else torch.float32
        return st
    if op in ("join", "join_bwd"):
        M, K = case["M"], case["K"]
        stream = torch.bfloat16 if case["stream"] == "bf16" else torch.float32
        st["H"] = _with_outliers(_normal(g, M, K, stream, 2.0), g, 20.0)
        st["B"] = _normal(g, M, K, torch.bfloat16, 0.5)
        weight = lambda: (1 + 0.1 * torch.randn(K, generator=g, device=_DEV)).to(torch.bfloat16)
        st["gamma_pre"] = weight()
        st["gamma_post"] = weight() if case["post"] else None
        st["gate"] = None
        if case["gate"] == "channel":
            st["gate"] = _normal(g, 1, K, torch.bfloat16)[0]
        elif case["gate"] == "full":
            st["gate"] = _normal(g, M, K, torch.bfloat16)
        st["alpha"], st["eps"] = 0.5, 1e-6
        if op == "join_bwd":
            st["dX"] = _normal(g, M, K, torch.bfloat16, 0.1)
            st["dH"] = _normal(g, M, K, stream, 0.1)
        return st
    M, V = case["M"], case["V"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    x = _normal(g, M, V, dtype, 2.5)
    # the token that was drawn is a likely one; some positions (prompt, padding) have none
    st["tokens"] = torch.randint(0, V, (M,), generator=g, device=_DEV)
    x[torch.arange(M, device=_DEV), st["tokens"]] += 12
    if M >= 8:
        st["tokens"][torch.randperm(M, generator=g, device=_DEV)[:M // 8]] = -1
    st["logits"] = x
    if op == "logprobs_bwd":
        T = case["temp"]
        st["logp"], st["peak"], st["log_sum"], st["entropy"] = (torch.empty(M, device=_DEV) for _ in range(4))
        for r in range(0, M, 256):
            z = x[r:r + 256].double() / T
            peak = z.amax(-1, keepdim=True)
            log_sum = (z - peak).exp().sum(-1, keepdim=True).log()
            z = z - peak - log_sum
            tok = st["tokens"][r:r + 256]
            st["logp"][r:r + 256] = z.gather(1, tok.clamp_min(0)[:, None])[:, 0] * (tok >= 0)
            st["peak"][r:r + 256] = x[r:r + 256].amax(-1).float()
            st["log_sum"][r:r + 256] = log_sum[:, 0]
            st["entropy"][r:r + 256] = -(z.exp() * z).sum(-1)
        st["dlogp"] = torch.randn(M, generator=g, device=_DEV)
        st["dentropy"] = torch.full((M,), -0.01, device=_DEV) if case["entropy"] else None
    return st


# ------------------------------------------------------------------------------------------------ one pass

def run(st):
    op = st["case"]["op"]
    if own:
        import paper_2607_26515_b200 as rq
        if op == "gemv":
            return rq.w4a16_gemv(st["X"], st["codes"], st["side"], st["case"]["fmt"], out_dtype=st["out"])
        if op == "join":
            h, x = rq.block_join(st["H"], st["B"], st["gamma_pre"], st["gamma_post"], st["gate"], act=st["case"]["act"],
                                 alpha=st["alpha"], eps=st["eps"])
            return {"H": h, "X": x}
        if op == "join_bwd":
            return rq.block_join_backward(st["dH"], st["dX"], st["H"], st["B"], st["gamma_pre"], st["gamma_post"], st["gate"],
                                          act=st["case"]["act"], alpha=st["alpha"], eps=st["eps"])
        if op == "logprobs":
            return rq.token_logprobs(st["logits"], st["tokens"], temperature=st["case"]["temp"], top=st["case"]["top"])
        return rq.token_logprobs_backward(st["logits"], st["tokens"], st["logp"], st["peak"], st["log_sum"], st["entropy"],
                                          st["dlogp"], st["dentropy"], temperature=st["case"]["temp"])
    return {"gemv": _gemv, "join": _join, "join_bwd": _join_bwd, "logprobs": _logprobs, "logprobs_bwd": _logprobs_bwd}[op](st)


def _gemv(st):
    c, side = st["codes"], st["side"]
    N, K = c.shape[0], c.shape[1] * 2
    nib = torch.stack((c & 15, c >> 4), -1).view(N, K)
    mag, sign = (nib & 7).int(), 1 - (nib >> 3).float() * 2
    if st["case"]["fmt"] == "hif4":
        bits = lambda lo, n: (side[..., None] >> torch.arange(lo, lo + n, device=_DEV, dtype=torch.int32)) & 1
        s1 = (1 + (side & 3).float() / 4) * torch.exp2(((side >> 2 & 63) - 48).float())
        e = bits(8, 8)[..., None] + bits(16, 16).view(N, K // 64, 8, 2)
        w = (sign * mag / 4).view(N, K // 64, 8, 2, 4) * torch.exp2(e.float())[..., None] * s1[..., None, None, None]
    else:
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=_DEV)
        w = (sign * table[mag]).view(N, K // 32, 32) * torch.exp2(side.float() - 127)[..., None]
    return (st["X"].float() @ w.view(N, K).t()).to(st["out"])


def _norm(x, eps):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)


def _gate(st):
    if st["gate"] is None:
        return None, None
    G = st["gate"].float()
    if st["case"]["act"] == "linear":
        return G, torch.ones_like(G)
    s = 1 / (1 + torch.exp(-G))
    return s, s * (1 - s)


def _join(st):
    p = st["B"].float()
    if st["gamma_post"] is not None:
        p = _norm(p, st["eps"]) * st["gamma_post"].float()
    gate, _ = _gate(st)
    if gate is not None:
        p = p * gate
    h = st["H"].float() + st["alpha"] * p
    return {"H": h.to(st["H"].dtype), "X": (_norm(h, st["eps"]) * st["gamma_pre"].float()).to(torch.bfloat16)}


def _norm_grad(u, x, eps):
    """Gradient of _norm at x for the gradient u of its result."""
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    n = x * r
    return r * (u - n * (u * n).mean(-1, keepdim=True))


def _join_bwd(st):
    h, b, dx = st["H"].float(), st["B"].float(), st["dX"].float()
    out = {"dgamma_pre": (dx * _norm(h, st["eps"])).sum(0)}
    dh = st["dH"].float() + _norm_grad(dx * st["gamma_pre"].float(), h, st["eps"])
    post = st["gamma_post"]
    n = b if post is None else _norm(b, st["eps"])
    p = n if post is None else n * post.float()
    gate, slope = _gate(st)
    dp = st["alpha"] * dh
    if gate is not None:
        dg = dp * p * slope
        out["dgate"] = dg.sum(0) if st["gate"].dim() == 1 else dg.to(torch.bfloat16)
        dp = dp * gate
    if post is not None:
        out["dgamma_post"] = (dp * n).sum(0)
        dp = _norm_grad(dp * post.float(), b, st["eps"])
    out["dH"], out["dB"] = dh.to(st["H"].dtype), dp.to(torch.bfloat16)
    return out


def _logprobs(st):
    x, tok, top, T = st["logits"].float(), st["tokens"], st["case"]["top"], st["case"]["temp"]
    m = x.max(-1, keepdim=True)
    z = (x - m.values) / T
    e = torch.exp(z)
    # the largest term is 1: the others are summed apart, so that a log-probability near 0 keeps its digits
    others = e.scatter(1, m.indices, 0.0).sum(-1, keepdim=True)
    log_s = torch.log1p(others)
    logp = torch.where(tok >= 0, (z.gather(1, tok.clamp_min(0)[:, None]) - log_s)[:, 0], torch.zeros_like(log_s[:, 0]))
    out = {"logp": logp, "entropy": (log_s - (z * e).sum(-1, keepdim=True) / (1 + others))[:, 0], "peak": m.values[:, 0],
           "log_sum": log_s[:, 0]}
    if top:
        # one whole number for each logit that orders by value, then by lower place
        bits = (x + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 2 ** 32 - torch.arange(x.shape[1], device=_DEV)
        ids = torch.topk(order, top, -1).values.neg() % 2 ** 32
        out["top_ids"], out["top_logp"] = ids.int(), z.gather(1, ids) - log_s
    return out


def _logprobs_bwd(st):
    x, tok, T = st["logits"].float(), st["tokens"], st["case"]["temp"]
    z = (x - st["peak"][:, None]) / T - st["log_sum"][:, None]
    p = torch.exp(z)
    there = tok >= 0
    dlogp = torch.where(there, st["dlogp"], torch.zeros_like(st["dlogp"]))
    d = -p * dlogp[:, None]
    hot = -torch.expm1(st["logp"]) * dlogp
    if st["dentropy"] is not None:
        d = d - p * (z + st["entropy"][:, None]) * st["dentropy"][:, None]
        hot = hot - torch.exp(st["logp"]) * (st["logp"] + st["entropy"]) * st["dentropy"]
    at = tok.clamp_min(0)[:, None]
    d.scatter_(1, at, torch.where(there[:, None], hot[:, None], d.gather(1, at)))
    return (d / T).to(st["logits"].dtype)


# ------------------------------------------------------------------------------------------------ 64-bit values

def exact(case, seed):
    """What run returns, from the definitions in 64 bits, a block of rows at a time."""
    st = prepare(case, seed)
    op = case["op"]
    f8 = torch.float64
    if op == "gemv":
        M, N, K = case["M"], case["N"], case["K"]
        x, out = st["X"].to(f8), torch.empty((M, N), dtype=f8, device=_DEV)
        k = torch.arange(K, device=_DEV)
        s1p2 = torch.tensor([(-1) ** (c >> 3) * (c & 7) / 4 for c in range(16)], dtype=f8, device=_DEV)
        e2m1 = torch.tensor([v * s for s in (1, -1) for v in (0, 0.5, 1, 1.5, 2, 3, 4, 6)], dtype=f8, device=_DEV)
        for r in range(0, N, 4096):
            c, side = st["codes"][r:r + 4096].long(), st["side"][r:r + 4096].long()
            code = (c[:, k // 2] >> (k % 2) * 4) & 15
            if case["fmt"] == "hif4":
                m = side[:, k // 64] & 0xFFFFFFFF
                e = ((m >> 2) & 63) - 48 + ((m >> (8 + k % 64 // 8)) & 1) + ((m >> (16 + k % 64 // 4)) & 1)
                w = s1p2[code] * (1 + (m & 3) / 4) * torch.pow(2.0, e.to(f8))
            else:
                w = e2m1[code] * torch.pow(2.0, (side[:, k // 32] - 127).to(f8))
            out[:, r:r + 4096] = x @ w.T
        return out
    if op in ("join", "join_bwd"):
        M, K, alpha, eps = case["M"], case["K"], st["alpha"], st["eps"]
        parts, sums = {}, {}
        one = torch.ones(K, dtype=f8, device=_DEV)
        wpre = st["gamma_pre"].to(f8)
        wpost = one if st["gamma_post"] is None else st["gamma_post"].to(f8)
        for r in range(0, M, 2048):
            at = slice(r, r + 2048)
            h, b = st["H"][at].to(f8), st["B"][at].to(f8)
            G = one if st["gate"] is None else (st["gate"] if st["gate"].dim() == 1 else st["gate"][at]).to(f8)
            act = G if case["act"] == "linear" else torch.sigmoid(G)
            if st["gate"] is None:
                act = one
            slope = torch.ones_like(G) if case["act"] == "linear" else act * (1 - act)
            rb = 1 / torch.sqrt(b.square().mean(1, keepdim=True) + eps) if st["gamma_post"] is not None else torch.ones_like(b[:, :1])
            if op == "join":
                h = h + alpha * act * wpost * b * rb
                x = h * wpre / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
                got = {"H": h, "X": x}
            else:
                dx = st["dX"][at].to(f8)
                rh = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
                u = dx * wpre
                dh = st["dH"][at].to(f8) + rh * u - h * rh ** 3 * (u * h).mean(1, keepdim=True)
                dn = alpha * dh * act * wpost
                db = dn
                if st["gamma_post"] is not None:
                    db = rb * dn - b * rb ** 3 * (dn * b).mean(1, keepdim=True)
                got = {"dH": dh, "dB": db}
                col = {"dgamma_pre": (dx * h * rh).sum(0)}
                if st["gamma_post"] is not None:
                    col["dgamma_post"] = (alpha * dh * act * b * rb).sum(0)
                if st["gate"] is not None:
                    dg = alpha * dh * wpost * b * rb * slope
                    if st["gate"].dim() == 1:
                        col["dgate"] = dg.sum(0)
                    else:
                        got["dgate"] = dg
                for name, v in col.items():
                    sums[name] = sums.get(name, 0) + v
            for name, v in got.items():
                parts.setdefault(name, []).append(v)
        return {**{name: torch.cat(v) for name, v in parts.items()}, **sums}
    M, T = case["M"], case["temp"]
    rows = []
    for r in range(0, M, 256):
        at = slice(r, r + 256)
        x, tok = st["logits"][at].to(f8), st["tokens"][at]
        there = (tok >= 0).to(f8)
        hot = torch.zeros_like(x)
        hot[torch.arange(x.shape[0], device=_DEV), tok.clamp_min(0)] = there
        lse = torch.logsumexp(x / T, 1, keepdim=True)
        logp = x / T - lse
        p = torch.exp(logp)
        H = -(p * logp).sum(1, keepdim=True)
        if op == "logprobs":
            row = {"logp": (hot * logp).sum(1), "entropy": H[:, 0], "peak": x.amax(1), "log_sum": (lse - x.amax(1, keepdim=True) / T)[:, 0]}
            if case["top"]:
                best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
                row["top_ids"], row["top_logp"] = best.int(), logp.gather(1, best)
        else:
            d = st["dlogp"][at].to(f8)[:, None] * (hot - p * there[:, None])
            if st["dentropy"] is not None:
                d = d - st["dentropy"][at].to(f8)[:, None] * p * (logp + H)
            row = {"d": d / T}
        rows.append(row)
    out = {name: torch.cat([row[name] for row in rows]) for name in rows[0]}
    return out["d"] if op == "logprobs_bwd" else out
