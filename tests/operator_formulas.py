"""The operators of the residual stream and of the token log-probabilities from their definitions, in the precision of their
inputs (64 bits in the tests), and how large the terms of each result are, which is what a rounding error scales with."""
import torch


def _act(G, act):
    if G is None:
        return 1.0, 0.0
    if act == "linear":
        return G, torch.ones_like(G)
    s = torch.sigmoid(G)
    return s, s * (1 - s)


def _r(x, eps):
    return 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)


def join(H, B, gamma_pre, gamma_post, gate, act, alpha, eps):
    p = B if gamma_post is None else B * _r(B, eps) * gamma_post
    g, _ = _act(gate, act)
    h = H + alpha * g * p
    return h, None if gamma_pre is None else h * _r(h, eps) * gamma_pre


def _backward(dHo, dX, h, B, gamma_pre, gamma_post, gate, act, alpha, eps, sizes):
    """The gradients, or (`sizes`) the sums of their terms' magnitudes."""
    a = torch.abs if sizes else (lambda t: t)
    minus = 1 if sizes else -1
    r = _r(h, eps)
    xh = a(h * r)
    out = {}
    dh = a(dHo) if dHo is not None else torch.zeros_like(h)
    if dX is not None:
        u = a(dX * gamma_pre)
        dh = dh + r * (u + minus * xh * (u * xh).mean(-1, keepdim=True))
        out["dgamma_pre"] = (a(dX) * xh).sum(0)
    rb = _r(B, eps) if gamma_post is not None else torch.ones_like(r)
    n = a(B * rb)
    w = a(gamma_post) if gamma_post is not None else 1.0
    g, slope = _act(gate, act)
    g = a(g) if gate is not None else 1.0
    dp = (abs(alpha) if sizes else alpha) * dh
    if gate is not None:
        dg = dp * n * w * a(slope)
        out["dgate"] = dg.sum(0) if gate.dim() == 1 else dg
    v = dp * g * w
    if gamma_post is not None:
        out["dgamma_post"] = (dp * g * n).sum(0)
        out["dB"] = rb * (v + minus * n * (v * n).mean(-1, keepdim=True))
    else:
        out["dB"] = v
    out["dH"] = dh
    return out


def join_gradients(*args):
    return _backward(*args, sizes=False)


def join_gradient_sizes(*args):
    return _backward(*args, sizes=True)


def log_softmax(z):
    """Relative to the largest value: next to 2^127, lse and z differ by less than their spacing."""
    z = z - z.amax(-1, keepdim=True)
    return z - z.exp().sum(-1, keepdim=True).log()


def logprobs(x, tok, T, top=0):
    z = x / T
    logp = log_softmax(z)
    p = logp.exp()
    there = (tok >= 0) & (tok < x.shape[1])
    picked = logp.gather(1, torch.where(there, tok, torch.zeros_like(tok))[:, None])[:, 0]
    out = {"logp": torch.where(there, picked, torch.zeros_like(picked)), "peak": x.amax(-1),
           "log_sum": -logp.amax(-1), "entropy": -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(-1)}
    if top:
        ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
        out["top_ids"], out["top_logp"] = ids.int(), logp.gather(1, ids)
    return out


def logprobs_gradient(x, tok, dlogp, dent, T):
    z = x / T
    logp = log_softmax(z)
    p = logp.exp()
    there = (tok >= 0) & (tok < x.shape[1])
    d = -p * (dlogp * there)[:, None]
    d[torch.arange(x.shape[0], device=x.device)[there], tok[there]] += dlogp[there]
    if dent is not None:
        plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
        d = d - dent[:, None] * (plogp - p * plogp.sum(-1, keepdim=True))
    return d / T
