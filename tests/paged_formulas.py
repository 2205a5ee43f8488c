"""Rotation into a paged cache, attention over it and the verification of drafts from their definitions, in 64 bits, one sequence at
a time in plain loops, and how large the terms of an attention row are, which is what a rounding error scales with."""
import math

import torch

F64 = torch.float64


def spans(q_start, kv_len, T, max_keys):
    """(first row, new tokens, keys) of every sequence, cut as the header says."""
    out = []
    for b in range(len(kv_len)):
        lo = min(max(q_start[b], 0), T)
        out.append((lo, max(min(q_start[b + 1], T) - lo, 0), min(max(kv_len[b], 0), max_keys)))
    return out


def gather(cache, table_row, n):
    """Keys 0 .. n - 1 of a sequence [n, heads, d]; those of pages outside the cache are zeros."""
    P, page = cache.shape[:2]
    out = torch.zeros((n,) + tuple(cache.shape[2:]), dtype=F64, device=cache.device)
    for i in range((n + page - 1) // page):
        m, id = min(page, n - i * page), int(table_row[i])
        if 0 <= id < P:
            out[i * page:i * page + m] = cache[id, :m].double()
    return out


def rope_append(qkv, bias, k_cache, v_cache, q_start, kv_len, table, inv_freq, pairs, positions=None):
    """(q, k_cache, v_cache) in 64 bits; rows of no sequence are NaN in q."""
    P, page, Hkv, D = k_cache.shape
    T = qkv.shape[0]
    x = qkv.double() + (0 if bias is None else bias.double())
    x = x.view(T, -1, D)
    Hq, rot = x.shape[1] - 2 * Hkv, 2 * len(inv_freq)
    q = torch.full((T, Hq, D), float("nan"), dtype=F64, device=qkv.device)
    kc, vc = k_cache.double(), v_cache.double()
    for b, (lo, n, kv) in enumerate(spans(q_start, kv_len, T, table.shape[1] * page)):
        for i in range(n):
            place = kv - n + i
            pos = place if positions is None else int(positions[lo + i])
            a = pos * inv_freq
            c, s = torch.cos(a), torch.sin(a)
            y = x[lo + i].clone()
            if pairs:
                f, g = x[lo + i, :Hq + Hkv, 0:rot:2], x[lo + i, :Hq + Hkv, 1:rot:2]
                y[:Hq + Hkv, 0:rot:2], y[:Hq + Hkv, 1:rot:2] = f * c - g * s, g * c + f * s
            else:
                f, g = x[lo + i, :Hq + Hkv, :rot // 2], x[lo + i, :Hq + Hkv, rot // 2:rot]
                y[:Hq + Hkv, :rot // 2], y[:Hq + Hkv, rot // 2:rot] = f * c - g * s, g * c + f * s
            q[lo + i] = y[:Hq]
            if place >= 0 and 0 <= int(table[b, place // page]) < P:
                kc[int(table[b, place // page]), place % page] = y[Hq:Hq + Hkv]
                vc[int(table[b, place // page]), place % page] = y[Hq + Hkv:]
    return q.view(T, Hq * D), kc, vc


def attention(q, k_cache, v_cache, q_start, kv_len, table, scale):
    """(out, lse, sum p |v|, largest scale sum |q k| of a row's keys); rows of no sequence are NaN.  Masked keys are left out, so
    what they hold does not matter."""
    P, page, Hkv, D = k_cache.shape
    T, W = q.shape
    Hq = W // D
    out, size = (torch.full((T, Hq, D), float("nan"), dtype=F64, device=q.device) for _ in range(2))
    lse, terms = (torch.full((T, Hq), float("nan"), dtype=F64, device=q.device) for _ in range(2))
    for b, (lo, n, kv) in enumerate(spans(q_start, kv_len, T, table.shape[1] * page)):
        row = table[b].tolist()
        k, v = gather(k_cache, row, kv), gather(v_cache, row, kv)
        finite = bool(torch.isfinite(v).all() and torch.isfinite(k).all())
        g = Hq // Hkv
        # sequences without strange values all tokens at once, the others token by token
        step = max(1, min(n, 40_000_000 // max(1, kv * Hq))) if finite else 1
        for i in range(0, n, step):
            m = min(step, n - i)
            keys = max(0, min(kv - n + i + m, kv))
            at = slice(lo + i, lo + i + m)
            x = q[at].double().view(m, Hkv, g, D)
            s = torch.einsum("mhgd,khd->mhgk", x, k[:keys]) * scale
            seen = torch.arange(keys, device=q.device)[None] <= torch.arange(kv - n + i, kv - n + i + m, device=q.device)[:, None]
            s = torch.where(seen[:, None, None], s, float("-inf"))
            none = ~seen.any(1)
            top = s.amax(-1, keepdim=True) if keys else torch.zeros((m, Hkv, g, 1), dtype=F64, device=q.device)
            top = torch.where(none[:, None, None, None], torch.zeros_like(top), top)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True)
            p = torch.where(none[:, None, None, None], torch.zeros_like(p), p / total)
            out[at] = torch.einsum("mhgk,khd->mhgd", p, v[:keys]).reshape(m, Hq, D)
            size[at] = torch.einsum("mhgk,khd->mhgd", p, v[:keys].abs()).reshape(m, Hq, D)
            lse[at] = (top + total.log())[..., 0].reshape(m, Hq)
            a = torch.einsum("mhgd,khd->mhgk", x.abs(), k[:keys].abs()) * scale
            a = torch.where(seen[:, None, None], a, torch.zeros_like(a))
            terms[at] = a.amax(-1).reshape(m, Hq) if keys else torch.zeros((m, Hq), dtype=F64, device=q.device)
    return out.view(T, W), lse, size.view(T, W), terms


def verify(logits, row_start, drafts, u, noise, draft_logits, draft_peak, draft_log_sum, T):
    """(accepted, tokens, logp) as lists; None in rows of no sequence."""
    R, V = logits.shape
    accepted, tokens, logps = [], [None] * R, [None] * R
    for b in range(len(row_start) - 1):
        lo = min(max(row_start[b], 0), R)
        n = max(min(row_start[b + 1], R) - lo, 0)
        kept, over = 0, False
        for i in range(n):
            r = lo + i
            if over:
                tokens[r], logps[r] = -1, 0.0
                continue
            z, x = logits[r].double(), int(drafts[r])
            usable = not bool(torch.isnan(z).any()) and float(z.max()) < math.inf and float(z.max()) > -math.inf
            lp = torch.log_softmax(z / (T or 1.0), 0)
            p = lp.exp()
            some = i < n - 1 and 0 <= x < V
            if T == 0:
                token = int(torch.nonzero(z == z.max())[0, 0]) if usable else -1
                ok = some and usable and token == x
            else:
                if draft_logits is not None:
                    q = torch.exp((draft_logits[r].double() - draft_peak[r].double()) / T - draft_log_sum[r].double())
                else:
                    q = torch.zeros_like(p)
                    if some:
                        q[x] = 1.0
                ok = some and usable and float(p[x]) > 0 and float(u[r]) * float(q[x]) < float(p[x])
                token = -1
                if not ok and usable:
                    w = torch.relu(p - q) if some else p
                    w = p if float(w.max()) == 0 else w
                    token = int(torch.argmax(w / noise[b].double()))
            if ok:
                kept += 1
                tokens[r], logps[r] = x, float(lp[x])
            else:
                over = True
                tokens[r], logps[r] = token, float(lp[token]) if token >= 0 else 0.0
        accepted.append(kept)
    return accepted, tokens, logps
