"""Measured cases of the operators that a rollout step calls between the qkv and the output projection and behind the head.

append   rotation of queries and keys, keys and values into their slots of a paged cache
attn     attention of the new tokens of several sequences over a paged cache
verify   drafted tokens accepted or replaced by the target's probabilities, from given random numbers

`run` computes the plain form in elementary torch operations, or, where `own` is true, calls the library.
"""
import math
import random

import torch

own = False

_DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases
#
# Lengths of a case: every sequence has new_lo .. new_hi new tokens behind past_lo .. past_hi earlier ones, drawn from `lens`.

def listed():
    return [
        # one decoded token of the smaller model: launch and memory latency
        _append("append 1 token", 1, 1, 1, 1500, 1500, 16, 2, 128, 128, 16, bias=True),
        # a prefill of eight prompts through the larger model
        _append("append prefill", 8, 2048, 2048, 0, 0, 28, 4, 128, 128, 64, bias=True),
        # ragged chunks far into their sequences, small heads, half of each rotated in neighbouring pairs, 32-bit projections
        _append("append ragged, pairs, fp32", 37, 1, 90, 20000, 500000, 14, 2, 64, 32, 16, pairs=True, dtype="f32"),
        # one sequence being decoded: latency, the cache of one sequence over the whole device
        _attn("attn decode 1 sequence", 1, 1, 1, 4000, 4000, 16, 2, 128, 16),
        # a rollout batch being decoded: reading the cache
        _attn("attn decode batch", 64, 1, 1, 2000, 12000, 28, 4, 128, 16),
        # drafted tokens of a batch, a cache with a page's heads apart
        _attn("attn drafts", 24, 2, 6, 500, 9000, 16, 2, 128, 32, layout="head"),
        # one long prompt from the beginning
        _attn("attn prefill", 1, 8192, 8192, 0, 0, 28, 4, 128, 64),
        # a chunk of each of two prompts behind long beginnings
        _attn("attn chunk over long context", 2, 500, 520, 30000, 33000, 16, 2, 128, 128),
        # a mixed batch: decoded tokens and short chunks, small heads, pages that do not divide a tile
        _attn("attn mixed, small heads", 40, 1, 300, 0, 3000, 14, 2, 64, 24),
        # one sequence with four drafts
        _verify("verify 1 sequence", 1, 5, 5, 131072, "bf16", "logits"),
        # a rollout batch with four drafts each
        _verify("verify batch", 64, 5, 5, 131072, "bf16", "logits"),
        # drafts without probabilities (from the text itself), ragged, odd vocabulary, 32-bit logits
        _verify("verify looked-up drafts, odd vocabulary", 41, 1, 8, 50001, "f32", "sure"),
    ]


def _append(name, B, new_lo, new_hi, past_lo, past_hi, Hq, Hkv, D, rot, page, bias=False, pairs=False, dtype="bf16", lens=1):
    return {"name": name, "op": "append", "B": B, "new_lo": new_lo, "new_hi": new_hi, "past_lo": past_lo, "past_hi": past_hi, "Hq": Hq,
            "Hkv": Hkv, "D": D, "rot": rot, "page": page, "bias": bias, "pairs": pairs, "dtype": dtype, "lens": lens}


def _attn(name, B, new_lo, new_hi, past_lo, past_hi, Hq, Hkv, D, page, layout="token", lens=1):
    return {"name": name, "op": "attn", "B": B, "new_lo": new_lo, "new_hi": new_hi, "past_lo": past_lo, "past_hi": past_hi, "Hq": Hq,
            "Hkv": Hkv, "D": D, "page": page, "layout": layout, "lens": lens}


def _verify(name, B, rows_lo, rows_hi, V, dtype, drafts, temp=1.0, lens=1):
    return {"name": name, "op": "verify", "B": B, "rows_lo": rows_lo, "rows_hi": rows_hi, "V": V, "dtype": dtype, "drafts": drafts,
            "temp": temp, "lens": lens}


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


_HEADS = [(16, 2, 128), (28, 4, 128), (14, 2, 64), (8, 8, 128), (12, 4, 64), (32, 1, 128)]
_PAGES = [8, 16, 24, 32, 64, 128, 256]


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "attn", "verify", "verify"])
    lens = rng.randrange(1 << 30)
    if op == "verify":
        V = _log_uniform(rng, 200, 160000)
        dtype = rng.choice(["bf16", "f32"])
        hi = rng.randint(1, 9)
        B = _log_uniform(rng, 1, max(1, min(256, 40_000_000 // (V * hi) // (1 if dtype == "bf16" else 2))))
        return {k: v for k, v in _verify("", B, rng.randint(1, hi), hi, V, dtype, rng.choice(["logits", "sure", "greedy"]),
                                         rng.choice([0.7, 1.0, 1.3]), lens).items() if k != "name"}
    Hq, Hkv, D = rng.choice(_HEADS)
    page = rng.choice(_PAGES)
    if op == "append":
        T = _log_uniform(rng, 1, 14000)
        B = _log_uniform(rng, 1, min(T, 200))
        hi = max(1, T // B)
        past = rng.choice([0, _log_uniform(rng, 1, 30000), _log_uniform(rng, 30000, 900000)])
        return {k: v for k, v in _append("", B, max(1, hi // 3), hi, past // 2, past, Hq, Hkv, D, rng.choice([D, D, D // 2]), page,
                                         rng.random() < 0.5, rng.random() < 0.3, rng.choice(["bf16", "f32"]), lens).items() if k != "name"}
    while True:
        kind = rng.choice(["decode", "decode", "drafts", "chunk", "mixed"])
        hi = {"decode": 1, "drafts": rng.randint(2, 8)}.get(kind) or _log_uniform(rng, 9, 4096)
        lo = 1 if kind == "mixed" else max(1, hi // 2)
        past = rng.choice([0, _log_uniform(rng, 1, 40000), _log_uniform(rng, 100, 10000)])
        case = _attn("", _log_uniform(rng, 1, 128), lo, hi, past // 4, past, Hq, Hkv, D, page, rng.choice(["token", "head"]), lens)
        w = work(case)
        if w["flops"] <= 4.0e11 and w["bytes"] <= 1.0e9:
            return {k: v for k, v in case.items() if k != "name"}


def _lengths(case):
    """(new, past) tokens of every sequence."""
    rng = random.Random(case["lens"])
    return [(rng.randint(case["new_lo"], case["new_hi"]), rng.randint(case["past_lo"], case["past_hi"])) for _ in range(case["B"])]


def _row_counts(case):
    rng = random.Random(case["lens"])
    return [rng.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["B"])]


def work(case):
    if case["op"] == "verify":
        R, B, V, b = sum(_row_counts(case)), case["B"], case["V"], 2 if case["dtype"] == "bf16" else 4
        drawn = {"logits": B * V * (b + 4), "sure": B * V * 4, "greedy": 0}[case["drafts"]]
        return {"bytes": R * V * b + drawn + R * 36, "flops": 6 * R * V + 8 * B * V}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    lens = _lengths(case)
    T = sum(n for n, _ in lens)
    if case["op"] == "append":
        b = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": T * (Hq + 2 * Hkv) * D * (b + 2) + case["rot"] * 4, "flops": 3 * T * (Hq + Hkv) * case["rot"]}
    keys = sum(n + p for n, p in lens)
    pairs = sum(n * p + n * (n + 1) // 2 for n, p in lens)
    return {"bytes": 4 * T * Hq * D + 4 * keys * Hkv * D, "flops": 4 * D * Hq * pairs}


# ------------------------------------------------------------------------------------------------ inputs

def _rows(M, K, dtype):
    """[M, K] whose rows start on 16-byte boundaries."""
    return torch.empty((M, (K + 7) // 8 * 8), dtype=dtype, device=_DEV)[:, :K]


def _normal(g, M, K, dtype, std=1.0):
    out = _rows(M, K, dtype)
    step = max(1, 40_000_000 // K)
    for r in range(0, M, step):
        n = min(step, M - r)
        out[r:r + n] = torch.randn((n, K), generator=g, device=_DEV) * std
    return out


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=_DEV)


def _paged(case, g, lens):
    """Lengths, page table and an empty cache whose pages are dealt out in any order; a few stay free."""
    page, Hkv, D = case["page"], case["Hkv"], case["D"]
    used = [(n + p + page - 1) // page for n, p in lens]
    # far into a sequence an append test keeps only the pages that it writes
    first = [p // page if case["op"] == "append" else 0 for _, p in lens]
    P = sum(u - f for u, f in zip(used, first)) + 3
    order = torch.randperm(P, generator=g, device=_DEV).to(torch.int32)
    table = torch.full((len(lens), max(used)), -1, dtype=torch.int32, device=_DEV)
    at = 0
    for b, (u, f) in enumerate(zip(used, first)):
        table[b, f:u] = order[at:at + u - f]
        at += u - f
    starts = [0]
    for n, _ in lens:
        starts.append(starts[-1] + n)
    st = {"q_start": _ints(starts), "kv_len": _ints([n + p for n, p in lens]), "page_table": table, "lens": lens}
    if case.get("layout") == "head":  # a page's heads apart, keys and values in one buffer
        both = _normal(g, P * 2 * Hkv * page, D, torch.bfloat16).view(P, 2, Hkv, page, D).transpose(2, 3)
        st["k_cache"], st["v_cache"] = both[:, 0], both[:, 1]
    else:
        st["k_cache"] = _normal(g, P * page * Hkv, D, torch.bfloat16).view(P, page, Hkv, D)
        st["v_cache"] = _normal(g, P * page * Hkv, D, torch.bfloat16).view(P, page, Hkv, D)
    return st


def prepare(case, seed):
    g = torch.Generator(device=_DEV).manual_seed(seed)
    if case["op"] == "verify":
        return {"case": case, **_verify_inputs(case, g)}
    lens = _lengths(case)
    T = sum(n for n, _ in lens)
    st = {"case": case, **_paged(case, g, lens)}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["op"] == "append":
        st["qkv"] = _normal(g, T, (Hq + 2 * Hkv) * D, torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        st["bias"] = _normal(g, 1, (Hq + 2 * Hkv) * D, torch.bfloat16)[0] if case["bias"] else None
        j = torch.arange(case["rot"] // 2, dtype=torch.float64, device=_DEV)
        st["inv_freq"] = 1e6 ** (-2 * j / case["rot"])
        return st
    # scores of a few units: some keys take most of a row's weight
    st["q"] = _normal(g, T, Hq * D, torch.bfloat16, 2.0)
    st["scale"] = D ** -0.5
    st["max_new"] = max(n for n, _ in lens)
    if own:
        import paper_2607_26515_b200 as rq
        nbytes = rq.paged_attention_workspace_bytes(T, case["B"], Hq, Hkv, D, st["max_new"])
        st["workspace"] = rq.alloc_workspace(nbytes)
    return st


def _verify_inputs(case, g):
    counts = _row_counts(case)
    B, R, V, T = case["B"], sum(counts), case["V"], case["temp"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    st = {"row_start": _ints(starts), "counts": counts}
    x = _normal(g, R, V, dtype, 2.5)
    at = torch.arange(R, device=_DEV)
    drafts = torch.randint(0, V, (R,), generator=g, device=_DEV)
    # the drafted token is a likely one, for the target in most rows
    likely = 3 + 9 * torch.rand((R,), generator=g, device=_DEV) if case["drafts"] != "greedy" else 16 * torch.rand((R,), generator=g, device=_DEV)
    x[at, drafts] = (x[at, drafts].float() + likely).to(dtype)
    st["logits"], st["drafts"] = x, drafts
    if case["drafts"] == "greedy":
        return st
    st["u"] = torch.rand((R,), generator=g, device=_DEV)
    e = _rows(B, V, torch.float32)
    for b in range(B):
        e[b] = torch.empty(V, device=_DEV).exponential_(generator=g).clamp_min_(1e-30)
    st["noise"] = e
    if case["drafts"] == "logits":
        d = _rows(R, V, dtype)
        st["draft_peak"], st["draft_log_sum"] = torch.empty(R, device=_DEV), torch.empty(R, device=_DEV)
        for r in range(0, R, 64):
            n = min(64, R - r)
            d[r:r + n] = x[r:r + n].float() + torch.randn((n, V), generator=g, device=_DEV) * 0.5
            z = d[r:r + n].double()
            st["draft_peak"][r:r + n] = z.amax(-1)
            st["draft_log_sum"][r:r + n] = ((z - z.amax(-1, keepdim=True)) / T).exp().sum(-1).log()
        st["draft_logits"] = d
    return st


# ------------------------------------------------------------------------------------------------ one pass

def run(st):
    case = st["case"]
    if own:
        import paper_2607_26515_b200 as rq
        if case["op"] == "append":
            q = rq.rope_append(st["qkv"], st["k_cache"], st["v_cache"], st["q_start"], st["kv_len"], st["page_table"], st["inv_freq"],
                               bias=st["bias"], pairs=case["pairs"])
            return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
        if case["op"] == "attn":
            out, lse = rq.paged_attention(st["q"], st["k_cache"], st["v_cache"], st["q_start"], st["kv_len"], st["page_table"],
                                          scale=st["scale"], max_new=st["max_new"], lse=True, workspace=st["workspace"])
            return {"out": out, "lse": lse}
        if case["drafts"] == "greedy":
            return rq.verify_drafts(st["logits"], st["row_start"], st["drafts"], temperature=0.0)
        return rq.verify_drafts(st["logits"], st["row_start"], st["drafts"], st["u"], st["noise"], st.get("draft_logits"),
                                st.get("draft_peak"), st.get("draft_log_sum"), temperature=case["temp"])
    return {"append": _append_plain, "attn": _attn_plain, "verify": _verify_plain}[case["op"]](st)


def _append_plain(st):
    case = st["case"]
    Hq, Hkv, D, rot, page = (case[k] for k in ("Hq", "Hkv", "D", "rot", "page"))
    start, kv_len = st["q_start"].long(), st["kv_len"].long()
    x = st["qkv"].float()
    if st["bias"] is not None:
        x = x + st["bias"].float()
    T = x.shape[0]
    tok = torch.arange(T, device=_DEV)
    seq = torch.searchsorted(start, tok, right=True) - 1
    pos = tok - start[seq + 1] + kv_len[seq]
    angle = pos.double()[:, None] * st["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.view(T, Hq + 2 * Hkv, D)
    turn = x[:, :Hq + Hkv, :rot]
    if case["pairs"]:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = turn[..., :rot // 2], turn[..., rot // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    qk = torch.cat((turned, x[:, :Hq + Hkv, rot:]), -1).to(torch.bfloat16)
    where = st["page_table"].long()[seq, pos // page], pos % page
    st["k_cache"][where] = qk[:, Hq:]
    st["v_cache"][where] = x[:, Hq + Hkv:].to(torch.bfloat16)
    return {"q": qk[:, :Hq].reshape(T, Hq * D), "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def _attn_plain(st):
    case = st["case"]
    Hq, Hkv, D, page = (case[k] for k in ("Hq", "Hkv", "D", "page"))
    G = Hq // Hkv
    out, lse = torch.empty_like(st["q"]), torch.empty((st["q"].shape[0], Hq), device=_DEV)
    at = 0
    for b, (n, past) in enumerate(st["lens"]):
        L = n + past
        ids = st["page_table"][b, :(L + page - 1) // page].long()
        k = st["k_cache"][ids].flatten(0, 1)[:L].float().permute(1, 2, 0)
        v = st["v_cache"][ids].flatten(0, 1)[:L].float().transpose(0, 1)
        step = max(1, 200_000_000 // (Hq * L))
        for i in range(0, n, step):
            m = min(step, n - i)
            rows = slice(at + i, at + i + m)
            q = st["q"][rows].float().view(m, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, m * G, D)
            s = (q @ k * st["scale"]).view(Hkv, m, G, L)
            if i + past + m > 1:
                mask = torch.arange(L, device=_DEV)[None, :] > torch.arange(past + i, past + i + m, device=_DEV)[:, None]
                s.masked_fill_(mask[None, :, None, :], float("-inf"))
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True)
            o = (p.view(Hkv, m * G, L) @ v).view(Hkv, m, G, D) / total
            out[rows] = o.permute(1, 0, 2, 3).reshape(m, Hq * D).to(torch.bfloat16)
            lse[rows] = (top + torch.log(total))[..., 0].permute(1, 0, 2).reshape(m, Hq)
        at += n
    return {"out": out, "lse": lse}


def _verify_plain(st):
    """Decisions in 64 bits: a token is kept or drawn next to a border of real numbers."""
    case = st["case"]
    x, drafts, V, B = st["logits"], st["drafts"], case["V"], case["B"]
    start = st["row_start"].long()
    R = x.shape[0]
    row = torch.arange(R, device=_DEV)
    seq = torch.searchsorted(start, row, right=True) - 1
    last = row == start[seq + 1] - 1
    T = case["temp"] if case["drafts"] != "greedy" else 1.0
    best, peak, log_sum = (torch.empty(R, dtype=t, device=_DEV) for t in (torch.int64, torch.float64, torch.float64))
    for r in range(0, R, 64):
        z = x[r:r + 64].double()
        peak[r:r + 64] = z.amax(-1)
        best[r:r + 64] = (z == z.amax(-1, keepdim=True)).to(torch.uint8).argmax(-1)
        z = (z - z.amax(-1, keepdim=True)) / T
        log_sum[r:r + 64] = z.exp().sum(-1).log()
    logp = (x[row, drafts].double() - peak) / T - log_sum
    if case["drafts"] == "greedy":
        keep = drafts == best
    else:
        logq = torch.zeros_like(logp)
        if case["drafts"] == "logits":
            logq = (st["draft_logits"][row, drafts].double() - st["draft_peak"].double()) / T - st["draft_log_sum"].double()
        keep = st["u"].double() < torch.exp(logp - logq)
    keep &= ~last
    # rows kept from each sequence's first on
    fails = torch.cumsum((~keep).long(), 0)
    before = torch.where(start[seq] > 0, fails[start[seq] - 1], torch.zeros_like(fails))
    kept = fails == before
    accepted = torch.zeros(B, dtype=torch.int64, device=_DEV).index_add_(0, seq, kept.long())
    at = start[:-1] + accepted
    if case["drafts"] == "greedy":
        drawn = best[at]
    else:
        drawn = torch.empty(B, dtype=torch.int64, device=_DEV)
        for b in range(0, B, 32):
            r = at[b:b + 32]
            p = torch.exp((x[r].double() - peak[r, None]) / T - log_sum[r, None])
            w = p.clone()
            if case["drafts"] == "logits":
                q = torch.exp((st["draft_logits"][r].double() - st["draft_peak"][r, None].double()) / T - st["draft_log_sum"][r, None].double())
                w = torch.where(last[r, None], w, (w - q).clamp_min(0))
            else:
                w[torch.arange(len(r), device=_DEV), drafts[r]] *= last[r]
            none = (w.amax(-1, keepdim=True) == 0)
            drawn[b:b + 32] = (torch.where(none, p, w) / st["noise"][b:b + 32].double()).argmax(-1)
    tokens = torch.where(kept, drafts, torch.full_like(drafts, -1))
    tokens[at] = drawn
    values = torch.where(kept, logp, torch.zeros_like(logp))
    values[at] = (x[at, drawn].double() - peak[at]) / T - log_sum[at]
    return {"accepted": accepted.int(), "tokens": tokens, "logp": values.float()}


# ------------------------------------------------------------------------------------------------ 64-bit values

def exact(case, seed):
    """What run returns, from the definitions in 64 bits, one sequence at a time."""
    st = prepare(case, seed)
    f8 = torch.float64
    if case["op"] == "append":
        Hq, Hkv, D, rot, page = (case[k] for k in ("Hq", "Hkv", "D", "rot", "page"))
        W = (Hq + 2 * Hkv) * D
        kc, vc = st["k_cache"].to(f8), st["v_cache"].to(f8)
        qs, at = [], 0
        # the element that each one is turned with, and the sign of its part
        d = torch.arange(D, device=_DEV)
        if case["pairs"]:
            mate, freq, sign = d ^ 1, d // 2, torch.where(d % 2 == 0, -1.0, 1.0)
        else:
            mate, freq, sign = (d + rot // 2) % rot, d % max(1, rot // 2), torch.where(d < rot // 2, -1.0, 1.0)
        mate, freq = torch.where(d < rot, mate, d), torch.where(d < rot, freq, torch.zeros_like(d))
        for b, (n, past) in enumerate(st["lens"]):
            x = st["qkv"][at:at + n].to(f8) + (st["bias"].to(f8) if st["bias"] is not None else torch.zeros(W, dtype=f8, device=_DEV))
            x = x.reshape(n, Hq + 2 * Hkv, D)
            pos = torch.arange(past, past + n, device=_DEV)
            a = torch.outer(pos.to(f8), st["inv_freq"])[:, freq]
            c, s = torch.where(d < rot, a.cos(), 1.0), torch.where(d < rot, a.sin() * sign.to(f8), 0.0)
            y = x * c[:, None] + x[:, :, mate] * s[:, None]
            qs.append(y[:, :Hq].reshape(n, Hq * D))
            slot = st["page_table"][b].long()[pos // page] * page + pos % page
            for cache, new in ((kc, y[:, Hq:Hq + Hkv]), (vc, x[:, Hq + Hkv:])):
                cache[slot // page, slot % page] = new
            at += n
        return {"q": torch.cat(qs), "k_cache": kc, "v_cache": vc}
    if case["op"] == "attn":
        Hq, Hkv, D, page = (case[k] for k in ("Hq", "Hkv", "D", "page"))
        G, outs, lses, at = Hq // Hkv, [], [], 0
        for b, (n, past) in enumerate(st["lens"]):
            L = n + past
            j = torch.arange(L, device=_DEV)
            slot = st["page_table"][b].long()[j // page], j % page
            k, v = st["k_cache"][slot].to(f8), st["v_cache"][slot].to(f8)
            out, lse = torch.empty((n, Hq, D), dtype=f8, device=_DEV), torch.empty((n, Hq), dtype=f8, device=_DEV)
            step = max(1, 60_000_000 // L)
            for h in range(Hq):
                for i in range(0, n, step):
                    q = st["q"][at + i:at + min(i + step, n), h * D:(h + 1) * D].to(f8)
                    s = torch.einsum("id,jd->ij", q, k[:, h // G]) * st["scale"]
                    seen = j[None] <= torch.arange(past + i, past + i + q.shape[0], device=_DEV)[:, None]
                    s = torch.where(seen, s, float("-inf"))
                    lse[i:i + step, h] = torch.logsumexp(s, 1)
                    out[i:i + step, h] = torch.softmax(s, 1) @ v[:, h // G]
            outs.append(out.reshape(n, Hq * D))
            lses.append(lse)
            at += n
        return {"out": torch.cat(outs), "lse": torch.cat(lses)}
    V, B, temp = case["V"], case["B"], case["temp"]
    R = sum(st["counts"])
    accepted = torch.zeros(B, dtype=torch.int32)
    tokens, logps = torch.full((R,), -1, dtype=torch.int64), torch.zeros(R, dtype=f8)
    drafts = st["drafts"].tolist()
    us = st["u"].tolist() if "u" in st else None
    first = 0
    for b, n in enumerate(st["counts"]):
        for i in range(n):
            r = first + i
            z = st["logits"][r].to(f8)
            lp = torch.log_softmax(z / (1.0 if case["drafts"] == "greedy" else temp), 0)
            x, final = drafts[r], i == n - 1
            if case["drafts"] == "greedy":
                top = int(torch.nonzero(z == z.max())[0, 0])
                ok, token = (not final) and top == x, top
            else:
                p = lp.exp()
                if case["drafts"] == "logits":
                    q = torch.exp((st["draft_logits"][r].to(f8) - st["draft_peak"][r].to(f8)) / temp - st["draft_log_sum"][r].to(f8))
                else:
                    q = torch.zeros_like(p)
                    q[x] = 1.0
                ok = (not final) and us[r] * float(q[x]) < float(p[x])
                if not ok:
                    w = p if final else torch.relu(p - q)
                    w = p if float(w.max()) == 0 else w
                    token = int(torch.argmax(w / st["noise"][b].to(f8)))
            tokens[r] = x if ok else token
            logps[r] = lp[tokens[r]]
            if not ok:
                break
            accepted[b] += 1
        first += n
    return {"accepted": accepted.to(_DEV), "tokens": tokens.to(_DEV), "logp": logps.to(_DEV)}
