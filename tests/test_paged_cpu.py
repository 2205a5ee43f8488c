"""Host-side refusals of rotation into a paged cache, attention over it and verification of drafts (no device work), and the
formulas that the GPU tests hold them to, checked against other ways to compute them."""
import ctypes

import pytest
import torch

import paged_formulas as formulas

OK, NULL, SHAPE, ALIGN, WORKSPACE, PATTERN = 0, 1, 2, 3, 4, 5
P = 0x100000  # an aligned address that no call below gets far enough to use


@pytest.fixture(scope="module")
def lib():
    from paper_2607_26515_b200 import binding, build
    build.build()
    return binding.lib()


CACHE = dict(k=P, v=P, pages=10, page_size=16, kv_heads=2, head_dim=128, k_page=4096, k_row=256, k_head=128, v_page=4096, v_row=256, v_head=128)
SEQS = dict(q_start=P, kv_len=P, page_table=P, count=3, max_pages=4, ld_table=4)
ROPE = dict(qkv=P, dtype=0, T=5, ldqkv=2560, Hq=16, Hkv=2, D=128, bias=P, inv_freq=P, rot=128, pairs=0, positions=P, cache=CACHE, seqs=SEQS, Q=P,
            ldq=2048, stream=None)
ATTN = dict(Q=P, T=5, ldq=2048, Hq=16, Hkv=2, D=128, cache=CACHE, seqs=SEQS, max_new=1, scale=0.1, O=P, ldo=2048, lse=P, ws=P, ws_bytes=1 << 34,
            stream=None)

PAGED_BAD = [
    (NULL, dict(cache=None)), (NULL, dict(seqs=None)), (NULL, dict(cache=dict(k=None))), (NULL, dict(cache=dict(v=None))),
    (NULL, dict(seqs=dict(q_start=None))), (NULL, dict(seqs=dict(kv_len=None))), (NULL, dict(seqs=dict(page_table=None))),
    (SHAPE, dict(T=0)), (SHAPE, dict(T=-4)), (SHAPE, dict(T=2 ** 31)), (SHAPE, dict(T=2 ** 27)), (SHAPE, dict(Hq=15)), (SHAPE, dict(Hq=0)),
    (SHAPE, dict(Hkv=0)), (SHAPE, dict(Hkv=1)), (SHAPE, dict(D=96)), (SHAPE, dict(D=64)), (SHAPE, dict(cache=dict(head_dim=64))),
    (SHAPE, dict(Hq=258)), (SHAPE, dict(cache=dict(kv_heads=4))), (SHAPE, dict(seqs=dict(count=0))), (SHAPE, dict(seqs=dict(count=4097))),
    (SHAPE, dict(cache=dict(pages=0))), (SHAPE, dict(cache=dict(pages=2 ** 31))), (SHAPE, dict(cache=dict(page_size=12))),
    (SHAPE, dict(cache=dict(page_size=0))), (SHAPE, dict(cache=dict(page_size=65544))), (SHAPE, dict(seqs=dict(max_pages=0))),
    (SHAPE, dict(seqs=dict(max_pages=2 ** 27, ld_table=2 ** 27))),
    (ALIGN, dict(cache=dict(k=P + 8))), (ALIGN, dict(cache=dict(v=P + 2))), (ALIGN, dict(cache=dict(k_row=252))), (ALIGN, dict(cache=dict(v_head=4))),
    (ALIGN, dict(cache=dict(k_page=-4096))), (ALIGN, dict(cache=dict(v_page=2 ** 36))), (ALIGN, dict(seqs=dict(q_start=P + 2))),
    (ALIGN, dict(seqs=dict(kv_len=P + 1))), (ALIGN, dict(seqs=dict(page_table=P + 2))), (ALIGN, dict(seqs=dict(ld_table=3))),
]
ROPE_BAD = PAGED_BAD + [
    (NULL, dict(qkv=None)), (NULL, dict(Q=None)), (NULL, dict(inv_freq=None)), (PATTERN, dict(dtype=2)), (PATTERN, dict(dtype=-1)),
    (SHAPE, dict(rot=-16)), (SHAPE, dict(rot=144)), (SHAPE, dict(rot=24)),
    (ALIGN, dict(qkv=P + 2)), (ALIGN, dict(ldqkv=2552)), (ALIGN, dict(ldqkv=2564)), (ALIGN, dict(Q=P + 8)), (ALIGN, dict(ldq=2040)),
    (ALIGN, dict(bias=P + 8)), (ALIGN, dict(inv_freq=P + 4)), (ALIGN, dict(positions=P + 2)),
]
ATTN_BAD = PAGED_BAD + [
    (NULL, dict(Q=None)), (NULL, dict(O=None)), (SHAPE, dict(scale=0.0)), (SHAPE, dict(scale=-0.1)), (SHAPE, dict(scale=float("nan"))),
    (SHAPE, dict(scale=float("inf"))), (ALIGN, dict(Q=P + 8)), (ALIGN, dict(ldq=2047)), (ALIGN, dict(O=P + 4)), (ALIGN, dict(ldo=8)),
    (ALIGN, dict(lse=P + 2)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws=P + 128)), (WORKSPACE, dict(ws_bytes=4096)),
]


class _PagedCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v")] + [(n, ctypes.c_int64) for n in CACHE if n not in ("k", "v")]


class _Sequences(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q_start", "kv_len", "page_table")] + [(n, ctypes.c_int64) for n in ("count", "max_pages", "ld_table")]


def call(fn, args, changes):
    got, held = [], []
    for name, value in args.items():
        if name in ("cache", "seqs"):
            change = changes.get(name, {})
            if change is None:
                got.append(None)
                continue
            assert set(change) <= set(value), change
            held.append((_PagedCache if name == "cache" else _Sequences)(**{**value, **change}))
            got.append(ctypes.addressof(held[-1]))
        else:
            got.append(changes.get(name, value))
    assert set(changes) <= set(args), changes
    return fn(*got)


@pytest.mark.parametrize("status, changes", ROPE_BAD)
def test_rope_append_refuses(lib, status, changes):
    assert call(lib.resq_rope_append, ROPE, changes) == status
    assert lib.resq_last_error()


@pytest.mark.parametrize("status, changes", ATTN_BAD)
def test_paged_attention_refuses(lib, status, changes):
    assert call(lib.resq_paged_attention, ATTN, changes) == status
    assert lib.resq_last_error()


VERIFY = dict(logits=P, dtype=0, R=10, V=100, ld=104, row_start=P, count=2, drafts=P, u=P, noise=P, lde=104, draft_logits=P, ldd=104, draft_peak=P,
              draft_log_sum=P, temperature=1.0, accepted=P, tokens=P, logp=P, ws=P, ws_bytes=1 << 20, stream=None)
VERIFY_BAD = [
    (NULL, dict(logits=None)), (NULL, dict(row_start=None)), (NULL, dict(drafts=None)), (NULL, dict(accepted=None)), (NULL, dict(tokens=None)),
    (NULL, dict(logp=None)), (NULL, dict(u=None)), (NULL, dict(noise=None)), (NULL, dict(draft_peak=None)), (NULL, dict(draft_log_sum=None)),
    (PATTERN, dict(dtype=3)), (SHAPE, dict(R=0)), (SHAPE, dict(R=2 ** 31)), (SHAPE, dict(V=0)), (SHAPE, dict(V=2 ** 28 + 8, ld=2 ** 28 + 8)),
    (SHAPE, dict(count=0)), (SHAPE, dict(count=4097)), (SHAPE, dict(temperature=-1.0)), (SHAPE, dict(temperature=1e-9)),
    (SHAPE, dict(temperature=float("nan"))), (SHAPE, dict(temperature=1e7)),
    (ALIGN, dict(logits=P + 2)), (ALIGN, dict(ld=96)), (ALIGN, dict(ld=100)), (ALIGN, dict(noise=P + 4)), (ALIGN, dict(lde=96)), (ALIGN, dict(lde=102)),
    (ALIGN, dict(draft_logits=P + 8)), (ALIGN, dict(ldd=99)), (ALIGN, dict(drafts=P + 4)), (ALIGN, dict(tokens=P + 4)), (ALIGN, dict(row_start=P + 2)),
    (ALIGN, dict(u=P + 1)), (ALIGN, dict(accepted=P + 2)), (ALIGN, dict(logp=P + 2)), (ALIGN, dict(draft_peak=P + 2)), (ALIGN, dict(draft_log_sum=P + 2)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws=P + 64)), (WORKSPACE, dict(ws_bytes=256)),
]


@pytest.mark.parametrize("status, changes", VERIFY_BAD)
def test_verify_drafts_refuses(lib, status, changes):
    assert set(changes) <= set(VERIFY)
    assert lib.resq_verify_drafts(*{**VERIFY, **changes}.values()) == status
    assert lib.resq_last_error()


def test_workspace_queries(lib):
    assert lib.resq_verify_drafts_workspace_bytes(0) == 0 and lib.resq_verify_drafts_workspace_bytes(1000) >= 16000
    q = lib.resq_paged_attention_workspace_bytes
    assert q(0, 1, 16, 2, 128, 1) == 0 and q(1, 1, 15, 2, 128, 1) == 0 and q(1, 1, 16, 2, 96, 1) == 0
    assert q(4, 4, 16, 2, 128, 1) > 0 and q(4, 4, 16, 2, 128, 1) <= q(4000, 4, 16, 2, 128, 0)
    # one more byte is enough, one less is not
    n = q(5, 3, 16, 2, 128, 1)
    assert call(lib.resq_paged_attention, ATTN, dict(ws_bytes=n - 1)) == WORKSPACE


def test_packed_structs_have_the_layout_of_the_header():
    from paper_2607_26515_b200 import binding
    cache, seqs = _PagedCache(*range(1, 13)), _Sequences(*range(21, 27))
    assert bytes(cache) == binding._PAGED_CACHE.pack(*range(1, 13)) and bytes(seqs) == binding._SEQUENCES.pack(*range(21, 27))


def test_binding_refuses_on_the_cpu():
    """The Python calls name what is wrong before anything reaches the library."""
    import paper_2607_26515_b200 as m
    t = torch.zeros((2, 256), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="qkv must be a 2-D CUDA tensor"):
        m.rope_append(t, t, t, t, t, t, t)
    with pytest.raises(ValueError, match="q must be a 2-D CUDA tensor"):
        m.paged_attention(t, t, t, t, t, t)
    with pytest.raises(ValueError, match="logits must be a 2-D CUDA tensor"):
        m.verify_drafts(t, t, t)


# ------------------------------------------------------------------------------------------------ the formulas themselves

def test_attention_formula_against_a_loop():
    g = torch.Generator().manual_seed(0)
    page, Hkv, D, Hq = 8, 2, 64, 4
    k, v = (torch.randn((6, page, Hkv, D), generator=g) for _ in range(2))
    table = torch.tensor([[4, 1, -1], [3, 0, 2]])
    q_start, kv_len = [0, 3, 5], [12, 20]
    q = torch.randn((5, Hq * D), generator=g)
    out, lse, _, _ = formulas.attention(q, k, v, q_start, kv_len, table, 0.2)
    for t in range(5):
        b = 0 if t < 3 else 1
        last = kv_len[b] - (q_start[b + 1] - q_start[b]) + t - q_start[b]
        for h in range(Hq):
            x = q[t, h * D:(h + 1) * D].double()
            s, vs = [], []
            for j in range(last + 1):
                id = int(table[b, j // page])
                kj, vj = (k[id, j % page, h // 2], v[id, j % page, h // 2]) if id >= 0 else (torch.zeros(D), torch.zeros(D))
                s.append(0.2 * float(x @ kj.double()))
                vs.append(vj.double())
            s = torch.tensor(s, dtype=torch.float64)
            p = (s - s.max()).exp() / (s - s.max()).exp().sum()
            assert torch.allclose(out[t, h * D:(h + 1) * D], sum(pj * vj for pj, vj in zip(p, vs)), atol=1e-12)
            assert abs(float(lse[t, h]) - float(torch.logsumexp(s, 0))) < 1e-12


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_formula_is_a_rotation_of_complex_numbers(pairs):
    g = torch.Generator().manual_seed(1)
    D, rot = 64, 32
    qkv = torch.randn((3, 3 * D), generator=g)
    k, v = (torch.zeros((2, 8, 1, D)) for _ in range(2))
    inv = 100.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / 8)
    q, kc, vc = formulas.rope_append(qkv, None, k, v, [0, 3], [9], torch.tensor([[1, 0]]), inv, pairs)
    for i in range(3):
        x = qkv[i].double().view(3, D)
        for head, got in ((0, q[i]), (1, kc[0 if 6 + i >= 8 else 1, (6 + i) % 8, 0])):
            re, im = (x[head, :rot:2], x[head, 1:rot:2]) if pairs else (x[head, :rot // 2], x[head, rot // 2:rot])
            z = torch.complex(re, im) * torch.exp(1j * (6 + i) * inv)
            a, b = (got[:rot:2], got[1:rot:2]) if pairs else (got[:rot // 2], got[rot // 2:rot])
            assert torch.allclose(a, z.real, atol=1e-12) and torch.allclose(b, z.imag, atol=1e-12)
            assert torch.equal(got[rot:], x[head, rot:])
        assert torch.equal(vc[0 if 6 + i >= 8 else 1, (6 + i) % 8, 0], x[2])


def test_verify_formula_draws_from_the_target():
    """The chance that a token comes out, summed over the drafts: min(q, p) + (1 - sum min) residual = p."""
    g = torch.Generator().manual_seed(2)
    z, zq = torch.randn(7, generator=g).double(), torch.randn(7, generator=g).double()
    p, q = torch.softmax(z, 0), torch.softmax(zq, 0)
    kept = torch.minimum(p, q)
    rest = torch.relu(p - q)
    assert torch.allclose(kept + (1 - kept.sum()) * rest / rest.sum(), p)
    # the formula keeps exactly while u q < p
    for x in range(7):
        for u, want in ((float(p[x] / q[x]) * (1 - 1e-9), 1), (float(p[x] / q[x]) * (1 + 1e-9), 0)):
            got = formulas.verify(z.expand(2, 7), [0, 2], torch.tensor([x, 0]), torch.tensor([u, 0.5], dtype=torch.float64), torch.ones((1, 7)), zq.expand(2, 7),
                                  zq.max().expand(2), torch.log((zq - zq.max()).exp().sum()).expand(2), 1.0)
            assert got[0] == [want]
