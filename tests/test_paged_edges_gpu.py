"""What the operators on a paged cache do at their edges, against their definitions in 64 bits (paged_formulas.py; tolerances of
attention as in test_paged_gpu.py)."""
import pytest
import torch

from test_paged_gpu import BF, NAN, Paged, rq

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
