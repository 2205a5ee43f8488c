"""Refusals of the operators on a paged cache and of the verification of drafts that their tables of refusals do not hold (no device work)."""
import pytest

from test_paged_cpu import ALIGN, ATTN, ROPE, SHAPE, call, lib  # noqa: F401


# every stride of a cache that is written to, where more than one of its kind exists
@pytest.mark.parametrize("name", ["k_page", "k_row", "k_head", "v_page", "v_row", "v_head"])
@pytest.mark.parametrize("stride", [0, 8, 120])
def test_rope_append_refuses_slots_that_share_memory(lib, name, stride):
    assert call(lib.resq_rope_append, ROPE, dict(cache={name: stride})) == ALIGN
    assert b"share memory" in lib.resq_last_error()


@pytest.mark.parametrize("name, only", [("k_page", dict(pages=1)), ("v_page", dict(pages=1))])
def test_rope_append_takes_any_stride_of_a_single_one(lib, name, only):
    # (rot is refused behind the strides: nothing is launched)
    assert call(lib.resq_rope_append, ROPE, dict(cache={name: 0, **only}, rot=24)) == SHAPE
    assert b"rot" in lib.resq_last_error()


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38, -0.0])
def test_paged_attention_refuses_scales_without_a_place_in_fp32(lib, scale):
    """scale / ln 2 is what scores are multiplied by."""
    assert call(lib.resq_paged_attention, ATTN, dict(scale=scale)) == SHAPE
    assert b"scale" in lib.resq_last_error()
