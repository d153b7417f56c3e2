"""Strides and sizes that the operators over a paged cache refuse (no GPU)."""

import pytest

import paper_2511_06605_amd as dl

from test_decode_host import attention, cache, refused


@pytest.mark.parametrize("field,value", [
    ("page_stride", -1), ("page_stride", 1 << 32), ("token_stride", -64), ("token_stride", 1 << 32), ("head_stride", -1), ("head_stride", (1 << 46) + 1),
    ("scale_page_stride", -1), ("scale_page_stride", 1 << 30), ("scale_token_stride", -2), ("scale_token_stride", 1 << 30), ("scale_head_stride", -1),
    ("scale_head_stride", (1 << 44) + 1), ("k_scale", 6), ("v_scale", 1)])
def test_strides_and_alignments_that_are_refused(field, value):
    c = cache()
    r = attention(c)
    setattr(c.desc, field, value)
    refused(lambda: dl.dl_prefix_attention_workspace(r), field=field, value=value)


@pytest.mark.parametrize("field,value", [("page_stride", (1 << 32) - 1), ("token_stride", 0), ("scale_page_stride", (1 << 30) - 1), ("head_stride", 1 << 46)])
def test_strides_up_to_the_limits(field, value):
    c = cache()
    r = attention(c)
    setattr(c.desc, field, value)
    assert dl.dl_prefix_attention_workspace(r) >= 65536


def test_rows_of_a_call():
    """batch * q_tokens * q_heads, at most half of DL_MAX_ROWS."""
    r = attention()
    r.desc.q_tokens, r.desc.q_heads = 8, 4
    r.desc.batch = dl.DL_MAX_ROWS // 64
    assert dl.dl_prefix_attention_workspace(r) >= 65536
    r.desc.batch += 1
    refused(lambda: dl.dl_prefix_attention_workspace(r), batch=r.desc.batch)
