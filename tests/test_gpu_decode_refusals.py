"""Calls of the operators over a paged cache that are refused: a status, nothing enqueued, nothing written."""

import ctypes

import pytest
import torch

import paper_2511_06605_amd as dl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield
    dl.dl_shutdown()


def refused(call, *args):
    with pytest.raises(dl.DlError) as e:
        call(*args, torch.cuda.current_stream())
    assert e.value.status == dl.DL_ERR_INVALID


def cache():
    codes = lambda: torch.zeros((4, 16, 2, 64), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)  # noqa: E731
    scale = lambda: torch.zeros((4, 16, 2), device="cuda")  # noqa: E731
    return dl.KvCache(codes(), codes(), scale(), scale())


@pytest.mark.parametrize("field,value", [("slots", None), ("slots", 4), ("type", 3), ("type", -1), ("tokens", -1), ("tokens", 1 << 31), ("tokens", 1 << 62),
                                         ("reserved", 1), ("k", 2)])
def test_rows(field, value):
    c = cache()
    rows = dl.KvRows(torch.ones((3, 2, 64), device="cuda"), None, torch.arange(3, device="cuda"))
    setattr(rows.desc, field, value)
    refused(dl.dl_kv_write, c, rows)
    refused(dl.dl_kv_read, c, rows)
    assert not c._tensors[0].view(torch.uint8).any()


@pytest.mark.parametrize("field,value", [("k", None), ("k_scale", None), ("k_scale", 2), ("format", 5), ("head_dim", 63), ("heads", 0), ("page_tokens", 0)])
def test_cache(field, value):
    c = cache()
    rows = dl.KvRows(torch.ones((3, 2, 64), device="cuda"), torch.ones((3, 2, 64), device="cuda"), torch.arange(3, device="cuda"))
    values = dl.KvRows(None, torch.ones((3, 2, 64), device="cuda"), torch.arange(3, device="cuda"))
    setattr(c.desc, field, value)
    L, s = dl.binding.lib(), torch.cuda.current_stream().cuda_stream
    assert L.dl_kv_write(c.at, rows.at, s) == dl.DL_ERR_INVALID and L.dl_kv_read(c.at, rows.at, s) == dl.DL_ERR_INVALID
    if value is None:  # the side that is not there is not asked for
        dl.dl_kv_write(c, values, torch.cuda.current_stream())


def test_null_structs():
    L, s = dl.binding.lib(), torch.cuda.current_stream().cuda_stream
    c = cache()
    rows = dl.KvRows(torch.ones((3, 2, 64), device="cuda"), None, torch.arange(3, device="cuda"))
    for call in (L.dl_kv_write, L.dl_kv_read, L.dl_prefix_attention):
        assert call(None, rows.at, s) == dl.DL_ERR_INVALID and call(c.at, None, s) == dl.DL_ERR_INVALID
    assert L.dl_verify_draft(None, s) == dl.DL_ERR_INVALID
    assert L.dl_prefix_attention_workspace(c.at, None) == dl.DL_ERR_INVALID and L.dl_verify_draft_workspace(None) == dl.DL_ERR_INVALID


@pytest.mark.parametrize("field,value", [
    ("q", None), ("out", None), ("q", 1), ("pages", None), ("lens", None), ("prefix_pages", None), ("lens", 6), ("lse", 2), ("workspace", None),
    ("workspace_bytes", 1000), ("workspace", 8), ("type", 0), ("max_pages", -1), ("q_heads", 3)])
def test_attention(field, value):
    c = cache()
    q = torch.ones((2, 1, 4, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    r = dl.PrefixAttention(c, q, out, torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.ones((2,), dtype=torch.int32, device="cuda"),
                           prefix_pages=torch.zeros((1,), dtype=torch.int32, device="cuda"), prefix_tokens=5, lse=torch.zeros((2, 1, 4), device="cuda"))
    r.use_workspace(torch.zeros(dl.dl_prefix_attention_workspace(r), dtype=torch.uint8, device="cuda"))
    setattr(r.desc, field, value)
    refused(dl.dl_prefix_attention, r)
    assert bool((out == 7).all())


@pytest.mark.parametrize("field,value", [
    ("target", None), ("target", 2), ("draft", 1), ("draft_tokens", None), ("uniform", None), ("race", None), ("race", 2), ("tokens", None),
    ("accepted", None), ("draft_lens", 1), ("workspace", None), ("workspace", 24), ("workspace_bytes", 10), ("vocab", 0), ("drafts", 64)])
def test_verification(field, value):
    tokens, accepted = torch.full((2, 4), 7, dtype=torch.int32, device="cuda"), torch.full((2,), 7, dtype=torch.int32, device="cuda")
    V = 9000
    r = dl.DraftVerify(torch.ones((2, 4, V), device="cuda"), torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((2, 3), device="cuda"),
                       torch.ones((2, V), device="cuda"), tokens, accepted, draft_probs=torch.ones((2, 3, V), device="cuda"))
    r.use_workspace(torch.zeros(dl.dl_verify_draft_workspace(r), dtype=torch.uint8, device="cuda"))
    setattr(r.desc, field, value)
    refused(dl.dl_verify_draft, r)
    assert bool((tokens == 7).all()) and bool((accepted == 7).all())


def test_other_modes_change_nothing():
    """Always one-shot, on the caller's stream."""
    c = cache()
    x = torch.randn((5, 2, 64), device="cuda")
    back = torch.zeros_like(x)
    at = torch.arange(5, device="cuda")
    dl.dl_prelaunch_start()
    try:
        for mode in (dl.DL_MODE_PRELAUNCH, dl.DL_MODE_SIGNAL, dl.DL_MODE_AUTO):
            dl.dl_set_mode(mode)
            back.zero_()
            dl.dl_kv_write(c, dl.KvRows(x, None, at), torch.cuda.current_stream())
            dl.dl_kv_read(c, dl.KvRows(back, None, at), torch.cuda.current_stream())
            assert dl.dl_last_mode() == dl.DL_MODE_ONESHOT
            torch.cuda.synchronize()
            assert bool((back - x).abs().max() < 0.5) and bool(back.any())
        assert ctypes.sizeof(c.desc) == 104
    finally:
        dl.dl_set_mode(dl.DL_MODE_ONESHOT)
        dl.dl_prelaunch_stop()
