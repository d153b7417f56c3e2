"""Calls of the operators that take a prompt into a bounded cache that are refused: a status, nothing enqueued, nothing written."""

import pytest
import torch

import paper_2511_06605_amd as dl

from test_gpu_decode_refusals import cache, refused

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield
    dl.dl_shutdown()


def zeros(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def rotate():
    q, k, i = (torch.ones((3, h, 64), device="cuda") for h in (4, 2, 1))
    return dl.NormRotate(q, k, zeros(3, 4, 64), zeros(3, 2, 64), q_weight=i[0, 0], k_weight=i[0, 0], table=zeros(9, 64), positions=torch.arange(3, device="cuda"))


def packed():
    return torch.ones((6, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda"), zeros(2, 2, dtype=torch.int32), \
        torch.tensor([2, 4], dtype=torch.int32, device="cuda")


def chunk():
    q, starts, pages, lens = packed()
    r = dl.ChunkAttention(cache(), q, torch.zeros_like(q), starts, pages, lens, lse=zeros(6, 4))
    r.use_workspace(zeros(dl.dl_chunk_attention_workspace(r), dtype=torch.uint8))
    return r


def weigh():
    q, starts, pages, lens = packed()
    r = dl.KvWeigh(cache(), q, zeros(6, 4), starts, pages, lens, zeros(2, 32), before=torch.ones((2, 32), device="cuda"))
    r.use_workspace(zeros(dl.dl_kv_weigh_workspace(r), dtype=torch.uint8))
    return r


def evict():
    _, _, pages, lens = packed()
    r = dl.KvEvict(cache(), torch.ones((2, 32), device="cuda"), pages, lens, torch.ones_like(pages)[:, :1], torch.full((2, 3), 7, dtype=torch.int32, device="cuda"),
                   torch.full((2,), 7, dtype=torch.int32, device="cuda"))
    r.use_workspace(zeros(dl.dl_kv_evict_workspace(r), dtype=torch.uint8))
    return r


@pytest.mark.parametrize("field,value", [
    ("type", 3), ("type", -1), ("reserved", 1), ("head_dim", 0), ("head_dim", 72), ("head_dim", 272), ("rotary", 8), ("rotary", 80), ("rotary", -16), ("neighbours", 2),
    ("eps", -1.0), ("eps", float("nan")), ("q_heads", -1), ("k_heads", 65536), ("tokens", -1), ("tokens", 1 << 27), ("tokens", 1 << 62), ("table_rows", -1), ("table_rows", 1 << 31),
    ("q_out", None), ("k_out", None), ("q", 2), ("k_out", 1), ("table", None), ("table", 2), ("positions", None), ("positions", 4), ("q_weight", 2)])
def test_norm_rotate(field, value):
    r = rotate()
    setattr(r.desc, field, value)
    refused(dl.dl_norm_rotate, r)
    assert not r._tensors[2].any() and not r._tensors[3].any()


@pytest.mark.parametrize("field,value", [
    ("type", 0), ("batch", -1), ("batch", 65536), ("tokens", -1), ("q_heads", 3), ("max_pages", -1), ("q", None), ("q", 1), ("out", None), ("out", 1), ("lse", 2),
    ("q_starts", None), ("q_starts", 2), ("pages", None), ("lens", None), ("lens", 1), ("workspace", None), ("workspace", 8), ("workspace_bytes", 65535)])
def test_chunk_attention(field, value):
    r = chunk()
    setattr(r.desc, field, value)
    refused(dl.dl_chunk_attention, r)
    assert not r._tensors[1].any()


@pytest.mark.parametrize("field,value", [
    ("type", 0), ("batch", -1), ("batch", 65536), ("tokens", -1), ("q_heads", 3), ("max_pages", -1), ("q", None), ("q", 1), ("lse", None), ("lse", 2), ("weights", None),
    ("weights", 2), ("before", 2), ("q_starts", None), ("pages", None), ("lens", None), ("workspace", None), ("workspace", 8), ("workspace_bytes", 65535)])
def test_weigh(field, value):
    r = weigh()
    setattr(r.desc, field, value)
    refused(dl.dl_kv_weigh, r)
    assert not r._tensors[5].any()


@pytest.mark.parametrize("field,value", [
    ("batch", -1), ("batch", 65536), ("keep", -1), ("first", 4), ("recent", 4), ("max_pages", -1), ("weights", None), ("weights", 2), ("pages", None), ("lens", None),
    ("to_pages", None), ("kept", None), ("kept", 2), ("kept_lens", None), ("kept_weights", 2), ("workspace", None), ("workspace", 8), ("workspace_bytes", 65535)])
def test_evict(field, value):
    r = evict()
    setattr(r.desc, field, value)
    refused(dl.dl_kv_evict, r)
    assert (r._tensors[4] == 7).all() and (r._tensors[5] == 7).all()


def test_evict_into_what_it_reads():
    r = evict()
    r.desc.kept_lens = r.desc.lens
    refused(dl.dl_kv_evict, r)
    r = evict()
    r.desc.kept_weights = r.desc.weights
    refused(dl.dl_kv_evict, r)
    assert (r._tensors[4] == 7).all() and (r._tensors[5] == 7).all()


def test_null_structs_and_caches_without_codes():
    L, s = dl.binding.lib(), torch.cuda.current_stream().cuda_stream
    assert L.dl_norm_rotate(None, s) == dl.DL_ERR_INVALID
    for call, make in ((L.dl_chunk_attention, chunk), (L.dl_kv_weigh, weigh), (L.dl_kv_evict, evict)):
        r = make()
        assert call(None, r.at, s) == dl.DL_ERR_INVALID and call(r.cache.at, None, s) == dl.DL_ERR_INVALID
        r.cache.desc.k_scale = None
        assert call(r.cache.at, r.at, s) == dl.DL_ERR_INVALID
        r = make()
        r.cache.desc.v = None  # keys alone are enough for what reads nothing else
        assert call(r.cache.at, r.at, s) == (dl.DL_OK if call is L.dl_kv_weigh else dl.DL_ERR_INVALID)
    torch.cuda.synchronize()


def test_what_is_not_refused():
    for call, make in ((dl.dl_norm_rotate, rotate), (dl.dl_chunk_attention, chunk), (dl.dl_kv_weigh, weigh), (dl.dl_kv_evict, evict)):
        call(make(), torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert dl.dl_last_mode() == dl.DL_MODE_ONESHOT
