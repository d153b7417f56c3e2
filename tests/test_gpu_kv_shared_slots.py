"""Tokens of one write that share a slot (dl_kv_write, dl_kv_read): what the header says of them, no more and no less."""

import os
import re

import numpy as np
import pytest
import torch

import paper_2511_06605_amd as dl

import decode_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_header_does_not_promise_one_of_the_rows():
    """A row's codes and its scale are stores of several lanes: nothing makes those of one row win together."""
    said = re.sub(r"[\s*]+", " ", open(os.path.join(ROOT, "include", "dmalatte.h")).read())
    assert "leave either row" not in said
    assert "The slots of a call of dl_kv_write differ from each other" in said


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["fp8", "int8"])
def test_other_slots_are_not_affected(kind):
    torch.cuda.set_device(0)
    dl.dl_init(0)
    try:
        rng = np.random.default_rng(1)
        tokens, pages, page, heads, dim = 3000, 100, 16, 2, 128
        slots = rng.integers(-1, pages * page, tokens)
        x = torch.from_numpy(rng.standard_normal((tokens, heads, dim))).float().cuda()
        codes = torch.full((pages, page, heads, dim), 0x55, dtype=torch.uint8, device="cuda").view(decode_ref.CODE[kind])
        scale = torch.full((pages, page, heads), 5.0, device="cuda")
        cache = dl.KvCache(codes, codes, scale, scale)
        at, stream = torch.from_numpy(slots).cuda(), torch.cuda.current_stream()
        dl.dl_kv_write(cache, dl.KvRows(x, None, at), stream)
        y, z = decode_ref.quantised(x.double().cpu().numpy(), kind)
        got = decode_ref.code_values(codes).reshape(pages * page, heads, dim)
        got_scale = scale.cpu().numpy().reshape(pages * page, heads)
        filler = decode_ref.code_values(torch.full((1,), 0x55, dtype=torch.uint8).view(decode_ref.CODE[kind]))[0]
        shared = 0
        for s in range(pages * page):
            mine = np.flatnonzero(slots == s)
            if len(mine) == 0:
                assert (got[s] == filler).all() and (got_scale[s] == 5).all()
            else:
                shared += len(mine) > 1
                assert (got[s] == y[mine]).any(0).all() and (got_scale[s] == z[mine]).any(0).all()
        assert shared > 100
        # a slot that is read more than once
        back = torch.full_like(x, 3.0)
        dl.dl_kv_read(cache, dl.KvRows(back, None, at), stream)
        want = np.where((slots >= 0)[:, None, None], got[slots].astype(np.float32) * got_scale[slots][..., None], np.float32(0))
        assert np.array_equal(back.cpu().numpy(), want)
    finally:
        dl.dl_shutdown()
