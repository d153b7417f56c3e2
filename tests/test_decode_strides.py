"""Strides of dimensions of size one, where nothing is stepped over: they say nothing, and refuse nothing (no GPU)."""

import pytest

import paper_2511_06605_amd as dl

from test_decode_host import Fake


def cache(shape, k=None, v=None, k_scale=None, v_scale=None):
    return dl.KvCache(Fake(shape, "int8", stride=k), Fake(shape, "int8", stride=v), Fake(shape[:3], "float32", stride=k_scale),
                      Fake(shape[:3], "float32", stride=v_scale))


@pytest.mark.parametrize("shape,k,v,k_scale,v_scale", [
    ((1, 16, 2, 64), (2048, 128, 64, 1), (4096, 128, 64, 1), (32, 2, 1), (7, 2, 1)),       # one page
    ((5, 1, 2, 64), (128, 128, 64, 1), (128, 9, 64, 1), (2, 2, 1), (2, 5, 1)),             # one token a page
    ((5, 16, 1, 64), (1024, 64, 64, 1), (1024, 64, 1, 1), (16, 1, 1), (16, 1, 16)),        # one head
    ((1, 16, 1, 64), (1 << 40, 64, 1 << 50, 1), (1024, 64, 64, 1), (1 << 40, 1, 1 << 50), (16, 1, 1)),  # a page of a far larger thing
    ((0, 16, 2, 64), (2048, 128, 64, 1), (4096, 128, 64, 1), (32, 2, 1), (64, 2, 1))])     # none
def test_dimensions_of_one(shape, k, v, k_scale, v_scale):
    c = cache(shape, k, v, k_scale, v_scale)
    plain = cache(shape)
    for name, n in zip(("page", "token", "head"), shape):
        for prefix in ("", "scale_"):
            got, packed = (getattr(x.desc, prefix + name + "_stride") for x in (c, plain))
            assert got == packed == 0 if n <= 1 else got == packed
    q = Fake((2, 1, shape[2], 64), "bfloat16")
    r = dl.PrefixAttention(c, q, q, Fake((2, 3), "int32"), Fake((2,), "int32"))
    assert dl.dl_prefix_attention_workspace(r) >= 65536


@pytest.mark.parametrize("k,v,k_scale,v_scale", [
    ((2048, 128, 64, 1), (4096, 128, 64, 1), None, None), (None, None, (32, 2, 1), (32, 1, 16))])
def test_strides_that_differ(k, v, k_scale, v_scale):
    with pytest.raises(ValueError):
        cache((2, 16, 2, 64), k, v, k_scale, v_scale)
