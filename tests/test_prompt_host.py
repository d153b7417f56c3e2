"""What the operators that take a prompt into a bounded cache decide on the host: struct layouts, refusals, sizes of workspaces.  No GPU:
addresses are made up and never followed."""

import ctypes
import os
import re
import subprocess

import pytest

import paper_2511_06605_amd as dl
from paper_2511_06605_amd import binding

from test_decode_host import Fake, cache, refused

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STRUCTS = {"dl_norm_rotate_args": binding.NormRotateDesc, "dl_chunk_attention_args": binding.ChunkAttentionDesc,
           "dl_kv_weigh_args": binding.KvWeighDesc, "dl_kv_evict_args": binding.KvEvictDesc}


def test_structs_have_the_layout_of_the_header(tmp_path):
    """Names in the header's order, and the offsets that a C compiler gives them."""
    header = open(os.path.join(ROOT, "include", "dmalatte.h")).read()
    lines = []
    for name, cls in STRUCTS.items():
        body = re.sub(r"/\*.*?\*/", "", header[header.index("typedef struct %s {" % name):header.index("} %s;" % name)], flags=re.S)
        declared = [re.search(r"(\w+)$", part.strip()).group(1) for line in body.split("{")[1].split(";") for part in line.split(",") if part.strip()]
        assert declared == [f[0] for f in cls._fields_], name
        lines.append('printf("%%zu", sizeof(%s));' % name)
        lines += ['printf(" %%zu", offsetof(%s, %s));' % (name, f) for f in declared]
        lines.append('printf("\\n");')
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include "dmalatte.h"\nint main(void) { %s return 0; }\n' % "\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    said = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()
    for line, (name, cls) in zip(said, STRUCTS.items()):
        got = [int(v) for v in line.split()]
        assert got == [ctypes.sizeof(cls)] + [getattr(cls, f[0]).offset for f in cls._fields_], name


def rotate(T=3, q_heads=4, k_heads=2, dim=64, dtype="bfloat16", **more):
    args = dict(q=Fake((T, q_heads, dim), dtype), k=Fake((T, k_heads, dim), dtype), q_weight=Fake((dim,), "float32"), k_weight=Fake((dim,), "float32"),
                table=Fake((100, dim), "float32"), positions=Fake((T,), "int64"))
    args.update(more)
    return dl.NormRotate(**args)


def packed(T=6, q_heads=4, dim=64, batch=3, width=5):
    return dict(q=Fake((T, q_heads, dim), "bfloat16"), q_starts=Fake((batch + 1,), "int32"), pages=Fake((batch, width), "int32"), lens=Fake((batch,), "int32"))


def chunk(c=None, **more):
    own = {k: more.pop(k) for k in ("T", "q_heads", "dim", "batch", "width") if k in more}
    args = packed(**own)
    args.update(out=Fake(args["q"].shape, "bfloat16"))
    args.update(more)
    return dl.ChunkAttention(c or cache(), **args)


def weigh(c=None, **more):
    own = {k: more.pop(k) for k in ("T", "q_heads", "dim", "batch", "width") if k in more}
    args = packed(**own)
    args.update(lse=Fake(args["q"].shape[:2], "float32"), weights=Fake((args["pages"].shape[0], args["pages"].shape[1] * 16), "float32"))
    args.update(more)
    return dl.KvWeigh(c or cache(), **args)


def evict(c=None, batch=3, width=5, keep=20, **more):
    args = dict(weights=Fake((batch, width * 16), "float32"), pages=Fake((batch, width), "int32"), lens=Fake((batch,), "int32"),
                to_pages=Fake((batch, -(-keep // 16)), "int32"), kept=Fake((batch, keep), "int32"), kept_lens=Fake((batch,), "int32"),
                kept_weights=Fake((batch, keep), "float32"))
    args.update(more)
    return dl.KvEvict(c or cache(), **args)


CALLS = [(dl.dl_norm_rotate, rotate), (dl.dl_chunk_attention, chunk), (dl.dl_kv_weigh, weigh), (dl.dl_kv_evict, evict)]


def test_nothing_runs_before_init():
    for call, make in CALLS:
        with pytest.raises(dl.DlError) as e:
            call(make())
        assert e.value.status == dl.DL_ERR_STATE


def test_descriptors_refuse_what_does_not_fit():
    f = Fake
    for make in (
            lambda: dl.NormRotate(None, None),
            lambda: rotate(q=f((3, 4, 64), "int8")),
            lambda: rotate(k=f((3, 2, 64), "float16")),
            lambda: rotate(k=f((4, 2, 64), "bfloat16")),
            lambda: rotate(k=f((3, 2, 32), "bfloat16")),
            lambda: rotate(q=f((3, 4), "bfloat16")),
            lambda: rotate(q_out=f((3, 5, 64), "bfloat16")),
            lambda: rotate(q_out=f((3, 4, 64), "float32")),
            lambda: rotate(q_out=f((3, 4, 64), "bfloat16", stride=(512, 128, 2))),
            lambda: rotate(q_weight=f((64,), "bfloat16")),
            lambda: rotate(k_weight=f((32,), "float32")),
            lambda: rotate(k=None),
            lambda: rotate(positions=None),
            lambda: rotate(positions=f((3,), "int32")),
            lambda: rotate(positions=f((4,), "int64")),
            lambda: rotate(table=f((100, 64), "float16")),
            lambda: rotate(table=f((100, 64), "float32", is_cuda=False)),
            lambda: chunk(dim=128),
            lambda: chunk(q=f((6, 4, 64), "float32")),
            lambda: chunk(q=f((6, 1, 4, 64), "bfloat16")),
            lambda: chunk(out=f((6, 4, 64), "float16")),
            lambda: chunk(out=f((5, 4, 64), "bfloat16")),
            lambda: chunk(q_starts=f((3,), "int32")),
            lambda: chunk(q_starts=f((4,), "int64")),
            lambda: chunk(pages=f((2, 5), "int32")),
            lambda: chunk(pages=f((3, 5), "int32", stride=(10, 2))),
            lambda: chunk(lens=f((3,), "int64")),
            lambda: chunk(lse=f((6, 4), "float32", stride=(8, 2))),
            lambda: chunk(lse=f((6, 4), "bfloat16")),
            lambda: weigh(lse=f((6, 3), "float32")),
            lambda: weigh(weights=f((3, 79), "float32")),
            lambda: weigh(weights=f((3, 80), "float16")),
            lambda: weigh(before=f((2, 80), "float32")),
            lambda: weigh(before=f((3, 80), "float32", stride=(160, 2))),
            lambda: evict(weights=f((3, 79), "float32")),
            lambda: evict(to_pages=f((3, 1), "int32")),
            lambda: evict(kept=f((60,), "int32")),
            lambda: evict(kept=f((3, 20), "int64")),
            lambda: evict(kept=f((3, 20), "int32", stride=(40, 1))),
            lambda: evict(kept_lens=f((2,), "int32")),
            lambda: evict(kept_weights=f((3, 19), "float32")),
            lambda: evict(lens=f((3,), "int32", is_cuda=False))):
        with pytest.raises(ValueError):
            make()


def test_empty_tensors_have_no_strides_to_refuse():
    assert rotate(T=0, q=Fake((0, 4, 64), "bfloat16", stride=(1, 1, 0))).desc.tokens == 0


@pytest.mark.parametrize("field,value", [
    ("format", 2), ("heads", 0), ("heads", 65536), ("heads", 3), ("head_dim", 72), ("head_dim", 272), ("page_tokens", 0), ("page_tokens", 65537),
    ("pages", -1), ("pages", 1 << 31), ("page_stride", -1), ("token_stride", 1 << 32), ("k_scale", 2)])
def test_caches_that_are_refused(field, value):
    c = cache()
    sizes = [(dl.dl_chunk_attention_workspace, chunk(c)), (dl.dl_kv_weigh_workspace, weigh(c)), (dl.dl_kv_evict_workspace, evict(c))]
    setattr(c.desc, field, value)
    for f, r in sizes:
        if (field, value) != ("heads", 3) or f is not dl.dl_kv_evict_workspace:  # (no queries there to share the heads)
            refused(lambda: f(r), field=field, value=value)


@pytest.mark.parametrize("field,value", [
    ("type", dl.DL_TYPE_F32), ("type", 3), ("batch", -1), ("batch", 65536), ("tokens", -1), ("tokens", 1 << 62), ("tokens", 1 << 25), ("q_heads", 3), ("q_heads", -2),
    ("q_heads", (1 << 31) - 2), ("max_pages", -1), ("max_pages", (1 << 26) + 1), ("max_pages", 1 << 62)])
def test_packed_queries_that_are_refused(field, value):
    for f, r in ((dl.dl_chunk_attention_workspace, chunk()), (dl.dl_kv_weigh_workspace, weigh())):
        setattr(r.desc, field, value)
        refused(lambda: f(r), field=field, value=value)


def test_weights_of_more_tokens_than_32_bits_count_are_refused():
    r = weigh()
    r.desc.max_pages, r.desc.batch = 1 << 26, 2
    refused(lambda: dl.dl_kv_weigh_workspace(r))


@pytest.mark.parametrize("field,value", [
    ("batch", -1), ("batch", 65536), ("keep", -1), ("keep", 1 << 25), ("first", -1), ("recent", -1), ("first", 21), ("recent", 21), ("recent", (1 << 31) - 1),
    ("max_pages", -1), ("max_pages", (1 << 26) + 1), ("max_pages", 1 << 62)])
def test_evictions_that_are_refused(field, value):
    r = evict()
    setattr(r.desc, field, value)
    refused(lambda: dl.dl_kv_evict_workspace(r), field=field, value=value)
    r = evict()
    r.desc.first, r.desc.recent = 10, 11
    refused(lambda: dl.dl_kv_evict_workspace(r))


def test_workspaces():
    """At least the control words, and no more than two rounds of workgroups leave behind, whatever the lengths may become."""
    for f, make in ((dl.dl_chunk_attention_workspace, chunk), (dl.dl_kv_weigh_workspace, weigh), (dl.dl_kv_evict_workspace, evict)):
        assert f(make()) >= 65536
        assert f(make(batch=0)) >= 65536
    assert dl.dl_chunk_attention_workspace(chunk(T=8000, batch=16, width=1 << 16)) <= 2 * 512 * 128 * (64 * 4 + 8) + (1 << 20)


def test_strides_are_those_of_the_tensors():
    wide = lambda heads: Fake((3, heads, 64), "bfloat16", stride=(1000, 70, 1))  # noqa: E731
    d = rotate(q=wide(4), k=wide(2), k_out=Fake((3, 2, 64), "bfloat16")).desc
    assert (d.q_token_stride, d.q_head_stride, d.q_out_token_stride, d.q_out_head_stride) == (1000, 70, 1000, 70)
    assert (d.k_token_stride, d.k_out_token_stride, d.k_out_head_stride, d.rotary, d.table_rows) == (1000, 128, 64, 64, 100)
    assert d.q_out == d.q
    d = evict(weights=Fake((3, 80), "float32", stride=(200, 1)), kept_weights=Fake((3, 20), "float32", stride=(90, 1))).desc
    assert (d.weights_stride, d.kept_weights_stride, d.keep, d.max_pages) == (200, 90, 20, 5)
