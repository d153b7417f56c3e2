"""What the operators over a paged cache decide on the host: struct layouts, refusals, sizes of workspaces.  No GPU: addresses are made
up and never followed."""

import ctypes
import os
import re
import subprocess

import pytest

import paper_2511_06605_amd as dl
from paper_2511_06605_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STRUCTS = {"dl_kv_cache": binding.KvCacheDesc, "dl_kv_rows": binding.KvRowsDesc, "dl_prefix_attention_args": binding.PrefixAttentionDesc,
           "dl_verify_draft_args": binding.VerifyDraftDesc}


class Fake:
    """As much of a tensor as the descriptors look at."""

    def __init__(self, shape, dtype, stride=None, at=1 << 20, is_cuda=True):
        self.shape, self.dtype, self.at, self.is_cuda = tuple(shape), dtype, at, is_cuda
        self._stride = tuple(stride) if stride else self._packed()

    def _packed(self):
        s, out = 1, []
        for n in reversed(self.shape):
            out.append(s)
            s *= n
        return tuple(reversed(out))

    def data_ptr(self):
        return self.at

    def stride(self):
        return self._stride

    def numel(self):
        n = 1
        for v in self.shape:
            n *= v
        return n

    def element_size(self):
        return {"uint8": 1}[self.dtype]

    def is_contiguous(self):
        return self._stride == self._packed()


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


def cache(pages=10, page=16, heads=2, dim=64, dtype="float8_e4m3fn", **more):
    shape = (pages, page, heads, dim)
    return dl.KvCache(Fake(shape, dtype), Fake(shape, dtype), Fake(shape[:3], "float32"), Fake(shape[:3], "float32"))


def attention(c=None, batch=3, q_tokens=2, q_heads=4, dim=64, width=5, prefix=0, **more):
    shape = (batch, q_tokens, q_heads, dim)
    args = dict(q=Fake(shape, "bfloat16"), out=Fake(shape, "bfloat16"), pages=Fake((batch, width), "int32"), lens=Fake((batch,), "int32"),
                prefix_pages=Fake((-(-prefix // 16),), "int32"), prefix_tokens=prefix)
    args.update(more)
    return dl.PrefixAttention(c or cache(), **args)


def verify(batch=3, drafts=4, vocab=100, dtype="float32", **more):
    args = dict(target=Fake((batch, drafts + 1, vocab), dtype), draft_tokens=Fake((batch, drafts), "int32"), uniform=Fake((batch, drafts), "float32"),
                race=Fake((batch, vocab), "float32"), tokens=Fake((batch, drafts + 1), "int32"), accepted=Fake((batch,), "int32"),
                draft_probs=Fake((batch, drafts, vocab), dtype))
    args.update(more)
    return dl.DraftVerify(**args)


def test_nothing_runs_before_init():
    with pytest.raises(dl.DlError) as e:
        dl.dl_kv_write(cache(), dl.KvRows(Fake((3, 2, 64), "float32"), None, Fake((3,), "int64")))
    assert e.value.status == dl.DL_ERR_STATE
    for call, request in ((dl.dl_prefix_attention, attention()), (dl.dl_verify_draft, verify())):
        with pytest.raises(dl.DlError) as e:
            call(request)
        assert e.value.status == dl.DL_ERR_STATE


def test_descriptors_refuse_what_does_not_fit():
    for make in (
            lambda: dl.KvCache(Fake((1, 16, 2, 64), "float32"), Fake((1, 16, 2, 64), "float32"), Fake((1, 16, 2), "float32"), Fake((1, 16, 2), "float32")),
            lambda: dl.KvCache(Fake((1, 16, 2, 64), "int8"), Fake((1, 16, 2, 64), "float8_e4m3fn"), Fake((1, 16, 2), "float32"), Fake((1, 16, 2), "float32")),
            lambda: dl.KvCache(Fake((1, 16, 2, 64), "int8"), Fake((1, 16, 2, 64), "int8"), Fake((1, 16, 1), "float32"), Fake((1, 16, 2), "float32")),
            lambda: dl.KvCache(Fake((1, 16, 2, 64), "int8"), Fake((1, 16, 2, 64), "int8", stride=(4096, 256, 64, 1)), Fake((1, 16, 2), "float32"), Fake((1, 16, 2), "float32")),
            lambda: dl.KvCache(Fake((1, 16, 2, 64), "int8", stride=(2048, 128, 1, 2)), Fake((1, 16, 2, 64), "int8"), Fake((1, 16, 2), "float32"), Fake((1, 16, 2), "float32")),
            lambda: dl.KvCache(Fake((1, 16, 2, 64), "int8", is_cuda=False), Fake((1, 16, 2, 64), "int8"), Fake((1, 16, 2), "float32"), Fake((1, 16, 2), "float32")),
            lambda: dl.KvRows(None, None, Fake((3,), "int64")),
            lambda: dl.KvRows(Fake((3, 2, 64), "float32"), Fake((3, 2, 64), "bfloat16"), Fake((3,), "int64")),
            lambda: dl.KvRows(Fake((3, 2, 64), "int8"), None, Fake((3,), "int64")),
            lambda: dl.KvRows(Fake((3, 2, 64), "float32"), None, Fake((3,), "int32")),
            lambda: dl.KvRows(Fake((3, 2, 64), "float32"), None, Fake((4,), "int64")),
            lambda: attention(dim=128),
            lambda: attention(q=Fake((3, 2, 4, 64), "float32")),
            lambda: attention(out=Fake((3, 2, 4, 64), "float16")),
            lambda: attention(lens=Fake((2,), "int32")),
            lambda: attention(pages=Fake((3, 5), "int64")),
            lambda: attention(prefix_tokens=100),
            lambda: attention(lse=Fake((3, 2, 4), "float32", stride=(16, 8, 2))),
            lambda: verify(draft_tokens=Fake((3, 4), "int64")),
            lambda: verify(race=Fake((3, 99), "float32")),
            lambda: verify(draft_probs=Fake((3, 4, 100), "float16")),
            lambda: verify(tokens=Fake((3, 4), "int32"))):
        with pytest.raises(ValueError):
            make()
    with pytest.raises(ValueError):
        dl.dl_kv_write(cache(), dl.KvRows(Fake((3, 1, 64), "float32"), None, Fake((3,), "int64")))


def refused(f, **fields):
    with pytest.raises(dl.DlError) as e:
        f()
    assert e.value.status == dl.DL_ERR_INVALID, fields


@pytest.mark.parametrize("field,value", [
    ("format", 2), ("format", -1), ("heads", 0), ("heads", 65536), ("heads", 3), ("head_dim", 0), ("head_dim", 8), ("head_dim", 72), ("head_dim", 272),
    ("page_tokens", 0), ("page_tokens", 65537), ("pages", -1), ("pages", 1 << 31)])
def test_caches_that_are_refused(field, value):
    c = cache()
    r = attention(c)
    setattr(c.desc, field, value)
    refused(lambda: dl.dl_prefix_attention_workspace(r), field=field, value=value)


@pytest.mark.parametrize("field,value", [
    ("type", dl.DL_TYPE_F32), ("type", 3), ("batch", -1), ("q_tokens", -1), ("q_heads", 3), ("q_heads", -2), ("prefix_tokens", -1),
    ("prefix_tokens", (1 << 30) + 1), ("max_pages", -1), ("max_pages", (1 << 26) + 1), ("max_pages", 1 << 62), ("reserved", 1), ("batch", 1 << 30)])
def test_attention_that_is_refused(field, value):
    r = attention()
    setattr(r.desc, field, value)
    refused(lambda: dl.dl_prefix_attention_workspace(r), field=field, value=value)


@pytest.mark.parametrize("field,value", [
    ("type", 3), ("type", -1), ("batch", -1), ("batch", (1 << 20) + 1), ("drafts", -1), ("drafts", 64), ("vocab", 0), ("vocab", (1 << 30) + 1)])
def test_verification_that_is_refused(field, value):
    r = verify()
    setattr(r.desc, field, value)
    refused(lambda: dl.dl_verify_draft_workspace(r), field=field, value=value)


def test_workspaces():
    """At least the control words; with the rows, and never more than a few times 256 compute units' worth of pieces."""
    least = dl.dl_prefix_attention_workspace(attention(batch=0))
    assert least >= 65536 and dl.dl_verify_draft_workspace(verify()) >= 65536
    small, large = (dl.dl_prefix_attention_workspace(attention(batch=b, prefix=4000, prefix_pages=Fake((250,), "int32"))) for b in (1, 500))
    assert least < small < large
    # 131 072 rows of 64 floats: with the lengths at their limits no more than 64 pieces each
    wide = dl.dl_prefix_attention_workspace(attention(batch=16384, width=1 << 16))
    assert wide <= 64 * 131072 * (64 * 4 + 8) + (1 << 20)


def test_a_workspace_is_named_with_its_size():
    r = attention()
    w = Fake((1 << 20,), "uint8", at=1 << 30)
    r.use_workspace(w)
    assert r.desc.workspace == 1 << 30 and r.desc.workspace_bytes == 1 << 20
    with pytest.raises(ValueError):
        r.use_workspace(Fake((64,), "uint8", is_cuda=False))
