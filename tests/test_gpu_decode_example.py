"""The example that runs the copies and the operators over a paged cache together; it checks its last step itself."""

import importlib.util
import os

import pytest
import torch

import paper_2511_06605_amd as dl

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decode_step", os.path.join(ROOT, "examples", "decode_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield module
    dl.dl_shutdown()


@pytest.mark.parametrize("kind,dtype,batch,prefix,drafts", [("fp8", "bfloat16", 8, 2000, 4), ("int8", "float16", 1, 33, 1), ("int8", "bfloat16", 3, 5, 7)])
def test_decoding_with_drafts(example, kind, dtype, batch, prefix, drafts):
    r = example.run(batch=batch, prefix=prefix, drafts=drafts, steps=4, kind=kind, dtype=dtype)
    assert len(r["texts"]) == batch and all(len(t) >= 4 for t in r["texts"])
    assert sum(len(t) for t in r["texts"]) == r["accepted"] + 4 * batch
    assert 0 <= r["accepted"] <= r["proposed"]


@pytest.mark.parametrize("tokens,heads", [((1 << 26) + 1, 2), (1 << 27, 2), ((1 << 27) + 1, 1)])
def test_more_rows_than_a_launch_holds(example, tokens, heads):
    """Refused before anything is looked at (the rows that are named are not there)."""
    codes = lambda: torch.zeros((4, 16, heads, 64), dtype=torch.uint8, device="cuda").view(torch.int8)  # noqa: E731
    scale = lambda: torch.zeros((4, 16, heads), device="cuda")  # noqa: E731
    c = dl.KvCache(codes(), codes(), scale(), scale())
    rows = dl.KvRows(torch.ones((3, heads, 64), device="cuda"), None, torch.arange(3, device="cuda"))
    rows.desc.tokens = tokens
    for call in (dl.dl_kv_write, dl.dl_kv_read):
        with pytest.raises(dl.DlError) as e:
            call(c, rows, torch.cuda.current_stream())
        assert e.value.status == dl.DL_ERR_INVALID
