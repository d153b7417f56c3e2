"""The operators that take a prompt into a bounded cache, run together by the example, which checks every step itself."""

import importlib.util
import os

import pytest
import torch

import paper_2511_06605_amd as dl

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("long_prompt", os.path.join(ROOT, "examples", "long_prompt.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield module
    dl.dl_shutdown()


@pytest.mark.parametrize("more", [
    {}, {"kind": "int8", "dtype": "float16"}, {"batch": 1, "prompt": 70, "chunk": 1, "keep": 40, "recent": 5}, {"prompt": 600, "chunk": 600, "keep": 700},
    {"batch": 3, "prompt": 900, "chunk": 333, "keep": 100, "first": 0, "recent": 0, "dim": 128, "page": 24, "q_heads": 12, "heads": 3},
    {"batch": 1, "prompt": 700, "chunk": 500, "keep": 300, "q_heads": 32, "heads": 1}])
def test_prompts_are_cut(example, more):
    r = example.run(**more)
    keep = more.get("keep", 512)
    assert r["kept"] == [min(n, keep) for n in r["lens"]]
