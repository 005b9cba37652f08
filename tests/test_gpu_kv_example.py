"""The example that learns centres, fills a cache and decodes over it."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("kv_codes_example",
                                                  os.path.join(ROOT, "examples", "kv_codes.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("kw", [dict(), dict(heads=1, group=8, sub=2, dtype=torch.float16, page=32),
                                dict(heads=1, dim=96, sub=8, centres=200, group=1)])
def test_example(kw):
    got = load().run(prompt=300, steps=3, **kw)
    sub = kw.get("sub", 4)
    assert got["codes"] * 2 * sub == got["plain"]
    # learned centres keep most of a vector: one centre at the mean would leave 1
    assert got["key"] < 0.6 and got["value"] < 0.6
    # over the same keys and values only roundings differ: of the output (2^-9 of
    # bf16), and of the plain form's fp32
    assert got["same"] < 2.0 ** -8
