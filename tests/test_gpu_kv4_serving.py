"""The serving example against the same stack without a cache.

The stack adds up, per layer, some six roundings to bf16 (2^-9 each, of sums as large as the
residual, several times what a layer adds), which move a few codes by one: below 2^-4 of what it
has added after four layers.  Rounding to 4 bits moves keys and values by 2^-3.5, and so do all
of their errors together not reach 2^-1; entries under another position or page would.
"""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_kv4.py")


@pytest.mark.parametrize("args", [[], ["--layers", "2", "--batch", "33", "--prompt", "300", "--piece", "50", "--steps", "5"],
                                  ["--layers", "3", "--batch", "5", "--prompt", "200", "--piece", "7", "--steps", "70"]])
def test_stack_with_and_without_the_cache(args):
    spec = importlib.util.spec_from_file_location("serve_kv4", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.serve(args)
    assert r["mixed"] >= 1
    assert r["model"] <= 2.0 ** -4 and r["read"] <= 1.5 * 2.0 ** -8
    assert r["model"] < r["exact"] <= 2.0 ** -1
