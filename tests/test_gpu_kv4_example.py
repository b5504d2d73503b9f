"""The serving example end to end.  Its outputs are bf16: 2^-8 of the largest, and half as
much for probabilities of 11 bits and fp32 sums."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_kv4.py")


@pytest.mark.parametrize("args", [[], ["--layers", "1", "--batch", "1", "--prompt", "1", "--steps", "70"],
                                  ["--layers", "2", "--batch", "33", "--prompt", "300", "--steps", "5"]])
def test_example(args):
    spec = importlib.util.spec_from_file_location("serve_kv4", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main(args) <= 1.5 * 2.0 ** -8
