"""The serving example with pages that a score selects: it runs, its last outputs are those of
64 bits over the selected pages (bf16's rounding, 2^-8, and the products'), and with as many
pages as there are it is the example without a selection."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_kv4.py")


def serve(args):
    spec = importlib.util.spec_from_file_location("serve_kv4", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m.serve(args)


@pytest.mark.parametrize("pages", [2, 5])
def test_selected_pages(pages):
    r = serve(["--layers", "2", "--batch", "5", "--prompt", "700", "--steps", "20", "--pages", str(pages)])
    assert r["read"] <= 1.5 * 2.0 ** -8


def test_all_pages():
    args = ["--layers", "2", "--batch", "7", "--prompt", "300", "--steps", "9"]
    a, b = serve(args), serve(args + ["--pages", "12"])
    assert b["model"] <= 2.0 ** -4 and b["read"] <= 1.5 * 2.0 ** -8
    assert a["tokens"] == b["tokens"] and a["pages"] == b["pages"]
    assert abs(a["model"] - b["model"]) < 1e-3
