"""What the page plan refuses of buffers that overlap, before any CUDA call."""
import pytest

from test_kv4 import A, _plan, lib  # noqa: F401

WRITTEN = {"table": 32, "kv_len": 8, "row_start": 12, "slot": 16, "pos": 8, "free_head_out": 4}
READ = {"len": 8, "n_new": 8, "free_pages": 16, "free_head": 4}


def at(name):
    return getattr(_plan(), name)


@pytest.mark.parametrize("written", list(WRITTEN))
@pytest.mark.parametrize("other", list(READ) + list(WRITTEN))
def test_plan_refuses_overlapping_buffers(lib, written, other):  # noqa: F811
    if written == other:
        return
    size = {**WRITTEN, **READ}[other]
    for where in (at(other), at(other) + size - 4, at(other) - WRITTEN[written] + 4):
        assert lib.buddy_page_plan(_plan(**{written: where}), None, None) == 1, where - A

