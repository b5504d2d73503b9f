"""CPU checks of the CUDA sources for faults that no GPU run may be made to show."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2606_09514_gb300" / "csrc"


def code(path):
    """The file without comments."""
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", path.read_text(), flags=re.S)


def kernels(text):
    """(name, body) of each kernel."""
    for m in re.finditer(r"__global__", text):
        end = text.index("{", text.index(")", re.compile(r"\b\w+_kernel\s*\(").search(text, m.start()).end()))
        depth, at = 1, end + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield re.search(r"(\w+_kernel)\s*\(", text[m.start():end]).group(1), text[end:at]


def remote_kernels():
    for f in sorted(CSRC.glob("*.cu")):
        for name, body in kernels(code(f)):
            if "dsmem_addr" in body:
                yield pytest.param(body, id=name)


# A CTA's shared memory may be accessed by its cluster only once it has started:
# a cluster barrier comes before the first access.
@pytest.mark.parametrize("body", list(remote_kernels()))
def test_cluster_barrier_before_remote_shared_memory(body):
    before = body[:body.index("dsmem_addr")]
    started = "cluster_arrive_started" in before and "cluster_wait_started" in before
    assert started or "cluster_sync" in before


def test_remote_kernels_are_found():
    assert {p.id for p in remote_kernels()} == {"attn_cl_kernel", "gemm_pf_kernel", "pool_refresh_kernel"}


# What a function keeps between calls would be shared by contexts on other devices and
# by host threads: only constants may be static in a function.
def test_no_state_kept_in_functions():
    found = [f"{f.name}: {line.strip()}" for f in sorted(CSRC.glob("*.cu*")) + sorted(CSRC.glob("*.h"))
             for line in code(f).splitlines() if re.match(r"\s+static\s+(?!const\b|constexpr\b)", line)]
    assert not found


# The active mask says which lanes happen to be together, not which have to take part: after
# waits that lanes end one by one it may hold some of them.
def test_no_warp_intrinsic_goes_by_the_active_mask():
    found = [f.name for f in sorted(CSRC.glob("*.cu*")) if "__activemask" in code(f)]
    assert not found


# A commit follows the MMAs of the thread that makes it: where an elected thread issues
# them, lane 0 need not be that thread.
@pytest.mark.parametrize("path", [pytest.param(f, id=f.name) for f in sorted(CSRC.glob("*.cu"))
                                  if "mma_commit" in f.read_text() and "elect_one()" in f.read_text()])
def test_commits_are_made_by_the_thread_that_issues(path):
    text = code(path)
    for m in re.finditer(r"mma_commit", text):
        before = text[:m.start()]
        assert before.rfind("elect_one()") > before.rfind("lane == 0"), text[m.start() - 80:m.end() + 20]


# setmaxnreg.inc takes from what the block was launched with and waits for ever for more: the
# host compares the kernel's registers with what its roles ask for before it launches it.
def test_register_splits_are_checked_before_the_launch():
    for f in sorted(CSRC.glob("*.cu")):
        text = code(f)
        if "setmaxnreg.inc" in text:
            assert "numRegs" in text and "static_assert" in text, f.name


# Queries and keys may be turned in place: their rows are not read through the path of data
# that no one writes while the kernel runs.
def test_rows_that_may_be_written_are_read_by_ordinary_loads():
    text = code(CSRC / "kv4_rows.cu")
    loaders = re.findall(r"struct Raw8<\w+> \{.*?\n\};", text, flags=re.S)
    assert len(loaders) == 2 and not any(re.search(r"__ldg|\.nc\b", x) for x in loaders)
