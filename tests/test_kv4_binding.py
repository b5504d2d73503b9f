"""How the binding and the build get along with the compiled calls of the 4-bit cache."""
import importlib.metadata
import shutil
import subprocess
import sys

import pytest
import torch

from paper_2606_09514_gb300 import binding, build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


@pytest.fixture
def without_calls(monkeypatch):
    import paper_2606_09514_gb300 as pkg
    monkeypatch.setitem(sys.modules, "paper_2606_09514_gb300._calls", None)     # an import raises ImportError
    monkeypatch.delattr(pkg, "_calls", raising=False)


def test_the_library_loads_without_the_compiled_calls(without_calls):
    lib = binding.load_library(binding.LIB_PATH)
    assert lib.buddy_budget_to_k(0.5, 32) > 0


def test_the_cache_names_what_is_missing(without_calls, monkeypatch):
    monkeypatch.setattr(binding, "_lib", binding.load_library(binding.LIB_PATH))
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(RuntimeError, match="_calls"):
        binding.buddy_page_plan(z, z, 16, z.view(4, 1), z, z, z, z, z.long(), z, z)
    with pytest.raises(RuntimeError, match="_calls"):
        binding.buddy_qk_norm_rope(None, z, z, (z, z), None, z)


def test_the_compiled_calls_are_built_for_the_torch_that_is_there(monkeypatch, tmp_path):
    """Another version of torch builds them anew, the same one does not."""
    real_run, real_version, version, built = subprocess.run, importlib.metadata.version, [None], []

    def run(cmd, *a, **kw):
        if build.CALLS + ".tmp" not in cmd:
            return real_run(cmd, *a, **kw)
        built.append(version[0])
        shutil.copy(build.CALLS, build.CALLS + ".tmp")
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(importlib.metadata, "version",
                        lambda name: version[0] if name == "torch" and version[0] else real_version(name))
    monkeypatch.setattr(build, "CALLS_FOR", str(tmp_path / "for"), raising=False)
    for v in (None, None, "9.9.9", "9.9.9", None):
        version[0] = v
        build.build()
    assert built == [None, "9.9.9", None]
