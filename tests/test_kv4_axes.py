"""Position axes without a GPU: layouts, the C struct, and what the entries refuse."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2606_09514_gb300 as pkg
from oracle import kv4_oracle as O
from paper_2606_09514_gb300 import binding as B
from test_kv4_refusals import elsewhere, fake_cache, refused, rows

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "buddy.h")
fakes = [pytest.mark.skipif(torch.cuda.is_available(), reason="fake tensors of devices that are not there"),
         pytest.mark.filterwarnings("ignore")]


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2606_09514_gb300 import build
    build.build()
    return pkg.load_library()


def axis_of(hd, sections, interleaved=False):
    a = pkg.buddy_rope_axes(hd, sections, interleaved)
    assert a.head_dim == hd and a.n_axes == len(sections)
    return list(a.axis)[:hd // 2]


def test_sections():
    assert axis_of(128, (16, 24, 24)) == [0] * 16 + [1] * 24 + [2] * 24
    assert axis_of(64, (0, 32)) == [1] * 32
    assert axis_of(64, (32,)) == [0] * 32
    # in turn: 0 1 2 0 1 2 ... and what is left of the longest
    assert axis_of(128, (24, 20, 20), True) == [0, 1, 2] * 20 + [0] * 4
    assert axis_of(64, (2, 30), True) == [0, 1, 0, 1] + [1] * 28


@pytest.mark.parametrize("hd,sections", [(64, (8, 12)), (64, ()), (64, (33, -1)), (64, (8, 8, 8, 4, 4)), (96, (16, 32)),
                                         (128, (16, 24, 25))])
def test_sections_that_are_not_a_heads(hd, sections):
    with pytest.raises(ValueError):
        pkg.buddy_rope_axes(hd, sections)


def test_oracle_turns_by_axis():
    rng = np.random.default_rng(0)
    x, pos = rng.standard_normal((3, 2, 64)), np.array([[0, 5, 9], [3, 5, 1]])
    axis = [0] * 10 + [1] * 22
    y = O.norm_rope_axes(x, None, pos, axis, 1e4, 1e-6)
    z = torch.complex(torch.tensor(x[..., :32]), torch.tensor(x[..., 32:]))
    angle = torch.tensor([[float(pos[axis[j], t]) * 1e4 ** (-j / 32) for j in range(32)] for t in range(3)])[:, None]
    z = z * torch.polar(torch.ones_like(angle), angle)
    np.testing.assert_allclose(y, torch.cat([z.real, z.imag], -1).numpy(), rtol=1e-5, atol=1e-5)
    same = np.array([[4, 5, 9]] * 2)
    np.testing.assert_array_equal(O.norm_rope_axes(x, None, same, axis, 1e4, 1e-6), O.norm_rope(x, None, same[0], 1e4, 1e-6))


def test_struct_matches_the_header(tmp_path):
    src = tmp_path / "l.c"
    fields = [f for f, _ in B.RopeAxes._fields_[:-1]]
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "{HEADER}"\nint main(void){{'
                   + "".join(f'printf("%zu ", offsetof(buddy_rope_axes, {f}));' for f in fields)
                   + 'printf("%zu", sizeof(buddy_rope_axes));return 0;}')
    subprocess.run(["gcc", "-o", tmp_path / "l", src], check=True)
    got = [int(x) for x in subprocess.run([tmp_path / "l"], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(B.RopeAxes, f).offset for f in fields] + [B.RopeAxes.head_dim.offset]


def test_entries_refuse(lib):
    """Before any CUDA call: the addresses are made up and not read."""
    p = 0x10000
    r = B.buddy_qk_rows(4, 6, 2, 64, 1, 8, 1e-6, p, p, 1024, 1024, None, None, p, p, p, p, p, 1024, 1024)
    cache = B.buddy_kv4_cache(p, p, 3, 16, 2, 64)
    good = pkg.buddy_rope_axes(64, (8, 12, 12))

    def both(axes, rows=r, c=cache):
        ref = None if axes is None else ctypes.byref(axes)
        return {lib.buddy_qk_norm_rope_axes(ctypes.byref(rows), ref, None, None),
                lib.buddy_kv4_append_axes(ctypes.byref(c), ctypes.byref(rows), ref, p, 1024, p, None, None)}

    assert both(None) == {B.BUDDY_ERR_ARG}
    for n_axes, stride, j, axis in ((0, 4, 0, 0), (5, 4, 0, 0), (3, -1, 0, 0), (3, 4, 31, 3), (2, 4, 31, 2)):
        bad = B.RopeAxes.from_buffer_copy(good)
        bad.n_axes, bad.pos_stride, bad.axis[j] = n_axes, stride, axis
        assert both(bad) == {B.BUDDY_ERR_ARG}, (n_axes, stride, j, axis)
    wrong_rows = B.buddy_qk_rows.from_buffer_copy(r)
    wrong_rows.head_dim = 96
    assert both(good, wrong_rows) == {B.BUDDY_ERR_ARG}
    assert lib.buddy_kv4_append_axes(ctypes.byref(cache), ctypes.byref(r), ctypes.byref(good), p + 4, 1024, p, None,
                                     None) == B.BUDDY_ERR_ARG


class TestFakes:
    pytestmark = fakes

    def good(self, hd=64):
        t = rows(hd)
        t.update(pos=torch.empty(3, 4, dtype=torch.int32, device="cuda:0"), axes=pkg.buddy_rope_axes(hd, (hd // 4, hd // 8, hd // 8)))
        return t

    def test_positions(self):
        with FakeTensorMode():
            i32 = dict(dtype=torch.int32, device="cuda:0")
            for bad in (torch.empty(4, **i32), torch.empty(2, 4, **i32), torch.empty(4, 3, **i32), torch.empty(3, 5, **i32),
                        torch.empty(4, 3, **i32).t(), torch.empty(3, 4, device="cuda:0"), torch.empty(1, 3, 4, **i32),
                        torch.empty(3, 8, **i32)[:, ::2]):
                refused(pkg.buddy_qk_norm_rope, self.good(), "pos", bad, "pos")

    def test_axes_of_another_head(self):
        with FakeTensorMode():
            refused(pkg.buddy_qk_norm_rope, self.good(), "axes", pkg.buddy_rope_axes(128, (16, 24, 24)), "axes")
            with pytest.raises(TypeError, match="axes"):
                pkg.buddy_qk_norm_rope(**{**self.good(), "axes": (8, 12, 12)})

    def test_one_device(self):
        with FakeTensorMode():
            good = self.good()
            elsewhere(pkg.buddy_qk_norm_rope, good, "k")
            good.update(v=torch.empty(4, 2, 64, device="cuda:0"), slot=torch.empty(4, dtype=torch.int64, device="cuda:0"))
            elsewhere(fake_cache().buddy_kv4_append, good, "k")
            refused(fake_cache("cuda:1").buddy_kv4_append, good, "flags", good["flags"], "device")
