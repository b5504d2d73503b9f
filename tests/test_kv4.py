"""The paged 4-bit cache without a GPU: the oracle's pins, the C structs, and what
the entries refuse before any CUDA call."""
import ctypes
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2606_09514_gb300 import build as b
    b.build()
    import paper_2606_09514_gb300 as pkg
    return pkg.load_library()


# ------------------------------------------------------------------ oracle pins
def test_scale_has_seven_bits_and_codes_are_nearest():
    rng = np.random.default_rng(0)
    for mag in (1e-8, 1e-4, 1.0, 300.0, 6000.0):
        x = rng.standard_normal((50, 64)) * mag
        codes, s = O.quantise(x)
        assert codes.min() >= 1 and codes.max() <= 15
        m, _ = np.frexp(s[s > 0])
        assert np.all(m * 128 == np.round(m * 128))
        if mag >= 1e-4:   # f16's normal range: the largest code is used, nothing is off by more than half a step
            err = np.abs(O.values(codes, s) - x)
            fine = np.repeat(s, 32, -1) < O.MAX_SCALE
            assert np.all((err <= np.repeat(s, 32, -1) * 0.5 + 1e-12)[fine])
            assert np.all(np.abs(codes - 8).reshape(50, 2, 32).max(-1) == 7)


def test_special_groups():
    x = np.zeros((4, 32))
    x[1, 3] = np.nan
    x[2, 5] = np.inf
    x[3] = 2.0 ** -30
    codes, s = O.quantise(x)
    assert s[0, 0] == 0 and np.all(codes[0] == 8)
    assert np.isnan(s[1, 0])
    assert s[2, 0] == 896 and codes[2, 5] == 15
    assert s[3, 0] == 0 and np.all(codes[3] == 8)      # below half's smallest step


@pytest.mark.parametrize("page,hd", [(16, 64), (64, 128)])
def test_pack_and_unpack_are_inverse(page, hd):
    rng = np.random.default_rng(1)
    codes = rng.integers(0, 16, (3, 2, page, hd))
    s = rng.integers(64, 128, (3, 2, page, hd // 32)) / 256.0
    b = O.blocks(codes, s)
    assert b.shape == (3, 2, page * (hd // 2 + hd // 16))
    np.testing.assert_array_equal(O.entries(b, page, hd), O.values(codes, s))
    # channel 0 is the lowest nibble of the first byte, channel 1 the lowest of the third
    assert np.all((b[0, 0, 0] & 15) == codes[0, 0, 0, 0]) and np.all((b[0, 0, 2] & 15) == codes[0, 0, 0, 1])


def test_attention_is_torch_softmax():
    rng = np.random.default_rng(2)
    q, k, v = (rng.standard_normal(s) for s in ((3, 6, 64), (2, 10, 64), (2, 10, 64)))
    got = O.attention(q, k, v, 3, 0.125)
    mask = torch.ones(3, 10, dtype=torch.bool).tril(7)
    want = torch.nn.functional.scaled_dot_product_attention(
        torch.tensor(q).transpose(0, 1), torch.tensor(k).repeat_interleave(3, 0), torch.tensor(v).repeat_interleave(3, 0),
        attn_mask=mask, scale=0.125).transpose(0, 1)
    np.testing.assert_allclose(got, want.numpy(), rtol=1e-12, atol=1e-13)
    assert np.all(O.attention(q, k[:, :0], v[:, :0], 3, 0.125) == 0)


def test_norm_rope_is_torch():
    rng = np.random.default_rng(3)
    x, g, pos = rng.standard_normal((4, 3, 64)), rng.uniform(0.5, 1.5, 64), np.array([0, 1, 77, 5000])
    y = torch.nn.functional.rms_norm(torch.tensor(x), (64,), torch.tensor(g), 1e-5).numpy()
    f = 1e4 ** (-np.arange(32) / 32)
    z = (y[..., :32] + 1j * y[..., 32:]) * np.exp(1j * pos[:, None, None] * f)
    np.testing.assert_allclose(O.norm_rope(x, g, pos, 1e4, 1e-5), np.concatenate([z.real, z.imag], -1), atol=1e-12)


def test_plan_of_a_known_case():
    table, kv, rows, slot, pos, head = O.page_plan([0, 3, 4], [2, 1, 5], 4, -np.ones((3, 4), int), [9, 8, 7, 6], 0)
    assert list(kv) == [2, 4, 9] and list(rows) == [0, 2, 3, 8] and head == 3
    assert table[0, 0] == 9 and table[1, 0] == -1 and list(table[2]) == [-1, 8, 7, -1]
    assert list(slot) == [36, 37, -1 * 4 + 3, 32, 33, 34, 35, 28] and list(pos) == [0, 1, 3, 4, 5, 6, 7, 8]


# ------------------------------------------------------------------ C boundary
def test_ctypes_structs_match_c_layout():
    from paper_2606_09514_gb300 import binding as B
    header = os.path.join(ROOT, "include", "buddy.h")
    names = ("buddy_kv4_cache", "buddy_page_plan_args", "buddy_qk_rows", "buddy_kv4_attention_args")
    lines = ["#include <stdio.h>", "#include <stddef.h>", f'#include "{header}"', "int main(void){"]
    for n in names:
        lines.append(f'printf("{n} %zu\\n", sizeof({n}));')
        lines += [f'printf("{n}.{f} %zu\\n", offsetof({n}, {f}));' for f, _ in getattr(B, n)._fields_]
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "l.c"), os.path.join(d, "l")
        open(src, "w").write("\n".join(lines + ["return 0;}"]))
        subprocess.run(["gcc", "-o", exe, src], check=True)
        out = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split("\n")
    got = dict(x.split() for x in out if x)
    for n in names:
        cls = getattr(B, n)
        assert int(got[n]) == ctypes.sizeof(cls), n
        for f, _ in cls._fields_:
            assert int(got[f"{n}.{f}"]) == getattr(cls, f).offset, (n, f)


A = 0x100000   # made-up device addresses: every call below is refused before they are used


def _cache(**kw):
    from paper_2606_09514_gb300 import binding as B
    return B.buddy_kv4_cache(**{**dict(k_pages=A, v_pages=A, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64), **kw})


def _plan(**kw):
    from paper_2606_09514_gb300 import binding as B
    good = dict(batch=2, page_size=16, max_pages=4, n_free=4, n_tok=2, len=A, n_new=A + 64, table=A + 128,
                free_pages=A + 256, free_head=A + 512, kv_len=A + 576, row_start=A + 640, slot=A + 704, pos=A + 768,
                free_head_out=A + 832)
    return B.buddy_page_plan_args(**{**good, **kw})


def _rows(**kw):
    from paper_2606_09514_gb300 import binding as B
    good = dict(n_tok=2, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=1, max_pos=64, eps=1e-6, q=A, k=A, q_stride=256,
                k_stride=128, q_gain=A, k_gain=A, pos=A, rope_cos=A, rope_sin=A, q_out=A, k_out=A, q_out_stride=256,
                k_out_stride=128)
    return B.buddy_qk_rows(**{**good, **kw})


def _attn(**kw):
    from paper_2606_09514_gb300 import binding as B
    good = dict(batch=2, n_tok=2, max_new=1, n_q_heads=4, q_dtype=1, out_dtype=1, max_pages=4, scale=0.0, q=A, out=A + 4096,
                q_stride=256, out_stride=256, row_start=None, kv_len=A, table=A, workspace=A, workspace_bytes=1 << 40)
    return B.buddy_kv4_attention_args(**{**good, **kw})


BAD_CACHE = [dict(k_pages=None), dict(v_pages=None), dict(k_pages=A + 8), dict(n_pages=0), dict(page_size=8),
             dict(page_size=48), dict(page_size=256), dict(n_kv_heads=0), dict(head_dim=96), dict(n_kv_heads=2000)]


@pytest.mark.parametrize("bad", [dict(batch=0), dict(batch=20000), dict(page_size=0), dict(page_size=24),
                                 dict(max_pages=0), dict(n_free=-1), dict(n_tok=-1), dict(len=None), dict(n_new=None),
                                 dict(table=None), dict(free_pages=None), dict(free_head=None), dict(kv_len=None),
                                 dict(row_start=None), dict(slot=None), dict(pos=None), dict(free_head_out=None),
                                 dict(kv_len=A), dict(kv_len=A + 64), dict(free_head_out=A + 512)])
def test_plan_refuses(lib, bad):
    assert lib.buddy_page_plan(_plan(**bad), None, None) == 1


BAD_ROWS = [dict(n_tok=-1), dict(n_q_heads=-1), dict(n_kv_heads=0), dict(head_dim=80), dict(dtype=2), dict(dtype=-1),
            dict(max_pos=0), dict(eps=0.0), dict(eps=float("nan")), dict(q=None), dict(k=None), dict(q=A + 2),
            dict(k=A + 8), dict(q_stride=257), dict(k_stride=132), dict(q_gain=A + 4), dict(k_gain=A + 4), dict(pos=None),
            dict(rope_cos=None), dict(rope_sin=A + 4), dict(q_out=None), dict(q_out_stride=4), dict(k_out=A + 2)]


@pytest.mark.parametrize("bad", BAD_ROWS + [dict(k_out=None)])
def test_norm_refuses(lib, bad):
    assert lib.buddy_qk_norm_rope(_rows(**bad), None, None) == 1


@pytest.mark.parametrize("bad", BAD_ROWS + [dict(n_kv_heads=1), dict(head_dim=128)])
def test_append_refuses_rows(lib, bad):
    assert lib.buddy_kv4_append(_cache(), _rows(**bad), A, 128, A, None, None) == 1


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_cache_refused_everywhere(lib, bad):
    c = _cache(**bad)
    assert lib.buddy_kv4_append(c, _rows(), A, 128, A, None, None) == 1
    assert lib.buddy_kv4_read(c, 1, A, 0, A, A, None, None) == 1
    assert lib.buddy_kv4_attention(c, _attn(), None, None) == 1


def test_append_and_read_refuse_the_rest(lib):
    assert lib.buddy_kv4_append(_cache(), _rows(), None, 128, A, None, None) == 1
    assert lib.buddy_kv4_append(_cache(), _rows(), A + 2, 128, A, None, None) == 1
    assert lib.buddy_kv4_append(_cache(), _rows(), A, 129, A, None, None) == 1
    assert lib.buddy_kv4_append(_cache(), _rows(), A, 128, None, None, None) == 1
    assert lib.buddy_kv4_read(_cache(), -1, A, 0, A, A, None, None) == 1
    assert lib.buddy_kv4_read(_cache(), 1, None, 0, A, A, None, None) == 1
    assert lib.buddy_kv4_read(_cache(), 1, A, 3, A, A, None, None) == 1
    assert lib.buddy_kv4_read(_cache(), 1, A, 0, A + 4, A, None, None) == 1
    assert lib.buddy_kv4_read(_cache(), 0, None, 0, A, A, None, None) == 0
    assert lib.buddy_rope_table(None, A, 8, 64, 1e4, None) == 1
    assert lib.buddy_rope_table(A, A, 0, 64, 1e4, None) == 1
    assert lib.buddy_rope_table(A, A, 8, 32, 1e4, None) == 1
    assert lib.buddy_rope_table(A, A, 8, 64, -1.0, None) == 1


@pytest.mark.parametrize("bad", [dict(batch=0), dict(batch=20000), dict(n_tok=-1), dict(max_new=0), dict(n_q_heads=3),
                                 dict(n_q_heads=0), dict(n_q_heads=18), dict(q_dtype=2), dict(out_dtype=-1),
                                 dict(max_pages=0), dict(max_pages=1 << 28), dict(scale=-1.0), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(q=None), dict(out=None), dict(q=A + 4), dict(out=A + 2),
                                 dict(q_stride=250), dict(out_stride=1), dict(kv_len=None), dict(table=None),
                                 dict(workspace=None), dict(workspace=A + 16), dict(workspace_bytes=0), dict(n_tok=3),
                                 dict(max_new=2)])
def test_attention_refuses(lib, bad):
    assert lib.buddy_kv4_attention(_cache(), _attn(**bad), None, None) == 1


def test_workspace_of_refused_sizes(lib):
    assert lib.buddy_kv4_attention_workspace(3, 2, 64, 1) == -1
    assert lib.buddy_kv4_attention_workspace(4, 2, 72, 1) == -1
    assert lib.buddy_kv4_attention_workspace(4, 2, 64, 0) == -1


def test_binding_refuses_tensors_on_the_host(lib):
    import paper_2606_09514_gb300 as pkg
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        pkg.buddy_page_plan(z, z, 16, z.view(4, 1), z, z, z, z, z.long(), z, z)
    x = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):
        pkg.buddy_qk_norm_rope(x, x, z, (x[0], x[0]), x, x)
    with pytest.raises(ValueError):
        pkg.KV4Cache(torch.zeros(2, 2, 576, dtype=torch.uint8), torch.zeros(2, 2, 576, dtype=torch.uint8), 16)
