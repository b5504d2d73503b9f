"""Attention over selected pages without a GPU: the oracle's pins, the C structs, and what the
entries refuse."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2606_09514_gb300 as pkg
from oracle import kv4_oracle as O
from paper_2606_09514_gb300 import binding as B
from test_kv4_refusals import elsewhere, fake_cache, refused

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "buddy.h")
P = 0x10000          # an address that is not read


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2606_09514_gb300 import build
    build.build()
    return pkg.load_library()


# ------------------------------------------------------------------ oracle pins
def test_scores_are_the_formula():
    rng = np.random.default_rng(0)
    q, lo = rng.standard_normal((6, 128)), rng.standard_normal((9, 2, 1, 128))
    bounds = np.concatenate([lo, lo + rng.random((9, 2, 1, 128))], 2)
    got = O.page_scores(q, bounds)
    for g in range(2):
        for n in range(9):
            want = sum(max(x * a, x * b) for row in q[3 * g:3 * g + 3] for x, a, b in zip(row, *bounds[n, g]))
            assert abs(got[g, n] - want) < 1e-3 * max(1.0, abs(want))


def test_scores_bound_the_products():
    rng = np.random.default_rng(1)
    keys, q = rng.standard_normal((4, 2, 16, 64)), rng.standard_normal((4, 64))
    score = O.page_scores(q, O.page_bounds(keys, 16, 64))
    for g in range(2):
        s = np.einsum("hd,npd->hnp", q[2 * g:2 * g + 2], keys[:, g])
        assert np.all(s.max(-1).sum(0) <= score[g] + 1e-4)


def test_bounds_stop_at_the_end():
    keys = np.zeros((2, 1, 16, 64))
    keys[1, 0, 3], keys[1, 0, 4] = 5.0, -7.0
    assert O.page_bounds(keys, 16, 20)[1].max() == 5 and O.page_bounds(keys, 16, 20)[1].min() == 0
    assert O.page_bounds(keys, 16, 21)[1].min() == -7


def test_the_order_of_a_sum():
    """Halves inside eight neighbours, then over the eights: not from left to right."""
    x = np.zeros(64, np.float32)
    x[0], x[4], x[1] = 2.0 ** 24, -2.0 ** 24, 1.0       # (0 + 4) first: the one is not lost
    assert O._eights(x) == 1
    x[4], x[32] = 0, -2.0 ** 24                          # eights 0 and 4 first, after the one was lost
    assert O._eights(x) == 0


def test_selection():
    s = [0.0, 3.0, 1.0, 3.0, np.nan, None, 2.0, 9.0]
    assert O.select(s, 8, 1, 1) == list(range(8))
    assert O.select(s, 3, 1, 1) == [0, 4, 7]
    assert O.select(s, 4, 1, 1) == [0, 1, 4, 7]          # of two threes the first
    assert O.select(s, 5, 0, 1) == [1, 3, 4, 6, 7]
    assert O.select(s, 7, 1, 1) == [0, 1, 2, 3, 4, 6, 7]
    assert O.select(s, 3, 1, 2) == [0, 6, 7]


# ------------------------------------------------------------------ the C ABI
def test_structs_match_the_header(tmp_path):
    src = tmp_path / "l.c"
    structs = {"buddy_kv4_seqs": B.buddy_kv4_seqs, "buddy_kv4_select_args": B.buddy_kv4_select_args}
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "{HEADER}"\nint main(void){{' + "".join(
        f'printf("%zu ", sizeof({n}));' + "".join(f'printf("%zu ", offsetof({n}, {f}));' for f, _ in c._fields_)
        for n, c in structs.items()) + "return 0;}")
    subprocess.run(["gcc", "-o", tmp_path / "l", src], check=True)
    got = [int(x) for x in subprocess.run([tmp_path / "l"], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for c in structs.values():
        want += [ctypes.sizeof(c)] + [getattr(c, f).offset for f, _ in c._fields_]
    assert got == want


def cache():
    return B.buddy_kv4_cache(P, P, 3, 16, 2, 64)


def seqs(**kw):
    return B.buddy_kv4_seqs(**{**dict(batch=4, n_tok=4, max_new=1, max_pages=8, row_start=None, kv_len=P, table=P), **kw})


BAD_SEQS = [dict(batch=0), dict(batch=16385), dict(n_tok=-1), dict(max_new=0), dict(max_pages=0), dict(max_pages=2 ** 27),
            dict(kv_len=None), dict(table=None), dict(n_tok=5), dict(max_new=2)]


@pytest.mark.parametrize("bad", BAD_SEQS + [dict(bounds=None), dict(bounds=P + 2), dict(page_size=24), dict(head_dim=96)])
def test_bounds_refuse(lib, bad):
    c, at = cache(), bad.get("bounds", P)
    for f in ("page_size", "head_dim"):
        setattr(c, f, bad.get(f, getattr(c, f)))
    s = seqs(**{k: v for k, v in bad.items() if k not in ("bounds", "page_size", "head_dim")})
    assert lib.buddy_kv4_bounds(ctypes.byref(c), ctypes.byref(s), at, None, None) == B.BUDDY_ERR_ARG
    assert lib.buddy_kv4_bounds(None, ctypes.byref(seqs()), P, None, None) == B.BUDDY_ERR_ARG
    assert lib.buddy_kv4_bounds(ctypes.byref(cache()), None, P, None, None) == B.BUDDY_ERR_ARG


@pytest.mark.parametrize("bad", [dict(s=seqs(**b)) for b in BAD_SEQS] + [
    dict(n_q_heads=1), dict(n_q_heads=5), dict(n_q_heads=18), dict(q_dtype=2), dict(budget=1), dict(first=-1), dict(last=0),
    dict(first=2 ** 31 - 1, last=2), dict(q=None), dict(q=P + 8), dict(q_stride=257), dict(bounds=None), dict(bounds=P + 8),
    dict(pages=None), dict(visible=None), dict(s=seqs(max_pages=40001))])
def test_select_refuses(lib, bad):
    good = dict(s=seqs(), n_q_heads=4, q_dtype=1, budget=4, first=1, last=1, q=P, q_stride=256, bounds=P, pages=P, visible=P)
    a = B.buddy_kv4_select_args(**{**good, **bad})
    want = B.BUDDY_ERR_RANGE if a.s.max_pages == 40001 else B.BUDDY_ERR_ARG
    assert lib.buddy_kv4_select(ctypes.byref(cache()), ctypes.byref(a), None, None) == want
    assert lib.buddy_kv4_select(ctypes.byref(cache()), None, None, None) == B.BUDDY_ERR_ARG


@pytest.mark.parametrize("bad", [dict(row_start=P), dict(max_new=2), dict(n_tok=3), dict(batch=-1), dict(batch=16385, n_tok=16385),
                                 dict(workspace_bytes=100), dict(kv_len=None), dict(table=None), dict(max_pages=2 ** 27), dict(q=P + 8), dict(out_stride=250)])
def test_attention_refuses(lib, bad):
    good = dict(batch=4, n_tok=4, max_new=1, n_q_heads=4, q_dtype=1, out_dtype=1, max_pages=4, scale=0.0, q=P, out=P,
                q_stride=256, out_stride=256, row_start=None, kv_len=P, table=P, workspace=P, workspace_bytes=1 << 30)
    a = B.buddy_kv4_attention_args(**{**good, **bad})
    assert lib.buddy_kv4_attention_pages(ctypes.byref(cache()), ctypes.byref(a), None, None) == B.BUDDY_ERR_ARG
    none = B.buddy_kv4_attention_args(**{**good, "batch": 0, "n_tok": 0, "kv_len": None, "table": None})
    assert lib.buddy_kv4_attention_pages(ctypes.byref(cache()), ctypes.byref(none), None, None) == B.BUDDY_OK


# ------------------------------------------------------------------ tensors
@pytest.mark.skipif(torch.cuda.is_available(), reason="fake tensors of devices that are not there")
@pytest.mark.filterwarnings("ignore")
class TestFakes:
    def good(self):
        t = dict(device="cuda:0")
        i32 = dict(dtype=torch.int32, **t)
        q = torch.empty(5, 4, 64, **t)
        seq = dict(kv_len=torch.empty(3, **i32), table=torch.empty(3, 7, **i32), row_start=torch.empty(4, **i32),
                   flags=torch.empty(1, **i32))
        bounds = torch.empty(3, 2, 2, 64, dtype=torch.float16, **t)
        lists = dict(pages=torch.empty(5, 2, 4, **i32), visible=torch.empty(5, **i32))
        return {"buddy_kv4_bounds": dict(bounds=bounds, max_new=3, **seq),
                "buddy_kv4_select": dict(q=q, bounds=bounds, max_new=3, **seq, **lists),
                "buddy_kv4_attention_pages": dict(q=q, out=torch.empty_like(q), flags=seq["flags"],
                                                  workspace=torch.empty(4096, dtype=torch.uint8, **t), **lists)}

    def test_one_device(self):
        with FakeTensorMode():
            for name, good in self.good().items():
                elsewhere(getattr(fake_cache(), name), good, None)
                refused(getattr(fake_cache("cuda:1"), name), good, "flags", good["flags"], "device")

    def test_shapes_and_types(self):
        with FakeTensorMode():
            t = dict(device="cuda:0")
            i32 = dict(dtype=torch.int32, **t)
            half = dict(dtype=torch.float16, **t)
            bad = {"bounds": [torch.empty(3, 2, 2, 64, **t), torch.empty(3, 2, 2, 128, **half), torch.empty(4, 2, 2, 64, **half),
                              torch.empty(3, 2, 128, **half), torch.empty(3, 1, 2, 64, **half),
                              torch.empty(3, 2, 64, 2, **half).transpose(2, 3), torch.empty(3, 2, 2, 64, dtype=torch.float16)],
                   "kv_len": [torch.empty(3, dtype=torch.int64, **t), torch.empty(6, **i32)[::2]],
                   "table": [torch.empty(21, **i32), torch.empty(4, 7, **i32), torch.empty(7, 3, **i32).t()],
                   "row_start": [torch.empty(3, **i32), torch.empty(4, dtype=torch.int64, **t)],
                   "flags": [torch.empty(0, **i32), torch.empty(1, dtype=torch.uint8, **t)],
                   "q": [torch.empty(5, 256, **t), torch.empty(5, 4, 128, **t), torch.empty(5, 64, 4, **t).transpose(1, 2)],
                   "pages": [torch.empty(5, 8, **i32), torch.empty(4, 2, 4, **i32), torch.empty(5, 3, 4, **i32),
                             torch.empty(5, 2, 4, dtype=torch.int64, **t), torch.empty(5, 2, 8, **i32)[..., :4]],
                   "visible": [torch.empty(4, **i32), torch.empty(5, **t)],
                   "workspace": [torch.empty(4096, **i32)], "out": [torch.empty(5, 4, 128, **t), torch.empty(4, 4, 64, **t)]}
            for name, good in self.good().items():
                for arg in good:
                    for value in bad.get(arg, []):
                        refused(getattr(fake_cache(), name), good, arg, value, arg)

    def test_numbers(self):
        with FakeTensorMode():
            good = self.good()["buddy_kv4_select"]
            for arg in ("first", "last", "max_new"):
                with pytest.raises(OverflowError):
                    fake_cache().buddy_kv4_select(**{**good, arg: 2 ** 31})


def test_first_memory_is_reached_after_a_cluster_barrier():
    """The kernels that write to the first CTA of their cluster: it has started, and waits for them."""
    from test_kernel_sources import CSRC, code, kernels
    found = [body for name, body in kernels(code(CSRC / "kv4_pages.cu")) if "put_first" in body]
    assert len(found) == 1
    for body in found:
        first, last = body.index("put_first"), body.rindex("put_first")
        assert body.index("cluster_arrive_started") < body.index("cluster_wait_started") < first
        assert "cluster_sync" in body[last:]


def test_no_count_over_a_lists_entries_passes_32_bits():
    """A list may have 2^31 - 1 entries, and as many first and last pages: a signed counter that goes up to
    them in steps, or a product with the tokens, would pass 2^31, and the loop not end."""
    from test_kernel_sources import CSRC, code
    text = code(CSRC / "kv4_pages.cu")
    loops = re.findall(r"for \((\w+) (\w+) = [^;]*; \2 < ([^;]*); \2 \+= THREADS\)", text)
    assert any("budget" in end for _, _, end in loops) and any("ends" in end for _, _, end in loops)
    for kind, _, end in loops:
        if re.search(r"budget|first|last", end):
            assert kind in ("unsigned", "int64_t"), end
    assert re.search(r"int ends = min\(a\.first \+ a\.last, kSelMaxPages\);", text)
    assert int(re.search(r"kSelMaxPages = (\d+);", text).group(1)) * 4 + 256 < 2 ** 31
