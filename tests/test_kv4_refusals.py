"""What the 4-bit cache's calls refuse of CUDA tensors, shown without a GPU: fake tensors have
a type, a device and a shape, and a refused call gets no further."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2606_09514_gb300 as pkg

pytestmark = [pytest.mark.skipif(torch.cuda.is_available(), reason="fake tensors of devices that are not there"),
              pytest.mark.filterwarnings("ignore")]


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2606_09514_gb300 import build
    build.build()


def rows(hd=64, device="cuda:0"):
    t = dict(device=device)
    return dict(q=torch.empty(4, 6, hd, **t), k=torch.empty(4, 2, hd, **t), pos=torch.empty(4, dtype=torch.int32, **t),
                rope=(torch.empty(8, hd // 2, **t), torch.empty(8, hd // 2, **t)), q_out=torch.empty(4, 6, hd, **t),
                k_out=torch.empty(4, 2, hd, **t), q_gain=torch.empty(hd, **t), k_gain=torch.empty(hd, **t),
                flags=torch.empty(1, dtype=torch.int32, **t))


def refused(call, good, name, value, match):
    with pytest.raises(ValueError, match=match):
        call(**{**good, name: value})


@pytest.mark.parametrize("hd", [64, 128])
def test_rotary_tables_of_another_layout(hd):
    """Tables with both halves [positions, head_dim], flat, transposed ones, or of different lengths would be
    read in bounds and turn every head by another token's angles."""
    with FakeTensorMode():
        good = rows(hd)
        co, si = good["rope"]
        both = torch.empty(8, hd, device="cuda:0")
        flat = torch.empty(8 * hd // 2, device="cuda:0")
        more = torch.empty(9, hd // 2, device="cuda:0")
        turned = torch.empty(hd // 2, 8, device="cuda:0")
        deep = torch.empty(8, 1, hd // 2, device="cuda:0")
        for bad in (both, flat, turned, deep, torch.empty(16, hd // 4, device="cuda:0")):
            refused(pkg.buddy_qk_norm_rope, good, "rope", (bad, si), "cos")
            refused(pkg.buddy_qk_norm_rope, good, "rope", (co, bad), "sin")
            refused(pkg.buddy_qk_norm_rope, good, "rope", (bad, bad), "cos")
        refused(pkg.buddy_qk_norm_rope, good, "rope", (co, more), "sin")
        refused(pkg.buddy_qk_norm_rope, good, "rope", (more, si), "sin")


# ------------------------------------------------------------------ devices
# The library launches where the call's tensors are: one that is elsewhere is refused.
def elsewhere(call, good, first, **names):
    """Every tensor of a call but its first on another device."""
    for name, value in good.items():
        if name == first or not isinstance(value, torch.Tensor):
            continue
        other = torch.empty_strided(value.size(), value.stride(), dtype=value.dtype, device="cuda:1")
        refused(call, good, name, other, f"{names.get(name, name)}.*device")


def test_row_calls_want_one_device():
    with FakeTensorMode():
        good = rows()
        elsewhere(pkg.buddy_qk_norm_rope, good, "k")
        for k, name in ((0, "cos"), (1, "sin")):
            rope = list(good["rope"])
            rope[k] = torch.empty(8, 32, device="cuda:1")
            refused(pkg.buddy_qk_norm_rope, good, "rope", tuple(rope), f"{name}.*device")
        cache = fake_cache()
        good.update(v=torch.empty(4, 2, 64, device="cuda:0"), slot=torch.empty(4, dtype=torch.int64, device="cuda:0"))
        elsewhere(cache.buddy_kv4_append, good, "k")
        refused(fake_cache("cuda:1").buddy_kv4_append, good, "flags", good["flags"], "device")


def fake_cache(device="cuda:0"):
    return pkg.KV4Cache(*(torch.empty(3, 2, 16 * 36, dtype=torch.uint8, device=device) for _ in range(2)), 16)


def test_plan_wants_one_device():
    i32 = dict(dtype=torch.int32, device="cuda:0")
    with FakeTensorMode():
        good = dict(slot=torch.empty(3, dtype=torch.int64, device="cuda:0"), length=torch.empty(2, **i32),
                    n_new=torch.empty(2, **i32), page_size=16, table=torch.empty(2, 4, **i32),
                    free_pages=torch.empty(8, **i32), free_head=torch.empty(1, **i32), kv_len=torch.empty(2, **i32),
                    row_start=torch.empty(3, **i32), pos=torch.empty(3, **i32), free_head_out=torch.empty(1, **i32),
                    flags=torch.empty(1, **i32))
        elsewhere(pkg.buddy_page_plan, good, "slot")


def test_read_and_attention_want_one_device():
    with FakeTensorMode():
        t = dict(device="cuda:0")
        cache = fake_cache()
        out = torch.empty(3, 2, 64, **t)
        read = dict(slot=torch.empty(3, dtype=torch.int64, **t), k_out=out, v_out=out,
                    flags=torch.empty(1, dtype=torch.int32, **t))
        elsewhere(cache.buddy_kv4_read, read, None, slot="(slot|pages)")
        i32 = dict(dtype=torch.int32, **t)
        att = dict(q=torch.empty(3, 4, 64, **t), kv_len=torch.empty(3, **i32), table=torch.empty(3, 2, **i32),
                   out=torch.empty(3, 4, 64, **t), row_start=torch.empty(4, **i32), flags=torch.empty(1, **i32),
                   workspace=torch.empty(4096, dtype=torch.uint8, **t))
        elsewhere(cache.buddy_kv4_attention, att, None, q="(q|pages)")


def test_pages_are_on_one_device():
    with FakeTensorMode():
        k, v = (torch.empty(3, 2, 16 * 36, dtype=torch.uint8, device=d) for d in ("cuda:0", "cuda:1"))
        with pytest.raises(ValueError, match="v_pages.*device"):
            pkg.KV4Cache(k, v, 16)
