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
