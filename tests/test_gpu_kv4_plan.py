"""The page plan at the ends of its ranges."""
import pytest
import torch

from test_gpu_kv4 import flags, i32, pkg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_new,page", [(2 ** 31 - 1, 1), (5, 16)])
def test_plan_of_nearly_2_to_the_31_tokens(n_new, page):
    """As many slots as 32 bits count, all of them new tokens' (and as many pages), or nearly
    all of them behind the last token."""
    n_tok = 2 ** 31 - 1
    pages = -(-n_new // page)
    free = torch.arange(pages, device="cuda", dtype=torch.int32)
    table = torch.full((1, pages), -9, device="cuda", dtype=torch.int32)
    slot = torch.full((n_tok,), -9, device="cuda", dtype=torch.int64)
    pos = torch.full((n_tok,), -9, device="cuda", dtype=torch.int32)
    kv, rows, head, fl = i32([-9]), i32([-9, -9]), i32([-9]), flags()
    pkg().buddy_page_plan(i32([0]), i32([n_new]), page, table, free, i32([0]), kv, rows, slot, pos, head, fl)
    torch.cuda.synchronize()
    assert fl.item() == 0 and kv.item() == n_new and rows.tolist() == [0, n_new] and head.item() == pages
    assert torch.equal(table[0], free)
    step = 2 ** 27                                # (compared in pieces)
    for t0 in range(0, n_tok, step):
        t1 = min(n_tok, t0 + step)
        want = torch.arange(t0, t1, device="cuda")
        want[want >= n_new] = -1
        assert torch.equal(slot[t0:t1], want) and torch.equal(pos[t0:t1], want.int()), t0
    del slot, pos, table, free, want
    torch.cuda.empty_cache()
