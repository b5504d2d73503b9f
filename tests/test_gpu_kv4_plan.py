"""The page plan at the ends of its ranges."""
import pytest
import torch

from test_gpu_kv4 import flags, i32, make_plan, pkg, run_plan

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


def test_plan_takes_buffers_that_touch():
    """Every buffer of a call out of one allocation, one right behind the other."""
    length, n_new, page = [15, 0, 33], [3, 20, 1], 16
    want, _ = make_plan(length, n_new, page)
    run_plan(want, page)
    t, _ = make_plan(length, n_new, page)
    names = ["slot", "kv_len", "length", "table", "n_new", "row_start", "free", "pos", "head", "head_out"]
    words = [t[n].numel() * t[n].element_size() // 4 for n in names]
    buf, at = torch.zeros(sum(words), dtype=torch.int32, device="cuda"), 0
    for name, w in zip(names, words):
        x = buf[at:at + w].view(t[name].dtype).view(t[name].shape)
        x.copy_(t[name])
        t[name], at = x, at + w
    run_plan(t, page)
    assert all(torch.equal(t[n], want[n]) for n in names) and t["flags"].item() == 0


def test_plan_without_new_tokens_or_free_pages():
    t, _ = make_plan([15, 16], [0, 0], 16, n_tok=0)
    t["free"] = t["free"][:0]
    t["head"].zero_()
    got = run_plan(t, 16)
    assert got["flags"][0] == 0 and got["kv_len"].tolist() == [15, 16] and got["row_start"].tolist() == [0, 0, 0]
    assert got["head_out"][0] == 0
