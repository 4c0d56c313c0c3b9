"""The plan with a stack of free pages shorter than the pool: its entries and no others are dealt out,
whatever the count on the device says."""
import numpy as np
import pytest

from test_gpu_paged import EXHAUSTED, RANGE, cg, i32, torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("held,count,flags", [(3, 3, 0), (3, 2, EXHAUSTED), (3, 5, RANGE), (3, 40, RANGE), (3, 10 ** 6, RANGE),
                                              (0, 0, EXHAUSTED), (0, 7, RANGE | EXHAUSTED), (3, -1, RANGE | EXHAUSTED), (64, 50, 0)])
def test_a_stack_shorter_than_the_pool(held, count, flags):
    """Three pages wanted. Behind the stack's entries lie numbers that would pass for pages."""
    n_pages, n = 40, 48
    memory = i32(np.arange(64) % n_pages)
    stack = memory[:held]
    bt = torch.full((1, 4), -1, dtype=torch.int32, device="cuda")
    lens, cu, pos, left = i32([0]), i32([0, 0]), i32(np.zeros(n)), i32([77])
    slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    pages = cg.Pages(n_pages=n_pages, page=16, n_req=1, max_pages=4)
    cg.page_plan(pages, i32([0]), i32([n]), stack, i32([count]), bt, lens, cu, pos, slots, left)
    if held == 64:
        flags = RANGE           # a stack larger than the pool counts as one of n_pages
    assert cg.get_status() == flags
    have = max(0, min(count, held, n_pages))
    want = [have - 1 - k if k < have else -1 for k in range(3)]
    assert bt[0].tolist() == want + [-1] and left.item() == have - 3
    assert slots.tolist() == [want[t // 16] * 16 + t % 16 if want[t // 16] >= 0 else -1 for t in range(n)]


def test_an_empty_stack_without_memory():
    pages = cg.Pages(n_pages=4, page=16, n_req=1, max_pages=1)
    bt, lens, cu, pos, left = i32([[2]]), i32([0]), i32([0, 0]), i32([0]), i32([0])
    slots = torch.zeros(1, dtype=torch.int64, device="cuda")
    cg.page_plan(pages, i32([5]), i32([1]), torch.empty(0, dtype=torch.int32, device="cuda"), i32([0]), bt, lens, cu, pos, slots, left)
    assert cg.get_status() == 0 and slots.item() == 37 and left.item() == 0
