"""Release of requests whose block table holds entries that are no pages: those a program has given back
itself (a window's old pages, -1), those a plan could not fill (-1), and wrong ones."""
import numpy as np
import pytest

from test_gpu_paged import RANGE, _attend, _case, _check, cg, i32, torch

pytestmark = pytest.mark.gpu

PAD = -9


def _release(page, n_pages, lens, done, table, free, count=None):
    """The stack, its count and the lengths after a release; eight words behind the stack stay."""
    table = np.asarray(table)
    stack = i32(np.concatenate([free, np.full(n_pages - len(free) + 8, PAD)]))
    left, lens_left = i32([77]), i32(np.full(len(lens), 77))
    pages = cg.Pages(n_pages=n_pages, page=page, n_req=len(lens), max_pages=table.shape[1])
    cg.page_release(pages, i32(lens), i32(done), i32(table), stack, i32([len(free) if count is None else count]), lens_left, left)
    stack = stack.cpu().tolist()
    assert stack[n_pages:] == [PAD] * 8
    return stack[:n_pages], left.item(), lens_left.cpu().tolist()


@pytest.mark.parametrize("n_req,page,holes,wrong", [(1, 16, 0.5, 0.0), (60, 16, 0.3, 0.0), (60, 16, 1.0, 0.0), (700, 64, 0.2, 0.1),
                                                    (2048, 16, 0.9, 0.0), (4100, 32, 0.3, 0.05)])
def test_entries_that_are_no_pages(n_req, page, holes, wrong):
    rng = np.random.default_rng(n_req)
    lens = rng.integers(0, 40 * page, n_req)
    need = -(-lens // page)
    table = np.full((n_req, 43), -1)
    n_pages = int(need.sum()) + 50
    perm = rng.permutation(n_pages)
    table[np.arange(43) < need[:, None]] = perm[:need.sum()]
    table[rng.random(table.shape) < holes] = -1
    bad = (rng.random(table.shape) < wrong) & (np.arange(43) < need[:, None])
    table[bad] = rng.choice([n_pages, -2, 2 ** 31 - 1, -2 ** 31], bad.sum())
    done = (rng.random(n_req) < 0.5).astype(int)
    done[0] = 1
    free = perm[need.sum():]
    stack, left, lens_left = _release(page, n_pages, lens, done, table, free)
    back = [int(e) for i in range(n_req) if done[i] for e in table[i, :need[i]] if 0 <= e < n_pages]
    assert stack == list(free) + back + [PAD] * (n_pages - len(free) - len(back))
    assert left == len(free) + len(back)
    assert lens_left == [0 if f else int(x) for x, f in zip(lens, done)]
    assert cg.get_status() == (RANGE if (bad & (done[:, None] != 0)).any() else 0)


def test_long_lines():
    """More entries than the kernel takes at a time, holes among them, requests of very different size."""
    rng = np.random.default_rng(8)
    lens = np.array([0, 16 * 30000, 5, 16 * 2048, 16 * 9999 + 1, 0, 16 * 1])
    need = -(-lens // 16)
    n_pages = int(need.sum()) + 3
    table = np.full((7, 30001), -1)
    table[np.arange(30001) < need[:, None]] = rng.permutation(n_pages)[:need.sum()]
    table[rng.random(table.shape) < 0.1] = -1
    done = np.array([1, 1, 1, 0, 1, 1, 1])
    stack, left, _ = _release(16, n_pages, lens, done, table, [])
    back = [int(e) for i in range(7) if done[i] for e in table[i, :need[i]] if e >= 0]
    assert stack == back + [PAD] * (n_pages - len(back)) and left == len(back) and cg.get_status() == 0


def test_more_pages_than_the_stack_holds():
    """A page that two requests name: what finds no room is dropped, with the flag."""
    table = [[0, 1, 2], [2, 3, 0]]
    stack, left, _ = _release(16, 5, [48, 48], [1, 1], table, [4])
    assert stack == [4, 0, 1, 2, 2] and left == 5 and cg.get_status() == RANGE


def test_lengths_beyond_the_table():
    stack, left, lens_left = _release(16, 8, [1000, -5, 16], [1, 1, 0], [[3, 5], [1, 2], [4, -1]], [7])
    assert stack[:3] == [7, 3, 5] and left == 3 and lens_left == [0, 0, 16] and cg.get_status() == RANGE


def test_a_window_gives_pages_back_and_the_stack_drains():
    """A windowed request whose first pages are back on the stack attends as before; its release gives the
    rest, and a plan then takes every page of the pool once."""
    c = _case("bf16", 128, 2, 4, 16, [300, 40], [1, 1], window=100, sinks=3, seed=41)
    want, _ = _attend(c)
    table, n_pages = c["table"].copy(), c["pool"].shape[1]
    given = [j for j in range(300 // 16 + 1) if j * 16 >= 3 and (j + 1) * 16 <= 300 - 100]
    free = [p for p in range(n_pages) if p not in table] + [int(table[0, j]) for j in given]
    table[0, given] = -1
    out, lse = _attend(dict(c, table=table))
    assert torch.equal(out, want) and cg.get_status() == 0
    _check(c, out, lse)
    stack, left, _ = _release(16, n_pages, [300, 40], [1, 1], table, free)
    assert left == n_pages and sorted(stack) == list(range(n_pages)) and cg.get_status() == 0
    # all of it for one new request
    pages = cg.Pages(n_pages=n_pages, page=16, n_req=1, max_pages=n_pages)
    bt, n = torch.full((1, n_pages), -1, dtype=torch.int32, device="cuda"), 16 * n_pages
    lens, cu, pos, left = i32([0]), i32([0, 0]), i32(np.zeros(n)), i32([0])
    slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    cg.page_plan(pages, i32([0]), i32([n]), i32(stack), i32([n_pages]), bt, lens, cu, pos, slots, left)
    assert sorted(bt[0].tolist()) == list(range(n_pages)) and left.item() == 0 and (slots >= 0).all() and cg.get_status() == 0


def test_after_a_plan_that_ran_out():
    """Its -1 entries, if the plan is kept all the same, do not come onto the stack."""
    pages = cg.Pages(n_pages=4, page=16, n_req=1, max_pages=6)
    bt = torch.full((1, 6), -1, dtype=torch.int32, device="cuda")
    lens, cu, pos, left = i32([0]), i32([0, 0]), i32(np.zeros(96)), i32([0])
    slots = torch.zeros(96, dtype=torch.int64, device="cuda")
    cg.page_plan(pages, i32([0]), i32([96]), i32([0, 1, 2, 3]), i32([4]), bt, lens, cu, pos, slots, left)
    assert cg.get_status() == 8 and bt.tolist() == [[3, 2, 1, 0, -1, -1]]
    stack, left, _ = _release(16, 4, [96], [1], bt.cpu().numpy(), [])
    assert stack == [3, 2, 1, 0] and left == 4 and cg.get_status() == 0
