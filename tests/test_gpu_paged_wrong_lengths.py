"""Plans and releases with lengths that are wrong by far: the flag, and nothing written outside the arrays."""
import numpy as np
import pytest

from test_gpu_paged import EXHAUSTED, RANGE, cg, i32, torch

pytestmark = pytest.mark.gpu

FILL, EDGE = -5, 1 << 20


def _guarded(n, dtype=torch.int32):
    flat = torch.full((n + 2 * EDGE,), FILL, dtype=dtype, device="cuda")
    return flat, flat[EDGE:EDGE + n]


def _edges_stay(flat):
    return bool((flat[:EDGE] == FILL).all() and (flat[-EDGE:] == FILL).all())


@pytest.mark.parametrize("n_req,max_pages", [(65536, 33000), (300, 5000), (1, 7)])
def test_a_plan_of_far_too_many_tokens(n_req, max_pages):
    """Each request asks for as many tokens as the whole call may have: in the largest case for 2^31 pages
    and more, in a table of 8.7 GB. The first request gets its pages, as far as there are any; no more than
    n_tok + n_req entries are dealt out."""
    page, n_pages = 16, 1000
    n_tok = page * max_pages
    flat, table = _guarded(n_req * max_pages)
    pages = cg.Pages(n_pages=n_pages, page=page, n_req=n_req, max_pages=max_pages)
    ones = torch.ones(n_req, dtype=torch.int32, device="cuda")
    fp, pos = _guarded(n_tok)
    fs, slots = _guarded(n_tok, torch.int64)
    lens, cu, left = torch.empty_like(ones), i32(np.zeros(n_req + 1)), i32([0])
    cg.page_plan(pages, ones * 0, ones * n_tok, torch.arange(n_pages, dtype=torch.int32, device="cuda"), i32([n_pages]), table, lens, cu,
                 pos, slots, left)
    flags = cg.get_status()
    too_few = n_req * max_pages > n_pages
    assert flags == (RANGE if n_req > 1 else 0) | (EXHAUSTED if too_few else 0)
    assert _edges_stay(flat) and _edges_stay(fp) and _edges_stay(fs)
    given = min(n_req * max_pages, n_tok + n_req)
    assert int((table[:given] == FILL).sum()) == 0 and bool((table[given:] == FILL).all())
    assert int((table[:given] >= 0).sum()) == min(given, n_pages)
    have = min(max_pages, n_pages)
    assert table[:have].tolist() == list(range(n_pages - 1, n_pages - 1 - have, -1))
    assert left.item() == max(n_pages - n_req * max_pages, -(2 ** 31 - 1))
    assert torch.equal(pos, torch.arange(n_tok, dtype=torch.int32, device="cuda"))
    want = torch.where(pos // page < have, (n_pages - 1 - pos // page) * page + pos % page, -1)
    assert torch.equal(slots, want.long())


def test_a_release_of_far_too_many_pages():
    """Every request claims a full row of a wide table of -1: 2^31 entries and more, none of them a page."""
    n_req, max_pages = 65536, 33000
    pages = cg.Pages(n_pages=64, page=16, n_req=n_req, max_pages=max_pages)
    table = torch.full((n_req, max_pages), -1, dtype=torch.int32, device="cuda")
    table[5, 7], table[n_req - 1, max_pages - 1], table[40000, 3] = 9, 11, 64
    ones = torch.ones(n_req, dtype=torch.int32, device="cuda")
    fs, stack = _guarded(64)
    lens_left, left = torch.empty_like(ones), i32([0])
    cg.page_release(pages, ones * 16 * max_pages, ones, table, stack, i32([3]), lens_left, left)
    assert cg.get_status() == RANGE
    assert stack[3:5].tolist() == [9, 11] and left.item() == 5 and _edges_stay(fs) and not lens_left.any()
    assert bool((stack[:3] == FILL).all() and (stack[5:] == FILL).all())
