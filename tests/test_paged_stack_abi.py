"""Refusals of the plan with a sized stack, before any device work."""
import os

import pytest

cg = pytest.importorskip("paper_2607_20538_gb300")
paged = cg.paged
FAKE = 0x10000


def test_refusals():
    if not os.path.exists(cg.lib_path()):
        from paper_2607_20538_gb300 import build
        build.build()
    p = cg.Pages(n_pages=8, page=16, n_req=2, max_pages=4).c()
    plan = paged._fn("cg_page_plan_stack")
    good = [p, 4, FAKE, FAKE, FAKE, 3, FAKE, FAKE, 0x20000, FAKE, FAKE, FAKE, 0x20000, None]
    for at, v in ((0, None), (1, -1), (2, None), (4, None), (4, FAKE + 1), (5, -1), (6, None), (8, FAKE), (12, FAKE)):
        bad = list(good)
        bad[at] = v
        assert plan(*bad) == -1, at
    old = [p, 4, FAKE, FAKE, None, FAKE, FAKE, 0x20000, FAKE, FAKE, FAKE, 0x20000, None]
    assert paged._fn("cg_page_plan")(*old) == -1
    assert paged._fn("cg_page_plan")(None, *old[1:4], FAKE, *old[5:]) == -1
