"""Outputs whose rows lie on one another (a stride of 0, as of an expanded tensor) are refused before any
device work; inputs may be like that, and so may an output's dimension of one element."""
import os

import pytest

cg = pytest.importorskip("paper_2607_20538_gb300")
paged = cg.paged
FAKE = 0x10000


@pytest.fixture(autouse=True, scope="module")
def built():
    if not os.path.exists(cg.lib_path()):
        from paper_2607_20538_gb300 import build
        build.build()


def _attention(n_tok, n_rep, H, strides):
    p, h = cg.Pages(n_pages=8, page=16, H=H, d=128, n_req=2, max_pages=4), cg.PagedAttention(n_rep, 4, 0.1)
    # a workspace that is too small: what passes the strides stops there
    rc = paged._fn("cg_paged_attention")(p.c(), paged._attn(p, h, n_tok, *strides), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, 64, None)
    return rc, cg.load().cg_last_error().decode()


@pytest.mark.parametrize("n_tok,n_rep,H,strides,refused", [
    (2, 4, 2, (1024, 128, 0, 128), True), (2, 4, 2, (1024, 128, 1024, 0), True), (2, 1, 2, (1024, 128, 1024, 0), True),
    (2, 4, 2, (0, 0, 1024, 128), False), (1, 4, 2, (1024, 128, 0, 128), False), (2, 1, 1, (1024, 128, 1024, 0), False),
])
def test_attention(n_tok, n_rep, H, strides, refused):
    rc, message = _attention(n_tok, n_rep, H, strides)
    assert rc == -1 and ("workspace" in message) != refused and ("stride" in message) == refused


@pytest.mark.parametrize("tok,head", [(0, 128), (256, 0)])
def test_rotary_and_append(tok, head):
    r = cg.Rotary(rot=64).c()
    f = paged._fn("cg_rotary")
    assert f(r, 0, 4, 2, 128, FAKE, 256, 128, FAKE, FAKE, FAKE, tok, head, None) == -1
    assert "stride" in cg.load().cg_last_error().decode()
    g = paged._fn("cg_rotary_append")
    p = cg.Pages(n_pages=8, page=16, H=2, d=128).c()
    args = [FAKE] * 8 + [None]
    assert g(p, r, 4, 2, paged._CStrides(256, 128, 256, 128, 256, 128, tok, head), *args) == -1
    assert "stride" in cg.load().cg_last_error().decode()
