"""A paged attention call of one token waits for the host: what lies between the caller and the library stays as short as it was.
Python calls are counted, which a clock would only show among other programs' noise."""
from __future__ import annotations

import os
import sys

import pytest

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")
paged = cg.paged

PAGES, HOW = cg.Pages(n_pages=8, page=16, H=2, d=64, n_req=2, max_pages=4), cg.PagedAttention(4, 1, 0.1)


@pytest.fixture
def made(monkeypatch):
    if not os.path.exists(cg.lib_path()):
        from paper_2607_20538_gb300 import build
        build.build()
    made = []
    fn = lambda *a: made.append(a) or 0  # noqa: E731
    monkeypatch.setattr(paged, "_device", lambda: -1)
    monkeypatch.setattr(paged, "_stream", lambda stream: 0)
    monkeypatch.setattr(paged, "_fn", lambda name: fn if name == "cg_paged_attention" else pytest.fail(name))
    monkeypatch.setattr(paged, "_ws_bytes", {(64, 4, 1, torch.device("cpu")): 100})
    return made


@pytest.mark.parametrize("own,most", [(False, 19), (True, 17)])
def test_python_calls_of_a_paged_attention(own, most, made):
    """The call itself, device, two of heads, type, two structs (four), four addresses, function, the library, stream and check; without a
    workspace of one's own that and the stream it is for."""
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q, pool = torch.zeros(2, 8, 64, dtype=torch.bfloat16), torch.zeros(2, 8, 2, 16, 64, dtype=torch.bfloat16)
    args = (PAGES, HOW, q, pool, i32(2, 4), i32(2), i32(3), torch.empty_like(q))
    kw = dict(workspace=torch.zeros(1000, dtype=torch.uint8)) if own else {}
    cg.paged_attention(*args, **kw)
    calls = []

    def note(frame, event, arg):
        if event == "call":
            calls.append(frame.f_code.co_name)

    sys.setprofile(note)
    try:
        cg.paged_attention(*args, **kw)
    finally:
        sys.setprofile(None)
    assert len(made) == 2 and made[0] == made[1] and len(calls) <= most, calls
