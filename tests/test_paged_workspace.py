"""Which paged attention calls share the workspace that the binding keeps for the default stream: a call
is up to three launches, so calls that two host threads make at the same time must not."""
import os
import threading

import pytest

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")
paged = cg.paged

PAGES, HOW = cg.Pages(n_pages=8, page=16, H=2, d=64, n_req=2, max_pages=4), cg.PagedAttention(4, 40, 0.1)


@pytest.fixture(autouse=True)
def default_stream(monkeypatch):
    if not os.path.exists(cg.lib_path()):
        from paper_2607_20538_gb300 import build
        build.build()
    monkeypatch.setattr(paged, "_stream", lambda stream: 0)


def test_threads_do_not_share_the_kept_workspace():
    """Four threads that are all inside their calls at the same time, two calls each."""
    got, gate = {}, threading.Barrier(4)

    def calls(name):
        gate.wait()
        first = paged._workspace(PAGES, HOW, 10, torch.device("cpu"))
        gate.wait()
        got[name] = first, paged._workspace(PAGES, HOW, 10, torch.device("cpu"))
        gate.wait()

    threads = [threading.Thread(target=calls, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(a is b for a, b in got.values())
    assert len({a.data_ptr() for a, _ in got.values()}) == 4


def test_a_thread_keeps_one_workspace_that_grows():
    device = torch.device("cpu")
    small = paged._workspace(PAGES, cg.PagedAttention(4, 1, 0.1), 1, device)
    large = paged._workspace(PAGES, HOW, 10, device)
    assert large.nbytes >= cg.paged_attention_workspace_bytes(PAGES, HOW, 10) > small.nbytes
    assert paged._workspace(PAGES, cg.PagedAttention(4, 1, 0.1), 1, device) is large
