"""The bounded waits of the paged attention kernels give up cleanly: with a limit that no pipeline stage
can meet the call comes back with CG_FLAG_PIPE_TIMEOUT, its copies and products drained, and the next
call, with the normal limit, gives what the call before gave, bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")

pytestmark = pytest.mark.gpu
ENV = "CODECGAUGE_PIPE_WAIT_NS"


@pytest.mark.parametrize("d,ctx,new", [
    (128, [3000, 40], [1, 1]), (256, [3000, 40], [1, 1]), (64, [900, 0, 17], [300, 200, 65]), (128, [2000], [333]),
    (256, [500, 3], [200, 90]), (128, [700, 800], [1, 400]),
])
def test_wait_limit(d, ctx, new, monkeypatch):
    H, n_rep, page = 2, 4, 16
    gen = torch.Generator(device="cuda").manual_seed(d)
    n_req, n_tok = len(ctx), sum(new)
    per = max(-(-(c + n) // page) for c, n in zip(ctx, new))
    pages = cg.Pages(n_pages=n_req * per, page=page, H=H, d=d, n_req=n_req, max_pages=per)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    pool, q = rnd(2, n_req * per, H, page, d), rnd(n_tok, H * n_rep, d)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
    table = i32(np.random.default_rng(d).permutation(n_req * per).reshape(n_req, per))
    lens, cu = i32(np.add(ctx, new)), i32(np.concatenate([[0], np.cumsum(new)]))
    how = cg.PagedAttention(n_rep, max(new), d ** -0.5)

    def go():
        out = torch.zeros_like(q)
        cg.paged_attention(pages, how, q, pool, table, lens, cu, out)
        return out, cg.get_status()

    before, flags = go()
    assert flags == 0
    monkeypatch.setenv(ENV, "100")
    _, flags = go()
    assert flags & cg.CG_FLAG_PIPE_TIMEOUT
    monkeypatch.delenv(ENV)
    after, flags = go()
    assert flags == 0 and torch.equal(after, before)
