"""The bounded waits of the block product give up cleanly: with a limit that no copy or product can meet the call comes back
with CG_FLAG_PIPE_TIMEOUT, its copies and products drained, and the next call, with the normal limit, gives what the call
before gave, bit for bit."""
import pytest

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")

pytestmark = pytest.mark.gpu
ENV = "CODECGAUGE_PIPE_WAIT_NS"


@pytest.mark.parametrize("M,N,K", [(17, 6144, 4096), (30, 1000, 1040), (60, 500, 4096), (333, 1000, 4112), (1000, 2000, 528), (4000, 6144, 1024)])
def test_wait_limit(M, N, K, monkeypatch):
    gen = torch.Generator(device="cuda").manual_seed(M)
    make = lambda R: torch.randint(0, 120, (R, K), generator=gen, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)  # noqa: E731
    x, w, nb = make(M), make(N), -(-K // 128)
    xs, ws = torch.rand(M, nb, generator=gen, device="cuda"), torch.rand(-(-N // 128), nb, generator=gen, device="cuda")

    def go():
        out = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
        cg.block8_matmul(x, xs, w, ws, out)
        return out, cg.get_status()

    before, flags = go()
    assert flags == 0
    monkeypatch.setenv(ENV, "100")
    _, flags = go()
    assert flags & cg.CG_FLAG_PIPE_TIMEOUT
    monkeypatch.delenv(ENV)
    after, flags = go()
    assert flags == 0 and torch.equal(after, before)
