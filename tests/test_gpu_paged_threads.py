"""Calls from several host threads. Two that attend on the default stream at the same time: each gets
what it gets alone, bit for bit, and nothing is written past its outputs. A thread whose first use of
the GPU is a call of the library."""
import threading

import numpy as np
import pytest

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")

pytestmark = pytest.mark.gpu

CALLS = 150


def _in_a_new_thread(call):
    failed = []

    def run():
        try:
            call()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    assert not failed


def _state(seed, lens, new, n_rep, d, window):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    H, page, per, r = 2, 16, -(-max(lens) // 16), len(lens)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
    n = sum(new)
    pages = cg.Pages(n_pages=r * per, page=page, H=H, d=d, n_req=r, max_pages=per)
    how = cg.PagedAttention(n_rep, max(new), d ** -0.5, window)
    args = (pages, how, rnd(n, H * n_rep, d), rnd(2, r * per, H, page, d), i32(np.arange(r * per).reshape(r, per)), i32(lens),
            i32(np.concatenate([[0], np.cumsum(new)])))
    # outputs with rows of NaN behind them
    out = torch.full((n + 300, H * n_rep, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n + 300, H * n_rep), float("nan"), device="cuda")
    return args, out, lse, n


@pytest.mark.parametrize("other", [dict(lens=[900, 40, 333], new=[200, 1, 90], n_rep=4, d=128, window=0),
                                   dict(lens=[500, 700], new=[1, 60], n_rep=7, d=64, window=100),
                                   dict(lens=[260], new=[260], n_rep=2, d=256, window=0)])
def test_two_threads_on_the_default_stream(other):
    states = [_state(1, [70, 300, 1500], [40, 2, 33], 4, 128, 0), _state(2, **other)]
    want = []
    for args, out, lse, n in states:
        cg.paged_attention(*args, out[:n], lse[:n])
        want.append((out[:n].clone(), lse[:n].clone()))
    torch.cuda.synchronize()
    gate, wrong = threading.Barrier(len(states)), []

    def work(k):
        try:
            args, out, lse, n = states[k]
            gate.wait()
            for i in range(CALLS):
                cg.paged_attention(*args, out[:n], lse[:n])
                if i % 10 == 9 and not (torch.equal(out[:n], want[k][0]) and torch.equal(lse[:n], want[k][1])):
                    wrong.append((k, i))
        except Exception as e:  # noqa: BLE001
            wrong.append((k, e))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(states))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong
    for _, out, lse, n in states:
        assert torch.isnan(out[n:]).all() and torch.isnan(lse[n:]).all()
    assert cg.get_status() == 0


@pytest.mark.parametrize("lens,new", [([300, 40], [1, 1]), ([300, 90], [60, 45])])
def test_attention_as_a_threads_first_call(lens, new):
    """Everything the call needs is there, so that nothing but the call itself touches the GPU."""
    args, out, lse, n = _state(3, lens, new, 4, 128, 0)
    cg.paged_attention(*args, out[:n], lse[:n])
    want, o = out[:n].clone(), out[:n].zero_()
    ws = torch.empty(cg.paged_attention_workspace_bytes(*args[:2], n), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    _in_a_new_thread(lambda: cg.paged_attention(*args, o, lse[:n], ws))
    assert torch.equal(o, want) and cg.get_status() == 0


def test_codec_as_a_threads_first_call():
    """The tensor-core encode and decode: tensor maps, like the attention."""
    shape, params = cg.Shape(2, 1, 4, 256, 128), cg.Params(cg.CG_BLOCK_UNIFORM, 128, 4, block=64)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(2, 2, 1, 4, 256, 128, generator=gen, device="cuda").bfloat16()
    g = torch.linalg.qr(torch.randn(2 * 2 * 4, 128, 128, generator=gen, device="cuda"))[0].contiguous()
    a, b = cg.alloc_outputs(shape, params), cg.alloc_outputs(shape, params)
    y, z = torch.empty_like(x), torch.empty_like(x)
    cg.encode(shape, params, x, g, *a[:2])
    cg.decode(shape, params, *a[:2], None, g, y)
    torch.cuda.synchronize()
    _in_a_new_thread(lambda: cg.encode(shape, params, x, g, *b[:2]))
    torch.cuda.synchronize()
    _in_a_new_thread(lambda: cg.decode(shape, params, *b[:2], None, g, z))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(y, z) and cg.get_status() == 0
