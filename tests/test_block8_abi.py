"""The 8-bit block matrices without a GPU: refusals before any device work, by the library and by the binding."""
import os

import pytest

from test_paged_devices import OnDevice

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")
paged = cg.paged

FAKE = 0x10000
E4M3, BF16, F32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cg.lib_path()):
        from paper_2607_20538_gb300 import build
        build.build()
    return cg.load()


def _encode(dtype=0, R=3, K=256, rows=1, x=FAKE, xs=256, codes=2 * FAKE, cs=256, scales=3 * FAKE):
    return paged._fn("cg_block8_encode")(dtype, R, K, rows, x, xs, codes, cs, scales, None)


def _matmul(dtype=0, M=3, N=5, K=256, x=FAKE, xs=256, x_scales=2 * FAKE, w=3 * FAKE, ws=256, w_scales=4 * FAKE, out=5 * FAKE, os=5):
    return paged._fn("cg_block8_matmul")(dtype, M, N, K, x, xs, x_scales, w, ws, w_scales, out, os, None)


BIG = 1 << 31


@pytest.mark.parametrize("call,kw,code", [
    (_encode, dict(dtype=2), -1), (_encode, dict(R=-1), -1), (_encode, dict(R=BIG), -4), (_encode, dict(K=0), -1), (_encode, dict(K=24), -1),
    (_encode, dict(K=BIG), -4), (_encode, dict(rows=2), -1), (_encode, dict(rows=0), -1), (_encode, dict(xs=248), -1), (_encode, dict(xs=260), -1),
    (_encode, dict(cs=240), -1), (_encode, dict(cs=264), -1), (_encode, dict(cs=1 << 40), -1), (_encode, dict(xs=-256), -1), (_encode, dict(x=None), -1),
    (_encode, dict(codes=None), -1), (_encode, dict(scales=None), -1), (_encode, dict(x=FAKE + 8), -1), (_encode, dict(codes=FAKE + 8), -1),
    (_encode, dict(scales=FAKE + 2), -1),
    (_matmul, dict(dtype=-1), -1), (_matmul, dict(M=-1), -1), (_matmul, dict(N=-1), -1), (_matmul, dict(M=BIG), -4), (_matmul, dict(N=BIG), -4),
    (_matmul, dict(K=40), -1), (_matmul, dict(K=0), -1), (_matmul, dict(K=BIG), -4), (_matmul, dict(xs=240), -1), (_matmul, dict(xs=264), -1),
    (_matmul, dict(ws=240), -1), (_matmul, dict(ws=257), -1), (_matmul, dict(os=4), -1), (_matmul, dict(os=-5), -1), (_matmul, dict(x=None), -1),
    (_matmul, dict(x_scales=None), -1), (_matmul, dict(w=None), -1), (_matmul, dict(w_scales=None), -1), (_matmul, dict(out=None), -1),
    (_matmul, dict(x=FAKE + 8), -1), (_matmul, dict(w=FAKE + 8), -1), (_matmul, dict(x_scales=FAKE + 2), -1), (_matmul, dict(out=FAKE + 1), -1),
    (_matmul, dict(out=FAKE), -1),
])
def test_refusals(lib, call, kw, code):
    assert call(**kw) == code
    assert lib.cg_last_error().decode()


@pytest.mark.parametrize("call,kw", [
    (_encode, dict(codes=FAKE)), (_encode, dict(scales=FAKE)), (_encode, dict(scales=2 * FAKE)), (_matmul, dict(out=3 * FAKE)), (_matmul, dict(out=2 * FAKE)),
    (_matmul, dict(out=4 * FAKE)),
])
def test_outputs_in_the_place_of_others(lib, call, kw):
    assert call(**kw) == -1 and b"overlap" in lib.cg_last_error()


def test_nothing_to_do(lib):
    assert _encode(R=0) == 0 and _matmul(M=0) == 0 and _matmul(N=0) == 0
    assert _encode(R=0, x=None, codes=None, scales=None) == 0


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(paged, "_fn", lambda name: lambda *a: made.append(a) or 0)
    monkeypatch.setattr(paged, "_device", lambda: 0)
    monkeypatch.setattr(paged, "_stream", lambda stream: 0)
    return made


def _tensors(call):
    if call == "encode":
        return dict(x=([130, 272], BF16), codes=([130, 272], E4M3), scales=([130, 3], F32))
    if call == "square":
        return dict(x=([130, 272], BF16), codes=([130, 272], E4M3), scales=([2, 3], F32))
    return dict(x=([7, 272], E4M3), x_scales=([7, 3], F32), w=([130, 272], E4M3), w_scales=([2, 3], F32), out=([7, 130], BF16))


def _make(call, t, **kw):
    {"encode": lambda: cg.block8_encode(**t, **kw), "square": lambda: cg.block8_encode(**t, rows=128, **kw),
     "matmul": lambda: cg.block8_matmul(**t, **kw)}[call]()


@pytest.mark.parametrize("call", ["encode", "square", "matmul"])
def test_every_tensor_is_checked(call, calls):
    """On the call's device, of the right type and shape, its rows contiguous."""
    shapes = _tensors(call)
    make = lambda **other: {k: other.get(k, OnDevice(*v)) for k, v in shapes.items()}  # noqa: E731
    _make(call, make())
    assert len(calls) == 1
    for name, (shape, dt) in shapes.items():
        across = OnDevice(shape[::-1], dt)
        across._t = across._t.t()
        for t in (OnDevice(shape, dt, 1), OnDevice(shape, dt, -1), OnDevice([shape[0] + 128, shape[1]], dt), OnDevice([shape[0], shape[1] + 128], dt),
                  OnDevice(shape, torch.int32), OnDevice(shape[1:], dt), across):
            with pytest.raises(cg.CodecGaugeError) as e:
                _make(call, make(**{name: t}))
            assert e.value.code == -1, name
    assert len(calls) == 1
    if call != "matmul":
        with pytest.raises(cg.CodecGaugeError):
            cg.block8_encode(**make(), rows=64)


def test_strides_of_one_row_are_not_used(calls):
    x = OnDevice([1, 272], E4M3)
    x._t = x._t.as_strided([1, 272], [3, 1])
    t = {k: OnDevice(*v) for k, v in dict(x_scales=([1, 3], F32), w=([130, 272], E4M3), w_scales=([2, 3], F32), out=([1, 130], BF16)).items()}
    cg.block8_matmul(x, **t)
    assert calls[0][5] == 0 and calls[0][11] == 0
