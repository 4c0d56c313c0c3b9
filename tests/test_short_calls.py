"""The short way of calls from Python (csrc/cg_calls.cpp) gives the library what the Python functions give it, or nothing."""
from __future__ import annotations

import ctypes
import importlib.util
import os
import shutil

import pytest
import torch

import paper_2607_20538_gb300 as cg
from paper_2607_20538_gb300 import build, paged

BF16, FP16, F32, I32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.int32, torch.float8_e4m3fn
NAMES = ["tree_plan", "tree_attention", "tree_commit", "block8_encode", "block8_matmul"]
PAGES = cg.Pages(8, 16, 2, 128, 2, 4)
HOW = cg.PagedAttention(4, 5, 0.1)


class Calls:
    """A copy of the module whose entry points write down what they are given. Its tensors are on the CPU, whose
    number as a device is -1."""

    def __init__(self, tmp_path, monkeypatch):
        if not os.path.exists(build.CALLS):
            pytest.skip("built where Python's and torch's headers are")
        copy = str(tmp_path / "_calls.so")
        shutil.copy(build.CALLS, copy)
        spec = importlib.util.spec_from_file_location("_calls", copy)
        self.module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(self.module)
        self.made, self.rc = [], 0
        self._keep = [ctypes.CFUNCTYPE(ctypes.c_int, *paged._ARGS["cg_" + n])(self._note(n)) for n in NAMES]
        self.module.setup(torch.Tensor, *(ctypes.cast(f, ctypes.c_void_p).value for f in self._keep))
        monkeypatch.setattr(paged, "_short", False)
        monkeypatch.setattr(paged, "_device", lambda: -1)
        monkeypatch.setattr(paged, "_stream", lambda stream: 7)
        monkeypatch.setattr(paged, "_fn", lambda name: self._note(name[3:]))

    def _note(self, name):
        structs = {"tree_attention": (28, 56), "tree_commit": (28,)}.get(name, ())

        def note(*a):
            a = list(a)
            for i, size in enumerate(structs):
                a[i] = (a[i] if isinstance(a[i], bytes) else ctypes.string_at(a[i], size))[:size]
            self.made.append((name, tuple(None if v == 0 else v for v in a)))
            return self.rc
        return note

    def both(self, name, kw, python):
        """What the two ways give the library; None: nothing."""
        self.made.clear()
        rc = getattr(self.module, name)(*ARGS[name](kw))
        short = self.made.copy()
        assert (rc is None) == (not short)
        self.made.clear()
        try:
            python(kw)
        except cg.CodecGaugeError as e:
            assert e.code == -1
        return short, self.made.copy()


@pytest.fixture
def calls(tmp_path, monkeypatch):
    return Calls(tmp_path, monkeypatch)


def _t(*shape, dtype=I32):
    return torch.empty(shape, dtype=dtype)


def _plan():
    return dict(max_new=5, window=0, sinks=0, parents=_t(6), seq_lens=_t(2), cu_new=_t(3), positions=_t(5), masks=_t(5, 1))


def _attention():
    return dict(pages=PAGES, how=HOW, q=_t(5, 8, 128, dtype=BF16), pool=_t(2, 8, 2, 16, 128, dtype=BF16), block_table=_t(2, 4), seq_lens=_t(2),
                cu_new=_t(3), positions=_t(5), masks=_t(5, 2), out=_t(5, 8, 128, dtype=BF16), lse=_t(5, 8, dtype=F32),
                workspace=_t(1000, dtype=torch.uint8))


def _commit():
    return dict(pages=PAGES, max_new=5, parents=_t(5), leaves=_t(2), seq_lens=_t(2), cu_new=_t(3), block_table=_t(2, 4),
                pool=_t(3, 2, 8, 2, 16, 128, dtype=BF16), lens_left=_t(2), free_pages=_t(8), free_count=_t(1), free_left=_t(1))


def _encode():
    return dict(x=_t(130, 272, dtype=BF16), codes=_t(130, 272, dtype=E4M3), scales=_t(130, 3, dtype=F32), rows=1)


def _matmul():
    return dict(x=_t(7, 272, dtype=E4M3), x_scales=_t(7, 3, dtype=F32), w=_t(130, 272, dtype=E4M3), w_scales=_t(2, 3, dtype=F32),
                out=_t(7, 130, dtype=BF16))


KW = dict(tree_plan=_plan, tree_attention=_attention, tree_commit=_commit, block8_encode=_encode, block8_matmul=_matmul)
ARGS = {n: (lambda kw: (*kw.values(), -1, 7)) for n in NAMES}
PYTHON = {n: (lambda kw, n=n: getattr(cg, n)(**kw)) for n in NAMES}


def _other(name, key, value):
    """Values in the place of a good one; some fit too."""
    if not isinstance(value, torch.Tensor):
        if isinstance(value, int):
            return [value + 1, -1, 128, 2 ** 31, -2 ** 31 - 1, True]
        if key == "pages":
            return [value._replace(**{f: v}) for f in value._fields for v in (1, 2 ** 31)]
        return [value._replace(**{f: v}) for f in value._fields for v in (1, 3, 2 ** 31)] + [value._replace(scale=s) for s in (1e39, float("inf"), 2)]
    s = list(value.shape)
    out = [torch.empty(s[:i] + [s[i] + d] + s[i + 1:], dtype=value.dtype) for i in range(len(s)) for d in (-1, 1, 128) if s[i] + d >= 0]
    out += [torch.empty(s, dtype=d) for d in (BF16, FP16, F32, I32, torch.int64, E4M3) if d is not value.dtype]
    out += [torch.empty([1, *s], dtype=value.dtype), torch.empty(s[1:], dtype=value.dtype), torch.empty(s, dtype=value.dtype, device="meta")]
    out += [torch.empty([*s[:i], 2 * s[i], *s[i + 1:]], dtype=value.dtype)[(slice(None),) * i + (slice(None, None, 2),)] for i in range(len(s))]
    out += [torch.empty(s[::-1], dtype=value.dtype).permute(*range(len(s))[::-1])]
    out += [torch.empty([*s[:i], 3 * s[i], *s[i + 1:]], dtype=value.dtype).narrow(i, s[i], s[i]) for i in range(len(s))]
    return out


@pytest.mark.parametrize("name", NAMES)
def test_same_call(name, calls):
    kw = KW[name]()
    short, python = calls.both(name, kw, PYTHON[name])
    assert len(short) == 1 and short == python
    optional = {"tree_attention": (dict(lse=None), dict(positions=None)),
                "tree_commit": (dict(pool=None), dict(pool=_t(2, 8, 2, 16, 128, dtype=FP16)),
                                dict.fromkeys(("lens_left", "free_pages", "free_count", "free_left"))),
                "block8_encode": (dict(rows=128, scales=_t(2, 3, dtype=F32)), dict(x=_t(130, 272, dtype=FP16))),
                "block8_matmul": (dict(out=_t(7, 130, dtype=FP16)),
                                  dict(x=_t(1, 272, dtype=E4M3).as_strided([1, 272], [3, 1]), x_scales=_t(1, 3, dtype=F32), out=_t(1, 130, dtype=BF16)))}
    for change in optional.get(name, ()):
        short, python = calls.both(name, dict(kw, **change), PYTHON[name])
        assert len(short) == 1 and short == python, list(change)


@pytest.mark.parametrize("name", NAMES)
def test_other_arguments(name, calls):
    """Whatever one argument is: where the short way calls, the Python function makes the same call; where the Python
    function refuses, the short way does not call."""
    kw = KW[name]()
    took = refused = 0
    for key, value in kw.items():
        for v in [*_other(name, key, value), None, 1.5, "x", object()]:
            try:
                short, python = calls.both(name, dict(kw, **{key: v}), PYTHON[name])
            except (AttributeError, TypeError, ValueError, RuntimeError):   # (a thing that is no tensor or number)
                assert not calls.made
                assert getattr(calls.module, name)(*ARGS[name](dict(kw, **{key: v}))) is None, (key, v)
                continue
            assert not short or short == python, (key, v)
            took += bool(short)
            refused += not python
            if short != python:      # (what only the longer way takes is nothing that a program passes in a loop)
                assert python and not isinstance(v, torch.Tensor), (key, v)
    assert took >= 3 and refused >= 20


def test_the_librarys_status_comes_back(calls):
    calls.rc = -2
    assert calls.module.block8_encode(*ARGS["block8_encode"](_encode())) == -2
    assert calls.module.block8_encode() is None and calls.module.tree_plan(1, 2, 3) is None


def test_a_status_raises(monkeypatch):
    class Short:
        tree_plan = staticmethod(lambda *a: a[0])

    monkeypatch.setattr(paged, "_short", Short)
    assert paged._took("tree_plan", 0) and not paged._took("tree_plan", None)
    with pytest.raises(cg.CodecGaugeError) as e:
        paged._took("tree_plan", -2)
    assert e.value.code == -2


def _step(device="cuda"):
    """One step of two trees and a product: the outputs of the five calls."""
    g = torch.Generator().manual_seed(3)
    i32 = lambda v: torch.tensor(v, dtype=I32, device=device)  # noqa: E731
    rand = lambda *s: torch.randn(s, generator=g).to(device)  # noqa: E731
    parents, lens, cu, table = i32([-1, 0, 0, -1, 0]), i32([21, 18]), i32([0, 3, 5]), i32([[3, 5, -1, -1], [1, 0, -1, -1]])
    positions, masks = torch.full((5,), -1, dtype=I32, device=device), torch.zeros((5, 1), dtype=I32, device=device)
    cg.tree_plan(3, parents, lens, cu, positions, masks)
    pool, q = rand(2, 8, 2, 16, 128).to(BF16), rand(5, 8, 128).to(BF16)
    out, lse = torch.empty_like(q), torch.empty((5, 8), dtype=F32, device=device)
    cg.tree_attention(PAGES, HOW, q, pool, table, lens, cu, positions, masks, out, lse)
    left, free, count, free_left = i32([0, 0]), i32([2, 4, 6, 7, 0, 0, 0, 0]), i32([4]), i32([0])
    cg.tree_commit(PAGES, 3, parents, i32([2, -1]), lens, cu, table, pool, left, free, count, free_left)
    x, w = rand(7, 272).to(BF16), rand(130, 272).to(BF16)
    xc, wc = torch.empty((7, 272), dtype=E4M3, device=device), torch.empty((130, 272), dtype=E4M3, device=device)
    xs, ws = torch.empty((7, 3), dtype=F32, device=device), torch.empty((2, 3), dtype=F32, device=device)
    y = torch.empty((7, 130), dtype=BF16, device=device)
    cg.block8_encode(x, xc, xs)
    cg.block8_encode(w, wc, ws, rows=128)
    cg.block8_matmul(xc, xs, wc, ws, y)
    return [t.cpu() for t in (positions, masks, out, lse, pool, left, free, free_left, xc.view(torch.uint8), xs, wc.view(torch.uint8), ws, y)]


@pytest.mark.gpu
def test_a_step_goes_the_short_way(monkeypatch):
    """And gives what it gives by Python and ctypes."""
    if not os.path.exists(build.CALLS):
        pytest.skip("built where Python's and torch's headers are")
    by_ctypes = []
    fn = paged._fn
    monkeypatch.setattr(paged, "_fn", lambda name: by_ctypes.append(name) or fn(name))
    monkeypatch.setattr(paged, "_short", None)
    short = _step()
    assert not [n for n in by_ctypes if "workspace_bytes" not in n]
    monkeypatch.setattr(paged, "_short", False)
    longer = _step()
    assert len([n for n in by_ctypes if "workspace_bytes" not in n]) == 6
    assert all(torch.equal(a, b) for a, b in zip(short, longer))
    assert cg.get_status() == 0


@pytest.mark.gpu
def test_a_tensor_elsewhere_is_refused():
    x, codes, scales = (t.cuda() for t in list(_encode().values())[:3])
    with pytest.raises(cg.CodecGaugeError, match="scales"):
        cg.block8_encode(x, codes, scales.cpu())
    with pytest.raises(cg.CodecGaugeError, match="q:"):
        cg.tree_attention(**dict({k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in _attention().items()}, q=_attention()["q"]))
