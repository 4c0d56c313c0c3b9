"""The draft-tree operators without a GPU: refusals before any device work, by the library and by the binding."""
import os

import numpy as np
import pytest

import tree_ref as ref
from test_paged_devices import OnDevice

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")
paged = cg.paged

FAKE = 0x10000
GOOD = dict(n_pages=8, page=16, H=2, d=128, n_req=2, max_pages=4)
HOW = dict(n_rep=4, max_new=5, scale=0.1)
I32, BF16, U8 = torch.int32, torch.bfloat16, torch.uint8


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cg.lib_path()):
        from paper_2607_20538_gb300 import build
        build.build()
    return cg.load()


def _plan(n_req=2, n_tok=5, max_new=5, window=0, sinks=0, parents=FAKE, lens=2 * FAKE, cu=3 * FAKE, positions=4 * FAKE, masks=5 * FAKE, words=1):
    return paged._fn("cg_tree_plan")(n_req, n_tok, max_new, window, sinks, parents, lens, cu, positions, masks, words, None)


def _attention(pages=GOOD, how=HOW, n_tok=2, strides=(1024, 128, 1024, 128), q=FAKE, out=FAKE, masks=FAKE, positions=FAKE, words=1, ws=1 << 30, dtype=0):
    p, h = cg.Pages(**pages), cg.PagedAttention(**how)
    return paged._fn("cg_tree_attention")(p.c(dtype), paged._attn(p, h, n_tok, *strides), words, q, FAKE, FAKE, FAKE, FAKE, positions, masks,
                                          out, None, FAKE, ws, None)


def _commit(pages=GOOD, n_tok=5, max_new=5, layers=1, parents=FAKE, leaves=2 * FAKE, lens=3 * FAKE, cu=4 * FAKE, table=5 * FAKE, pool=6 * FAKE,
            left=7 * FAKE, free=8 * FAKE, count=9 * FAKE, free_left=10 * FAKE, dtype=0):
    return paged._fn("cg_tree_commit")(cg.Pages(**pages).c(dtype), n_tok, max_new, layers, parents, leaves, lens, cu, table, pool, left, free, count,
                                       free_left, None)


@pytest.mark.parametrize("call,kw,code", [
    (_plan, dict(n_req=0), -1), (_plan, dict(n_req=65537), -1), (_plan, dict(n_tok=-1), -1), (_plan, dict(max_new=-1), -1),
    (_plan, dict(max_new=8193, words=300), -1), (_plan, dict(max_new=33), -1), (_plan, dict(words=0), -1), (_plan, dict(window=-1), -1),
    (_plan, dict(sinks=2), -1), (_plan, dict(window=4, sinks=-1), -1), (_plan, dict(parents=None), -1), (_plan, dict(lens=None), -1),
    (_plan, dict(cu=None), -1), (_plan, dict(positions=None), -1), (_plan, dict(masks=None), -1), (_plan, dict(masks=FAKE + 2), -1),
    (_plan, dict(positions=FAKE), -1), (_plan, dict(masks=2 * FAKE), -1), (_plan, dict(masks=4 * FAKE), -1),
    (_attention, dict(pages=dict(GOOD, page=24)), -1), (_attention, dict(pages=dict(GOOD, d=96)), -2), (_attention, dict(how=dict(HOW, n_rep=65)), -1),
    (_attention, dict(how=dict(HOW, sinks=4)), -1), (_attention, dict(words=0), -1), (_attention, dict(how=dict(HOW, max_new=33)), -1),
    (_attention, dict(masks=None), -1), (_attention, dict(how=dict(HOW, window=8), positions=None), -1), (_attention, dict(masks=FAKE + 2), -1),
    (_attention, dict(q=None), -1), (_attention, dict(q=FAKE + 8), -1), (_attention, dict(ws=64), -1), (_attention, dict(strides=(1020, 128, 1024, 128)), -1),
    (_attention, dict(strides=(1024, 128, 0, 128)), -1), (_attention, dict(dtype=2), -1),
    (_commit, dict(pages=dict(GOOD, page=24)), -1), (_commit, dict(pages=dict(GOOD, H=0)), -1), (_commit, dict(pages=dict(GOOD, d=96)), -2),
    (_commit, dict(n_tok=-1), -1), (_commit, dict(max_new=8193), -1), (_commit, dict(layers=0), -1), (_commit, dict(layers=-1), -1),
    (_commit, dict(layers=65537), -1), (_commit, dict(pool=None), -1), (_commit, dict(pool=FAKE + 8), -1), (_commit, dict(parents=None), -1),
    (_commit, dict(leaves=None), -1), (_commit, dict(lens=None), -1), (_commit, dict(cu=None), -1), (_commit, dict(table=None), -1),
    (_commit, dict(left=None), -1), (_commit, dict(free=None), -1), (_commit, dict(count=None), -1), (_commit, dict(free_left=None), -1),
    (_commit, dict(left=3 * FAKE), -1), (_commit, dict(free_left=9 * FAKE), -1), (_commit, dict(left=7 * FAKE + 1), -1), (_commit, dict(dtype=3), -1),
])
def test_refusals(lib, call, kw, code):
    assert call(**kw) == code
    assert lib.cg_last_error().decode()


def test_nothing_to_do(lib):
    assert _attention(n_tok=0) == 0 and _attention(how=dict(HOW, max_new=0)) == 0
    assert _commit(pool=None, layers=0, left=None, free=None, count=None, free_left=None) == 0


def _tensors(call):
    if call == "plan":
        return dict(parents=([5], I32), seq_lens=([2], I32), cu_new=([3], I32), positions=([5], I32), masks=([5, 1], I32))
    if call == "attention":
        return dict(q=([5, 8, 128], BF16), pool=([2, 8, 2, 16, 128], BF16), block_table=([2, 4], I32), seq_lens=([2], I32), cu_new=([3], I32),
                    positions=([5], I32), masks=([5, 1], I32), out=([5, 8, 128], BF16), lse=([5, 8], torch.float32), workspace=([1 << 20], U8))
    return dict(parents=([5], I32), leaves=([2], I32), seq_lens=([2], I32), cu_new=([3], I32), block_table=([2, 4], I32),
                pool=([3, 2, 8, 2, 16, 128], BF16), lens_left=([2], I32), free_pages=([8], I32), free_count=([1], I32), free_left=([1], I32))


def _make(call, t, **kw):
    pages = cg.Pages(**GOOD)
    {"plan": lambda: cg.tree_plan(5, **t, **kw), "attention": lambda: cg.tree_attention(pages, cg.PagedAttention(4, 5, 0.1), **t, **kw),
     "commit": lambda: cg.tree_commit(pages, 5, **t, **kw)}[call]()


@pytest.mark.parametrize("kw", [
    *(dict([(o, i * FAKE)]) for o in ("left", "free", "free_left") for i in (1, 2, 3, 4, 5, 9)), dict(left=8 * FAKE), dict(free_left=7 * FAKE), dict(free_left=8 * FAKE),
])
def test_commit_in_the_place_of_others(lib, kw):
    assert _commit(**kw) == -1 and b"alias" in lib.cg_last_error()


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(paged, "_fn", lambda name: lambda *a: made.append(name) or 0)
    monkeypatch.setattr(paged, "_device", lambda: 0)
    monkeypatch.setattr(paged, "_stream", lambda stream: 0)
    return made


@pytest.mark.parametrize("call", ["plan", "attention", "commit"])
def test_every_tensor_is_checked(call, calls):
    """On the call's device, of the right type and size, contiguous where it has to be."""
    shapes = _tensors(call)
    make = lambda **other: {k: other.get(k, OnDevice(*v)) for k, v in shapes.items()}  # noqa: E731
    _make(call, make())
    assert len(calls) == 1
    for name, (shape, dt) in shapes.items():
        bad = [OnDevice(shape, dt, 1), OnDevice(shape, dt, -1)]
        if name not in ("seq_lens",) or call != "plan":      # (the plan's number of requests is seq_lens')
            less = [shape[0] - 1, *shape[1:]] if name != "pool" else [*shape[:-1], 64]
            bad += [OnDevice(less, dt)] if name != "workspace" and (call, name) != ("commit", "parents") else []
        if name not in ("q", "out", "workspace", "pool"):
            bad += [OnDevice(shape, torch.int64)]
        for t in bad:
            if name == "positions" and call == "plan" and t.shape != torch.Size(shape):
                t = OnDevice([6], dt)                       # more rows than parents
            with pytest.raises(cg.CodecGaugeError) as e:
                _make(call, make(**{name: t}))
            assert e.value.code == -1
    assert len(calls) == 1


def test_what_goes_together(calls):
    t = {k: OnDevice(*v) for k, v in _tensors("commit").items()}
    with pytest.raises(cg.CodecGaugeError):
        _make("commit", dict(t, free_left=None))
    _make("commit", dict(t, pool=None))
    _make("commit", {k: (None if k in ("lens_left", "free_pages", "free_count", "free_left") else v) for k, v in t.items()})
    a = {k: OnDevice(*v) for k, v in _tensors("attention").items()}
    _make("attention", dict(a, positions=None))
    with pytest.raises(cg.CodecGaugeError):
        cg.tree_attention(cg.Pages(**GOOD), cg.PagedAttention(4, 5, 0.1, window=8), **dict(a, positions=None))


def test_plain_forms():
    """The plain forms on a tree that was drawn by hand:  0 - 1 - 3,  0 - 2,  4 (behind the history)."""
    parents, lens, cu = [-1, 0, 0, 1, -1], [12], [0, 5]
    pos, masks = ref.plan(parents, lens, cu, 5, 1)
    assert pos.tolist() == [7, 8, 8, 9, 7] and masks[:, 0].tolist() == [0b1, 0b11, 0b101, 0b1011, 0b10000]
    assert ref.plan(parents, lens, cu, 5, 1, window=2)[1][:, 0].tolist() == [0b1, 0b11, 0b101, 0b1010, 0b10000]
    assert ref.plan(parents, lens, cu, 5, 1, window=1, sinks=8)[1][:, 0].tolist() == [0b1, 0b11, 0b101, 0b1001, 0b10000]
    assert np.array_equal(ref.pack(ref.unpack(masks)), masks)
    pool = np.arange(2 * 3 * 1 * 4 * 1).reshape(2, 3, 1, 4, 1)
    got, left, stack, count = ref.commit(4, 3, parents, [3], lens, cu, np.array([[2, 0, 1]]), pool, [-9, -9, -9], 0)
    # rows 7, 8, 10 stay, stay and move to 9: page 1 (tokens 8 - 11)
    assert left == [10] and count == 0 and got[0, 1, 0, :, 0].tolist() == [4, 6, 6, 7] and got[0, 0, 0, :, 0].tolist() == [0, 1, 2, 3]
    assert ref.path([-1, 5], 1) == ([1], True)
