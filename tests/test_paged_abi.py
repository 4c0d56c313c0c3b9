"""Paged operators without a GPU: refusals before any device work, the rotary table, and what the
plain forms of the GPU tests rest on."""
import ctypes
import math
import os

import numpy as np
import pytest

import paged_ref as ref

cg = pytest.importorskip("paper_2607_20538_gb300")
paged = cg.paged


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cg.lib_path()):
        from paper_2607_20538_gb300 import build
        build.build()
    return cg.load()


FAKE = 0x10000
GOOD = dict(n_pages=8, page=16, H=2, d=128, n_req=2, max_pages=4)
HOW = dict(n_rep=4, max_new=1, scale=0.1)


def _attention(pages=GOOD, how=HOW, n_tok=2, strides=(1024, 128, 1024, 128), q=FAKE, out=FAKE, ws=1 << 30, dtype=0):
    p, h = cg.Pages(**pages), cg.PagedAttention(**how)
    return paged._fn("cg_paged_attention")(p.c(dtype), paged._attn(p, h, n_tok, *strides), q, FAKE, FAKE, FAKE, FAKE, out,
                                           None, FAKE, ws, None)


@pytest.mark.parametrize("kw,code", [
    (dict(pages=dict(GOOD, page=24)), -1), (dict(pages=dict(GOOD, page=8)), -1), (dict(pages=dict(GOOD, page=512)), -1),
    (dict(pages=dict(GOOD, n_pages=0)), -1), (dict(pages=dict(GOOD, n_pages=1 << 28)), -4),
    (dict(pages=dict(GOOD, H=0)), -1), (dict(pages=dict(GOOD, H=1025)), -1), (dict(pages=dict(GOOD, d=96)), -2),
    (dict(pages=dict(GOOD, d=32)), -2), (dict(pages=dict(GOOD, n_req=0)), -1), (dict(pages=dict(GOOD, max_pages=0)), -1),
    (dict(pages=dict(GOOD, max_pages=1 << 27)), -4), (dict(dtype=2), -1),
    (dict(how=dict(HOW, n_rep=0)), -1), (dict(how=dict(HOW, n_rep=65)), -1), (dict(how=dict(HOW, window=-1)), -1),
    (dict(how=dict(HOW, sinks=4)), -1), (dict(how=dict(HOW, window=8, sinks=-1)), -1),
    (dict(how=dict(HOW, scale=math.nan)), -1), (dict(how=dict(HOW, scale=math.inf)), -1), (dict(how=dict(HOW, max_new=-1)), -1),
    (dict(n_tok=-1), -1), (dict(n_tok=1 << 30), -4), (dict(strides=(1020, 128, 1024, 128)), -1), (dict(strides=(1024, 128, -8, 128)), -1),
    (dict(q=None), -1), (dict(out=None), -1), (dict(q=FAKE + 8), -1), (dict(ws=64), -1),
])
def test_attention_refusals(lib, kw, code):
    assert _attention(**kw) == code
    assert lib.cg_last_error().decode()


def test_attention_nothing_to_do(lib):
    assert _attention(n_tok=0) == 0
    assert _attention(how=dict(HOW, max_new=0)) == 0


def test_workspace_bytes(lib):
    pages, how = cg.Pages(**GOOD), cg.PagedAttention(**HOW)
    assert cg.paged_attention_workspace_bytes(pages, how, 2) > 0
    with pytest.raises(cg.CodecGaugeError):
        cg.paged_attention_workspace_bytes(cg.Pages(**dict(GOOD, d=32)), how, 2)


def test_plan_and_release_refusals(lib):
    p = cg.Pages(**GOOD).c()
    good = [p, 4] + [FAKE, FAKE, FAKE, FAKE, FAKE, 0x20000, FAKE, FAKE, FAKE, 0x20000, None]
    plan = paged._fn("cg_page_plan")
    for at, v in ((0, cg.Pages(**dict(GOOD, page=20)).c()), (0, cg.Pages(**dict(GOOD, n_req=65537)).c()), (1, -1),
                  (2, None), (5, None), (6, None), (9, None), (9, FAKE + 4), (10, FAKE + 8), (7, FAKE), (11, FAKE), (3, FAKE + 2)):
        bad = list(good)
        bad[at] = v
        assert plan(*bad) == -1, at
    release = paged._fn("cg_page_release")
    good = [p, FAKE, FAKE, FAKE, FAKE, FAKE, 0x20000, 0x20000, None]
    for at, v in ((1, None), (4, None), (6, FAKE), (7, FAKE), (2, FAKE + 1)):
        bad = list(good)
        bad[at] = v
        assert release(*bad) == -1, at


def test_rotary_refusals(lib):
    f = paged._fn("cg_rotary")
    R = lambda **k: cg.Rotary(**{**dict(rot=64), **k}).c()  # noqa: E731
    good = [R(), 0, 4, 2, 128, FAKE, 256, 128, FAKE, FAKE, FAKE, 256, 128, None]
    for at, v, code in ((0, R(rot=24), -1), (0, R(rot=144), -1), (0, R(mscale=math.nan), -1), (1, 7, -1), (2, -1, -1),
                        (4, 96, -2), (5, None, -1), (5, FAKE + 2, -1), (6, 100, -1), (8, None, -1), (9, None, -1),
                        (10, None, -1), (12, -8, -1)):
        bad = list(good)
        bad[at] = v
        assert f(*bad) == code, at
    assert f(*(good[:2] + [0] + good[3:])) == 0          # no tokens: nothing to do
    g = paged._fn("cg_rotary_append")
    S = lambda *v: paged._CStrides(*v)  # noqa: E731
    good = [cg.Pages(**GOOD).c(), R(), 4, 8, S(1024, 128, 256, 128, 256, 128, 1024, 128), FAKE, FAKE, FAKE, FAKE, FAKE,
            FAKE, FAKE, FAKE, None]
    for at, v, code in ((0, cg.Pages(**dict(GOOD, d=32)).c(), -2), (1, R(rot=8), -1), (3, -1, -1),
                        (4, S(1024, 128, 250, 128, 256, 128, 1024, 128), -1), (5, None, -1), (6, None, -1), (7, FAKE + 8, -1),
                        (9, None, -1), (9, FAKE + 4, -1), (10, None, -1), (12, None, -1)):
        bad = list(good)
        bad[at] = v
        assert g(*bad) == code, at


@pytest.mark.parametrize("kind,factor,low,high", [(0, 1.0, 1.0, 4.0), (1, 4.0, 1.0, 4.0), (2, 8.0, 1.0, 4.0), (3, 4.0, 1.0, 32.0),
                                                  (3, 0.5, 1.0, 32.0)])
@pytest.mark.parametrize("rot", [16, 64, 128, 256])
def test_rotary_table_is_the_formula(lib, kind, factor, low, high, rot):
    """Against the rules written out: double arithmetic is good to a few 2^-53 of a frequency (pow and
    log within 2 ulp, five operations), that is 2^-46 of it with room."""
    base, orig = 10000.0, 8192.0
    t, m = cg.rotary_table(rot, cg.RopeScaling(kind, base, factor, orig, low, high), device="cpu")
    at = lambda n: rot * math.log(orig / (2 * math.pi * n)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
    for c in range(rot // 2):
        f = math.exp(-2 * c / rot * math.log(base))
        x = 1.0
        if kind == 1:
            x = 0.0
        elif kind == 2:
            x = min(max((orig * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
        elif kind == 3:
            x = 1 - min(max((c - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
        want = (f / factor * (1 - x) + f * x) / (2 * math.pi)
        got = (int(t[c]) % (1 << 64)) / 2.0 ** 64
        assert abs(got - want) <= 2.0 ** -46 * want, (c, got, want)
    assert m == pytest.approx(0.1 * math.log(factor) + 1 if kind == 3 and factor > 1 else 1.0, rel=1e-6)


def test_rotary_table_refusals(lib):
    for rot, kw in ((0, {}), (24, {}), (272, {}), (64, dict(base=1.0)), (64, dict(kind=5)), (64, dict(kind=1, factor=0.0)),
                    (64, dict(kind=2, factor=2.0, low=4.0, high=1.0)), (64, dict(kind=3, factor=2.0, original=0.0))):
        with pytest.raises(cg.CodecGaugeError) as e:
            cg.rotary_table(rot, cg.RopeScaling(**kw), device="cpu")
        assert e.value.code == -1


def test_a_table_without_scaling_is_within_half_a_unit(lib):
    """2^64 f / 2 pi is rounded to a whole number: frequencies of 1 (c = 0) give 2^64 / 2 pi."""
    t, _ = cg.rotary_table(64, device="cpu")
    assert abs(int(t[0]) - (1 << 64) / (2 * math.pi)) <= 2048     # 2^64 / 2 pi has 62 bits, a double 53


def test_plain_attention_is_the_softmax(lib):
    """The plain form of the GPU tests against torch's own attention in float64 (causal, shared heads)."""
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(1)
    H, rep, d, page, n = 2, 3, 64, 16, 37
    pool = rng.normal(size=(2, 4, H, page, d))
    table = np.array([[2, 0, 3]])
    q = rng.normal(size=(n, H * rep, d))
    o, lse, mag, big = ref.attention(q, pool, table, [n], [0, n], rep, 0.2)
    K, V = (torch.from_numpy(pool[x][table[0]].transpose(1, 0, 2, 3).reshape(H, -1, d)[:, :n]) for x in (0, 1))
    Q = torch.from_numpy(q).permute(1, 0, 2)
    want = torch.nn.functional.scaled_dot_product_attention(Q, K.repeat_interleave(rep, 0), V.repeat_interleave(rep, 0),
                                                            is_causal=True, scale=0.2)
    assert np.allclose(o, want.permute(1, 0, 2).numpy(), atol=1e-12)
    # one token: its own value, and its score as the log-sum-exp
    assert np.allclose(o[0, 0], pool[1, 2, 0, 0]) and np.isclose(lse[0, 0], 0.2 * (q[0, 0] @ pool[0, 2, 0, 0]))


def test_plain_rotation_is_a_rotation(lib):
    rng = np.random.default_rng(2)
    x = rng.normal(size=(3, 2, 32))
    table = [int(2 ** 64 * f / (2 * math.pi)) for f in (1.0, 0.1)] + [0] * 6
    for inter in (False, True):
        y = ref.rotate(x, [0, 1, 1 << 40], table, inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[0], x[0])
        a, b = (0, 1) if inter else (0, 8)
        assert np.allclose(y[1, :, a], x[1, :, a] * math.cos(1) - x[1, :, b] * math.sin(1), atol=1e-9)
        assert np.allclose(ref.rotate(y, [0, 1, 1 << 40], table, inter, transpose=True), x)
