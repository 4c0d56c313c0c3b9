"""The serving example: plan, rotary append, attention and release together, against 64-bit histories
kept request by request without pages; and its run as a program."""
import os
import subprocess
import sys

import numpy as np
import pytest

import paged_ref as ref

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


def num(t):
    return t.detach().cpu().to(torch.float64).numpy()


@pytest.mark.parametrize("dtype,H,n_rep,d,page,window,sinks", [
    ("bf16", 2, 4, 128, 16, 0, 0), ("fp16", 1, 3, 64, 32, 0, 0), ("bf16", 2, 7, 64, 16, 29, 3), ("fp16", 1, 2, 256, 64, 0, 0),
])
def test_steps_against_histories(dtype, H, n_rep, d, page, window, sinks):
    from paged_serving import PagedLayer, tokens
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    layer = PagedLayer(n_req=4, max_tokens=400, H=H, n_rep=n_rep, d=d, page=page, window=window, sinks=sinks, dtype=dt)
    gen = torch.Generator(device="cuda").manual_seed(d + page)
    freq = layer.table.cpu().numpy().astype(np.uint64)
    keys, vals = [[] for _ in range(4)], [[] for _ in range(4)]
    all_pages = layer.pages.n_pages
    # prompts (one request waits), single tokens, a chunk beside them, request 1 done and replaced
    for new, done in [([70, 33, 0, 150], None), ([1, 1, 1, 1], None), ([1, 1, 40, 0], None), ([1, 1, 1, 1], [0, 1, 0, 0]),
                      ([1, 21, 1, 1], None), ([1, 1, 1, 1], None)]:
        n = sum(new)
        q, k, v = tokens(n, layer, gen)
        o = num(layer.step(torch.tensor(new, dtype=torch.int32, device="cuda"), q, k, v, max_new=max(new)))
        q, k, v = num(q), num(k), num(v)
        at = 0
        for i, m in enumerate(new):
            pos = range(len(keys[i]), len(keys[i]) + m)
            rows = slice(at, at + m)
            at += m
            if not m:
                continue
            qr = ref.rotate(q[rows], pos, freq, False, layer.mscale)
            keys[i] += list(ref.rotate(k[rows], pos, freq, False, layer.mscale))
            vals[i] += list(v[rows])
            # one page that holds the whole history
            pool = np.stack([np.array(keys[i]), np.array(vals[i])]).transpose(0, 2, 1, 3)[:, None]
            want, _, mag, big = ref.attention(qr, pool, np.zeros((1, 1), int), [len(keys[i])], [0, m], n_rep, d ** -0.5, window, sinks)
            tol, _ = ref.attention_tolerance(dtype == "fp16", d, want, mag, big)
            # the turned query and key are rounded to 16 bits each: a score moves by 2 u of its |q||k|
            u = 2.0 ** -11 if dtype == "fp16" else 2.0 ** -8
            tol = tol + 2 * (2.01 * u * big[..., None]) * mag
            assert np.all(np.abs(o[rows] - want) <= tol)
        if done:
            layer.release(torch.tensor(done, dtype=torch.int32, device="cuda"))
            for i in np.flatnonzero(done):
                keys[i], vals[i] = [], []
        lens = [len(x) for x in keys]
        assert layer.lens.tolist() == lens
        assert int(layer.free_count) == all_pages - sum(-(-x // page) for x in lens)
    assert cg.get_status() == 0


def test_program():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "paged_serving.py"), "--steps", "3", "--bits", "8"],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert "lengths [90, 37, 1504, 260]" in r.stdout and "attention off by" in r.stdout


def test_kept_workspace():
    """Calls of different workspace sizes one after the other on the default stream, against calls with
    a workspace of their own."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    cases = []
    for d, n_rep, lens, new in [(64, 2, [70, 300], [1, 1]), (128, 4, [500, 40, 333], [90, 1, 200]), (64, 2, [70, 300], [1, 1]),
                                (256, 1, [200], [200]), (128, 4, [9, 1000], [1, 1])]:
        H, page, per = 2, 16, 64
        pages = cg.Pages(n_pages=len(lens) * per, page=page, H=H, d=d, n_req=len(lens), max_pages=per)
        rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
        i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
        q = rnd(sum(new), H * n_rep, d)
        cases.append((pages, cg.PagedAttention(n_rep, max(new), d ** -0.5), q, rnd(2, len(lens) * per, H, page, d),
                      i32(np.arange(len(lens) * per).reshape(len(lens), per)), i32(lens), i32(np.concatenate([[0], np.cumsum(new)]))))
    kept = [torch.empty_like(c[2]) for c in cases]
    for c, o in zip(cases, kept):
        cg.paged_attention(*c, o)
    for c, o in zip(cases, kept):
        own = torch.empty_like(o)
        ws = torch.empty(cg.paged_attention_workspace_bytes(c[0], c[1], own.shape[0]), dtype=torch.uint8, device="cuda")
        cg.paged_attention(*c, own, workspace=ws)
        assert torch.equal(own, o)
