"""The serving example's step of drafted trees: afterwards the layer stands where one stands that took the accepted tokens alone."""
import os
import sys

import numpy as np
import pytest

import tree_ref as ref

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.mark.parametrize("dtype,H,n_rep,d,page,window,sinks", [("bf16", 2, 4, 128, 16, 0, 0), ("fp16", 1, 3, 64, 32, 29, 3), ("bf16", 1, 1, 256, 16, 0, 0)])
def test_verify(dtype, H, n_rep, d, page, window, sinks):
    from paged_serving import PagedLayer, tokens
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    make = lambda: PagedLayer(n_req=3, max_tokens=200, H=H, n_rep=n_rep, d=d, page=page, window=window, sinks=sinks, dtype=dt)  # noqa: E731
    trees, alone = make(), make()
    gen, rng = torch.Generator(device="cuda").manual_seed(d), np.random.default_rng(d)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    prompt = tokens(80, trees, gen)
    for layer in (trees, alone):
        layer.step(i32([50, 0, 30]), *prompt, max_new=50)
    for _ in range(3):
        n = [int(rng.integers(1, 40)), int(rng.integers(0, 5)), 9]
        parents = [ref.random_parents(rng, k) for k in n]
        leaves = [int(rng.integers(-1, k)) if k else -1 for k in n]
        x = tokens(sum(n), trees, gen)
        o = trees.verify(i32(n), i32([p for q in parents for p in q]), *x, max_new=max(n), accept=lambda o: i32(leaves))
        start = np.cumsum([0, *n])
        paths = [ref.path(p, e)[0] if e >= 0 else [] for p, e in zip(parents, leaves)]
        took = [int(c) + b for c, line in zip(start, paths) for b in line]
        want = alone.step(i32([len(line) for line in paths]), *(t[took] for t in x), max_new=40)
        assert cg.get_status() == 0 and trees.lens.tolist() == alone.lens.tolist() and int(trees.free_count) == int(alone.free_count)
        # each is off by the rounding of its weights and of itself
        u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
        if took:
            assert (o[took].float() - want.float()).abs().max() <= 4 * u * x[2].float().abs().max()
    one = tokens(3, trees, gen)
    a, b = (layer.step(i32([1, 1, 1]), *one, max_new=1) for layer in (trees, alone))
    assert (a.float() - b.float()).abs().max() <= 4 * u * one[2].float().abs().max()
