"""Every visible value row counts exactly once, wherever it lies in a long history: all scores are equal,
and token t's value is 1 in one channel, t mod d for the even KV heads and t div d mod d for the odd ones, so
that an output is the number of visible tokens of that name over their number. Weights are equal powers
of two and the sums whole numbers below 2^24 of them, so an output is off by its rounding (u), and by the
division (2^-22). One row more, less or in another's place moves a name's count, at most 128, by 1, which
is more than u = 2^-8."""
import numpy as np
import pytest

from test_gpu_paged import _attend, _case, cg, num, torch

pytestmark = pytest.mark.gpu

CASES = {
    "one_long": dict(lens=[12000], new=[1]), "one_long_page_256": dict(lens=[12771], new=[1], page=256), "one_d64": dict(lens=[6300], new=[1], d=64, rep=7),
    "one_d256": dict(lens=[9001], new=[1], d=256, rep=2), "ragged": dict(lens=[12000, 1, 63, 64, 65, 4097, 700, 9999], new=[1] * 8),
    "window": dict(lens=[12000, 5000, 30], new=[1] * 3, window=3001, sinks=77), "few_tokens": dict(lens=[7000, 300], new=[4, 3], page=32),
    "prompt": dict(lens=[1500], new=[1500]), "prompt_d64": dict(lens=[900], new=[900], d=64, rep=5), "chunk_after_long": dict(lens=[12300], new=[300]),
    "chunk_d256": dict(lens=[5000], new=[130], d=256, rep=2), "chunks_mixed": dict(lens=[8000, 2000, 333, 12000], new=[90, 1, 333, 1], page=64),
    "chunks_window": dict(lens=[9000, 2222], new=[500, 64], window=1500, sinks=300, rep=7),
    "chunk_rep33": dict(lens=[3000], new=[20], rep=33, d=64),
}


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("name", list(CASES))
def test_every_row_counts_once(name, dtype):
    kw = dict(dict(dtype=dtype, d=128, H=2, rep=4, page=16, seed=len(name)), **CASES[name])
    c = _case(**kw, poison=True)
    d, H, rep, window, sinks = c["d"], c["H"], c["rep"], c["window"], c["sinks"]
    c["q"].zero_()
    counts = np.zeros(c["q"].shape)
    for i, n in enumerate(c["lens"]):
        held = np.arange(n)
        held = held[c["table"][i, held // c["page"]] >= 0]      # (a windowed request's old pages are gone)
        ids, at = torch.from_numpy(c["table"][i, held // c["page"]].astype(np.int64)), torch.from_numpy(held % c["page"])
        seen = ~torch.isnan(c["pool"][0, ids, 0, at, 0].float()).numpy()
        for h in range(H):
            token = held // d % d if h % 2 else held % d
            rows = torch.zeros(len(held), d, dtype=c["pool"].dtype)
            rows[np.arange(len(held)), token] = 1
            rows[~torch.from_numpy(seen)] = float("nan")
            c["pool"][1, ids, h, at] = rows
        new = c["cu"][i + 1] - c["cu"][i]
        for k in range(new):
            t = np.arange(n - new + k + 1)
            if window:
                t = t[(t > n - new + k - window) | (t < sinks)]
            for h in range(H):
                r = slice(h * rep, (h + 1) * rep)
                counts[c["cu"][i] + k, r] = np.bincount(t // d % d if h % 2 else t % d, minlength=d) / len(t)
    out, lse = _attend(c)
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    err, got = np.abs(num(out) - counts), num(out)
    assert np.isfinite(got).all() and (err <= (u + 2.0 ** -22) * counts).all(), f"worst {(err / np.maximum(counts, 1e-9)).max():.3g}"
    assert cg.get_status() == 0
