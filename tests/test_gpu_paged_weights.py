"""What the weights of the paged attention are rounded to, and the range they leave to the values."""
import numpy as np
import pytest

import paged_ref as ref
from test_gpu_paged import _attend, _case, cg, num, torch

pytestmark = pytest.mark.gpu


def _set_scores(c, scores):
    """Keys that give every query of request i the scores[i], as exponents of 2, with the scale returned:
    queries are 1 in two channels and 0 elsewhere, the keys' two hold the whole part and the fraction."""
    c["q"].zero_()
    c["q"][:, :, :2] = 1
    c["pool"][0].zero_()
    for i, s in enumerate(scores):
        t = np.arange(len(s))
        ids, at = torch.from_numpy(c["table"][i, t // c["page"]].astype(np.int64)), torch.from_numpy(t % c["page"])
        whole = np.floor(s)
        for ch, part in ((0, whole), (1, s - whole)):
            c["pool"][0][ids, :, at, ch] = torch.from_numpy(part).to(c["pool"].dtype)[:, None]
    return float(np.log(2.0))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rep", [3, 4])
@pytest.mark.parametrize("whole", [1, 5, 7])
def test_the_largest_weight_is_not_rounded(dtype, rep, whole):
    """Decode rows whose last token outweighs all others by 2^whole times a number halfway between two of 16
    bits; an earlier block holds the second largest score. The largest weight is a power of two, so an
    output is off by its own rounding, u |o|, and by the rounding of the other weights, u times their sum
    of p |v|, beside what fp32 leaves (paged_ref.attention_tolerance). 400 requests, so that most tiles are
    whole in one CTA and the blocks follow one another there."""
    n, n_req, u = 128, 400, 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    c = _case(dtype, 64, 2, rep, 16, [n] * n_req, [1] * n_req, seed=3)
    s = np.full(n, -24.0)
    s[60], s[127] = 0.0, whole + np.log2(1 + u)
    scale = _set_scores(c, [s] * n_req)
    out, lse = _attend(c, scale)
    want, wl, mag, big = ref.attention(num(c["q"]), num(c["pool"]), c["table"], c["lens"], c["cu"], rep, scale)
    v = num(c["pool"])[1][c["table"][:, (n - 1) // 16], :, (n - 1) % 16].repeat(rep, 1)
    k = num(c["pool"])[0][c["table"][:, (n - 1) // 16], :, (n - 1) % 16].repeat(rep, 1)
    top = np.exp(scale * k[..., :2].sum(-1) - wl)[..., None] * np.abs(v)
    ds = (64 + 8) * 2.0 ** -24 * big + 2.0 ** -19
    tol = u * np.abs(want) + u * (mag - top) + (2 * ds[..., None] + 2.0 ** -24) * mag + 2.0 ** -24
    err = np.abs(num(out) - want)
    assert (err <= tol).all(), f"worst error / bound {(err / tol).max():.3g}"
    assert cg.get_status() == 0


@pytest.mark.parametrize("power", [118, 110, 0, -100, -120])
@pytest.mark.parametrize("d,lens,new", [(128, [700], [1]), (128, [700], [300]), (64, [700, 300], [300, 40]), (256, [500], [200])])
def test_the_range_of_values(d, lens, new, power):
    """bf16 values of about 2^power under scores that climb by up to 2^15 from the first tokens to the last:
    an output is a mean of values, finite wherever they leave fp32 room for the sum over the tokens. Off by
    at most paged_ref.attention_tolerance, in units of 2^power (what fp32 does not hold below 2^-126 adds
    2^-149 a token to a sum of weights of 2^-16 at least: 2^-123 for 1000 tokens)."""
    c = _case("bf16", d, 2, 2, 16, lens, new, seed=7)
    rng = np.random.default_rng(7)
    scale = _set_scores(c, [np.sort(rng.uniform(0, 15, n)) for n in lens])
    unit = c["pool"].clone()
    c["pool"][1] = (c["pool"][1].double() * 2.0 ** power).to(c["pool"].dtype)
    unit[1] = (c["pool"][1].double() * 2.0 ** -power).to(unit.dtype)
    out, lse = _attend(c, scale)
    want, wl, mag, big = ref.attention(num(c["q"]), num(unit), c["table"], c["lens"], c["cu"], 2, scale)
    to, tl = ref.attention_tolerance(False, d, want, mag, big)
    got = num(out) * 2.0 ** -power
    assert np.isfinite(got).all()
    err, to = np.abs(got - want), to + 2.0 ** (-123 - power) + 2.0 ** (-133 - power)
    assert (err <= to).all(), f"worst error / bound {(err / to).max():.3g}"
    assert (np.abs(num(lse) - wl) <= tl + 2.0 ** -22 * np.abs(wl)).all()
