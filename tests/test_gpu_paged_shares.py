"""How the paged attention's work is dealt to CTAs: a whole tile each, equal shares with cuts inside tiles,
between tiles and among a tile's start; many short tiles beside long ones. Against the 64-bit form, with
the bounds of paged_ref.attention_tolerance."""
import numpy as np
import pytest

from test_gpu_paged import _attend, _case, _check, cg

pytestmark = pytest.mark.gpu


def _ragged(n, lo, hi, new_hi, seed):
    rng = np.random.default_rng(seed)
    new = rng.integers(1, new_hi + 1, n)
    return [int(x) for x in rng.integers(lo, hi + 1, n) + new], [int(x) for x in new]


def _cases():
    out = {}
    # tiles of 128-row halves: as many as CTAs, a few more, fewer; one long request among short ones
    for name, n, H in (("fit", 38, 4), ("over", 39, 4), ("few", 7, 2), ("many", 90, 4)):
        lens, new = _ragged(n, 0, 300, 50, n)
        out["chunks_" + name] = dict(lens=lens, new=[max(x, 17) for x in new], H=H, rep=2, d=64)
        out["chunks_" + name]["lens"] = [a + max(b, 17) for a, b in zip(lens, new)]
    out["chunks_long_one"] = dict(lens=[2600] + [40] * 9, new=[90] + [40] * 9, H=2, rep=4)
    out["chunks_long_one_d256"] = dict(lens=[1500] + [40] * 4, new=[70] + [40] * 4, H=2, rep=2, d=256)
    out["chunks_window"] = dict(lens=[900, 1300, 64, 700], new=[300, 41, 64, 1], H=2, rep=7, window=150, sinks=3, page=16)
    # around the size where a prompt's tiles are cut
    for n in (255, 256, 600, 1100):
        out[f"prompt_{n}"] = dict(lens=[n], new=[n], H=3, rep=4, d=64)
    # tiles of 16 rows: very short ones, beside long ones, with and without a window
    lens, _ = _ragged(120, 0, 130, 1, 5)
    out["rows_short"] = dict(lens=lens, new=[1] * 120, H=4, rep=2)
    out["rows_short_and_long"] = dict(lens=lens[:60] + [9000], new=[1] * 61, H=4, rep=2, page=16)
    out["rows_window"] = dict(lens=lens[:50] + [3000, 5000], new=[1] * 52, H=4, rep=2, page=16, window=700, sinks=4)
    out["rows_four_tokens"] = dict(lens=[x + 4 for x in lens[:70]] + [2500], new=[4] * 71, H=2, rep=3)
    out["rows_one_chunk"] = dict(lens=[1 + i % 64 for i in range(200)], new=[1] * 200, H=2, rep=8)
    out["rows_d256"] = dict(lens=lens[:40] + [3000], new=[1] * 41, H=2, rep=2, d=256)
    return out


CASES = _cases()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("name", list(CASES))
def test_shares(name, dtype):
    kw = dict(dict(dtype=dtype, d=128, page=32, seed=len(name)), **CASES[name])
    c = _case(**kw)
    out, lse = _attend(c)
    _check(c, out, lse)
    again, lse2 = _attend(c)
    assert (again == out).all() and (lse2 == lse).all()
    assert cg.get_status() == 0


@pytest.mark.parametrize("d", [64, 128, 256])
def test_workspace_is_sized_once(d):
    """A workspace sized for many requests serves one, and one for the most rows serves fewer."""
    torch = pytest.importorskip("torch")
    pages = cg.Pages(n_pages=64, page=16, H=2, d=d, n_req=50, max_pages=40)
    sizes = [cg.paged_attention_workspace_bytes(pages, cg.PagedAttention(4, new, 0.1), 50 * new) for new in (1, 2, 3, 4, 5, 40)]
    assert sizes == sorted(sizes)
    for new in (1, 2, 4, 5, 40):
        c = _case("bf16", d, 2, 4, 16, [500], [new])
        one = cg.Pages(n_pages=c["pool"].shape[1], page=16, H=2, d=d, n_req=1, max_pages=c["table"].shape[1])
        how = cg.PagedAttention(4, new, d ** -0.5)
        ws = torch.empty(cg.paged_attention_workspace_bytes(pages, how, 50 * new), dtype=torch.uint8, device="cuda")
        q = c["q"].cuda()
        out, lse = torch.empty_like(q), torch.empty(new, 8, device="cuda")
        t = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
        cg.paged_attention(one, how, q, c["pool"].cuda(), t(c["table"]), t(c["lens"]), t(c["cu"]), out, lse, workspace=ws)
        _check(c, out, lse)
