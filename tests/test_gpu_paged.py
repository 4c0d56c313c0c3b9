"""The paged operators on the GPU against their plain 64-bit forms (paged_ref.py): page plan and
release, rotary and its append into the pool, attention over the pages. Tolerances are derived in
paged_ref.attention_tolerance and beside the rotary tests; whole numbers are equal."""
import numpy as np
import pytest

import paged_ref as ref

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")

pytestmark = pytest.mark.gpu

RANGE, EXHAUSTED = 16, 8
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


def num(t):
    return t.detach().cpu().to(torch.float64).numpy()


# ------------------------------------------------------------------------------------ plan
def _plan(page, n_pages, ctx, new, free_pages, free_count, table, n_tok):
    r = len(ctx)
    pages = cg.Pages(n_pages=n_pages, page=page, n_req=r, max_pages=table.shape[1])
    bt = i32(table)
    out = [torch.full((r,), 77, dtype=torch.int32, device="cuda"), torch.full((r + 1,), 77, dtype=torch.int32, device="cuda"),
           torch.full((n_tok,), 77, dtype=torch.int32, device="cuda"), torch.full((n_tok,), 77, dtype=torch.int64, device="cuda"),
           torch.full((1,), 77, dtype=torch.int32, device="cuda")]
    stack = np.concatenate([np.asarray(free_pages, np.int32), np.full(n_pages - len(free_pages), -9, np.int32)])
    cg.page_plan(pages, i32(ctx), i32(new), i32(stack), i32([free_count]), bt, *out)
    return [x.cpu().numpy() for x in (bt, *out)]


def _table_for(page, ctx, new, rng, spare):
    have = [-(-c // page) for c in ctx]
    total = sum(-(-(c + n) // page) for c, n in zip(ctx, new)) + spare
    perm = rng.permutation(total)
    table = np.full((len(ctx), max(-(-(c + n) // page) for c, n in zip(ctx, new)) + 2), -1)
    at = 0
    for i, h in enumerate(have):
        table[i, :h] = perm[at:at + h]
        at += h
    return table, perm[at:], total


@pytest.mark.parametrize("n_req,page,ctx_max,new_max,pad", [
    (1, 16, 0, 1, 0), (1, 64, 100, 0, 3), (3, 16, 40, 20, 0), (256, 64, 9000, 1, 0), (333, 16, 900, 70, 5),
    (2048, 32, 100, 3, 1), (2049, 16, 50, 3, 0), (5000, 256, 300, 2, 1111), (7, 128, 5, 5000, 0),
])
def test_plan(n_req, page, ctx_max, new_max, pad):
    rng = np.random.default_rng(n_req)
    ctx = rng.integers(0, ctx_max + 1, n_req)
    new = rng.integers(0, new_max + 1, n_req) if new_max > 1 else np.full(n_req, new_max)
    table, free, n_pages = _table_for(page, ctx, new, rng, spare=3)
    n_tok = int(new.sum()) + pad
    got = _plan(page, n_pages, ctx, new, free, len(free), table, n_tok)
    want = ref.plan(page, n_pages, ctx, new, free, len(free), table, n_tok)
    assert cg.get_status() == 0
    for g, w, what in zip(got, want, ("block_table", "seq_lens", "cu_new", "positions", "slots", "free_left")):
        assert np.array_equal(g, np.asarray(w).reshape(g.shape)), what


def test_plan_out_of_pages():
    """Tokens whose page is lacking get slot -1, free_left says how many pages lack; what was read is
    unchanged, so the plan can be made again with fewer tokens."""
    table = np.full((2, 4), -1)
    table[0, 0] = 5
    bt, lens, cu, pos, slots, left = _plan(16, 8, [10, 0], [30, 20], [3], 1, table, 50)
    assert cg.get_status() == EXHAUSTED
    assert left[0] == 1 - 4 and list(lens) == [40, 20] and list(cu) == [0, 30, 50]
    assert bt[0, 0] == 5 and bt[0, 1] == 3
    assert list(slots[:6]) == [5 * 16 + k for k in range(10, 16)] and list(slots[6:22]) == [3 * 16 + k for k in range(16)]
    assert (slots[22:] == -1).all() and pos[22] == 32


def test_plan_bad_lengths():
    table = np.full((4, 2), -1)
    # a negative length, a negative number of new tokens, one that outgrows its two pages, more than n_tok
    bt, lens, cu, pos, slots, left = _plan(16, 8, [-3, 0, 0, 0], [2, -1, 40, 99], [0, 1, 2, 3, 4], 5, table, 42)
    assert cg.get_status() == RANGE
    assert list(cu) == [0, 2, 2, 42, 42] and (slots[2:34] >= 0).all() and (slots[34:] == -1).all()
    # a free stack that holds a page the pool has not
    bt, lens, cu, pos, slots, left = _plan(16, 4, [0], [1], [9], 1, np.full((1, 1), -1), 1)
    assert cg.get_status() == RANGE and slots[0] == -1
    # a table entry of a token already held that is no page
    _, _, _, _, slots, _ = _plan(16, 4, [3], [1], [1], 1, np.full((1, 1), 4), 1)
    assert cg.get_status() == RANGE and slots[0] == -1


@pytest.mark.parametrize("n_req,page", [(1, 16), (50, 16), (2100, 64)])
def test_release(n_req, page):
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 200, n_req)
    table, free, n_pages = _table_for(page, lens, np.zeros(n_req, int), rng, spare=4)
    done = (rng.random(n_req) < 0.4).astype(np.int32)
    stack = i32(np.concatenate([free, np.full(n_pages - len(free), -9)]))
    left, lens_left = i32([77]), i32(np.full(n_req, 77))
    pages = cg.Pages(n_pages=n_pages, page=page, n_req=n_req, max_pages=table.shape[1])
    cg.page_release(pages, i32(lens), i32(done), i32(table), stack, i32([len(free)]), lens_left, left)
    assert cg.get_status() == 0
    back = [int(table[i, j]) for i in range(n_req) if done[i] for j in range(-(-int(lens[i]) // page))]
    assert left.item() == len(free) + len(back)
    assert stack.cpu().tolist() == list(free) + back + [-9] * (n_pages - len(free) - len(back))
    assert lens_left.cpu().tolist() == [0 if f else int(x) for x, f in zip(lens, done)]


# ------------------------------------------------------------------------------------ rotary
def _unit(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,rot,inter,transpose", [(128, 128, False, False), (128, 128, True, False), (128, 32, False, True),
                                                   (64, 16, True, True), (64, 64, False, False), (256, 240, True, False),
                                                   (256, 256, False, True), (128, 0, False, False)])
def test_rotary(dtype, d, rot, inter, transpose):
    """Cosine and sine are within 2^-22 (the angle's fraction is rounded at 2^-25 of a turn: 2^-22 of a
    radian; sincospi adds 2^-23); products and sums add a few 2^-24; the result is rounded once (u)."""
    rng = np.random.default_rng(d + rot)
    n, heads = 9, 3
    pos = np.array([0, 1, 2, 77, 4095, 131071, 10 ** 6 + 1, 2 ** 24 + 1, 2 ** 31 - 1])
    x = torch.from_numpy(rng.normal(size=(n, heads, d))).to(DT[dtype]).cuda()
    table, m = cg.rotary_table(rot, cg.RopeScaling(3, 500000.0, 4.0, 8192.0, 1.0, 32.0)) if rot else (torch.empty(0, dtype=torch.int64).cuda(), 1.0)
    out = torch.empty_like(x)
    cg.rotary(cg.Rotary(rot, inter, m, transpose), x, i32(pos), table, out)
    want = ref.rotate(num(x), pos, table.cpu().tolist(), inter, m, transpose)
    pair = np.abs(num(x)).max() * 2 * m
    assert (np.abs(num(out) - want) <= _unit(dtype) * np.abs(want) + 2.0 ** -20 * pair + 2.0 ** -24).all()
    assert np.array_equal(num(out)[..., rot:], num(x)[..., rot:])
    cg.rotary(cg.Rotary(rot, inter, m, transpose), x, i32(pos), table, x)      # in place
    assert torch.equal(x, out)


@pytest.mark.parametrize("inter", [False, True])
def test_rotary_transpose_is_the_gradient(inter):
    """<R x, y> = <x, R^T y> (each side off by the rounding of 16-bit results), and R^T y against the
    differences of <R x, y> in x, channel by channel: the map is linear, so a step of 1 has no error of
    its own and the two roundings of R (x + e) and R x bound it."""
    rng = np.random.default_rng(5)
    d, rot = 64, 48
    table, m = cg.rotary_table(rot, cg.RopeScaling(base=100.0))
    fwd, bwd = cg.Rotary(rot, inter, 1.25), cg.Rotary(rot, inter, 1.25, True)
    x, y = (torch.from_numpy(rng.normal(size=(1, 1, d))).to(torch.float16).cuda() for _ in range(2))
    pos, u = i32([12345]), 2.0 ** -11
    gx = torch.empty_like(x)
    cg.rotary(bwd, y, pos, table, gx)
    steps = x.expand(d + 1, 1, d).clone()
    steps[torch.arange(d), 0, torch.arange(d)] += 1
    out = torch.empty_like(steps)
    cg.rotary(fwd, steps, pos.expand(d + 1).contiguous(), table, out)
    moved = num(steps)[:d, 0] - num(steps)[d:, 0]                       # the step after its own rounding
    diff = (num(out)[:d, 0] - num(out)[d:, 0]) @ num(y)[0, 0] / moved[np.arange(d), np.arange(d)]
    bound = 2 * u * (np.abs(num(out)).max(0)[0] @ np.abs(num(y)[0, 0])) + u * np.abs(num(gx)[0, 0]) + 1e-5
    assert (np.abs(diff - num(gx)[0, 0]) <= bound).all()
    a, b = float((num(out)[d, 0] * num(y)[0, 0]).sum()), float((num(x)[0, 0] * num(gx)[0, 0]).sum())
    assert abs(a - b) <= u * (np.abs(num(out)[d, 0] * num(y)[0, 0]).sum() + np.abs(num(x)[0, 0] * num(gx)[0, 0]).sum()) + 1e-4
    want = ref.rotate(num(y), [12345], table.cpu().tolist(), inter, 1.25, True)
    assert (np.abs(want - num(gx)) <= u * np.abs(want) + 2.0 ** -18).all()


@pytest.mark.parametrize("dtype,d,rot,H,rep,page,n", [("bf16", 128, 128, 2, 4, 64, 1), ("fp16", 64, 32, 3, 5, 16, 70),
                                                       ("bf16", 256, 64, 1, 1, 32, 33), ("bf16", 128, 64, 5, 7, 256, 300)])
def test_rotary_append(dtype, d, rot, H, rep, page, n):
    """Slices of a fused projection in, queries out with another order of dimensions, keys and values at
    their slots; slot -1 and a slot outside the pool write nothing."""
    rng = np.random.default_rng(n)
    n_pages, hq = -(-n // page) + 2, H * rep
    qkv = torch.from_numpy(rng.normal(size=(n, (hq + 2 * H) * d))).to(DT[dtype]).cuda()
    q, k, v = (t.view(n, -1, d) for t in qkv.split([hq * d, H * d, H * d], 1))
    pool = torch.from_numpy(rng.normal(size=(2, n_pages, H, page, d))).to(DT[dtype]).cuda()
    before = num(pool)
    slots = rng.permutation(n_pages * page)[:n]
    bad = n > 3
    if bad:
        slots[1], slots[2] = -1, n_pages * page
    pos = rng.integers(0, 50000, n)
    table, _ = cg.rotary_table(rot)
    out = torch.empty(hq, n, d, dtype=DT[dtype], device="cuda").transpose(0, 1)
    pages = cg.Pages(n_pages=n_pages, page=page, H=H, d=d)
    cg.rotary_append(pages, cg.Rotary(rot), q, k, v, i32(pos), torch.from_numpy(slots).cuda(), table, out, pool)
    assert cg.get_status() == (RANGE if bad else 0)
    T = table.cpu().tolist()
    near = lambda got, want: (np.abs(got - want) <= _unit(dtype) * np.abs(want) + 2.0 ** -18).all()  # noqa: E731
    assert near(num(out), ref.rotate(num(q), pos, T, False))
    want, keys = before.copy(), ref.rotate(num(k), pos, T, False)
    for t, s in enumerate(slots):
        if 0 <= s < n_pages * page:
            want[0, s // page, :, s % page], want[1, s // page, :, s % page] = keys[t], num(v)[t]
    got = num(pool)
    assert near(got[0], want[0]) and np.array_equal(got[1], want[1])
    touched = np.zeros(n_pages * page, bool)
    touched[[s for s in slots if 0 <= s < n_pages * page]] = True
    rows = got[0].transpose(0, 2, 1, 3).reshape(n_pages * page, -1)
    assert np.array_equal(rows[~touched], before[0].transpose(0, 2, 1, 3).reshape(n_pages * page, -1)[~touched])
    # keys and values alone, and queries in place
    pool2 = torch.from_numpy(before).to(DT[dtype]).cuda()
    cg.rotary_append(pages, cg.Rotary(rot), None, k, v, i32(pos), torch.from_numpy(slots).cuda(), table, None, pool2)
    cg.rotary_append(pages, cg.Rotary(rot), q, k, v, i32(pos), torch.from_numpy(slots).cuda(), table, q, pool2)
    cg.get_status()
    assert torch.equal(pool2, pool) and torch.equal(q, out)


# ------------------------------------------------------------------------------------ attention
def _case(dtype, d, H, rep, page, lens, new, window=0, sinks=0, seed=0, poison=False, spread=1.0):
    """A pool whose used pages hold keys and values; with poison, everything that no query sees holds
    NaN and pages that no query needs have no entry in the table."""
    rng = np.random.default_rng(seed)
    r, n = len(lens), int(sum(new))
    need = [-(-x // page) for x in lens]
    n_pages = sum(need) + 2
    table = np.full((r, max(need) + 1), -1)
    perm, at = rng.permutation(n_pages), 0
    for i, k in enumerate(need):
        table[i, :k] = perm[at:at + k]
        at += k
    pool = torch.from_numpy(rng.normal(size=(2, n_pages, H, page, d)) * np.array([spread, 1.0]).reshape(2, 1, 1, 1, 1)).to(DT[dtype])
    cu = np.concatenate([[0], np.cumsum(new)]).astype(int)
    q = torch.from_numpy(rng.normal(size=(n, H * rep, d))).to(DT[dtype])
    if poison:
        seen = np.zeros((n_pages, page), bool)
        for i in range(r):
            for p in range(max(0, lens[i] - new[i]), lens[i]):
                t = np.arange(p + 1)
                if window:
                    t = t[(t > p - window) | (t < sinks)]
                seen[table[i, t // page], t % page] = True
        keep = torch.from_numpy(seen)[None, :, None, :, None]
        pool = torch.where(keep, pool, torch.full((), float("nan"), dtype=pool.dtype))
        for i in range(r):
            for j in range(need[i]):
                if not seen[table[i, j]].any():
                    table[i, j] = -1
    return dict(dtype=dtype, q=q, pool=pool, table=table, lens=list(lens), cu=cu, H=H, rep=rep, d=d, page=page, window=window, sinks=sinks)


def _attend(c, scale=None, stream=None, q=None, out=None, lse=True, max_new=None):
    scale = c["d"] ** -0.5 if scale is None else scale
    pages = cg.Pages(n_pages=c["pool"].shape[1], page=c["page"], H=c["H"], d=c["d"], n_req=len(c["lens"]), max_pages=c["table"].shape[1])
    n = c["q"].shape[0]
    new = np.diff(c["cu"])
    how = cg.PagedAttention(c["rep"], int(new.max()) if max_new is None else max_new, scale, c["window"], c["sinks"])
    q = c["q"].cuda() if q is None else q
    out = torch.full_like(q, float("nan")) if out is None else out
    lse = torch.full((n, c["H"] * c["rep"]), float("nan"), device="cuda") if lse else None
    cg.paged_attention(pages, how, q, c["pool"].cuda(), i32(c["table"]), i32(c["lens"]), i32(c["cu"]), out, lse)
    return out, lse


def _check(c, out, lse, scale=None):
    scale = c["d"] ** -0.5 if scale is None else scale
    want, wl, mag, big = ref.attention(num(c["q"]), num(c["pool"]), c["table"], c["lens"], c["cu"], c["rep"], scale, c["window"], c["sinks"])
    to, tl = ref.attention_tolerance(c["dtype"] == "fp16", c["d"], want, mag, big)
    got = num(out)
    assert np.isfinite(got).all()
    err = np.abs(got - want)
    assert (err <= to).all(), f"worst error / bound {(err / to).max():.3g}"
    if lse is not None:
        gl, none = num(lse), np.isinf(wl)
        assert np.array_equal(np.isneginf(gl), none)
        assert (np.abs(gl - wl)[~none] <= (tl + 2.0 ** -22 * np.abs(np.where(none, 0, wl)))[~none]).all()


CASES = {
    # one token of one request: lengths around tile and page ends
    "one_1": dict(lens=[1], new=[1]), "one_2": dict(lens=[2], new=[1]), "one_63": dict(lens=[63], new=[1]),
    "one_64": dict(lens=[64], new=[1]), "one_65": dict(lens=[65], new=[1], page=16), "one_1000": dict(lens=[1000], new=[1], page=16),
    "one_5000": dict(lens=[5000], new=[1], H=1, rep=8, page=256),
    # ragged decode batches, each head layout
    "decode_rep1": dict(lens=[5, 700, 64, 129, 1, 333], new=[1] * 6, rep=1, page=32),
    "decode_rep7_fp16": dict(lens=[5, 700, 64, 129, 1, 333], new=[1] * 6, rep=7, dtype="fp16", H=3),
    "decode_rep16": dict(lens=[90, 300], new=[1, 1], rep=16), "decode_rep17": dict(lens=[90, 300], new=[1, 1], rep=17, H=1),
    "decode_rep64": dict(lens=[200, 70], new=[1, 1], rep=64, H=1),
    "decode_d64": dict(lens=[5, 700, 64], new=[1] * 3, d=64, page=128), "decode_d256": dict(lens=[5, 700, 64], new=[1] * 3, d=256),
    "decode_d256_fp16": dict(lens=[257, 31], new=[1] * 2, d=256, dtype="fp16", page=16),
    # a few new tokens, none for some requests, a request without tokens
    "few": dict(lens=[40, 3, 130, 77], new=[2, 3, 0, 4], rep=4), "none_held": dict(lens=[0, 20, 0], new=[0, 1, 0]),
    "few_odd": dict(lens=[100, 101, 102], new=[5, 3, 7], rep=3, dtype="fp16", page=16, d=64),
    # chunks and whole prompts
    "prompt_17": dict(lens=[17], new=[17]), "prompt_128": dict(lens=[128], new=[128], H=1, rep=2), "prompt_300": dict(lens=[300], new=[300], H=1, rep=3),
    "chunk_64_after_200": dict(lens=[264], new=[64], H=1, page=16), "chunks": dict(lens=[150, 400, 90], new=[37, 130, 90], H=1, rep=4, dtype="fp16"),
    "chunk_d64": dict(lens=[150, 333], new=[37, 70], d=64, rep=5, H=2, page=16), "chunk_d256": dict(lens=[150, 200], new=[37, 40], d=256, rep=2, H=1),
    "chunk_rep64": dict(lens=[40], new=[9], rep=64, H=1), "chunk_rep33": dict(lens=[300], new=[20], rep=33, H=1, d=64),
    "mixed": dict(lens=[600, 1, 90, 257], new=[1, 1, 90, 1], H=2), "mixed_d64": dict(lens=[600, 31, 90, 257], new=[1, 31, 40, 1], H=2, d=64, dtype="fp16", page=16),
    # windows and sinks
    "window_1": dict(lens=[100, 7], new=[1, 7], window=1), "window_decode": dict(lens=[1000, 40, 130], new=[1] * 3, window=100, sinks=4, page=16),
    "window_only_sinks_far": dict(lens=[900], new=[1], window=5, sinks=130, page=16), "window_chunk": dict(lens=[700, 300], new=[100, 50], window=64, sinks=3, H=1, page=16),
    "window_chunk_fp16_d64": dict(lens=[500, 260], new=[200, 33], window=150, sinks=70, H=1, d=64, dtype="fp16"),
    "window_longer_than_all": dict(lens=[80, 30], new=[4, 30], window=5000, sinks=2),
    "window_chunk_d256": dict(lens=[300], new=[60], window=90, sinks=5, d=256, H=1, rep=3),
    # concentrated and wide scores
    "peaked": dict(lens=[500, 90], new=[1, 40], spread=8.0, H=1), "peaked_fp16": dict(lens=[500, 90], new=[1, 40], spread=8.0, H=1, dtype="fp16"),
}


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("poison", [False, True])
def test_attention(name, poison):
    kw = dict(dtype="bf16", d=128, H=2, rep=4, page=64)
    kw.update(CASES[name])
    c = _case(**kw, seed=len(name), poison=poison)
    out, lse = _attend(c)
    assert cg.get_status() == 0
    _check(c, out, lse)


@pytest.mark.parametrize("scale", [-0.1, 0.0, 1e-3, 3.0])
def test_attention_scales(scale):
    c = _case("bf16", 128, 1, 4, 32, [300, 90], [1, 40], seed=8)
    _check(c, *_attend(c, scale), scale)


def test_rows_that_see_nothing():
    """More new tokens than tokens: the first rows stand before the request and see nothing."""
    for new, rep in ((5, 2), (40, 4)):
        c = _case("bf16", 128, 2, rep, 16, [3, 20], [new, 1], seed=9)
        out, lse = _attend(c)
        _check(c, out, lse)
        assert (out[:new - 3] == 0).all() and torch.isneginf(lse[:new - 3]).all()
        c["lens"] = [0, 20]
        out, lse = _attend(c)
        assert (out[:new] == 0).all() and torch.isneginf(lse[:new]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rep,new", [(2, 6), (4, 60)])
def test_special_values_reach_only_rows_that_see_them(dtype, rep, new):
    """Infinities and NaN in values (and keys) of new tokens: rows before them are as if they were not
    there, rows that see them get what the sum of p v gives."""
    c = _case(dtype, 128, 1, rep, 16, [new + 100], [new], seed=11)
    clean, _ = _attend(c)
    at, h = 100 + new // 2, 0
    pg, off = c["table"][0, at // 16], at % 16
    c["pool"][1, pg, h, off, 3] = float("inf")
    c["pool"][1, pg, h, off, 5] = float("nan")
    c["pool"][1, pg, h, off, 64] = float("-inf")
    out, _ = _attend(c)
    k = new // 2
    assert torch.equal(out[:k], clean[:k])
    assert torch.isposinf(out[k:, :, 3]).all() and torch.isnan(out[k:, :, 5]).all() and torch.isneginf(out[k:, :, 64]).all()
    rest = [x for x in range(128) if x not in (3, 5, 64)]
    assert torch.equal(out[k:, :, rest], clean[k:, :, rest])
    c["pool"][0, pg, h, off, 7] = float("nan")             # a key too: every row that sees it is NaN
    out, lse = _attend(c)
    assert torch.equal(out[:k], clean[:k]) and torch.isnan(out[k:]).all() and torch.isnan(lse[k:]).all()
    assert cg.get_status() == 0


@pytest.mark.parametrize("lens,new", [([300, 40], [1, 1]), ([300, 90], [60, 45])])
def test_strides_streams_and_no_lse(lens, new):
    """Queries inside a fused projection, outputs head-major, a stream of the caller's own."""
    c = _case("bf16", 128, 2, 4, 64, lens, new, seed=12)
    want, _ = _attend(c)
    n, hq = c["q"].shape[:2]
    fused = torch.full((n, hq + 3, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    fused[:, 2:2 + hq] = c["q"].cuda()
    out = torch.full((hq, n, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = _attend(c, q=fused[:, 2:2 + hq], out=out.transpose(0, 1), lse=False)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("lens,new", [([300, 40], [1, 1]), ([300, 90], [60, 45])])
def test_graph_replay_follows_the_lengths(lens, new):
    """A captured call reads lengths and tables on the device: replayed after they change."""
    c = _case("bf16", 128, 2, 4, 64, lens, new, seed=13)
    pages = cg.Pages(n_pages=c["pool"].shape[1], page=64, H=2, d=128, n_req=2, max_pages=c["table"].shape[1])
    how = cg.PagedAttention(4, max(new), 128 ** -0.5)
    q, pool, table, ln, cu = c["q"].cuda(), c["pool"].cuda(), i32(c["table"]), i32(c["lens"]), i32(c["cu"])
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    ws = torch.empty(cg.paged_attention_workspace_bytes(pages, how, q.shape[0]), dtype=torch.uint8, device="cuda")
    call = lambda: cg.paged_attention(pages, how, q, pool, table, ln, cu, out, lse, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for cut in (0, 1, 30):
        c["lens"] = [max(x - cut, n) for x, n in zip(lens, new)]
        ln.copy_(i32(c["lens"]))
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        _check(c, out, lse)


def test_same_inputs_same_bits():
    for lens, new in (([3000, 40, 777], [1, 1, 1]), ([700, 90], [200, 45])):
        c = _case("bf16", 128, 2, 4, 64, lens, new, seed=14)
        a, la = _attend(c)
        for _ in range(3):
            b, lb = _attend(c)
            assert torch.equal(a, b) and torch.equal(la, lb)


def test_bad_tables_and_lengths_raise_the_flag():
    c = _case("bf16", 128, 1, 2, 16, [100, 50], [1, 1], seed=15)
    _attend(c)
    assert cg.get_status() == 0
    good = c["table"].copy()
    for bad in (-1, c["pool"].shape[1], 2 ** 31 - 1, -2 ** 31):
        c["table"] = good.copy()
        c["table"][0, 2] = bad
        out, _ = _attend(c)
        assert cg.get_status() == RANGE
    c["table"] = good
    clean, _ = _attend(c)
    for lens, cu in (([10 ** 6, 50], [0, 1, 2]), ([-4, 50], [0, 1, 2]), ([100, 50], [0, 5, 2])):
        d = dict(c, lens=lens, cu=np.array(cu))
        out, _ = _attend(d, max_new=1)
        assert cg.get_status() == RANGE
        if cu == [0, 1, 2]:
            assert torch.isnan(out[0]).all() and torch.equal(out[1], clean[1])
    d = _case("bf16", 128, 1, 2, 16, [100, 50], [9, 1], seed=15)      # more new tokens than max_new
    out, _ = _attend(d, max_new=4)
    assert cg.get_status() == RANGE and torch.isnan(out[:9]).all()


@pytest.mark.parametrize("lens,new", [([300, 900], [1, 1]), ([300, 900], [30, 200])])
def test_offsets_past_32_bits(lens, new):
    """Pages at the end of a pool of more than 2^32 bytes (and 2^31 elements) in each half."""
    c = _case("bf16", 128, 8, 2, 64, lens, new, seed=16)
    n_big = (1 << 32) // (8 * 64 * 128 * 2) + 40
    pool = torch.zeros(2, n_big, 8, 64, 128, dtype=torch.bfloat16, device="cuda")
    k = c["pool"].shape[1]
    pool[:, n_big - k:] = c["pool"].cuda()
    want, wl = _attend(c)
    big = dict(c, table=np.where(c["table"] >= 0, c["table"] + n_big - k, -1))
    pages = cg.Pages(n_pages=n_big, page=64, H=8, d=128, n_req=2, max_pages=c["table"].shape[1])
    q = c["q"].cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    cg.paged_attention(pages, cg.PagedAttention(2, max(new), 128 ** -0.5), q, pool, i32(big["table"]), i32(c["lens"]), i32(c["cu"]), out, lse)
    assert torch.equal(out, want) and torch.equal(lse, wl)
    # the append writes there too
    slots = torch.tensor([n_big * 64 - 1, n_big * 64 - 70], device="cuda")
    kv = torch.randn(2, 2, 8, 128, device="cuda").bfloat16()
    table, _ = cg.rotary_table(128)
    cg.rotary_append(pages, cg.Rotary(128), None, kv[0], kv[1], i32([0, 0]), slots, table, None, pool)
    assert cg.get_status() == 0
    assert torch.equal(pool[0, -1, :, 63], kv[0, 0]) and torch.equal(pool[1, -2, :, 58], kv[1, 1])


def test_binding_refusals():
    c = _case("bf16", 128, 2, 4, 64, [30], [1])
    q = c["q"].cuda()
    for kw in (dict(q=q.float()), dict(q=q[:, :4]), dict(out=q.half()), dict(q=q.transpose(1, 2)), dict(q=q.cpu())):
        with pytest.raises(cg.CodecGaugeError) as e:
            _attend(c, **kw)
        assert e.value.code == -1
    pages = cg.Pages(n_pages=c["pool"].shape[1], page=64, H=2, d=128, n_req=1, max_pages=2)
    out, lens, cu, table = torch.empty_like(q), i32([30]), i32([0, 1]), i32(c["table"])
    how = cg.PagedAttention(4, 1, 0.1)
    for bad in (dict(pool=c["pool"].cuda().half()), dict(pool=c["pool"]), dict(table=table.long()), dict(lens=lens[:0]),
                dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        kw = dict(pool=c["pool"].cuda(), table=table, lens=lens, workspace=None)
        kw.update(bad)
        with pytest.raises(cg.CodecGaugeError):
            cg.paged_attention(pages, how, q, kw["pool"], kw["table"], kw["lens"], cu, out, None, kw["workspace"])


@pytest.mark.parametrize("rep,new", [(4, 1), (4, 50), (7, 50)])
def test_broadcast_queries(rep, new):
    """Queries whose token or head stride is 0 (one query for every head, or for every token)."""
    c = _case("bf16", 128, 2, rep, 16, [new + 70], [new], seed=17)
    q = c["q"].cuda()
    for b in (q[:, :1].expand(-1, 2 * rep, -1), q[:1].expand(new, -1, -1), q[:1, :1].expand(new, 2 * rep, -1)):
        got, lse = _attend(c, q=b, out=torch.full_like(q, float("nan")))
        _check(dict(c, q=b.contiguous().cpu()), got, lse)


@pytest.mark.parametrize("rep", [1, 2, 3, 5, 6, 7, 9, 11, 16, 17, 31, 48, 63])
def test_every_head_group(rep):
    """Rows per tile are whole tokens of n_rep rows, which leaves some of the 128 empty."""
    c = _case("bf16", 64, 1, rep, 16, [300, 20], [290, 3], seed=rep)
    _check(c, *_attend(c))


@pytest.mark.parametrize("kw", [dict(lens=[9000], new=[64], H=8), dict(lens=[3000, 700, 2100], new=[300, 500, 41], H=2, window=600, sinks=5, rep=7, page=16),
                                dict(lens=[4000, 900], new=[60, 900], H=2, d=64, page=16)])
def test_many_calls_in_a_row(kw):
    """No wait of the pipelines gives up, and every call gives the same bits, over many calls on two
    caches in turn (copies land in any order)."""
    base = dict(dtype="bf16", d=128, rep=4, page=64)
    base.update(kw)
    cases = [_case(**base, seed=s) for s in (21, 22)]
    state = []
    for c in cases:
        pages = cg.Pages(n_pages=c["pool"].shape[1], page=c["page"], H=c["H"], d=c["d"], n_req=len(c["lens"]), max_pages=c["table"].shape[1])
        how = cg.PagedAttention(c["rep"], int(np.diff(c["cu"]).max()), c["d"] ** -0.5, c["window"], c["sinks"])
        q = c["q"].cuda()
        state.append((pages, how, q, c["pool"].cuda(), i32(c["table"]), i32(c["lens"]), i32(c["cu"]), torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")))
        cg.paged_attention(*state[-1])
    first = [(s[7].clone(), s[8].clone()) for s in state]
    for k in range(400):
        cg.paged_attention(*state[k % 2])
        if k % 40 > 37:
            assert torch.equal(state[k % 2][7], first[k % 2][0]) and torch.equal(state[k % 2][8], first[k % 2][1])
    assert cg.get_status() == 0
    for c, f in zip(cases, first):
        _check(c, *f)
