"""The draft-tree operators on the GPU against their plain forms (tree_ref.py). Whole numbers and moved rows are equal;
the attention's tolerances are those of paged_ref.attention_tolerance, derived there."""
import numpy as np
import pytest

import paged_ref
import tree_ref as ref

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")

pytestmark = pytest.mark.gpu

RANGE = 16
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def i32(v):
    return torch.tensor(np.asarray(v).astype(np.int64), dtype=torch.int32).cuda() if np.asarray(v).dtype != np.uint32 \
        else torch.from_numpy(np.asarray(v).view(np.int32).copy()).cuda()


def num(t):
    return t.detach().cpu().to(torch.float64).numpy()


# ------------------------------------------------------------------------------------ plan
def _plan(parents, lens, cu, n_tok, words, max_new, window=0, sinks=0):
    pos = torch.full((n_tok,), 77, dtype=torch.int32, device="cuda")
    masks = torch.full((n_tok, words), 77, dtype=torch.int32, device="cuda")
    p = np.full(n_tok, 1 << 20)
    p[:len(parents)] = parents
    cg.tree_plan(max_new, i32(p), i32(lens), i32(cu), pos, masks, window, sinks)
    return pos.cpu().numpy(), masks.cpu().numpy().view(np.uint32)


@pytest.mark.parametrize("n_req,most,ctx,window,sinks,pad,more", [
    (1, 1, 0, 0, 0, 0, 0), (1, 8, 1000, 0, 0, 3, 0), (3, 31, 10, 0, 0, 0, 0), (3, 32, 10, 0, 0, 0, 0), (3, 33, 10, 0, 0, 2, 1), (40, 64, 500, 0, 0, 5, 0),
    (300, 70, 90, 7, 0, 0, 0), (300, 70, 9, 5, 12, 1, 2), (2, 700, 20, 33, 25, 0, 0), (5, 200, 0, 1, 0, 0, 0), (5, 90, 0, 2, 1, 400, 0),
])
def test_plan(n_req, most, ctx, window, sinks, pad, more):
    rng = np.random.default_rng(n_req + most)
    n = rng.integers(0, most + 1, n_req)
    n[-1] = most
    parents = [ref.random_parents(rng, k, rng.random()) for k in n]
    lens, cu = rng.integers(0, ctx + 1, n_req) + n, np.concatenate([[0], np.cumsum(n)])
    words, n_tok = -(-most // 32) + more, int(cu[-1]) + pad
    flat = [p for q in parents for p in q]
    got = _plan(flat, lens, cu, n_tok, words, most, window, sinks)
    assert cg.get_status() == 0
    want = ref.plan(flat, lens, cu, n_tok, words, window, sinks)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


@pytest.mark.parametrize("kind", ["chain", "star", "all_roots", "comb"])
def test_plan_of_the_largest_tree(kind):
    n = 8192
    k = np.arange(n)
    parents = {"chain": k - 1, "star": np.where(k, 0, -1), "all_roots": np.full(n, -1), "comb": np.where(k % 2, k - 1, k - 2)}[kind]
    parents[0] = -1
    got = _plan(parents, [n + 5], [0, n], n, 256, n, 0, 0)
    assert cg.get_status() == 0
    want = ref.plan(parents.tolist(), [n + 5], [0, n], n, 256)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_plan_of_what_does_not_fit():
    """Parents that are no earlier node count as -1; requests whose lengths do not fit have no nodes, and their rows
    are left as they are."""
    got = _plan([-1, 1, 0, -5, 9, 4], [8], [0, 6], 6, 1, 6)
    assert cg.get_status() == RANGE
    want = ref.plan([-1, -1, 0, -1, -1, 4], [8], [0, 6], 6, 1)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    # a negative length, more nodes than tokens, more than max_new
    for lens, cu, max_new in (([-1, 6], [0, 2, 4], 3), ([1, 6], [0, 2, 4], 3), ([9, 6], [0, 4, 6], 3), ([9, 6], [-2, 2, 4], 3), ([9, 6], [5, 2, 4], 3)):
        pos, masks = _plan([-1] * 6, lens, cu, 6, 1, max_new)
        assert cg.get_status() == RANGE
        assert (pos[2 if cu[0] <= 0 else 0:cu[1]] == 77).all()
        assert (pos[cu[1]:cu[2]] == 4).all() and (pos[cu[2]:] == 0).all() and (masks[cu[2]:] == 0).all()
    pos, _ = _plan([-1] * 6, [9, 6], [0, 2, 9], 6, 1, 3)              # more than the rows
    assert cg.get_status() == RANGE and (pos[:2] == 7).all() and (pos[2:] == 77).all()


# ------------------------------------------------------------------------------------ attention
def _case(dtype="bf16", d=128, H=2, rep=4, page=16, ctx=(70,), nodes=(9,), window=0, sinks=0, seed=0, spread=1.0, masks=None, pad=0):
    """Pools whose rows behind the requests hold NaN, and of windowed requests the pages that nobody sees too (their
    entries are -1); masks: a tree's, or any bits."""
    rng = np.random.default_rng(seed)
    ctx, nodes = np.array(ctx), np.array(nodes)
    lens, cu, r = ctx + nodes, np.concatenate([[0], np.cumsum(nodes)]), len(ctx)
    n, most, need = int(cu[-1]) + pad, int(max(nodes)), -(-lens // page)
    n_pages, words = int(need.sum()) + 2, max(1, -(-most // 32))
    perm, at = rng.permutation(n_pages), 0
    table = np.full((r, int(max(need)) + 1), -1)
    seen = np.zeros((n_pages, page), bool)
    for i in range(r):
        table[i, :need[i]] = perm[at:at + need[i]]
        at += need[i]
        t = np.arange(lens[i])
        if window and nodes[i]:
            t = t[(t > ctx[i] - window) | (t < sinks)]
        seen[table[i, t // page], t % page] = True
        for j in range(need[i]):
            if not seen[table[i, j]].any():
                table[i, j] = -1
    pool = torch.from_numpy(rng.normal(size=(2, n_pages, H, page, d)) * np.array([spread, 1.0]).reshape(2, 1, 1, 1, 1)).to(DT[dtype])
    pool = torch.where(torch.from_numpy(seen)[None, :, None, :, None], pool, torch.full((), float("nan"), dtype=pool.dtype))
    flat = [p for k in nodes for p in ref.random_parents(rng, k)]
    pos, tree = ref.plan(flat, lens, cu, n, words, window, sinks)
    if masks == "any":       # bits behind the last node among them, and rows without any
        tree = rng.integers(0, 1 << 32, (n, words), dtype=np.uint32)
        tree[rng.random(n) < 0.2] = 0
        pos = np.array([rng.integers(0, k + 1) for c in nodes for k in range(c)] + [0] * pad) + np.repeat(np.append(ctx, 0), np.append(nodes, pad))
    q = torch.from_numpy(rng.normal(size=(n, H * rep, d))).to(DT[dtype])
    return dict(dtype=dtype, q=q, pool=pool, table=table, lens=lens, cu=cu, H=H, rep=rep, d=d, page=page, window=window, sinks=sinks, pos=pos,
                masks=tree, most=most)


def _attend(c, scale=None, q=None, out=None, pool=None, **kw):
    scale = c["d"] ** -0.5 if scale is None else scale
    pages = cg.Pages(n_pages=c["pool"].shape[1], page=c["page"], H=c["H"], d=c["d"], n_req=len(c["lens"]), max_pages=c["table"].shape[1])
    how = cg.PagedAttention(c["rep"], c["most"], scale, c["window"], c["sinks"])
    q = c["q"].cuda() if q is None else q
    out = torch.full_like(q, 77.0) if out is None else out
    lse = torch.full(q.shape[:2], 77.0, device="cuda")
    cg.tree_attention(pages, how, q, c["pool"].cuda() if pool is None else pool, i32(c["table"]), i32(c["lens"]), i32(c["cu"]),
                      i32(c["pos"]) if c["window"] else None, i32(c["masks"]), out, lse, **kw)
    return out, lse


def _check(c, out, lse, scale=None):
    scale = c["d"] ** -0.5 if scale is None else scale
    n = int(c["cu"][-1])
    want, wl, mag, big = ref.attention(num(c["q"]), num(c["pool"]), c["table"], c["lens"], c["cu"], c["masks"], c["pos"], c["rep"], scale,
                                       c["window"], c["sinks"])
    to, tl = paged_ref.attention_tolerance(c["dtype"] == "fp16", c["d"], want, mag, big)
    got, gl, none = num(out)[:n], num(lse)[:n], np.isinf(wl)[:n]
    assert np.isfinite(got).all()
    err = np.abs(got - want[:n])
    assert (err <= to[:n]).all(), f"worst error / bound {(err / to[:n]).max():.3g}"
    assert np.array_equal(np.isneginf(gl), none)
    assert (np.abs(gl - wl[:n])[~none] <= (tl[:n] + 2.0 ** -22 * np.abs(np.where(none, 0, wl[:n])))[~none]).all()
    assert (num(out)[n:] == 77).all() and (num(lse)[n:] == 77).all()       # rows behind the last request


CASES = {
    "one_alone": dict(ctx=[0], nodes=[1], rep=1), "one_after_1": dict(ctx=[1], nodes=[1]), "one_after_63": dict(ctx=[63], nodes=[1], page=64),
    "pair_after_64": dict(ctx=[64], nodes=[2], page=64, rep=2), "no_history": dict(ctx=[0], nodes=[40]), "no_history_few": dict(ctx=[0, 0], nodes=[3, 2]),
    "few_rows": dict(ctx=[200, 5, 90], nodes=[3, 4, 1], rep=4), "few_rows_d64": dict(ctx=[200, 5, 90], nodes=[3, 4, 1], rep=4, d=64, dtype="fp16"),
    "few_rows_d256": dict(ctx=[200, 5, 90], nodes=[3, 4, 1], rep=4, d=256), "few_of_many": dict(ctx=[300, 20, 0, 131], nodes=[2, 40, 0, 16], rep=8, H=1),
    "nodes_over_words": dict(ctx=[50], nodes=[33], rep=1), "nodes_63": dict(ctx=[127], nodes=[63], rep=3, page=32), "nodes_64": dict(ctx=[128], nodes=[64], H=1),
    "nodes_65_fp16": dict(ctx=[129], nodes=[65], H=1, dtype="fp16"), "nodes_over_tiles": dict(ctx=[100], nodes=[150], H=1, rep=4),
    "nodes_500": dict(ctx=[17], nodes=[500], H=1, rep=1), "rep7": dict(ctx=[77, 300], nodes=[20, 37], rep=7, H=1), "rep33": dict(ctx=[30], nodes=[9], rep=33, H=1),
    "d64": dict(ctx=[300, 45], nodes=[60, 31], d=64, page=128), "d256": dict(ctx=[300, 45], nodes=[60, 31], d=256, H=1), "long": dict(ctx=[5000, 700], nodes=[12, 64], H=1),
    "d256_fp16_alone": dict(ctx=[260], nodes=[17], d=256, H=1, dtype="fp16", rep=2), "page256": dict(ctx=[255, 257], nodes=[2, 70], page=256, H=1),
    "window": dict(ctx=[500, 30], nodes=[30, 40], window=100, sinks=4), "window_few": dict(ctx=[500, 30], nodes=[3, 2], window=100, sinks=4),
    "window_1": dict(ctx=[90], nodes=[20], window=1), "window_in_tree": dict(ctx=[10, 0], nodes=[90, 70], window=5, sinks=12), "window_d64": dict(
        ctx=[400], nodes=[50], window=130, sinks=70, d=64, H=1, dtype="fp16"), "window_d256": dict(ctx=[400], nodes=[50], window=40, d=256, H=1, rep=2),
    "window_longer_than_all": dict(ctx=[40], nodes=[30], window=5000, sinks=3),
    "any": dict(ctx=[100, 0, 30], nodes=[50, 37, 4], masks="any"), "any_few": dict(ctx=[100, 0, 30], nodes=[2, 4, 3], masks="any"),
    "any_window": dict(ctx=[300, 0], nodes=[50, 37], masks="any", window=40, sinks=3, H=1), "any_few_window": dict(ctx=[300, 0], nodes=[4, 3], masks="any", window=40),
    "peaked": dict(ctx=[300, 40], nodes=[40, 3], spread=8.0, H=1), "peaked_fp16": dict(ctx=[300, 40], nodes=[40, 3], spread=8.0, H=1, dtype="fp16"),
    "padded": dict(ctx=[30, 40], nodes=[3, 20], pad=7),
}


@pytest.mark.parametrize("d", [64, 128, 256])
def test_every_cut_of_a_tree(d):
    """One tree after histories of one tile after the other: the shares of the CTAs begin and end at every place of a tile."""
    for ctx in list(range(120, 1700, 128)) + [127, 128, 129, 255, 256, 257, 3000]:
        c = _case(ctx=[ctx], nodes=[9], H=1, rep=3, d=d, seed=ctx)
        out, lse = _attend(c)
        assert cg.get_status() == 0
        _check(c, out, lse)


@pytest.mark.parametrize("name", list(CASES))
def test_attention(name):
    c = _case(**CASES[name], seed=len(name))
    out, lse = _attend(c)
    assert cg.get_status() == 0
    _check(c, out, lse)


@pytest.mark.parametrize("scale", [-0.1, 0.0, 2.0])
def test_attention_scales(scale):
    for nodes in ((40,), (3, 2)):
        c = _case(ctx=[90] * len(nodes), nodes=nodes, H=1)
        _check(c, *_attend(c, scale), scale)


def test_rows_that_see_nothing():
    for nodes in ([40], [3, 2]):
        c = _case(ctx=[0] * len(nodes), nodes=nodes)
        c["masks"][:] = 0
        out, lse = _attend(c)
        assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("nodes,dtype,d", [((60,), "bf16", 128), ((4, 3), "fp16", 128), ((50,), "fp16", 64), ((30,), "bf16", 256)])
def test_special_values_reach_who_sees_them(nodes, dtype, d):
    """Infinities and NaN in one node's key and value change the rows that see the node, and no bit of the others."""
    c = _case(dtype=dtype, d=d, ctx=[100] * len(nodes), nodes=nodes, H=1)
    clean, lse = _attend(c)
    j = 1
    sees = (c["masks"][:, 0] >> j & 1).astype(bool)
    sees[nodes[0]:] = False
    assert sees.any() and not sees.all()
    t = c["lens"][0] - nodes[0] + j
    at = (c["table"][0, t // c["page"]], 0, t % c["page"])
    for half, value in ((1, float("nan")), (1, float("inf")), (1, float("-inf")), (0, float("nan"))):
        pool = c["pool"].clone()
        pool[half][at] = value
        out, l2 = _attend(c, pool=pool.cuda())
        other = torch.from_numpy(~sees).cuda()
        assert torch.equal(out[other], clean[other]) and torch.equal(l2[other], lse[other])
        got = out[~other].float()
        assert (torch.isnan(got) if value != value else got == value).all()


def test_longer_rows_of_masks():
    """More words than the nodes need: their bits count for nothing."""
    for nodes in ([40, 3], [4, 2]):
        c = _case(ctx=[70, 300], nodes=nodes)
        want, lse = _attend(c)
        more = np.full((c["masks"].shape[0], 3), 0xffffffff, np.uint32)
        wide = dict(c, masks=np.concatenate([c["masks"], more], 1))
        out, l2 = _attend(wide)
        assert torch.equal(out, want) and torch.equal(l2, lse) and cg.get_status() == 0


def test_queries_shared_by_heads():
    """A stride of 0: one query for all heads of a token."""
    for nodes in ([50, 3], [4, 2]):
        c = _case(ctx=[70, 300], nodes=nodes)
        one = c["q"][:, :1].cuda()
        c["q"] = one.expand(-1, c["H"] * c["rep"], -1).contiguous().cpu()
        want, lse = _attend(c)
        out, l2 = _attend(c, q=one.expand(-1, c["H"] * c["rep"], -1), out=torch.full_like(want, 77.0))
        assert torch.equal(out, want) and torch.equal(l2, lse)
        _check(c, out, lse)


def test_plan_without_rows():
    got = _plan([], [3, 0], [0, 0, 0], 0, 1, 0)
    assert got[0].size == 0 and cg.get_status() == 0
    got = _plan([], [3, 0], [0, 0, 0], 4, 1, 5)
    assert (got[0] == 0).all() and (got[1] == 0).all() and cg.get_status() == 0


def test_a_chain_is_paged_attention():
    """With a chain's masks the rows see what paged_attention's see."""
    for ctx, nodes in (([100, 7], [30, 50]), ([100, 7], [2, 4])):
        c = _case(ctx=ctx, nodes=nodes)
        flat = [k - 1 for n in nodes for k in range(n)]
        c["pos"], c["masks"] = ref.plan(flat, c["lens"], c["cu"], int(c["cu"][-1]), c["masks"].shape[1])
        out, lse = _attend(c)
        pages = cg.Pages(n_pages=c["pool"].shape[1], page=c["page"], H=c["H"], d=c["d"], n_req=2, max_pages=c["table"].shape[1])
        plain, l2 = torch.empty_like(out), torch.empty_like(lse)
        cg.paged_attention(pages, cg.PagedAttention(c["rep"], c["most"], c["d"] ** -0.5), c["q"].cuda(), c["pool"].cuda(), i32(c["table"]),
                           i32(c["lens"]), i32(c["cu"]), plain, l2)
        _check(c, out, lse)
        _check(c, plain, l2)


def test_strides_streams_and_workspaces():
    """A slice of a fused projection in, heads-first out, on a side stream with its own workspace; the same twice."""
    c = _case(ctx=[300, 20, 90], nodes=[30, 3, 64])
    n, hq, d = c["q"].shape
    fused = torch.full((n, hq + 4, d), float("nan"), dtype=c["q"].dtype, device="cuda")
    fused[:, 2:2 + hq] = c["q"].cuda()
    out = torch.full((hq, n, d), 77.0, dtype=c["q"].dtype, device="cuda").transpose(0, 1)
    pages = cg.Pages(n_pages=c["pool"].shape[1], page=c["page"], H=c["H"], d=d, n_req=3, max_pages=c["table"].shape[1])
    ws = torch.empty(cg.paged_attention_workspace_bytes(pages, cg.PagedAttention(c["rep"], c["most"], 1.0), n), dtype=torch.uint8, device="cuda")
    pool = c["pool"].cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, lse = _attend(c, q=fused[:, 2:2 + hq], out=out, pool=pool, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    _check(c, got, lse)
    again, l2 = _attend(c, pool=pool)
    assert torch.equal(again, got) and torch.equal(lse, l2)


def test_attention_of_what_does_not_fit():
    for nodes in ([4, 3], [40, 30]):
        c = _case(ctx=[90, 60], nodes=nodes)
        bad = dict(c, lens=np.array([nodes[0] - 1, c["lens"][1]]))            # more nodes than tokens
        out, lse = _attend(bad)
        assert cg.get_status() == RANGE and (out[:nodes[0]] == 77).all() and (lse[:nodes[0]] == 77).all()
        good, l2 = _attend(c)
        assert cg.get_status() == 0 and torch.equal(out[nodes[0]:], good[nodes[0]:])
        c = _case(ctx=[90, 60], nodes=nodes, window=50)
        good, l2 = _attend(c)
        far = dict(c, pos=c["pos"].copy())
        far["pos"][0], far["pos"][1] = 10 ** 9, -5                            # count as the nearest that fit
        out, lse = _attend(far)
        assert cg.get_status() == RANGE
        far["pos"][0], far["pos"][1] = 90, 90
        _check(far, out, lse)
        assert cg.get_status() == 0


# ------------------------------------------------------------------------------------ commit
def _commit_case(n_req, page, ctx, most, layers, H, d, seed=0, dtype=torch.bfloat16):
    rng = np.random.default_rng(seed)
    nodes = rng.integers(0, most + 1, n_req)
    nodes[-1] = most
    held = rng.integers(0, ctx + 1, n_req)
    lens, cu = held + nodes, np.concatenate([[0], np.cumsum(nodes)])
    parents = [ref.random_parents(rng, k, rng.random()) for k in nodes]
    leaves = [int(rng.integers(-1, k)) if k else -1 for k in nodes]
    leaves[-1] = most - 1
    need = -(-lens // page)
    n_pages = int(need.sum()) + 5
    perm, at = rng.permutation(n_pages), 0
    table = np.full((n_req, int(max(need)) + 1), -1)
    for i in range(n_req):
        table[i, :need[i]] = perm[at:at + need[i]]
        at += need[i]
    stack = np.full(n_pages, -9)
    stack[:3] = perm[at:at + 3]
    pool = torch.from_numpy(rng.normal(size=(layers, 2, n_pages, H, page, d))).to(dtype)
    return dict(page=page, H=H, d=d, n_pages=n_pages, parents=[p for q in parents for p in q], leaves=leaves, lens=lens, cu=cu, table=table, pool=pool,
                stack=stack, count=3, most=most)


def _commit(c, rows=True, give=True, pool=None):
    pages = cg.Pages(n_pages=c["n_pages"], page=c["page"], H=c["H"], d=c["d"], n_req=len(c["lens"]), max_pages=c["table"].shape[1])
    pool = c["pool"].cuda() if pool is None else pool
    left, stack, free_left = i32(np.full(len(c["lens"]), 77)), i32(c["stack"]), i32([77])
    given = [left, stack, i32([c["count"]]), free_left] if give else []
    cg.tree_commit(pages, c["most"], i32(c["parents"]), i32(c["leaves"]), i32(c["lens"]), i32(c["cu"]), i32(c["table"]), pool if rows else None, *given)
    return pool.cpu(), left.cpu().tolist(), stack.cpu().tolist(), free_left.item()


def _committed(c):
    bits = c["pool"].view(torch.int16).numpy()
    pool, left, stack, count = ref.commit(c["page"], c["n_pages"], c["parents"], c["leaves"], c["lens"], c["cu"], c["table"], bits, c["stack"], c["count"])
    return torch.from_numpy(pool), [int(x) for x in left], [int(x) for x in stack], int(count)


@pytest.mark.parametrize("n_req,page,ctx,most,layers,H,d", [
    (1, 16, 0, 1, 1, 1, 64), (1, 64, 500, 8, 1, 8, 128), (7, 16, 90, 40, 3, 2, 128), (64, 32, 100, 48, 2, 3, 64), (5, 256, 300, 33, 1, 2, 256),
    (1030, 16, 20, 9, 1, 1, 64), (3, 16, 5, 700, 2, 1, 64), (1, 16, 0, 96, 16, 8, 128),
])
def test_commit(n_req, page, ctx, most, layers, H, d):
    c = _commit_case(n_req, page, ctx, most, layers, H, d, seed=most)
    want = _committed(c)
    got = _commit(c)
    assert cg.get_status() == 0
    assert got[1] == want[1] and got[2] == want[2] and got[3] == want[3]
    assert torch.equal(got[0].view(torch.int16), want[0])
    # lengths and pages alone, and rows alone; one layer without its dimension
    assert _commit(c, rows=False)[1:] == want[1:]
    only = _commit(c, give=False)
    assert torch.equal(only[0].view(torch.int16), want[0]) and only[1] == [77] * n_req
    one = _commit(c, pool=c["pool"][0].clone().cuda())
    assert torch.equal(one[0].view(torch.int16), want[0][0]) and cg.get_status() == 0


def test_commit_in_a_pool_past_32_bits():
    """Pages of the pool's end, whose rows lie beyond 2^31 elements."""
    H, page, d, n_pages, n = 16, 256, 256, 1100, 300
    pool = torch.zeros(2, n_pages, H, page, d, dtype=torch.bfloat16, device="cuda")
    table = np.array([[n_pages - 1, n_pages - 2]])
    for j in (0, 1):
        pool[:, table[0, j]] = torch.randn(2, H, page, d, device="cuda").bfloat16()
    c = dict(page=page, H=H, d=d, n_pages=2, parents=ref.random_parents(np.random.default_rng(1), n), leaves=[n - 1], lens=np.array([n + 5]), cu=np.array([0, n]),
             table=np.array([[1, 0]]), pool=pool[None, :, n_pages - 2:].cpu(), stack=np.full(2, -9), count=0, most=n)
    want = _committed(c)
    pages = cg.Pages(n_pages=n_pages, page=page, H=H, d=d, n_req=1, max_pages=2)
    left, stack, free_left = i32([77]), i32(np.full(n_pages, -9)), i32([77])
    cg.tree_commit(pages, n, i32(c["parents"]), i32(c["leaves"]), i32(c["lens"]), i32(c["cu"]), i32(table), pool, left, stack, i32([0]), free_left)
    assert cg.get_status() == 0 and left.tolist() == want[1] and free_left.item() == want[3]
    assert torch.equal(pool[:, n_pages - 2:].cpu().view(torch.int16), want[0][0])


def test_commit_of_the_largest_tree():
    c = _commit_case(1, 16, 3, 8192, 1, 1, 64)
    for parents in ([-1 if k == 0 else max(0, k - 2) for k in range(8192)], [k - 1 for k in range(8192)], [-1] * 8192):
        c["parents"] = parents
        want, got = _committed(c), _commit(c)
        assert got[1:] == want[1:] and torch.equal(got[0].view(torch.int16), want[0]) and cg.get_status() == 0


def test_commit_of_what_does_not_fit():
    c = _commit_case(4, 16, 60, 30, 1, 1, 64, seed=3)
    # a leaf that is no node, and a parent that is none
    for i, leaf in ((3, 30), (3, -2)):
        b = dict(c, leaves=c["leaves"][:i] + [leaf] + c["leaves"][i + 1:])
        want, got = _committed(dict(b, leaves=c["leaves"][:i] + [-1])), _commit(b)
        assert cg.get_status() == RANGE and got[1:] == want[1:] and torch.equal(got[0].view(torch.int16), want[0])
    b = dict(c, parents=list(c["parents"]))
    root = int(c["cu"][3]) + ref.path(c["parents"][c["cu"][3]:], 29)[0][0]
    b["parents"][root] = 1 << 30
    want, got = _committed(b), _commit(b)
    assert cg.get_status() == RANGE and got[1:] == want[1:] and torch.equal(got[0].view(torch.int16), want[0])
    # lengths that do not fit: nothing moves, nothing comes back, the length stays
    b = dict(c, lens=np.array([*c["lens"][:3], 29]), leaves=c["leaves"][:3] + [29])
    want = _committed(dict(c, leaves=c["leaves"][:3] + [29]))
    got = _commit(b)
    assert cg.get_status() == RANGE and got[1][:3] == want[1][:3] and got[1][3] == 29
    back = int(np.sum([-(-int(n) // 16) - -(-m // 16) for n, m in zip(c["lens"][:3], want[1][:3])]))
    assert got[3] == 3 + back and got[2][:3 + back] == want[2][:3 + back]
    # entries that are no pages: their rows stay where they are
    b = dict(c, table=c["table"].copy())
    b["table"][3, (c["lens"][3] - 30) // 16] = c["n_pages"]
    want, got = _committed(b), _commit(b)
    assert cg.get_status() == RANGE and got[1:] == want[1:] and torch.equal(got[0].view(torch.int16), want[0])
    # a stack without room
    b = dict(c, count=c["n_pages"], leaves=[-1] * 4)
    got = _commit(b)
    assert cg.get_status() == RANGE and got[3] == c["n_pages"] and got[2] == [int(x) for x in c["stack"]]


# ------------------------------------------------------------------------------------ a step
@pytest.mark.parametrize("graph", [False, True])
def test_a_step(graph):
    """Trees through plan, append, attention and commit, and then one more token: its keys and values, the lengths
    and its output are those of a cache that took the accepted tokens one by one. Eager, and as a graph that is
    replayed on other trees."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    H, rep, d, page, r, most, layers = 2, 4, 128, 16, 3, 21, 2
    n_pages, max_pages = 60, 20
    pages = cg.Pages(n_pages=n_pages, page=page, H=H, d=d, n_req=r, max_pages=max_pages)
    how = cg.PagedAttention(rep, most, d ** -0.5)
    turn, (freqs, _) = cg.Rotary(rot=d), cg.rotary_table(d)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    e32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731

    class Cache:
        def __init__(self):
            self.pool = torch.zeros(layers, 2, n_pages, H, page, d, dtype=torch.bfloat16, device="cuda")
            self.table, self.free, self.count = torch.full((r, max_pages), -1, dtype=torch.int32, device="cuda"), i32(np.arange(n_pages)), i32([n_pages])
            self.lens = e32(r)

        def plan(self, new, n):
            """Lengths behind the step, first rows, positions and slots."""
            lens, cu, pos, slots, left = e32(r), e32(r + 1), e32(n), torch.zeros(n, dtype=torch.int64, device="cuda"), e32(1)
            cg.page_plan(pages, self.lens, new, self.free, self.count, self.table, lens, cu, pos, slots, left)
            self.count.copy_(left)
            return lens, cu, pos, slots

        def take(self, q, k, v, pos, slots):
            turned = [torch.empty_like(x) for x in q]
            for x in range(layers):
                cg.rotary_append(pages, turn, q[x], k[x], v[x], pos, slots, freqs, turned[x], self.pool[x])
            return turned

        def one_by_one(self, q, k, v, new):
            """Tokens in order, as paged_attention takes them; the outputs of the last layer's."""
            n = q.shape[1]
            lens, cu, pos, slots = self.plan(new, n)
            turned = self.take(q, k, v, pos, slots)
            out = torch.empty_like(turned[0])
            cg.paged_attention(pages, how, turned[-1], self.pool[-1], self.table, lens, cu, out)
            self.lens.copy_(lens)
            return out

    ours, plain = Cache(), Cache()
    prompt = i32([40, 5, 0])
    x = rand(layers, 45, H * rep, d), rand(layers, 45, H, d), rand(layers, 45, H, d)
    how_prompt, how = how, how._replace(max_new=40)
    assert torch.equal(ours.one_by_one(*x, prompt), plain.one_by_one(*x, prompt))
    how = how_prompt

    new, n = i32([21, 13, 8]), 42
    parents, leaves = e32(n), e32(r)
    q, k, v = rand(layers, n, H * rep, d), rand(layers, n, H, d), rand(layers, n, H, d)
    out, positions, masks, left, free_left = torch.empty_like(q[0]), e32(n), e32(n, 1), e32(r), e32(1)

    def step():
        lens, cu, _, slots = ours.plan(new, n)
        cg.tree_plan(most, parents, lens, cu, positions, masks)
        turned = ours.take(q, k, v, positions, slots)
        cg.tree_attention(pages, how, turned[-1], ours.pool[-1], ours.table, lens, cu, positions, masks, out)
        cg.tree_commit(pages, most, parents, leaves, lens, cu, ours.table, ours.pool, left, ours.free, ours.count, free_left)
        ours.lens.copy_(left)
        ours.count.copy_(free_left)

    run = step
    if graph:
        state = [t.clone() for t in (ours.pool, ours.table, ours.free, ours.count, ours.lens)]
        parents.copy_(i32([-1] * n))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for t, s in zip((ours.pool, ours.table, ours.free, ours.count, ours.lens), state):
            t.copy_(s)
        run = g.replay
    rng = np.random.default_rng(4)
    cu = [0, 21, 34, 42]
    for turn_no in range(3):
        trees = [ref.random_parents(rng, c) for c in (21, 13, 8)]
        leaf = [20, int(rng.integers(0, 13)), -1 if turn_no == 1 else 7]
        parents.copy_(i32([p for t in trees for p in t]))
        leaves.copy_(i32(leaf))
        for t in (q, k, v):
            t.copy_(rand(*t.shape))
        run()
        assert cg.get_status() == 0
        lines = [ref.path(t, e)[0] if e >= 0 else [] for t, e in zip(trees, leaf)]
        took = torch.tensor([c + b for c, line in zip(cu, lines) for b in line], device="cuda")
        want = plain.one_by_one(q[:, took], k[:, took], v[:, took], i32([len(x) for x in lines]))
        assert torch.equal(ours.lens, plain.lens)
        used = [-(-int(x) // page) for x in plain.lens]
        assert n_pages - ours.count.item() == sum(used) == n_pages - plain.count.item()
        for i, length in enumerate(plain.lens.tolist()):
            rows = lambda c: c.pool[:, :, c.table[i, :used[i]].long()].transpose(3, 4).reshape(layers, 2, used[i] * page, H, d)[:, :, :length]  # noqa: E731
            assert torch.equal(rows(ours), rows(plain))
        # both outputs are within a rounding of the same exact value, and their weights each within another
        assert (out[took].float() - want.float()).abs().max() <= 4 * 2.0 ** -8 * want.float().abs().max()
