"""Cases of the draft-tree operators over the paged cache, and of the 8-bit products around them.

A program that drafts trees of tokens checks a whole tree in one step. Per request the tree's nodes are new
tokens of the paged cache, in an order in which a node's parent stands before it; in one layer the step is
    tree plan       parents -> positions (tokens held + depth) and, per node, a mask of its ancestors
    tree attention  every node over its request's history and its own ancestors
    tree commit     the accepted path's keys and values move up behind the history, spare pages go back
with products in 8 bits before and after the attention:
    block8 encode   a scale for each block of 128 channels (weights: of 128 x 128), codes in e4m3
    block8 matmul   codes times codes, blocks summed in 32 bits with their scales
`run` is one pass of one of them: in elementary torch operations, or by the library's calls.
"""
import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = torch.float8_e4m3fn
BLOCK, TOP = 128, 448.0


# ------------------------------------------------------------------------------- cases
def listed():
    return [
        # one request, a small tree: latency
        dict(name="plan_tree_1", op="tree_plan", n_req=1, ctx=1000, nodes=8, ragged=False, window=0, sinks=0, shape=1),
        # a large batch of ragged trees, for layers under a sliding window
        dict(name="plan_tree_256", op="tree_plan", n_req=256, ctx=9000, nodes=64, ragged=True, window=4096, sinks=4, shape=2),
        # one request, a small tree after a short history: latency
        dict(name="tree_1x1000", op="tree_attention", n_req=1, ctx=1000, nodes=8, H=8, n_rep=4, d=128, dtype="bf16", page=64,
             window=0, sinks=0, ragged=False, shape=3),
        # a verify step of a batch: trees of up to 64 nodes after ragged histories, the 8B-shaped heads
        dict(name="tree_16x64", op="tree_attention", n_req=16, ctx=16384, nodes=64, H=8, n_rep=4, d=128, dtype="bf16", page=64,
             window=0, sinks=0, ragged=True, shape=4),
        # the 27B-shaped heads under a sliding window with sinks, trees of an odd size, small pages
        dict(name="tree_window_41", op="tree_attention", n_req=41, ctx=16384, nodes=25, H=16, n_rep=2, d=128, dtype="fp16",
             page=32, window=4096, sinks=4, ragged=True, shape=5),
        # one request's accepted path in one layer: latency
        dict(name="commit_1", op="tree_commit", n_req=1, ctx=500, nodes=8, layers=1, H=8, d=128, dtype="bf16", page=64,
             ragged=False, shape=6),
        # the accepted paths of a batch in the pools of 16 layers
        dict(name="commit_64", op="tree_commit", n_req=64, ctx=300, nodes=48, layers=16, H=8, d=128, dtype="bf16", page=64,
             ragged=True, shape=7),
        # the activations of one token
        dict(name="encode_1", op="encode", M=1, K=4096, rows=1, dtype="bf16"),
        # the activations of a prompt
        dict(name="encode_8192", op="encode", M=8192, K=4096, rows=1, dtype="bf16"),
        # one token through a projection to queries, keys and values of 32 + 8 + 8 heads of 128
        dict(name="matmul_1", op="matmul", M=1, N=6144, K=4096, dtype="bf16"),
        # the nodes of a few trees, sizes that end inside tiles and blocks
        dict(name="matmul_333", op="matmul", M=333, N=1000, K=4112, dtype="fp16"),
        # a prompt through the same projection
        dict(name="matmul_8192", op="matmul", M=8192, N=6144, K=4096, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree_plan", "tree_attention", "tree_attention", "tree_commit", "encode", "matmul", "matmul"])
    pages = [16, 32, 64, 128, 256]
    while True:
        if op == "tree_plan":
            c = dict(op=op, n_req=_log(rng, 1, 256), ctx=_log(rng, 1, 20000), nodes=_log(rng, 1, 512), ragged=True,
                     window=rng.choice([0, 0, _log(rng, 1, 4096)]), sinks=0, shape=rng.randrange(1 << 20))
            if c["window"]:
                c["sinks"] = rng.choice([0, 4])
            if work(c)["bytes"] <= work(listed()[1])["bytes"]:
                return c
        elif op == "tree_attention":
            windowed = rng.random() < 0.4
            c = dict(op=op, n_req=_log(rng, 1, 64), ctx=_log(rng, 1, 32768), nodes=_log(rng, 1, 200), H=rng.choice([1, 2, 4, 8, 16]),
                     n_rep=rng.choice([1, 2, 3, 4, 5, 7, 8]), d=rng.choice([64, 128, 128, 128, 256]), dtype=rng.choice(["bf16", "fp16"]),
                     page=rng.choice(pages), window=_log(rng, 16, 8192) if windowed else 0,
                     sinks=rng.choice([0, 1, 4, 33]) if windowed else 0, ragged=rng.random() < 0.7, shape=rng.randrange(1 << 20))
            ctx, nodes = lengths(c)
            longest = max(a + b for a, b in zip(ctx, nodes))
            scores = c["n_req"] * c["H"] * c["n_rep"] * max(nodes) * longest * 4      # of the plain form, padded
            gathered = 2 * c["n_req"] * longest * c["H"] * c["d"] * 4
            w, top = work(c), work(listed()[3])
            if scores <= 12e9 and gathered <= 18e9 and w["flops"] <= top["flops"] and w["bytes"] <= 1.5 * top["bytes"]:
                return c
        elif op == "tree_commit":
            c = dict(op=op, n_req=_log(rng, 1, 96), ctx=_log(rng, 1, 600), nodes=_log(rng, 1, 96), layers=rng.choice([1, 1, 2, 7, 16]),
                     H=rng.choice([1, 2, 4, 8, 16]), d=rng.choice([64, 128, 128, 256]), dtype=rng.choice(["bf16", "fp16"]),
                     page=rng.choice(pages), ragged=True, shape=rng.randrange(1 << 20))
            ctx, nodes = lengths(c)
            n_pages = sum(_up(a + b, c["page"]) for a, b in zip(ctx, nodes)) + 3
            if work(c)["bytes"] <= work(listed()[6])["bytes"] and c["layers"] * n_pages * c["H"] * c["page"] * c["d"] * 4 <= 2.5e9:
                return c
        elif op == "encode":
            c = dict(op=op, M=_log(rng, 1, 16384), K=16 * _log(rng, 1, 1024), rows=rng.choice([1, 1, BLOCK]), dtype=rng.choice(["bf16", "fp16"]))
            if work(c)["bytes"] <= work(listed()[8])["bytes"]:
                return c
        else:
            c = dict(op=op, M=_log(rng, 1, 16384), N=_log(rng, 8, 16384), K=16 * _log(rng, 1, 1024), dtype=rng.choice(["bf16", "fp16"]))
            w, top = work(c), work(listed()[11])
            if w["flops"] <= top["flops"] and w["bytes"] <= top["bytes"]:
                return c


def lengths(c):
    """Tokens that each request holds before the step, and the nodes of its tree (by the case alone)."""
    r = random.Random(c["shape"])
    ctx = [r.randrange(c["ctx"] + 1) if c["ragged"] else c["ctx"] for _ in range(c["n_req"])]
    nodes = [(0 if r.random() < 0.04 and i else 1 + r.randrange(c["nodes"])) if c["ragged"] else c["nodes"] for i in range(c["n_req"])]
    nodes[-1] = c["nodes"]                                # the case's largest is there
    return ctx, nodes


def trees(c, salt=0):
    """Each request's parents (-1: the last token held), and its accepted node (-1: none)."""
    r = random.Random(c["shape"] + 1 + 7919 * salt)
    parents, leaves = [], []
    for n in lengths(c)[1]:
        p = []
        for k in range(n):
            x = r.random()
            p.append(-1 if k == 0 or x < 0.1 else k - 1 if x < 0.4 else r.randrange(max(0, k - 12), k))
        parents.append(p)
        leaves.append(-1 if n == 0 or r.random() < 0.1 else r.randrange(n // 2, n))
    return parents, leaves


def _paths(parents):
    """Every node's path from the root to itself."""
    paths = []
    for k, p in enumerate(parents):
        paths.append((paths[p] if p >= 0 else []) + [k])
    return paths


def _up(n, page):
    return -(-n // page)


def _words(n):
    return max(1, _up(n, 32))


def work(c):
    if c["op"] == "tree_plan":
        n = sum(lengths(c)[1])
        return {"bytes": 8 * c["n_req"] + 8 * n + 4 * n * _words(c["nodes"]), "flops": 0}
    if c["op"] == "encode":
        M, K = c["M"], c["K"]
        return {"bytes": 3 * M * K + 4 * _up(M, c["rows"]) * _up(K, BLOCK), "flops": 3 * M * K}
    if c["op"] == "matmul":
        M, N, K = c["M"], c["N"], c["K"]
        b = _up(K, BLOCK)
        return {"bytes": M * K + N * K + 4 * b * (M + _up(N, BLOCK)) + 2 * M * N, "flops": 2 * M * N * K}
    ctx, nodes = lengths(c)
    parents, leaves = trees(c)
    if c["op"] == "tree_commit":
        moved = sum(sum(a != b for a, b in enumerate(_paths(p)[x])) for p, x in zip(parents, leaves) if x >= 0)
        back = sum(_up(a + b, c["page"]) - _up(a + (len(_paths(p)[x]) if x >= 0 else 0), c["page"])
                   for a, b, p, x in zip(ctx, nodes, parents, leaves))
        return {"bytes": 8 * moved * c["layers"] * c["H"] * c["d"] + 20 * c["n_req"] + 4 * sum(nodes) + 8 * back, "flops": 0}
    w, read, pairs = c["window"], 0, 0
    for a, b, p in zip(ctx, nodes, parents):
        for path in _paths(p):
            at = a + len(path) - 1                        # the node's position
            lo = max(0, at - w + 1) if w else 0           # first token of its window
            pairs += max(0, a - lo) + min(lo, a, c["sinks"]) if w else a
            pairs += sum(1 for k in range(len(path)) if not w or len(path) - 1 - k < w or a + k < c["sinks"])
        if b:
            lo = min(a, max(0, a - w + 1)) if w else 0
            read += a + b - lo + min(c["sinks"] if w else 0, lo)
    hq, n = c["H"] * c["n_rep"], sum(nodes)
    return {"bytes": 4 * read * c["H"] * c["d"] + 4 * n * hq * c["d"] + 4 * n * hq + 4 * n * (1 + _words(c["nodes"])),
            "flops": 4 * pairs * hq * c["d"]}


# ------------------------------------------------------------------------------ inputs
def _spread(n, gen):
    """Per-channel sizes: a spread, and a few channels ten times as large."""
    s = torch.exp(0.5 * torch.randn(n, device="cuda", generator=gen))
    s[torch.randperm(n, device="cuda", generator=gen)[:max(1, n // 64)]] *= 10
    return s


def _coded(x, rows):
    """Codes and scales of a matrix, as a program has them from a checkpoint."""
    M, K = x.shape
    s = torch.zeros(_up(M, rows) * rows, _up(K, BLOCK) * BLOCK, device=x.device)
    s[:M, :K] = x.abs()
    s = s.view(_up(M, rows), rows, _up(K, BLOCK), BLOCK).amax((1, 3)) / TOP
    wide = s.repeat_interleave(rows, 0)[:M].repeat_interleave(BLOCK, 1)[:, :K]
    return (x / wide).nan_to_num(0.0).to(E4M3), s


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    empty = lambda n, t: torch.empty(n, dtype=t, device="cuda")        # noqa: E731
    randn = lambda *n: torch.randn(*n, device="cuda", generator=gen)   # noqa: E731
    if c["op"] == "encode":
        M, K = c["M"], c["K"]
        return dict(c=c, x=(randn(M, K) * _spread(K, gen)).to(DT[c["dtype"]]), codes=empty((M, K), E4M3),
                    scales=empty((_up(M, c["rows"]), _up(K, BLOCK)), torch.float32))
    if c["op"] == "matmul":
        M, N, K = c["M"], c["N"], c["K"]
        x, xs = _coded(randn(M, K) * _spread(K, gen), 1)
        w, ws = _coded(randn(N, K) / math.sqrt(K), BLOCK)
        return dict(c=c, x=x, x_scales=xs, w=w, w_scales=ws, out=empty((M, N), DT[c["dtype"]]))
    ctx, nodes = lengths(c)
    parents, leaves = trees(c, seed if c["op"] == "tree_plan" else 0)
    order = list(range(c["n_req"]))
    random.Random(seed).shuffle(order)                    # the same work for every seed, in another order
    ctx, nodes, parents, leaves = ([v[i] for i in order] for v in (ctx, nodes, parents, leaves))
    lens = [a + b for a, b in zip(ctx, nodes)]
    cu = [0]
    for b in nodes:
        cu.append(cu[-1] + b)
    n, words = cu[-1], _words(c["nodes"])
    s = dict(c=c, parents=i32([p for q in parents for p in q]), seq_lens=i32(lens), cu_new=i32(cu), positions=empty(n, torch.int32),
             masks=empty((n, words), torch.int32))
    if c["op"] == "tree_plan":
        return s
    page, dt, H, d = c["page"], DT[c["dtype"]], c["H"], c["d"]
    need = [_up(x, page) for x in lens]
    n_pages, layers = sum(need) + 3, c.get("layers", 1)
    perm = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((c["n_req"], max(need) + 1), -1, dtype=torch.int32, device="cuda")
    need_t = torch.tensor(need)
    rows = torch.repeat_interleave(torch.arange(c["n_req"]), need_t)
    cols = torch.arange(sum(need)) - torch.repeat_interleave(torch.cumsum(need_t, 0) - need_t, need_t)
    table[rows.cuda(), cols.cuda()] = perm[:sum(need)]
    pool = torch.empty(layers, 2, n_pages, H, page, d, dtype=dt, device="cuda")
    size = _spread(H * d, gen).view(H, 1, d)
    step = max(1, (1 << 27) // (H * page * d))
    for layer in pool:
        for a in range(0, n_pages, step):
            b = min(n_pages, a + step)
            layer[0, a:b] = randn(b - a, H, page, d) * size
            layer[1, a:b] = randn(b - a, H, page, d)
    s.update(block_table=table, pool=pool)
    if c["op"] == "tree_commit":
        # two pages are free; the last one is nobody's
        free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        free[:2] = perm[sum(need):sum(need) + 2]
        s.update(leaves=i32(leaves), free_pages=free, free_count=i32([2]), nobody=perm[-1:].long(), lens_left=empty(c["n_req"], torch.int32),
                 free_left=empty(1, torch.int32), most_back=sum(_up(x, page) - _up(a, page) for x, a in zip(lens, ctx)))
        return s
    at, bits = [], torch.zeros(n, words * 32, dtype=torch.bool)
    for a, p, c0 in zip(ctx, parents, cu):
        for k, path in enumerate(_paths(p)):
            at.append(a + len(path) - 1)
            bits[c0 + k, [b for j, b in enumerate(path) if not c["window"] or len(path) - 1 - j < c["window"] or a + j < c["sinks"]]] = True
    packed = (bits.view(n, words, 32).long() << torch.arange(32)).sum(-1)
    s.update(positions=i32(at), masks=torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32).cuda(), pool=pool[0],
             max_len=max(lens), scale=d ** -0.5, q=randn(n, H * c["n_rep"], d).to(dt), out=empty((n, H * c["n_rep"], d), dt),
             lse=empty((n, H * c["n_rep"]), torch.float32))
    return s


# --------------------------------------------------------------------------- plain forms
def _padded(s):
    """Per request and node (padded to the largest tree): its token, and whether there is one."""
    cu = s["cu_new"].long()
    k = torch.arange(s["c"]["nodes"], device="cuda")
    have = k < (cu[1:] - cu[:-1])[:, None]
    return torch.where(have, cu[:-1, None] + k, 0), have


def _reach(s):
    """[request, node, node]: the second is the first or an ancestor of it. Powers of (1 + parent) by squaring."""
    tok, have = _padded(s)
    n = tok.shape[1]
    k = torch.arange(n, device="cuda")
    parent = torch.where(have, s["parents"].long()[tok], -1)
    a = ((parent[..., None] == k) | (k[:, None] == k)).float()
    for _ in range(max(1, n - 1).bit_length()):
        a = (torch.matmul(a, a) > 0).float()
    return a, tok, have


def _plain_tree_plan(s):
    c = s["c"]
    a, tok, have = _reach(s)
    depth = a.sum(-1).long() - 1
    cu, lens = s["cu_new"].long(), s["seq_lens"].long()
    ctx = (lens - (cu[1:] - cu[:-1]))[:, None]
    see = a > 0
    if c["window"]:
        see &= (depth[:, :, None] - depth[:, None] < c["window"]) | ((ctx + depth)[:, None] < c["sinks"])
    n, words = s["positions"].numel(), _words(c["nodes"])
    r = torch.repeat_interleave(torch.arange(c["n_req"], device="cuda"), cu[1:] - cu[:-1], output_size=n)
    at = torch.arange(n, device="cuda") - cu[r]
    bits = torch.zeros(n, words * 32, dtype=torch.int64, device="cuda")
    bits[:, :see.shape[2]] = see[r, at].long()
    packed = (bits.view(n, words, 32) << torch.arange(32, device="cuda")).sum(-1)
    s["positions"].copy_((ctx + depth)[r, at])
    s["masks"].copy_(torch.where(packed >= 1 << 31, packed - (1 << 32), packed))
    return dict(positions=s["positions"], masks=s["masks"])


def _plain_tree_attention(s):
    c, page, H, d, rep = s["c"], s["c"]["page"], s["c"]["H"], s["c"]["d"], s["c"]["n_rep"]
    n_req, n, width, most = c["n_req"], s["q"].shape[0], _up(s["max_len"], page), c["nodes"]
    ids = s["block_table"][:, :width].long().clamp(min=0)
    # [n_req, H, tokens, d] in 32 bits
    k = s["pool"][0][ids].permute(0, 2, 1, 3, 4).float().reshape(n_req, H, width * page, d)
    v = s["pool"][1][ids].permute(0, 2, 1, 3, 4).float().reshape(n_req, H, width * page, d)
    tok, _ = _padded(s)
    q = s["q"][tok].view(n_req, most, H, rep, d).permute(0, 2, 1, 3, 4).float().reshape(n_req, H, most * rep, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    cu, lens = s["cu_new"].long(), s["seq_lens"].long()
    ctx = (lens - (cu[1:] - cu[:-1]))[:, None, None]
    t = torch.arange(width * page, device="cuda")
    j = (t - ctx).clamp(0, most - 1).expand(n_req, most, -1)                          # node at token t
    node = torch.gather(s["masks"][tok], 2, j >> 5) >> (j & 31).int() & 1
    see = t < ctx
    if c["window"]:
        see = see & ((t > s["positions"].long()[tok][..., None] - c["window"]) | (t < c["sinks"]))
    see = torch.where(t >= ctx, (node > 0) & (t < lens[:, None, None]), see)
    x.view(n_req, H, most, rep, -1).masked_fill_(~see[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v) / total
    lse = top + torch.log(total)
    r = torch.repeat_interleave(torch.arange(n_req, device="cuda"), cu[1:] - cu[:-1], output_size=n)
    at = torch.arange(n, device="cuda") - cu[r]
    o = o.view(n_req, H, most, rep, d)[r, :, at].reshape(n, H * rep, d)
    return dict(out=o.to(s["q"].dtype), lse=lse.view(n_req, H, most, rep)[r, :, at].reshape(n, H * rep))


def _plain_tree_commit(s):
    c, page, pool, table = s["c"], s["c"]["page"], s["pool"], s["block_table"].long()
    a, _, have = _reach(s)
    cu, lens, leaf = s["cu_new"].long(), s["seq_lens"].long(), s["leaves"].long()
    ctx = lens - (cu[1:] - cu[:-1])
    row = torch.arange(c["n_req"], device="cuda")
    path = (a[row, leaf.clamp(min=0)] > 0) & (leaf >= 0)[:, None] & have
    k = torch.arange(c["nodes"], device="cuda")
    src, dst = ctx[:, None] + k, ctx[:, None] + torch.cumsum(path, 1) - 1

    def place(p):                                          # page and row; nodes off the path: a row that is nobody's
        p = torch.where(path, p, 0)
        return torch.where(path, table[row[:, None], p // page], s["nobody"]).view(-1), torch.where(path, p % page, 0).view(-1)
    pg, off = place(src)
    rows = pool[:, :, pg, :, off]
    pg, off = place(dst)
    pool[:, :, pg, :, off] = rows
    keep = ctx + path.sum(1)
    back = (lens + page - 1) // page - (keep + page - 1) // page
    upto = torch.cumsum(back, 0)
    i = torch.arange(s["most_back"], device="cuda")
    used = i < upto[-1]
    r = torch.where(used, torch.searchsorted(upto, i, right=True), 0)
    col = torch.where(used, ((keep + page - 1) // page)[r] + i - (upto - back)[r], 0)
    to = torch.where(used, s["free_count"].long() + i, 0)
    free = s["free_pages"]
    free[to] = torch.where(used, s["block_table"][r, col], free[to])
    return dict(pool=pool, lens_left=keep.int(), free_pages=free, free_left=(s["free_count"] + upto[-1]).int())


def _plain_encode(s):
    c, x = s["c"], s["x"].float()
    M, K, rows = c["M"], c["K"], c["rows"]
    a = torch.zeros(_up(M, rows) * rows, _up(K, BLOCK) * BLOCK, device="cuda")
    a[:M, :K] = x.abs()
    # (by a tensor: a quotient by a number is a product with its rounded reciprocal)
    scales = a.view(_up(M, rows), rows, _up(K, BLOCK), BLOCK).amax((1, 3)) / torch.full((), TOP, device="cuda")
    wide = scales.repeat_interleave(rows, 0)[:M].repeat_interleave(BLOCK, 1)[:, :K]
    return dict(codes=torch.where(wide > 0, x / wide, 0.0).to(E4M3), scales=scales)


def _plain_matmul(s):
    M, N, K = s["c"]["M"], s["c"]["N"], s["c"]["K"]
    x = s["x"].float() * s["x_scales"].repeat_interleave(BLOCK, 1)[:, :K]
    w = s["w"].float() * s["w_scales"].repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1)[:, :K]
    return torch.matmul(x, w.T).to(s["out"].dtype)


def run(s):
    c = s["c"]
    if not own:
        return {"tree_plan": _plain_tree_plan, "tree_attention": _plain_tree_attention, "tree_commit": _plain_tree_commit,
                "encode": _plain_encode, "matmul": _plain_matmul}[c["op"]](s)
    import paper_2607_20538_gb300 as cg
    if c["op"] == "tree_plan":
        cg.tree_plan(c["nodes"], s["parents"], s["seq_lens"], s["cu_new"], s["positions"], s["masks"], window=c["window"], sinks=c["sinks"])
        return dict(positions=s["positions"], masks=s["masks"])
    if c["op"] == "tree_attention":
        pages = cg.Pages(n_pages=s["pool"].shape[1], page=c["page"], H=c["H"], d=c["d"], n_req=c["n_req"], max_pages=s["block_table"].shape[1])
        how = cg.PagedAttention(n_rep=c["n_rep"], max_new=c["nodes"], scale=s["scale"], window=c["window"], sinks=c["sinks"])
        cg.tree_attention(pages, how, s["q"], s["pool"], s["block_table"], s["seq_lens"], s["cu_new"], s["positions"], s["masks"],
                          s["out"], s["lse"])
        return dict(out=s["out"], lse=s["lse"])
    if c["op"] == "tree_commit":
        pages = cg.Pages(n_pages=s["pool"].shape[2], page=c["page"], H=c["H"], d=c["d"], n_req=c["n_req"], max_pages=s["block_table"].shape[1])
        cg.tree_commit(pages, c["nodes"], s["parents"], s["leaves"], s["seq_lens"], s["cu_new"], s["block_table"], s["pool"], s["lens_left"],
                       s["free_pages"], s["free_count"], s["free_left"])
        return {k: s[k] for k in ("pool", "lens_left", "free_pages", "free_left")}
    if c["op"] == "encode":
        cg.block8_encode(s["x"], s["codes"], s["scales"], rows=c["rows"])
        return dict(codes=s["codes"], scales=s["scales"])
    cg.block8_matmul(s["x"], s["x_scales"], s["w"], s["w_scales"], s["out"])
    return s["out"]


# ------------------------------------------------------------------------- from the definition
def exact(c, seed):
    """What run returns, from the definition in 64 bits."""
    if c["op"] in ("tree_plan", "tree_commit"):
        return None                                       # whole numbers, and rows that only move
    s = prepare(c, seed)
    if c["op"] == "encode":
        x, M, K, rows = s["x"].double(), c["M"], c["K"], c["rows"]
        scales = torch.stack([torch.stack([x[r:r + rows, k:k + BLOCK].abs().amax() for k in range(0, K, BLOCK)]) for r in range(0, M, rows)]) / TOP \
            if rows > 1 else torch.stack([x[:, k:k + BLOCK].abs().amax(1) for k in range(0, K, BLOCK)], 1) / TOP
        r, k = torch.arange(M, device="cuda") // rows, torch.arange(K, device="cuda") // BLOCK
        return dict(codes=(x / scales[r[:, None], k]).nan_to_num(0.0), scales=scales)
    if c["op"] == "matmul":
        M, N, K = c["M"], c["N"], c["K"]
        out = torch.zeros(M, N, dtype=torch.float64, device="cuda")
        n = torch.arange(N, device="cuda") // BLOCK
        for b, k in enumerate(range(0, K, BLOCK)):
            out += (s["x"][:, k:k + BLOCK].double() @ s["w"][:, k:k + BLOCK].double().T) * s["x_scales"][:, b, None].double() * s["w_scales"][n, b].double()
        return out
    H, rep, d, page, w = c["H"], c["n_rep"], c["d"], c["page"], c["window"]
    lens, cu, parents = s["seq_lens"].tolist(), s["cu_new"].tolist(), s["parents"].tolist()
    out = torch.empty(cu[-1], H * rep, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(cu[-1], H * rep, dtype=torch.float64, device="cuda")
    for i, (length, lo, hi) in enumerate(zip(lens, cu, cu[1:])):
        a, ids = length - (hi - lo), s["block_table"][i, :_up(length, page)].long()
        seen = torch.zeros(hi - lo, length, dtype=torch.bool)
        for k, path in enumerate(_paths(parents[lo:hi])):
            line = torch.tensor(list(range(a)) + [a + b for b in path])               # the tokens that lead to the node, in order
            p = torch.arange(len(line))
            seen[k, line if not w else line[(p > len(line) - 1 - w) | (p < c["sinks"])]] = True
        for h in range(H if hi > lo else 0):
            key, val = (s["pool"][x, ids, h].double().reshape(-1, d)[:length] for x in (0, 1))
            x = torch.einsum("nrd,td->rnt", s["q"][lo:hi, h * rep:(h + 1) * rep].double(), key) * s["scale"]
            x = torch.where(seen.cuda(), x, -math.inf)
            z = torch.logsumexp(x, -1)
            lse[lo:hi, h * rep:(h + 1) * rep] = z.T
            out[lo:hi, h * rep:(h + 1) * rep] = torch.einsum("rnt,td->nrd", torch.exp(x - z[..., None]), val)
    return dict(out=out, lse=lse)
