"""Cases of the paged-cache operators: page plan, rotary append and paged attention.

A paged cache keeps the keys and values of many requests in one pool of fixed-size pages,
pool[2][n_pages][H][page][d] (0 keys, 1 values), which is the codec's cache layout with one layer
and the pages as the batch. One serving step of one layer is
    plan       lengths -> pages for the new tokens, positions and pool slots of every token
    rotary     queries and keys turned by their positions, keys and values put into their slots
    attention  the new tokens' queries over the pages of their own request (causal, with an
               optional sliding window and first tokens that stay visible)
`run` is one pass of one of them: in elementary torch operations, or by the library's calls.
"""
import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token for each of 256 running requests: what every decode step plans
        dict(name="plan_decode_256", op="plan", n_req=256, ctx=8192, new=1, page=64, ragged=True, singles=1.0, shape=1),
        # a large batch of prompts of very different lengths, small pages
        dict(name="plan_prompts_333", op="plan", n_req=333, ctx=900, new=2047, page=16, ragged=True, singles=0.0, shape=2),
        # one token of one request: latency
        dict(name="rotary_token_1", op="rotary", n_tok=1, ctx=1000, H=8, n_rep=4, d=128, rot=128, dtype="bf16",
             interleaved=False, base=500000.0, scaling="none", factor=1.0, page=64),
        # a decode batch, 7 query heads per KV head, half of the head turned, stretched context
        dict(name="rotary_decode_193", op="rotary", n_tok=193, ctx=32768, H=4, n_rep=7, d=128, rot=64, dtype="fp16",
             interleaved=True, base=10000.0, scaling="yarn", factor=4.0, page=16),
        # a long prompt of the 8B-shaped cache, long-context frequencies
        dict(name="rotary_prompt_16384", op="rotary", n_tok=16384, ctx=0, H=8, n_rep=4, d=128, rot=128, dtype="bf16",
             interleaved=False, base=500000.0, scaling="bands", factor=8.0, page=64),
        # one short request, one token: latency
        dict(name="decode_1x1000", op="attention", n_req=1, ctx=999, new=1, H=8, n_rep=4, d=128, dtype="bf16", page=64,
             window=0, sinks=0, ragged=False, singles=1.0, shape=3),
        # one token for each of 64 histories of 16k tokens (the rolling step's layer)
        dict(name="decode_64x16384", op="attention", n_req=64, ctx=16383, new=1, H=8, n_rep=4, d=128, dtype="bf16",
             page=64, window=0, sinks=0, ragged=False, singles=1.0, shape=4),
        # a ragged decode batch under a sliding window with sinks, the 27B-shaped heads
        dict(name="decode_window_41", op="attention", n_req=41, ctx=32768, new=1, H=16, n_rep=2, d=128, dtype="fp16",
             page=32, window=4096, sinks=4, ragged=True, singles=1.0, shape=5),
        # a prompt chunk that follows 32k tokens already in the cache
        dict(name="chunk_2048_over_32k", op="attention", n_req=1, ctx=32768, new=2048, H=8, n_rep=4, d=128,
             dtype="bf16", page=64, window=0, sinks=0, ragged=False, singles=0.0, shape=6),
        # ragged chunks under a window, 7 query heads per KV head
        dict(name="chunk_window_5", op="attention", n_req=5, ctx=9000, new=1111, H=4, n_rep=7, d=128, dtype="fp16",
             page=16, window=2000, sinks=5, ragged=True, singles=0.0, shape=7),
        # a whole prompt of the 8B shape
        dict(name="prompt_8192", op="attention", n_req=1, ctx=0, new=8192, H=8, n_rep=4, d=128, dtype="bf16", page=64,
             window=0, sinks=0, ragged=False, singles=0.0, shape=8),
        # a mixed step: most requests decode, some bring a chunk; 64-channel heads
        dict(name="mixed_17", op="attention", n_req=17, ctx=5000, new=700, H=8, n_rep=5, d=64, dtype="bf16", page=16,
             window=0, sinks=0, ragged=True, singles=0.75, shape=9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "rotary", "attention", "attention", "attention"])
    top = {o: max((work(c) for c in listed() if c["op"] == o), key=lambda w: w["bytes"] + w["flops"] / 100)
           for o in ("plan", "rotary")}
    while True:
        if op == "plan":
            one = rng.random() < 0.5
            c = dict(op=op, n_req=_log(rng, 1, 2048), ctx=_log(rng, 1, 20000), new=1 if one else _log(rng, 2, 2047),
                     page=rng.choice([16, 32, 64, 128, 256]), ragged=True, singles=1.0 if one else rng.choice([0.0, 0.5]),
                     shape=rng.randrange(1 << 20))
            if work(c)["bytes"] <= top[op]["bytes"]:
                return c
        elif op == "rotary":
            d = rng.choice([64, 128, 128, 256])
            c = dict(op=op, n_tok=_log(rng, 1, 16384), ctx=_log(rng, 1, 60000), H=rng.choice([1, 2, 4, 8, 16]),
                     n_rep=rng.choice([1, 2, 3, 4, 7, 8]), d=d, rot=rng.choice([d, d, d // 2, d // 4]),
                     dtype=rng.choice(["bf16", "fp16"]), interleaved=rng.random() < 0.5,
                     base=rng.choice([10000.0, 500000.0, 1000000.0]), scaling=rng.choice(["none", "linear", "bands", "yarn"]),
                     factor=rng.choice([2.0, 4.0, 8.0]), page=rng.choice([16, 32, 64, 128, 256]))
            if work(c)["bytes"] <= top[op]["bytes"]:
                return c
        else:
            kind = rng.choice(["decode", "decode", "chunk", "mixed"])
            windowed = rng.random() < 0.4
            c = dict(op=op, n_req=_log(rng, 1, 8 if kind == "chunk" else 96), ctx=_log(rng, 1, 32768),
                     new=1 if kind == "decode" else _log(rng, 2, 4096), H=rng.choice([1, 2, 4, 8, 16]),
                     n_rep=rng.choice([1, 2, 3, 4, 5, 7, 8]), d=rng.choice([64, 128, 128, 128, 256]),
                     dtype=rng.choice(["bf16", "fp16"]), page=rng.choice([16, 32, 64, 128, 256]),
                     window=_log(rng, 16, 8192) if windowed else 0, sinks=rng.choice([0, 1, 4, 33]) if windowed else 0,
                     ragged=rng.random() < 0.7, singles={"decode": 1.0, "chunk": 0.0, "mixed": 0.8}[kind],
                     shape=rng.randrange(1 << 20))
            ctx, new = lengths(c)
            longest = max(a + b for a, b in zip(ctx, new))
            scores = c["n_req"] * c["H"] * c["n_rep"] * max(new) * longest * 4       # of the plain form, padded
            gathered = 2 * c["n_req"] * longest * c["H"] * c["d"] * 4
            w = work(c)
            if sum(new) and scores <= 12e9 and gathered <= 18e9 and w["flops"] <= 6e11 and w["bytes"] <= 4.4e9:
                return c


def lengths(c):
    """Tokens each request holds before the step, and its new ones (by the case alone)."""
    r = random.Random(c["shape"])
    ctx, new = [], []
    for i in range(c["n_req"]):
        ctx.append(r.randrange(c["ctx"] + 1) if c["ragged"] else c["ctx"])
        if not c["ragged"]:
            new.append(c["new"])
        elif r.random() < c["singles"]:
            new.append(1)
        else:
            new.append(0 if r.random() < 0.03 and i else 1 + r.randrange(c["new"]))
    if max(new) < c["new"]:
        new[-1] = c["new"]           # the case's longest is there
    return ctx, new


def _pages(n, page):
    return -(-n // page)


def _visible(c, p):
    """Tokens that the query at position p sees."""
    w = c["window"]
    return p + 1 if not w or p + 1 <= w else w + min(c["sinks"], p + 1 - w)


def work(c):
    if c["op"] == "plan":
        ctx, new = lengths(c)
        touched = sum(_pages(a + b, c["page"]) - a // c["page"] for a, b in zip(ctx, new) if b)
        fresh = sum(_pages(a + b, c["page"]) - _pages(a, c["page"]) for a, b in zip(ctx, new))
        return {"bytes": 16 * c["n_req"] + 12 * sum(new) + 4 * touched + 8 * fresh, "flops": 0}
    if c["op"] == "rotary":
        vec = 2 * c["d"] * c["n_tok"]
        heads = c["H"] * c["n_rep"] + c["H"]
        return {"bytes": 2 * vec * (heads + c["H"]) + 12 * c["n_tok"] + 4 * c["rot"], "flops": 3 * c["rot"] * heads * c["n_tok"]}
    ctx, new = lengths(c)
    w, pairs, read = c["window"], 0, 0
    for a, b in zip(ctx, new):
        # sum over p in [a, a + b) of _visible(p)
        def upto(n):                                      # sum over p in [0, n)
            if not w or n <= w:
                return n * (n + 1) // 2
            m, s = n - w, c["sinks"]                      # positions beyond the window's length
            k = min(m, s)
            return w * (w + 1) // 2 + m * w + k * (k + 1) // 2 + (m - k) * s
        pairs += upto(a + b) - upto(a)
        if b:
            lo = max(0, a + 1 - w) if w else 0            # the first query's window starts here
            read += a + b - lo + min(c["sinks"] if w else 0, lo)
    hq, n = c["H"] * c["n_rep"], sum(new)
    return {"bytes": 4 * read * c["H"] * c["d"] + 4 * n * hq * c["d"] + 4 * n * hq, "flops": 4 * pairs * hq * c["d"]}


# ------------------------------------------------------------------------------ inputs
def frequencies(c):
    """Angle per position of every pair of channels, and what cosine and sine are multiplied by."""
    n, base, s = c["rot"] // 2, c["base"], c["factor"]
    f = [base ** (-2.0 * i / c["rot"]) for i in range(n)]
    if c["scaling"] == "linear":                          # positions interpolated
        return [x / s for x in f], 1.0
    if c["scaling"] == "bands":                           # long wavelengths interpolated, short ones kept, a ramp between
        low, high, orig = 1.0, 4.0, 8192.0
        g = []
        for x in f:
            turns = orig * x / (2 * math.pi)
            t = min(1.0, max(0.0, (turns - low) / (high - low)))
            g.append((1 - t) * x / s + t * x)
        return g, 1.0
    if c["scaling"] == "yarn":                            # a ramp over the pair index, and a temperature
        orig, fast, slow = 8192.0, 32.0, 1.0
        at = lambda turns: c["rot"] * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), c["rot"] - 1)
        g = []
        for i, x in enumerate(f):
            t = 1 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3)))
            g.append((1 - t) * x / s + t * x)
        return g, 0.1 * math.log(s) + 1.0
    return f, 1.0


def _key_scale(H, d, gen):
    """Per-channel size of the keys: a spread, and a few channels ten times as large."""
    s = torch.exp(0.5 * torch.randn(H, 1, d, device="cuda", generator=gen))
    s[:, :, torch.randperm(d, device="cuda", generator=gen)[:4]] *= 10
    return s


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    empty = lambda n, t: torch.empty(n, dtype=t, device="cuda")        # noqa: E731
    page = c["page"]
    if c["op"] == "plan":
        ctx, new = lengths(c)
        have = [_pages(a, page) for a in ctx]
        need = sum(_pages(a + b, page) for a, b in zip(ctx, new)) + 5
        width = max(_pages(a + b, page) for a, b in zip(ctx, new)) + 1
        perm = torch.randperm(need, device="cuda", generator=gen).to(torch.int32)
        table = torch.full((c["n_req"], width), -1, dtype=torch.int32, device="cuda")
        rows = torch.repeat_interleave(torch.arange(c["n_req"]), torch.tensor(have))
        cols = torch.arange(sum(have)) - torch.repeat_interleave(torch.cumsum(torch.tensor(have), 0) - torch.tensor(have), torch.tensor(have))
        table[rows.cuda(), cols.cuda()] = perm[:sum(have)]
        n = sum(new)
        return dict(c=c, n_tok=n, n_pages=need, ctx_lens=i32(ctx), new_lens=i32(new), free_pages=perm[sum(have):].clone(),
                    free_count=i32([need - sum(have)]), block_table=table,
                    seq_lens=empty(c["n_req"], torch.int32), cu_new=empty(c["n_req"] + 1, torch.int32),
                    positions=empty(n, torch.int32), slots=empty(n, torch.int64), free_left=empty(1, torch.int32))
    dt, H, d = DT[c["dtype"]], c["H"], c["d"]
    hq = H * c["n_rep"]
    if c["op"] == "rotary":
        n = c["n_tok"]
        qkv = torch.randn(n, (hq + 2 * H) * d, device="cuda", generator=gen).to(dt)        # a fused projection's output
        q, k, v = (x.view(n, -1, d) for x in qkv.split([hq * d, H * d, H * d], dim=1))
        n_pages = _pages(n, page) + 3
        f, m = frequencies(c)
        turns = [round(x / (2 * math.pi) * 2 ** 64) % 2 ** 64 for x in f]                   # in 2^-64 of a turn
        pool = torch.randn(2, n_pages, H, page, d, device="cuda", generator=gen).to(dt)
        ids = torch.randperm(n_pages, device="cuda", generator=gen)
        t = torch.arange(n, device="cuda")
        # a prompt's positions run on; a decode batch has one of its own per token
        pos = t + c["ctx"] if c["ctx"] == 0 else torch.randint(0, c["ctx"], (n,), device="cuda", generator=gen)
        return dict(c=c, q=q, k=k, v=v, pool=pool, q_out=empty((n, hq, d), dt), positions=pos.to(torch.int32),
                    slots=ids[t // page] * page + t % page, mscale=m,
                    inv_freq=torch.tensor(f, dtype=torch.float32, device="cuda"),
                    table=torch.tensor([x - 2 ** 64 if x >= 2 ** 63 else x for x in turns], dtype=torch.int64, device="cuda"))
    ctx, new = lengths(c)
    lens = [a + b for a, b in zip(ctx, new)]
    n, need = sum(new), [_pages(x, page) for x in lens]
    n_pages = sum(need) + 2
    pool = torch.empty(2, n_pages, H, page, d, dtype=dt, device="cuda")
    ks = _key_scale(H, d, gen)
    step = max(1, (1 << 27) // (H * page * d))
    for a in range(0, n_pages, step):
        b = min(n_pages, a + step)
        pool[0, a:b] = torch.randn(b - a, H, page, d, device="cuda", generator=gen) * ks
        pool[1, a:b] = torch.randn(b - a, H, page, d, device="cuda", generator=gen)
    table = torch.full((c["n_req"], max(need) + 1), -1, dtype=torch.int32, device="cuda")
    perm = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    need_t = torch.tensor(need)
    rows = torch.repeat_interleave(torch.arange(c["n_req"]), need_t)
    cols = torch.arange(sum(need)) - torch.repeat_interleave(torch.cumsum(need_t, 0) - need_t, need_t)
    table[rows.cuda(), cols.cuda()] = perm[:sum(need)]
    cu = [0]
    for b in new:
        cu.append(cu[-1] + b)
    return dict(c=c, max_len=max(lens), scale=d ** -0.5, pool=pool, block_table=table, seq_lens=i32(lens), cu_new=i32(cu),
                q=torch.randn(n, hq, d, device="cuda", generator=gen).to(dt), out=empty((n, hq, d), dt),
                lse=empty((n, hq), torch.float32))


# --------------------------------------------------------------------------- plain forms
def _plain_plan(s):
    page = s["c"]["page"]
    ctx, new = s["ctx_lens"].long(), s["new_lens"].long()
    lens = ctx + new
    have = (ctx + page - 1) // page
    fresh = (lens + page - 1) // page - have
    total = int(s["free_pages"].numel())                  # a bound that the host knows
    upto = torch.cumsum(fresh, 0)
    j = torch.arange(total, device="cuda")
    row = torch.searchsorted(upto, j, right=True)
    used = j < upto[-1]
    row = torch.where(used, row, 0)
    col = torch.where(used, have[row] + j - (upto - fresh)[row], s["block_table"].shape[1] - 1)
    at = torch.where(used, s["free_count"].long() - 1 - j, 0)
    table = s["block_table"]
    table[row, col] = torch.where(used, s["free_pages"][at], table[row, col])
    cu = torch.zeros(new.numel() + 1, dtype=torch.int64, device="cuda")
    cu[1:] = torch.cumsum(new, 0)
    t = torch.arange(s["n_tok"], device="cuda")
    r = torch.searchsorted(cu[1:], t, right=True)
    pos = ctx[r] + t - cu[r]
    return dict(block_table=table, seq_lens=lens.int(), cu_new=cu.int(), positions=pos.int(),
                slots=table[r, pos // page].long() * page + pos % page, free_left=(s["free_count"] - upto[-1]).int())


def _turn(x, cos, sin, rot, interleaved):
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * cos - b * sin, b * cos + a * sin
    y = x.clone()
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = u, v
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = u, v
    return y


def _plain_rotary(s):
    c, pool, page = s["c"], s["pool"], s["c"]["page"]
    angle = s["positions"].float()[:, None] * s["inv_freq"][None]
    cos, sin = (torch.cos(angle) * s["mscale"])[:, None], (torch.sin(angle) * s["mscale"])[:, None]
    s["q_out"].copy_(_turn(s["q"], cos, sin, c["rot"], c["interleaved"]))
    at, off = s["slots"] // page, s["slots"] % page
    pool[0][at, :, off] = _turn(s["k"], cos, sin, c["rot"], c["interleaved"]).to(pool.dtype)
    pool[1][at, :, off] = s["v"]
    return dict(q=s["q_out"], pool=pool)


def _plain_attention(s):
    c, page, H, d, rep = s["c"], s["c"]["page"], s["c"]["H"], s["c"]["d"], s["c"]["n_rep"]
    n_req, n, width = c["n_req"], s["q"].shape[0], _pages(s["max_len"], page)
    ids = s["block_table"][:, :width].long().clamp(min=0)
    # [n_req, H, tokens, d] in 32 bits
    k = s["pool"][0][ids].permute(0, 2, 1, 3, 4).float().reshape(n_req, H, width * page, d)
    v = s["pool"][1][ids].permute(0, 2, 1, 3, 4).float().reshape(n_req, H, width * page, d)
    cu, lens = s["cu_new"].long(), s["seq_lens"].long()
    i = torch.arange(c["new"], device="cuda")
    tok = (cu[:-1, None] + i).clamp(max=n - 1)                                      # padded to the longest chunk
    q = s["q"][tok].view(n_req, c["new"], H, rep, d).permute(0, 2, 1, 3, 4).float().reshape(n_req, H, c["new"] * rep, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    pos = (lens - (cu[1:] - cu[:-1]))[:, None] + i                                   # [n_req, new]
    t = torch.arange(width * page, device="cuda")
    hide = t > pos[..., None]
    if c["window"]:
        hide |= (t <= pos[..., None] - c["window"]) & (t >= c["sinks"])
    hide |= t >= lens[:, None, None]
    x.view(n_req, H, c["new"], rep, -1).masked_fill_(hide[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v) / total
    lse = top + torch.log(total)
    r = torch.repeat_interleave(torch.arange(n_req, device="cuda"), cu[1:] - cu[:-1], output_size=n)
    at = torch.arange(n, device="cuda") - cu[r]
    o = o.view(n_req, H, c["new"], rep, d)[r, :, at].reshape(n, H * rep, d)
    return dict(out=o.to(s["q"].dtype), lse=lse.view(n_req, H, c["new"], rep)[r, :, at].reshape(n, H * rep))


def run(s):
    c = s["c"]
    if not own:
        return {"plan": _plain_plan, "rotary": _plain_rotary, "attention": _plain_attention}[c["op"]](s)
    import paper_2607_20538_gb300 as cg
    if c["op"] == "plan":
        pages = cg.Pages(n_pages=s["n_pages"], page=c["page"], n_req=c["n_req"], max_pages=s["block_table"].shape[1])
        cg.page_plan(pages, s["ctx_lens"], s["new_lens"], s["free_pages"], s["free_count"], s["block_table"], s["seq_lens"],
                     s["cu_new"], s["positions"], s["slots"], s["free_left"])
        return {k: s[k] for k in ("block_table", "seq_lens", "cu_new", "positions", "slots", "free_left")}
    if c["op"] == "rotary":
        pages = cg.Pages(n_pages=s["pool"].shape[1], page=c["page"], H=c["H"], d=c["d"])
        turn = cg.Rotary(rot=c["rot"], interleaved=c["interleaved"], mscale=s["mscale"])
        cg.rotary_append(pages, turn, s["q"], s["k"], s["v"], s["positions"], s["slots"], s["table"], s["q_out"], s["pool"])
        return dict(q=s["q_out"], pool=s["pool"])
    pages = cg.Pages(n_pages=s["pool"].shape[1], page=c["page"], H=c["H"], d=c["d"], n_req=c["n_req"],
                     max_pages=s["block_table"].shape[1])
    how = cg.PagedAttention(n_rep=c["n_rep"], max_new=c["new"], scale=s["scale"], window=c["window"], sinks=c["sinks"])
    cg.paged_attention(pages, how, s["q"], s["pool"], s["block_table"], s["seq_lens"], s["cu_new"], s["out"], s["lse"])
    return dict(out=s["out"], lse=s["lse"])


# ------------------------------------------------------------------------- from the definition
def exact(c, seed):
    """What run returns, from the definition in 64 bits."""
    if c["op"] == "plan":
        return None                                       # whole numbers
    s = prepare(c, seed)
    if c["op"] == "rotary":
        f, m = frequencies(c)
        z = torch.exp(1j * s["positions"].double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda")) * m
        n, half = c["rot"], c["rot"] // 2

        def turned(x):
            x = x.double().clone()
            pairs = x[..., :n].reshape(*x.shape[:2], half, 2) if c["interleaved"] else x[..., :n].reshape(*x.shape[:2], 2, half).transpose(2, 3)
            w = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z[:, None])
            x[..., :n] = (w if c["interleaved"] else w.transpose(2, 3)).reshape(*x.shape[:2], n)
            return x
        pool = s["pool"].double().permute(0, 1, 3, 2, 4).reshape(2, -1, c["H"], c["d"])
        pool[0, s["slots"]] = turned(s["k"])
        pool[1, s["slots"]] = s["v"].double()
        pool = pool.reshape(2, -1, c["page"], c["H"], c["d"]).permute(0, 1, 3, 2, 4).contiguous()
        return dict(q=turned(s["q"]), pool=pool)
    w = work(c)
    if w["flops"] > 3e12:
        return None
    ctx, new = lengths(c)
    H, rep, d, page = c["H"], c["n_rep"], c["d"], c["page"]
    out = torch.empty(sum(new), H * rep, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(sum(new), H * rep, dtype=torch.float64, device="cuda")
    at = 0
    for i, (a, b) in enumerate(zip(ctx, new)):
        ids = s["block_table"][i, :_pages(a + b, page)].long()
        for h in range(H if b else 0):
            k, v = (s["pool"][x, ids, h].double().reshape(-1, d)[:a + b] for x in (0, 1))
            for lo in range(0, b, 512):
                hi = min(b, lo + 512)
                q = s["q"][at + lo:at + hi, h * rep:(h + 1) * rep].double()
                p, t = torch.arange(a + lo, a + hi, device="cuda")[:, None], torch.arange(a + b, device="cuda")
                seen = t <= p
                if c["window"]:
                    seen &= (t > p - c["window"]) | (t < c["sinks"])
                x = torch.einsum("nrd,td->rnt", q, k) * s["scale"]
                x = torch.where(seen, x, -math.inf)
                z = torch.logsumexp(x, -1)
                lse[at + lo:at + hi, h * rep:(h + 1) * rep] = z.T
                out[at + lo:at + hi, h * rep:(h + 1) * rep] = torch.einsum("rnt,td->nrd", torch.exp(x - z[..., None]), v)
        at += b
    return dict(out=out, lse=lse)
