"""Library calls with nothing between them, each of which reads what the one before wrote, or writes over what it still reads, or
writes where it has written: kernels that come while the one before ends wait for it. Against the same calls with the GPU waited for
after each. The older calls of the paged cache, whose kernels are launched in the plain way or let the next one come early, are among
them."""
from __future__ import annotations

import pytest
import torch

import paper_2607_20538_gb300 as cg

pytestmark = pytest.mark.gpu
BF16, F32, I32, I64, U8, E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.uint8, torch.float8_e4m3fn
PAGE, H, D, REP, PAGES = 16, 2, 128, 4, 1024
WIDTH = H * REP * D       # channels of a row of queries: those that the products take


def _i32(*s):
    return torch.zeros(s, dtype=I32, device="cuda")


class World:
    """All buffers of a step, made before it. The requests' last pages are the pool's first ones, in order, so that a matrix of
    `moved` rows over the pool's start is what a commit moves."""

    def __init__(self, nodes: int, rows: int, n_req: int = 4, ctx: int = 3000):
        self.nodes, self.rows, self.n_req, n = nodes, rows, n_req, nodes * n_req
        per = -(-(ctx + nodes) // PAGE)
        self.pages, self.how = cg.Pages(PAGES, PAGE, H, D, n_req, per), cg.PagedAttention(REP, nodes, D ** -0.5)
        self.last = last = -(-nodes // PAGE) + 1          # pages of a request that may hold nodes
        self.lens0 = torch.tensor([ctx + nodes - PAGE * i for i in range(n_req)], dtype=I32, device="cuda")
        self.ctx0 = self.lens0 - nodes
        self.cu0 = torch.arange(n_req + 1, dtype=I32, device="cuda") * nodes
        table = (torch.randperm(PAGES - n_req * last, generator=torch.Generator().manual_seed(5)) + n_req * last)[:n_req * per].view(n_req, per)
        for i in range(n_req):
            end = -(-int(self.lens0[i]) // PAGE)
            table[i, end - last:end] = torch.arange(i * last, (i + 1) * last)
        self.table0 = table.to(I32).cuda().contiguous()
        free = sorted(set(range(PAGES)) - set(table.view(-1).tolist()))
        self.stack0 = torch.tensor(free + [0] * (PAGES - len(free)), dtype=I32, device="cuda")
        self.count0 = torch.tensor([len(free)], dtype=I32, device="cuda")
        tokens = [[int(self.ctx0[i]) + k for k in range(nodes)] for i in range(n_req)]
        self.slots0 = torch.tensor([int(table[i, t // PAGE]) * PAGE + t % PAGE for i in range(n_req) for t in tokens[i]], dtype=I64, device="cuda")
        self.done0 = torch.arange(n_req, dtype=I32, device="cuda") % 2
        self.turn, self.frequencies = cg.Rotary(D), cg.rotary_table(D)[0]
        self.new = torch.full((n_req,), nodes, dtype=I32, device="cuda")
        b = self.b = {}
        b["lens"], b["cu"], b["table"], b["ctx"] = self.lens0.clone(), self.cu0.clone(), self.table0.clone(), self.ctx0.clone()
        b["parents"], b["leaves"], b["positions"], b["masks"] = _i32(n), _i32(n_req), _i32(n), _i32(n, -(-nodes // 32))
        b["slots"] = torch.zeros(n, dtype=I64, device="cuda")
        b["chain"], b["done"] = _i32(n), _i32(n_req)
        b["left"], b["stack"], b["count"], b["free_left"] = _i32(n_req), _i32(PAGES), _i32(1), _i32(1)
        new = lambda dt, *s: torch.empty(s, dtype=dt, device="cuda")  # noqa: E731
        b["pool"] = new(BF16, 2, PAGES, H, PAGE, D)
        b["q"], b["k"], b["v"] = (new(BF16, n, h, D) for h in (H * REP, H, H))
        b["turned"], b["out"] = torch.empty_like(b["q"]), torch.empty_like(b["q"])
        self.moved = n_req * last * H * PAGE
        for x, codes, scales, r, k in (("x", "codes", "scales", rows, WIDTH), ("out", "nc", "ns", n, WIDTH), ("pool", "pc", "ps", self.moved, D),
                                       ("small", "sc", "ss", 4096, 256)):
            b[codes], b[scales] = new(E4M3, r, k), new(F32, r, k // 128)
            if x not in b:
                b[x] = new(BF16, r, k)
        b["w"], b["wc"], b["ws"], b["y"] = new(BF16, 640, WIDTH), new(E4M3, 640, WIDTH), new(F32, 5, WIDTH // 128), new(BF16, rows, 640)
        b["ws2"] = new(U8, cg.paged_attention_workspace_bytes(self.pages, self.how, n))
        seeded = lambda i: torch.Generator(device="cuda").manual_seed(i)  # noqa: E731
        self.noise = {k: torch.randn(v.shape, generator=seeded(i), device="cuda").to(BF16) for i, (k, v) in enumerate(b.items()) if v.dtype is BF16}
        self.codes0 = {k: torch.randint(0, 0x78, v.shape, generator=seeded(i), device="cuda", dtype=U8) for i, (k, v) in enumerate(b.items())
                       if v.dtype is E4M3}
        node = torch.arange(n, device="cuda", dtype=I32) % nodes
        self.parents0, self.chain0 = node * 3 // 4 - 1, node - 1
        self.leaves0 = torch.tensor([nodes - 1 - i % 2 for i in range(n_req)], dtype=I32, device="cuda")
        self.reset()
        self.call("tree_plan")
        self.masks0, self.positions0 = b["masks"].clone(), b["positions"].clone()

    def reset(self):
        b = self.b
        for k, v in self.noise.items():
            b[k].copy_(v)
        for k, v in self.codes0.items():
            b[k].view(U8).copy_(v)
        for k in ("scales", "ws", "ns", "ps", "ss"):
            b[k].fill_(1.0)
        for k, v in b.items():
            if v.dtype in (I32, I64):
                v.copy_(getattr(self, k + "0")) if hasattr(self, k + "0") else v.zero_()

    def call(self, name, **kw):
        b = dict(self.b, **kw)
        n, k = self.nodes * self.n_req, self.nodes
        if name == "tree_plan":
            cg.tree_plan(k, b["parents"], b["lens"], b["cu"], b["positions"], b["masks"])
        elif name == "tree_attention":
            cg.tree_attention(self.pages, self.how, b["q"], b["pool"], b["table"], b["lens"], b["cu"], b["positions"], b["masks"], b["out"],
                              workspace=b["ws2"])
        elif name == "paged_attention":
            cg.paged_attention(self.pages, self.how, b["q"], b["pool"], b["table"], b["lens"], b["cu"], b["out"], workspace=b["ws2"])
        elif name == "tree_commit":
            cg.tree_commit(self.pages, k, b["parents"], b["leaves"], b["lens"], b["cu"], b["table"], b["pool"], b["left"], b["stack"], b["count"],
                           b["free_left"])
        elif name == "page_plan":
            cg.page_plan(self.pages, b["ctx"], self.new, b["stack"], b["count"], b["table"], b["lens"], b["cu"], b["positions"], b["slots"],
                         b["free_left"])
        elif name == "page_release":
            cg.page_release(self.pages, b["lens"], b["done"], b["table"], b["stack"], b["count"], b["left"], b["free_left"])
        elif name == "rotary_append":
            cg.rotary_append(self.pages, self.turn, b["q"], b["k"], b["v"], b["positions"], b["slots"], self.frequencies, b["turned"],
                             b["pool"])
        elif name == "encode":
            cg.block8_encode(b["x"], b["codes"], b["scales"])
        elif name == "encode_w":
            cg.block8_encode(b["w"], b["wc"], b["ws"], rows=128)
        elif name == "encode_queries":                            # of the nodes
            cg.block8_encode(b["out"].view(n, WIDTH), b["nc"], b["ns"])
        elif name == "encode_moved":
            cg.block8_encode(b["pool"].view(-1, D)[:self.moved], b["pc"], b["ps"])
        else:
            assert name == "matmul"
            cg.block8_matmul(b["codes"], b["scales"], b["wc"], b["ws"], b["y"])

    def results(self):
        return {k: v.view(U8).clone() for k, v in self.b.items() if k != "ws2"}


def _small_over(key):
    """An encoding whose codes lie in the place of the buffer `key` (all of it, or the first MB)."""
    def call(w):
        t = w.b[key].view(-1).view(U8)
        rows = min(4096, t.numel() // 256)
        cg.block8_encode(w.b["small"][:rows], t[:rows * 256].view(rows, 256).view(E4M3), w.b["ss"][:rows])
    return call


def _just(name, **kw):
    return lambda w: w.call(name, **{k: v(w) for k, v in kw.items()})


CHAINS = {
    # what the one before wrote
    "encode, matmul": [_just("encode"), _just("matmul")],
    "encode_w, matmul": [_just("encode_w"), _just("matmul")],
    "matmul, encode of its result": [_just("matmul"), lambda w: cg.block8_encode(w.b["y"][:, :256], w.b["sc"][:w.rows], w.b["ss"][:w.rows])],
    "matmul, matmul into the same": [_just("matmul"), _just("matmul", codes=lambda w: w.b["wc"][:w.rows] if w.rows <= 640 else w.b["codes"])],
    "plan, attention": [_just("tree_plan"), _just("tree_attention")],
    "attention, encode": [_just("tree_attention"), _just("encode_queries")],
    "commit, encode of moved rows": [_just("tree_commit"), _just("encode_moved")],
    "commit, attention over moved rows": [_just("tree_commit"), _just("tree_attention")],
    "commit, plan of what is left": [_just("tree_commit"), _just("tree_plan", lens=lambda w: w.b["left"])],
    # what the one before may still read
    "matmul, encode over its codes": [_just("matmul"), _just("encode")],
    "matmul, encode_w over its codes": [_just("matmul"), _just("encode_w")],
    "attention, plan over its masks": [_just("tree_attention"), _just("tree_plan", parents=lambda w: w.b["chain"])],
    "attention, commit of rows that it reads": [_just("tree_attention"), _just("tree_commit")],
    "attention, codes over its queries": [_just("tree_attention"), _small_over("q")],
    "attention, codes over its pool": [_just("tree_attention"), _small_over("pool")],
    "encode, attention over its input": [_just("encode_queries"), _just("tree_attention")],
    "encode_moved, commit": [_just("encode_moved"), _just("tree_commit")],
    "plan, commit over its lengths": [_just("tree_plan", lens=lambda w: w.b["ctx"], cu=lambda w: w.b["cu"]), _just("tree_commit", left=lambda w: w.b["ctx"])],
    "commit, codes over its pool": [_just("tree_commit"), _small_over("pool")],
    # with the calls of before
    "page_plan, plan": [_just("page_plan"), _just("tree_plan")],
    "plan, page_plan over its lengths": [_just("tree_plan"), _just("page_plan", ctx=lambda w: w.b["left"])],
    "rotary_append, attention": [_just("rotary_append"), _just("tree_attention", q=lambda w: w.b["turned"])],
    "rotary_append, encode": [_just("rotary_append"), _just("encode_queries", out=lambda w: w.b["turned"])],
    "attention, rotary_append over its pool": [_just("tree_attention"), _just("rotary_append")],
    "commit, rotary_append": [_just("tree_commit"), _just("rotary_append")],
    "paged, encode": [_just("paged_attention"), _just("encode_queries")],
    "paged, codes over its queries": [_just("paged_attention"), _small_over("q")],
    "paged, codes over its pool": [_just("paged_attention"), _small_over("pool")],
    "paged, commit of rows that it reads": [_just("paged_attention"), _just("tree_commit")],
    "paged, attention": [_just("paged_attention"), _just("tree_attention")],
    "attention, paged": [_just("tree_attention"), _just("paged_attention", out=lambda w: w.b["turned"])],
    "paged, matmul, encode": [_just("paged_attention"), _just("matmul"), _just("encode_queries")],
    "commit, page_release": [_just("tree_commit"), _just("page_release", lens=lambda w: w.b["left"], left=lambda w: w.b["ctx"], count=lambda w: w.b["free_left"],
                                                         free_left=lambda w: w.b["count"])],
    "page_release, plan": [_just("page_release"), _just("tree_plan", lens=lambda w: w.b["left"])],
    # a whole step, twice
    "step": 2 * [_just("page_plan"), _just("tree_plan"), _just("rotary_append"), _just("tree_attention", q=lambda w: w.b["turned"]), _just("encode_queries"),
                 _just("encode"), _just("encode_w"), _just("matmul"), _just("encode"),
                 _just("tree_commit", count=lambda w: w.b["free_left"], free_left=lambda w: w.b["count"]), _just("encode_moved"), _just("paged_attention"),
                 _just("encode_queries"), _just("matmul"), _just("page_release", lens=lambda w: w.b["left"], left=lambda w: w.b["ctx"])],
}


@pytest.mark.parametrize("nodes,rows", [(3, 5), (3, 300), (20, 60), (20, 4000)])
def test_chains(nodes, rows):
    """Each in a stream, behind a kernel long enough for all its launches to be there before its first one starts, and in a graph."""
    w = World(nodes, rows)
    stream = torch.cuda.Stream()
    moved = 0
    for name, calls in CHAINS.items():
        w.reset()
        for c in calls:
            c(w)
            torch.cuda.synchronize()
        want = w.results()
        w.reset()
        if "commit" in name:
            start = w.b["pool"].view(U8).view(-1)[:w.moved * D * 2]
            before = start.clone()
            w.call("tree_commit")
            moved += not torch.equal(before, start)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for _ in range(3):
                w.reset()
                torch.cuda._sleep(1500000)
                for c in calls:
                    c(w)
                got = w.results()
                stream.synchronize()
                assert all(torch.equal(got[k], want[k]) for k in want), (name, [k for k in want if not torch.equal(got[k], want[k])])
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                for c in calls:
                    c(w)
            for _ in range(3):
                w.reset()
                graph.replay()
                got = w.results()
                stream.synchronize()
                assert all(torch.equal(got[k], want[k]) for k in want), (name, "graph", [k for k in want if not torch.equal(got[k], want[k])])
        torch.cuda.synchronize()
    assert moved >= 5          # the rows that a commit moves are among those that the encoding reads
    cg.get_status()            # (lengths that a chain mixes up may raise the flag of wrong lengths)
