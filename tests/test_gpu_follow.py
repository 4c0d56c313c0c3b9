"""Calls one behind the other, whose kernels come on while the one before ends: each sees what was written before it, and
what it reads is not written over early. Against the same calls with the GPU waited for after each."""
from __future__ import annotations

import threading

import pytest
import torch

import paper_2607_20538_gb300 as cg

pytestmark = pytest.mark.gpu
BF16, F32, I32, E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn
PAGE, H, D, REP, PAGES = 16, 2, 128, 4, 512


class Chain:
    """A step in which each call reads what the one before wrote, into the same buffers every time. nodes: of a tree (up to 4
    go to the attention's kernel for few rows, of which the next call's CTAs may come beside all of it); rows: of a product."""

    def __init__(self, nodes: int, rows: int, n_req: int = 3, ctx: int = 900):
        dev, self.nodes, self.n_req, n = "cuda", nodes, n_req, nodes * n_req
        per = -(-(ctx + nodes) // PAGE)
        i32 = lambda *s: torch.zeros(s, dtype=I32, device=dev)  # noqa: E731
        self.pages, self.how = cg.Pages(PAGES, PAGE, H, D, n_req, per), cg.PagedAttention(REP, nodes, D ** -0.5)
        self.lens = torch.tensor([ctx + nodes - 37 * i for i in range(n_req)], dtype=I32, device=dev)
        self.cu = torch.arange(n_req + 1, dtype=I32, device=dev) * nodes
        self.table = torch.randperm(PAGES, device=dev)[:n_req * per].to(I32).view(n_req, per).contiguous()
        self.parents, self.leaves, self.positions, self.masks = i32(n), i32(n_req), i32(n), i32(n, -(-nodes // 32))
        self.pool, self.q = torch.empty((2, PAGES, H, PAGE, D), dtype=BF16, device=dev), torch.empty((n, H * REP, D), dtype=BF16, device=dev)
        self.out = torch.empty_like(self.q)
        self.left, self.stack, self.count, self.free_left = i32(n_req), i32(PAGES), i32(1), i32(1)
        k = H * REP * D
        self.x = self.out.view(n, k).repeat(-(-rows // n), 1)[:rows].contiguous()
        self.codes, self.scales = torch.empty((rows, k), dtype=E4M3, device=dev), torch.empty((rows, k // 128), device=dev)
        self.w, self.wc, self.ws = (torch.empty((640, k), dtype=t, device=dev) for t in (BF16, E4M3, F32))
        self.ws = torch.empty((5, k // 128), device=dev)
        self.y = torch.empty((rows, 640), dtype=BF16, device=dev)
        self.workspace = torch.empty(cg.paged_attention_workspace_bytes(self.pages, self.how, n), dtype=torch.uint8, device=dev)
        self.seed = torch.zeros(1, device=dev)

    def step(self, after=lambda: None):
        n, r = self.nodes * self.n_req, self.n_req

        def noise(t, a):     # (values of the seed alone, by kernels that are there just before the call that reads them)
            i = torch.arange(t.numel(), device=t.device, dtype=F32).view(t.shape)
            t.copy_(torch.sin(i * 0.7311 + self.seed * a))
            after()

        node = torch.arange(n, device="cuda", dtype=I32) % self.nodes
        noise(self.pool, 3.1)
        noise(self.q, 1.7)
        self.parents.copy_(torch.minimum(node - 1, (node * 7 + self.seed.to(I32)) % torch.clamp(node, min=1)))
        cg.tree_plan(self.nodes, self.parents, self.lens, self.cu, self.positions, self.masks)
        after()
        cg.tree_attention(self.pages, self.how, self.q, self.pool, self.table, self.lens, self.cu, self.positions, self.masks, self.out,
                          workspace=self.workspace)
        after()
        rows = self.x.shape[0]
        self.x.copy_(self.out.view(n, -1)[torch.arange(rows, device="cuda") % n])
        cg.block8_encode(self.x, self.codes, self.scales)
        after()
        self.x.zero_()
        noise(self.w, 0.9)
        cg.block8_encode(self.w, self.wc, self.ws, rows=128)
        after()
        self.w.zero_()
        cg.block8_matmul(self.codes, self.scales, self.wc, self.ws, self.y)
        after()
        cg.block8_encode(self.y[:, :256], self.codes[:, :256], self.scales[:, :2].contiguous())    # over what the product read
        after()
        self.leaves.copy_((torch.arange(r, device="cuda") * 5 + self.seed).to(I32) % self.nodes)
        self.stack.zero_()
        self.count.zero_()
        cg.tree_commit(self.pages, self.nodes, self.parents, self.leaves, self.lens, self.cu, self.table, self.pool, self.left, self.stack,
                       self.count, self.free_left)
        after()
        cg.block8_encode(self.pool.view(-1, 1024)[:rows], self.wcodes(rows), self.wscales(rows))   # rows that have just moved
        after()
        cg.tree_plan(self.nodes, self.parents, self.left + self.nodes, self.cu, self.positions, self.masks)
        after()

    def wcodes(self, rows):
        return self._keep("_c", lambda: torch.empty((rows, 1024), dtype=E4M3, device="cuda"))

    def wscales(self, rows):
        return self._keep("_s", lambda: torch.empty((rows, 8), device="cuda"))

    def _keep(self, name, make):
        if not hasattr(self, name):
            setattr(self, name, make())
        return getattr(self, name)

    def results(self):
        return [t.clone() for t in (self.pool, self.positions, self.masks, self.out, self.codes.view(torch.uint8), self.scales, self.wc.view(torch.uint8),
                                    self.ws, self.y, self.left, self.stack, self.free_left, self._c.view(torch.uint8), self._s)]


SIZES = [(3, 5), (3, 300), (20, 5), (20, 60), (20, 2000)]
STEPS = 6


def _waited(c):
    want = []
    for k in range(STEPS):
        c.seed.fill_(float(k + 1))
        c.step(after=torch.cuda.synchronize)
        want.append(c.results())
    assert cg.get_status() == 0
    return want


def _same(got, want):
    for k, (g, w) in enumerate(zip(got, want)):
        for i, (a, b) in enumerate(zip(g, w)):
            assert torch.equal(a, b), (k, i)


@pytest.mark.parametrize("nodes,rows", SIZES)
def test_in_a_stream(nodes, rows):
    c = Chain(nodes, rows)
    want = _waited(c)
    for _ in range(4):
        got = []
        for k in range(STEPS):
            c.seed.fill_(float(k + 1))
            c.step()
            got.append(c.results())
        _same(got, want)
    assert cg.get_status() == 0


@pytest.mark.parametrize("nodes,rows", SIZES)
def test_in_a_graph(nodes, rows):
    c = Chain(nodes, rows)
    want = _waited(c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.step()
    for _ in range(4):
        got = []
        for k in range(STEPS):
            c.seed.fill_(float(k + 1))
            graph.replay()
            got.append(c.results())
        _same(got, want)
    assert cg.get_status() == 0


def _product(rows):
    x, w = torch.randn(rows, 1024, device="cuda").to(BF16), torch.randn(640, 1024, device="cuda").to(BF16)
    t = dict(x=x, w=w, xc=torch.empty_like(x, dtype=E4M3), wc=torch.empty_like(w, dtype=E4M3), xs=torch.empty((rows, 8), device="cuda"),
             ws=torch.empty((5, 8), device="cuda"), y=torch.empty((rows, 640), dtype=BF16, device="cuda"))
    return t


@pytest.mark.parametrize("rows", [5, 60, 2000])
@pytest.mark.parametrize("captured", [False, True])
def test_over_two_streams(rows, captured):
    """x and w are coded in a stream each; the product waits for both, the next step for the product. Copies and fills
    stand before the calls, and a call is a capture's first and its last."""
    t = _product(rows)
    side, main = torch.cuda.Stream(), torch.cuda.Stream()
    want = torch.empty_like(t["y"])
    cg.block8_encode(t["x"], t["xc"], t["xs"])
    cg.block8_encode(t["w"], t["wc"], t["ws"], rows=128)
    cg.block8_matmul(t["xc"], t["xs"], t["wc"], t["ws"], want)
    torch.cuda.synchronize()

    def step():
        cg.block8_encode(t["x"], t["xc"], t["xs"])
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            t["wc"].view(torch.uint8).zero_()
            t["ws"].zero_()
            cg.block8_encode(t["w"], t["wc"], t["ws"], rows=128)
        t["y"].zero_()
        t["xs"].copy_(t["xs"].clone())
        torch.cuda.current_stream().wait_stream(side)
        cg.block8_matmul(t["xc"], t["xs"], t["wc"], t["ws"], t["y"])

    side.wait_stream(torch.cuda.current_stream())
    main.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(main):
        step()
        torch.cuda.synchronize()
        assert torch.equal(t["y"], want)
        run = step
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=main):
                step()
            run = graph.replay
        for _ in range(20):
            t["y"].fill_(7.0)
            run()
            assert torch.equal(t["y"].clone(), want)
    assert cg.get_status() == 0


def test_four_threads():
    """Each with a stream and buffers of its own."""
    chains = [Chain(*s) for s in ((3, 5), (20, 300), (7, 60), (20, 5))]
    want = [_waited(c) for c in chains]
    got, failed = [None] * len(chains), []

    def run(k):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(3):
                    got[k] = []
                    for n in range(STEPS):
                        chains[k].seed.fill_(float(n + 1))
                        chains[k].step()
                        got[k].append(chains[k].results())
            stream.synchronize()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(k,)) for k in range(len(chains))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    for g, w in zip(got, want):
        _same(g, w)
    assert cg.get_status() == 0
