"""A small serving loop of one attention layer on a paged cache.

Each step takes the new tokens of a batch of requests (a prompt, a chunk or one token each) through
    page_plan        pages for them out of the free stack, positions and pool slots
    rotary_append    queries and keys turned by their positions, keys and values into their pages
    paged_attention  the new tokens over the pages of their own request
and page_release gives a finished request's pages back. Drafted continuations of the requests go through
    tree_plan        positions and masks of each tree's nodes
    tree_attention   the nodes over their request's pages and their own ancestors
    tree_commit      the accepted path's keys and values move up, spare pages go back
instead of paged_attention. The pool is at the same time a cache of the
codec (one layer, the pages as the batch): at the end all pages are encoded and restored, and the next
token attends over the restored pages.

    python examples/paged_serving.py [--steps 16] [--bits 4]
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_20538_gb300 as cg  # noqa: E402
from paper_2607_20538_gb300 import paged, synth  # noqa: E402


class PagedLayer:
    """Pool, block table and free stack of one layer, and what one step needs beside its tokens."""

    def __init__(self, n_req, max_tokens, H=8, n_rep=4, d=128, page=64, n_pages=None, window=0, sinks=0, dtype=torch.bfloat16,
                 base=500000.0, device="cuda"):
        self.max_pages = -(-max_tokens // page)
        self.pages = cg.Pages(n_pages or n_req * self.max_pages, page, H, d, n_req, self.max_pages)
        self.n_rep, self.window, self.sinks, self.device = n_rep, window, sinks, device
        i32 = dict(dtype=torch.int32, device=device)
        n = self.pages.n_pages
        # every page starts with finite contents: what no token has written yet is coded too
        self.pool = torch.zeros(2, n, H, page, d, dtype=dtype, device=device)
        self.block_table = torch.full((n_req, self.max_pages), -1, **i32)
        self.free_pages = torch.arange(n, **i32)
        self.free_count, self.free_left = torch.full((1,), n, **i32), torch.empty(1, **i32)
        self.lens, self.next_lens, self.cu_new = torch.zeros(n_req, **i32), torch.empty(n_req, **i32), torch.empty(n_req + 1, **i32)
        self.table, self.mscale = cg.rotary_table(d, cg.RopeScaling(kind=paged.CG_ROPE_BANDS, base=base, factor=8.0), device)
        self.turn = cg.Rotary(rot=d, mscale=self.mscale)

    def step(self, new_lens, q, k, v, max_new, out=None, pool=None):
        """New tokens of every request, in the requests' order: q [n][H * n_rep][d], k and v [n][H][d];
        new_lens [n_req] (int32, device), none above max_new. Returns o, like q. With `pool` the pages
        are read from there instead (the new tokens are put there too)."""
        n = k.shape[0]
        pool = self.pool if pool is None else pool
        out = torch.empty_like(q) if out is None else out
        positions = torch.empty(n, dtype=torch.int32, device=self.device)
        slots = torch.empty(n, dtype=torch.int64, device=self.device)
        cg.page_plan(self.pages, self.lens, new_lens, self.free_pages, self.free_count, self.block_table, self.next_lens, self.cu_new,
                     positions, slots, self.free_left)
        turned = torch.empty_like(q)
        cg.rotary_append(self.pages, self.turn, q, k, v, positions, slots, self.table, turned, pool)
        how = cg.PagedAttention(self.n_rep, max_new, 1.0 / math.sqrt(self.pages.d), self.window, self.sinks)
        cg.paged_attention(self.pages, how, turned, pool, self.block_table, self.next_lens, self.cu_new, out)
        self.lens, self.next_lens = self.next_lens, self.lens
        self.free_count, self.free_left = self.free_left, self.free_count
        return out

    def verify(self, new_lens, parents, q, k, v, max_new, accept):
        """Drafted trees of every request as one step: parents int32 [n] (a node's place in its tree, -1: the last token held), q, k,
        v as in step. accept(o) gives each request's accepted node (int32 [n_req], -1: none) from the nodes' outputs; those on
        its path stay. Returns o."""
        n = k.shape[0]
        i32 = dict(dtype=torch.int32, device=self.device)
        positions, masks, kept = torch.empty(n, **i32), torch.empty(n, -(-max_new // 32), **i32), torch.empty_like(self.lens)
        slots = torch.empty(n, dtype=torch.int64, device=self.device)
        cg.page_plan(self.pages, self.lens, new_lens, self.free_pages, self.free_count, self.block_table, self.next_lens, self.cu_new,
                     positions, slots, self.free_left)
        cg.tree_plan(max_new, parents, self.next_lens, self.cu_new, positions, masks, self.window, self.sinks)
        turned, out = torch.empty_like(q), torch.empty_like(q)
        cg.rotary_append(self.pages, self.turn, q, k, v, positions, slots, self.table, turned, self.pool)
        how = cg.PagedAttention(self.n_rep, max_new, 1.0 / math.sqrt(self.pages.d), self.window, self.sinks)
        cg.tree_attention(self.pages, how, turned, self.pool, self.block_table, self.next_lens, self.cu_new, positions, masks, out)
        cg.tree_commit(self.pages, max_new, parents, accept(out), self.next_lens, self.cu_new, self.block_table, self.pool, kept,
                       self.free_pages, self.free_left, self.free_count)
        self.lens = kept
        return out

    def release(self, done):
        """Give back the pages of the requests whose flag (int32 [n_req]) is set."""
        cg.page_release(self.pages, self.lens, done, self.block_table, self.free_pages, self.free_count, self.next_lens, self.free_left)
        self.lens, self.next_lens = self.next_lens, self.lens
        self.free_count, self.free_left = self.free_left, self.free_count

    def coded(self, bits=4, group=64, seed=0):
        """The pool through the codec: encoded with random orthogonal gauges and restored, and the
        codes' bytes per byte of the pool."""
        p = self.pages
        shape, params = cg.Shape(1, p.n_pages, p.H, p.page, p.d), cg.Params(cg.CG_BLOCK_UNIFORM, group, bits, block=group)
        rng = np.random.default_rng(seed)
        gauges = np.stack([synth.random_orthogonal(group, rng) for _ in range(2 * p.H * (p.d // group))]).astype(np.float32)
        gauges = torch.from_numpy(gauges).to(self.device)
        n_codes, n_scales, _ = cg.packed_bytes(shape, params)
        codes = torch.empty(n_codes, dtype=torch.uint8, device=self.device)
        scales = torch.empty(n_scales, dtype=torch.uint8, device=self.device)
        restored = torch.empty_like(self.pool)
        cg.encode(shape, params, self.pool, gauges, codes, scales)
        cg.decode(shape, params, codes, scales, None, gauges, restored)
        return restored, (n_codes + n_scales) / (2 * self.pool.numel())


def tokens(n, layer, gen):
    p = layer.pages
    make = lambda heads: torch.randn(n, heads, p.d, generator=gen, device=layer.device).to(layer.pool.dtype)  # noqa: E731
    return make(p.H * layer.n_rep), make(p.H), make(p.H)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=16, help="single-token steps after the prompts")
    ap.add_argument("--bits", type=int, default=4, choices=[2, 3, 4, 6, 8])
    a = ap.parse_args(argv)
    prompts = [700, 33, 1500, 256]
    layer = PagedLayer(n_req=len(prompts), max_tokens=max(prompts) + a.steps + 64)
    gen = torch.Generator(device=layer.device).manual_seed(0)
    i32 = dict(dtype=torch.int32, device=layer.device)

    layer.step(torch.tensor(prompts, **i32), *tokens(sum(prompts), layer, gen), max_new=max(prompts))
    ones = torch.ones(len(prompts), **i32)
    for _ in range(a.steps):
        layer.step(ones, *tokens(len(prompts), layer, gen), max_new=1)
    print(f"{sum(prompts)} prompt tokens and {a.steps} steps: {layer.pages.n_pages - int(layer.free_count)} pages of {layer.pages.page} in use")

    # request 0 is done; request 1's slot stays, and a new prompt takes the freed one
    layer.release(torch.tensor([1, 0, 0, 0], **i32))
    new = torch.tensor([90, 1, 1, 1], **i32)
    layer.step(new, *tokens(93, layer, gen), max_new=90)
    print(f"after a release and a new prompt of 90: lengths {layer.lens.tolist()}, "
          f"{layer.pages.n_pages - int(layer.free_count)} pages in use")

    # a drafted tree of 6 nodes for each request: two continuations of two tokens and one of one behind a common first;
    # here the first node's second child is accepted for all, which leaves two tokens
    parents = torch.tensor([-1, 0, 1, 0, 3, 0] * len(prompts), **i32)
    layer.verify(6 * ones, parents, *tokens(6 * len(prompts), layer, gen), max_new=6, accept=lambda o: 3 * ones)
    print(f"after a step of drafted trees: lengths {layer.lens.tolist()}, {layer.pages.n_pages - int(layer.free_count)} pages in use")

    # the same next token over the pages and over the pages as the codec restores them
    restored, ratio = layer.coded(a.bits)
    state = layer.lens, layer.next_lens, layer.free_count, layer.free_left, layer.block_table.clone()
    x = tokens(len(prompts), layer, gen)
    over_pages = layer.step(ones, *x, max_new=1)
    layer.lens, layer.next_lens, layer.free_count, layer.free_left = state[:4]
    layer.block_table.copy_(state[4])
    over_codes = layer.step(ones, *x, max_new=1, pool=restored)
    diff = (over_codes.float() - over_pages.float()).norm() / over_pages.float().norm()
    print(f"{a.bits}-bit pages ({100 * ratio:.0f} % of the bytes): attention off by {100 * float(diff):.1f} %")
    flags = cg.get_status()
    if flags:
        raise SystemExit(f"status flags {flags:#x}")
    return float(diff)


if __name__ == "__main__":
    main()
