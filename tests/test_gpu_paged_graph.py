"""A whole serving step (plan, rotary append, attention) and a release in a CUDA graph: replayed, they follow
the lengths, tables and stack that the replay before left on the device."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("new", [[1, 1, 1], [7, 1, 20]])
def test_steps_and_release_in_a_graph(new):
    from paged_serving import PagedLayer, tokens
    i32 = dict(dtype=torch.int32, device="cuda")
    make = lambda: PagedLayer(n_req=3, max_tokens=400, H=2, n_rep=4, d=64, page=16)  # noqa: E731
    eager, graphed = make(), make()
    gen = torch.Generator(device="cuda").manual_seed(6)
    prompt, n = [70, 3, 45], sum(new)
    x = tokens(sum(prompt), eager, gen)
    for layer in (eager, graphed):
        layer.step(torch.tensor(prompt, **i32), *x, max_new=70)
    lens, done = torch.tensor(new, **i32), torch.tensor([0, 1, 0], **i32)
    stream = torch.cuda.Stream()
    held = [tokens(n, graphed, gen) for _ in range(2)]
    out = [torch.empty_like(t[0]) for t in held]
    # one step, and a release that leaves the second request at 0 tokens; then another step and release: the
    # layer's two sets of lengths and counts are back in their places
    saved = [t.clone() for t in (graphed.pool, graphed.block_table, graphed.lens, graphed.free_pages, graphed.free_count)]

    def steps():
        for t, o in zip(held, out):
            graphed.step(lens, *t, max_new=max(new), out=o)
            graphed.release(done)

    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        steps()                                     # warm-up, undone below
    torch.cuda.current_stream().wait_stream(stream)
    for t, s in zip((graphed.pool, graphed.block_table, graphed.lens, graphed.free_pages, graphed.free_count), saved):
        t.copy_(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        steps()
    for _ in range(4):
        for t in held:
            for a, b in zip(t, tokens(n, graphed, gen)):
                a.copy_(b)
        g.replay()
        for t, o in zip(held, out):
            want = eager.step(lens, *t, max_new=max(new))
            eager.release(done)
            assert torch.equal(o, want)
        assert torch.equal(graphed.lens, eager.lens) and torch.equal(graphed.free_count, eager.free_count)
        assert torch.equal(graphed.block_table, eager.block_table) and torch.equal(graphed.free_pages, eager.free_pages)
    assert torch.equal(graphed.pool, eager.pool) and graphed.lens.tolist() == [70 + 8 * new[0], 0, 45 + 8 * new[2]]
    assert cg.get_status() == 0
