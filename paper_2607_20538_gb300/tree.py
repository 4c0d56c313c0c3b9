"""Trees of drafted tokens over the paged cache: plan, attention and commit (``include/codecgauge_tree.h``).

Bindings of the C entry points with the same names, in the manner of ``paged.py``.
"""
from __future__ import annotations

from . import _check
from . import paged as _p
from .paged import PagedAttention, Pages


def _masks(masks, n: int, dev: int):
    """Address and words a row of the masks [n][words] on the device."""
    if masks.dtype is not _p._INT32 or masks.get_device() != dev or masks.dim() != 2 or masks.shape[0] != n or not masks.is_contiguous():
        _p._bad(f"masks: expected a contiguous int32 tensor [{n}, words] on device {dev}")
    return masks.data_ptr(), masks.shape[1]


def tree_plan(max_new: int, parents, seq_lens, cu_new, positions, masks, window: int = 0, sinks: int = 0, stream=None) -> None:
    """Positions and masks of the nodes of every request's tree (cg_tree_plan). The number of requests is
    seq_lens.numel(), of rows positions.numel(); masks int32 [rows][words], 32 words >= max_new."""
    dev = _p._device()
    if dev >= 0 and _p._took("tree_plan", max_new, window, sinks, parents, seq_lens, cu_new, positions, masks, dev, _p._stream(stream)):
        return
    r, n = seq_lens.numel(), positions.numel()
    mp, words = _masks(masks, n, dev)
    _check(_p._fn("cg_tree_plan")(
        r, n, max_new, window, sinks, _p._i32("parents", parents, n, dev), _p._i32("seq_lens", seq_lens, r, dev),
        _p._i32("cu_new", cu_new, r + 1, dev), _p._i32("positions", positions, n, dev), mp, words, _p._stream(stream)))


def tree_attention(pages: Pages, how: PagedAttention, q, pool, block_table, seq_lens, cu_new, positions, masks, out, lse=None,
                   workspace=None, stream=None) -> None:
    """paged_attention of the nodes: each over its request's history and the nodes of its mask
    (cg_tree_attention). positions may be None without a window; the workspace is paged_attention's."""
    n, dev = q.shape[0], _p._device()
    if q.get_device() == dev:
        room = _p._workspace(pages, how, n, q.device, stream) if workspace is None else workspace
        if _p._took("tree_attention", pages, how, q, pool, block_table, seq_lens, cu_new, positions, masks, out, lse, room, dev,
                    _p._stream(stream)):
            return
    mp, words = _masks(masks, n, dev)
    if positions is None and how.window:
        _p._bad("positions: needed with a window")
    pp = None if positions is None else _p._i32("positions", positions, n, dev)
    _p.paged_attention(pages, how, q, pool, block_table, seq_lens, cu_new, out, lse, workspace, stream, _tree=(words, pp, mp))


def tree_commit(pages: Pages, max_new: int, parents, leaves, seq_lens, cu_new, block_table, pool, lens_left=None, free_pages=None,
                free_count=None, free_left=None, stream=None) -> None:
    """Keys and values of the accepted paths move up behind the history, the pages that no token is left in go
    back on the stack (cg_tree_commit). leaves: each request's accepted node, -1: none. pool: one layer's
    [2][n_pages][H][page][d], several [layers][2][n_pages][H][page][d], or None (lengths and pages alone); without
    lens_left, free_pages, free_count and free_left only rows move."""
    dev = _p._device()
    if dev >= 0 and _p._took("tree_commit", pages, max_new, parents, leaves, seq_lens, cu_new, block_table, pool, lens_left,
                             free_pages, free_count, free_left, dev, _p._stream(stream)):
        return
    n, r = parents.numel(), pages.n_req
    layers, pp, elem = 0, None, _p.CG_BF16
    if pool is not None:
        layers, elem = (pool.shape[0] if pool.dim() == 6 else 1), _p._elem(pool)
        if pool.shape[-5:] != (2, pages.n_pages, pages.H, pages.page, pages.d) or pool.dim() not in (5, 6) or not pool.is_contiguous() \
                or pool.get_device() != dev or layers < 1:
            _p._bad(f"pool: expected a contiguous tensor [layers, 2, {pages.n_pages}, {pages.H}, {pages.page}, {pages.d}] on device {dev}, "
                    f"got {list(pool.shape)}")
        pp = pool.data_ptr()
    give = [lens_left, free_pages, free_count, free_left]
    if any(t is None for t in give) and not all(t is None for t in give):
        _p._bad("lens_left, free_pages, free_count and free_left go together")
    lp, fp, cp, op = (None,) * 4 if lens_left is None else (
        _p._i32("lens_left", lens_left, r, dev), _p._i32("free_pages", free_pages, pages.n_pages, dev),
        _p._i32("free_count", free_count, 1, dev), _p._i32("free_left", free_left, 1, dev))
    _check(_p._fn("cg_tree_commit")(
        pages.c(elem), n, max_new, layers, _p._i32("parents", parents, n, dev), _p._i32("leaves", leaves, r, dev),
        _p._i32("seq_lens", seq_lens, r, dev), _p._i32("cu_new", cu_new, r + 1, dev),
        _p._i32("block_table", block_table, r * pages.max_pages, dev), pp, lp, fp, cp, op, _p._stream(stream)))
