"""Paged KV cache: page plan, rotary append and paged attention (``include/codecgauge_paged.h``).

Bindings of the C entry points with the same names; the tensors' shapes, types and strides are
checked here, everything else by the library. A pool is a tensor [2][n_pages][H][page][d] (bf16 or
fp16; 0 keys, 1 values), the codec's cache layout with one layer and the pages as the batch.
"""
from __future__ import annotations

import ctypes
import struct
import threading
from typing import NamedTuple

import torch

from . import CodecGaugeError, _check, load

CG_BF16, CG_FP16 = 0, 1
CG_ROPE_NONE, CG_ROPE_LINEAR, CG_ROPE_BANDS, CG_ROPE_YARN = 0, 1, 2, 3


def _packed(fmt: str):
    """The C struct of these members (native sizes and alignment) as bytes: their address is what the
    entry points take. A third of the time of a ctypes.Structure, in calls of a few microseconds."""
    pack = struct.Struct("@" + fmt).pack

    def make(*members) -> bytes:
        try:
            return pack(*members)
        except (struct.error, OverflowError) as e:
            raise CodecGaugeError(-1, f"a parameter does not fit its type: {e}") from None
    return make


_CPages = _packed("7i")        # dtype, n_pages, page, H, d, n_req, max_pages
_CRotary = _packed("3if")      # rot, interleaved, transpose, mscale
_CScaling = _packed("i5d")     # kind, base, factor, original, low, high
_CStrides = _packed("8q")      # q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head
_CPagedAttn = _packed("5if4q")  # n_tok, n_rep, max_new, window, sinks, scale, q_tok, q_head, o_tok, o_head


class Pages(NamedTuple):
    """Pool geometry (n_pages pages of `page` tokens, H KV heads of d channels) and block table
    [n_req][max_pages]. The plan and the release use neither H nor d."""
    n_pages: int
    page: int
    H: int = 1
    d: int = 128
    n_req: int = 1
    max_pages: int = 1

    def c(self, dtype: int = CG_BF16) -> bytes:
        return _CPages(dtype, self.n_pages, self.page, self.H, self.d, self.n_req, self.max_pages)


class Rotary(NamedTuple):
    """The first `rot` channels of a head turn; see cg_rotary_params."""
    rot: int
    interleaved: bool = False
    mscale: float = 1.0
    transpose: bool = False

    def c(self) -> bytes:
        return _CRotary(self.rot, int(self.interleaved), int(self.transpose), self.mscale)


class RopeScaling(NamedTuple):
    """Frequency rule of rotary_table: kind CG_ROPE_NONE, _LINEAR, _BANDS or _YARN."""
    kind: int = CG_ROPE_NONE
    base: float = 10000.0
    factor: float = 1.0
    original: float = 8192.0
    low: float = 1.0
    high: float = 4.0


class PagedAttention(NamedTuple):
    """n_rep query heads per KV head, at most max_new new tokens per request; see cg_paged_attn."""
    n_rep: int
    max_new: int
    scale: float
    window: int = 0
    sinks: int = 0


_vp, _ci32, _ci64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
_ARGS = {   # the first pointers are to parameter structs
    "cg_page_plan": [_vp, _ci32] + [_vp] * 11,
    "cg_page_plan_stack": [_vp, _ci32, _vp, _vp, _vp, _ci32] + [_vp] * 8,
    "cg_page_release": [_vp] + [_vp] * 8,
    "cg_rotary_table": [_ci32, _vp, _vp, ctypes.POINTER(ctypes.c_float)],
    "cg_rotary": [_vp, _ci32, _ci32, _ci32, _ci32, _vp, _ci64, _ci64, _vp, _vp, _vp, _ci64, _ci64, _vp],
    "cg_rotary_append": [_vp, _vp, _ci32, _ci32, _vp] + [_vp] * 9,
    "cg_paged_attention_workspace_bytes": [_vp, _vp, ctypes.POINTER(ctypes.c_size_t)],
    "cg_paged_attention": [_vp, _vp] + [_vp] * 8 + [ctypes.c_size_t, _vp],
}
_fns = {}
_ws_bytes = {}


def _fn(name: str):
    f = _fns.get(name)
    if f is None:
        f = getattr(load(), name)
        f.restype = ctypes.c_int
        f.argtypes = _ARGS[name]
        _fns[name] = f
    return f


def _bad(msg: str):
    raise CodecGaugeError(-1, msg)


_INT32, _INT64, _FLOAT32 = torch.int32, torch.int64, torch.float32
_ELEM = {torch.bfloat16: CG_BF16, torch.float16: CG_FP16}


def _elem(t) -> int:
    e = _ELEM.get(t.dtype)
    if e is None:
        _bad(f"expected a bfloat16 or float16 tensor, got {t.dtype}")
    return e


# The current stream's handle without a Stream object around it, where torch has that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _device() -> int:
    """The current device, on which a call launches; -2, where no tensor is, without a GPU."""
    try:
        return _get_device()
    except RuntimeError:
        return -2


def _stream(stream) -> int:
    if stream is not None:
        if getattr(stream, "device_index", _device()) != _device():
            _bad(f"stream: on device {stream.device_index}, the current one is {_device()}")
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(_get_device())
    return torch.cuda.current_stream().cuda_stream


# In the checks, dev is the device that the call launches on.
def _i32(name: str, t, n: int, dev: int) -> int:
    """Address of a contiguous array of at least n 32-bit integers on the device."""
    if t.dtype is not _INT32 or t.get_device() != dev or t.numel() < n or not t.is_contiguous():
        _bad(f"{name}: expected a contiguous int32 device tensor of at least {n} elements, on device {dev}")
    return t.data_ptr()


def _i64(name: str, t, n: int, dev: int) -> int:
    if t.dtype is not _INT64 or t.get_device() != dev or t.numel() < n or not t.is_contiguous():
        _bad(f"{name}: expected a contiguous int64 device tensor of at least {n} elements, on device {dev}")
    return t.data_ptr()


def _heads(name: str, t, n_tok: int, heads: int, d: int, dtype, dev: int):
    """Checks a [n_tok][heads][d] tensor on the device; returns its address and its two strides."""
    if t.shape != (n_tok, heads, d):
        _bad(f"{name}: expected shape [{n_tok}, {heads}, {d}], got {list(t.shape)}")
    if t.dtype is not dtype or t.get_device() != dev:
        _bad(f"{name}: expected a {dtype} tensor on device {dev}")
    tok, head, one = t.stride()
    if one != 1:
        _bad(f"{name}: the last dimension must be contiguous")
    # the stride of a dimension of one element is never used
    return t.data_ptr(), (tok if n_tok > 1 else 0), (head if heads > 1 else 0)


def _pool(pages: Pages, pool, dev: int) -> int:
    if pool.shape != (2, pages.n_pages, pages.H, pages.page, pages.d) or not pool.is_contiguous() or pool.get_device() != dev:
        _bad(f"pool: expected a contiguous tensor [2, {pages.n_pages}, {pages.H}, {pages.page}, {pages.d}] on device {dev}, "
             f"got {list(pool.shape)}")
    return pool.data_ptr()


def page_plan(pages: Pages, ctx_lens, new_lens, free_pages, free_count, block_table, seq_lens, cu_new, positions, slots,
              free_left, stream=None) -> None:
    """Pages for the new tokens of every request, and positions and slots of all new tokens
    (cg_page_plan_stack). The number of tokens planned for is positions.numel(), the stack's size
    free_pages.numel(), which may be less than n_pages, and 0."""
    n, r, dev = positions.numel(), pages.n_req, _device()
    _check(_fn("cg_page_plan_stack")(
        pages.c(), n, _i32("ctx_lens", ctx_lens, r, dev), _i32("new_lens", new_lens, r, dev),
        _i32("free_pages", free_pages, 0, dev), free_pages.numel(), _i32("free_count", free_count, 1, dev),
        _i32("block_table", block_table, r * pages.max_pages, dev), _i32("seq_lens", seq_lens, r, dev),
        _i32("cu_new", cu_new, r + 1, dev), _i32("positions", positions, n, dev), _i64("slots", slots, n, dev),
        _i32("free_left", free_left, 1, dev), _stream(stream)))


def page_release(pages: Pages, lens, done, block_table, free_pages, free_count, lens_left, free_left, stream=None) -> None:
    """Give back the pages of the requests whose done flag (int32) is set (cg_page_release)."""
    r, dev = pages.n_req, _device()
    _check(_fn("cg_page_release")(
        pages.c(), _i32("lens", lens, r, dev), _i32("done", done, r, dev), _i32("block_table", block_table, r * pages.max_pages, dev),
        _i32("free_pages", free_pages, pages.n_pages, dev), _i32("free_count", free_count, 1, dev),
        _i32("lens_left", lens_left, r, dev), _i32("free_left", free_left, 1, dev), _stream(stream)))


def rotary_table(rot: int, scaling: RopeScaling = RopeScaling(), device="cuda"):
    """Frequencies of rot / 2 pairs as a device tensor (int64, 2^-64 of a turn per position), and mscale."""
    host = torch.empty(max(rot // 2, 0), dtype=torch.int64)
    m = ctypes.c_float()
    c = _CScaling(scaling.kind, scaling.base, scaling.factor, scaling.original, scaling.low, scaling.high)
    _check(_fn("cg_rotary_table")(rot, c, host.data_ptr(), m))
    return host.to(device), m.value


def rotary(turn: Rotary, x, positions, table, out, stream=None) -> None:
    """out = rotary(x), [n_tok][heads][d] (cg_rotary); out may be x."""
    if x.dim() != 3:
        _bad("x: expected [n_tok, heads, d]")
    (n, heads, d), dev = x.shape, _device()
    xp, xt, xh = _heads("x", x, n, heads, d, x.dtype, dev)
    op, ot, oh = _heads("out", out, n, heads, d, x.dtype, dev)
    _check(_fn("cg_rotary")(turn.c(), _elem(x), n, heads, d, xp, xt, xh, _i32("positions", positions, n, dev),
                            _i64("table", table, turn.rot // 2, dev) if turn.rot else None, op, ot, oh, _stream(stream)))


def rotary_append(pages: Pages, turn: Rotary, q, k, v, positions, slots, table, q_out, pool, stream=None) -> None:
    """q_out = rotary(q); rotary(k) and v into the pool at their slots (cg_rotary_append). q and
    q_out may be None, or the same tensor."""
    n, dev = k.shape[0], _device()
    hq = 0 if q is None else q.shape[1]
    if k.dtype is not pool.dtype:
        _bad(f"k: expected the pool's type {pool.dtype}, got {k.dtype}")
    kp, kt, kh = _heads("k", k, n, pages.H, pages.d, pool.dtype, dev)
    vp, vt, vh = _heads("v", v, n, pages.H, pages.d, pool.dtype, dev)
    qp, qt, qh = _heads("q", q, n, hq, pages.d, pool.dtype, dev) if hq else (None, 0, 0)
    op, ot, oh = _heads("q_out", q_out, n, hq, pages.d, pool.dtype, dev) if hq else (None, 0, 0)
    _check(_fn("cg_rotary_append")(
        pages.c(_elem(pool)), turn.c(), n, hq, _CStrides(qt, qh, kt, kh, vt, vh, ot, oh), qp, kp, vp,
        _i32("positions", positions, n, dev), _i64("slots", slots, n, dev),
        _i64("table", table, turn.rot // 2, dev) if turn.rot else None, op, _pool(pages, pool, dev), _stream(stream)))


def _attn(pages: Pages, how: PagedAttention, n: int, qt=0, qh=0, ot=0, oh=0) -> bytes:
    return _CPagedAttn(n, how.n_rep, how.max_new, how.window, how.sinks, how.scale, qt, qh, ot, oh)


def paged_attention_workspace_bytes(pages: Pages, how: PagedAttention, n_tok: int) -> int:
    """Workspace bytes of paged_attention for n_tok query rows."""
    v = ctypes.c_size_t()
    _check(_fn("cg_paged_attention_workspace_bytes")(pages.c(), _attn(pages, how, n_tok), v))
    return v.value


class _Kept(threading.local):
    """Workspaces (by device) of one host thread's calls on the default stream. The calls of one thread
    follow one another there; those of two threads may mix their launches, of which a call has up to
    three, so that each thread needs its own."""

    def __init__(self):
        self.by_device = {}


_kept = _Kept()


def _workspace(pages: Pages, how: PagedAttention, n: int, device):
    key = (pages.d, how.n_rep, how.max_new, device)   # all that the size depends on
    nbytes = _ws_bytes.get(key)
    if nbytes is None:
        nbytes = _ws_bytes[key] = paged_attention_workspace_bytes(pages, how, n)
    if _stream(None) != 0:      # other streams end; the default one does not, and is never captured
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    mine = _kept.by_device
    kept = mine.get(device)
    if kept is None or kept.nbytes < nbytes:
        kept = mine[device] = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return kept


def paged_attention(pages: Pages, how: PagedAttention, q, pool, block_table, seq_lens, cu_new, out, lse=None,
                    workspace=None, stream=None) -> None:
    """Attention of the new tokens' queries q [n_tok][H * n_rep][d] over their requests' pages
    (cg_paged_attention). Without a workspace the call takes one from torch's allocator, on the
    current stream (pass one to run on another); the default stream's is kept for the next call of the
    same host thread, until the thread ends. A workspace that is passed serves calls made one after the
    other: two threads must not pass the same one at the same time."""
    n, hq, dev = q.shape[0], pages.H * how.n_rep, _device()
    qp, qt, qh = _heads("q", q, n, hq, pages.d, pool.dtype, dev)
    op, ot, oh = _heads("out", out, n, hq, pages.d, pool.dtype, dev)
    lp = None
    if lse is not None:
        if lse.dtype is not _FLOAT32 or lse.get_device() != dev or not lse.is_contiguous() or lse.numel() < n * hq:
            _bad(f"lse: expected a contiguous float32 tensor [{n}, {hq}] on device {dev}")
        lp = lse.data_ptr()
    cp, ca = pages.c(_elem(pool)), _attn(pages, how, n, qt, qh, ot, oh)
    if workspace is None:
        if stream is not None and stream != torch.cuda.current_stream():
            _bad("workspace: needed on a stream that is not the current one")
        workspace = _workspace(pages, how, n, q.device)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        _bad(f"workspace: expected a contiguous tensor on device {dev}")
    r = pages.n_req
    _check(_fn("cg_paged_attention")(
        cp, ca, qp, _pool(pages, pool, dev), _i32("block_table", block_table, r * pages.max_pages, dev),
        _i32("seq_lens", seq_lens, r, dev), _i32("cu_new", cu_new, r + 1, dev), op, lp, workspace.data_ptr(),
        workspace.nbytes, _stream(stream)))
