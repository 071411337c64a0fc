"""Binding of the paged KV cache (include/presto.h): the attention that reads
it, the append that fills it and the bookkeeping of its pages.

As in ``_lib``: argument marshalling and checks only.  The calls run on the
device of their tensors, on that device's current stream unless one is given.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from ._lib import PRESTO_DT_BF16, PRESTO_DT_F32, PRESTO_DT_FP4, PagedAttnDesc, PagesDesc, _check, _ptr, lib


_I32 = torch.int32
_DT = {torch.bfloat16: PRESTO_DT_BF16, torch.float32: PRESTO_DT_F32}


# (A decode step of a small batch is bound by the host: every check of the two
# functions costs 0.1 us, and the calls look at their usual tensors in one
# expression before they come here to say which one is wrong.)
def _same(dev: int, names: str, *ts) -> None:
    """Tensors on GPU `dev` (None: left out)."""
    for i, t in enumerate(ts):
        if t is not None and (t.get_device() != dev or dev < 0):
            raise ValueError(f"{names.split()[i]} must be a tensor on the GPU of the others")


def _book(dev: int, names: str, *ts) -> None:
    """int32 bookkeeping tensors, contiguous, on GPU `dev`."""
    for i, t in enumerate(ts):
        if t is not None and (t.dtype is not _I32 or t.get_device() != dev or dev < 0 or not t.is_contiguous()):
            raise ValueError(f"{names.split()[i]} must be a contiguous int32 tensor on the GPU of the others")


def _vector(name, t, n):
    if t is not None and t.shape != (n,):
        raise ValueError(f"{name} must be of shape [{n}], not {list(t.shape)}")


def _int32(bits: int) -> None:
    """Numbers, or-ed together, that the C interface holds in 32 bits: ctypes
    would cut them to their low half without a word.  (One outside of them
    shows unless a negative one stands beside it, which the library refuses.)"""
    if not -1 <= bits >> 31 <= 0:
        raise ValueError("a size, length or window does not fit 32 bits")


def _one_by_one(*numbers: int) -> None:
    for x in numbers:
        _int32(x)


_current = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream


def _empty(stream, shape, dtype, device, returned: bool = True) -> torch.Tensor:
    """A tensor for a call on `stream`.  The allocator orders a block's uses
    within one stream: taken on the current stream for a call on another, it may
    be one that kernels of the current stream, freed but not through, still
    write.  So it is taken on the call's own, and what the caller gets is noted
    for the current stream, where it is used next."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if returned:
        t.record_stream(torch.cuda.current_stream(device))
    return t


def _launch(call, who: str, dev: int, stream, *args) -> None:
    """Enqueues call(*args, stream) on GPU `dev`."""
    if stream is None:
        queue = _raw_stream(dev)
    else:
        if stream.device.index != dev:
            raise ValueError(f"the stream belongs to {stream.device}, the tensors to GPU {dev}")
        queue = stream.cuda_stream
    if dev == _current():
        status = call(*args, queue)
    else:
        with torch.cuda.device(dev):
            status = call(*args, queue)
    if status:
        _check(status, who)


def _pool(k, v, cols, batch, layers: bool) -> PagesDesc:
    """Descriptor of the pools k, v: [pages, page, hkv, dim], or with a leading
    layer dimension where `layers` allows it."""
    shape, stride = k.shape, k.stride()
    if v.shape != shape or v.stride() != stride or v.dtype is not k.dtype:
        raise ValueError("k_pages and v_pages must have one shape, stride and type")
    return _pool_of(shape, stride, k.dtype, batch, cols, layers)


@functools.lru_cache(maxsize=64)
def _pool_of(shape, stride, dtype, batch, cols, layers) -> PagesDesc:
    """The same from sizes alone (a program has few pools; not to be changed).
    Pools of bytes are 4-bit caches [pages, hkv, page / 16, 17 dim / 2]."""
    _one_by_one(*shape, batch, cols)
    if dtype not in _DT and dtype is not torch.uint8:
        raise TypeError(f"unsupported dtype {dtype}")
    n_layers, layer_stride = 1, 0
    if len(shape) == 5 and layers:
        n_layers, layer_stride, shape, stride = shape[0], stride[0], shape[1:], stride[1:]
    elif len(shape) != 4:
        raise ValueError("the page pools must be [pages, page, hkv, dim]" + (" or with layers first" if layers else ""))
    n, n2, n3, n4 = shape
    s_page, s_2, s_3, s_4 = stride
    if (s_4 != 1 or s_3 != n4 or s_2 != n3 * n4) and 0 not in shape:
        raise ValueError("a page must be contiguous")
    if dtype is torch.uint8:
        hkv, page, d, dt = n2, 16 * n3, n4 * 2 // 17, PRESTO_DT_FP4
        if d * 17 != n4 * 2:
            raise ValueError("the last dimension of a 4-bit pool must be 17 dim / 2 bytes")
        page_units = n2 * n3 * n4
    else:
        page, hkv, d, dt = n2, n3, n4, _DT[dtype]
        page_units = page * hkv * d
    # (the stride of a single page or layer is free: the default, 0)
    if n <= 1:
        s_page = 0
    elif s_page < page_units:
        raise ValueError("pages must not overlap")
    if n_layers == 1:
        layer_stride = 0
    elif layer_stride < (n - 1) * s_page + page_units and (
            layer_stride < page_units or s_page < (n_layers - 1) * layer_stride + page_units):
        raise ValueError("layers must not overlap")  # (they may lie one behind the other or page by page)
    return PagesDesc(batch, cols, n, page, hkv, d, dt, n_layers, s_page, layer_stride)


def _books(refs, page_table, page_size) -> PagesDesc:
    """Descriptor for the calls that look at the books only."""
    batch, cols = page_table.shape
    return _books_of(batch, cols, refs.shape[0], page_size)


@functools.lru_cache(maxsize=64)
def _books_of(batch, cols, pages, page_size) -> PagesDesc:
    _one_by_one(batch, cols, pages, page_size)
    return PagesDesc(batch, cols, pages, page_size, 1, 64, 0, 1, 0, 0)


def _rows(name, t, heads, d):
    """Token rows [n, heads, dim], any stride between tokens; the stride."""
    return _rows_of(name, t.shape, t.stride(), heads, d)


def _rows_of(name, shape, stride, heads, d):
    if len(shape) != 3 or shape[1] != heads or shape[2] != d:
        raise ValueError(f"{name} must be [tokens, {heads}, {d}]")
    if (stride[2] != 1 or (stride[1] != d and heads > 1)) and 0 not in shape:
        raise ValueError(f"the heads of a token of {name} must be contiguous")
    if shape[0] <= 1:
        return 0
    if stride[0] < heads * d:  # (0 would mean the default)
        raise ValueError(f"the tokens of {name} must not overlap")
    return stride[0]


def _attn_desc(q, k_pages, v_pages, page_table, batch, max_q, max_ctx, scale, window, sinks, total_ctx):
    table = page_table.shape
    if len(table) != 2 or table[0] != batch:
        raise ValueError("page_table must be [sequences, columns]")
    pages = _pool(k_pages, v_pages, table[1], batch, False)
    if q.dtype is not k_pages.dtype:
        raise TypeError("q and the pages must be of one type")
    d = pages.head_dim
    n, hq = q.shape[:2]
    stride = _rows("q", q, hq, d)
    if max_ctx is None:
        max_ctx = pages.max_pages * pages.page_size
    _int32(max_q | max_ctx | window | sinks)
    return PagedAttnDesc(pages, hq, max_q, max_ctx, window, sinks, d ** -0.5 if scale is None else scale, n, stride,
                         total_ctx)


def _room(workspace, dev: int) -> int:
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the GPU of the others")
    return workspace.nbytes


def _attend(who, call, need_of, q, q_offsets, k_pages, v_pages, page_table, ctx, desc, out, flags, workspace, stream):
    dev = q.get_device()
    if not (0 <= dev == k_pages.get_device() == v_pages.get_device() == page_table.get_device() == ctx.get_device()
            and page_table.dtype is _I32 is ctx.dtype and page_table.is_contiguous() and ctx.is_contiguous()):
        _same(dev, "q k_pages v_pages", q, k_pages, v_pages)
        _book(dev, "page_table ctx", page_table, ctx)
    if q_offsets is not None or flags is not None:
        _book(dev, "q_offsets flags", q_offsets, flags)
    ref, ws, nb = ctypes.byref(desc), workspace, 0
    if out is None:
        out = _empty(stream, q.shape, q.dtype, q.device)
    elif out.shape != q.shape or out.dtype is not q.dtype or not out.is_contiguous() or out.get_device() != dev:
        raise ValueError("out must be a contiguous tensor of q's shape and type on its GPU")
    if ws is None:
        nb = need_of(ref)
        if nb:
            ws = _empty(stream, nb, torch.uint8, q.device, returned=False)
    else:
        nb = _room(ws, dev)
    head = (ref, q.data_ptr()) if q_offsets is None else (ref, q.data_ptr(), q_offsets.data_ptr())
    _launch(call, who, dev, stream, *head, k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(),
            ctx.data_ptr(), out.data_ptr(), _ptr(flags), _ptr(ws), nb)
    return out


def presto_paged_attention(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                           page_table: torch.Tensor, ctx: torch.Tensor, *, max_ctx: int | None = None,
                           scale: float | None = None, window: int = 0, sinks: int = 0, total_ctx: int = 0,
                           out=None, flags=None, workspace=None, stream=None) -> torch.Tensor:
    """One new token per sequence: q [b, Hq, d] at position ctx[b] - 1 over the
    cached positions it sees (all up to its own, or with a window the last
    `window` of them and the first `sinks`)."""
    b = q.shape[0]
    desc = _attn_desc(q, k_pages, v_pages, page_table, b, 1, max_ctx, scale, window, sinks, total_ctx)
    _vector("ctx", ctx, b)
    L = lib()
    return _attend("presto_paged_attention", L.presto_paged_attention, L.presto_paged_attention_workspace, q, None,
                   k_pages, v_pages, page_table, ctx, desc, out, flags, workspace, stream)


def presto_window_attention(q: torch.Tensor, q_offsets: torch.Tensor, max_q: int, k_pages: torch.Tensor,
                            v_pages: torch.Tensor, page_table: torch.Tensor, ctx: torch.Tensor, *,
                            max_ctx: int | None = None, scale: float | None = None, window: int = 0,
                            sinks: int = 0, total_ctx: int = 0, out=None, flags=None, workspace=None,
                            stream=None) -> torch.Tensor:
    """A ragged batch of new tokens: rows q_offsets[b] .. q_offsets[b+1] - 1 of
    q [total, Hq, d] are the last positions of sequence b, at most max_q."""
    b = q_offsets.shape[0] - 1
    desc = _attn_desc(q, k_pages, v_pages, page_table, b, max_q, max_ctx, scale, window, sinks, total_ctx)
    _vector("q_offsets", q_offsets, b + 1)
    _vector("ctx", ctx, b)
    L = lib()
    return _attend("presto_window_attention", L.presto_window_attention, L.presto_window_attention_workspace, q,
                   q_offsets, k_pages, v_pages, page_table, ctx, desc, out, flags, workspace, stream)


def paged_attention_workspace(q: torch.Tensor, k_pages: torch.Tensor, page_table: torch.Tensor, *, max_q: int = 1,
                              max_ctx: int | None = None, window: int = 0, sinks: int = 0,
                              total_ctx: int = 0) -> torch.Tensor:
    """A workspace for calls with just these sizes and hints:
    presto_window_attention with these queries and max_q, and
    presto_paged_attention on this batch.  A call with fewer queries, a smaller
    max_q or max_ctx or another total_ctx may be split further and need more
    (too small a workspace is refused before anything runs): a program asks once
    per shape that it uses, or passes none."""
    desc = _attn_desc(q, k_pages, k_pages, page_table, page_table.shape[0], max_q, max_ctx, None, window, sinks,
                      total_ctx)
    need = max(lib().presto_window_attention_workspace(ctypes.byref(desc)),
               lib().presto_paged_attention_workspace(ctypes.byref(desc)), 16)
    return torch.empty(need, dtype=torch.uint8, device=q.device)


def _pages_call(who, refs, dev, desc, args, flags, workspace, stream):
    """args: the call's pointers up to flags."""
    L, ref, ws = lib(), ctypes.byref(desc), workspace
    if ws is None:
        ws = _empty(stream, max(L.presto_pages_workspace(ref), 16), torch.uint8, refs.device, returned=False)
    _launch(getattr(L, who), who, dev, stream, ref, *args, _ptr(flags), ws.data_ptr(), _room(ws, dev))


def pages_workspace(refs: torch.Tensor, page_table: torch.Tensor) -> torch.Tensor:
    """A workspace for every presto_pages_* call on these books."""
    need = lib().presto_pages_workspace(ctypes.byref(_books(refs, page_table, 16)))
    return torch.empty(max(need, 16), dtype=torch.uint8, device=refs.device)


def _check_books(refs, page_table, ctx, names: str = "", *more):
    if page_table.dim() != 2 or refs.dim() != 1:
        raise ValueError("page_table must be [sequences, columns] and refs [pages]")
    dev = refs.get_device()
    _book(dev, "refs page_table ctx " + names, refs, page_table, ctx, *more)
    if ctx is not None:
        _vector("ctx", ctx, page_table.shape[0])
    return dev


def presto_pages_reserve(refs: torch.Tensor, page_table: torch.Tensor, ctx: torch.Tensor, page_size: int,
                         add: torch.Tensor | None = None, extra: int = 0, *, out=None, flags=None, workspace=None,
                         stream=None) -> torch.Tensor:
    """Gives pages to the positions ctx .. ctx + add + extra - 1 and returns the
    new lengths (in `out`, which may be ctx); refs and page_table are updated
    in place.  A sequence the pool has no pages for keeps its length."""
    _one_by_one(page_size, extra)
    dev = _check_books(refs, page_table, ctx, "add out flags", add, out, flags)
    b = page_table.shape[0]
    _vector("add", add, b)
    _vector("out", out, b)
    if out is None:
        out = _empty(stream, ctx.shape, _I32, ctx.device)
    _pages_call("presto_pages_reserve", refs, dev, _books(refs, page_table, page_size),
                (refs.data_ptr(), page_table.data_ptr(), ctx.data_ptr(), _ptr(add), extra, out.data_ptr()), flags,
                workspace, stream)
    return out


def presto_append_kv(k_new: torch.Tensor, v_new: torch.Tensor, offsets: torch.Tensor, max_new: int,
                     k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, ctx: torch.Tensor,
                     ctx_new: torch.Tensor, *, flags=None, stream=None) -> None:
    """Writes rows offsets[b] + i of k_new, v_new [rows, Hkv, d] to positions
    ctx[b] + i < ctx_new[b] of the cache, at most max_new per sequence."""
    _int32(max_new)
    dev = k_new.get_device()
    b = offsets.shape[0] - 1
    if not (0 <= dev == v_new.get_device() == k_pages.get_device() == v_pages.get_device()):
        _same(dev, "k_new v_new k_pages v_pages", k_new, v_new, k_pages, v_pages)
    _book(dev, "offsets page_table ctx ctx_new flags", offsets, page_table, ctx, ctx_new, flags)
    _vector("offsets", offsets, b + 1)
    table = page_table.shape
    if len(table) != 2 or table[0] != b:
        raise ValueError("page_table must be [sequences, columns]")
    _vector("ctx", ctx, b)
    _vector("ctx_new", ctx_new, b)
    desc = _pool(k_pages, v_pages, table[1], b, False)
    if k_new.dtype is not k_pages.dtype or v_new.dtype is not k_pages.dtype:
        raise TypeError("the new rows and the pages must be of one type")
    hkv, d = k_pages.shape[2:]
    stride = _rows("k_new", k_new, hkv, d)
    if v_new.shape != k_new.shape or _rows("v_new", v_new, hkv, d) != stride:
        raise ValueError("k_new and v_new must have one shape and stride")
    _launch(lib().presto_append_kv, "presto_append_kv", dev, stream, ctypes.byref(desc), k_new.data_ptr(),
            v_new.data_ptr(), k_new.shape[0], stride, offsets.data_ptr(), max_new, k_pages.data_ptr(),
            v_pages.data_ptr(), page_table.data_ptr(), ctx.data_ptr(), ctx_new.data_ptr(), _ptr(flags))


def presto_pages_fork(refs: torch.Tensor, page_table: torch.Tensor, ctx: torch.Tensor, parent: torch.Tensor,
                      child: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, *, flags=None,
                      workspace=None, stream=None) -> None:
    """Sequence child[i] (empty) becomes a copy of parent[i]: full pages shared,
    the rows of the last one copied in all layers of k_pages, v_pages
    [layers, pages, page, Hkv, d] (or of one layer, without that dimension)."""
    dev = _check_books(refs, page_table, ctx, "parent child flags", parent, child, flags)
    _same(dev, "k_pages v_pages", k_pages, v_pages)
    n = parent.numel()
    _vector("parent", parent, n)
    _vector("child", child, n)
    desc = _pool(k_pages, v_pages, page_table.shape[1], page_table.shape[0], True)
    _vector("refs", refs, desc.num_pages)
    _pages_call("presto_pages_fork", refs, dev, desc,
                (_ptr(refs), _ptr(page_table), _ptr(ctx), _ptr(parent), _ptr(child), n, _ptr(k_pages),
                 _ptr(v_pages)), flags, workspace, stream)


def presto_pages_free(refs: torch.Tensor, page_table: torch.Tensor, ctx: torch.Tensor, rows: torch.Tensor, *,
                      flags=None, stream=None) -> None:
    """Drops the sequences `rows`: their references go, their lengths are 0."""
    dev = _check_books(refs, page_table, ctx, "rows flags", rows, flags)
    n = rows.numel()
    _vector("rows", rows, n)
    _launch(lib().presto_pages_free, "presto_pages_free", dev, stream, ctypes.byref(_books(refs, page_table, 16)),
            refs.data_ptr(), page_table.data_ptr(), ctx.data_ptr(), rows.data_ptr(), n, _ptr(flags))


def presto_pages_trim(refs: torch.Tensor, page_table: torch.Tensor, ctx: torch.Tensor, page_size: int, window: int,
                      sinks: int = 0, *, flags=None, stream=None) -> None:
    """Drops the pages that no query from position ctx - 1 on sees under the
    window and sinks."""
    _one_by_one(page_size, window, sinks)
    dev = _check_books(refs, page_table, ctx, "flags", flags)
    _launch(lib().presto_pages_trim, "presto_pages_trim", dev, stream,
            ctypes.byref(_books(refs, page_table, page_size)), refs.data_ptr(), page_table.data_ptr(), ctx.data_ptr(),
            window, sinks, _ptr(flags))


def presto_pages_compact(refs: torch.Tensor, page_table: torch.Tensor, k_pages: torch.Tensor,
                         v_pages: torch.Tensor, *, out=None, flags=None, workspace=None, stream=None) -> dict:
    """Moves the live pages to the front of the pool, in all layers.  Returns
    the books afterwards: refs, page_table, n_live [1] (or fills those of
    `out`, where refs and page_table may be the arguments themselves, and
    page_map [pages], each live page's new number, if it is there)."""
    dev = _check_books(refs, page_table, None, "flags", flags)
    _same(dev, "k_pages v_pages", k_pages, v_pages)
    if out is None:
        out = {name: _empty(stream, shape, _I32, refs.device)
               for name, shape in (("refs", refs.shape), ("page_table", page_table.shape), ("n_live", 1))}
    page_map = out.get("page_map")
    _book(dev, "out_refs out_page_table n_live page_map", out["refs"], out["page_table"], out["n_live"], page_map)
    desc = _pool(k_pages, v_pages, page_table.shape[1], page_table.shape[0], True)
    _vector("refs", refs, desc.num_pages)
    _vector("out refs", out["refs"], desc.num_pages)
    if out["page_table"].shape != page_table.shape:
        raise ValueError("out page_table must be of page_table's shape")
    _vector("n_live", out["n_live"], 1)
    _vector("page_map", page_map, desc.num_pages)
    _pages_call("presto_pages_compact", refs, dev, desc,
                (_ptr(refs), _ptr(out["refs"]), _ptr(page_table), _ptr(out["page_table"]), _ptr(out["n_live"]),
                 _ptr(page_map), _ptr(k_pages), _ptr(v_pages)), flags, workspace, stream)
    return out
