"""Binding of the operators around a decoding step (include/presto.h): rotary
positions, the append that rotates on the way, the 4-bit cache and its
attention, and the draw of a token.

As in ``_paged``: argument marshalling and checks only.  The calls run on the
device of their tensors, on that device's current stream unless one is given.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from ._lib import (PRESTO_ROPE_RAMP_LOG, PRESTO_ROPE_RAMP_NONE, PRESTO_ROPE_RAMP_TURNS, AppendDesc, PagedAttnDesc,
                   PagesDesc, RopeDesc, RopeFreqDesc, _check, _ptr, lib)
from ._paged import (_DT, _I32, _book, _empty, _int32, _launch, _one_by_one, _pool, _pool_of, _room, _rows, _rows_of,
                     _same, _vector)

_RAMPS = {None: PRESTO_ROPE_RAMP_NONE, "turns": PRESTO_ROPE_RAMP_TURNS, "log": PRESTO_ROPE_RAMP_LOG}


def _type(t) -> int:
    dt = _DT.get(t.dtype)
    if dt is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return dt


# ---------------------------------------------------------------------------
# rotary positions

def presto_rope_steps(rot_dim: int, *, base: float = 10000.0, factor: float = 1.0, original: float = 0.0,
                      low: float = 0.0, high: float = 0.0, ramp: str | None = None, frequencies=None) -> torch.Tensor:
    """The angles of one position as 64-bit fractions of a turn: int64
    [rot_dim / 2] on the host (the bits of unsigned words)."""
    _one_by_one(rot_dim)
    if ramp not in _RAMPS:
        raise ValueError(f"ramp must be one of {list(_RAMPS)}")
    out = torch.empty(max(rot_dim // 2, 1), dtype=torch.int64)
    desc = RopeFreqDesc(rot_dim, _RAMPS[ramp], base, factor, original, low, high)
    freq = None
    if frequencies is not None:
        freq = torch.as_tensor(frequencies, dtype=torch.float64).cpu().contiguous()
        _vector("frequencies", freq, rot_dim // 2)
    _check(lib().presto_rope_steps(ctypes.byref(desc), _ptr(freq), out.data_ptr()), "presto_rope_steps")
    return out


class RopePlan:
    """A rotation: its table of angles on one device, and what the calls need
    beside it.  A program makes one per model and device."""

    __slots__ = ("desc", "steps", "ref", "device_index", "address")

    def __init__(self, rot_dim: int, interleaved: bool, magnitude: float, steps: torch.Tensor):
        self.desc = RopeDesc(rot_dim, int(bool(interleaved)), magnitude)
        self.ref = ctypes.byref(self.desc)
        self.steps, self.device_index, self.address = steps, steps.get_device(), steps.data_ptr()


def rope_plan(rot_dim: int, *, base: float = 10000.0, interleaved: bool = False, factor: float = 1.0,
              original: float = 0.0, low: float = 0.0, high: float = 0.0, ramp: str | None = None,
              magnitude: float = 1.0, frequencies=None, device="cuda") -> RopePlan:
    """Rotation of the first rot_dim values of a head, pairs (i, i + rot_dim / 2)
    or, interleaved, (2 i, 2 i + 1), by base^(-2 i / rot_dim) per position.
    Long contexts: all frequencies divided by `factor`, or with ramp "turns" or
    "log" those of pairs that turn less than `low` times over `original`
    positions, and partly those up to `high` times.  `frequencies`: given one by
    one instead."""
    steps = presto_rope_steps(rot_dim, base=base, factor=factor, original=original, low=low, high=high, ramp=ramp,
                              frequencies=frequencies)
    return RopePlan(rot_dim, interleaved, magnitude, steps.to(device))


def _plan_on(plan: RopePlan, dev: int) -> None:
    if plan.device_index != dev:
        raise ValueError("the plan must be on the GPU of the tensors")


# (Calls on few rows are bound by the host: what follows from sizes alone is
# looked up, and the usual tensors are looked at in one expression before they
# are gone through to say which one is wrong.)
@functools.lru_cache(maxsize=64)
def _rope_of(shape, stride, out_shape, out_stride):
    if len(shape) != 3:
        raise ValueError("x must be [rows, heads, dim]")
    n, heads, d = shape
    _one_by_one(heads, d)
    from_ = _rows_of("x", shape, stride, heads, d)
    if out_shape != shape:
        raise ValueError("out must be a tensor of x's shape and type on its GPU")
    return n, heads, d, from_, _rows_of("out", out_shape, out_stride, heads, d)


def presto_rope(x: torch.Tensor, positions: torch.Tensor, plan: RopePlan, *, out=None, stream=None) -> torch.Tensor:
    """x [rows, heads, dim] rotated by positions [rows] (int32): in `out`, which
    may be x itself, or a new tensor."""
    dt, dev = _type(x), x.get_device()
    if out is None:
        out = _empty(stream, x.shape, x.dtype, x.device)
    n, heads, d, stride, to = _rope_of(x.shape, x.stride(), out.shape, out.stride())
    if not (0 <= dev == positions.get_device() == out.get_device() == plan.device_index and out.dtype is x.dtype
            and positions.dtype is _I32 and positions.is_contiguous() and positions.shape == (n,)):
        _book(dev, "positions", positions)
        _vector("positions", positions, n)
        _plan_on(plan, dev)
        raise ValueError("out must be a tensor of x's shape and type on its GPU")
    _launch(lib().presto_rope, "presto_rope", dev, stream, plan.ref, plan.address, dt, x.data_ptr(), stride, n, heads,
            d, positions.data_ptr(), out.data_ptr(), to)
    return out


# ---------------------------------------------------------------------------
# the cache

def quant_pages(pages: int, page_size: int, hkv: int, dim: int, *, layers: int | None = None,
                device="cuda") -> torch.Tensor:
    """A pool of a 4-bit cache (K or V): uint8 [pages, hkv, page_size / 16,
    17 dim / 2], or with layers first.  Its contents are undefined."""
    if page_size % 16:
        raise ValueError("page_size must be a multiple of 16")
    shape = (pages, hkv, page_size // 16, 17 * dim // 2)
    return torch.empty(shape if layers is None else (layers, *shape), dtype=torch.uint8, device=device)


def _cached(k_pages, v_pages, page_table, offsets, ctx, ctx_new, flags, dev) -> PagesDesc:
    """Descriptor of the pools, and the checks of the books beside them."""
    b = offsets.shape[0] - 1
    _book(dev, "offsets page_table ctx ctx_new flags", offsets, page_table, ctx, ctx_new, flags)
    _vector("offsets", offsets, b + 1)
    table = page_table.shape
    if len(table) != 2 or table[0] != b:
        raise ValueError("page_table must be [sequences, columns]")
    _vector("ctx", ctx, b)
    _vector("ctx_new", ctx_new, b)
    return _pool(k_pages, v_pages, table[1], b, False)


@functools.lru_cache(maxsize=64)
def _append_of(shape, k_stride, v_stride, q_shape, q_stride, out_stride, dt, max_new, pool, pool_stride, pool_type,
               cols, batch):
    """Descriptor of presto_append_rope from sizes alone, and a reference to it
    (not to be changed)."""
    _int32(max_new)
    pages = _pool_of(pool, pool_stride, pool_type, batch, cols, False)
    strides = [_rows_of(name, shape, s, pages.hkv, pages.head_dim) for name, s in (("k_new", k_stride),
                                                                                  ("v_new", v_stride))]
    hq, q_strides = 0, (0, 0)
    if q_shape is not None:
        if len(q_shape) != 3 or q_shape[0] != shape[0]:
            raise ValueError("q must be [tokens, heads, dim] of k_new's type on its GPU")
        hq = q_shape[1]
        q_strides = [_rows_of(name, q_shape, s, hq, pages.head_dim) for name, s in (("q", q_stride),
                                                                                   ("out", out_stride))]
    desc = AppendDesc(pages, dt, hq, max_new, shape[0], *q_strides, *strides)
    return desc, ctypes.byref(desc)


def presto_append_rope(plan: RopePlan | None, q: torch.Tensor | None, k_new: torch.Tensor, v_new: torch.Tensor,
                       offsets: torch.Tensor, max_new: int, k_pages: torch.Tensor, v_pages: torch.Tensor,
                       page_table: torch.Tensor, ctx: torch.Tensor, ctx_new: torch.Tensor, *, out=None, flags=None,
                       stream=None):
    """presto_append_kv with the new keys rotated by their positions (plan None:
    as they are), into a cache of the rows' type or of 4 bits; with q [rows, Hq,
    d] given, its rows rotated alike into `out` (may be q), which is returned."""
    dev, dtype, dt, table, pool, pool_stride = (k_new.get_device(), k_new.dtype, _type(k_new), page_table.shape,
                                                k_pages.shape, k_pages.stride())
    b = offsets.shape[0] - 1
    if not (0 <= dev == v_new.get_device() == k_pages.get_device() == v_pages.get_device() == offsets.get_device()
            == page_table.get_device() == ctx.get_device() == ctx_new.get_device()
            and offsets.dtype is _I32 is page_table.dtype and ctx.dtype is _I32 is ctx_new.dtype
            and offsets.is_contiguous() and page_table.is_contiguous() and ctx.is_contiguous()
            and ctx_new.is_contiguous() and len(table) == 2 and table[0] == b and offsets.shape == (b + 1,)
            and ctx.shape == (b,) == ctx_new.shape and v_new.shape == k_new.shape and v_new.dtype is dtype
            and k_pages.dtype in (dtype, torch.uint8)
            and v_pages.shape == pool and v_pages.stride() == pool_stride and v_pages.dtype is k_pages.dtype):
        _same(dev, "k_new v_new k_pages v_pages", k_new, v_new, k_pages, v_pages)
        _cached(k_pages, v_pages, page_table, offsets, ctx, ctx_new, flags, dev)
        if v_new.dtype is not dtype or k_pages.dtype not in (dtype, torch.uint8):
            raise TypeError("the new rows and the pages must be of one type, or the pages of 4 bits")
        raise ValueError("k_new and v_new must have one shape")
    if flags is not None:
        _book(dev, "flags", flags)
    q_shape = q_stride = out_stride = None
    if q is not None:
        q_shape, q_stride = q.shape, q.stride()
        if out is None:
            out = _empty(stream, q_shape, q.dtype, q.device)
        elif out.shape != q_shape or out.dtype is not q.dtype or out.get_device() != q.get_device():
            raise ValueError("out must be a tensor of q's shape and type on its GPU")
        if q.get_device() != dev or q.dtype is not dtype:
            raise ValueError("q must be [tokens, heads, dim] of k_new's type on its GPU")
        out_stride = out.stride()
    elif out is not None:
        raise ValueError("out without q")
    if plan is not None:
        _plan_on(plan, dev)
    _, ref = _append_of(k_new.shape, k_new.stride(), v_new.stride(), q_shape, q_stride, out_stride, dt, max_new, pool,
                        pool_stride, k_pages.dtype, table[1], b)
    _launch(lib().presto_append_rope, "presto_append_rope", dev, stream, ref, None if plan is None else plan.ref,
            None if plan is None else plan.address, _ptr(q), k_new.data_ptr(), v_new.data_ptr(), offsets.data_ptr(),
            _ptr(out), k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), ctx.data_ptr(),
            ctx_new.data_ptr(), _ptr(flags))
    return out


def presto_read_kv(k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, ctx: torch.Tensor,
                   ctx_new: torch.Tensor, offsets: torch.Tensor, max_new: int, *, rows: int | None = None,
                   dtype: torch.dtype | None = None, out=None, flags=None, stream=None):
    """Positions ctx[b] .. ctx_new[b] - 1 of the cache as rows offsets[b] + i of
    (k, v), [rows, Hkv, d]: those of `out`, or new ones of `rows` rows, zeros
    where nothing is read (of the pool's type; of a 4-bit pool bf16 unless
    `dtype` says otherwise)."""
    _int32(max_new)
    dev = k_pages.get_device()
    _same(dev, "k_pages v_pages", k_pages, v_pages)
    pages = _cached(k_pages, v_pages, page_table, offsets, ctx, ctx_new, flags, dev)
    if out is None:
        if rows is None:
            raise ValueError("rows, or out, must be given")
        if dtype is None:
            dtype = torch.bfloat16 if k_pages.dtype is torch.uint8 else k_pages.dtype
        shape = (rows, pages.hkv, pages.head_dim)
        out = tuple(_empty(stream, shape, dtype, k_pages.device) for _ in range(2))
        if stream is None:
            for t in out:
                t.zero_()
        else:
            with torch.cuda.stream(stream):
                for t in out:
                    t.zero_()
    k, v = out
    dt = _type(k)
    if v.dtype is not k.dtype or v.shape != k.shape:
        raise ValueError("the outputs must have one shape and type")
    if k_pages.dtype not in (k.dtype, torch.uint8):
        raise TypeError("the outputs must be of the pages' type, or the pages of 4 bits")
    _same(dev, "k v", k, v)
    k_stride, v_stride = (_rows(name, t, pages.hkv, pages.head_dim) for name, t in (("k", k), ("v", v)))
    desc = AppendDesc(pages, dt, 0, max_new, k.shape[0], 0, 0, k_stride, v_stride)
    _launch(lib().presto_read_kv, "presto_read_kv", dev, stream, ctypes.byref(desc), k_pages.data_ptr(),
            v_pages.data_ptr(), page_table.data_ptr(), ctx.data_ptr(), ctx_new.data_ptr(), offsets.data_ptr(),
            k.data_ptr(), v.data_ptr(), _ptr(flags))
    return out


@functools.lru_cache(maxsize=64)
def _queries_of(shape, stride, pool, pool_stride, pool_type, table, batch):
    """(pages, heads, rows, stride of a row) of an attention, from sizes alone."""
    if len(table) != 2 or table[0] != batch:
        raise ValueError("page_table must be [sequences, columns]")
    if pool_type is not torch.uint8:
        raise TypeError("the pages must be of 4 bits (uint8)")
    pages = _pool_of(pool, pool_stride, pool_type, batch, table[1], False)
    if len(shape) != 3:
        raise ValueError("q must be [tokens, heads, dim]")
    return pages, shape[1], shape[0], _rows_of("q", shape, stride, shape[1], pages.head_dim)


def _quant_desc(q, k_pages, v_pages, page_table, batch, max_q, max_ctx, scale, window, sinks, total_ctx):
    pool, pool_stride = k_pages.shape, k_pages.stride()
    if v_pages.shape != pool or v_pages.stride() != pool_stride or v_pages.dtype is not k_pages.dtype:
        raise ValueError("k_pages and v_pages must have one shape, stride and type")
    pages, hq, n, stride = _queries_of(q.shape, q.stride(), pool, pool_stride, k_pages.dtype, page_table.shape, batch)
    if max_ctx is None:
        max_ctx = pages.max_pages * pages.page_size
    _int32(max_q | max_ctx | window | sinks)
    return PagedAttnDesc(pages, hq, max_q, max_ctx, window, sinks, pages.head_dim ** -0.5 if scale is None else scale,
                         n, stride, total_ctx)


def presto_quant_attention(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor,
                           ctx: torch.Tensor, *, q_offsets: torch.Tensor | None = None, max_q: int = 1,
                           max_ctx: int | None = None, scale: float | None = None, window: int = 0, sinks: int = 0,
                           total_ctx: int = 0, out=None, flags=None, workspace=None, stream=None) -> torch.Tensor:
    """Attention over a 4-bit cache: one new token per sequence, q [b, Hq, d] at
    position ctx[b] - 1, or with q_offsets [b + 1] a ragged batch of new tokens,
    rows q_offsets[b] .. q_offsets[b+1] - 1 of q, at most max_q per sequence."""
    b = q.shape[0] if q_offsets is None else q_offsets.shape[0] - 1
    dt, dev = _type(q), q.get_device()
    desc = _quant_desc(q, k_pages, v_pages, page_table, b, 1 if q_offsets is None else max_q, max_ctx, scale, window,
                       sinks, total_ctx)
    if not (0 <= dev == k_pages.get_device() == v_pages.get_device() == page_table.get_device() == ctx.get_device()
            and page_table.dtype is _I32 is ctx.dtype and page_table.is_contiguous() and ctx.is_contiguous()
            and ctx.shape == (b,)):
        _same(dev, "q k_pages v_pages", q, k_pages, v_pages)
        _book(dev, "page_table ctx", page_table, ctx)
        _vector("ctx", ctx, b)
    if q_offsets is not None or flags is not None:
        _book(dev, "q_offsets flags", q_offsets, flags)
        _vector("q_offsets", q_offsets, b + 1)
    L, ref, ws, nb = lib(), ctypes.byref(desc), workspace, 0
    if out is None:
        out = _empty(stream, q.shape, q.dtype, q.device)
    elif out.shape != q.shape or out.dtype is not q.dtype or not out.is_contiguous() or out.get_device() != dev:
        raise ValueError("out must be a contiguous tensor of q's shape and type on its GPU")
    if ws is None:
        nb = L.presto_quant_attention_workspace(ref, dt, q_offsets is not None)
        if nb:
            ws = _empty(stream, nb, torch.uint8, q.device, returned=False)
    else:
        nb = _room(ws, dev)
    _launch(L.presto_quant_attention, "presto_quant_attention", dev, stream, ref, dt, q.data_ptr(), _ptr(q_offsets),
            k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), ctx.data_ptr(), out.data_ptr(), _ptr(flags),
            _ptr(ws), nb)
    return out


def quant_attention_workspace(q: torch.Tensor, k_pages: torch.Tensor, page_table: torch.Tensor, *, max_q: int = 1,
                              max_ctx: int | None = None, window: int = 0, sinks: int = 0,
                              total_ctx: int = 0) -> torch.Tensor:
    """A workspace for presto_quant_attention calls with just these sizes and
    hints, with q_offsets and, on one token per sequence, without (another size
    may be split further and need more: it is asked for per shape)."""
    desc = _quant_desc(q, k_pages, k_pages, page_table, page_table.shape[0], max_q, max_ctx, None, window, sinks,
                       total_ctx)
    need = max(lib().presto_quant_attention_workspace(ctypes.byref(desc), _type(q), ragged) for ragged in (0, 1))
    return torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)


# ---------------------------------------------------------------------------
# sampling

def _logits(logits) -> int:
    if logits.dim() != 2 or (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError("logits must be [rows, vocab], contiguous in vocab")
    if logits.shape[0] > 1 and logits.stride(0) < logits.shape[1]:
        raise ValueError("the rows of logits must not overlap")
    return _type(logits)


def presto_sample(logits: torch.Tensor, u: torch.Tensor, *, temperature=None, top_k=None, top_p=None, min_p=None,
                  out=None, logprob=None, flags=None, workspace=None, stream=None):
    """A token of each row of logits [rows, V], drawn with u [rows] in [0, 1):
    (token int32 [rows], the log of its share fp32 [rows]).  temperature, top_p,
    min_p: fp32 [rows], top_k: int32 [rows], on the GPU; None: 1, and no cut."""
    dt, dev = _logits(logits), logits.get_device()
    n, vocab = logits.shape
    stride = max(logits.stride(0), vocab) if n > 1 else vocab
    _one_by_one(vocab)
    for name, t in (("u", u), ("temperature", temperature), ("top_p", top_p), ("min_p", min_p), ("logprob", logprob)):
        if t is not None and (t.dtype is not torch.float32 or t.get_device() != dev or dev < 0 or t.shape != (n,)
                              or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous fp32 tensor [{n}] on the GPU of the logits")
    _book(dev, "top_k out flags", top_k, out, flags)
    _vector("top_k", top_k, n)
    _vector("out", out, n)
    if out is None:
        out = _empty(stream, (n,), _I32, logits.device)
    if logprob is None:
        logprob = _empty(stream, (n,), torch.float32, logits.device)
    L, ws, nb = lib(), workspace, 0
    if ws is None:
        nb = L.presto_sample_workspace(dt, n, vocab)
        if nb:
            ws = _empty(stream, nb, torch.uint8, logits.device, returned=False)
    else:
        nb = _room(ws, dev)
    _launch(L.presto_sample, "presto_sample", dev, stream, dt, logits.data_ptr(), n, vocab, stride, u.data_ptr(),
            _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), out.data_ptr(), logprob.data_ptr(), _ptr(flags),
            _ptr(ws), nb)
    return out, logprob


def sample_workspace(logits: torch.Tensor) -> torch.Tensor:
    """A workspace for presto_sample on logits of this shape and type."""
    need = lib().presto_sample_workspace(_logits(logits), *logits.shape)
    return torch.empty(max(need, 16), dtype=torch.uint8, device=logits.device)
