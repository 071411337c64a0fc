"""What the binding says about sizes.  Numbers that do not fit the C interface's 32 bits are refused: cut to their
low half, a window of 2^32 would be none at all (no GPU)."""
import ctypes

import pytest
import torch

import paper_2607_22634_amd as P
from paper_2607_22634_amd import _paged

FAR = [1 << 31, 1 << 32, (1 << 32) + 5, -(1 << 31) - 1, -(1 << 32), 1 << 64]


def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


@pytest.mark.parametrize("value", FAR)
@pytest.mark.parametrize("name", ["max_ctx", "window", "sinks", "max_q"])
def test_attention_refuses_numbers_past_32_bits(name, value):
    q, k = torch.zeros(1, 4, 64), torch.zeros(3, 16, 2, 64)
    kw = {name: value}
    with pytest.raises(ValueError, match="32 bits"):
        P.paged_attention_workspace(q, k, _i32(1, 2), **kw)
    most = kw.pop("max_q", 1)
    with pytest.raises(ValueError, match="32 bits"):
        P.presto_window_attention(q, _i32(2), most, k, k, _i32(1, 2), _i32(1), **kw)
    if kw:
        with pytest.raises(ValueError, match="32 bits"):
            P.presto_paged_attention(q, k, k, _i32(1, 2), _i32(1), **kw)
        with pytest.raises(ValueError, match="32 bits"):  # whatever stands beside it
            P.presto_paged_attention(q, k, k, _i32(1, 2), _i32(1), **{"window": 7, "sinks": 3, **kw})


@pytest.mark.parametrize("value", FAR)
def test_books_refuse_numbers_past_32_bits(value):
    refs, table, ctx = _i32(3), _i32(1, 2), _i32(1)
    k = torch.zeros(3, 16, 2, 64)
    for call in (lambda: P.presto_pages_reserve(refs, table, ctx, value, extra=1),
                 lambda: P.presto_pages_reserve(refs, table, ctx, 16, extra=value),
                 lambda: P.presto_pages_trim(refs, table, ctx, value, 5),
                 lambda: P.presto_pages_trim(refs, table, ctx, 16, value),
                 lambda: P.presto_pages_trim(refs, table, ctx, 16, 5, value),
                 lambda: P.presto_append_kv(k[0], k[0], _i32(2), value, k, k, table, ctx, ctx)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


@pytest.mark.parametrize("value", FAR[:3])
def test_sizes_past_32_bits(value):
    """Tables and pools of more sequences, columns or pages."""
    for args in ((value, 2, 3, 16), (1, value, 3, 16), (1, 2, value, 16)):
        with pytest.raises(ValueError, match="32 bits"):
            _paged._books_of(*args)
    page = 16 * 2 * 64
    with pytest.raises(ValueError, match="32 bits"):
        _paged._pool_of((value, 16, 2, 64), (page, 128, 64, 1), torch.float32, 1, 2, False)
    with pytest.raises(ValueError, match="32 bits"):
        _paged._pool_of((value, 1, 16, 2, 64), (page, page, 128, 64, 1), torch.float32, 1, 2, True)


def test_ordinary_numbers_pass():
    q, k = torch.zeros(1, 4, 64), torch.zeros(3, 16, 2, 64)
    for kw in (dict(window=5, sinks=1), dict(max_ctx=32), dict(max_ctx=0), dict(max_q=20)):
        assert P.paged_attention_workspace(q, k, _i32(1, 2), **kw).numel() >= 16


def _need(entry, **over):
    pool = P.PagesDesc(1, 2048, 3000, 16, 8, 128, P.PRESTO_DT_BF16, 1, 0, 0)
    desc = P.PagedAttnDesc(pool, 32, 1, 32768, 0, 0, 0.1, 1, 0, 0)
    for name, value in over.items():
        setattr(desc, name, value)
    return desc, getattr(P.lib(), entry + "_workspace")(ctypes.byref(desc))


def test_workspaces_are_for_the_sizes_they_were_asked_for():
    """A shorter chunk may need more than a longer one, a shorter context or
    another hint more or less; what is asked for a shape is what its call
    wants, and a call is refused with less."""
    entry, fake = "presto_window_attention", ctypes.c_void_p(0x1000)  # never dereferenced: the checks fail first
    sizes = {n: _need(entry, max_q=n, total_q=n)[1] for n in (4096, 2048, 512, 8)}
    assert sizes[512] > sizes[2048] and sizes[512] > sizes[4096]
    for n, need in sizes.items():
        desc, again = _need(entry, max_q=n, total_q=n)
        assert again == need
        if need:
            for room in (need - 1, min(sizes.values())):
                status = P.lib().presto_window_attention(ctypes.byref(desc), *[fake] * 7, None, fake, room, None)
                assert status == P.PRESTO_ERR_WORKSPACE


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", [(32, 8, 128), (20, 1, 64), (4, 4, 64)])
def test_the_binding_asks_for_its_own_call(dtype, heads):
    """paged_attention_workspace against what the two entry points ask for,
    over chunks, contexts and hints."""
    hq, hkv, d = heads
    dt = P.PRESTO_DT_BF16 if dtype is torch.bfloat16 else P.PRESTO_DT_F32
    for batch, most, ctx in ((1, 1, 40), (1, 9, 30000), (3, 512, 30000), (5, 70, 2000), (1, 4096, 32768)):
        cols = 2048
        k = torch.empty(4, 16, hkv, d, dtype=dtype)
        q = torch.empty(batch * most, hq, d, dtype=dtype)
        for total, window in ((0, 0), (batch * ctx, 0), (0, 1000)):
            got = P.paged_attention_workspace(q, k, _i32(batch, cols), max_q=most, max_ctx=ctx, total_ctx=total,
                                              window=window).numel()
            pool = P.PagesDesc(batch, cols, 4, 16, hkv, d, dt, 1, 0, 0)
            desc = P.PagedAttnDesc(pool, hq, most, ctx, window, 0, 0.1, batch * most, 0, total)
            for entry in ("presto_window_attention", "presto_paged_attention"):
                assert got >= getattr(P.lib(), entry + "_workspace")(ctypes.byref(desc))
