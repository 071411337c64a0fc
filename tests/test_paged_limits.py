"""Numbers that do not fit the C interface's 32 bits are refused: cut to their
low half, a window of 2^32 would be none at all (no GPU)."""
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
