"""Host-only checks of the paged cache: what its entry points refuse before
anything is launched, workspace sizes, and the reference itself (no GPU)."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2607_22634_amd as P
from paper_2607_22634_amd import _paged

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: the checks fail first


def pages(**over):
    d = P.PagesDesc(4, 64, 300, 16, 8, 128, P.PRESTO_DT_BF16, 1, 0, 0)
    for k, v in over.items():
        setattr(d, k, v)
    return d


def attn(pool=None, **over):
    d = P.PagedAttnDesc(pool or pages(), 32, 8, 1000, 0, 0, 0.1, 32, 0, 0)
    for k, v in over.items():
        setattr(d, k, v)
    return d


BAD_POOLS = [dict(page_size=8), dict(page_size=48), dict(page_size=2048), dict(head_dim=96), dict(hkv=0), dict(hkv=5000),
             dict(num_pages=0), dict(max_pages=0), dict(max_pages=(1 << 20) + 1), dict(max_pages=1 << 20, page_size=1024),
             dict(batch=1 << 23), dict(batch=1 << 20, max_pages=1 << 12, page_size=16), dict(layers=0), dict(dt=7), dict(batch=-1), dict(page_stride=16 * 8 * 128 - 8),
             dict(page_stride=16 * 8 * 128 + 4), dict(layer_stride=-8), dict(layer_stride=12), dict(page_stride=1 << 62)]
BAD_ATTN = [dict(hq=12), dict(hq=0), dict(max_ctx=-1), dict(max_ctx=64 * 16 + 1), dict(max_q=-1), dict(window=-1),
            dict(window=(1 << 30) + 1), dict(sinks=-1), dict(scale=0.0), dict(scale=float("nan")), dict(total_q=-1),
            dict(total_q=1 << 30), dict(total_ctx=-1), dict(q_stride=32 * 128 - 8), dict(q_stride=32 * 128 + 4),
            dict(max_q=1 << 30)]


def _attend(d, decode):
    lib = P.lib()
    if decode:
        return lib.presto_paged_attention(ctypes.byref(d), *[FAKE] * 6, None, FAKE, 1 << 40, None)
    return lib.presto_window_attention(ctypes.byref(d), *[FAKE] * 7, None, FAKE, 1 << 40, None)


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("over", BAD_POOLS)
def test_attention_refuses_bad_pools(over, decode):
    assert _attend(attn(pages(**over)), decode) == P.PRESTO_ERR_INVALID_ARG
    assert P.lib().presto_last_error()


@pytest.mark.parametrize("over", BAD_ATTN)
def test_window_attention_refuses_bad_descriptors(over):
    assert _attend(attn(**over), False) == P.PRESTO_ERR_INVALID_ARG
    assert b"presto_window_attention" in P.lib().presto_last_error()
    assert P.lib().presto_window_attention_workspace(ctypes.byref(attn(**over))) == 0


@pytest.mark.parametrize("over", [o for o in BAD_ATTN if not {"max_q", "total_q"} & set(o)])
def test_paged_attention_refuses_bad_descriptors(over):
    assert _attend(attn(**over), True) == P.PRESTO_ERR_INVALID_ARG


def test_attention_refuses_null_and_misaligned_tensors():
    lib, d = P.lib(), attn()
    assert lib.presto_paged_attention(None, *[FAKE] * 6, None, FAKE, 1 << 40, None) == P.PRESTO_ERR_INVALID_ARG
    for i in range(6):
        args = [FAKE] * 6
        args[i] = None
        assert lib.presto_paged_attention(ctypes.byref(d), *args, None, FAKE, 1 << 40, None) == P.PRESTO_ERR_INVALID_ARG
    for i in (0, 1, 2, 5):
        args = [FAKE] * 6
        args[i] = ctypes.c_void_p(0x1008)
        assert lib.presto_paged_attention(ctypes.byref(d), *args, None, FAKE, 1 << 40, None) == P.PRESTO_ERR_INVALID_ARG
        assert b"aligned" in lib.presto_last_error()


def test_attention_refuses_a_small_workspace():
    d = attn(pages(batch=1, max_pages=4096), max_q=1, max_ctx=60000, total_q=1)
    need = P.lib().presto_window_attention_workspace(ctypes.byref(d))
    assert need > 0 and need == P.lib().presto_paged_attention_workspace(ctypes.byref(d))
    for ws, nb in ((FAKE, need - 1), (None, need)):
        st = P.lib().presto_paged_attention(ctypes.byref(d), *[FAKE] * 6, None, ws, nb, None)
        assert st == P.PRESTO_ERR_WORKSPACE


def test_empty_calls_do_nothing():
    lib = P.lib()
    for d in (attn(pages(batch=0)), attn(max_q=0), attn(total_q=0)):
        assert lib.presto_window_attention(ctypes.byref(d), *[None] * 9, 0, None) == P.PRESTO_OK
    p = pages(batch=0)
    assert lib.presto_paged_attention(ctypes.byref(attn(p)), *[None] * 8, 0, None) == P.PRESTO_OK
    assert lib.presto_pages_reserve(ctypes.byref(p), None, None, None, None, 1, None, None, None, 0, None) == P.PRESTO_OK
    assert lib.presto_append_kv(ctypes.byref(p), None, None, 4, 0, None, 3, *[None] * 7) == P.PRESTO_OK
    assert lib.presto_append_kv(ctypes.byref(pages()), None, None, 0, 0, None, 3, *[None] * 7) == P.PRESTO_OK
    assert lib.presto_pages_fork(ctypes.byref(pages()), *[None] * 5, 0, *[None] * 4, 0, None) == P.PRESTO_OK
    assert lib.presto_pages_free(ctypes.byref(pages()), *[None] * 4, 0, None, None) == P.PRESTO_OK
    assert lib.presto_pages_trim(ctypes.byref(p), None, None, None, 5, 0, None, None) == P.PRESTO_OK


@pytest.mark.parametrize("over", BAD_POOLS)
def test_books_refuse_bad_pools(over):
    lib, d = P.lib(), pages(**over)
    bad = P.PRESTO_ERR_INVALID_ARG
    assert lib.presto_pages_reserve(ctypes.byref(d), *[FAKE] * 4, 1, FAKE, None, FAKE, 1 << 40, None) == bad
    assert lib.presto_append_kv(ctypes.byref(d), FAKE, FAKE, 4, 0, FAKE, 3, *[FAKE] * 5, None, None) == bad
    assert lib.presto_pages_fork(ctypes.byref(d), *[FAKE] * 5, 1, FAKE, FAKE, None, FAKE, 1 << 40, None) == bad
    assert lib.presto_pages_free(ctypes.byref(d), *[FAKE] * 4, 1, None, None) == bad
    assert lib.presto_pages_trim(ctypes.byref(d), *[FAKE] * 3, 5, 0, None, None) == bad
    assert lib.presto_pages_compact(ctypes.byref(d), *[FAKE] * 8, None, FAKE, 1 << 40, None) == bad
    assert lib.presto_pages_workspace(ctypes.byref(d)) == 0


def test_books_refuse_bad_arguments():
    lib, d = P.lib(), pages()
    bad = P.PRESTO_ERR_INVALID_ARG
    need = lib.presto_pages_workspace(ctypes.byref(d))
    assert need >= 300 * 4
    assert lib.presto_pages_reserve(ctypes.byref(d), *[FAKE] * 4, -1, FAKE, None, FAKE, need, None) == bad
    assert lib.presto_pages_reserve(ctypes.byref(d), *[FAKE] * 4, 1, None, None, FAKE, need, None) == bad
    assert lib.presto_pages_reserve(ctypes.byref(d), *[FAKE] * 4, 1, FAKE, None, FAKE, need - 1, None) == P.PRESTO_ERR_WORKSPACE
    for n in (-1, 5):
        assert lib.presto_pages_fork(ctypes.byref(d), *[FAKE] * 5, n, FAKE, FAKE, None, FAKE, need, None) == bad
        assert lib.presto_pages_free(ctypes.byref(d), *[FAKE] * 4, n, None, None) == bad
    assert lib.presto_pages_fork(ctypes.byref(d), *[FAKE] * 5, 1, FAKE, FAKE, None, None, 0, None) == P.PRESTO_ERR_WORKSPACE
    assert lib.presto_pages_compact(ctypes.byref(d), *[FAKE] * 8, None, FAKE, need - 1, None) == P.PRESTO_ERR_WORKSPACE
    for w, s in ((0, 0), (-1, 0), (5, -1)):
        assert lib.presto_pages_trim(ctypes.byref(d), *[FAKE] * 3, w, s, None, None) == bad
    for rows, stride, most in ((-1, 0, 3), (1 << 31, 0, 3), (4, 8, 3), (4, 8 * 128 + 4, 3), (4, 0, -1)):
        assert lib.presto_append_kv(ctypes.byref(d), FAKE, FAKE, rows, stride, FAKE, most, *[FAKE] * 5, None, None) == bad


def test_workspace_needs_no_more_for_smaller_calls():
    """A workspace sized for the longest context and most tokens serves the
    short calls of the same batch too."""
    lib = P.lib()
    for batch in (1, 3, 16):
        pool = pages(batch=batch, max_pages=4096)
        sizes = [lib.presto_paged_attention_workspace(ctypes.byref(attn(pool, max_ctx=c))) for c in (0, 1, 500, 60000)]
        assert sizes[0] == sizes[1] == 0 and sizes[-1] >= max(sizes)


def test_binding_refuses_host_tensors():
    q = torch.zeros(1, 4, 64)
    k = torch.zeros(3, 16, 2, 64)
    t, c = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        P.presto_paged_attention(q, k, k, t, c)
    with pytest.raises(ValueError):
        P.presto_pages_reserve(torch.zeros(3, dtype=torch.int32), t, c, 16, extra=1)


def test_binding_refuses_overlapping_tokens_and_layers():
    k = torch.zeros(4, 16, 2, 64)
    table, ctx, offs = torch.zeros(3, 2, dtype=torch.int32), torch.ones(3, dtype=torch.int32), torch.arange(4).int()
    for q in (torch.zeros(1, 4, 64).expand(3, 4, 64), torch.zeros(600).as_strided((3, 4, 64), (64, 64, 1))):
        with pytest.raises(ValueError, match="overlap"):
            P.presto_paged_attention(q, k, k, table, ctx)
        with pytest.raises(ValueError, match="overlap"):
            P.presto_window_attention(q, offs, 1, k, k, table, ctx)
        with pytest.raises(ValueError, match="overlap"):
            P.paged_attention_workspace(q, k, table)
    pool = _paged._pool
    for stride in ((2048 * 4, 2048), (2048, 2048 * 5), (4096, 4096 * 5)):  # layer by layer, page by page, of pairs
        p = torch.zeros(5 * 4 * 4096).as_strided((5, 4, 16, 2, 64), (*stride, 128, 64, 1))
        d = pool(p, p, 2, 3, True)
        assert (d.layer_stride, d.page_stride) == stride
    for stride in ((2048 * 3, 2048), (2048, 2048 * 4), (4096, 4096 * 4), (0, 2048)):
        p = torch.zeros(5 * 4 * 4096).as_strided((5, 4, 16, 2, 64), (*stride, 128, 64, 1))
        with pytest.raises(ValueError, match="overlap"):
            pool(p, p, 2, 3, True)
    with pytest.raises(ValueError, match="contiguous"):
        _paged._room(torch.zeros(1, dtype=torch.uint8).expand(64), -1)


def test_reference_attention_on_a_case_by_hand():
    k = np.array([[[0.0]], [[np.log(3.0)]], [[5.0]]])
    v = np.array([[[1.0]], [[5.0]], [[100.0]]])
    o, _ = R.attention(np.ones((1, 1, 1)), k, v, 1, scale=1.0)
    assert np.allclose(o, (1 + 3 * 5) / 4)
    o, _ = R.attention(np.ones((1, 1, 1)), k, v, 2, window=1, sinks=1, scale=1.0)
    assert np.allclose(o, (1 + np.exp(5) * 100) / (1 + np.exp(5)))
    o, _ = R.attention(np.ones((2, 1, 1)), k, v, -1, scale=1.0)
    assert o[0, 0, 0] == 0 and np.allclose(o[1], 1)


def test_reference_books_by_hand():
    b = R.Books([0] * 6, [[-1] * 4 for _ in range(3)], [0, 0, 0], 16)
    b.ctx = b.reserve([20, 0, 16], 0)
    assert b.table[0][:2] == [0, 1] and b.table[2][0] == 2 and b.ctx == [20, 0, 16]
    assert b.fork([0], [1]) == [(1, 3, 4)] and b.table[1][:2] == [0, 3] and b.refs == [2, 1, 1, 1, 0, 0]
    b.free([0])
    assert b.refs == [1, 0, 1, 1, 0, 0] and b.ctx == [0, 20, 16]
    moves, to, live = b.compact()
    assert moves == [(3, 1, 16)] and live == 3 and b.table[1][:2] == [0, 1] and to == [0, -1, 2, 1, -1, -1]


def test_calls_too_large_for_one_grid_are_refused():
    """More workgroups, or query rows, than a launch can number."""
    lib = P.lib()
    big = attn(pages(batch=(1 << 23) - 1, max_pages=2), max_ctx=32, max_q=1, total_q=(1 << 23) - 1)
    for fn, n in ((lib.presto_paged_attention, 6), (lib.presto_window_attention, 7)):
        assert fn(ctypes.byref(big), *[FAKE] * n, None, FAKE, 1 << 40, None) == P.PRESTO_ERR_UNSUPPORTED
    wide = attn(pages(batch=64, max_pages=1 << 16), max_ctx=1 << 20, max_q=1 << 20, total_q=64 << 20)
    assert _attend(wide, False) == P.PRESTO_ERR_UNSUPPORTED
    d = pages(batch=1 << 20, max_pages=1024)
    assert lib.presto_append_kv(ctypes.byref(d), FAKE, FAKE, 1 << 30, 0, FAKE, 1000, *[FAKE] * 5, None, None) == \
        P.PRESTO_ERR_INVALID_ARG


@pytest.mark.parametrize("n", [1, 2, 5, 8, 9, 33, 64, 127, 1000, 4096])
def test_workspaces_hold_the_partials(n):
    """Whatever the plan, the workspace is either none or room for one partial
    of every row at least, and the same each time it is asked for."""
    lib = P.lib()
    for dt, hkv, d in itertools.product((P.PRESTO_DT_BF16, P.PRESTO_DT_F32), (1, 8), (64, 128)):
        for batch, ctx, window, total in itertools.product((1, 5, 70, 3000), (0, 17, 4100, 150000), (0, 500), (0, 1)):
            pool = pages(batch=batch, max_pages=9400, hkv=hkv, head_dim=d, dt=dt)
            a = attn(pool, hq=hkv * 4, max_q=n, max_ctx=ctx, window=window, sinks=4, total_q=batch * n,
                     total_ctx=total * batch * ctx)
            need = lib.presto_window_attention_workspace(ctypes.byref(a))
            assert need == lib.presto_window_attention_workspace(ctypes.byref(a))
            assert need == 0 or need >= hkv * 4 * n * (d * 4 + 8)
