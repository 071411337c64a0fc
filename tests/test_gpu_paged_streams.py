"""Calls of the paged cache on a stream that is not the current one, while the
current one is still at work on memory that has been given back."""
import numpy as np
import pytest
import torch

import paper_2607_22634_amd as P
from test_gpu_paged import Cache, ints, queries

pytestmark = pytest.mark.gpu


def _after_late_writes(shapes, call):
    """call() with blocks of these (shape, dtype) just freed on the current
    stream, whose last writers have not started"""
    busy = torch.empty(1 << 28, device="cuda")
    torch.cuda.synchronize()
    for _ in range(60):  # (some 10 ms of work)
        busy.fill_(1.0)
    late = [torch.empty(s, dtype=t, device="cuda") for s, t in shapes]
    for t in late:
        t.view(torch.uint8).fill_(0xff)
    del late, t
    got = call()
    torch.cuda.synchronize()
    return got


def test_outputs_and_workspaces_are_not_written_by_earlier_work():
    rng = np.random.default_rng(60)
    c = Cache(rng, [9000, 40, 5000], [1] * 3, 64, 2, 128, "bf16")
    q = queries(rng, 3, 8, 128, "bf16")
    want = P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx)
    ws = P.paged_attention_workspace(q, c.k, c.table)
    assert ws.numel() > 16  # cut, so that the call needs one
    s = torch.cuda.Stream()
    for _ in range(3):
        got = _after_late_writes([(q.shape, q.dtype), (ws.shape, ws.dtype)],
                                 lambda: P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx, stream=s))
        assert torch.equal(got, want)


def test_books_are_not_written_by_earlier_work():
    page, B, pages = 16, 300, 4000
    add = ints([(7 * b) % 90 for b in range(B)])

    def books():
        return torch.zeros(pages, dtype=torch.int32, device="cuda"), ints([[-1] * 8] * B), ints([0] * B)

    refs, table, ctx = books()
    want = P.presto_pages_reserve(refs, table, ctx, page, add)
    ws, s = P.pages_workspace(refs, table), torch.cuda.Stream()
    late = [(ctx.shape, ctx.dtype), (ws.shape, ws.dtype)]
    got_books = books()
    got = _after_late_writes(late, lambda: P.presto_pages_reserve(*got_books, page, add, stream=s))
    assert torch.equal(got, want)
    assert torch.equal(got_books[0], refs) and torch.equal(got_books[1], table)
    refs[::3] = 0
    k = torch.randn(1, pages, page, 1, 64, device="cuda")
    kw = dict(refs=refs, page_table=table, k_pages=k.clone(), v_pages=k.clone())
    want = P.presto_pages_compact(**kw)
    late = [(refs.shape, refs.dtype), (table.shape, table.dtype), (1, torch.int32), (ws.shape, ws.dtype)]
    kw.update(k_pages=k.clone(), v_pages=k.clone())
    got = _after_late_writes(late, lambda: P.presto_pages_compact(**kw, stream=s))
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_a_stream_of_a_capture():
    """Tensors made during a capture, with the captured stream given."""
    rng = np.random.default_rng(61)
    c = Cache(rng, [3000, 70], [1] * 2, 64, 2, 128, "bf16")
    q = queries(rng, 2, 8, 128, "bf16")
    want = P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx)
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        out = P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx, stream=s)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx), want)
