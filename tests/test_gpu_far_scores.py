"""Attention over scores that all lie far below zero.  The kernels keep a lazy
reference per row, and a row that has seen nothing yet starts from 0: weighed
against that, terms below 2^-126 are flushed to zero while others are not.

Queries and keys are made such that a score is `far` (log2 units) plus noise of
2: their first components' product, and the product of the others."""
import math

import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2607_22634_amd as P
import synthetic as sy
from brute import anc_from_parent
from gpu_util import to_dev, to_host
from test_gpu_paged import Cache, flag, ints, queries

pytestmark = pytest.mark.gpu
SCALE = math.log(2.0)  # scores in log2 units are the products themselves
FAR = [-122.0, -126.0, -128.0, -140.0, -1000.0]


def _far(x, first):
    """[..., d]: the first component, and noise that makes 2 of a product"""
    x = x * (4.0 / (x.shape[-1] - 1)) ** 0.25
    x[..., 0] = first
    return x


def _far_cache(c, far):
    c.k_h.copy_(_far(c.k_h.float(), far / 8))  # (NaN where nothing sees it stays in the other components)
    c.k.copy_(c.k_h)


@pytest.mark.parametrize("far", FAR)
@pytest.mark.parametrize("dtype,batch,n,past,heads,window,sinks", [
    ("bf16", 2, 1000, 400, (16, 8, 64), 400, 0), ("bf16", 1, 1000, 100, (16, 16, 128), 100, 0),
    ("bf16", 1, 1000, 800, (8, 8, 128), 800, 0), ("bf16", 1, 1000, 800, (8, 8, 128), 800, 5),
    ("bf16", 1, 512, 3000, (8, 2, 128), 0, 0), ("bf16", 1, 40, 900, (4, 2, 64), 100, 0),
    ("f32", 1, 300, 900, (8, 2, 64), 200, 0)])
def test_prompts_of_far_scores(dtype, batch, n, past, heads, window, sinks, far):
    """Windowed prompts, whose later rows see nothing of their block's first
    keys, cut and uncut, and causal ones."""
    hq, hkv, d = heads
    rng = np.random.default_rng([50, n, past, window])
    L = past + n
    c = Cache(rng, [L] * batch, [n] * batch, 64, hkv, d, dtype, window, sinks)
    _far_cache(c, far)
    q = queries(rng, batch * n, hq, d, dtype)
    q.copy_(_far(q.float(), 8.0))
    f = flag()
    out = P.presto_window_attention(q, ints([n * b for b in range(batch + 1)]), n, c.k, c.v, c.table, c.ctx, scale=SCALE,
                                    window=window, sinks=sinks, flags=f)
    assert f.item() == 0
    got, qh = out.double().cpu().numpy(), q.double().cpu().numpy()
    k, v = c.rows(batch - 1)
    for i in range(0, n, 13):
        r = (batch - 1) * n + i
        want, bound = R.attention(qh[r:r + 1], k, v, past + i, window, sinks, SCALE, dtype)
        err = np.abs(got[r:r + 1] - want)
        assert (err <= bound).all(), (i, (err / bound).max())


@pytest.mark.parametrize("far", FAR)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_of_far_scores(dtype, far):
    rng = np.random.default_rng(51)
    ctx = [1, 40, 700, 5000]
    c = Cache(rng, ctx, [1] * 4, 32, 2, 128, dtype)
    _far_cache(c, far)
    q = queries(rng, 4, 8, 128, dtype)
    q.copy_(_far(q.float(), 8.0))
    out = P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx, scale=SCALE).double().cpu().numpy()
    qh = q.double().cpu().numpy()
    for b in range(4):
        k, v = c.rows(b)
        want, bound = R.attention(qh[b:b + 1], k, v, ctx[b] - 1, 0, 0, SCALE, dtype)
        assert (np.abs(out[b:b + 1] - want) <= bound).all(), b


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,past", [(1, 0), (1, 700), (5, 40), (600, 500)])
def test_scores_of_minus_infinity(dtype, n, past):
    """Keys whose score is -inf weigh nothing beside others; a query that sees
    no others gets zeros."""
    rng = np.random.default_rng([53, n, past])
    L, page = past + n, 32
    c = Cache(rng, [L], [n], page, 2, 64, dtype)
    q = queries(rng, n, 4, 64, dtype)
    q[..., 0] = 8.0
    lost = np.arange(L) < L // 3 if L > 1 else np.ones(1, bool)
    for head in range(2):
        dead = lost if head == 0 else np.ones(L, bool)  # KV head 1: all of them
        for j in np.flatnonzero(dead):
            p = int(c.table_h[0, j // page])
            c.k_h[p, j % page, head, 0] = float("-inf")
    c.k.copy_(c.k_h)
    out = P.presto_window_attention(q, ints([0, n]), n, c.k, c.v, c.table, c.ctx).double().cpu().numpy()
    assert not out[:, 2:].any()
    k, v = c.rows(0)
    some = sorted({0, n // 2, n - 1})
    for i in some:
        live = ~lost & (np.arange(L) <= past + i)
        if not live.any():
            assert not out[i, :2].any()
            continue
        want, bound = R.attention(q[i:i + 1, :2].double().cpu().numpy(), k[live, :1], v[live, :1], int(live.sum()) - 1,
                                  0, 0, None, dtype)
        assert (np.abs(out[i:i + 1, :2] - want) <= bound).all(), i


@pytest.mark.parametrize("far", FAR)
@pytest.mark.parametrize("dtype,N,hq,hkv,d", [("bf16", 9, 8, 2, 128), ("bf16", 33, 8, 8, 64), ("bf16", 70, 16, 2, 128),
                                              ("bf16", 257, 8, 1, 64), ("f32", 33, 4, 2, 64)])
def test_trees_of_far_scores(dtype, N, hq, hkv, d, far):
    """Trees of few nodes, whose rows' waves share the keys of one block among
    them, and of many, over contexts of several lengths."""
    rng = np.random.default_rng([52, N, hq])
    ctx = np.array([0, 40, 300, 2000], np.int32)
    b = len(ctx)
    n_nodes = np.array([N, N, max(N // 2, 1), N], np.int32)
    parent = np.full((b, N), -1, np.int32)
    for s in range(b):
        for n in range(1, int(n_nodes[s])):
            parent[s, n] = n - 1 if s == 1 else rng.integers(0, n)
    anc = anc_from_parent(parent, n_nodes, N)
    offs = np.zeros(b + 1, np.int32)
    offs[1:] = np.cumsum(ctx)
    rows = int(offs[-1])
    draw = lambda *s: rng.standard_normal(s, dtype=np.float32)
    q, kc, kt = (sy.cast(_far(draw(*s), x), dtype)
                 for s, x in (((b, N, hq, d), 8.0), ((rows, hkv, d), far / 8), ((b, N, hkv, d), far / 8)))
    vc, vt = sy.cast(draw(rows, hkv, d), dtype), sy.cast(draw(b, N, hkv, d), dtype)
    out = P.presto_tree_attention(to_dev(q, dtype), to_dev(kc, dtype), to_dev(vc, dtype), to_dev(offs), to_dev(kt, dtype),
                                  to_dev(vt, dtype), to_dev(anc), to_dev(n_nodes), int(ctx.max()), SCALE)
    got = sy.as_f32(to_host(out), dtype).astype(np.float64)
    q, kc, vc, kt, vt = (sy.as_f32(x, dtype).astype(np.float64) for x in (q, kc, vc, kt, vt))
    for s in range(b):
        for n in sorted({0, 1, int(n_nodes[s]) // 2, int(n_nodes[s]) - 1}):
            path = [n]
            while path[-1] > 0:
                path.append(int(parent[s, path[-1]]))
            k, v = (np.concatenate([c[offs[s]:offs[s + 1]], t[s, path]]) for c, t in ((kc, kt), (vc, vt)))
            want, bound = R.attention(q[s, n:n + 1], k, v, len(k) - 1, 0, 0, SCALE, dtype)
            # (the bound once more: split contexts round their parts to bf16, by
            # half a step of at most the sum that the bound is made of)
            assert (np.abs(got[s, n:n + 1] - want) <= 2 * bound).all(), (s, n)
