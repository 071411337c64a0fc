"""Decoding in bf16 holds its probabilities to more bits than one bf16 has:
what is left of the error is the output's own rounding."""
import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2607_22634_amd as P
from test_gpu_paged import Cache, ints, queries

pytestmark = pytest.mark.gpu


def _tight(q, k, v, pos0, window, sinks):
    """The 64-bit output and the bound of paged_ref.attention with another
    rounding of p: to two bf16, the second of which holds what the first left
    (at most 2^-8 of p) to 2^-8 of itself, so 2^-16 in all.  Everything else is
    that of fp32 arithmetic; then half a step of the bf16 output."""
    want, fp32 = R.attention(q, k, v, pos0, window, sinks, None, "f32")
    A, _ = R.attention(q, k, np.abs(v), pos0, window, sinks, None, "f32")
    inner = fp32 + 1.01 * 2.0 ** -16 * (A + np.abs(want))
    return want, inner + 2.0 ** -8 * (np.abs(want) + inner)


@pytest.mark.parametrize("heads", [(32, 8, 128), (7, 1, 128), (6, 6, 64), (20, 1, 64), (64, 1, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 5)])
@pytest.mark.parametrize("hint", [False, True])
def test_decode_rounds_its_output_only(heads, window, sinks, hint):
    hq, hkv, d = heads
    rng = np.random.default_rng([70, hq, d, window])
    ctx = [1, 2, 5, 17, 64, 300, 1000, 3000]
    c = Cache(rng, ctx, [1] * len(ctx), 16, hkv, d, "bf16", window, sinks)
    q = queries(rng, len(ctx), hq, d, "bf16")
    out = P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx, max_ctx=3000, window=window, sinks=sinks,
                                   total_ctx=sum(ctx) if hint else 0).double().cpu().numpy()
    qh = q.double().cpu().numpy()
    for b, n in enumerate(ctx):
        want, bound = _tight(qh[b:b + 1], *c.rows(b), n - 1, window, sinks)
        err = np.abs(out[b:b + 1] - want)
        assert (err <= bound).all(), (n, (err / bound).max())


def test_short_chunks_round_their_output_only():
    rng = np.random.default_rng(71)
    hq, hkv, d, new, ctx = 16, 4, 128, [4, 1, 8, 3], [700, 900, 8, 5000]
    c = Cache(rng, ctx, new, 64, hkv, d, "bf16")
    offs = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = queries(rng, offs[-1], hq, d, "bf16")
    out = P.presto_window_attention(q, ints(offs), 8, c.k, c.v, c.table, c.ctx).double().cpu().numpy()
    qh = q.double().cpu().numpy()
    for b, (n, L) in enumerate(zip(new, ctx)):
        s = slice(offs[b], offs[b] + n)
        want, bound = _tight(qh[s], *c.rows(b), L - n, 0, 0)
        assert (np.abs(out[s] - want) <= bound).all(), b
