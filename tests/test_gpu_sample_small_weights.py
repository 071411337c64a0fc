"""Many tokens of little weight, which together are within reach of u: a million
of 2^-43 are 2^-23 of the largest one, and fp32 numbers below 1 come to 2^-24 of it.

The reference sums in 80-bit numbers, the tail by itself: what 2^20 small terms
lose, all rounded the same way when they are added to a large one, is what these
tests are about."""
import math

import numpy as np
import pytest
import torch

from test_gpu_rope import DT
from test_gpu_sample import draw

pytestmark = pytest.mark.gpu

LAST = 1 - 2.0 ** -24
# How far a running sum may be off, of itself.  The weights of a bin of several
# values are held in units of 2^-(62 - bits of vocab), at least 2^-41, of what its
# upper end weighs, rounded (a half), and a bin on the grid is at most 4 octaves
# wide: 2^-42 * 2^4 of each weight.  (A lost tail is 2^-24 of the sum and more.)
SUMS = 2.0 ** -38


def check(z, u, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """Rows of z, all alike, drawn with u[r]."""
    kw = {n: x for n, x in (("top_k", top_k), ("top_p", top_p), ("min_p", min_p)) if x}
    token, logprob, flags = draw(z, u, temperature=temperature, **kw)
    assert flags == 0
    row = z[0].double().cpu().numpy().astype(np.longdouble)
    order = np.argsort(-row, kind="stable")
    w = np.exp((row[order] - row[order[0]]) / np.longdouble(np.float32(temperature)))
    n = min(len(row), top_k or len(row))
    run = np.concatenate([w[:1], w[0] + np.cumsum(w[1:n])])
    if top_p < 1:
        n = min(n, int(np.searchsorted(run, np.longdouble(np.float32(top_p)) * run[-1])) + 1)
    n = min(n, int((w >= np.longdouble(np.float32(min_p))).sum()))
    run = run[:n]
    for r, x in enumerate(np.asarray(u, dtype=np.float32)):
        at = [min(int(np.searchsorted(run, (np.longdouble(x) + d) * run[-1], side="right")), n - 1)
              for d in (-2 * SUMS, 0.0, 2 * SUMS)]  # (the sum's error and the total's)
        assert token[r] in order[at[0]:at[2] + 1], (r, token[r], at)
        place = int(np.flatnonzero(order[at[0]:at[2] + 1] == token[r])[0]) + at[0]
        want = float(np.log(w[place] / run[-1]))
        # the total's error, and one rounding to fp32
        assert abs(logprob[r] - want) <= 2.0 ** -24 * abs(want) + SUMS
    return token


def rows_of(top, below, temperature, vocab, dtype, rng):
    """One largest logit, the others `below` octaves beneath it, and some of them
    half an octave more."""
    more = rng.choice([0.0, 0.5], vocab)
    z = top - (below + more) * math.log(2) * temperature
    z[rng.integers(vocab)] = top
    return torch.from_numpy(z.astype(np.float32)[None].repeat(4, 0)).to(DT[dtype]).cuda()


# (largest logit, temperature): on the grid that rows are counted on, above and
# below it, next to 0, and temperatures of all sizes
@pytest.mark.parametrize("top,temperature", [(3.0, 1.0), (200.0, 1.0), (-3.0, 1.0), (-200.0, 1.0), (2.0 ** -8, 1.2e-5),
                                             (0.0, 1.0), (0.0, 1e-4), (2e-9, 1e-10), (1e6, 3e4)])
@pytest.mark.parametrize("vocab", [1 << 20, 151936])
def test_the_tail_is_not_lost(vocab, top, temperature):
    rng = np.random.default_rng([32, vocab])
    # (as much weight as 2^20 tokens at 43 octaves have, 2^-23 and a little less)
    z = rows_of(top, 23 + math.log2(vocab), temperature, vocab, "f32", rng)
    u = [0.0, 0.5, 1 - 2.0 ** -23, LAST]
    token = check(z, u, temperature)
    assert token[3] != token[0]
    check(z, u, temperature, min_p=1e-18)
    check(z, u, temperature, top_k=vocab - 5)
    check(z, u, temperature, top_p=LAST)


def test_the_tail_of_a_bf16_row():
    """bf16 values within 2^-8 of 0, whose bin holds many."""
    rng = np.random.default_rng(33)
    z = rows_of(0.0, 43, 1e-4, 1 << 20, "bf16", rng)
    check(z, [0.0, 0.5, 1 - 2.0 ** -23, LAST], 1e-4)
