"""Rows whose allowed tokens are all alike and the others masked: places that lie
exactly on a border between two tokens go to the later one, as u times the sum is
then a running sum, which the one drawn has to exceed."""
import math

import numpy as np
import pytest
import torch

from test_gpu_rope import DT
from test_gpu_sample import draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1000, 5000, 70001])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 64, 300, 512, 700])
def test_equal_tokens_among_masked_ones(n, vocab, dtype):
    rng = np.random.default_rng([70, n, vocab])
    values = [1.5, -1.5, 0.0, 1e-3, -1e-3, 0.3, 100.3, -100.3, math.log(0.25), -9.7, 131.0, -131.0, 2.0 ** -8, -2.0 ** -8, 1e-30]
    eighths = np.arange(8) / 8
    z = torch.full((len(values), vocab), -math.inf)
    kept = []
    for r, x in enumerate(values):
        kept.append(np.sort(rng.choice(vocab, n, replace=False)))
        z[r, torch.from_numpy(kept[-1])] = x
    z[2, kept[2][::2]] = -0.0  # (equal to 0)
    z = z.to(DT[dtype]).cuda()
    for u in eighths:
        for kw, left in ((dict(), n), (dict(temperature=0.7), n), (dict(temperature=3.0), n), (dict(top_p=0.5), -(-n // 2)),
                         (dict(top_k=max(n // 2, 1)), max(n // 2, 1)), (dict(min_p=1.0), n),
                         (dict(top_k=n, top_p=0.25, min_p=0.5, temperature=1.3), -(-n // 4))):
            token, logprob, flags = draw(z, np.full(len(values), u), **kw)
            assert flags == 0
            want = [int(k[math.floor(u * left)]) for k in kept]  # (u * left is exact)
            assert token.tolist() == want, (u, kw, [values[r] for r in range(len(values)) if token[r] != want[r]])
            # the total is a whole number; one rounding to fp32
            assert (np.abs(logprob + math.log(left)) <= 2.0 ** -24 * math.log(left) + 2.0 ** -50).all()
