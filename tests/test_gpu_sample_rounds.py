"""Sampling calls of more rows than share a workspace, and rows of the longest
vocabularies, which are counted in more slices than others."""
import math

import numpy as np
import pytest
import torch

import paper_2607_22634_amd as P
from test_gpu_rope import DT
from test_gpu_sample import check, draw, f32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(2048, 1025), (2049, 1500), (4100, 1999)])
def test_rows_of_several_rounds(rows, vocab, dtype):
    rng = np.random.default_rng([60, rows])
    z = torch.from_numpy((rng.standard_normal((rows, vocab)) * 3).astype(np.float32)).to(DT[dtype]).cuda()
    u = rng.random(rows)
    kw = dict(temperature=rng.choice([0.0, 0.7, 1.0, 30.0], rows), top_k=rng.choice([0, 1, 40, 1000], rows),
              top_p=rng.choice([1.0, 0.3, 0.95], rows), min_p=rng.choice([0.0, 0.05], rows))
    token, logprob, flags = draw(z, u, **kw)
    assert flags == 0
    for lo, hi in ((0, 40), (2028, 2068), (4080, 4100)):
        lo, hi = min(lo, rows - 20), min(hi, rows)
        part = slice(lo, hi)
        one = {n: x[part] for n, x in kw.items()}
        t, p, _ = draw(z[part], u[part], **one)
        assert (t == token[part]).all() and (p == logprob[part]).all()
        check(z[part], u[part], **one)
    # a bad row of a later round is its own
    z[rows - 1, vocab - 1] = math.nan
    t, p, flags = draw(z, u, **kw)
    assert flags == P.PRESTO_FLAG_NAN_LOGITS and t[-1] == -1 and math.isnan(p[-1])
    assert (t[:-1] == token[:-1]).all() and (p[:-1] == logprob[:-1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [524288, 524289, (1 << 20) - 1, 1 << 20])
def test_the_longest_rows(vocab, dtype):
    """Among them rows whose likely tokens, cuts and draws lie in the last slices."""
    rng = np.random.default_rng([61, vocab])
    z = torch.from_numpy((rng.standard_normal((6, vocab)) * 3).astype(np.float32))
    z[1, vocab - 40000:] += 12
    z[2, vocab - 700:] += 20
    z[3, vocab - 1] = 60
    z[4, :vocab - 300] = -math.inf
    z = z.to(DT[dtype]).cuda()
    for u in (0.0, 0.61, 1 - 2.0 ** -24):
        check(z, np.full(6, u))
    check(z, rng.random(6), top_k=500, top_p=0.9)
    check(z, rng.random(6), top_k=[vocab, 40000, 600, 2, 299, 7], min_p=1e-5)
    check(z, rng.random(6), temperature=[0.0, 0.8, 2.0, 1.0, 1e-3, 0.5], top_p=0.99)
    ws = P.sample_workspace(z)
    for at in (vocab - 1, vocab - 32768, 524287):
        y = z.clone()
        y[5, at] = math.nan
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        token, logprob = P.presto_sample(y, f32(np.full(6, 0.5)), workspace=ws, flags=flags)
        assert flags.item() == P.PRESTO_FLAG_NAN_LOGITS
        assert token[5] == -1 and torch.isnan(logprob[5]) and (token[:5] >= 0).all()
