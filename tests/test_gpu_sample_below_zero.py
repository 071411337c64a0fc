"""Rows of which no logit is above zero (log-probabilities, logits less their
maximum), rows whose largest logits lie next to 0, and masked rows at high
temperatures: draws and cuts against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from test_gpu_rope import DT
from test_gpu_sample import check, draw

pytestmark = pytest.mark.gpu


def settings(rng, rows, vocab):
    return dict(temperature=rng.choice([0.0, 0.1, 0.7, 1.0, 1.5, 30.0], rows),
                top_k=rng.choice([0, 1, 2, 5, 40, 1000, vocab, 1 << 30], rows),
                top_p=rng.choice([1.0, 0.0, 1e-6, 0.3, 0.9, 0.95, 0.999, 2.0], rows),
                min_p=rng.choice([0.0, 1e-4, 0.05, 0.3, 1.0], rows))


def each(z, rng):
    rows, vocab = z.shape
    u = rng.random(rows)
    u[:3] = [0.0, 2.0 ** -30, 1 - 2.0 ** -24]
    kw = settings(rng, rows, vocab)
    check(z, u)
    for name in kw:
        check(z, u, **{name: kw[name]})
    check(z, u, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1025, 5000, 50257, 151936])
@pytest.mark.parametrize("kind", ["log-softmax", "less the maximum", "shifted", "confident"])
def test_rows_below_zero(kind, vocab, dtype):
    rng = np.random.default_rng([40, vocab])
    z = torch.from_numpy((rng.standard_normal((16, vocab)) * 3).astype(np.float32))
    if kind == "confident":  # log-probabilities with one next to 0
        z[torch.arange(16), torch.from_numpy(rng.integers(0, vocab, 16))] = torch.linspace(20, 60, 16)
    if kind in ("log-softmax", "confident"):
        z = torch.log_softmax(z.double(), -1).float()
    elif kind == "less the maximum":
        z = z - z.amax(-1, keepdim=True)
    else:
        z = z - z.amax(-1, keepdim=True) - torch.logspace(-3, 2, 16)[:, None]
    assert (z <= 0).all()
    each(z.to(DT[dtype]).cuda(), rng)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_mirrored_bins(dtype):
    """Rows whose largest logit walks over both sides of 0, next to every border
    between bins that matters: 2^-8, 0 and the ends of the grid, +-2^7."""
    rng = np.random.default_rng(41)
    tops = [s * x for x in (2.0 ** -9, 2.0 ** -8 * (1 - 2.0 ** -8), 2.0 ** -8, 2.0 ** -8 * (1 + 2.0 ** -7), 0.5, 1.0, 127.0, 127.5, 128.0, 129.0)
            for s in (1, -1)] + [0.0, -0.0]
    z = torch.from_numpy(-np.abs(rng.standard_normal((len(tops), 3000)) * 2).astype(np.float32))
    z = z + torch.tensor(tops, dtype=torch.float32)[:, None]
    z[:, 77] = z[:, 1999] = torch.tensor(tops, dtype=torch.float32)
    each(z.to(DT[dtype]).cuda(), rng)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("keep", [2, 30, 400, 3000])
def test_masked_rows_at_high_temperatures(keep, dtype):
    rng = np.random.default_rng([42, keep])
    z = torch.full((12, 20000), -math.inf)
    for r in range(12):
        at = torch.from_numpy(rng.choice(20000, keep, replace=False))
        z[r, at] = torch.from_numpy((rng.standard_normal(keep) * 2 + (r - 6)).astype(np.float32))
    z = z.to(DT[dtype]).cuda()
    u = rng.random(12)
    for temperature in (0.5, 3.0, 10.0, 1e3, 1e30):
        check(z, u, temperature=temperature)
        check(z, u, temperature=temperature, top_k=keep // 2 + 1, top_p=0.9, min_p=0.01)
    token, _, _ = draw(z, np.full(12, 1 - 2.0 ** -24), temperature=1e30)
    assert torch.isfinite(z[torch.arange(12), torch.from_numpy(token).long()]).all()
    # masked with a lowest finite number, which is drawn as any other
    low = torch.where(torch.isinf(z), torch.finfo(DT[dtype]).min, z.float()).to(z.dtype)
    check(low, u, temperature=10.0)
    check(low, u, temperature=float(np.float32(3e38)), top_k=keep + 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_low_temperatures_next_to_zero(dtype):
    rng = np.random.default_rng(43)
    z = torch.from_numpy((rng.standard_normal((8, 4000)) * 2.0 ** -9).astype(np.float32)).to(DT[dtype]).cuda()
    u = rng.random(8)
    for offset in (0.0, 2.0 ** -8, -2.0 ** -8, 0.5, -0.5):
        y = (z.float() + offset).to(z.dtype)
        for temperature in (1e-5, 3e-4, 2e-3, 4e-3, 0.02, 1.0):
            check(y, u, temperature=temperature)
            check(y, u, temperature=temperature, top_p=0.7, top_k=1500, min_p=1e-3)
