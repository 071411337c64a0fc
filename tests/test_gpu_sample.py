"""Draws of tokens on the GPU against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2607_22634_amd as P
import step_ref as S
from test_gpu_rope import DT

pytestmark = pytest.mark.gpu


def f32(x):
    return torch.tensor(np.asarray(x, dtype=np.float32), device="cuda")


def draw(z, u, **kw):
    """z [rows, V] tensor; settings as lists or one value for all rows"""
    rows, args = z.shape[0], {}
    for name, x in kw.items():
        x = np.broadcast_to(np.asarray(x), (rows,)).copy()
        args[name] = torch.tensor(x, dtype=torch.int32 if name == "top_k" else torch.float32, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    token, logprob = P.presto_sample(z, f32(u), flags=flags, **args)
    return token.cpu().numpy(), logprob.double().cpu().numpy(), flags.item()


def check(z, u, **kw):
    token, logprob, flags = draw(z, u, **kw)
    assert flags == 0
    zd = z.double().cpu().numpy()
    u = np.asarray(u, dtype=np.float32)
    for r in range(z.shape[0]):
        one = {n: np.broadcast_to(np.asarray(x), (z.shape[0],))[r] for n, x in kw.items()}
        one = {n: int(x) if n == "top_k" else float(np.float32(x)) for n, x in one.items()}
        want, log, near = S.sample(zd[r], float(u[r]), **one)
        assert token[r] in near, (r, token[r], want, one, u[r])
        if token[r] == want:
            # y ln 2 - log of the sum, in fp64; the sum to about 2^-40
            assert abs(logprob[r] - log) <= 2.0 ** -24 * abs(log) + 1e-9


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 63, 1000, 4097, 32000, 151936])
@pytest.mark.parametrize("sigma", [0.05, 1.0, 4.0])
def test_settings(vocab, sigma, dtype):
    rng = np.random.default_rng([20, vocab])
    rows = 24
    z = torch.from_numpy((rng.standard_normal((rows, vocab)) * sigma).astype(np.float32)).to(DT[dtype]).cuda()
    u = rng.random(rows)
    u[:3] = [0.0, 2.0 ** -30, 1 - 2.0 ** -24]
    kw = dict(temperature=rng.choice([0.0, 0.1, 0.7, 1.0, 1.5, 30.0], rows), top_k=rng.choice([0, 1, 2, 5, 40, 1000, vocab, 1 << 30], rows),
              top_p=rng.choice([1.0, 0.0, 1e-6, 0.3, 0.9, 0.95, 0.999, 2.0], rows), min_p=rng.choice([0.0, 1e-4, 0.05, 0.3, 1.0], rows))
    check(z, u)
    check(z, u, temperature=kw["temperature"])
    check(z, u, top_k=kw["top_k"])
    check(z, u, top_p=kw["top_p"])
    check(z, u, min_p=kw["min_p"])
    check(z, u, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_each_token_of_a_small_row_gets_its_share(dtype):
    rng = np.random.default_rng(21)
    z = torch.from_numpy(rng.standard_normal(9).astype(np.float32)).to(DT[dtype]).cuda()
    n = 4000
    u = (np.arange(n) + 0.5) / n
    check(z.expand(n, 9).contiguous(), u)
    token, _, _ = draw(z.expand(n, 9).contiguous(), u, temperature=0.8)
    w = np.exp(z.double().cpu().numpy() / float(np.float32(0.8)))
    assert (np.abs(np.bincount(token, minlength=9) - n * w / w.sum()) <= 1.01).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5, 1024, 1025, 5000, 70001])
def test_equal_logits_go_by_id(vocab, dtype):
    z = torch.full((8, vocab), 1.5, dtype=DT[dtype], device="cuda")
    u = np.array([0.0, 0.1, 0.25, 0.5, 0.75, 0.9, 0.999, 1 - 2.0 ** -24], dtype=np.float32)
    token, logprob, _ = draw(z, u)
    assert (token == np.minimum(np.floor(u.astype(np.float64) * vocab), vocab - 1)).all()
    token, _, _ = draw(z, u, top_k=4)
    assert (token == np.floor(u.astype(np.float64) * min(4, vocab))).all()
    token, _, _ = draw(z, u, top_p=0.5)
    n = math.ceil(vocab / 2)
    assert (token == np.minimum(np.floor(u.astype(np.float64) * n), n - 1)).all()
    token, _, _ = draw(z, u, min_p=1.0)
    assert (token == np.minimum(np.floor(u.astype(np.float64) * vocab), vocab - 1)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_values_many_ties(dtype):
    rng = np.random.default_rng(22)
    z = torch.from_numpy(rng.choice([-3.0, -0.0, 0.0, 0.5, 2.0], (16, 20000)).astype(np.float32)).to(DT[dtype]).cuda()
    check(z, rng.random(16))
    check(z, rng.random(16), top_k=7001, top_p=0.97)
    check(z, rng.random(16), min_p=0.1, temperature=2.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1e-3, 1e3, 1e30])
def test_wide_and_narrow_ranges(scale, dtype):
    """Logits of any size: all but equal, or one far above the others."""
    rng = np.random.default_rng(23)
    z = torch.from_numpy((rng.standard_normal((12, 3000)) * scale).astype(np.float32)).to(DT[dtype]).cuda()
    check(z, rng.random(12))
    check(z, rng.random(12), top_p=0.9)
    check(z, rng.random(12), temperature=max(scale, 1e-37), top_p=0.9, top_k=500)
    for offset in (-50.0, 20.0):
        check((z.float() + offset).to(z.dtype), rng.random(12), top_k=100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [6000, 100000])
def test_places_around_zero(vocab, dtype):
    """Draws, and each of the cuts, among logits within 2^-8 of 0, where bf16 values
    lie closer than elsewhere (and unaligned ends of a slice's pieces)."""
    rng = np.random.default_rng(28)
    wide = torch.from_numpy(rng.standard_normal((8, vocab + 3)).astype(np.float32)).to(DT[dtype]).cuda()
    z = wide[:, 3:]
    zd = np.sort(z.double().cpu().numpy(), -1)[:, ::-1]
    w = np.exp(zd - zd[:, :1])
    at = (zd > 0).sum(1) + rng.integers(-4, 5, 8)  # a place in the order next to 0
    share = np.array([w[r, :at[r]].sum() / w[r].sum() for r in range(8)])
    assert (np.abs(zd[np.arange(8), at]) < 2.0 ** -8).all()
    check(z, share)
    check(z, rng.random(8), top_k=at.astype(np.int32))
    check(z, np.full(8, 1 - 2.0 ** -24), top_k=at.astype(np.int32))
    check(z, np.full(8, 1 - 2.0 ** -24), top_p=share.astype(np.float32))
    check(z, np.full(8, 1 - 2.0 ** -24), min_p=w[np.arange(8), at].astype(np.float32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_logits(dtype):
    rng = np.random.default_rng(24)
    z = torch.from_numpy(rng.standard_normal((6, 5000)).astype(np.float32)).to(DT[dtype])
    for r, low in enumerate((-math.inf, torch.finfo(DT[dtype]).min, -1e30, -math.inf, -math.inf, -1e4)):
        keep = rng.choice(5000, 1 if r == 4 else 20, replace=False)
        mask = torch.ones(5000, dtype=torch.bool)
        mask[keep] = False
        z[r, mask] = low
    z = z.cuda()
    for u in (0.0, 0.37, 1 - 2.0 ** -24):
        check(z, np.full(6, u))
        check(z, np.full(6, u), top_k=50, top_p=0.95, min_p=0.01)
    # masked throughout with the lowest finite value: all tokens weigh the same
    z = torch.full((2, 700), torch.finfo(DT[dtype]).min, dtype=DT[dtype], device="cuda")
    assert draw(z, [0.0, 0.5])[0].tolist() == [0, 350]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_token(dtype):
    z = torch.zeros(5, 300, dtype=DT[dtype], device="cuda")
    z[0, 7], z[1, 299], z[2] = math.nan, math.inf, -math.inf
    z[3, 1:] = -math.inf
    for kw in (dict(), dict(temperature=0.0), dict(top_k=3)):
        token, logprob, flags = draw(z, [0.5] * 5, **kw)
        assert flags == P.PRESTO_FLAG_NAN_LOGITS
        assert token[:4].tolist() == [-1, -1, -1, 0] and np.isnan(logprob[:3]).all() and logprob[3] == 0
        assert token[4] >= 0


def test_settings_out_of_range():
    rng = np.random.default_rng(25)
    row = torch.from_numpy(rng.standard_normal(100).astype(np.float32)).cuda()
    z = row.expand(8, 100).contiguous()
    best = int(row.argmax())
    assert (draw(z, [0.9] * 8, temperature=[0.0, -1.0, math.nan, -0.0, -math.inf, 0.0, 0.0, 0.0])[0] == best).all()
    plain = draw(z, [0.9] * 8)[0]
    for kw in (dict(top_k=-3), dict(top_k=0), dict(top_p=math.nan), dict(top_p=math.inf), dict(min_p=math.nan), dict(min_p=-1.0)):
        assert (draw(z, [0.9] * 8, **kw)[0] == plain).all()
    assert (draw(z, [0.9] * 8, top_p=-1.0)[0] == best).all()
    assert (draw(z, [0.9] * 8, min_p=7.0)[0] == best).all()
    first, last = draw(z, [0.0] * 8)[0], draw(z, [1 - 2.0 ** -24] * 8)[0]
    assert (draw(z, [-1.0, math.nan, -math.inf, 0, 0, 0, 0, 0])[0] == first).all()
    assert (draw(z, [1.0, 2.0, math.inf, 1, 1, 1, 1, 1])[0] == last).all()
    inf = draw(z, np.linspace(0, 0.99, 8), temperature=math.inf)[0]  # all weigh the same
    order = np.argsort(-row.cpu().numpy(), kind="stable")
    assert (inf == order[np.floor(np.linspace(0, 0.99, 8).astype(np.float32).astype(np.float64) * 100).astype(int)]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_and_unaligned_rows(dtype):
    rng = np.random.default_rng(26)
    wide = torch.from_numpy(rng.standard_normal((9, 1031)).astype(np.float32)).to(DT[dtype]).cuda()
    u = rng.random(9)
    for lo, hi in ((0, 1031), (1, 1030), (3, 4), (5, 900), (7, 12)):
        view = wide[:, lo:hi]
        a, la, _ = draw(view, u, temperature=0.7)
        b, lb, _ = draw(view.contiguous(), u, temperature=0.7)
        assert (a == b).all() and (la == lb).all()
        check(view.contiguous(), u, temperature=0.7)


def test_many_rows_and_repeats():
    rng = np.random.default_rng(27)
    z = torch.from_numpy((rng.standard_normal((3000, 257)) * 3).astype(np.float32)).cuda()
    u = rng.random(3000)
    a, b = draw(z, u, top_p=0.9), draw(z, u, top_p=0.9)
    assert (a[0] == b[0]).all() and (a[1] == b[1]).all()
    check(z[:200], u[:200], top_p=0.9)


def test_binding_refuses():
    z, u = torch.zeros(2, 8, device="cuda"), torch.zeros(2, device="cuda")
    for kw in (dict(temperature=torch.ones(3, device="cuda")), dict(top_k=torch.ones(2, device="cuda")),
               dict(top_p=torch.ones(2)), dict(min_p=torch.ones(2, device="cuda").double()),
               dict(out=torch.zeros(2, device="cuda")), dict(logprob=torch.zeros(4, device="cuda")[::2])):
        with pytest.raises(ValueError):
            P.presto_sample(z, u, **kw)
    token, logprob = P.presto_sample(z[:0], u[:0])
    assert token.shape == (0,) and logprob.shape == (0,)
