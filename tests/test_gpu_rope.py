"""Rotary positions on the GPU against the rotation in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2607_22634_amd as P
import step_ref as S

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a rounding step, relative


def tensor(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DT[dtype]).cuda()


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def bound(y, size, magnitude, dtype):
    """Errors in units of 2^-24: the angle's conversion to fp32 and its scaling
    4 (times at most 0.6, the largest |x cos x| or |x sin x| up to an eighth of
    a turn), either series 3, the magnitude 1, the product with a value 1 and
    the sum of the products 1 are under 10 times |a| + |b|; half a step of the
    output on top of what is stored."""
    inner = 10 * 2.0 ** -24 * size
    return inner + HALF[dtype] * (np.abs(y) + inner)


def check(x, pos, plan, freq, interleaved, magnitude, dtype, out):
    y, size = S.rotate(x.double().cpu().numpy(), pos, freq, interleaved, magnitude)
    got = out.double().cpu().numpy()
    turned = np.zeros(x.shape[-1], dtype=bool)
    turned[:2 * len(freq)] = True
    assert (np.abs(got - y) <= bound(y, size, magnitude, dtype))[..., turned].all()
    assert (got == y)[..., ~turned].all()  # (as they were)


FAR = [0, 1, 2, 7, 100, 8191, 131071, 1000003, 2 ** 31 - 1, -1, -5, -2 ** 31]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,dim,rot", [(40, 128, 128), (1, 8, 8), (3, 8, 2), (7, 16, 12), (5, 64, 64), (9, 64, 32),
                                           (2, 72, 72), (13, 80, 80), (4, 96, 90), (6, 128, 64), (3, 128, 22),
                                           (2, 192, 192), (65, 192, 64), (5, 256, 256), (1, 256, 130)])
def test_rotation(heads, dim, rot, interleaved, dtype):
    rng = np.random.default_rng([1, heads, dim, rot])
    pos = np.array(FAR + rng.integers(0, 200000, 9).tolist())
    x = tensor(rng, (len(pos), heads, dim), dtype)
    plan = P.rope_plan(rot, base=500000.0, interleaved=interleaved)
    before = x.clone()
    out = P.presto_rope(x, ints(pos), plan)
    check(before, pos, plan, S.frequencies(rot, 500000.0), interleaved, 1.0, dtype, out)
    assert torch.equal(x, before)
    same = x.clone()
    assert P.presto_rope(same, ints(pos), plan, out=same) is same
    assert torch.equal(same, out)


@pytest.mark.parametrize("kw", [dict(factor=4.0), dict(factor=8.0, original=8192.0, low=1.0, high=4.0, ramp="turns"),
                                dict(factor=16.0, original=4096.0, low=1.0, high=32.0, ramp="log", base=1e6)])
@pytest.mark.parametrize("magnitude", [1.0, 1.277, -0.5, 0.0])
def test_scaled_frequencies(kw, magnitude):
    rng = np.random.default_rng(2)
    pos = np.array([0, 5, 77, 4095, 4096, 65535, 10 ** 6])
    x = tensor(rng, (len(pos), 6, 128), "f32")
    plan = P.rope_plan(128, magnitude=magnitude, **kw)
    m = float(np.float32(magnitude))
    y, size = S.rotate(x.double().cpu().numpy(), pos, S.frequencies(128, **kw), False, m)
    got = P.presto_rope(x, ints(pos), plan).double().cpu().numpy()
    assert (np.abs(got - y) <= bound(y, np.abs(size), m, "f32") + 1e-300).all()


def test_given_frequencies():
    rng = np.random.default_rng(3)
    f = np.concatenate([10.0 ** rng.uniform(-9, 5, 15), [0.0]])
    x, pos = tensor(rng, (50, 3, 32), "f32"), rng.integers(-1000, 1000, 50)
    plan = P.rope_plan(32, frequencies=f)
    # angles of up to 1e8 hold 2^-53 of themselves in the reference
    y, size = S.rotate(x.double().cpu().numpy(), pos, f)
    got = P.presto_rope(x, ints(pos), plan).double().cpu().numpy()
    assert (np.abs(got - y) <= bound(y, size, 1.0, "f32") + 1e8 * 2.0 ** -52 * size).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 2, 33, 528, 5000])
def test_queries_and_keys_in_place_in_a_projection(rows, dtype):
    """The front heads of wider rows, in place: the rest stays as it was."""
    rng = np.random.default_rng([4, rows])
    wide = tensor(rng, (rows, 12, 64), dtype)
    before = wide.clone()
    pos = rng.integers(0, 9000, rows)
    plan = P.rope_plan(64)
    x = wide[:, :9]
    P.presto_rope(x, ints(pos), plan, out=x)
    check(before[:, :9], pos, plan, S.frequencies(64), False, 1.0, dtype, wide[:, :9])
    assert torch.equal(wide[:, 9:], before[:, 9:])
    other = torch.full((rows, 11, 64), 7.0, dtype=wide.dtype, device="cuda")
    P.presto_rope(before[:, :9], ints(pos), plan, out=other[:, 1:10])
    assert torch.equal(other[:, 1:10], wide[:, :9])
    assert (other[:, 0] == 7).all() and (other[:, 10] == 7).all()


def test_a_position_undoes_its_opposite():
    rng = np.random.default_rng(5)
    x, pos = tensor(rng, (100, 4, 128), "f32"), rng.integers(0, 10 ** 6, 100)
    plan = P.rope_plan(128, interleaved=True)
    back = P.presto_rope(P.presto_rope(x, ints(pos), plan), ints(-pos), plan)
    _, size = S.rotate(x.double().cpu().numpy(), pos, S.frequencies(128), True)
    # two rotations of the same angle's sine and cosine: each off by at most
    # 11 * 2^-24 of |a| + |b|, which the first leaves at most sqrt(2) larger
    assert (np.abs((back - x).double().cpu().numpy()) <= (1 + math.sqrt(2)) * 11 * 2.0 ** -24 * size).all()


def test_values_that_are_not_finite_reach_their_pair_only():
    x = torch.ones(1, 2, 64, device="cuda")
    x[0, 0, 3], x[0, 1, 40] = math.nan, math.inf
    out = P.presto_rope(x, ints([5]), P.rope_plan(32))
    bad = ~torch.isfinite(out[0])
    assert bad[0].nonzero().flatten().tolist() == [3, 19]
    assert bad[1].nonzero().flatten().tolist() == [40] and out[0, 1, 40] == math.inf  # (behind the rotated part)
    out = P.presto_rope(x, ints([5]), P.rope_plan(64, interleaved=True))
    bad = ~torch.isfinite(out[0])
    assert bad[0].nonzero().flatten().tolist() == [2, 3] and bad[1].nonzero().flatten().tolist() == [40, 41]


def test_no_rows_and_refusals():
    plan = P.rope_plan(64)
    assert P.presto_rope(torch.empty(0, 4, 64, device="cuda"), ints([]), plan).shape == (0, 4, 64)
    x, pos = torch.zeros(3, 4, 64, device="cuda"), ints([1, 2, 3])
    with pytest.raises(P.PrestoError):
        P.presto_rope(torch.zeros(3, 4, 60, device="cuda"), pos, plan)
    with pytest.raises(P.PrestoError):
        P.presto_rope(torch.zeros(3, 4, 32, device="cuda"), pos, plan)  # shorter than what rotates
    with pytest.raises(ValueError):
        P.presto_rope(x, pos.long(), plan)
    with pytest.raises(ValueError):
        P.presto_rope(x, pos[:2], plan)
    with pytest.raises(ValueError):
        P.presto_rope(x, pos, P.rope_plan(64, device="cpu"))
    with pytest.raises(ValueError, match="overlap"):
        P.presto_rope(x[:1].expand(3, 4, 64), pos, plan)
    with pytest.raises(ValueError):
        P.presto_rope(x, pos, plan, out=x[:, :2])
    with pytest.raises(TypeError):
        P.presto_rope(x.half(), pos, plan)
