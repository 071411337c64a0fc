"""Exponent bytes above those that are written (253, 254 and 255) make a group of
K or V read as NaN, whatever its codes, in every call that reads the cache."""
import numpy as np
import pytest
import torch

import paper_2607_22634_amd as P
import step_ref as S
from test_gpu_quant import Quant
from test_gpu_rope import ints, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("exponent", [253, 254, 255])
@pytest.mark.parametrize("new", [1, 9, 70])
@pytest.mark.parametrize("dim", [64, 128])
def test_high_exponents_read_as_nan(dim, new, exponent, dtype):
    """As in the test of groups that are not finite, with codes of 0 and of numbers."""
    rng = np.random.default_rng([31, dim, exponent])
    L, hkv, G = 90, 2, 3
    for pool, is_v in (("kh", False), ("vh", True)):
        for zero in (False, True):
            c = Quant(rng, [L, 80], 16, hkv, dim)
            q = tensor(rng, (2 * new, hkv * G, dim), dtype)
            args = dict(q_offsets=ints([0, new, 2 * new]), max_q=new)
            key, head, grp = L - new // 2 - 1, 1, 1
            page, row = c.where(0, [key])
            block = getattr(c, pool)[page[0], head, row[0] // 16]
            code_at, exp_at = (x[row[0] % 16, 32 * grp:32 * grp + 32] for x in S.offsets(dim, is_v))
            if zero:
                block[code_at] = 0
            c.upload()
            good = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, **args)
            assert torch.isfinite(good).all()
            block[exp_at] = exponent
            c.upload()
            out = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, **args)
            bad = torch.zeros_like(out, dtype=torch.bool)
            sees = torch.arange(L - new, L, device="cuda") >= key
            dims = slice(32 * grp, 32 * grp + 32) if is_v else slice(0, dim)
            bad[:new, head * G:(head + 1) * G, dims] = sees[:, None, None]
            assert torch.equal(torch.isnan(out), bad)
            assert torch.equal(out[~bad], good[~bad])
            back = P.presto_read_kv(c.k, c.v, c.table, ints([0, 0]), c.ctx, ints([0, L, L + 80]), L, rows=L + 80)
            nan = [torch.isnan(t).nonzero() for t in back]
            assert len(nan[not is_v]) == 0 and nan[is_v].tolist() == [[key, head, 32 * grp + i] for i in range(32)]
