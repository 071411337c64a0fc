"""Rows that hold a NaN or +inf anywhere draw nothing, wherever in a row, or in
the stretch of it that a workgroup counts, the value lies."""
import numpy as np
import pytest
import torch

import paper_2607_22634_amd as P
from test_gpu_rope import DT
from test_gpu_sample import f32

pytestmark = pytest.mark.gpu

# quiet NaNs of both signs, NaNs with the least payload, +inf
BAD = {"bf16": [0x7fc0, 0xffc0, 0x7f81, 0xff81, 0x7f80],
       "f32": [0x7fc00000, 0xffc00000, 0x7f800001, 0xff800001, 0x7f800000]}
MINUS_INF = {"bf16": 0xff80, "f32": 0xff800000}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,skip", [(1025, 0), (1025, 3), (4097, 5), (4104, 0), (20001, 0), (20001, 1), (32000, 0), (70001, 7)])
@pytest.mark.parametrize("masked", [False, True])
def test_what_is_not_finite_is_seen_at_every_end(vocab, skip, masked, dtype):
    """One bad value per row, in turn at each of the first and last eight places of
    every 64 (stretches begin at multiples of 64), among numbers or among -inf;
    row starts that are 16-byte aligned and that are not."""
    rng = np.random.default_rng([30, vocab, skip])
    rows = 65
    wide = torch.from_numpy(rng.standard_normal((rows, vocab + skip)).astype(np.float32)).to(DT[dtype]).cuda()
    z = wide[:, skip:]
    bits = z.view(torch.int16 if dtype == "bf16" else torch.int32)
    kind = np.uint16 if dtype == "bf16" else np.uint32

    def pattern(x):
        return torch.from_numpy(np.asarray(x, dtype=kind).view(np.int16 if dtype == "bf16" else np.int32)).cuda()

    if masked:  # all but the last row, and every row's first 40 and a third of the others
        hide = torch.rand(rows, vocab, device="cuda") < 2 / 3
        hide[:, :40] = False
        hide[-1] = False
        bits[hide] = pattern([MINUS_INF[dtype]])[0]
    i = np.arange(vocab)
    places = i[(i % 64 < 8) | (i % 64 >= 56) | (i >= vocab - 8)]
    u = f32(rng.random(rows))
    row = torch.arange(rows - 1, device="cuda")
    for at in range(0, len(places), rows - 1):
        where = torch.from_numpy(np.resize(places[at:at + rows - 1], rows - 1)).cuda()
        old = bits[row, where]
        bits[row, where] = pattern(np.resize(np.roll(BAD[dtype], at // (rows - 1)), rows - 1))
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        token, logprob = P.presto_sample(z, u, flags=flags)
        assert flags.item() == P.PRESTO_FLAG_NAN_LOGITS
        missed = (token[:-1] != -1) | ~torch.isnan(logprob[:-1])
        assert not missed.any(), [(int(r), int(where[r])) for r in missed.nonzero()[:4]]
        assert token[-1] >= 0 and torch.isfinite(logprob[-1])
        bits[row, where] = old
    flags.zero_()
    token, _ = P.presto_sample(z, u, flags=flags)
    assert flags.item() == 0 and (token >= 0).all()
