"""4-bit attention whose contexts are cut into pieces that a second kernel joins:
new tokens, windows, sinks, groups that are not finite and batches of many
sequences; and pieces so long that a wave looks pages up more than once."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2607_22634_amd as P
import step_ref as S
from paper_2607_22634_amd._lib import lib
from paper_2607_22634_amd._paged import _DT
from paper_2607_22634_amd._step import _quant_desc
from test_gpu_quant import Quant
from test_gpu_rope import ints, tensor

pytestmark = pytest.mark.gpu


def reference(q, k, v, pos0, window, sinks, dtype, short):
    """All of test_gpu_quant.tight at once: q [n, hq, d], k, v [L, hkv, d] (fp64)."""
    n, hq, d = q.shape
    L, hkv = k.shape[:2]
    q, k, v = (torch.from_numpy(np.ascontiguousarray(x)) for x in (q, k, v))
    k, v = (x.repeat_interleave(hq // hkv, 1).transpose(0, 1).contiguous() for x in (k, v))  # [hq, L, d]
    q = q.transpose(0, 1).contiguous()
    pos, j = pos0 + torch.arange(n)[:, None], torch.arange(L)[None]
    ok = j <= pos
    if window:
        ok &= (j > pos - window) | (j < sinks)
    scale = d ** -0.5
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
    s = s.masked_fill(~ok, -torch.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-1e300))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
    o, A = torch.matmul(p, v), torch.matmul(p, v.abs())
    mag = (torch.matmul(q.abs(), k.abs().transpose(1, 2).contiguous()) * scale).masked_fill(~ok, 0).amax(-1, keepdim=True)
    count = ok.sum(-1)[None, :, None]
    half = 2.0 ** -24
    e = 2 * (d + 3) * half * mag + 2.0 ** -18 + (count + 64) * half
    bound = e * (1 + 2 * e) * (A + o.abs()) + half * (o.abs() * (1 + 2 * e) + 2 * e * A) + 1e-30
    if dtype == "f32":
        bound = bound + 1.01 * 2.0 ** -23 * (A + o.abs()) + half * o.abs()
    else:
        bound = bound + 1.01 * (2.0 ** -16 if short else 2.0 ** -8) * (A + o.abs())
        bound = bound + 2.0 ** -8 * (o.abs() + bound)
    return o.transpose(0, 1).numpy(), bound.transpose(0, 1).numpy()


def pieces(q, c, ragged=True, max_q=1, max_ctx=None, window=0, sinks=0, total_ctx=0):
    """whether a call is cut (only then it needs a workspace)"""
    desc = _quant_desc(q, c.k, c.v, c.table, c.table.shape[0], max_q, max_ctx, None, window, sinks, total_ctx)
    return lib().presto_quant_attention_workspace(ctypes.byref(desc), _DT[q.dtype], ragged) > 0


CHUNKS = {  # context and new tokens of each sequence; the last pieces of rows that lie
    # side by side end at, before and behind a border between pieces
    "two": ([3100, 3391], [2, 2]),
    "nine": ([3223, 3136], [9, 5]),
    "forty": ([3400, 3105, 700], [40, 1, 33]),
    "hundreds": ([3400, 3333], [130, 61]),
    "more than cached": ([3100, 50], [64, 130]),
    "border": ([3584 + 70, 3584 + 5], [130, 130]),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,dim,page", [(8, 2, 128, 64), (3, 1, 64, 16)])
@pytest.mark.parametrize("chunk", CHUNKS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (900, 40), (1500, 200), (2900, 70)])
def test_new_tokens_over_pieces(window, sinks, chunk, hq, hkv, dim, page, dtype):
    ctx, new = CHUNKS[chunk]
    rng = np.random.default_rng([50, dim, sum(ctx), window])
    c = Quant(rng, ctx, page, hkv, dim, sigma=1.5)
    offs = 1 + np.concatenate([[0], np.cumsum(new)])
    q = tensor(rng, (int(offs[-1]) + 2, hq, dim), dtype)
    most = max(new)
    for kw in (dict(), dict(max_ctx=max(ctx), total_ctx=sum(ctx))):
        assert pieces(q, c, max_q=most, window=window, sinks=sinks, **kw)
        out = torch.full_like(q, 7.0)
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        args = dict(q_offsets=ints(offs), max_q=most, window=window, sinks=sinks, flags=flags, **kw)
        P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, out=out, **args)
        assert flags.item() == 0
        assert torch.equal(out, P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, out=torch.full_like(q, 7.0), **args))
        assert (out[:1] == 7).all() and (out[offs[-1]:] == 7).all()
        got, qd = out.double().cpu().numpy(), q.double().cpu().numpy()
        for b, (n, L) in enumerate(zip(new, ctx)):
            s = slice(offs[b], offs[b] + n)
            want, bound = reference(qd[s], *c.rows(b), L - n, window, sinks, dtype, most * hq // hkv < 128)
            err = np.abs(got[s] - want)
            assert (err <= bound).all(), (b, (err / bound).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 9, 130])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1200, 50)])
def test_groups_that_are_not_finite_through_the_pieces(window, sinks, new, dim, dtype):
    rng = np.random.default_rng([51, dim, new])
    L, hkv, G = 3300, 2, 3
    c = Quant(rng, [L, 2000], 64, hkv, dim)
    q = tensor(rng, (2 * new, hkv * G, dim), dtype)
    args = dict(q_offsets=ints([0, new, 2 * new]), max_q=new, window=window, sinks=sinks)
    assert pieces(q, c, max_q=new, window=window, sinks=sinks)
    good = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, **args)
    assert torch.isfinite(good).all()
    qd = q.double().cpu().numpy()
    want, bound = (np.concatenate(x) for x in zip(*(
        reference(qd[b * new:(b + 1) * new], *c.rows(b), c.ctx_h[b] - new, window, sinks, dtype, new * G < 128)
        for b in range(2))))
    head, grp = 1, 1
    for key in (3, 1700, L - 1200 + 40, L - new // 2 - 1):
        for pool, is_v in (("kh", False), ("vh", True)):
            page, row = c.where(0, [key])
            block = getattr(c, pool)[page[0], head, row[0] // 16]
            at = S.offsets(dim, is_v)[1][row[0] % 16, 32 * grp]
            old = block[at]
            block[at] = 255
            c.upload()
            out = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, **args)
            block[at] = old
            pos = torch.arange(L - new, L, device="cuda")
            sees = (pos >= key) & ((window == 0) | (key > pos - window) | (key < sinks))
            bad = torch.zeros_like(out, dtype=torch.bool)
            dims = slice(32 * grp, 32 * grp + 32) if is_v else slice(0, dim)
            bad[:new, head * G:(head + 1) * G, dims] = sees[:, None, None]
            assert torch.equal(torch.isnan(out), bad), (key, is_v)
            # (a NaN score makes its wave choose the references of all its rows anew,
            # which rounds the others differently)
            if is_v:
                assert torch.equal(out[~bad], good[~bad]), key
            else:
                rest = ~bad.cpu().numpy()
                assert (np.abs(out.double().cpu().numpy() - want) <= bound)[rest].all(), key


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,longest", [(65, 900), (130, 1500), (256, 900), (300, 1500)])
@pytest.mark.parametrize("hint", [False, True])
def test_many_sequences_in_pieces(hint, batch, longest, dtype):
    """Pieces are counted over 64 sequences at a time, up to 256 of them."""
    rng = np.random.default_rng([52, batch])
    lens = rng.integers(0, longest // 3, batch)
    lens[[0, 5, batch // 2, batch - 2]] = [longest, 0, longest - 33, longest - 1]
    lens[batch - 1] = 0 if batch % 2 else 700
    c = Quant(rng, lens.tolist(), 64, 1, 64)
    q = tensor(rng, (batch, 4, 64), dtype)
    kw = dict(max_ctx=longest, total_ctx=int(lens.sum())) if hint else {}
    if dtype == "bf16" or batch < 257 or hint:
        assert pieces(q, c, False, **kw)
    out = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, **kw)
    assert torch.equal(out, P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, **kw))
    got, qd = out.double().cpu().numpy(), q.double().cpu().numpy()
    for b in range(batch):
        if lens[b] == 0:
            assert (got[b] == 0).all()
            continue
        want, bound = reference(qd[b:b + 1], *c.rows(b), int(lens[b]) - 1, 0, 0, dtype, True)
        assert (np.abs(got[b:b + 1] - want) <= bound).all(), b


def repeated(c, times):
    """c's one sequence `times` over: its table again and again"""
    c.table_h = np.tile(c.table_h, (1, times))
    c.ctx_h = [c.ctx_h[0] * times]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 3, 130])
@pytest.mark.parametrize("window,sinks", [(0, 0), (4900, 100)])
def test_waves_of_many_tiles(window, sinks, new, dtype):
    """So many heads and sequences that contexts are not cut: 9000 keys are 282
    tiles, 71 and 141 to a wave, which looks up the pages of 32 at a time.  (The
    pages are few and repeat.)"""
    rng = np.random.default_rng([53, new])
    hkv, dim, batch = 64, 64, 16 if new < 130 else 4
    c = Quant(rng, [512], 32, hkv, dim, spare=5)
    repeated(c, 18)
    n_keys = 9000
    table = np.full((batch, c.table_h.shape[1]), -1)
    table[0], table[1:, 0] = c.table_h[0], c.table_h[0, 3]
    c.table, c.ctx = ints(table), ints([n_keys] + [7] * (batch - 1))
    offs = np.concatenate([[0], [new], new + 1 + np.arange(batch - 1)])
    q = tensor(rng, (int(offs[-1]), hkv, dim), dtype)
    kw = dict(max_ctx=n_keys, window=window, sinks=sinks, max_q=new)
    if window == 0:
        assert not pieces(q, c, **kw)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, q_offsets=ints(offs), flags=flags, **kw)
    assert flags.item() == 0
    heads = [0, 17, 63]
    at = c.where(0, range(n_keys))
    k, v = (S.read(np.ascontiguousarray(x[:, heads]), is_v, *at) for x, is_v in ((c.kh, False), (c.vh, True)))
    got, qd = (t[:new, heads].double().cpu().numpy() for t in (out, q))
    want, bound = reference(qd, k, v, n_keys - new, window, sinks, dtype, new < 128)
    err = np.abs(got - want)
    assert (err <= bound).all(), (err / bound).max()
    # a page that is missing behind the first lookup, and one that nothing sees
    table[0, 9000 // 32 - 40] = -1
    flags.zero_()
    P.presto_quant_attention(q, c.k, c.v, ints(table), c.ctx, q_offsets=ints(offs), flags=flags, **kw)
    assert flags.item() == P.PRESTO_FLAG_BAD_PAGE


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_offsets_leave_other_rows_as_they_should_be(dtype):
    """Sequences whose offsets cannot be are left out, the others computed: which
    rows are written, and with what."""
    rng = np.random.default_rng(54)
    c = Quant(rng, [70, 75, 80, 90], 16, 1, 64)
    q = tensor(rng, (4, 2, 64), dtype)
    qd = q.double().cpu().numpy()
    # offsets: {row: (sequence, position)}; rows that two sequences claim are not looked at
    for offs, rows, shared in (([0, 3, 2, 4, 4], {0: (0, 67), 1: (0, 68), 3: (2, 79)}, [2]),
                               ([0, 1, 9, 9, 9], {0: (0, 69)}, []),
                               ([-1, 1, 2, 3, 4], {1: (1, 74), 2: (2, 79), 3: (3, 89)}, []),
                               ([0, 4, 4, 4, 4], {0: (0, 66), 1: (0, 67), 2: (0, 68)}, []),
                               ([0, 1, 3, 3, 2 ** 31 - 1], {0: (0, 69), 1: (1, 73), 2: (1, 74)}, []),
                               ([0, -2 ** 31, 1, 3, 4], {1: (2, 78), 2: (2, 79), 3: (3, 89)}, [])):
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 7.0)
        P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, q_offsets=ints(offs), max_q=3, out=out, flags=flags)
        assert flags.item() == P.PRESTO_FLAG_BAD_SEQ
        got = out.double().cpu().numpy()
        for r in range(4):
            if r in rows:
                b, pos = rows[r]
                want, bound = reference(qd[r:r + 1], *c.rows(b), pos, 0, 0, dtype, True)
                assert (np.abs(got[r:r + 1] - want) <= bound).all(), (offs, r)
            elif r not in shared:
                assert (got[r] == 7).all(), (offs, r)
