"""The 4-bit paged cache on the GPU: what the append stores, the way back, and
attention over it, against references in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2607_22634_amd as P
import step_ref as S
from test_gpu_rope import DT, bound as rope_bound, ints, tensor

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Quant:
    """A 4-bit cache of sequences with lengths ctx, in shuffled pages; whatever is
    not a cached row is random bytes, exponents of 255 among them."""

    def __init__(self, rng, ctx, page, hkv, dim, spare=3, sigma=1.0):
        self.page, self.hkv, self.dim, self.ctx_h = page, hkv, dim, list(ctx)
        cols = max([1] + [-(-c // page) for c in ctx])
        need = sum(-(-c // page) for c in ctx)
        order = rng.permutation(need + spare)
        self.table_h = np.full((len(ctx), cols), -1, dtype=np.int64)
        at = 0
        for b, c in enumerate(ctx):
            for x in range(-(-c // page)):
                self.table_h[b, x] = order[at]
                at += 1
        shape = (need + spare, hkv, page // 16, 17 * dim // 2)
        self.kh, self.vh = (rng.integers(0, 256, shape, dtype=np.uint8) for _ in range(2))
        self.kh[..., 8 * dim:][rng.random(shape[:3] + (dim // 2,)) < 0.1] = 255
        self.vh[..., 8 * dim:][rng.random(shape[:3] + (dim // 2,)) < 0.1] = 255
        for b, c in enumerate(ctx):
            for pool, is_v in ((self.kh, False), (self.vh, True)):
                S.write(pool, is_v, *self.where(b, range(c)), *S.encode(rng.standard_normal((c, hkv, dim)) * sigma))
        self.upload()

    def upload(self):
        self.k, self.v, self.table = dev(self.kh), dev(self.vh), ints(self.table_h)
        self.ctx = ints(self.ctx_h)

    def where(self, b, positions):
        p = np.asarray(list(positions), dtype=np.int64)
        return self.table_h[b, p // self.page], p % self.page

    def rows(self, b):
        """the cached K and V (fp64) [ctx, hkv, dim]"""
        at = self.where(b, range(self.ctx_h[b]))
        return S.read(self.kh, False, *at), S.read(self.vh, True, *at)


def tight(q, k, v, pos0, window, sinks, dtype, short=True):
    """The 64-bit output and a bound: as paged_ref.attention's for fp32
    arithmetic, probabilities held to two bf16 (2^-16, inputs of bf16; one, 2^-8,
    in long prompts) or three (2^-24), then half a step of the output."""
    want, inner = R.attention(q, k, v, pos0, window, sinks, None, "f32")
    A, _ = R.attention(q, k, np.abs(v), pos0, window, sinks, None, "f32")
    if dtype == "f32":
        return want, inner + 1.01 * 2.0 ** -23 * (A + np.abs(want)) + 2.0 ** -24 * np.abs(want)
    inner = inner + 1.01 * (2.0 ** -16 if short else 2.0 ** -8) * (A + np.abs(want))
    return want, inner + 2.0 ** -8 * (np.abs(want) + inner)


# ---------------------------------------------------------------------------
# the append and the way back

def books(rng, past, new, page, extra=2):
    cols = max(1, max(-(-(p + n) // page) for p, n in zip(past, new)))
    need = sum(-(-(p + n) // page) for p, n in zip(past, new))
    order, at = rng.permutation(need + extra), 0
    table = np.full((len(past), cols), -1, dtype=np.int64)
    for b, (p, n) in enumerate(zip(past, new)):
        for x in range(-(-(p + n) // page)):
            table[b, x] = order[at]
            at += 1
    return table, need + extra


PAST, NEW = [0, 3, 15, 16, 100, 31, 0], [1, 40, 1, 17, 0, 2, 33]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,hkv,hq,page", [(64, 1, 3, 16), (64, 8, 8, 64), (128, 1, 1, 32), (128, 8, 32, 16), (128, 5, 10, 128)])
@pytest.mark.parametrize("rot,interleaved", [(0, False), (None, False), (None, True), (40, False), (22, True)])
@pytest.mark.parametrize("quant", [True, False])
def test_append(dim, hkv, hq, page, rot, interleaved, dtype, quant):
    rot = dim if rot is None else rot
    rng = np.random.default_rng([6, dim, hkv, rot])
    table, pages = books(rng, PAST, NEW, page)
    offs = np.concatenate([[0], np.cumsum(NEW)])
    rows = int(offs[-1]) + 3  # rows behind the last sequence
    wide = tensor(rng, (rows, hq + 2 * hkv, dim), dtype)
    q, k, v = wide[:, :hq], wide[:, hq:hq + hkv], wide[:, hq + hkv:]
    if quant:
        k_pool, v_pool = (dev(rng.integers(0, 256, (pages, hkv, page // 16, 17 * dim // 2), dtype=np.uint8)) for _ in range(2))
    else:
        k_pool, v_pool = tensor(rng, (pages, page, hkv, dim), dtype), tensor(rng, (pages, page, hkv, dim), dtype)
    k0, v0 = k_pool.clone(), v_pool.clone()
    plan = P.rope_plan(rot, base=1e4, interleaved=interleaved) if rot else None
    freq = S.frequencies(rot, 1e4)
    ctx, ctx_new = ints(PAST), ints(np.add(PAST, NEW))
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((rows, hq, dim), 7.0, dtype=q.dtype, device="cuda")
    P.presto_append_rope(plan, q, k, v, ints(offs), max(NEW), k_pool, v_pool, ints(table), ctx, ctx_new, out=out, flags=flags)
    assert flags.item() == 0
    pos = np.concatenate([p + np.arange(n) for p, n in zip(PAST, NEW)])
    seq = np.repeat(np.arange(len(NEW)), NEW)
    n = len(pos)
    qd, kd, vd = (t[:n].double().cpu().numpy() for t in (q, k, v))
    want, size = S.rotate(qd, pos, freq, interleaved)
    got = out[:n].double().cpu().numpy()
    if rot:
        assert (np.abs(got - want) <= rope_bound(want, size, 1.0, dtype)).all()
    else:
        assert (got == want).all()
    assert (out[n:] == 7).all()
    at, row = table[seq, pos // page], pos % page
    kt, size = S.rotate(kd, pos, freq, interleaved)
    if not quant:
        kp = k_pool.double().cpu().numpy()[at, row]
        assert (np.abs(kp - kt) <= (rope_bound(kt, size, 1.0, dtype) if rot else 0)).all()
        assert torch.equal(v_pool[at, row], v[:n])
        k_pool[at, row], v_pool[at, row] = k0[at, row], v0[at, row]
        assert torch.equal(k_pool, k0) and torch.equal(v_pool, v0)  # nothing else was written
        return
    kp, vp = k_pool.cpu().numpy(), v_pool.cpu().numpy()
    # values without a rotation are exact, and so are their codes
    code, e = S.encode(vd)
    mine = v0.cpu().numpy()
    S.write(mine, True, at, row, code, e)
    assert (mine == vp).all()
    mine = k0.cpu().numpy()
    S.write(mine, False, at, row, *S.encode(kt))
    held, want = S.read(kp, False, at, row), S.held(kt)
    # where a rotated key is within its error of a border it may lie on either
    # side: of codes, or of exponents
    err = 10 * 2.0 ** -24 * size
    lo, hi = S.held(kt - err), S.held(kt + err)
    top = np.abs(kt).reshape(*kt.shape[:-1], -1, 32)
    e_err = err.reshape(top.shape).max(-1)
    near = S.exponents(np.repeat((top.max(-1) + e_err)[..., None], 32, -1).reshape(kt.shape)) != \
        S.exponents(np.repeat((top.max(-1) - e_err)[..., None], 32, -1).reshape(kt.shape))
    near = np.repeat(near[..., None], 32, -1).reshape(kt.shape)
    assert near.mean() < 1e-3
    assert ((held >= np.minimum(lo, hi)) & (held <= np.maximum(lo, hi)))[~near].all()
    assert (held == want)[~near].mean() > 0.999
    S.write(kp, False, at, row, *S.encode(kt))
    S.write(mine, False, at, row, *S.encode(kt))
    assert (kp == mine).all()  # nothing else was written
    # the way back
    for t in ([torch.bfloat16, torch.float32] if dtype == "bf16" else [torch.float32]):
        k2, v2 = P.presto_read_kv(k_pool, v_pool, ints(table), ctx, ctx_new, ints(offs), max(NEW), rows=rows, dtype=t)
        assert (k2[:n].double().cpu().numpy() == held).all() and (k2[n:] == 0).all()
        assert (v2[:n].double().cpu().numpy() == S.held(vd)).all() and (v2[n:] == 0).all()


def test_keys_on_a_border_turn_to_the_right_side():
    """bf16 keys half-way between two codes, at positions whose small angles move
    them by less than fp32 holds: the side that the exact rotation leaves them on."""
    rng = np.random.default_rng(7)
    dim, n = 128, 64
    k = np.tile(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]), (n, 1, 16)) * rng.choice([-1, 1], (n, 1, dim))
    kt = torch.from_numpy(k).to(torch.bfloat16).cuda()
    freq = 2.0 ** -rng.integers(26, 31, dim // 2).astype(np.float64)
    plan = P.rope_plan(dim, frequencies=freq)
    pool = [P.quant_pages(4, 16, 1, dim).zero_() for _ in range(2)]
    table = ints([[2, 0, 1, 3]])
    P.presto_append_rope(plan, None, kt, kt, ints([0, n]), n, *pool, table, ints([0]), ints([n]))
    got, _ = P.presto_read_kv(*pool, table, ints([0]), ints([n]), ints([0, n]), n, rows=n)
    want = S.held(S.rotate(k, np.arange(n), freq)[0])
    assert (got.double().cpu().numpy() == want).all()
    assert (S.held(k) != want).mean() > 0.1  # (the angles matter)


def test_keys_next_to_a_border_keep_their_side():
    """fp32 keys that the rotation takes to within 1e-10 .. 1e-8 of a border between
    two codes: cosines and sines in fp32 would take many of them across."""
    n, dim, past = 256, 128, 992
    rng = np.random.default_rng(77)
    freq = S.frequencies(dim)
    turn = (np.arange(n) + past)[:, None, None] * freq[:, None]
    c, s = np.cos(turn), np.sin(turn)
    border = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], (n, 64, 1)) * rng.choice([-1, 1], (n, 64, 1))
    border[:, ::32] = 6.25  # (the largest of a group: codes count in ones)
    # of 256 pairs (a, b) each the one that comes nearest
    b = rng.uniform(-2, 2, (n, 64, 1)).astype(np.float32) * (1 + np.arange(256) * 2.0 ** -22).astype(np.float32)
    a = ((border + b * s) / np.where(np.abs(c) > 0.3, c, 1)).astype(np.float32)
    off = np.abs(a * c - b * s - border)
    off = np.where((off > 1e-10) & (np.abs(c) > 0.3), off, 1.0)
    at = off.argmin(-1)[..., None]
    use = np.take_along_axis(off, at, -1)[..., 0] < 1e-8
    assert use.sum() > 5000
    k = np.zeros((n, 1, dim), dtype=np.float32)
    k[:, 0, :64] = np.where(use, np.take_along_axis(a, at, -1)[..., 0], 0)
    k[:, 0, 64:] = np.where(use, np.take_along_axis(b, at, -1)[..., 0], 0)
    want = S.held(S.rotate(k.astype(np.float64), np.arange(n) + past, freq)[0])
    pool = [P.quant_pages(n // 16, 16, 1, dim) for _ in range(2)]
    books = ints([[-1] * (past // 16) + list(range(n // 16))]), ints([past]), ints([past + n])
    kt = dev(k)
    P.presto_append_rope(P.rope_plan(dim), None, kt, kt, ints([0, n]), n, *pool, *books)
    got, _ = P.presto_read_kv(*pool, *books, ints([0, n]), n, rows=n, dtype=torch.float32)
    assert (got.double().cpu().numpy() == want).all()


def test_groups_that_are_not_finite_or_extreme():
    dim = 64
    x = torch.ones(6, 2, dim, device="cuda")
    x[0, 0, 5], x[1, 1, 40], x[2, 0, 0] = math.nan, math.inf, -math.inf
    x[3, 0] = 3.4e38
    x[4, 0, :32] = 1e-40
    x[4, 0, 32:] = 2.0 ** -119
    x[5] = 0.0
    x[5, 1, 7] = -0.0
    pool = [P.quant_pages(1, 16, 2, dim) for _ in range(2)]
    args = (ints([[0]]), ints([0]), ints([6]), ints([0, 6]), 6)
    P.presto_append_rope(None, None, x, x, args[3], 6, *pool, *args[:3])
    want = S.held(x.double().cpu().numpy())
    for got in P.presto_read_kv(*pool, *args, rows=6, dtype=torch.float32):
        got = got.double().cpu().numpy()
        assert ((got == want) | (np.isnan(got) & np.isnan(want))).all()
    assert want[3, 0, 0] == 6 * 2.0 ** 125
    assert np.isnan(want[0, 0, :32]).all() and np.isfinite(want[0, 0, 32:]).all()


@pytest.mark.parametrize("quant", [True, False])
def test_append_and_read_flag_what_does_not_fit(quant):
    rng = np.random.default_rng(8)
    dim, hkv, page, B = 64, 2, 16, 7
    #        fine, no page, bad page, shrinks, too long, offsets back, past the rows
    past, new = [3, 5, 16, 4, 60, 0, 2], [3, 2, 2, -1, 10, 2, 9]
    table = np.full((B, 4), -1)
    table[:, 0] = np.arange(B)
    table[1, 0], table[2, 1] = -1, 99
    table[4] = [8, 9, 10, 11]
    offs = [0, 3, 5, 7, 7, 17, 15, 24]
    rows = 23
    q, k = tensor(rng, (rows, 4, dim), "bf16"), tensor(rng, (rows, hkv, dim), "bf16")
    if quant:
        pool = [dev(rng.integers(0, 256, (12, hkv, 1, 17 * dim // 2), dtype=np.uint8)) for _ in range(2)]
    else:
        pool = [tensor(rng, (12, page, hkv, dim), "bf16") for _ in range(2)]
    before = [p.clone() for p in pool]
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    books_ = (ints(table), ints(past), ints(np.add(past, new)))
    out = torch.full_like(q, 7.0)
    P.presto_append_rope(P.rope_plan(dim), q, k, k, ints(offs), 9, *pool, *books_, out=out, flags=flags)
    assert flags.item() == P.PRESTO_FLAG_BAD_PAGE | P.PRESTO_FLAG_BAD_SEQ
    touched = (out != 7).flatten(1).any(1).nonzero().flatten().tolist()
    assert touched == [0, 1, 2, 3, 4, 5, 6]  # (without a page the keys are lost, the queries are not)
    changed = [p for p in range(12) if not torch.equal(pool[0][p], before[0][p])]
    assert changed == [0]
    flags.zero_()
    outs = [torch.full_like(k, 7.0) for _ in range(2)]
    P.presto_read_kv(*pool, *books_, ints(offs), 9, out=outs, flags=flags)
    assert flags.item() == P.PRESTO_FLAG_BAD_PAGE | P.PRESTO_FLAG_BAD_SEQ
    for t in outs:
        assert (t != 7).flatten(1).any(1).nonzero().flatten().tolist() == [0, 1, 2]


# ---------------------------------------------------------------------------
# forks and moves of 4-bit pages

@pytest.mark.parametrize("layers", [1, 3])
@pytest.mark.parametrize("dim,hkv,page", [(64, 1, 16), (128, 3, 64)])
def test_forks_and_moves(layers, dim, hkv, page):
    rng = np.random.default_rng([9, dim])
    n, B = 24, 5
    k, v = (dev(rng.integers(0, 256, (layers, n, hkv, page // 16, 17 * dim // 2), dtype=np.uint8)) for _ in range(2))
    refs, table, ctx = ints([0] * n), ints([[-1] * 4] * B), ints([0] * B)
    P.presto_pages_reserve(refs, table, ctx, page, ints([page + 3, 0, 2 * page, 5, 0]), out=ctx)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    want_k, want_v = k.clone(), v.clone()
    P.presto_pages_fork(refs, table, ctx, ints([0, 2]), ints([1, 4]), k, v, flags=flags)
    assert flags.item() == 0 and ctx.tolist() == [page + 3, page + 3, 2 * page, 5, 2 * page]
    t = table.tolist()
    assert t[1][0] == t[0][0] and t[1][1] != t[0][1] and t[4][:2] == t[2][:2]
    for pool, want in ((k, want_k), (v, want_v)):
        want[:, t[1][1]] = want[:, t[0][1]]
        assert torch.equal(pool, want)
    P.presto_pages_free(refs, table, ctx, ints([0, 2]))
    old = table.tolist()
    got = P.presto_pages_compact(refs, table, k, v)
    for pool, want in ((k, want_k), (v, want_v)):
        for b in (1, 3, 4):
            for x, e in enumerate(old[b]):
                if e >= 0:
                    assert torch.equal(pool[:, got["page_table"][b, x].item()], want[:, e])


# ---------------------------------------------------------------------------
# attention

CTX = [1, 2, 5, 16, 17, 31, 32, 33, 64, 100, 300, 0, 1000]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,dim,page", [(4, 2, 64, 16), (32, 8, 128, 64), (7, 1, 128, 16), (6, 6, 64, 32), (40, 2, 128, 256),
                                             (33, 1, 64, 16)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (50, 4), (33, 40), (200, 0)])
def test_decode(hq, hkv, dim, page, window, sinks, dtype):
    rng = np.random.default_rng([10, hq, dim, window])
    c = Quant(rng, CTX, page, hkv, dim)
    if window:  # pages that nothing sees have been given back
        for b, n in enumerate(CTX):
            for x in range(c.table_h.shape[1]):
                if x * page >= sinks and x * page + page <= n - window:
                    c.table_h[b, x] = -1
        table = ints(c.table_h)
    else:
        table = c.table
    q = tensor(rng, (len(CTX), hq, dim), dtype)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = P.presto_quant_attention(q, c.k, c.v, table, c.ctx, window=window, sinks=sinks, flags=flags)
    assert flags.item() == 0
    offs = ints(np.arange(len(CTX) + 1))
    again = P.presto_quant_attention(q, c.k, c.v, table, c.ctx, q_offsets=offs, max_q=1, window=window, sinks=sinks)
    assert torch.equal(out, again)
    hint = P.presto_quant_attention(q, c.k, c.v, table, c.ctx, max_ctx=1000, window=window, sinks=sinks, total_ctx=sum(CTX))
    qd = q.double().cpu().numpy()
    c.table_h = c.table.cpu().numpy()
    for b, n in enumerate(CTX):
        want, bound = tight(qd[b:b + 1], *c.rows(b), n - 1, window, sinks, dtype)
        for got in (out, hint):
            err = np.abs(got[b:b + 1].double().cpu().numpy() - want)
            assert (err <= bound).all(), (n, (err / bound).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,dim,page", [(4, 2, 64, 16), (8, 2, 128, 64), (5, 1, 128, 32), (3, 3, 64, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 1), (50, 4), (300, 35)])
def test_chunks(hq, hkv, dim, page, window, sinks, dtype):
    """Ragged new tokens; rows outside all sequences stay as they were."""
    rng = np.random.default_rng([11, hq, dim, window])
    ctx, new = [40, 7, 500, 33, 130, 64, 9], [40, 1, 77, 0, 130, 33, 12]  # (the last: more tokens than positions)
    c = Quant(rng, ctx, page, hkv, dim)
    offs = 2 + np.concatenate([[0], np.cumsum(new)])
    q = tensor(rng, (int(offs[-1]) + 5, hq, dim), dtype)
    for kw in (dict(), dict(max_ctx=500, total_ctx=sum(ctx))):
        out = torch.full_like(q, 7.0)
        P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, q_offsets=ints(offs), max_q=130, window=window, sinks=sinks,
                                 out=out, **kw)
        assert (out[:2] == 7).all() and (out[offs[-1]:] == 7).all()
        got, qd = out.double().cpu().numpy(), q.double().cpu().numpy()
        for b, (n, L) in enumerate(zip(new, ctx)):
            s = slice(offs[b], offs[b] + n)
            want, bound = tight(qd[s], *c.rows(b), L - n, window, sinks, dtype, False)
            assert (np.abs(got[s] - want) <= bound).all(), b
            if n > L:
                assert (got[offs[b]:offs[b] + n - L] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,ctx", [(1, 9000), (3, 4097), (40, 700)])
def test_split_contexts(batch, ctx, dtype):
    rng = np.random.default_rng([12, batch])
    lens = [ctx] + rng.integers(1, ctx, batch - 1).tolist()
    c = Quant(rng, lens, 64, 2, 128, sigma=2.0)
    q = tensor(rng, (batch, 8, 128), dtype)
    out = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx)
    assert torch.equal(out, P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx))
    qd, got = q.double().cpu().numpy(), out.double().cpu().numpy()
    for b in list(range(min(batch, 3))):
        want, bound = tight(qd[b:b + 1], *c.rows(b), lens[b] - 1, 0, 0, dtype)
        assert (np.abs(got[b:b + 1] - want) <= bound).all()


def test_queries_in_a_projection():
    rng = np.random.default_rng(13)
    c = Quant(rng, [70, 200], 16, 2, 64)
    wide = tensor(rng, (2, 12, 64), "bf16")
    q = wide[:, :8]
    assert torch.equal(P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx),
                       P.presto_quant_attention(q.contiguous(), c.k, c.v, c.table, c.ctx))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [-300.0, -90.0, 0.0, 90.0, 300.0])
def test_scores_far_from_zero(shift, dtype):
    """All scores around `shift`: one K group holds a constant that the query
    meets."""
    rng = np.random.default_rng(14)
    c = Quant(rng, [400, 33], 16, 1, 64)
    q = tensor(rng, (2, 4, 64), dtype)
    for b in range(2):
        at = c.where(b, range(c.ctx_h[b]))
        k = S.read(c.kh, False, *at)
        k[..., 32:] = 4.0
        S.write(c.kh, False, *at, *S.encode(k))
    c.upload()
    q[..., 32:] = shift * 8 / (32 * 4.0)
    out = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx).double().cpu().numpy()
    for b in range(2):
        want, bound = tight(q[b:b + 1].double().cpu().numpy(), *c.rows(b), c.ctx_h[b] - 1, 0, 0, dtype)
        assert (np.abs(out[b:b + 1] - want) <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 4, 40])
@pytest.mark.parametrize("way", [1, -1])
def test_scores_that_rise_and_fall(way, new, dtype):
    """One K group holds a value that grows (or falls) from tile to tile, by more
    and more: a row's reference has to move in each of them, or in none."""
    rng = np.random.default_rng(17)
    c = Quant(rng, [420, 420], 32, 1, 128)
    steps = np.array([2.0 ** (i // 2) * (1, 1.5)[i % 2] for i in range(14)])[::way]
    for b in range(2):
        at = c.where(b, range(420))
        k = S.read(c.kh, False, *at)
        k[..., 96:] = steps[np.arange(420) // 32][:, None, None]
        S.write(c.kh, False, *at, *S.encode(k))
    c.upload()
    q = tensor(rng, (2 * new, 8, 128), dtype)
    q[..., 96:] = 0.25
    out = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, q_offsets=ints([0, new, 2 * new]), max_q=new)
    out = out.double().cpu().numpy()
    for b in range(2):
        one = slice(b * new, (b + 1) * new)
        want, bound = tight(q[one].double().cpu().numpy(), *c.rows(b), 420 - new, 0, 0, dtype, new * 8 < 128)
        assert (np.abs(out[one] - want) <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 40])
def test_least_values(new, dtype):
    """Values of the least exponent under equal probabilities (queries of 0)."""
    rng = np.random.default_rng(16)
    c = Quant(rng, [60, 300], 16, 1, 128)
    for b in range(2):
        at = c.where(b, range(c.ctx_h[b]))
        S.write(c.vh, True, *at, *S.encode(rng.standard_normal((c.ctx_h[b], 1, 128)) * 2.0 ** -120))
    c.upload()
    q = torch.zeros(2 * new, 8, 128, dtype=DT[dtype], device="cuda")
    out = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, q_offsets=ints([0, new, 2 * new]), max_q=new)
    out = out.double().cpu().numpy()
    for b in range(2):
        one = slice(b * new, (b + 1) * new)
        want, bound = tight(q[one].double().cpu().numpy(), *c.rows(b), c.ctx_h[b] - new, 0, 0, dtype, new * 8 < 128)
        # (and half a step of the output's subnormal numbers)
        assert (np.abs(out[one] - want) <= bound + (2.0 ** -134 if dtype == "bf16" else 2.0 ** -150)).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 40])
def test_groups_that_are_not_finite_reach_who_sees_them(dim, new):
    rng = np.random.default_rng([15, dim])
    L, hkv, G = 90, 2, 3
    for pool, is_v in (("kh", False), ("vh", True)):
        c = Quant(rng, [L, 64], 16, hkv, dim)
        q = tensor(rng, (2 * new, hkv * G, dim), "bf16")
        offs = ints([0, new, 2 * new])
        args = dict(q_offsets=offs, max_q=new)
        good = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, **args)
        key, head, grp = L - new // 2 - 1, 1, 1
        page, row = c.where(0, [key])
        block = getattr(c, pool)[page[0], head, row[0] // 16]
        block[S.offsets(dim, is_v)[1][row[0] % 16, 32 * grp]] = 255
        c.upload()
        out = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, **args)
        bad = torch.zeros_like(out, dtype=torch.bool)
        sees = torch.arange(L - new, L, device="cuda") >= key
        dims = slice(32 * grp, 32 * grp + 32) if is_v else slice(0, dim)
        bad[:new, head * G:(head + 1) * G, dims] = sees[:, None, None]
        assert torch.equal(torch.isnan(out), bad)
        same = torch.where(bad, torch.zeros_like(out), out)
        assert torch.equal(same, torch.where(bad, torch.zeros_like(good), good))


def test_bad_books_are_flagged_and_do_not_fault():
    rng = np.random.default_rng(16)
    c = Quant(rng, [70, 70, 70, 70], 16, 1, 64)
    q = tensor(rng, (4, 2, 64), "bf16")
    good = P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx)
    for entry in (-1, 10 ** 6, -2 ** 31):
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        table = c.table.clone()
        table[1, 2] = entry
        out = P.presto_quant_attention(q, c.k, c.v, table, c.ctx, flags=flags)
        assert flags.item() == P.PRESTO_FLAG_BAD_PAGE
        k, v = (np.delete(x, np.s_[32:48], 0) for x in c.rows(1))
        want, bound = tight(q[1:2].double().cpu().numpy(), k, v, 53, 0, 0, "bf16")
        assert (np.abs(out[1:2].double().cpu().numpy() - want) <= bound).all()
        assert torch.equal(out[[0, 2, 3]], good[[0, 2, 3]])
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = P.presto_quant_attention(q, c.k, c.v, c.table, ints([70, -3, 10 ** 6, 70]), max_ctx=70, flags=flags)
    assert flags.item() == P.PRESTO_FLAG_BAD_SEQ
    assert (out[1] == 0).all() and torch.equal(out[[0, 2, 3]], good[[0, 2, 3]])
    for offs in ([0, 3, 2, 4, 4], [0, 1, 9, 9, 9], [-1, 1, 2, 3, 4], [0, 4, 4, 4, 4]):
        flags.zero_()
        out = torch.full_like(q, 7.0)
        P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, q_offsets=ints(offs), max_q=3, out=out, flags=flags)
        assert flags.item() == P.PRESTO_FLAG_BAD_SEQ
        assert (out[3] == 7).all() or offs[0] == -1 or offs[3] == 4


def test_no_sequences():
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    pool = P.quant_pages(1, 16, 2, 64)
    t = torch.empty(0, 1, dtype=torch.int32, device="cuda")
    assert P.presto_quant_attention(q, pool, pool, t, ints([])).shape == (0, 4, 64)
