"""GPU parity of the paged cache: the attention against a 64-bit reference
within bounds derived from the arithmetic (paged_ref), copies and books bit
for bit.  Whatever no query sees (free pages, rows past a sequence's end, rows
outside the window where nobody sees them) holds NaN."""
import itertools

import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2607_22634_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def flag():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


class Cache:
    """A shuffled pool holding sequences of the given lengths; positions that
    queries from ctx - n on do not see are left out, all else is NaN."""

    def __init__(self, rng, ctx, new, page, hkv, d, dtype, window=0, sinks=0, pair=False, spare=3):
        self.page, self.dtype, self.ctx_l, self.new = page, dtype, list(ctx), list(new)
        B = len(ctx)
        cols = max([1] + [-(-c // page) for c in ctx]) + 1
        table = np.full((B, cols), -1, np.int32)
        keep = []
        for b, (c, n) in enumerate(zip(ctx, new)):
            seen = np.zeros(c, bool)
            for pos in {max(c - n, 0), c - 1} if c else ():
                seen |= R.visible(pos, c, window, sinks)
            if window == 0 or n == 0 and c:
                seen[:] = True
            lo = max(c - n, 0) - window + 1
            if window:  # the union over the queries in between
                seen[max(lo, 0):] = True
            keep.append(seen)
        used = [(b, x) for b in range(B) for x in range(-(-ctx[b] // page)) if keep[b][x * page:(x + 1) * page].any()]
        pages = len(used) + spare
        order = rng.permutation(pages)
        shape = (pages, 2, page, hkv, d) if pair else (2, pages, page, hkv, d)
        both = torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(TYPES[dtype])
        self.k_h, self.v_h = (both[:, 0], both[:, 1]) if pair else (both[0], both[1])
        unseen = np.ones((pages, page), bool)
        for i, (b, x) in enumerate(used):
            table[b, x] = order[i]
            m = keep[b][x * page:(x + 1) * page]
            unseen[order[i], :len(m)] = ~m
        for pool in (self.k_h, self.v_h):
            pool[torch.from_numpy(unseen)] = float("nan")
        both = both.to(DEV)
        self.k, self.v = (both[:, 0], both[:, 1]) if pair else (both[0], both[1])
        self.table_h, self.table, self.ctx = table, ints(table.tolist()), ints(list(ctx))

    def rows(self, b):
        c = self.ctx_l[b]
        return [R.gather(p.double().numpy(), self.table_h[b], c) for p in (self.k_h, self.v_h)]


def queries(rng, n, hq, d, dtype, wide=False):
    """[n, hq, d], as a slice of a wider projection if `wide`"""
    t = torch.from_numpy(rng.standard_normal((n, hq + 3 if wide else hq, d), dtype=np.float32)).to(TYPES[dtype])
    full = t.to(DEV)
    return full[:, 1:hq + 1] if wide else full


def close(got, q, cache, offs, window, sinks, scale=None):
    got, qh = got.double().cpu().numpy(), q.double().cpu().numpy()
    for b, n in enumerate(cache.new):
        if n == 0:
            continue
        k, v = cache.rows(b)
        s = slice(offs[b], offs[b] + n)
        want, bound = R.attention(qh[s], k, v, cache.ctx_l[b] - n, window, sinks, scale, cache.dtype)
        err = np.abs(got[s] - want)
        assert (err <= bound).all(), (b, n, cache.ctx_l[b], np.nanmax(err / bound), np.isnan(err).sum())


HEADS = [(4, 2, 64), (32, 8, 128), (7, 1, 128), (6, 6, 64), (20, 1, 64), (40, 1, 128)]
MASKS = [(0, 0), (48, 4), (1, 0), (17, 33), (200, 130), (100000, 4)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("mask", MASKS)
def test_decode_matches_reference(dtype, heads, mask):
    hq, hkv, d = heads
    rng = np.random.default_rng([hq, hkv, d, *mask])
    ctx = [0, 1, 2, 15, 16, 17, 31, 33, 64, 65, 127, 300, 1000]
    page = [16, 32, 64, 256][(hq + mask[0]) % 4]
    c = Cache(rng, ctx, [1] * len(ctx), page, hkv, d, dtype, *mask, pair=hq % 2 == 0)
    q = queries(rng, len(ctx), hq, d, dtype, wide=hq % 3 == 0)
    f = flag()
    out = P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx, window=mask[0], sinks=mask[1], flags=f)
    torch.cuda.synchronize()
    assert f.item() == 0
    assert not out[0].any()
    c.new[0] = 0  # a sequence without a cached token: zeros
    close(out, q, c, list(range(len(ctx))), *mask)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("mask", MASKS)
def test_window_matches_reference(dtype, heads, mask):
    hq, hkv, d = heads
    rng = np.random.default_rng([1, hq, hkv, d, *mask])
    ctx = [5, 130, 0, 40, 64, 70, 200, 333]
    new = [5, 1, 0, 0, 64, 33, 2, 140]
    if hq * d > 2000:
        ctx, new = ctx[:5] + [150], new[:5] + [40]
    page = [16, 32, 64, 256][(hkv + mask[1]) % 4]
    c = Cache(rng, ctx, new, page, hkv, d, dtype, *mask)
    offs = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = queries(rng, offs[-1] + 2, hq, d, dtype, wide=hq % 3 == 1)
    out = torch.full((offs[-1] + 2, hq, d), 7.0, dtype=TYPES[dtype], device=DEV)
    f = flag()
    P.presto_window_attention(q, ints(offs), max(new), c.k, c.v, c.table, c.ctx, window=mask[0], sinks=mask[1],
                              out=out, flags=f)
    torch.cuda.synchronize()
    assert f.item() == 0
    assert (out[offs[-1]:] == 7).all()  # rows behind the last sequence
    close(out, q, c, offs, *mask)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,n,hint", [(1, 1, False), (3, 1, True), (2, 3, False), (2, 40, True)])
@pytest.mark.parametrize("mask", [(0, 0), (700, 20)])
def test_long_contexts_split_and_joined(dtype, batch, n, hint, mask):
    rng = np.random.default_rng([2, batch, n, *mask])
    ctx = [5000, 17, 2500][:batch]
    c = Cache(rng, ctx, [n] * batch, 64, 2, 128, dtype, *mask)
    offs = [n * b for b in range(batch + 1)]
    q = queries(rng, n * batch, 4, 128, dtype)
    kw = dict(window=mask[0], sinks=mask[1], max_ctx=5000, total_ctx=sum(ctx) if hint else 0)
    if n == 1:
        run = lambda **o: P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx, **kw, **o)
    else:
        run = lambda **o: P.presto_window_attention(q, ints(offs), n, c.k, c.v, c.table, c.ctx, **kw, **o)
    out = run()
    close(out, q, c, offs, *mask)
    again = run(workspace=torch.full((1 << 24,), 0xff, dtype=torch.uint8, device=DEV))
    assert torch.equal(out, again)  # whatever the workspace held


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,past,window", [(3, 50, 60), (90, 10, 60), (300, 0, 60), (90, 3000, 60), (90, 1000, 0),
                                           (3, 1500, 0), (200, 0, 0)])
def test_values_that_are_not_finite_reach_their_own_queries_only(dtype, n, past, window):
    """inf and NaN in K or V of single keys: queries that do not see the key
    are as they were, those that see it are not finite (or, for K = -inf, as
    the definition has it)."""
    rng = np.random.default_rng([3, n, past])
    L, hq, hkv, d, sinks = past + n, 4, 2, 64, 2
    c = Cache(rng, [L], [n], 32, hkv, d, dtype, window, sinks)
    q = queries(rng, n, hq, d, dtype)
    offs = ints([0, n])
    run = lambda: P.presto_window_attention(q, offs, n, c.k, c.v, c.table, c.ctx, window=window, sinks=sinks)
    base = run()
    for key, name, val in ((L - n // 2 - 1, "v", float("nan")), (L - 1, "v", float("inf")), (L - 1, "k", float("nan")),
                           (L - n, "v", float("-inf")), (L - n, "k", float("nan"))):
        page, row = int(c.table_h[0, key // 32]), key % 32
        for pool in (getattr(c, name), getattr(c, name + "_h")):
            pool[page, row, 1] = val  # KV head 1: query heads 2 and 3
        got = run()
        sees = np.array([R.visible(past + i, L, window, sinks)[key] for i in range(n)])
        assert torch.equal(got[:, :2], base[:, :2])
        k, v = c.rows(0)
        want, bound = R.attention(q.double().cpu().numpy(), k, v, past, window, sinks, None, dtype)
        g = got.double().cpu().numpy()
        with np.errstate(invalid="ignore"):
            assert (np.abs(g - want)[~sees] <= bound[~sees]).all(), (key, name, val)
        assert not np.isfinite(g[sees, 2:]).any(), (key, name, val)
        good = torch.from_numpy(rng.standard_normal((hkv, d), dtype=np.float32)).to(TYPES[dtype])
        getattr(c, name)[page, row], getattr(c, name + "_h")[page, row] = good.to(DEV), good
        base = run()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [5, 180])
def test_values_that_are_not_finite_in_a_long_context(dtype, n):
    """K and V that no query can leave out, and V that only some see, 20000
    keys into a sequence: every element is finite exactly where the
    definition's is, and right there."""
    rng = np.random.default_rng([33, n])
    past, hq, hkv, d = 20000, 4, 2, 64
    L = past + n
    c = Cache(rng, [L], [n], 64, hkv, d, dtype, 0, 0)
    q = queries(rng, n, hq, d, dtype)
    offs = ints([0, n])
    some = [0, n // 2, n - 1]

    def check():
        got = P.presto_window_attention(q, offs, n, c.k, c.v, c.table, c.ctx).double().cpu().numpy()
        k, v = c.rows(0)
        for i in some:
            with np.errstate(invalid="ignore"):
                want, bound = R.attention(q[i:i + 1].double().cpu().numpy(), k, v, past + i, 0, 0, None, dtype)
            fin = np.isfinite(want)
            assert (np.isfinite(got[i:i + 1]) == fin).all(), i
            assert (np.abs(got[i:i + 1][fin] - want[fin]) <= bound[fin]).all(), i

    def put(name, key, head, dim, val):
        page, row = int(c.table_h[0, key // 64]), key % 64
        for pool in (getattr(c, name), getattr(c, name + "_h")):
            pool[page, row, head, dim] = val

    put("v", 7, 1, 3, float("nan"))  # all queries of heads 2, 3: that dim
    check()
    put("v", past + n // 2, 1, 5, float("inf"))  # and one that queries from the middle on see
    check()
    put("k", 9000, 0, 3, float("nan"))  # all of heads 0, 1
    check()
    put("v", L - 1, 0, 0, float("nan"))
    check()


def _ragged(rng, batch, lo, hi):
    return [int(x) for x in rng.integers(lo, hi + 1, batch)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,most,past", [(1, 700, 0), (3, 150, 900), (70, 40, 60), (2100, 9, 12)])
def test_ragged_prompts_of_small_and_large_batches(dtype, batch, most, past):
    """Row blocks counted by length, by sequence and by grid; a sample of the
    sequences is compared (all rows of small batches)."""
    rng = np.random.default_rng([16, batch])
    new = _ragged(rng, batch, 0, most)
    new[-1] = most
    ctx = [n + p for n, p in zip(new, _ragged(rng, batch, 0, past))]
    mask = (0, 0) if batch % 2 else (50, 3)
    c = Cache(rng, ctx, new, 16, 1, 64, dtype, *mask)
    offs = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = queries(rng, offs[-1], 8, 64, dtype)
    f = flag()
    out = P.presto_window_attention(q, ints(offs), most, c.k, c.v, c.table, c.ctx, window=mask[0], sinks=mask[1],
                                    flags=f)
    assert f.item() == 0 and torch.isfinite(out).all()
    pick = set(range(batch)) if batch <= 3 else set(rng.choice(batch, 12, replace=False).tolist()) | {0, batch - 1}
    c.new = [n if b in pick else 0 for b, n in enumerate(new)]
    close(out, q, c, offs, *mask)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,hi", [(5, 4000), (40, 900), (130, 700), (2100, 600)])
@pytest.mark.parametrize("n", [1, 3])
def test_ragged_contexts_in_shares(dtype, batch, hi, n):
    """Batches of very different lengths, empty sequences among them, cut into
    equal shares (or too large a batch for that)."""
    rng = np.random.default_rng([17, batch, n])
    ctx = [int(x) for x in np.exp(rng.uniform(0, np.log(hi), batch))]
    ctx[batch // 2], ctx[-1] = 0, hi
    new = [min(n, x) if b % 5 else 0 for b, x in enumerate(ctx)] if n > 1 else [1] * batch
    d = 64 if batch > 100 else 128
    c = Cache(rng, ctx, [1] * batch, 16, 2, d, dtype)
    c.new = new
    offs = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = queries(rng, offs[-1], 6, d, dtype)
    f = flag()
    if n == 1:
        out = P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx, max_ctx=hi, flags=f)
    else:
        out = P.presto_window_attention(q, ints(offs), n, c.k, c.v, c.table, c.ctx, max_ctx=hi, flags=f)
    assert f.item() == 0 and torch.isfinite(out).all()
    pick = set(rng.choice(batch, min(batch, 14), replace=False).tolist()) | {0, batch - 1, batch // 2 - 1}
    assert n > 1 or not out[batch // 2].any()
    c.new = [x if b in pick and ctx[b] else 0 for b, x in enumerate(new)]
    close(out, q, c, offs, 0, 0)


def test_more_pages_than_one_workgroup_keeps():
    """A context whose page numbers do not fit the LDS of one workgroup."""
    rng = np.random.default_rng(18)
    L, n = 140000, 20
    c = Cache(rng, [L], [1], 16, 1, 64, "bf16")
    c.new = [n]
    q = queries(rng, n, 2, 64, "bf16")
    out = P.presto_window_attention(q, ints([0, n]), n, c.k, c.v, c.table, c.ctx)
    close(out, q, c, [0], 0, 0)


@pytest.mark.parametrize("heads,n,ctx", [((32, 8, 128), 130, 130), ((32, 8, 128), 600, 700), ((16, 1, 128), 100, 2000),
                                         ((12, 4, 64), 513, 900), ((8, 8, 64), 257, 257)])
def test_blocks_of_64_128_and_256_rows(heads, n, ctx):
    """The plans of short, long and wide prompts (heads x tokens), a sample of
    the rows against the reference."""
    rng = np.random.default_rng([19, n])
    hq, hkv, d = heads
    c = Cache(rng, [ctx], [n], 32, hkv, d, "bf16", 300, 4)
    q = queries(rng, n, hq, d, "bf16")
    out = P.presto_window_attention(q, ints([0, n]), n, c.k, c.v, c.table, c.ctx, window=300, sinks=4)
    k, v = c.rows(0)
    for i in sorted({0, 1, 15, 16, 63, 64, n // 2, n - 2, n - 1}):
        want, bound = R.attention(q[i:i + 1].double().cpu().numpy(), k, v, ctx - n + i, 300, 4)
        assert (np.abs(out[i:i + 1].double().cpu().numpy() - want) <= bound).all(), i


@pytest.mark.parametrize("dtype,heads,n,ctx", [("f32", (32, 8, 128), 900, 1500), ("f32", (32, 8, 64), 40, 50),
                                               ("f32", (8, 2, 128), 30, 6000), ("bf16", (32, 8, 128), 6, 9000),
                                               ("bf16", (32, 8, 128), 8, 200), ("bf16", (2, 1, 64), 13, 3001)])
@pytest.mark.parametrize("window", [0, 1000])
@pytest.mark.parametrize("batch", [1, 5])
def test_blocks_of_16_and_32_rows(dtype, heads, n, ctx, window, batch):
    """The plans of the kernel of rows on more than sixteen, uncut and cut, of
    even and ragged batches; a sample of the rows against the reference."""
    rng = np.random.default_rng([20, n, window, batch])
    hq, hkv, d = heads
    new = [n] + _ragged(rng, batch - 1, 1, n)
    lens = [ctx] + [int(x) for x in rng.integers(ctx // 2, ctx + 1, batch - 1)]
    lens = [max(a, b) for a, b in zip(lens, new)]
    c = Cache(rng, lens, new, 32, hkv, d, dtype, window, 4)
    offs = np.concatenate([[0], np.cumsum(new)]).tolist()
    q = queries(rng, offs[-1], hq, d, dtype)
    for total in (0, sum(lens)):
        out = P.presto_window_attention(q, ints(offs), n, c.k, c.v, c.table, c.ctx, max_ctx=max(lens), window=window,
                                        sinks=4 if window else 0, total_ctx=total)
        for b in {0, batch - 1}:
            k, v = c.rows(b)
            for i in sorted({0, min(16, new[b] - 1), new[b] // 2, new[b] - 1}):
                r = offs[b] + i
                want, bound = R.attention(q[r:r + 1].double().cpu().numpy(), k, v, lens[b] - new[b] + i, window,
                                          4 if window else 0, None, dtype)
                assert (np.abs(out[r:r + 1].double().cpu().numpy() - want) <= bound).all(), (b, i, total)


@pytest.mark.parametrize("batch,n,past,heads,page,window", [
    (2, 700, 2300, (16, 2, 128), 32, 0), (2, 700, 2300, (16, 2, 128), 64, 900), (2, 1000, 0, (16, 4, 64), 16, 0),
    (1, 2100, 500, (12, 2, 64), 128, 0), (1, 200, 140000, (8, 1, 64), 16, 0)])
def test_long_prompts_with_odd_values_and_missing_pages(batch, n, past, heads, page, window):
    """Prompts too long for the kernel of rows: a sample of the rows as they
    are, with V that is not finite at a key that some rows see and at one that
    all do, and with a page that is not there (its keys count as not visible)."""
    rng = np.random.default_rng([21, n, past, window])
    hq, hkv, d = heads
    sinks, L = 4 if window else 0, past + n
    c = Cache(rng, [L] * batch, [n] * batch, page, hkv, d, "bf16", window, sinks)
    q = queries(rng, batch * n, hq, d, "bf16")
    offs, b = ints([i * n for i in range(batch + 1)]), batch - 1
    some = sorted({0, 1, n // 3, n // 2, n // 2 + 1, n - 1})

    def check(gone=()):
        f = flag()
        out = P.presto_window_attention(q, offs, n, c.k, c.v, c.table, c.ctx, window=window, sinks=sinks, flags=f)
        assert f.item() == (P.PRESTO_FLAG_BAD_PAGE if gone else 0)
        k, v = c.rows(b)
        for i in some:
            ok = R.visible(past + i, L, window, sinks)
            ok[list(gone)] = False
            r, m = b * n + i, int(ok.sum())
            got = out[r:r + 1].double().cpu().numpy()
            with np.errstate(invalid="ignore"):
                want, bound = R.attention(q[r:r + 1].double().cpu().numpy(), k[ok], v[ok], m - 1, 0, 0, None, "bf16")
            fin = np.isfinite(want)
            assert (np.isfinite(got) == fin).all(), i
            assert (np.abs(got[fin] - want[fin]) <= bound[fin]).all(), i

    def put(name, key, head, dim, val):
        pg, row = int(c.table_h[b, key // page]), key % page
        for pool in (getattr(c, name), getattr(c, name + "_h")):
            pool[pg, row, head, dim] = val

    check()
    put("v", past + n // 2, hkv - 1, 3, float("inf"))
    check()
    put("v", past + n // 3 if window else 1, 0, 9, float("nan"))
    put("k", L - 1, 0, 0, float("nan"))
    check()
    col = (past + n // 2) // page if n > 300 else past // page  # (with the first of the odd values)
    c.table[b, col] = -1
    if n <= 1000:
        check(range(col * page, min((col + 1) * page, L)))


def test_equal_and_extreme_scores():
    """Scores far from 0, of one value, and growing along the sequence (the
    running reference moves at every tile)."""
    hq, hkv, d, L = 4, 2, 64, 700
    for dtype, kind in itertools.product(("bf16", "f32"), ("same", "rising", "falling", "large")):
        rng = np.random.default_rng(5)
        c = Cache(rng, [L, L], [1, 40], 64, hkv, d, dtype)
        q = queries(rng, 41, hq, d, dtype)
        if kind != "large":
            q[:] = 0
            q[..., 0] = 8.0
        for b in range(2):
            for j in range(L):
                p, r = int(c.table_h[b, j // 64]), j % 64
                x = {"same": 1.0, "rising": j / 8, "falling": (L - j) / 8, "large": None}[kind]
                if x is not None:
                    c.k_h[p, r, :, 0] = x
                else:
                    c.k_h[p, r] *= 16
        c.k.copy_(c.k_h)
        out = P.presto_window_attention(q, ints([0, 1, 41]), 40, c.k, c.v, c.table, c.ctx)
        close(out, q, c, [0, 1], 0, 0)


def test_rows_at_negative_positions_see_nothing():
    rng = np.random.default_rng(6)
    for dtype in TYPES:
        c = Cache(rng, [3, 0], [3, 0], 16, 2, 64, dtype)
        q = queries(rng, 45, 4, 64, dtype)
        out = P.presto_window_attention(q, ints([0, 40, 45]), 40, c.k, c.v, c.table, c.ctx)
        assert not out[:37].any() and not out[40:].any()
        close(out[37:40], q[37:40], c, [0, 3], 0, 0)


def test_lengths_and_offsets_outside_their_ranges_are_cut():
    rng = np.random.default_rng(7)
    for dtype in TYPES:
        c = Cache(rng, [40, 20, 33], [1, 1, 1], 16, 2, 64, dtype)
        q = queries(rng, 3, 4, 64, dtype)
        good = P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx, max_ctx=40)
        f = flag()
        out = P.presto_paged_attention(q, c.k, c.v, c.table, ints([40, -5, 1 << 30]), max_ctx=33, flags=f)
        assert f.item() == P.PRESTO_FLAG_BAD_SEQ
        assert not out[1].any() and torch.equal(out[2], good[2])
        for offs in ([0, 1, 0, 3], [-1, 1, 2, 3], [0, 1, 2, 9]):
            f = flag()
            got = torch.full_like(q, 7.0)
            P.presto_window_attention(q, ints(offs), 2, c.k, c.v, c.table, c.ctx, out=got, flags=f)
            assert f.item() == P.PRESTO_FLAG_BAD_SEQ
        assert torch.equal(got[:2], good[:2]) and (got[2] == 7).all()
        f = flag()  # more rows than max_q: the first ones
        got = torch.full_like(q, 7.0)
        P.presto_window_attention(q, ints([0, 3, 3, 3]), 2, c.k, c.v, c.table, c.ctx, out=got, flags=f)
        assert f.item() == P.PRESTO_FLAG_BAD_SEQ and (got[2] == 7).all()
        c.new, c.ctx_l = [3, 0, 0], [40, 20, 33]
        full = P.presto_window_attention(q, ints([0, 3, 3, 3]), 3, c.k, c.v, c.table, c.ctx)
        assert torch.equal(got[:2], full[:2])


@pytest.mark.parametrize("entry", [-1, 1 << 20, 1 << 30, -(1 << 31), 2 ** 31 - 1])
def test_pages_outside_the_pool_count_as_not_visible(entry):
    rng = np.random.default_rng(8)
    for dtype, n in itertools.product(TYPES, (1, 50)):
        c = Cache(rng, [100, 90], [n, n], 32, 2, 64, dtype)
        q = queries(rng, 2 * n, 4, 64, dtype)
        offs = ints([0, n, 2 * n])
        run = lambda f: P.presto_window_attention(q, offs, n, c.k, c.v, c.table, c.ctx, flags=f)
        f = flag()
        good = run(f)
        assert f.item() == 0
        c.table[0, 1] = entry  # positions 32 .. 63
        out = run(f)
        assert f.item() == P.PRESTO_FLAG_BAD_PAGE
        assert torch.equal(out[n:], good[n:])
        k, v = c.rows(0)
        cut = np.r_[0:32, 64:100]
        qh = q.double().cpu().numpy()
        i = n - 1  # the last query sees all other positions
        want, bound = R.attention(qh[i:i + 1], k[cut], v[cut], len(cut) - 1, dtype=dtype)
        assert (np.abs(out[i:i + 1].double().cpu().numpy() - want) <= bound).all()


def test_offsets_past_32_bits():
    """Pages beyond the first 2^32 bytes of the pool."""
    pages, page, hkv, d = 17000, 128, 8, 128  # 4.4 GB each
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GB of device memory")
    k = torch.zeros(pages, page, hkv, d, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros(pages, page, hkv, d, dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(9)
    c = Cache(rng, [500, 300], [1, 120], page, hkv, d, "bf16", spare=0)
    ids = [pages - 1, 16500, 3, 16999 - 5, 16400, 16999 - 9, 0][:c.k.shape[0]]
    for i, p in enumerate(ids):
        k[p], v[p] = c.k[i], c.v[i]
    table = torch.where(c.table >= 0, torch.tensor(ids, device=DEV)[c.table.clamp(min=0).long()].int(), c.table)
    q = queries(rng, 121, 32, d, "bf16")
    out = P.presto_window_attention(q, ints([0, 1, 121]), 120, k, v, table, c.ctx)
    same = P.presto_window_attention(q, ints([0, 1, 121]), 120, c.k, c.v, c.table, c.ctx)
    assert torch.equal(out, same)
    # an append, a fork and a compaction up there
    refs = torch.ones(pages, dtype=torch.int32, device=DEV)
    refs[16990] = refs[16991] = 0
    t, ctx = table.clone(), ints([500, 0])
    t[1] = -1
    new = queries(rng, 20, hkv, d, "bf16")
    ctx2 = P.presto_pages_reserve(refs, t, ctx, page, extra=20)
    assert ctx2.tolist() == [520, 20] and t[0, 4].item() == 16990 and t[1, 0].item() == 16991
    P.presto_append_kv(new, new + 1, ints([0, 20, 20]), 20, k, v, t, ctx, ctx2)
    assert torch.equal(k[t[0, 3].item(), 116:], new[:12]) and torch.equal(v[16990, :8], new[12:] + 1)
    refs[:] = 0
    refs[16990] = 1
    got = P.presto_pages_compact(refs, t, k, v)
    assert got["n_live"].item() == 1 and torch.equal(k[0, :8], new[12:]) and torch.equal(v[0, :8], new[12:] + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[1] * 9, [0, 17, 1, 0, 100, 33, 16, 15, 3]])
def test_append_writes_the_new_rows_only(dtype, new):
    rng = np.random.default_rng([10, sum(new)])
    hkv, d, page = 3, 64, 16
    past = [0, 1, 15, 16, 40, 0, 100, 31, 32]
    B = len(past)
    refs, table, ctx = torch.zeros(80, dtype=torch.int32, device=DEV), ints([[-1] * 14] * B), ints([0] * B)
    ctx = P.presto_pages_reserve(refs, table, ctx, page, ints(past))
    after = P.presto_pages_reserve(refs, table, ctx, page, ints(new))
    assert after.tolist() == [p + n for p, n in zip(past, new)]
    k, v = (torch.from_numpy(rng.standard_normal((80, page, hkv, d), dtype=np.float32)).to(DEV, TYPES[dtype])
            for _ in range(2))
    k0, v0 = k.clone(), v.clone()
    kn, vn = queries(rng, sum(new) + 4, hkv, d, dtype, wide=True), queries(rng, sum(new) + 4, hkv, d, dtype, wide=True)
    offs = np.concatenate([[0], np.cumsum(new)]).tolist()
    f = flag()
    P.presto_append_kv(kn, vn, ints(offs), max(new), k, v, table, ctx, after, flags=f)
    assert f.item() == 0
    for pool, ref, src in ((k, k0, kn), (v, v0, vn)):
        for b in range(B):
            for i in range(new[b]):
                j = past[b] + i
                ref[int(table[b, j // page]), j % page] = src[offs[b] + i]
        assert torch.equal(pool, ref)


def test_append_skips_what_it_cannot_write():
    hkv, d, page = 2, 64, 16
    k = torch.zeros(4, page, hkv, d, device=DEV)
    v = torch.zeros_like(k)
    new = torch.ones(40, hkv, d, device=DEV)
    table = ints([[0, -1], [1, 9], [2, 3]])

    def run(offs, most, ctx, after):
        f = flag()
        k.zero_()
        P.presto_append_kv(new, new, ints(offs), most, k, v, table, ints(ctx), ints(after), flags=f)
        return f.item(), [int(k[p].sum().item()) // (hkv * d) for p in range(4)]

    assert run([0, 4, 8, 12], 4, [14, 14, 14], [18, 18, 18]) == (P.PRESTO_FLAG_BAD_PAGE, [2, 2, 2, 2])
    assert run([0, 4, 8, 12], 4, [0, 0, 0], [0, 4, 2]) == (0, [0, 4, 2, 0])  # fewer rows than given
    seq = P.PRESTO_FLAG_BAD_SEQ
    assert run([0, 4, 8, 12], 3, [0, 0, 0], [4, 3, 3]) == (seq, [0, 3, 3, 0])  # past max_new
    assert run([0, 4, 8, 12], 9, [0, 0, 0], [5, 4, 4]) == (seq, [0, 4, 4, 0])  # past its rows
    assert run([0, 4, 8, 12], 9, [-1, 9, 0], [2, 8, 4]) == (seq, [0, 0, 4, 0])
    assert run([0, 4, 2, 41], 30, [0, 0, 0], [4, 0, 4]) == (seq, [4, 0, 0, 0])  # offsets out of order, past the rows
    assert run([-1, 4, 8, 12], 9, [0, 0, 28], [4, 4, 33]) == (seq, [0, 4, 0, 0])  # past the table


def _books_on_device(b):
    return ints(b.refs), ints(b.table), ints(b.ctx)


def _same_books(b, refs, table, ctx):
    assert refs.tolist() == b.refs
    assert table.tolist() == b.table
    assert ctx.tolist() == b.ctx


@pytest.mark.parametrize("seed", range(6))
def test_books_against_the_reference(seed):
    """A random serving history: every call's books, flags and pages."""
    rng = np.random.default_rng([11, seed])
    page, layers, hkv, d = [16, 64][seed % 2], 1 + seed % 3, 1 + seed % 2, 64
    B, pages, cols = [(3, 12, 6), (9, 40, 8), (70, 300, 9), (5, 5000, 40), (20, 90, 5), (40, 9000, 20)][seed]
    ref = R.Books([0] * pages, [[-1] * cols for _ in range(B)], [0] * B, page)
    refs, table, ctx = _books_on_device(ref)
    k, v = (torch.randn(layers, pages, page, hkv, d, device=DEV) for _ in range(2))
    kh, vh = k.clone(), v.clone()
    for step in range(60):
        f = flag()
        ref.flags = 0
        kind = rng.choice(["reserve", "reserve", "fork", "free", "trim", "compact"])
        moves = []
        if kind == "reserve":
            add = [int(x) for x in rng.integers(-1 if step % 7 == 0 else 0, [3, 2 * page, 1][step % 3] + 1, B)]
            add = add if step % 4 else None
            extra = int(rng.integers(0, 3))
            want = ref.reserve(add, extra)
            got = P.presto_pages_reserve(refs, table, ctx, page, None if add is None else ints(add), extra, flags=f)
            assert got.tolist() == want
            ref.ctx, ctx = want, got
        elif kind == "fork":
            n = int(rng.integers(1, B + 1))
            par, chi = rng.integers(0, B, n).tolist(), rng.integers(-1, B + 1, n).tolist()
            moves = ref.fork(par, chi)
            P.presto_pages_fork(refs, table, ctx, ints(par), ints(chi), k, v, flags=f)
        elif kind == "free":
            rows = rng.integers(-1 if step % 5 == 0 else 0, B, int(rng.integers(1, max(2, B // 2)))).tolist()
            ref.free(rows)
            P.presto_pages_free(refs, table, ctx, ints(rows), flags=f)
        elif kind == "trim":
            window, sinks = int(rng.integers(1, 3 * page)), int(rng.integers(0, 2 * page))
            ref.trim(window, sinks)
            P.presto_pages_trim(refs, table, ctx, page, window, sinks, flags=f)
        else:
            moves, to, live = ref.compact()
            out = dict(refs=refs, page_table=table, n_live=flag(), page_map=torch.empty_like(refs))
            if step % 2:  # books of their own
                out.update(refs=torch.empty_like(refs), page_table=torch.empty_like(table))
            got = P.presto_pages_compact(refs, table, k, v, out=out, flags=f)
            refs, table = got["refs"], got["page_table"]
            assert got["n_live"].item() == live and got["page_map"].tolist() == to
        torch.cuda.synchronize()
        assert f.item() == ref.flags, (step, kind)
        _same_books(ref, refs, table, ctx)
        for s, t, r in moves:
            for pool in (kh, vh):
                pool[:, t, :r] = pool[:, s, :r]
        assert torch.equal(k, kh) and torch.equal(v, vh), (step, kind)


def test_forks_that_cannot_be_made():
    page = 16
    base = R.Books([1, 1, 1, 0, 0, 0, 0, 0, 1], [[0, 1, -1], [-1] * 3, [-1] * 3, [2, 8, -1], [-1] * 3, [5, -1, -1], [50, -1, -1]],
                   [20, 0, 0, 32, 0, 3, 5], page)
    cases = [([0, 0], [1, 1]), ([0], [0]), ([0], [3]), ([0, 1], [1, 2]), ([1, 0], [2, 1]), ([5], [1]), ([6], [1]),
             ([-1, 7, 0, 0], [1, 1, -2, 7]), ([3, 3, 0, 0], [1, 2, 4, 4])]
    for par, chi in cases:
        ref = R.Books(base.refs, base.table, base.ctx, page)
        refs, table, ctx = _books_on_device(ref)
        k = torch.randn(2, 9, page, 1, 64, device=DEV)
        kh, f = k.clone(), flag()
        P.presto_pages_fork(refs, table, ctx, ints(par), ints(chi), k, k.clone(), flags=f)
        for s, t, r in ref.fork(par, chi):
            kh[:, t, :r] = kh[:, s, :r]
        _same_books(ref, refs, table, ctx)
        assert f.item() == ref.flags and torch.equal(k, kh), (par, chi)


def test_pools_of_page_pairs_and_spaced_layers():
    """K and V as the halves of one tensor of page pairs, and layers further
    apart than a pool is long: forks and compactions move just the pages."""
    page, hkv, d, pages, layers = 16, 2, 64, 10, 3
    room = torch.randn(layers, pages + 2, 2, page, hkv, d, device=DEV)
    ref0 = room.clone()
    both = room[:, :pages]
    k, v = both[:, :, 0], both[:, :, 1]
    ref = R.Books([1, 0, 1, 0, 0, 1, 0, 0, 0, 1], [[9, 5, 2], [0, -1, -1], [-1] * 3], [40, 7, 0], page)
    refs, table, ctx = _books_on_device(ref)
    P.presto_pages_fork(refs, table, ctx, ints([0]), ints([2]), k, v)
    moves = ref.fork([0], [2])
    got = P.presto_pages_compact(refs, table, k, v)
    moves += ref.compact()[0]
    _same_books(ref, got["refs"], got["page_table"], ctx)
    for s, t, r in moves:
        ref0[:, t, :, :r] = ref0[:, s, :, :r]
    assert torch.equal(room, ref0)


def test_layers_page_by_page():
    """[pages, layers, ...], as the call's [layers, pages, ...]."""
    page, hkv, d, pages, layers = 16, 2, 64, 10, 3
    room = torch.randn(2, pages, layers, page, hkv, d, device=DEV)
    ref0 = room.clone()
    k, v = room.transpose(1, 2)
    ref = R.Books([1, 0, 1, 0, 0, 1, 0, 0, 0, 1], [[9, 5, 2], [0, -1, -1], [-1] * 3], [40, 7, 0], page)
    refs, table, ctx = _books_on_device(ref)
    P.presto_pages_fork(refs, table, ctx, ints([0]), ints([2]), k, v)
    moves = ref.fork([0], [2])
    got = P.presto_pages_compact(refs, table, k, v)
    moves += ref.compact()[0]
    _same_books(ref, got["refs"], got["page_table"], ctx)
    for s, t, r in moves:
        ref0[:, t, :, :r] = ref0[:, s, :, :r]
    assert torch.equal(room, ref0)


@pytest.mark.parametrize("held", [0, 1])
def test_a_pool_of_one_page(held):
    refs, table = ints([held]), ints([[0 if held else -1, -1]])
    k = torch.randn(2, 1, 16, 1, 64, device=DEV)
    kh, f = k.clone(), flag()
    got = P.presto_pages_compact(refs, table, k, k.clone(), flags=f)
    assert got["refs"].tolist() == [held] and got["n_live"].tolist() == [held] and f.item() == 0
    assert torch.equal(got["page_table"], table) and torch.equal(k, kh)
    if held:  # and no room for a fork's page, but for one that shares the only one
        table, ctx = ints([[0, -1], [-1, -1], [-1, -1]]), ints([5, 0, 0])
        P.presto_pages_fork(refs, table, ctx, ints([0]), ints([1]), k, k.clone(), flags=f)
        assert f.item() == P.PRESTO_FLAG_NO_PAGES and ctx.tolist() == [5, 0, 0] and refs.tolist() == [1]
        ctx = ints([16, 0, 0])
        P.presto_pages_fork(refs, table, ctx, ints([0, 0]), ints([1, 2]), k, k.clone())
        assert ctx.tolist() == [16] * 3 and refs.tolist() == [3] and table[:, 0].tolist() == [0] * 3


@pytest.mark.parametrize("n", [1024, 1025, 3000])
def test_many_forks_at_once(n):
    """More forks than one workgroup keeps in LDS, children named twice among
    them, and fewer free pages than they need."""
    rng = np.random.default_rng([44, n])
    page, cols, parents, B = 16, 4, 40, n + 40
    ctx = [int(x) for x in rng.integers(1, cols * page + 1, parents)] + [0] * n
    used = [-(-c // page) for c in ctx]
    pages = sum(used) + n // 2
    order = iter(rng.permutation(pages).tolist())
    table = [[next(order) if x < u else -1 for x in range(cols)] for u in used]
    refs = [0] * pages
    for row in table:
        for e in row:
            refs[e] += e >= 0
    par = rng.integers(-1, parents, n).tolist()
    chi = (rng.permutation(n) + parents).tolist()
    for i in rng.integers(0, n, 50).tolist():
        chi[i] = int(rng.integers(0, B + 2))
    ref = R.Books(refs, table, ctx, page)
    dev = _books_on_device(ref)
    k, f = torch.randn(1, pages, page, 1, 64, device=DEV), flag()
    kh = k.cpu()
    P.presto_pages_fork(*dev, ints(par), ints(chi), k, k.clone(), flags=f)
    for s, t, r in ref.fork(par, chi):
        kh[:, t, :r] = kh[:, s, :r]
    _same_books(ref, *dev)
    assert f.item() == ref.flags and torch.equal(k.cpu(), kh)


def _dense(kv, q, pos0, window, sinks, dtype):
    k, v = (np.stack(x) for x in kv)
    return R.attention(q, k, v, pos0, window, sinks, None, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4)])
def test_a_serving_run(dtype, window, sinks):
    """Prompts, decode steps, forks, dropped sequences, trimmed and compacted
    pools, all as a program would run them, against K and V kept densely."""
    rng = np.random.default_rng([12, window])
    page, hq, hkv, d, B, pages = 16, 4, 2, 64, 6, 64
    k, v = (torch.full((pages, page, hkv, d), float("nan"), dtype=TYPES[dtype], device=DEV) for _ in range(2))
    refs, table, ctx = torch.zeros(pages, dtype=torch.int32, device=DEV), ints([[-1] * 16] * B), ints([0] * B)
    kv = [([], []) for _ in range(B)]
    f = flag()

    def step(new):
        nonlocal ctx
        offs = np.concatenate([[0], np.cumsum(new)]).tolist()
        q, kn, vn = (queries(rng, max(offs[-1], 1), h, d, dtype) for h in (hq, hkv, hkv))
        after = P.presto_pages_reserve(refs, table, ctx, page, ints(new), flags=f)
        P.presto_append_kv(kn, vn, ints(offs), max(new), k, v, table, ctx, after, flags=f)
        ctx = after
        if max(new) == 1 and min(new) == 1:
            out = P.presto_paged_attention(q, k, v, table, ctx, window=window, sinks=sinks, flags=f)
        else:
            out = P.presto_window_attention(q, ints(offs), max(new), k, v, table, ctx, window=window, sinks=sinks,
                                            flags=f)
        for b, n in enumerate(new):
            s = slice(offs[b], offs[b] + n)
            for dst, src in zip(kv[b], (kn, vn)):
                dst.extend(src[s].double().cpu().numpy())
            if n:
                want, bound = _dense(kv[b], q[s].double().cpu().numpy(), len(kv[b][0]) - n, window, sinks, dtype)
                got = out[s].double().cpu().numpy()
                assert (np.abs(got - want) <= bound).all(), (new, b)
        assert f.item() == 0

    step([37, 50, 0, 0, 0, 0])          # two prompts
    P.presto_pages_fork(refs, table, ctx, ints([0, 0, 1]), ints([2, 3, 4]), k, v, flags=f)
    for p, c in ((0, 2), (0, 3), (1, 4)):
        kv[c] = tuple(list(x) for x in kv[p])
    step([1, 1, 1, 1, 1, 70])           # decode, and a prompt beside it
    for _ in range(20):
        step([1] * B)
    if window:
        P.presto_pages_trim(refs, table, ctx, page, window, sinks, flags=f)
    P.presto_pages_free(refs, table, ctx, ints([0, 4]), flags=f)
    kv[0], kv[4] = ([], []), ([], [])
    step([0, 2, 3, 1, 33, 1])           # drafted chains, a new prompt in a dropped row
    out = P.presto_pages_compact(refs, table, k, v, flags=f)
    refs, table = out["refs"], out["page_table"]
    live = out["n_live"].item()
    assert (refs[:live] > 0).all() and not refs[live:].any() and table.max().item() < live
    step([5, 1, 1, 1, 1, 1])
    P.presto_pages_free(refs, table, ctx, ints(list(range(B))), flags=f)
    assert f.item() == 0 and not refs.any() and (table == -1).all() and not ctx.any()


def test_a_step_captured_into_a_graph():
    """Reserve, append and attention of a decode step, replayed with other
    inputs and eager work in between; every replay equals the eager step."""
    rng = np.random.default_rng(13)
    page, hq, hkv, d, B, pages = 16, 8, 2, 128, 3, 600
    c = Cache(rng, [30, 500, 2000], [1] * 3, page, hkv, d, "bf16", spare=0)
    k, v = (torch.zeros(pages, page, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    n0 = c.k.shape[0]
    k[:n0], v[:n0] = c.k.nan_to_num(), c.v.nan_to_num()
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    refs[:n0] = 1
    cols = 160
    table = torch.full((B, cols), -1, dtype=torch.int32, device=DEV)
    table[:, :c.table.shape[1]] = c.table
    q, kn, vn = (torch.zeros(B, h, d, dtype=torch.bfloat16, device=DEV) for h in (hq, hkv, hkv))
    offs = ints(list(range(B + 1)))

    def books():
        return dict(refs=refs.clone(), table=table.clone(), ctx=c.ctx.clone(), after=torch.empty_like(c.ctx),
                    k=k.clone(), v=v.clone(), out=torch.empty_like(q),
                    ws=P.paged_attention_workspace(q, k, table, max_ctx=2100), pws=P.pages_workspace(refs, table))

    def step(s):
        P.presto_pages_reserve(s["refs"], s["table"], s["ctx"], page, extra=1, out=s["after"], workspace=s["pws"])
        P.presto_append_kv(kn, vn, offs, 1, s["k"], s["v"], s["table"], s["ctx"], s["after"])
        P.presto_paged_attention(q, s["k"], s["v"], s["table"], s["after"], max_ctx=2100, out=s["out"],
                                 workspace=s["ws"])
        s["ctx"].copy_(s["after"])

    eager, cap = books(), books()
    warm = books()
    step(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cap)
    for i in range(20):
        for t in (q, kn, vn):
            t.copy_(torch.randn(t.shape, device=DEV))
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("refs", "table", "ctx", "k", "v", "out"):
            assert torch.equal(eager[name], cap[name]), (i, name)
    assert eager["ctx"].tolist() == [50, 520, 2020]


def test_calls_on_two_streams_and_a_given_one():
    rng = np.random.default_rng(14)
    c = Cache(rng, [3000, 100], [1, 1], 64, 2, 128, "bf16")
    q = queries(rng, 2, 4, 128, "bf16")
    want = P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [P.presto_paged_attention(q, c.k, c.v, c.table, c.ctx, stream=s) for _ in range(10) for s in (s1, s2)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_slots_read_as_pages():
    """A slot cache of presto_tree_attention is a pool of consecutive pages:
    one tree node decodes as one new token does."""
    rng = np.random.default_rng(15)
    hq, hkv, d, page, ctx = 8, 2, 128, 64, [700, 64]
    cache = [torch.from_numpy(rng.standard_normal((1024, hkv, d), dtype=np.float32)).to(DEV) for _ in range(2)]
    start = [128, 896]
    q = queries(rng, 2, hq, d, "f32")
    root = [torch.stack([x[s + n - 1] for s, n in zip(start, ctx)])[:, None].contiguous() for x in cache]
    tree = P.presto_tree_attention(q[:, None].contiguous(), cache[0], cache[1],
                                   ints([[s, n - 1] for s, n in zip(start, ctx)]), *root,
                                   torch.ones(2, 1, 1, dtype=torch.int64, device=DEV), ints([1, 1]), 1024,
                                   ctx_layout=P.PRESTO_CTX_SLOTS)
    pools = [x.view(16, page, hkv, d) for x in cache]
    table = ints([[s // page + i if i * page < n else -1 for i in range(11)] for s, n in zip(start, ctx)])
    out = P.presto_paged_attention(q, *pools, table, ints(ctx))
    for b, n in enumerate(ctx):
        kh, vh = (x[start[b]:start[b] + n].double().cpu().numpy() for x in cache)
        want, bound = R.attention(q[b:b + 1].double().cpu().numpy(), kh, vh, n - 1, dtype="f32")
        for got in (out[b], tree[b, 0]):
            assert (np.abs(got.double().cpu().numpy() - want[0]) <= bound[0]).all()


def test_binding_refusals():
    k = torch.zeros(4, 16, 2, 64, device=DEV)
    t, c, q = ints([[0, 1]]), ints([20]), torch.zeros(1, 4, 64, device=DEV)
    P.presto_paged_attention(q, k, k, t, c)
    bad = [dict(q=q.bfloat16()), dict(q=q[..., :32]), dict(q=q.cpu()), dict(k=k[:, :, :, ::2]), dict(k=k[:, ::2]),
           dict(v=k[:2]), dict(v=k.bfloat16()), dict(t=t.long()), dict(t=t.cpu()), dict(c=c.long()), dict(c=ints([1, 2])),
           dict(t=ints([[0, 1], [0, 1]])), dict(t=ints([[0, 1, 2, 3]])[:, ::2]), dict(k=k.half(), v=k.half(), q=q.half())]
    for over in bad:
        a = dict(q=q, k=k, v=k, t=t, c=c)
        a.update(over)
        with pytest.raises((ValueError, TypeError)):
            P.presto_paged_attention(a["q"], a["k"], a["v"], a["t"], a["c"])
    for kw in (dict(out=q.bfloat16()), dict(out=torch.zeros(2, 4, 64, device=DEV)), dict(flags=torch.zeros(1, device=DEV))):
        with pytest.raises(ValueError):
            P.presto_paged_attention(q, k, k, t, c, **kw)
    for kw in (dict(max_ctx=33), dict(window=-1), dict(scale=0.0)):
        with pytest.raises(P.PrestoError):
            P.presto_paged_attention(q, k, k, t, c, **kw)
    with pytest.raises(P.PrestoError):
        P.presto_paged_attention(torch.zeros(1, 3, 64, device=DEV), k, k, t, c)  # 3 query heads, 2 KV heads
    with pytest.raises(ValueError):
        P.presto_pages_fork(ints([0] * 3), t, c, ints([0]), ints([0]), k, k)  # 3 reference counts, 4 pages
    with pytest.raises(ValueError):
        P.presto_pages_compact(ints([0] * 4), t, k.expand(2, 4, 16, 2, 64), k.expand(2, 4, 16, 2, 64))
