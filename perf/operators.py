"""Performance cases of the paged KV cache: the attention that reads it, the
append that fills it and the bookkeeping of its pages.

A cache is a pool of pages [pages, page, hkv, dim] for K and one for V; the
page table [sequences, columns] int32 names the page of every `page`
consecutive positions of a sequence (-1: none), `ctx` [sequences] int32 its
length and `refs` [pages] int32 how many table entries hold a page.  Position
j is visible to a query at position p when j <= p and, with a window, j > p -
window or j < sinks.

Shapes are those of the synthetic workloads (32 query and 8 KV heads of
dimension 128, contexts of 1024 to 32768, 1 to 32 sequences, 36 layers) and
the ranges around them.
"""
import math
import random

import torch

own = False

DEV = "cuda"


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _esize(case):
    return 2 if case["dtype"] == "bf16" else 4


# ---------------------------------------------------------------------------
# the cases

def _decode(batch, lo, hi, dtype="bf16", hq=32, hkv=8, dim=128, page=64, window=0, sinks=0, shape=1):
    return dict(kind="decode", batch=batch, ctx_lo=lo, ctx_hi=hi, dtype=dtype, hq=hq, hkv=hkv, dim=dim, page=page,
                window=window, sinks=sinks, shape=shape)


def _prompt(batch, q_lo, q_hi, past_lo, past_hi, dtype="bf16", hq=32, hkv=8, dim=128, page=64, window=0, sinks=0,
            shape=1):
    return dict(kind="prompt", batch=batch, q_lo=q_lo, q_hi=q_hi, past_lo=past_lo, past_hi=past_hi, dtype=dtype,
                hq=hq, hkv=hkv, dim=dim, page=page, window=window, sinks=sinks, shape=shape)


def _append(batch, new_lo, new_hi, past_lo, past_hi, dtype="bf16", hkv=8, dim=128, page=64, shape=1):
    return dict(kind="append", batch=batch, new_lo=new_lo, new_hi=new_hi, past_lo=past_lo, past_hi=past_hi,
                dtype=dtype, hkv=hkv, dim=dim, page=page, shape=shape)


def _fork(batch, forks, lo, hi, layers, dtype="bf16", hkv=8, dim=128, page=64, shape=1):
    return dict(kind="fork", batch=batch, forks=forks, ctx_lo=lo, ctx_hi=hi, layers=layers, dtype=dtype, hkv=hkv,
                dim=dim, page=page, shape=shape)


def _compact(batch, lo, hi, layers, drop, dtype="bf16", hkv=8, dim=128, page=64, shape=1):
    return dict(kind="compact", batch=batch, ctx_lo=lo, ctx_hi=hi, layers=layers, drop=drop, dtype=dtype, hkv=hkv,
                dim=dim, page=page, shape=shape)


def listed():
    return [
        # the smallest call: a toy model in fp32 as one debugs with, a few
        # dozen cached tokens; launch latency
        dict(name="decode-tiny-f32", **_decode(1, 37, 37, "f32", 4, 2, 64, 16)),
        # interactive decoding of one sequence, one layer
        dict(name="decode-single", **_decode(1, 4096, 4096)),
        # a serving batch of ragged contexts in small pages
        dict(name="decode-ragged", **_decode(16, 1024, 8192, page=16, shape=3)),
        # long contexts: the cache is all of the work
        dict(name="decode-long", **_decode(16, 32768, 32768)),
        # a model with a sliding window and sinks deep in long sequences, the
        # pages outside the window given back
        dict(name="decode-window", **_decode(32, 6000, 32768, page=16, window=4096, sinks=4, shape=5)),
        # short ragged prompts of the toy model with a window
        dict(name="prompt-tiny-f32", **_prompt(3, 1, 77, 0, 50, "f32", 4, 2, 64, 16, window=48, sinks=4, shape=2)),
        # ragged prompts of a windowed model, some of them in their second chunk
        dict(name="prompt-window", **_prompt(4, 1000, 4096, 0, 4096, page=16, window=1024, sinks=4, shape=4)),
        # the chunk of a long prompt against all that is cached of it
        dict(name="prompt-long", **_prompt(4, 2048, 2048, 30720, 30720)),
        # a decode step of a serving batch: a page where the last one is full,
        # one token's K/V written
        dict(name="append-step", **_append(64, 1, 1, 1024, 8192, page=16, shape=6)),
        # ragged prompts written into the cache
        dict(name="append-prompts", **_append(8, 500, 4096, 0, 2000, shape=7)),
        # best-of-n sampling, 36 layers: the losers' pages given back, their
        # rows taken by forks of the others
        dict(name="pages-fork", **_fork(32, 16, 200, 2000, 36, page=16, shape=8)),
        # after half of the sequences have gone: the live pages moved to the
        # front of the pool, so that its tail can be given back
        dict(name="pages-compact", **_compact(16, 500, 2048, 36, 8, shape=9)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("decode", "decode", "prompt", "prompt", "append", "fork", "compact"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    hkv = rng.choice((1, 2, 4, 8))
    hq = hkv * rng.choice((1, 2, 3, 4, 5, 7, 8))
    dim = rng.choice((64, 128))
    page = rng.choice((16, 32, 64, 128, 256))
    shape = rng.randrange(10, 1 << 20)
    window, sinks = 0, 0
    if rng.random() < 0.5:
        window = _log(rng, 1, 8000)
        sinks = rng.choice((0, 1, 4, 4, 33, 130))
    if kind == "decode":
        batch = _log(rng, 1, 128)
        hi = _log(rng, 1, min(65536, 400000 // batch))
        lo = hi if rng.random() < 0.3 else _log(rng, 1, hi)
        return _decode(batch, lo, hi, dtype, hq, hkv, dim, page, window, sinks, shape)
    if kind == "prompt":
        batch = _log(rng, 1, 16)
        q_hi = _log(rng, 1, min(4096, 12000 // batch))
        q_lo = rng.choice((0, 1, q_hi, (q_hi + 1) // 2))
        past_hi = rng.choice((0, _log(rng, 1, 16000)))
        return _prompt(batch, q_lo, q_hi, rng.choice((0, past_hi)), past_hi, dtype, hq, hkv, dim, page, window, sinks,
                       shape)
    if kind == "append":
        batch = _log(rng, 1, 128)
        new_hi = _log(rng, 1, min(8192, 40000 // batch))
        new_lo = rng.choice((0, 1, new_hi))
        past_hi = rng.choice((0, _log(rng, 1, min(16000, 200000 // batch))))
        return _append(batch, new_lo, new_hi, 0, past_hi, dtype, hkv, dim, page, shape)
    layers = rng.choice((1, 2, 7, 24, 36))
    batch = _log(rng, 2, 48)
    hi = _log(rng, 1, min(4000, 1500000 // (batch * layers)))
    lo = rng.choice((1, hi, (hi + 1) // 2))
    if kind == "fork":
        return _fork(batch, rng.randint(1, batch // 2), lo, hi, layers, dtype, hkv, dim, page, shape)
    return _compact(batch, lo, hi, layers, rng.randint(0, batch), dtype, hkv, dim, page, shape)


# ---------------------------------------------------------------------------
# lengths and the pages in use: plain numbers that follow from the case alone

def _lengths(case, lo, hi, salt=0):
    rng = random.Random(case["shape"] * 7919 + salt)
    return [rng.randint(min(lo, hi), hi) for _ in range(case["batch"])]


def _some(new):
    return new if any(new) else [1] + new[1:]


def _plan(case):
    """(lengths before the call, new tokens, lengths after it)"""
    kind = case["kind"]
    if kind == "prompt":
        new = _some(_lengths(case, case["q_lo"], case["q_hi"]))
        past = _lengths(case, case["past_lo"], case["past_hi"], 1)
        return past, new, [p + n for p, n in zip(past, new)]
    if kind == "append":
        new = _some(_lengths(case, case["new_lo"], case["new_hi"]))
        past = _lengths(case, case["past_lo"], case["past_hi"], 1)
        return past, new, [p + n for p, n in zip(past, new)]
    ctx = _lengths(case, case["ctx_lo"], case["ctx_hi"])
    if kind == "decode":
        return ctx, [1] * len(ctx), ctx
    return ctx, [0] * len(ctx), ctx


def _visible(case, p):
    """how many keys a query at position p sees"""
    w, s = case["window"], case["sinks"]
    if p < 0:
        return 0
    if w == 0 or w > p:
        return p + 1
    return w + min(s, p + 1 - w)


def _covered(case, first, last):
    """how many keys the queries at positions first .. last see together"""
    w, s = case["window"], case["sinks"]
    if last < 0 or last < first:
        return 0
    if w == 0:
        return last + 1
    lo = max(0, max(first, 0) - w + 1)
    return last + 1 - lo + min(s, lo)


def work(case):
    e, kind = _esize(case), case["kind"]
    row = case["hkv"] * case["dim"] * e
    past, new, ctx = _plan(case)
    if kind in ("decode", "prompt"):
        head = case["hq"] * case["dim"]
        keys = sum(_covered(case, c - n, c - 1) for c, n in zip(ctx, new))
        pairs = sum(_visible(case, p) for c, n in zip(ctx, new) for p in range(c - n, c))
        return {"bytes": 2 * row * keys + 2 * sum(new) * head * e, "flops": 4 * head * pairs}
    if kind == "append":
        return {"bytes": 4 * row * sum(new), "flops": 0}
    page, layers = case["page"], case["layers"]
    if kind == "fork":
        return {"bytes": 4 * row * layers * sum(ctx[p] % page for p in _parents(case)), "flops": 0}
    moved = _moved(case)
    return {"bytes": 4 * row * page * layers * moved + 8 * _pool_pages(case), "flops": 0}


def _parents(case):
    """the sequences forked from: the upper half of the rows is the losers"""
    rng = random.Random(case["shape"] + 17)
    return [rng.randrange(case["batch"] - case["forks"]) for _ in range(case["forks"])]


def _pages_of(case, n):
    return (n + case["page"] - 1) // case["page"]


def _pool_pages(case):
    """pages of the pool: what the case holds at the end and some to spare"""
    past, new, ctx = _plan(case)
    pages = sum(_pages_of(case, c) for c in ctx)
    if case["kind"] == "fork":
        pages += case["forks"]
    if case.get("window"):
        pages = sum(len(_kept(case, c, n)) for c, n in zip(ctx, new))
    return pages + pages // 8 + 4


def _kept(case, c, n):
    """table columns of a sequence of length c that queries from position
    c - n on can still see (the others have been given back)"""
    cols, w = _pages_of(case, c), case.get("window", 0)
    if not w:
        return list(range(cols))
    first = max(0, c - n - w) // case["page"]
    head = _pages_of(case, case["sinks"])
    return [x for x in range(cols) if x < head or x >= first]


def _order(case, pages):
    """the order in which the pool's pages were handed out: a shuffled pool, as
    after some hours of serving"""
    order = list(range(pages))
    random.Random(case["shape"] + 29).shuffle(order)
    return order


def _dropped(case):
    rng = random.Random(case["shape"] + 31)
    return sorted(rng.sample(range(case["batch"]), case["drop"]))


def _moved(case):
    refs = _books(case)[1]
    live = sum(1 for r in refs if r > 0)
    return sum(1 for r in refs[live:] if r > 0)


def _books(case):
    """table rows, reference counts and lengths that a pass starts from"""
    past, new, ctx = _plan(case)
    kind, pages = case["kind"], _pool_pages(case)
    order = _order(case, pages)
    cols = max([1] + [_pages_of(case, c) for c in ctx]) + 1
    table, refs, at = [], [0] * pages, 0
    held = past if kind == "append" else ctx
    gone = set(_dropped(case)) if kind == "compact" else set()
    for b, c in enumerate(held):
        row = [-1] * cols
        if b not in gone:
            for x in (_kept(case, c, new[b]) if kind in ("decode", "prompt") else range(_pages_of(case, c))):
                row[x] = order[at]
                refs[order[at]] += 1
                at += 1
        elif kind == "compact":
            at += _pages_of(case, c)
        table.append(row)
    lens = [0 if b in gone else c for b, c in enumerate(held)]
    return table, refs, lens


# ---------------------------------------------------------------------------
# what a program has in hand before the call

def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt, kind = _dtype(case), case["kind"]
    hkv, dim, page = case["hkv"], case["dim"], case["page"]
    past, new, ctx = _plan(case)
    pages = _pool_pages(case)
    layers = case.get("layers", 0)

    def normal(*shape):
        return torch.randn(*shape, device=DEV, dtype=dt, generator=gen)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)

    table, refs, lens = _books(case)
    lead = (layers,) if layers else ()
    st = dict(case=case, k=normal(*lead, pages, page, hkv, dim), v=normal(*lead, pages, page, hkv, dim),
              table=ints(table), refs=ints(refs), ctx=ints(lens), past=past, new=new, lens=ctx,
              max_ctx=max(ctx), total=sum(ctx))
    offs = [0]
    for n in new:
        offs.append(offs[-1] + n)
    if kind == "decode":
        st["q"] = normal(case["batch"], case["hq"], dim)
    elif kind == "prompt":
        st["q"] = normal(offs[-1], case["hq"], dim)
    elif kind == "append":
        st["k_new"] = normal(offs[-1], hkv, dim)
        st["v_new"] = normal(offs[-1], hkv, dim)
        st["add"] = ints(new)
    elif kind == "fork":
        losers = list(range(case["batch"] - case["forks"], case["batch"]))
        st["parent"], st["child"] = ints(_parents(case)), ints(losers)
        st["parent_idx"], st["child_idx"] = st["parent"].long(), st["child"].long()
    st["offsets"], st["offs"], st["max_new"] = ints(offs), offs, max(new)
    if own:
        import paper_2607_22634_amd as P

        if kind in ("decode", "prompt"):
            st["out"] = torch.empty_like(st["q"])
            st["ws"] = P.paged_attention_workspace(
                st["q"], st["k"], st["table"], max_q=1 if kind == "decode" else st["max_new"],
                max_ctx=st["max_ctx"], window=case["window"], sinks=case["sinks"], total_ctx=st["total"])
        else:
            st["ws"] = P.pages_workspace(st["refs"], st["table"])
            st["ctx_new"] = torch.empty_like(st["ctx"])
            st["out"] = dict(refs=torch.empty_like(st["refs"]), page_table=torch.empty_like(st["table"]),
                             n_live=torch.empty(1, dtype=torch.int32, device=DEV))
    return st


# ---------------------------------------------------------------------------
# one pass

def run(st):
    return (_run_own if own else _run_plain)[st["case"]["kind"]](st)


def _own_decode(st):
    import paper_2607_22634_amd as P

    c = st["case"]
    return P.presto_paged_attention(st["q"], st["k"], st["v"], st["table"], st["ctx"], max_ctx=st["max_ctx"],
                                    window=c["window"], sinks=c["sinks"], total_ctx=st["total"], out=st["out"],
                                    workspace=st["ws"])


def _own_prompt(st):
    import paper_2607_22634_amd as P

    c = st["case"]
    return P.presto_window_attention(st["q"], st["offsets"], st["max_new"], st["k"], st["v"], st["table"], st["ctx"],
                                     max_ctx=st["max_ctx"], window=c["window"], sinks=c["sinks"],
                                     total_ctx=st["total"], out=st["out"], workspace=st["ws"])


def _own_append(st):
    import paper_2607_22634_amd as P

    ctx = P.presto_pages_reserve(st["refs"], st["table"], st["ctx"], st["case"]["page"], st["add"],
                                 out=st["ctx_new"], workspace=st["ws"])
    P.presto_append_kv(st["k_new"], st["v_new"], st["offsets"], st["max_new"], st["k"], st["v"], st["table"],
                       st["ctx"], ctx)
    return st["k"], st["v"], st["table"], st["refs"], ctx


def _own_fork(st):
    import paper_2607_22634_amd as P

    P.presto_pages_free(st["refs"], st["table"], st["ctx"], st["child"])
    P.presto_pages_fork(st["refs"], st["table"], st["ctx"], st["parent"], st["child"], st["k"], st["v"],
                        workspace=st["ws"])
    return st["k"], st["v"], st["table"], st["refs"], st["ctx"]


def _own_compact(st):
    import paper_2607_22634_amd as P

    got = P.presto_pages_compact(st["refs"], st["table"], st["k"], st["v"], out=st["out"], workspace=st["ws"])
    return st["k"], st["v"], got["page_table"], got["refs"], got["n_live"]


def _rows(pool, table, b, n):
    """the first n cached rows of sequence b, [n, hkv, dim] (a page that is
    not there reads as page 0: nothing sees its positions)"""
    page = pool.shape[1]
    ids = table[b, :(n + page - 1) // page].clamp(min=0).long()
    return pool[ids].flatten(0, 1)[:n]


def _attend(q, k, v, pos0, window, sinks, wide):
    """softmax attention of q [n, hq, d] at positions pos0 .. over k, v
    [L, hkv, d] in the type `wide`, one KV head and a bounded number of score
    rows at a time"""
    n, hq, d = q.shape
    hkv, length = k.shape[1], k.shape[0]
    group = hq // hkv
    out = torch.zeros(n, hq, d, dtype=wide, device=q.device)
    if n == 0 or length == 0:
        return out
    cols = torch.arange(length, device=q.device)
    step = max(1, (1 << 28) // (group * length))
    for g in range(hkv):
        kg, vg = k[:, g].to(wide), v[:, g].to(wide)
        for i in range(0, n, step):
            m = min(step, n - i)
            qg = q[i:i + m, g * group:(g + 1) * group].to(wide).reshape(m * group, d)
            s = (qg @ kg.t().contiguous() * d ** -0.5).reshape(m, group, length)
            pos = pos0 + i + torch.arange(m, device=q.device)[:, None]
            seen = cols <= pos
            if window:
                seen &= (cols > pos - window) | (cols < sinks)
            s = torch.where(seen[:, None], s, torch.full((), float("-inf"), dtype=wide, device=q.device))
            top = s.amax(-1, keepdim=True).clamp(min=torch.finfo(wide).min)
            e = torch.exp(s - top)
            z = e.sum(-1, keepdim=True)
            o = (e.reshape(m * group, length) @ vg).reshape(m, group, d)
            out[i:i + m, g * group:(g + 1) * group] = torch.where(z > 0, o / z.clamp(min=1e-30), torch.zeros_like(o))
    return out


def _attend_all(st, wide):
    c, out = st["case"], []
    for b, (n, total) in enumerate(zip(st["new"], st["lens"])):
        q = st["q"][st["offs"][b]:st["offs"][b] + n]
        out.append(_attend(q, _rows(st["k"], st["table"], b, total), _rows(st["v"], st["table"], b, total),
                           total - n, c["window"], c["sinks"], wide))
    return torch.cat(out)


def _plain_attention(st):
    return _attend_all(st, torch.float32).to(st["q"].dtype)


def _plain_append(st):
    c, page = st["case"], st["case"]["page"]
    table, refs, ctx = st["table"], st["refs"], st["ctx"]
    ctx_new = ctx + st["add"]
    # the pages that are missing, in order of sequence and column, get the
    # lowest free ones in order
    col = torch.arange(table.shape[1], device=DEV)
    need = (col >= ((ctx + page - 1) // page)[:, None]) & (col < ((ctx_new + page - 1) // page)[:, None]) & (table < 0)
    free = torch.argsort((refs > 0).to(torch.uint8), stable=True)
    rank = (need.flatten().cumsum(0) - 1).clamp(min=0, max=refs.numel() - 1)
    ids = free[rank].reshape(need.shape)
    table.copy_(torch.where(need, ids.to(torch.int32), table))
    refs.scatter_add_(0, ids.flatten(), need.flatten().to(torch.int32))
    for b, n in enumerate(st["new"]):
        pos = st["past"][b] + torch.arange(n, device=DEV)
        at = table[b, pos // page].long()
        src = slice(st["offs"][b], st["offs"][b] + n)
        st["k"][at, pos % page] = st["k_new"][src]
        st["v"][at, pos % page] = st["v_new"][src]
    return st["k"], st["v"], table, refs, ctx_new


def _plain_fork(st):
    page, table, refs, ctx = st["case"]["page"], st["table"], st["refs"], st["ctx"]
    parent, child = st["parent_idx"], st["child_idx"]
    # the losers' references go
    old = table[child]
    refs.scatter_add_(0, old.clamp(min=0).flatten().long(), -(old >= 0).flatten().to(torch.int32))
    table[child] = -1
    ctx[child] = 0
    # a child shares its parent's full pages and copies what the last one holds
    rows, n = table[parent], ctx[parent]
    full, part = (n // page)[:, None], n % page > 0
    col = torch.arange(table.shape[1], device=DEV)
    shared = (col < full) & (rows >= 0)
    refs.scatter_add_(0, rows.clamp(min=0).flatten().long(), shared.flatten().to(torch.int32))
    free = torch.argsort((refs > 0).to(torch.uint8), stable=True)
    # (a fork without a partial page copies some other free page onto itself)
    ids = part.to(torch.int64)
    rank = torch.where(part, ids.cumsum(0) - 1, ids.sum() + (1 - ids).cumsum(0) - 1)
    fresh = free[rank]
    last = torch.where(part, rows.gather(1, full.long().clamp(max=table.shape[1] - 1))[:, 0].long(), fresh)
    kept = torch.where(shared, rows, torch.full_like(rows, -1))
    table[child] = torch.where((col == full) & part[:, None], fresh.to(torch.int32)[:, None], kept)
    refs.scatter_add_(0, fresh, part.to(torch.int32))
    ctx[child] = n
    filled = (torch.arange(page, device=DEV) < (n % page)[:, None])[:, :, None, None]
    for pool in (st["k"], st["v"]):
        pool[:, fresh] = torch.where(filled, pool[:, last], pool[:, fresh])
    return st["k"], st["v"], table, refs, ctx


def _plain_compact(st):
    table, refs = st["table"], st["refs"]
    pages = refs.numel()
    live, at = refs > 0, torch.arange(pages, device=DEV)
    n_live = live.sum()
    src = torch.argsort((~(live & (at >= n_live))).to(torch.uint8), stable=True)
    dst = torch.argsort((~(~live & (at < n_live))).to(torch.uint8), stable=True)
    moves = (live & (at >= n_live)).sum()
    half = pages // 2 + 1
    src, dst = src[:half], dst[:half]
    src = torch.where(torch.arange(src.numel(), device=DEV) < moves, src, dst)  # past the moves: onto itself
    new_id = torch.where(live, at, torch.full_like(at, -1))
    slot = torch.where(src == dst, pages, src)  # (one slot more takes what does not move)
    to = torch.full((pages + 1,), -1, device=DEV).scatter_(0, slot, dst)[:pages]
    new_id = torch.where(live & (at >= n_live), to, new_id)
    out_refs = torch.zeros_like(refs).scatter_add_(0, new_id.clamp(min=0), torch.where(live, refs, 0))
    out_table = torch.where(table >= 0, new_id[table.clamp(min=0).long()].to(torch.int32), table)
    st["k"][:, dst] = st["k"][:, src]
    st["v"][:, dst] = st["v"][:, src]
    return st["k"], st["v"], out_table, out_refs, n_live.to(torch.int32).reshape(1)


_run_own = dict(decode=_own_decode, prompt=_own_prompt, append=_own_append, fork=_own_fork, compact=_own_compact)
_run_plain = dict(decode=_plain_attention, prompt=_plain_attention, append=_plain_append, fork=_plain_fork,
                  compact=_plain_compact)


# ---------------------------------------------------------------------------
# the definition in 64 bits

def exact(case, seed):
    if case["kind"] not in ("decode", "prompt"):
        return None  # copies and whole numbers
    if work(case)["flops"] > 8e12:
        return None
    st = prepare(case, seed)
    group, d, page = case["hq"] // case["hkv"], case["dim"], case["page"]
    w, sinks = case["window"], case["sinks"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    for b, (n, total) in enumerate(zip(st["new"], st["lens"])):
        # the rows by position, then one query head and a stretch of queries
        # at a time: a masked score takes no part in the sums at all
        j = torch.arange(total, device=DEV)
        at = st["table"][b].long()[j // page].clamp(min=0)
        for h in range(case["hq"] if n else 0):
            k = st["k"][at, j % page, h // group].double()
            v = st["v"][at, j % page, h // group].double()
            step = max(1, (1 << 26) // max(total, 1))
            for i in range(0, n, step):
                m = min(step, n - i)
                r = st["offs"][b] + i
                p = torch.arange(total - n + i, total - n + i + m, device=DEV)[:, None]
                seen = (j <= p) & ((p - j < w) | (j < sinks)) if w else j <= p
                s = st["q"][r:r + m, h].double() @ k.t().contiguous() / math.sqrt(d)
                s = s.masked_fill(~seen, -math.inf)
                s = torch.exp(s - s.max(1, keepdim=True).values)
                out[r:r + m, h] = (s / s.sum(1, keepdim=True)) @ v
    return out
