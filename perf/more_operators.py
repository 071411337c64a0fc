"""Performance cases of the operators around one step of plain decoding: the
rotation of queries and keys by their positions, the append that rotates on the
way, attention over a cache held in 4 bits, and the draw of a token.

Rotation: the pair (a, b) number i of a head at position p becomes
m (a cos t - b sin t, b cos t + a sin t) with t = p f_i; the first `rot` values
of a head rotate, in pairs (i, i + rot / 2) or, interleaved, (2 i, 2 i + 1).

A 4-bit cache holds every 32 values of a row as e2m1 codes (0, .5, 1, 1.5, 2,
3, 4, 6 and a sign) with one exponent byte E: code * 2^(E - 127), E the least
with 7 * 2^(E - 127) >= the largest magnitude, codes rounded to nearest even.
Pools are uint8 [pages, hkv, page / 16, 17 dim / 2]: of 16 positions of a head
the codes, then the exponents.  K: codes [16][dim / 2] in order, low nibble
first, and exponents [16][dim / 32].  V: with position 4 g + i and value x =
(dim / 16) n + y, codes [g][n][i][y / 2] and exponents [g][x / 32][i].

A token is drawn from logits z: weights w = exp((z - max z) / T), in order of z
(largest first, lower id first among equals) the first top_k of them, of those
the shortest head that has at least top_p of their sum, of those the ones of at
least min_p; then the first whose running sum exceeds u times their sum.

Shapes are those of the synthetic workloads (32 query and 8 KV heads of
dimension 128, vocabulary 151936, contexts of 1024 to 32768, 1 to 32 sequences
and more) and the ranges around them.
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

def _rope(rows, heads, dim, rot, inter, scaling, far, dtype="bf16", shape=1):
    return dict(kind="rope", rows=rows, heads=heads, dim=dim, rot=rot, inter=inter, scaling=scaling, far=far,
                dtype=dtype, shape=shape)


def _append(batch, new_lo, new_hi, past_lo, past_hi, quant, dtype="bf16", hq=32, hkv=8, dim=128, page=64, rot=128,
            inter=False, scaling="none", shape=1):
    return dict(kind="append", batch=batch, new_lo=new_lo, new_hi=new_hi, past_lo=past_lo, past_hi=past_hi,
                quant=quant, dtype=dtype, hq=hq, hkv=hkv, dim=dim, page=page, rot=rot, inter=inter, scaling=scaling,
                shape=shape)


def _attend(batch, q_lo, q_hi, past_lo, past_hi, dtype="bf16", hq=32, hkv=8, dim=128, page=64, window=0, sinks=0,
            shape=1):
    return dict(kind="attend", batch=batch, new_lo=q_lo, new_hi=q_hi, past_lo=past_lo, past_hi=past_hi, dtype=dtype,
                hq=hq, hkv=hkv, dim=dim, page=page, window=window, sinks=sinks, shape=shape)


def _sample(rows, vocab, settings, sigma=4.0, peaks=2, dtype="bf16", shape=1):
    return dict(kind="sample", rows=rows, vocab=vocab, settings=settings, sigma=sigma, peaks=peaks, dtype=dtype,
                shape=shape)


def listed():
    return [
        # the nodes of a batch of drafted trees before their verification:
        # queries and keys in a wider projection, positions by depth
        dict(name="rope-tree", **_rope(528, 40, 128, 128, False, "none", 8192)),
        # the prompts of a model with partly rotated heads, interleaved pairs
        # and frequencies stretched for long contexts
        dict(name="rope-long", **_rope(16384, 40, 128, 64, True, "ramp", 131072)),
        # a decode step of a serving batch into the bf16 cache
        dict(name="append-step", **_append(64, 1, 1, 1024, 8192, False, page=16, shape=2)),
        # ragged prompts written into the 4-bit cache
        dict(name="append-prompts", **_append(8, 500, 4096, 0, 2000, True, shape=3)),
        # a toy model in fp32, a few dozen cached tokens: launch latency
        dict(name="decode-tiny-f32", **_attend(1, 1, 1, 36, 36, "f32", 4, 2, 64, 16)),
        # a serving batch of ragged contexts in small pages
        dict(name="decode-ragged", **_attend(16, 1, 1, 1024, 8192, page=16, shape=4)),
        # long contexts, what a 4-bit cache is for: the cache is all of the work
        dict(name="decode-long", **_attend(16, 1, 1, 32767, 32767)),
        # one more chunk of a few prompts against what is cached of them
        dict(name="chunk", **_attend(4, 300, 512, 8000, 12288, shape=5)),
        # one interactive user
        dict(name="sample-single", **_sample(1, 151936, "usual")),
        # a serving batch, each request with settings of its own, some greedy
        dict(name="sample-serving", **_sample(64, 151936, "mixed", shape=6)),
        # draws from the whole distribution, as in collecting rollouts
        dict(name="sample-full", **_sample(512, 151936, "full", 2.0, 3, shape=7)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_SCALINGS = ("none", "none", "linear", "ramp", "logramp")


def draw(rng):
    kind = rng.choice(("rope", "append", "append", "decode", "decode", "chunk", "sample", "sample"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    shape = rng.randrange(10, 1 << 20)
    scaling, inter = rng.choice(_SCALINGS), rng.random() < 0.5
    if kind == "rope":
        dim = rng.choice((16, 32, 64, 72, 80, 96, 128, 128, 192, 256))
        rot = 2 * rng.randint(1, dim // 2) if rng.random() < 0.4 else dim
        heads = _log(rng, 1, 64)
        rows = _log(rng, 1, min(40000, 40000000 // (heads * dim)))
        return _rope(rows, heads, dim, rot, inter, scaling, _log(rng, 100, 1000000), dtype, shape)
    if kind == "sample":
        vocab = _log(rng, 200, 200000)
        rows = _log(rng, 1, min(1024, 40000000 // vocab))
        return _sample(rows, vocab, rng.choice(("usual", "mixed", "full")), rng.choice((1.0, 2.0, 4.0)),
                       rng.choice((0, 1, 3)), dtype, shape)
    hkv = rng.choice((1, 2, 4, 8))
    hq = hkv * rng.choice((1, 2, 3, 4, 5, 7, 8))
    dim, page = rng.choice((64, 128)), rng.choice((16, 32, 64, 128, 256))
    if kind == "append":
        rot = 2 * rng.randint(1, dim // 2) if rng.random() < 0.4 else dim
        batch = _log(rng, 1, 128)
        new_hi = _log(rng, 1, min(8192, 20000 // batch))
        past_hi = rng.choice((0, _log(rng, 1, min(16000, 100000 // batch))))
        return _append(batch, rng.choice((0, 1, new_hi)), new_hi, 0, past_hi, rng.random() < 0.6, dtype, hq, hkv, dim,
                       page, rot, inter, scaling, shape)
    window, sinks = 0, 0
    if rng.random() < 0.4:
        window, sinks = _log(rng, 1, 8000), rng.choice((0, 1, 4, 4, 33, 130))
    if kind == "decode":
        batch = _log(rng, 1, 128)
        hi = _log(rng, 1, min(65536, 400000 // batch))
        return _attend(batch, 1, 1, hi if rng.random() < 0.3 else _log(rng, 1, hi), hi, dtype, hq, hkv, dim, page,
                       window, sinks, shape)
    batch = _log(rng, 1, 16)
    q_hi = _log(rng, 2, min(1024, 4000 // batch))
    past_hi = rng.choice((0, _log(rng, 1, min(16000, 500000000 // (batch * q_hi * hq) - q_hi))))
    return _attend(batch, rng.choice((0, 1, q_hi, (q_hi + 1) // 2)), q_hi, rng.choice((0, past_hi)), past_hi, dtype,
                   hq, hkv, dim, page, window, sinks, shape)


# ---------------------------------------------------------------------------
# lengths, pages and frequencies: plain numbers that follow from the case alone

def _lengths(case, lo, hi, salt=0):
    rng = random.Random(case["shape"] * 7919 + salt)
    return [rng.randint(min(lo, hi), hi) for _ in range(case["batch"])]


def _plan(case):
    """(lengths before the call, new tokens, lengths after it)"""
    new = _lengths(case, case["new_lo"], case["new_hi"])
    new = new if any(new) else [1] + new[1:]
    past = _lengths(case, case["past_lo"], case["past_hi"], 1)
    return past, new, [p + n for p, n in zip(past, new)]


def _visible(case, p):
    """how many keys a query at position p sees"""
    w, s = case["window"], case["sinks"]
    return p + 1 if w == 0 or w > p else w + min(s, p + 1 - w)


def _covered(case, first, last):
    """how many keys the queries at positions first .. last see together"""
    w, s = case["window"], case["sinks"]
    if last < first:
        return 0
    lo = max(0, first - w + 1) if w else 0
    return last + 1 - lo + min(s, lo)


def _scaling(case):
    """(factor, original length, low, high, magnitude) of the case's frequencies"""
    return {"none": (1.0, 0.0, 0.0, 0.0, 1.0), "linear": (4.0, 0.0, 0.0, 0.0, 1.0), "ramp": (8.0, 8192.0, 1.0, 4.0, 1.0),
            "logramp": (16.0, 4096.0, 1.0, 32.0, 0.1 * math.log(16.0) + 1.0)}[case["scaling"]]


_BASE = 500000.0


def _frequencies(case):
    kind, rot = case["scaling"], case["rot"]
    factor, original, low, high, _ = _scaling(case)
    out = []
    for i in range(rot // 2):
        f = _BASE ** (-2.0 * i / rot)
        if kind == "linear":
            f /= factor
        elif kind in ("ramp", "logramp"):
            turns = original * f / (2.0 * math.pi)
            if kind == "ramp":
                keep = (turns - low) / (high - low)
            else:
                keep = (math.log(turns) - math.log(low)) / (math.log(high) - math.log(low))
            keep = min(max(keep, 0.0), 1.0)
            f = f * (keep + (1.0 - keep) / factor)
        out.append(f)
    return out


def work(case):
    e, kind = _esize(case), case["kind"]
    if kind == "rope":
        n = case["rows"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * e + 4 * case["rows"], "flops": 3 * n}
    if kind == "sample":
        return {"bytes": case["rows"] * (case["vocab"] * e + 24), "flops": 2 * case["rows"] * case["vocab"]}
    past, new, ctx = _plan(case)
    head, row = case["hq"] * case["dim"], case["hkv"] * case["dim"]
    if kind == "append":
        n = sum(new)
        held = row * 17 // 32 if case["quant"] else row * e
        back = 2 * (held + 2 * row) * n if case["quant"] else 0  # read back: out of the cache, and as bf16
        return {"bytes": (2 * head + 2 * row) * n * e + 2 * held * n + back, "flops": 3 * (head + row) * n}
    keys = sum(_covered(case, c - n, c - 1) for c, n in zip(ctx, new))
    pairs = sum(_visible(case, p) for c, n in zip(ctx, new) for p in range(c - n, c))
    return {"bytes": 2 * (row * 17 // 32) * keys + 2 * sum(new) * head * e, "flops": 4 * head * pairs}


def _pages_of(case, n):
    return (n + case["page"] - 1) // case["page"]


def _books(case):
    """(table rows, pages of the pool) of a shuffled pool, as after some hours of
    serving; pages that no query sees any more have been given back"""
    past, new, ctx = _plan(case)
    page, w = case["page"], case.get("window", 0)
    kept = []
    for c, n in zip(ctx, new):
        first = max(0, c - n - w) // page if w else 0
        kept.append([x for x in range(_pages_of(case, c)) if x >= first or x < _pages_of(case, case["sinks"])])
    pages = sum(len(k) for k in kept)
    pages += pages // 8 + 4
    order = list(range(pages))
    random.Random(case["shape"] + 29).shuffle(order)
    cols, table, at = max([1] + [_pages_of(case, c) for c in ctx]), [], 0
    for k in kept:
        row = [-1] * cols
        for x in k:
            row[x] = order[at]
            at += 1
        table.append(row)
    return table, pages


# ---------------------------------------------------------------------------
# the 4-bit format

def _encode(x):
    """codes [..., d] and exponent bytes [..., d / 32] (uint8) of the rows x [..., d]"""
    g = x.unflatten(-1, (-1, 32))
    m, k = torch.frexp(g.abs().amax(-1))
    e = torch.where(m <= 0.875, k - 3, k - 2)  # 7 = 0.875 * 2^3
    e = torch.where(m > 0, e, torch.full_like(e, -120)).clamp(min=-120)
    y = torch.ldexp(g, -e[..., None])
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = torch.where(torch.signbit(y), code + 8, code)
    return code.flatten(-2), (e + 127).to(torch.uint8)


def _pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _k_parts(pool, dim):
    """views of a K pool: codes [pages, hkv, blocks, 16, dim / 2], exponents [pages, hkv, blocks, 16, dim / 32]"""
    return pool[..., :8 * dim].unflatten(-1, (16, dim // 2)), pool[..., 8 * dim:].unflatten(-1, (16, dim // 32))


def _v_parts(pool, dim):
    """views of a V pool: codes [pages, hkv, blocks, 4, 16, 4, dim / 32], exponents [pages, hkv, blocks, 4, dim / 32, 4]"""
    return pool[..., :8 * dim].unflatten(-1, (4, 16, 4, dim // 32)), pool[..., 8 * dim:].unflatten(-1, (4, dim // 32, 4))


def _decode_values(packed, exps):
    """values (fp32) [..., d] of packed codes [..., d / 2] and exponents [..., d / 32]"""
    lut = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                       device=packed.device)
    code = torch.stack((packed & 15, packed >> 4), -1).flatten(-2).to(torch.int32)
    return torch.ldexp(lut[code].unflatten(-1, (-1, 32)), exps[..., None].to(torch.int32) - 127).flatten(-2)


# ---------------------------------------------------------------------------
# what a program has in hand before the call

def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt, kind = _dtype(case), case["kind"]
    st = dict(case=case)

    def normal(*shape, dtype=dt):
        return torch.randn(*shape, device=DEV, dtype=dtype, generator=gen)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)

    if kind == "sample":
        _prepare_sample(case, seed, st, normal, gen)
        return st
    dim = case["dim"]
    if kind in ("rope", "append"):
        st["freq"] = torch.tensor(_frequencies(case), dtype=torch.float64, device=DEV)
    if kind == "rope":
        # queries and keys at the front of the projection, values behind them
        wide = normal(case["rows"], (case["heads"] + 8) * dim)
        st["x"] = wide[:, :case["heads"] * dim].unflatten(1, (case["heads"], dim))
        st["pos"] = torch.randint(0, case["far"], (case["rows"],), device=DEV, generator=gen).to(torch.int32)
        if own:
            st["out"] = torch.empty(case["rows"], case["heads"], dim, device=DEV, dtype=dt)
    else:
        hq, hkv, page = case["hq"], case["hkv"], case["page"]
        past, new, ctx = _plan(case)
        table, pages = _books(case)
        offs = [0]
        for n in new:
            offs.append(offs[-1] + n)
        seq = [b for b, n in enumerate(new) for _ in range(n)]
        st |= dict(table=ints(table), ctx=ints(ctx), past=ints(past), offsets=ints(offs), max_new=max(new),
                   max_ctx=max(ctx), total=sum(ctx), seq=ints(seq).long(),
                   index=torch.arange(offs[-1], device=DEV) - ints(offs).long()[ints(seq).long()])
        if kind == "append":
            wide = normal(offs[-1], (hq + 2 * hkv) * dim).unflatten(1, (hq + 2 * hkv, dim))
            st["q"], st["k_new"], st["v_new"] = wide[:, :hq], wide[:, hq:hq + hkv], wide[:, hq + hkv:]
        else:
            st["q"] = normal(offs[-1], hq, dim)
        if kind == "attend" or case["quant"]:
            st["k"], st["v"] = (torch.empty(pages, hkv, page // 16, 17 * dim // 2, dtype=torch.uint8, device=DEV)
                                for _ in range(2))
            step = max(1, (1 << 27) // (page * hkv * dim))
            for p in range(0, pages, step):  # (a stretch of the pool at a time: room for its fp32 rows)
                n = min(step, pages - p)
                for name in ("k", "v"):
                    code, exps = _encode(normal(n, hkv, page // 16, 16, dim, dtype=torch.float32))
                    to = st[name][p:p + n]
                    if name == "k":
                        codes_to, exps_to = _k_parts(to, dim)
                        codes_to.copy_(_pack(code))
                        exps_to.copy_(exps)
                    else:
                        codes_to, exps_to = _v_parts(to, dim)
                        codes_to.copy_(_pack(code).unflatten(-1, (16, dim // 32)).unflatten(-3, (4, 4)).transpose(-2, -3))
                        exps_to.copy_(exps.unflatten(-2, (4, 4)).transpose(-1, -2))
        else:
            st["k"], st["v"] = normal(pages, page, hkv, dim), normal(pages, page, hkv, dim)
        if own:
            import paper_2607_22634_amd as P

            st["out"] = torch.empty(offs[-1], hq, dim, device=DEV, dtype=dt)
            if kind == "attend":
                st["ws"] = P.quant_attention_workspace(
                    st["q"], st["k"], st["table"], max_q=st["max_new"], max_ctx=st["max_ctx"], window=case["window"],
                    sinks=case["sinks"], total_ctx=st["total"])
            else:
                st["back"] = [torch.empty(offs[-1], hkv, dim, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    if own and kind in ("rope", "append"):
        import paper_2607_22634_amd as P

        factor, original, low, high, magnitude = _scaling(case)
        st["plan"] = P.rope_plan(case["rot"], base=_BASE, interleaved=case["inter"], factor=factor, original=original,
                                 low=low, high=high, ramp={"ramp": "turns", "logramp": "log"}.get(case["scaling"]),
                                 magnitude=magnitude, device=DEV)
    return st


def _prepare_sample(case, seed, st, normal, gen):
    rows, vocab = case["rows"], case["vocab"]
    z = normal(rows, vocab, dtype=torch.float32) * case["sigma"]
    if case["peaks"]:  # a few tokens that the model prefers
        at = torch.randint(0, vocab, (rows, case["peaks"]), device=DEV, generator=gen)
        height = 4 * torch.rand(rows, case["peaks"], device=DEV, generator=gen)
        z.scatter_(1, at, z.amax(1, keepdim=True) + height)
    st["logits"] = z.to(_dtype(case))
    st["u"] = torch.rand(rows, device=DEV, generator=gen)
    st["temperature"] = torch.ones(rows, device=DEV)
    st["top_k"] = st["top_p"] = st["min_p"] = None
    rng = random.Random(case["shape"])

    def pick(choices, dtype=torch.float32):
        return torch.tensor([rng.choice(choices) for _ in range(rows)], dtype=dtype, device=DEV)

    if case["settings"] == "usual":
        st["temperature"], st["top_k"] = pick((0.6, 0.7, 1.0)), pick((20, 50), torch.int32)
        st["top_p"] = pick((0.8, 0.9, 0.95))
    elif case["settings"] == "mixed":
        st["temperature"] = pick((0.0, 0.3, 0.7, 1.0, 1.5))
        st["top_k"] = pick((0, 0, 1, 7, 40, 1000, vocab), torch.int32)
        st["top_p"], st["min_p"] = pick((1.0, 1.0, 0.5, 0.9, 0.95, 0.999)), pick((0.0, 0.0, 0.02, 0.1))
    if own:
        import paper_2607_22634_amd as P

        st["token"] = torch.empty(rows, dtype=torch.int32, device=DEV)
        st["logprob"] = torch.empty(rows, device=DEV)
        st["ws"] = P.sample_workspace(st["logits"])


# ---------------------------------------------------------------------------
# one pass

def run(st):
    return (_run_own if own else _run_plain)[st["case"]["kind"]](st)


def _own_rope(st):
    import paper_2607_22634_amd as P

    return P.presto_rope(st["x"], st["pos"], st["plan"], out=st["out"])


def _own_append(st):
    import paper_2607_22634_amd as P

    q = P.presto_append_rope(st["plan"], st["q"], st["k_new"], st["v_new"], st["offsets"], st["max_new"], st["k"],
                             st["v"], st["table"], st["past"], st["ctx"], out=st["out"])
    if not st["case"]["quant"]:
        return q, st["k"], st["v"]
    k, v = P.presto_read_kv(st["k"], st["v"], st["table"], st["past"], st["ctx"], st["offsets"], st["max_new"],
                            out=st["back"])
    return q, k, v


def _own_attend(st):
    import paper_2607_22634_amd as P

    c = st["case"]
    return P.presto_quant_attention(st["q"], st["k"], st["v"], st["table"], st["ctx"], q_offsets=st["offsets"],
                                    max_q=st["max_new"], max_ctx=st["max_ctx"], window=c["window"], sinks=c["sinks"],
                                    total_ctx=st["total"], out=st["out"], workspace=st["ws"])


def _own_sample(st):
    import paper_2607_22634_amd as P

    return P.presto_sample(st["logits"], st["u"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                           min_p=st["min_p"], out=st["token"], logprob=st["logprob"], workspace=st["ws"])


def _rotate(st, x, pos, wide=torch.float32):
    """x [rows, heads, dim] rotated by its rows' positions, in the type `wide`"""
    c, rot = st["case"], st["case"]["rot"]
    turn = pos.double()[:, None] * st["freq"]
    magnitude = _scaling(c)[4]
    cos = (torch.cos(turn) * magnitude).to(wide)[:, None]
    sin = (torch.sin(turn) * magnitude).to(wide)[:, None]
    x = x.to(wide)
    if c["inter"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, x[..., rot:]), -1)


def _plain_rope(st):
    return _rotate(st, st["x"], st["pos"]).to(st["x"].dtype)


def _plain_append(st):
    c, seq = st["case"], st["seq"]
    pos = st["past"].long()[seq] + st["index"]
    at, row = st["table"].long()[seq, pos // c["page"]], pos % c["page"]
    q = _rotate(st, st["q"], pos).to(st["q"].dtype)
    if not c["quant"]:
        st["k"][at, row] = _rotate(st, st["k_new"], pos).to(st["k"].dtype)
        st["v"][at, row] = st["v_new"]
        return q, st["k"], st["v"]
    dim, blk, r = c["dim"], row // 16, row % 16
    k_codes, k_exps = _k_parts(st["k"], dim)
    v_codes, v_exps = _v_parts(st["v"], dim)
    # (in 64 bits: bf16 keys often lie on the border of two codes, and a turn by a
    # small angle leaves them a hair to one side of it)
    code, exps = _encode(_rotate(st, st["k_new"], pos, torch.float64))
    k_codes[at, :, blk, r], k_exps[at, :, blk, r] = _pack(code), exps
    code, exps = _encode(st["v_new"].float())
    v_codes[at, :, blk, r // 4, :, r % 4] = _pack(code).unflatten(-1, (16, dim // 32))
    v_exps[at, :, blk, r // 4, :, r % 4] = exps
    # and what the cache holds now
    k = _decode_values(k_codes[at, :, blk, r], k_exps[at, :, blk, r])
    v = _decode_values(v_codes[at, :, blk, r // 4, :, r % 4].flatten(-2), v_exps[at, :, blk, r // 4, :, r % 4])
    return q, k.to(torch.bfloat16), v.to(torch.bfloat16)


def _plain_attend(st):
    c, table, seq = st["case"], st["table"].clamp(min=0).long(), st["seq"]
    dim, hkv, hq, batch = c["dim"], c["hkv"], c["hq"], c["batch"]
    group, n = hq // hkv, st["max_new"]
    # every sequence's cache in order, as fp32 [batch, hkv, positions, dim]
    codes, exps = _k_parts(st["k"], dim)
    k = _decode_values(codes[table], exps[table]).transpose(1, 2).flatten(2, 4)
    codes, exps = _v_parts(st["v"], dim)
    v = _decode_values(codes[table].transpose(-2, -3).flatten(-2).flatten(-3, -2),
                       exps[table].transpose(-1, -2).flatten(-3, -2)).transpose(1, 2).flatten(2, 4)
    # the queries as [batch, hkv, (query, head), dim], rows of padding at the end of the short ones
    q = torch.zeros(batch, n, hq, dim, device=DEV)
    q[seq, st["index"]] = st["q"].float()
    q = q.unflatten(2, (hkv, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(dim ** -0.5).unflatten(2, (n, group))
    j = torch.arange(k.shape[2], device=DEV)
    new = (st["offsets"][1:] - st["offsets"][:-1]).long()
    p = ((st["ctx"].long() - new)[:, None] + torch.arange(n, device=DEV))[:, None, :, None, None]
    seen = j <= p
    if c["window"]:
        seen &= (j > p - c["window"]) | (j < c["sinks"])
    s.masked_fill_(~seen, float("-inf"))
    s -= s.amax(-1, keepdim=True)
    s.exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.flatten(2, 3), v).unflatten(2, (n, group)) / total
    return o.permute(0, 2, 1, 3, 4).flatten(2, 3)[seq, st["index"]].to(st["q"].dtype)


def _plain_sample(st):
    z, order = st["logits"].float().sort(dim=1, descending=True, stable=True)
    vocab = z.shape[1]
    t = st["temperature"].double()[:, None]
    greedy = t <= 0
    w = torch.exp((z - z[:, :1]).double() / torch.where(greedy, torch.ones_like(t), t))
    rank = torch.arange(vocab, device=DEV)
    if st["top_k"] is not None:
        k = st["top_k"].long()[:, None]
        w = torch.where(rank < torch.where(k <= 0, vocab, k), w, 0.0)
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        before = w.cumsum(1) - w
        w = torch.where((before < p * w.sum(1, keepdim=True)) | (p >= 1), w, 0.0)
    if st["min_p"] is not None:
        w = torch.where(w >= st["min_p"].double()[:, None], w, 0.0)
    w = torch.where(greedy & (rank > 0), 0.0, w)
    run = w.cumsum(1)
    total = run[:, -1:]
    at = torch.searchsorted(run, st["u"].double()[:, None] * total, right=True).clamp(max=vocab - 1)
    logprob = torch.log(w.gather(1, at) / total)[:, 0]
    return order.gather(1, at)[:, 0].to(torch.int32), logprob.float()


_run_own = dict(rope=_own_rope, append=_own_append, attend=_own_attend, sample=_own_sample)
_run_plain = dict(rope=_plain_rope, append=_plain_append, attend=_plain_attend, sample=_plain_sample)


# ---------------------------------------------------------------------------
# the definitions in 64 bits

def _turned(case, x, pos):
    """rotation as a product of complex numbers"""
    rot, rate = case["rot"], torch.tensor(_frequencies(case), dtype=torch.float64, device=DEV)
    angle = torch.outer(pos.double(), rate)
    unit = torch.polar(torch.full_like(angle, _scaling(case)[4]), angle)[:, None, :]
    y = x.double().clone()
    even, odd = (slice(0, rot, 2), slice(1, rot, 2)) if case["inter"] else (slice(0, rot // 2), slice(rot // 2, rot))
    turned = torch.complex(y[..., even].contiguous(), y[..., odd].contiguous()) * unit
    y[..., even], y[..., odd] = turned.real, turned.imag
    return y


def _nearest(x):
    """the values that the 4-bit format holds for the rows x (fp64)"""
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    scale = 2.0 ** torch.ceil(torch.log2(top.clamp(min=2.0 ** -110) / 7.0))
    y = g / scale
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
    return ((y / step).round() * step).clamp(-6, 6).mul(scale).flatten(-2)


def _held(pool, table, page, dim, head, length, is_v):
    """fp64 values [length, dim] of one sequence and KV head, byte by byte from the layout"""
    j = torch.arange(length, device=DEV)
    where = table.long()[j // page].clamp(min=0)
    block = pool[where, head, (j % page) // 16].long()  # [length, 17 dim / 2]
    r, x = (j % 16)[:, None], torch.arange(dim, device=DEV)[None, :]
    if is_v:
        per = dim // 16
        at = (((r // 4) * 16 + x // per) * 4 + r % 4) * (per // 2) + (x % per) // 2
        ex = 8 * dim + ((r // 4) * (dim // 32) + x // 32) * 4 + r % 4
    else:
        at, ex = r * (dim // 2) + x // 2, 8 * dim + r * (dim // 32) + x // 32
    nibble = (block.gather(1, at.expand(length, dim)) >> (4 * (x % 2))) & 15
    size = nibble & 7
    # e2m1: sign, two bits of exponent, one of mantissa
    mag = torch.where(size < 2, size.double() / 2, (1 + (size % 2).double() / 2) * 2.0 ** (size // 2 - 1).double())
    return torch.where(nibble > 7, -mag, mag) * 2.0 ** (block.gather(1, ex.expand(length, dim)) - 127).double()


def exact(case, seed):
    kind = case["kind"]
    if kind == "attend" and work(case)["flops"] > 4e12:
        return None
    st = prepare(case, seed)
    if kind == "rope":
        return _turned(case, st["x"], st["pos"])
    if kind == "append":
        pos = st["past"].double()[st["seq"]] + st["index"]
        q, k, v = _turned(case, st["q"], pos), _turned(case, st["k_new"], pos), st["v_new"].double()
        if case["quant"]:
            return q, _nearest(k), _nearest(v)
        at, row = st["table"].long()[st["seq"], (pos // case["page"]).long()], (pos % case["page"]).long()
        pools = [st["k"].double(), st["v"].double()]
        pools[0][at, row], pools[1][at, row] = k, v
        return q, pools[0], pools[1]
    if kind == "attend":
        past, new, ctx = _plan(case)
        w, sinks, group, dim = case["window"], case["sinks"], case["hq"] // case["hkv"], case["dim"]
        out, at = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV), 0
        for b, (n, length) in enumerate(zip(new, ctx)):
            j = torch.arange(length, device=DEV)
            p = torch.arange(length - n, length, device=DEV)[:, None]
            seen = (j <= p) & ((p - j < w) | (j < sinks)) if w else j <= p
            for h in range(case["hkv"] if n else 0):
                k, v = (_held(st[name], st["table"][b], case["page"], dim, h, length, name == "v") for name in "kv")
                for g in range(h * group, (h + 1) * group):
                    s = (st["q"][at:at + n, g].double() @ k.t().contiguous() / math.sqrt(dim)).masked_fill(~seen, -math.inf)
                    s = torch.exp(s - s.max(1, keepdim=True).values)
                    out[at:at + n, g] = (s / s.sum(1, keepdim=True)) @ v
            at += n
        return out
    return _exact_sample(case, st)


def _exact_sample(case, st):
    """one row after the other, the lists cut as the definition says"""
    tokens, logs = [], []
    for r in range(case["rows"]):
        z = st["logits"][r].double()
        order = torch.argsort(z, descending=True, stable=True)
        t = float(st["temperature"][r])
        if t <= 0:
            tokens.append(order[0])
            logs.append(torch.zeros((), dtype=torch.float64, device=DEV))
            continue
        w = torch.exp((z[order] - z[order[0]]) / t)
        if st["top_k"] is not None and int(st["top_k"][r]) > 0:
            w = w[:int(st["top_k"][r])]
        if st["top_p"] is not None and float(st["top_p"][r]) < 1:
            w = w[:int((torch.cumsum(w, 0) < float(st["top_p"][r]) * w.sum()).sum()) + 1]
        if st["min_p"] is not None:
            w = w[w >= float(st["min_p"][r])]
        n = min(int((torch.cumsum(w, 0) <= float(st["u"][r]) * w.sum()).sum()), w.numel() - 1)
        tokens.append(order[n])
        logs.append(torch.log(w[n] / w.sum()))
    return torch.stack(tokens).to(torch.int32), torch.stack(logs)
