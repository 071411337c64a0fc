"""The operators of a decoding step together, as a program uses them: append with
rotation, attention over the cache, a token drawn; captured into a graph, on
other streams, and prompt and single tokens against one another."""
import numpy as np
import pytest
import torch

import paper_2607_22634_amd as P
import step_ref as S
from test_gpu_paged_streams import _after_late_writes
from test_gpu_quant import Quant, dev, tight
from test_gpu_rope import ints, tensor

pytestmark = pytest.mark.gpu

HQ, HKV, D, PAGE, V = 8, 2, 128, 16, 1000


class Model:
    """One layer and a projection to logits: enough to decode with."""

    def __init__(self, batch, quant, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.batch, self.quant = batch, quant
        self.embed = torch.randn(V, (HQ + 2 * HKV) * D, device="cuda", generator=g).bfloat16()
        self.head = (torch.randn(HQ * D, V, device="cuda", generator=g) * 0.1).bfloat16()
        self.plan = P.rope_plan(96, base=1e4, interleaved=True)
        pages = 40
        self.refs, self.table, self.ctx = ints([0] * pages), ints([[-1] * 6] * batch), ints([0] * batch)
        if quant:
            self.k, self.v = (P.quant_pages(pages, PAGE, HKV, D) for _ in range(2))
        else:
            self.k, self.v = (torch.zeros(pages, PAGE, HKV, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.after = self.ctx.clone()
        self.temp = torch.full((batch,), 0.8, device="cuda")
        self.top_k = ints([50] * batch)

    def attend(self, q, offsets, max_new):
        if self.quant:
            return P.presto_quant_attention(q, self.k, self.v, self.table, self.after, q_offsets=offsets, max_q=max_new)
        return P.presto_window_attention(q, offsets, max_new, self.k, self.v, self.table, self.after)

    def step(self, tokens, offsets, max_new, add, u):
        """new tokens of all sequences; (logits of every token, the token drawn after each sequence's last)"""
        x = self.embed[tokens.long()].unflatten(1, (HQ + 2 * HKV, D))
        P.presto_pages_reserve(self.refs, self.table, self.ctx, PAGE, add, out=self.after)
        q = P.presto_append_rope(self.plan, x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], offsets, max_new, self.k, self.v,
                                 self.table, self.ctx, self.after)
        logits = self.attend(q, offsets, max_new).flatten(1) @ self.head
        self.ctx.copy_(self.after)
        token, logprob = P.presto_sample(logits[offsets[1:].long() - 1], u, temperature=self.temp, top_k=self.top_k)
        return logits, token, logprob


@pytest.mark.parametrize("quant", [False, True])
def test_a_prompt_at_once_and_token_by_token(quant):
    """The same cache and logits either way."""
    B, n = 3, 21
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(0, V, (B, n), device="cuda", generator=g, dtype=torch.int32)
    u = torch.full((B,), 0.5, device="cuda")
    a, b = Model(B, quant), Model(B, quant)
    la, ta, _ = a.step(tokens.flatten(), ints(np.arange(B + 1) * n), n, ints([n] * B), u)
    for i in range(n):
        lb, tb, _ = b.step(tokens[:, i], ints(np.arange(B + 1)), 1, ints([1] * B), u)
    assert torch.equal(a.ctx, b.ctx) and a.ctx.tolist() == [n] * B
    args = (ints([0] * B), a.ctx, ints(np.arange(B + 1) * n), n)
    for x, y in zip(P.presto_read_kv(a.k, a.v, a.table, *args, rows=B * n), P.presto_read_kv(b.k, b.v, b.table, *args, rows=B * n)):
        assert torch.equal(x, y)
    # the last logits: the attention's outputs differ by a rounding or two of
    # 2^-8 of the values' size, summed over 1024 products with weights of 0.1
    assert (la.view(B, n, V)[:, -1] - lb).float().abs().max() <= 2 * 2.0 ** -8 * 3 * 0.1 * 32 * 3


@pytest.mark.parametrize("quant", [False, True])
def test_a_step_in_a_graph(quant):
    """A captured step, replayed with new tokens and numbers between eager work,
    gives what the eager steps give, bit for bit."""
    B, steps = 5, 30
    g = torch.Generator(device="cuda").manual_seed(2)
    us = torch.rand(steps, B, device="cuda", generator=g)
    offsets, add = ints(np.arange(B + 1)), ints([1] * B)
    first = torch.randint(0, V, (B,), device="cuda", generator=g, dtype=torch.int32)

    eager, want, t = Model(B, quant), [], first
    for i in range(steps):
        _, t, lp = eager.step(t, offsets, 1, add, us[i])
        want.append((t.clone(), lp.clone()))

    m = Model(B, quant)
    token, u = first.clone(), us[0].clone()
    start = [x.clone() for x in (m.refs, m.table, m.ctx, m.after, m.k, m.v)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        m.step(token, offsets, 1, add, u)  # (warm up)
    torch.cuda.current_stream().wait_stream(s)
    for x, y in zip((m.refs, m.table, m.ctx, m.after, m.k, m.v), start):
        x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, t, lp = m.step(token, offsets, 1, add, u)
    for i in range(steps):
        u.copy_(us[i])
        graph.replay()
        if i % 7 == 0:
            torch.cuda.synchronize()
            torch.randn(1000, device="cuda").sum()
        assert torch.equal(t, want[i][0]) and torch.equal(lp, want[i][1]), i
        token.copy_(t)


def test_calls_on_another_stream():
    """Outputs and workspaces made for a call on a given stream."""
    rng = np.random.default_rng(30)
    c = Quant(rng, [9000, 40, 3000], 64, 2, 128)
    q = tensor(rng, (3, 8, 128), "bf16")
    plan, pos = P.rope_plan(128), ints([5, 6, 7])
    z, u = tensor(rng, (3, 50000), "f32"), torch.rand(3, device="cuda")
    args = (c.table, ints([0, 0, 0]), c.ctx, ints([0, 9000, 9040, 12040]), 9000)
    s = torch.cuda.Stream()
    ws = P.quant_attention_workspace(q, c.k, c.table)
    assert ws.numel() > 16  # cut, so that the call needs one
    kv = torch.Size((12040, 2, 128))
    for late, call in (
            ([(q.shape, q.dtype), (ws.shape, ws.dtype)], lambda **k: (P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, **k),)),
            ([(q.shape, q.dtype)], lambda **k: (P.presto_rope(q, pos, plan, **k),)),
            ([(kv, torch.bfloat16)] * 2, lambda **k: P.presto_read_kv(c.k, c.v, *args, rows=12040, **k)),
            ([((3,), torch.int32), ((3,), torch.float32)], lambda **k: P.presto_sample(z, u, **k))):
        want = call()
        for _ in range(2):
            got = _after_late_writes(late, lambda: call(stream=s))
            assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_two_streams_at_once():
    """Calls in flight together, each with a workspace of its own."""
    rng = np.random.default_rng(31)
    sets = [(Quant(rng, [5000, 700], 32, 2, 64), tensor(rng, (2, 6, 64), "bf16")) for _ in range(2)]
    want = [P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx) for c, q in sets]
    z = [tensor(rng, (40, 30000), "bf16") for _ in range(2)]
    u = torch.rand(40, device="cuda")
    drawn = [P.presto_sample(x, u) for x in z]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        got = []
        for (c, q), x, s in zip(sets, z, streams):
            got.append((P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, stream=s), *P.presto_sample(x, u, stream=s)))
        torch.cuda.synchronize()
        for g, w, d in zip(got, want, drawn):
            assert torch.equal(g[0], w) and torch.equal(g[1], d[0]) and torch.equal(g[2], d[1])


def test_nothing_but_its_outputs_is_written():
    """Guards around every output."""
    rng = np.random.default_rng(32)
    c = Quant(rng, [300, 5, 77], 16, 2, 64)
    q = tensor(rng, (3, 6, 64), "bf16")

    def guarded(shape, dtype):
        n = int(np.prod(shape)) * dtype.itemsize
        raw = torch.full((n + 512,), 0x5a, dtype=torch.uint8, device="cuda")
        return raw, raw[256:256 + n].view(dtype).view(shape)

    def check(raw):
        assert (raw[:256] == 0x5a).all() and (raw[-256:] == 0x5a).all()

    raw, out = guarded(q.shape, q.dtype)
    P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, out=out)
    check(raw)
    raw, out = guarded(q.shape, q.dtype)
    P.presto_rope(q, ints([1, 2, 3]), P.rope_plan(64), out=out)
    check(raw)
    (r1, a), (r2, b) = guarded((3,), torch.int32), guarded((3,), torch.float32)
    P.presto_sample(tensor(rng, (3, 999), "bf16"), torch.rand(3, device="cuda"), out=a, logprob=b)
    check(r1), check(r2)
    before = (c.k.clone(), c.v.clone())
    need = P.quant_attention_workspace(q, c.k, c.table).numel()
    raw, ws = guarded((max(need, 16),), torch.uint8)
    P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx, workspace=ws)
    check(raw)
    assert torch.equal(c.k, before[0]) and torch.equal(c.v, before[1])


def test_offsets_past_32_bits():
    """A pool whose last page lies beyond 2^32 bytes."""
    rng = np.random.default_rng(33)
    c = Quant(rng, [40], 16, 8, 128, spare=0)
    stride = 16 * 8 * 128 * 17 // 32
    n = (1 << 32) // stride + 8
    pools = [torch.empty(n, 8, 1, 1088, dtype=torch.uint8, device="cuda") for _ in range(2)]
    far = [n - 1, 3, n - 5]
    for x, e in enumerate(far):
        pools[0][e], pools[1][e] = c.k[c.table[0, x]], c.v[c.table[0, x]]
    q = tensor(rng, (1, 32, 128), "bf16")
    table = ints([far])
    assert torch.equal(P.presto_quant_attention(q, *pools, table, c.ctx), P.presto_quant_attention(q, c.k, c.v, c.table, c.ctx))
    k = tensor(rng, (1, 8, 128), "bf16")
    for pool, t in ((pools, table), ((c.k, c.v), c.table)):
        P.presto_append_rope(None, None, k, k, ints([0, 1]), 1, *pool, t, c.ctx, ints([41]))
    args = (ints([0]), ints([41]), ints([0, 41]), 41)
    for x, y in zip(P.presto_read_kv(*pools, table, *args, rows=41), P.presto_read_kv(c.k, c.v, c.table, *args, rows=41)):
        assert torch.equal(x, y)
