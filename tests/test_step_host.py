"""Host-only checks of the operators around a decoding step: what they refuse
before anything is launched, the table of angles, workspaces, and the references
themselves (no GPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2607_22634_amd as P
import step_ref as S

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: the checks fail first
BAD, OK = P.PRESTO_ERR_INVALID_ARG, P.PRESTO_OK


def pages(**over):
    d = P.PagesDesc(4, 64, 300, 16, 8, 128, P.PRESTO_DT_FP4, 1, 0, 0)
    for k, v in over.items():
        setattr(d, k, v)
    return d


def attn(pool=None, **over):
    d = P.PagedAttnDesc(pool or pages(), 32, 8, 1000, 0, 0, 0.1, 32, 0, 0)
    for k, v in over.items():
        setattr(d, k, v)
    return d


def append(pool=None, **over):
    d = P.AppendDesc(pool or pages(), P.PRESTO_DT_BF16, 32, 3, 4, 0, 0, 0, 0)
    for k, v in over.items():
        setattr(d, k, v)
    return d


def rope(**over):
    d = P.RopeDesc(128, 0, 1.0)
    for k, v in over.items():
        setattr(d, k, v)
    return d


# ---------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(factor=4.0), dict(base=0.5),
                                dict(base=500000.0, factor=8.0, original=8192.0, low=1.0, high=4.0, ramp="turns"),
                                dict(base=10000.0, factor=40.0, original=4096.0, low=1.0, high=32.0, ramp="log")])
@pytest.mark.parametrize("rot", [2, 20, 64, 128, 256])
def test_steps_are_fractions_of_a_turn(rot, kw):
    steps = P.presto_rope_steps(rot, **kw).numpy().view(np.uint64)
    want = S.frequencies(rot, **kw) / (2 * math.pi)
    # pow and the ramp round by a few 2^-53 of the frequency; a word holds 2^-64
    err = (steps.astype(np.float64) * 2.0 ** -64 - want % 1.0 + 0.5) % 1.0 - 0.5
    assert (np.abs(err) <= 16 * 2.0 ** -53 * np.maximum(want, 2.0 ** -9)).all()


def test_steps_of_given_frequencies():
    f = [0.0, 1.0, 2 * math.pi, math.pi, -1.0, 1e5, 1e-9]
    steps = P.presto_rope_steps(14, frequencies=f).numpy().view(np.uint64).astype(np.float64) * 2.0 ** -64
    want = np.array(f) / (2 * math.pi)
    err = (steps - want % 1.0 + 0.5) % 1.0 - 0.5
    assert (np.abs(err) <= 4 * 2.0 ** -53 * np.maximum(np.abs(want), 1)).all()


@pytest.mark.parametrize("rot,kw", [(0, {}), (3, {}), (258, {}), (-2, {}), (64, dict(base=0.0)), (64, dict(base=math.nan)),
                                    (64, dict(base=math.inf)), (64, dict(factor=0.0)), (64, dict(factor=-1.0)),
                                    (64, dict(ramp="turns", low=1.0, high=4.0)),
                                    (64, dict(ramp="turns", original=8.0, low=4.0, high=4.0)),
                                    (64, dict(ramp="log", original=8.0, low=0.0, high=4.0)),
                                    (64, dict(ramp="log", original=8.0, low=1.0, high=math.inf)),
                                    (4, dict(frequencies=[1.0, math.nan])), (4, dict(frequencies=[1.0, 2.0 ** 20])),
                                    (64, dict(base=1e-9)), (64, dict(factor=1e-7))])
def test_steps_refuse(rot, kw):
    with pytest.raises(P.PrestoError) as e:
        P.presto_rope_steps(rot, **kw)
    assert e.value.status == BAD


def test_steps_binding_refuses():
    with pytest.raises(ValueError):
        P.presto_rope_steps(8, ramp="yes")
    with pytest.raises(ValueError):
        P.presto_rope_steps(8, frequencies=[1.0])
    with pytest.raises(ValueError):
        P.presto_rope_steps(1 << 40)


def _rope(r=None, steps=FAKE, dt=0, x=FAKE, xs=0, rows=4, heads=8, dim=128, pos=FAKE, out=ctypes.c_void_p(0x2000), os=0):
    return P.lib().presto_rope(None if r is False else ctypes.byref(r or rope()), steps, dt, x, xs, rows, heads, dim,
                               pos, out, os, None)


@pytest.mark.parametrize("kw", [dict(r=False), dict(dt=2), dict(dt=7), dict(rows=-1), dict(rows=1 << 31), dict(heads=0),
                                dict(heads=65537), dict(dim=0), dict(dim=12), dict(dim=264), dict(xs=1016), dict(xs=1028),
                                dict(os=1016), dict(os=1 << 40), dict(steps=None), dict(steps=ctypes.c_void_p(0x1004)),
                                dict(x=None), dict(pos=None), dict(out=None), dict(x=ctypes.c_void_p(0x1008)),
                                dict(out=ctypes.c_void_p(0x2004)), dict(x=FAKE, out=FAKE, os=2048),
                                dict(r=rope(rot_dim=130)), dict(r=rope(rot_dim=7)), dict(r=rope(rot_dim=-2)),
                                dict(r=rope(interleaved=2)), dict(r=rope(magnitude=math.nan))])
def test_rope_refuses(kw):
    assert _rope(**kw) == BAD
    assert b"presto_rope" in P.lib().presto_last_error()


def test_rope_of_no_rows():
    assert _rope(rows=0, x=None, pos=None, out=None, steps=None) == OK


def _append(d=None, r=None, steps=FAKE, q=FAKE, k=FAKE, v=FAKE, off=FAKE, qo=ctypes.c_void_p(0x2000), kp=FAKE, vp=FAKE,
            table=FAKE, ctx=FAKE, new=FAKE):
    return P.lib().presto_append_rope(None if d is False else ctypes.byref(d or append()), ctypes.byref(r or rope()), steps,
                                      q, k, v, off, qo, kp, vp, table, ctx, new, None, None)


BAD_POOLS = [dict(page_size=8), dict(page_size=48), dict(head_dim=96), dict(hkv=0), dict(num_pages=0), dict(max_pages=0),
             dict(batch=-1), dict(dt=7), dict(layers=0), dict(page_stride=16 * 8 * 68 - 16), dict(page_stride=16 * 8 * 68 + 8),
             dict(layer_stride=-16)]
BAD_APPENDS = [dict(dt=2), dict(dt=5), dict(new_rows=-1), dict(new_rows=1 << 31), dict(max_new=-1), dict(max_new=1 << 22),
               dict(k_stride=1016), dict(k_stride=1028), dict(v_stride=8), dict(v_stride=1 << 40)]


@pytest.mark.parametrize("over", BAD_POOLS)
def test_cache_calls_refuse_bad_pools(over):
    d = pages(**over)
    assert _append(append(d)) == BAD
    assert P.lib().presto_read_kv(ctypes.byref(append(d)), *[FAKE] * 8, None, None) == BAD
    a = attn(d)
    assert P.lib().presto_quant_attention(ctypes.byref(a), 0, *[FAKE] * 7, None, FAKE, 1 << 40, None) == BAD or over == {}
    assert P.lib().presto_quant_attention_workspace(ctypes.byref(a), 0, 1) == 0


@pytest.mark.parametrize("over", BAD_APPENDS + [dict(hq=-1), dict(hq=65537), dict(q_stride=8), dict(q_out_stride=4097)])
def test_append_refuses_bad_descriptors(over):
    assert _append(append(**over)) == BAD
    assert b"presto_append_rope" in P.lib().presto_last_error()


@pytest.mark.parametrize("over", BAD_APPENDS)
def test_read_refuses_bad_descriptors(over):
    assert P.lib().presto_read_kv(ctypes.byref(append(**over)), *[FAKE] * 8, None, None) == BAD


@pytest.mark.parametrize("kw", [dict(d=False), dict(k=None), dict(v=None), dict(off=None), dict(qo=None), dict(kp=None),
                                dict(vp=None), dict(table=None), dict(ctx=None), dict(new=None), dict(steps=None),
                                dict(k=ctypes.c_void_p(0x1008)), dict(q=ctypes.c_void_p(0x1002)),
                                dict(vp=ctypes.c_void_p(0x1004)), dict(r=rope(rot_dim=130)), dict(r=rope(interleaved=-1)),
                                dict(q=FAKE, qo=FAKE, d=append(q_out_stride=8192))])
def test_append_refuses_bad_tensors(kw):
    assert _append(**kw) == BAD


def test_append_refuses_rows_and_pool_of_different_types():
    assert _append(append(pages(dt=P.PRESTO_DT_F32))) == BAD
    assert _append(append(pages(dt=P.PRESTO_DT_BF16), dt=P.PRESTO_DT_F32)) == BAD


def test_empty_appends_do_nothing():
    none = [None] * 12
    for d in (append(pages(batch=0)), append(max_new=0), append(new_rows=0)):
        assert P.lib().presto_append_rope(ctypes.byref(d), None, *none, None) == OK
        assert P.lib().presto_read_kv(ctypes.byref(d), *[None] * 10) == OK
    assert P.lib().presto_read_kv(ctypes.byref(append()), *[FAKE] * 6, None, None, None, None) == OK  # no output


def test_four_bit_pools_are_refused_where_nothing_reads_them():
    d = pages()
    a = P.PagedAttnDesc(d, 32, 8, 1000, 0, 0, 0.1, 32, 0, 0)
    lib = P.lib()
    assert lib.presto_paged_attention(ctypes.byref(a), *[FAKE] * 6, None, FAKE, 1 << 40, None) == BAD
    assert lib.presto_window_attention(ctypes.byref(a), *[FAKE] * 7, None, FAKE, 1 << 40, None) == BAD
    assert lib.presto_paged_attention_workspace(ctypes.byref(a)) == 0
    assert lib.presto_append_kv(ctypes.byref(d), FAKE, FAKE, 4, 0, FAKE, 3, *[FAKE] * 5, None, None) == BAD
    assert lib.presto_topk(2, None, 4, 1024, 1024, 2, *[None] * 6, 0, None) == BAD


BAD_ATTN = [dict(hq=12), dict(hq=0), dict(max_ctx=-1), dict(max_ctx=64 * 16 + 1), dict(max_q=-1), dict(window=-1),
            dict(window=(1 << 30) + 1), dict(sinks=-1), dict(scale=0.0), dict(scale=math.nan), dict(total_q=-1),
            dict(total_q=1 << 30), dict(total_ctx=-1), dict(q_stride=32 * 128 - 8), dict(q_stride=32 * 128 + 4),
            dict(max_q=1 << 30)]


@pytest.mark.parametrize("over", BAD_ATTN)
def test_attention_refuses_bad_descriptors(over):
    a = attn(**over)
    assert P.lib().presto_quant_attention(ctypes.byref(a), 0, *[FAKE] * 7, None, FAKE, 1 << 40, None) == BAD
    assert b"presto_quant_attention" in P.lib().presto_last_error()
    assert P.lib().presto_quant_attention_workspace(ctypes.byref(a), 0, 1) == 0


def test_attention_refuses_types_tensors_and_workspaces():
    lib = P.lib()
    a = attn()
    for dt in (2, 3, -1):
        assert lib.presto_quant_attention(ctypes.byref(a), dt, *[FAKE] * 7, None, FAKE, 1 << 40, None) == BAD
    for pool in (pages(dt=0), pages(dt=1)):
        assert lib.presto_quant_attention(ctypes.byref(attn(pool)), 0, *[FAKE] * 7, None, FAKE, 1 << 40, None) == BAD
    assert lib.presto_quant_attention(None, 0, *[FAKE] * 7, None, FAKE, 1 << 40, None) == BAD
    for i in (0, 2, 3, 4, 5, 6):
        args = [FAKE] * 7
        args[i] = None
        assert lib.presto_quant_attention(ctypes.byref(a), 0, *args, None, FAKE, 1 << 40, None) == BAD
    for i in (0, 2, 3, 6):
        args = [FAKE] * 7
        args[i] = ctypes.c_void_p(0x1008)
        assert lib.presto_quant_attention(ctypes.byref(a), 0, *args, None, FAKE, 1 << 40, None) == BAD
    d = attn(pages(batch=1, max_pages=4096), max_q=1, max_ctx=60000, total_q=1)
    need = lib.presto_quant_attention_workspace(ctypes.byref(d), 0, 0)
    assert need > 0 and need == lib.presto_quant_attention_workspace(ctypes.byref(d), 0, 1)
    for ws, nb in ((FAKE, need - 1), (None, need)):
        assert lib.presto_quant_attention(ctypes.byref(d), 0, FAKE, None, *[FAKE] * 5, None, ws, nb, None) == \
            P.PRESTO_ERR_WORKSPACE
    assert lib.presto_quant_attention(ctypes.byref(d), 0, FAKE, None, *[FAKE] * 5, None, ctypes.c_void_p(0x1008), need,
                                      None) == BAD
    for e in (attn(pages(batch=0)), attn(max_q=0), attn(total_q=0)):
        assert lib.presto_quant_attention(ctypes.byref(e), 0, None, FAKE, *[None] * 7, 0, None) == OK
    big = attn(pages(batch=(1 << 23) - 1, max_pages=2), max_ctx=32, max_q=1, total_q=(1 << 23) - 1)
    assert lib.presto_quant_attention(ctypes.byref(big), 0, *[FAKE] * 7, None, FAKE, 1 << 40, None) == \
        P.PRESTO_ERR_UNSUPPORTED


@pytest.mark.parametrize("dt", [0, 1])
def test_attention_workspaces_hold_the_partials(dt):
    """Either none or room for one partial of every row at least, the same each
    time it is asked for, and never beyond 2^23 workgroups."""
    for hkv, d in ((1, 64), (8, 128)):
        for batch in (1, 5, 70, 3000):
            for ctx in (0, 17, 4100, 150000):
                for n in (1, 7, 300):
                    for window, total in ((0, 0), (500, 0), (0, 1)):
                        pool = pages(batch=batch, max_pages=9400, hkv=hkv, head_dim=d)
                        a = attn(pool, hq=hkv * 4, max_q=n, max_ctx=ctx, window=window, sinks=4, total_q=batch * n,
                                 total_ctx=total * batch * ctx)
                        need = P.lib().presto_quant_attention_workspace(ctypes.byref(a), dt, 1)
                        assert need == P.lib().presto_quant_attention_workspace(ctypes.byref(a), dt, 1)
                        assert need == 0 or need >= batch * hkv * 4 * n * (d * 2 + 8)


def _sample(dt=0, z=FAKE, rows=4, vocab=1000, stride=1000, u=FAKE, token=FAKE):
    return P.lib().presto_sample(dt, z, rows, vocab, stride, u, None, None, None, None, token, None, None, FAKE, 1 << 40,
                                 None)


@pytest.mark.parametrize("kw", [dict(dt=2), dict(dt=9), dict(z=None), dict(u=None), dict(token=None), dict(rows=-1),
                                dict(rows=(1 << 21) + 1), dict(vocab=0), dict(vocab=(1 << 20) + 1, stride=1 << 21),
                                dict(stride=999), dict(stride=1 << 41), dict(z=ctypes.c_void_p(0x1001)),
                                dict(dt=1, z=ctypes.c_void_p(0x1002))])
def test_sample_refuses(kw):
    assert _sample(**kw) == BAD
    assert b"presto_sample" in P.lib().presto_last_error()


def test_sample_of_no_rows():
    assert _sample(rows=0, z=None, u=None, token=None) == OK


def test_binding_refuses_host_tensors_and_wrong_shapes():
    z = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        P.presto_sample(z, torch.zeros(2))
    with pytest.raises(ValueError):
        P.presto_sample(torch.zeros(8, 2).t(), torch.zeros(2))
    with pytest.raises(ValueError, match="overlap"):
        P.presto_sample(torch.zeros(1, 8).expand(2, 8), torch.zeros(2))
    with pytest.raises(TypeError):
        P.presto_sample(z.half(), torch.zeros(2))
    plan = P.rope_plan(64, device="cpu")
    with pytest.raises(ValueError):
        P.presto_rope(torch.zeros(2, 4, 64), torch.zeros(2, dtype=torch.int32), plan)
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    pool = P.quant_pages(3, 16, 2, 64, device="cpu")
    assert pool.shape == (3, 2, 1, 544)
    t, c = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        P.presto_quant_attention(q, pool, pool, t, c)
    with pytest.raises(TypeError):
        P.presto_quant_attention(q, torch.zeros(3, 16, 2, 64), torch.zeros(3, 16, 2, 64), t, c)
    with pytest.raises(ValueError, match="17 dim"):
        P.quant_attention_workspace(q, torch.zeros(3, 2, 1, 545, dtype=torch.uint8), t)
    with pytest.raises(ValueError):
        P.quant_pages(3, 24, 2, 64, device="cpu")
    with pytest.raises(ValueError):
        P.presto_append_rope(plan, q, q[:, :2], q[:, :2], torch.zeros(2, dtype=torch.int32), 1, pool, pool, t, c, c)


# ---------------------------------------------------------------------------
# the references

def test_reference_rotation_by_hand():
    x = np.array([[[3.0, 4.0, 5.0, 7.0]]])
    y, _ = S.rotate(x, [1], np.array([math.pi / 2]))  # one pair: values 0 and 1
    assert np.allclose(y, [[[-4, 3, 5, 7]]])
    y, _ = S.rotate(x, [1], np.array([math.pi / 2, math.pi]))
    assert np.allclose(y, [[[-5, -4, 3, -7]]])
    y, _ = S.rotate(x, [1], np.array([math.pi / 2, math.pi]), True, 2.0)
    assert np.allclose(y, [[[-8, 6, -10, -14]]])


def test_reference_format_by_hand():
    x = np.zeros(32)
    x[:8] = [7.0, 0.25, 0.26, -1.75, 2.5, 3.5, -5.0, 5.01]
    code, e = S.encode(x)
    assert e.tolist() == [127]
    assert S.decode(code, e)[:8].tolist() == [6.0, 0.0, 0.5, -2.0, 2.0, 4.0, -4.0, 6.0]
    x[0] = 7.01
    assert S.encode(x)[1].tolist() == [128]
    assert S.encode(np.full(32, 1.75 * 2.0 ** -118))[1].tolist() == [7]
    assert S.encode(np.full(32, 1.75 * 2.0 ** -117))[1].tolist() == [8]
    assert S.encode(np.zeros(32))[1].tolist() == [7]
    x[5] = np.nan
    assert S.encode(x)[1].tolist() == [255] and np.isnan(S.held(x)).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("is_v", [False, True])
def test_reference_layout_is_one_to_one(dim, is_v):
    co, eo = S.offsets(dim, is_v)
    assert sorted(co[:, ::2].ravel().tolist()) == list(range(8 * dim)) and (co[:, ::2] == co[:, 1::2]).all()
    assert sorted(eo[:, ::32].ravel().tolist()) == list(range(8 * dim, 17 * dim // 2))
    rng = np.random.default_rng(1)
    pool = rng.integers(0, 256, (3, 2, 4, 17 * dim // 2), dtype=np.uint8)
    page, row = np.array([2, 0, 2, 1]), np.array([5, 63, 17, 16])
    x = rng.standard_normal((4, 2, dim))
    S.write(pool, is_v, page, row, *S.encode(x))
    assert (S.read(pool, is_v, page, row) == S.held(x)).all()


def test_reference_draw_by_hand():
    z = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert [S.sample(z, u)[0] for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.91, 0.999)] == [1, 1, 3, 3, 2, 0, 0]
    assert [S.sample(z, u, top_k=2)[0] for u in (0.5, 0.6, 0.99)] == [1, 3, 3]
    assert [S.sample(z, u, top_p=0.7001)[0] for u in (0.4, 0.5, 0.8)] == [1, 3, 2]
    assert [S.sample(z, u, min_p=0.6)[0] for u in (0.5, 0.6)] == [1, 3]
    assert S.sample(z, 0.99, temperature=0.0)[0] == 1
    assert S.sample(z, 0.99, top_p=0.0)[0] == 1
    assert math.isclose(S.sample(z, 0.6, top_k=2)[1], math.log(3 / 7))
    assert S.sample(np.array([1.0, -np.inf, 1.0]), 0.9999)[0] == 2
