"""Plain references of the operators around a decoding step, in 64 bits and from
their definitions: rotation, the 4-bit format with its layout byte by byte, and
the draw of a token."""
from __future__ import annotations

import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def frequencies(rot, base=10000.0, factor=1.0, original=0.0, low=0.0, high=0.0, ramp=None):
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if ramp is None:
            out.append(f / factor)
            continue
        r = original * f / (2 * math.pi)
        g = (r - low) / (high - low) if ramp == "turns" else math.log(r / low) / math.log(high / low)
        g = min(max(g, 0.0), 1.0)
        out.append(f * g + f * (1 - g) / factor)
    return np.array(out)


def pairs(rot, interleaved):
    """indexes of the first and second values of the pairs"""
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotate(x, pos, freq, interleaved=False, magnitude=1.0):
    """x [n, heads, dim] (fp64) at positions pos [n], and the size of the terms
    of each output, |a| + |b| (0 where nothing turns)"""
    rot = 2 * len(freq)
    a, b = pairs(rot, interleaved)
    t = (np.asarray(pos, dtype=np.float64)[:, None] * freq)[:, None]
    y, size = x.copy(), np.zeros_like(x)
    y[..., a] = magnitude * (x[..., a] * np.cos(t) - x[..., b] * np.sin(t))
    y[..., b] = magnitude * (x[..., b] * np.cos(t) + x[..., a] * np.sin(t))
    size[..., a] = size[..., b] = magnitude * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, size


def exponents(x):
    """the exponent byte of every 32 values of x [..., d]"""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(g).max(-1)
    out = np.full(top.shape, 255, dtype=np.int64)
    ok = np.isfinite(g).all(-1)
    e = np.full(top.shape, 7, dtype=np.int64)
    pos = ok & (top > 0)
    with np.errstate(divide="ignore"):
        guess = np.floor(np.log2(np.where(pos, top, 1.0) / 7)).astype(np.int64)
    for k in (2, 1, 0, -1):  # the least that holds, whatever the logarithm rounds to
        fits = 7 * np.exp2((guess + k).astype(np.float64)) >= top
        e = np.where(pos & fits, np.maximum(guess + k + 127, 7), e)
    out[ok] = np.minimum(e, 252)[ok]
    return out


def encode(x):
    """codes [..., d] and exponent bytes [..., d / 32]"""
    x = np.asarray(x, dtype=np.float64)
    e = exponents(x)
    scale = np.exp2(np.where(e == 255, 127, e) - 127.0)[..., None]
    y = np.where((e == 255)[..., None], 0.0, x.reshape(*e.shape, 32) / scale)
    a = np.abs(y)
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    held = np.minimum(np.rint(a / step) * step, 6.0)
    code = np.searchsorted(GRID, held) + 8 * (np.signbit(y) & (e != 255)[..., None])
    return code.reshape(x.shape), e


def decode(code, exps):
    mag = GRID[code & 7] * np.where(code > 7, -1.0, 1.0)
    scale = np.where(exps == 255, np.nan, np.exp2(exps - 127.0))
    return (mag.reshape(*exps.shape, 32) * scale[..., None]).reshape(code.shape)


def held(x):
    return decode(*encode(x))


def offsets(dim, is_v):
    """of position r and value x in a block: the byte of the code, of the exponent"""
    r, x = np.arange(16)[:, None], np.arange(dim)[None]
    if not is_v:
        return r * (dim // 2) + x // 2, 8 * dim + r * (dim // 32) + x // 32
    g, i, per = r // 4, r % 4, dim // 16
    n, y = x // per, x % per
    return ((g * 16 + n) * 4 + i) * (per // 2) + y // 2, 8 * dim + (g * (dim // 32) + x // 32) * 4 + i


def write(pool, is_v, page, row, code, exps):
    """rows of a pool (uint8 [pages, hkv, page / 16, 17 dim / 2], in place): code
    [n, hkv, dim] and exps [n, hkv, dim / 32] at rows row[n] of pages page[n]"""
    dim = code.shape[-1]
    co, eo = offsets(dim, is_v)
    for n in range(len(page)):
        block = pool[page[n], :, row[n] // 16]  # [hkv, bytes], a view
        r = row[n] % 16
        block[:, co[r][::2]] = (code[n][:, 0::2] | code[n][:, 1::2] << 4).astype(np.uint8)
        block[:, eo[r][::32]] = exps[n].astype(np.uint8)


def read(pool, is_v, page, row):
    """the values (fp64) [n, hkv, dim] of rows row[n] of pages page[n]"""
    dim = pool.shape[-1] * 2 // 17
    co, eo = offsets(dim, is_v)
    out = []
    for p, r in zip(page, row):
        block = pool[p, :, r // 16]
        byte = block[:, co[r % 16]]
        code = (byte >> (4 * (np.arange(dim) % 2))) & 15
        out.append(decode(code.astype(np.int64), block[:, eo[r % 16][::32]].astype(np.int64)))
    return np.array(out).reshape(len(page), pool.shape[1], dim)


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The token, the log of its share, and the tokens within 1e-11 of the sum of
    the place drawn (more than one where a border is that near)."""
    z = np.asarray(z, dtype=np.float64)
    order = np.lexsort((np.arange(len(z)), -z))
    if not temperature > 0:
        return int(order[0]), 0.0, {int(order[0])}
    with np.errstate(invalid="ignore"):
        w = np.exp((z[order] - z[order[0]]) / temperature)
    w = np.where(np.isneginf(z[order]), 0.0, w)
    n = len(w)
    if top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        run = np.cumsum(w[:n])
        n = min(n, int(np.searchsorted(run, max(top_p, 0.0) * run[-1], side="left")) + 1)
    if min_p > 0:
        n = min(n, int((w >= min(min_p, 1.0)).sum()))
    run = np.cumsum(w[:n])
    u = min(max(u, 0.0), np.nextafter(np.float32(1), np.float32(0))) if u == u else 0.0
    at = [min(int(np.searchsorted(run, u * run[-1] + d * run[-1], side="right")), n - 1) for d in (-1e-11, 0, 1e-11)]
    return int(order[at[1]]), float(np.log(w[at[1]] / run[-1])), {int(order[i]) for i in range(at[0], at[2] + 1)}
