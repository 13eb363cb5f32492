"""The definitions of include/kv4.h and include/qk_rope.h in 64 bits on the CPU, value by value and byte by byte."""
import math

import numpy as np

GRID = [0, 0.5, 1, 1.5, 2, 3, 4, 6]


def block_codes(x):
    """(codes [32], scale byte) of 32 float64 values."""
    x = np.asarray(x, dtype=np.float64)
    if not np.isfinite(x).all():
        return np.zeros(32, np.uint8), 255
    top = np.abs(x).max()
    e = -23
    while e < 13 and top > 7 * 2.0 ** e:
        e += 1
    y = x / 2.0 ** e
    codes = np.zeros(32, np.uint8)
    for i, v in enumerate(y):
        gaps = [abs(abs(v) - g) for g in GRID]
        best = min(gaps)
        near = [c for c, g in enumerate(gaps) if g == best]
        code = near[0] if len(near) == 1 else [c for c in near if c % 2 == 0][0]
        codes[i] = code | (8 if math.copysign(1, v) < 0 else 0)
    return codes, e + 127


def token_place(d, tok, c):
    """Byte offsets in a group and half of channel c of token tok (0 .. 15): keys, values, their scales."""
    run = d // 16
    return (tok * (d // 2) + c // 2, 8 * d + (tok // 4) * 2 * d + (c // run) * (d // 8) + (tok % 4) * (d // 32) + c % run // 2, c % 2,
            16 * d + tok * (d // 32) + c // 32, 16 * d + d // 2 + (tok // 4) * (d // 8) + (c // 32) * 4 + tok % 4)


def put(cache, slot, head, k, v):
    """cache: uint8 numpy [pages, heads, page_size, d + d/16]; k, v: float64 [d]."""
    pages, heads, page, row = cache.shape
    d = row * 16 // 17
    place = slot % page
    g = cache[slot // page, head].reshape(-1)[(place // 16) * 17 * d:(place // 16 + 1) * 17 * d]
    for x, at, at_scale in ((k, 0, 3), (v, 1, 4)):
        for b in range(d // 32):
            codes, byte = block_codes(x[32 * b:32 * b + 32])
            for i, code in enumerate(codes):
                where = token_place(d, place % 16, 32 * b + i)
                keep = 0xf0 if where[2] == 0 else 0x0f
                g[where[at]] = (g[where[at]] & keep) | (int(code) << (4 * where[2]))
                g[where[at_scale]] = byte


def values(cache):
    """(k, v) float64 [pages, heads, page_size, d] of a whole cache."""
    pages, heads, page, row = cache.shape
    d = row * 16 // 17
    flat = cache.reshape(pages, heads, page // 16, 17 * d)
    grid = np.array(GRID + [-g for g in GRID])
    k, v = (np.empty((pages, heads, page // 16, 16, d)) for _ in range(2))
    for tok in range(16):
        for c in range(d):
            at = token_place(d, tok, c)
            for x, code, scale in ((k, at[0], at[3]), (v, at[1], at[4])):
                byte = flat[..., scale].astype(np.float64)
                x[..., tok, c] = grid[(flat[..., code] >> (4 * at[2])) & 15] * np.where(byte == 255, np.nan, 2.0 ** (byte - 127))
    return k.reshape(pages, heads, page, d), v.reshape(pages, heads, page, d)


def attention(q, kv, tables, lens, cu, causal, scale):
    """out [T, H, d], lse [T, H], and sum_j p_j |v_j| [T, H, d], for q float64 [T, H, d]; rows of nobody are NaN."""
    k_all, v_all = kv
    pages, heads, page, d = k_all.shape
    T, H, _ = q.shape
    out, lse, spread = np.full((T, H, d), np.nan), np.full((T, H), np.nan), np.full((T, H, d), np.nan)
    for b, n in enumerate(lens):
        n = max(0, min(int(n), tables.shape[1] * page))
        nq = cu[b + 1] - cu[b]
        keys = np.arange(n)
        page_of = tables[b][keys // page] if n else np.zeros(0, int)
        there = (page_of >= 0) & (page_of < pages)
        for i in range(nq):
            seen = keys[there & ((keys <= n - nq + i) if causal else True)]
            for a in range(H):
                h = a // (H // heads)
                t = cu[b] + i
                if not len(seen):
                    out[t, a], lse[t, a], spread[t, a] = 0, -np.inf, 0
                    continue
                k, v = (x[page_of[seen], h, seen % page] for x in (k_all, v_all))
                x = k @ q[t, a] * scale
                m = x.max()
                p = np.exp(x - m)
                lse[t, a] = m + np.log(p.sum())
                p /= p.sum()
                out[t, a], spread[t, a] = p @ v, p @ np.abs(v)
    return out, lse, spread


def rotate(x, c, s, interleaved, turn=1):
    d = x.shape[-1]
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :d // 2], x[..., d // 2:])
    y = np.empty_like(x)
    u, w = a * c - turn * b * s, b * c + turn * a * s
    if interleaved:
        y[..., 0::2], y[..., 1::2] = u, w
    else:
        y[..., :d // 2], y[..., d // 2:] = u, w
    return y


def norm_rope(x, w, c, s, eps, interleaved):
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    return rotate(x, c, s, interleaved)


def norm_rope_bwd(dy, x, w, c, s, eps, interleaved):
    """(dx, dw) by the formula; dw None without a weight."""
    g = rotate(dy, c, s, interleaved, turn=-1)
    if w is None:
        return g, None
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    h = g * w
    return r * (h - x * r * (h * x * r).mean(-1, keepdims=True)), (g * x * r).reshape(-1, x.shape[-1]).sum(0)
