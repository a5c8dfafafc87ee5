"""TEST INFRASTRUCTURE -- not the product.

Definitions of the sparse-attention operators in 64 bits and whole numbers, one page, one group, one row at a time: position
rotation, page bounds, page choice, attention over listed pages.
"""
from __future__ import annotations

import math

import numpy as np

from .fp8 import e4m3_decode
from .reference import _as_f64, bf16_to_f64


def f64_to_bf16_bits(x) -> np.ndarray:
    """64 -> 32 -> 16 bits, each to nearest, ties to even."""
    u = np.ascontiguousarray(x, dtype=np.float64).astype(np.float32).view(np.uint32)
    return ((u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) >> np.uint32(16)).astype(np.uint16)


def rope_reference(x, positions, inv_freq, interleaved=False, scale=1.0):
    """x [n, heads, d] (bf16 bits or float64) at the given positions -> float64."""
    x = np.array(_as_f64(x), copy=True)
    h = len(inv_freq)
    for t, pos in enumerate(positions):
        for j in range(h):
            a = float(pos) * float(np.float32(inv_freq[j]))
            c, s = math.cos(a) * scale, math.sin(a) * scale
            i1, i2 = (2 * j, 2 * j + 1) if interleaved else (j, j + h)
            x1, x2 = x[t, :, i1].copy(), x[t, :, i2].copy()
            x[t, :, i1] = x1 * c - x2 * s
            x[t, :, i2] = x2 * c + x1 * s
    return x


def bounds_exponent(amax: float) -> int:
    """Smallest e with amax <= 127 * 2^e, clamped to [-40, 96]."""
    if not amax > 0.0:
        return -40
    m, x = math.frexp(amax)                     # 127 = 0.9921875 * 2^7
    return max(-40, min(96, x - 7 if m <= 127 / 128 else x - 6))


def page_bounds(keys):
    """keys [tokens, d] float64 -> codes int8 [2, d], scale."""
    e = bounds_exponent(float(np.abs(keys).max()))
    hi, lo = keys.max(axis=0), keys.min(axis=0)
    codes = np.stack([np.ceil(np.ldexp(hi, -e)), np.floor(np.ldexp(lo, -e))])
    return np.clip(codes, -127, 127).astype(np.int8), np.float32(math.ldexp(1.0, e))


def page_bounds_reference(codes, scale, k_pool, k_scale, block_table, ctx_len, incr_len, P):
    """Bounds arrays after an update for tokens [C, C + L) of every row (copies); k_scale None: a bf16 pool (bits)."""
    codes, scale = codes.copy(), scale.copy()
    for r in range(len(ctx_len)):
        C, L = int(ctx_len[r]), int(incr_len[r])
        for lp in range(C // P, (C + L - 1) // P + 1) if L else ():
            page, n = int(block_table[r][lp]), min(P, C + L - lp * P)
            for h in range(k_pool.shape[1]):
                k = bf16_to_f64(k_pool[page, h, :n]) if k_scale is None else e4m3_decode(k_pool[page, h, :n]) * float(k_scale[page, h])
                codes[page, h], scale[page, h] = page_bounds(k)
    return codes, scale


def groups_of(ctx_len, incr_len, g):
    """(request, first new token, tokens, packed row of the first) of every group."""
    out, off = [], 0
    for r in range(len(ctx_len)):
        L = int(incr_len[r])
        out += [(r, i, min(g, L - i), off + i) for i in range(0, L, g)]
        off += L
    return out


def page_scores(q, codes, scale):
    """q [rows, d] float64 (a group's tokens x heads of one KV head); codes [pages, 2, d]; scale [pages] -> float32 [pages]."""
    amax = float(np.abs(q).max())
    f = 0
    if amax > 0.0:
        m, x = math.frexp(amax)
        f = x - 7 if m <= 127 / 128 else x - 6
    c = np.rint(np.ldexp(q, -f)).astype(np.int64)
    pos, neg = np.maximum(c, 0).sum(axis=0), np.minimum(c, 0).sum(axis=0)
    n = codes[:, 0].astype(np.int64) @ pos + codes[:, 1].astype(np.int64) @ neg
    assert np.abs(n).max(initial=0) < 2 ** 31
    return n.astype(np.float32) * scale


def select_reference(codes, scale, block_table, ctx_len, incr_len, q, P, budget, first_pages, last_pages, g):
    """int32 [groups, Hkv, budget]."""
    q = _as_f64(q)
    Hkv = codes.shape[1]
    G = q.shape[1] // Hkv
    groups = groups_of(ctx_len, incr_len, g)
    out = np.full((len(groups), Hkv, budget), -1, np.int32)
    for i, (r, t0, m, row) in enumerate(groups):
        lp0, lp1 = (int(ctx_len[r]) + t0) // P, (int(ctx_len[r]) + t0 + m - 1) // P
        always = [j for j in range(lp1 + 1) if j < first_pages or j > lp0 - last_pages]
        rest = [j for j in range(lp1 + 1) if j not in set(always)]
        left = min(len(rest), budget - len(always))
        for h in range(Hkv):
            pick = list(always)
            if left > 0:
                pages = np.asarray(block_table[r])[rest]
                there = (pages >= 0) & (pages < len(codes))                     # the others come last
                pages = np.where(there, pages, 0)
                s = page_scores(q[row:row + m, h * G:(h + 1) * G].reshape(m * G, -1), codes[pages, h], scale[pages, h])
                pick += [rest[j] for j in np.argsort(-np.where(there, s.astype(np.float64), -np.inf), kind="stable")[:left]]
            out[i, h, :len(pick)] = sorted(pick)
    return out


def sparse_attn_reference(k_rows, v_rows, ctx_len, incr_len, selected, q, P, scale, g):
    """k_rows / v_rows: per request [T, Hkv, d] float64 (all tokens).  Returns out [sum L, Hq, d] and, for error bounds, the same with
    |v| in the place of v, and the largest sum over channels of |q k| * scale of a row."""
    q = _as_f64(q)
    Hkv = selected.shape[1]
    G = q.shape[1] // Hkv
    out, mag, dots = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:2])
    for i, (r, t0, m, row) in enumerate(groups_of(ctx_len, incr_len, g)):
        last_page = (int(ctx_len[r]) + t0 + m - 1) // P
        for h in range(Hkv):
            pages = [int(e) for e in selected[i, h] if 0 <= e <= last_page]
            for t in range(m):
                p = int(ctx_len[r]) + t0 + t
                at = [x for e in pages for x in range(e * P, min((e + 1) * P, p + 1))]
                if not at:
                    continue
                k, v = k_rows[r][at, h], v_rows[r][at, h]
                for hq in range(h * G, (h + 1) * G):
                    s = (k @ q[row + t, hq]) * scale
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[row + t, hq], mag[row + t, hq] = w @ v, w @ np.abs(v)
                    dots[row + t, hq] = (np.abs(k) @ np.abs(q[row + t, hq])).max() * scale
    return out, mag, dots
