"""64-bit oracle of the cache operators (include/elsaa_cache.h), from their
definitions, in numpy, one sequence and head at a time. Shares no code with
the CUDA path.

A cache is a dict of arrays: k, v [pages, H_kv, page_size, d] uint8 codes,
k_scale, v_scale [pages, H_kv] float, bounds [pages, H_kv, 2, d] int8, table
[B, max_pages] int, lengths [B] int.
"""
import math

import numpy as np


def _table():
    """Value of every e4m3 code: sign, 4 exponent bits (bias 7), 3 mantissa
    bits; exponent 0 is subnormal, 0x7f and 0xff are NaN."""
    out = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        if e == 15 and m == 7:
            x = math.nan
        elif e == 0:
            x = m * 2.0 ** -9
        else:
            x = (8 + m) * 2.0 ** (e - 10)
        out[c] = -x if s else x
    return out


E4M3 = _table()
_POSITIVE = E4M3[:127]  # 0 .. 448, increasing


def encode(x):
    """Nearest e4m3 code (ties to even, saturating at 448), NaN as NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.searchsorted(_POSITIVE, np.where(np.isnan(a), 0.0, a))
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    up, dn = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    pick_hi = (up < dn) | ((up == dn) & (hi % 2 == 0))
    code = np.where(pick_hi | (_POSITIVE[hi] == a), hi, lo)
    code = np.where(np.isnan(x), 127, code)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def exponent(amax, top, low, high):
    """Least e in [low, high] with amax <= top 2^e."""
    if not amax > 0:
        return low
    e = math.frexp(amax / top)[1] - 2
    while amax > math.ldexp(top, e):
        e += 1
    return min(max(e, low), high)


def _amax(x):
    a = np.abs(x[~np.isnan(x)])
    a = np.minimum(a, float(np.finfo(np.float32).max))
    return float(a.max()) if a.size else 0.0


def _page(x):
    return exponent(_amax(x), 448.0, -64, 120)


def _extremes(codes):
    """ceil(max / 4), floor(min / 4) per channel, NaN left out."""
    y = E4M3[codes]
    hi = np.where(np.isnan(y), -np.inf, y).max(0)
    lo = np.where(np.isnan(y), np.inf, y).min(0)
    return np.ceil(hi / 4), np.floor(lo / 4)


def _box(hi, lo):
    """The bounds of a page; a channel without a number may hold anything."""
    none = hi < lo
    return np.stack([np.where(none, 112, hi), np.where(none, -112, lo)])


def append(c, k, v, new_len):
    """Updates c in place with rows k, v [B, H_kv, T, d]; lengths count
    them already."""
    ps = c["k"].shape[2]
    for b in range(len(c["lengths"])):
        end, n = int(c["lengths"][b]), int(new_len[b])
        start = end - n
        for p in range(start // ps, -(-end // ps) if n else 0):
            i = c["table"][b, p]
            r0, r1 = max(start - p * ps, 0), min(ps, end - p * ps)
            t0 = p * ps + r0 - start
            for x, new in (("k", k), ("v", v)):
                for h in range(c["k"].shape[1]):
                    rows = np.float64(new[b, h, t0:t0 + r1 - r0])
                    e = _page(rows)
                    drop = 1.0
                    if r0:
                        old = math.frexp(c[x + "_scale"][i, h])[1] - 1
                        e = max(e, old)
                        drop = 2.0 ** (old - e)
                        c[x][i, h, :r0] = encode(E4M3[c[x][i, h, :r0]] * drop)
                    c[x][i, h, r0:r1] = encode(rows / 2.0 ** e)
                    c[x + "_scale"][i, h] = 2.0 ** e
                    if x == "k":
                        hi, lo = _extremes(c[x][i, h, r0:r1])
                        if r0:
                            was = np.float64(c["bounds"][i, h]) * drop
                            hi = np.maximum(hi, np.ceil(was[0]))
                            lo = np.minimum(lo, np.floor(was[1]))
                        c["bounds"][i, h] = _box(hi, lo)


def _rows(c, x, b, h, pos):
    ps = c["k"].shape[2]
    pages = c["table"][b, pos // ps]
    return E4M3[c[x][pages, h, pos % ps]] * \
        np.float64(c[x + "_scale"][pages, h])[:, None]


def attention(c, q, new_len, scale, pages=None, skip=()):
    """O [B, H, T, d], lse [B, H, T], the weights' increments
    [B, H_kv, slots] and, per query, sum_i |q_i k_ij| at its largest (for
    error bounds) with the largest |v|. Rows t >= new_len are NaN. skip: pages
    (of the pool) that are treated as absent."""
    B, H, T, d = q.shape
    hkv, ps = c["k"].shape[1:3]
    G = H // hkv
    o = np.full(q.shape, np.nan)
    lse = np.full((B, H, T), np.nan)
    size = np.zeros((B, H, T))
    vmax = np.zeros((B, H, T))
    w = np.zeros((B, hkv, c["table"].shape[1] * ps))
    for b in range(B):
        n, end = int(new_len[b]), int(c["lengths"][b])
        for h in range(hkv):
            pos = np.arange(end)
            if pages is not None:
                pos = pos[np.isin(pos // ps, pages[b, h])]
            if len(pos) and len(skip):
                pos = pos[~np.isin(c["table"][b, pos // ps], skip)]
            k, v = _rows(c, "k", b, h, pos), _rows(c, "v", b, h, pos)
            for g in range(h * G, h * G + G):
                for t in range(n):
                    sees = pos <= end - n + t
                    if not sees.any():
                        o[b, g, t], lse[b, g, t] = 0.0, -np.inf
                        continue
                    x = np.float64(q[b, g, t])
                    s = k[sees] @ x * scale
                    top = s.max()
                    L = top + np.log(np.exp(s - top).sum())
                    p = np.exp(s - L)
                    o[b, g, t], lse[b, g, t] = p @ v[sees], L
                    w[b, h, pos[sees]] += p
                    size[b, g, t] = (np.abs(k[sees]) @ np.abs(x)).max() * scale
                    vmax[b, g, t] = np.abs(v[sees]).max()
    return o, lse, w, size, vmax


def select(c, q, new_len, n_sel, first, last):
    B, H, T, d = q.shape
    hkv, ps = c["k"].shape[1:3]
    G = H // hkv
    out = np.full((B, hkv, n_sel), -1, dtype=np.int32)
    for b in range(B):
        n, m = -(-int(c["lengths"][b]) // ps), int(new_len[b])
        if m == 0:
            continue
        for h in range(hkv):
            score = []
            for p in range(n):
                i = c["table"][b, p]
                hi, lo = np.float64(c["bounds"][i, h])
                best = -math.inf
                for x in np.float64(q[b, h * G:h * G + G, :m]).reshape(-1, d):
                    e = exponent(_amax(x), 127.0, -60, 120)
                    z = np.clip(np.rint(x / 2.0 ** e), -127, 127)
                    z = np.where(np.isnan(z), 0.0, z)
                    u = np.maximum(z * hi, z * lo).sum()
                    best = max(best, u * 2.0 ** e * 4 *
                               float(c["k_scale"][i, h]))
                if p < first or p >= n - last:
                    best = math.inf
                score.append(best)
            take = sorted(sorted(range(n), key=lambda p: (-score[p], p))
                          [:n_sel])
            out[b, h, :len(take)] = take
    return out


def evict(c, weight, keep, recent, dst, weight_out):
    """Updates the pages of dst in c and weight_out in place; returns
    (lengths, kept)."""
    B, width = dst.shape
    hkv, ps = c["k"].shape[1:3]
    kept = np.full((B, hkv, keep), -1, dtype=np.int32)
    counts = np.minimum(c["lengths"], keep).astype(np.int32)
    for b in range(B):
        n, m = int(c["lengths"][b]), int(counts[b])
        for h in range(hkv):
            safe = max(0, n - recent)
            w = np.float64(weight[b, h, :safe])
            key = np.where(np.isnan(w), -np.inf, w)
            order = np.lexsort((np.arange(safe), np.isnan(w), -key))
            take = np.sort(np.concatenate(
                [order[:max(0, m - (n - safe))], np.arange(safe, n)]))
            if n <= keep:
                take = np.arange(n)
            kept[b, h, :m] = take
            weight_out[b, h, :m] = weight[b, h, take]
            take = take.astype(np.int64)
            for x in "kv":
                rows = _rows(c, x, b, h, take)
                for p in range(-(-m // ps)):
                    r = rows[p * ps:(p + 1) * ps]
                    e = _page(r)
                    i = dst[b, p]
                    c[x][i, h, :len(r)] = encode(r / 2.0 ** e)
                    c[x + "_scale"][i, h] = 2.0 ** e
                    if x == "k":
                        hi, lo = _extremes(c[x][i, h, :len(r)])
                        c["bounds"][i, h] = _box(hi, lo)
    return counts, kept
