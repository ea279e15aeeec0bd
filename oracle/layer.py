"""64-bit oracle of rows and heads (include/elsaa_heads.h) and of exact
attention (include/elsaa_exact.h), from their definitions, in numpy, a
sequence and head at a time. Shares no code with the CUDA path.

Each function also returns, beside a value, the sums of magnitudes that bound
its rounding errors (`mag`, ...): a test derives its tolerance from them.
"""
import math

import numpy as np

# ---------------------------------------------------------------- heads


def angles(turns, axis, positions):
    """Angle [N, pairs] of every pair, positions [axes, N] of Python's or
    numpy's integers: the product modulo 2^64, exactly."""
    out = np.empty((positions.shape[1], len(turns)))
    for p, (t, a) in enumerate(zip(turns, axis)):
        for n in range(positions.shape[1]):
            f = int(positions[a, n]) * int(t) % (1 << 64)
            if f >= 1 << 63:
                f -= 1 << 64
            out[n, p] = 2 * math.pi * (f / 2.0 ** 64)
    return out


def _pairs(dim, interleaved):
    if interleaved:
        return np.arange(0, dim, 2), np.arange(1, dim, 2)
    return np.arange(dim // 2), np.arange(dim // 2, dim)


def rotate(x, ang, interleaved):
    """x [N, d] turned by ang [N, pairs]; and |lo| + |hi| per channel."""
    lo, hi = _pairs(2 * ang.shape[1], interleaved)
    y, mag = x.copy(), np.abs(x)
    c, s = np.cos(ang), np.sin(ang)
    y[:, lo] = x[:, lo] * c - x[:, hi] * s
    y[:, hi] = x[:, hi] * c + x[:, lo] * s
    mag[:, lo] = mag[:, hi] = np.abs(x[:, lo]) + np.abs(x[:, hi])
    return y, mag


def normed(x, w, eps):
    r = 1.0 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    return x * r * w


def head_forward(x, ang, interleaved, norm, w, eps):
    """One head's rows x [N, d] -> (out, mag)."""
    return rotate(normed(x, w, eps) if norm else x, ang, interleaved)


def head_backward(g, x, ang, interleaved, norm, w, eps):
    """g [copies, N, d], gradients of a head's copies -> dict(dx, dw) and the
    magnitudes of what they are sums of."""
    u, mag = rotate(g.sum(0), -ang, interleaved)
    mag = rotate(np.abs(g).sum(0), 0 * ang, interleaved)[1]
    if not norm:
        return dict(dx=u, dx_mag=mag, dw=None, dw_mag=None)
    r = 1.0 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    xh = x * r
    t = u * w
    m = (t * xh).mean(1, keepdims=True)
    at = mag * np.abs(w)
    return dict(dx=r * (t - xh * m),
                dx_mag=r * (at + np.abs(xh) *
                            (at * np.abs(xh)).mean(1, keepdims=True)),
                dw=(u * xh).sum(0), dw_mag=(mag * np.abs(xh)).sum(0))


# ---------------------------------------------------------------- exact


def visible(nq, nk, causal):
    """[nq, nk]: query row i sees key row j."""
    i, j = np.arange(nq)[:, None], np.arange(nk)[None]
    return (j <= i + nk - nq) if causal else (j >= 0) & (i >= 0)


def attend(q, k, v, scale, causal):
    """One head: q [nq, d], k, v [nk, d] -> dict(o, lse, o_mag = sum P |v|,
    s_mag = the largest scale sum |q k| a query sees)."""
    nq, nk = len(q), len(k)
    vis = visible(nq, nk, causal)
    s = np.where(vis, scale * (q @ k.T), -np.inf)
    sm = np.where(vis, scale * (np.abs(q) @ np.abs(k).T), 0.0)
    o = np.zeros((nq, v.shape[1]))
    o_mag = np.zeros_like(o)
    lse = np.full(nq, -np.inf)
    for i in range(nq):
        if not vis[i].any():
            continue
        top = s[i].max()
        e = np.exp(s[i] - top)
        lse[i] = top + math.log(e.sum())
        p = e / e.sum()
        o[i] = p @ np.where(vis[i][:, None], v, 0.0)
        o_mag[i] = p @ np.where(vis[i][:, None], np.abs(v), 0.0)
    return dict(o=o, lse=lse, o_mag=o_mag,
                s_mag=sm.max(1, initial=0.0)[:, None])


def attend_backward(q, k, v, o, lse, do, scale, causal):
    """One query head; o and lse are what the forward pass left. Returns dq,
    dk, dv and, for the bounds, P, dS and the matrices they came from."""
    vis = visible(len(q), len(k), causal)
    s = scale * (q @ k.T)
    p = np.where(vis, np.exp(np.where(vis, s - np.where(
        np.isfinite(lse), lse, 0.0)[:, None], 0.0)), 0.0)
    p[~np.isfinite(lse)] = 0.0
    dp = do @ v.T
    delta = (do * o).sum(1)[:, None]
    ds = p * (dp - delta)
    sm = np.where(vis, scale * (np.abs(q) @ np.abs(k).T), 0.0)
    dm = np.abs(do) @ np.abs(v).T + (np.abs(do) * np.abs(o)).sum(1)[:, None]
    return dict(dq=scale * (ds @ k), dk=scale * (ds.T @ q), dv=p.T @ do,
                p=p, ds=ds, s_mag=sm, dp_mag=dm)
