"""Exact attention of scores that fp32 holds to no fraction, or barely: against
64 bits, where these tell which key a row's weights go to."""
import math

import numpy as np
import pytest
import torch

import layer_cases as C
from paper_2607_20214_gb300 import elsaa as E

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "fp32"}
KINDS = [(BF, 0), (BF, E.ELSAA_IMPL_SIMT), (F32, 0)]
# whole walks, masked; few rows of many keys, divided among CTAs; a padded
# batch of grouped heads
SHAPES = [dict(H=2, Nq=150, Nk=150, causal=True), dict(H=1, Nq=40, Nk=2100),
          dict(B=2, H=4, Hkv=2, Nq=140, Nk=1100, causal=True, ql=[140, 33],
               kl=[1100, 600])]


def large(d, dtype, kind, B=1, H=1, Hkv=1, Nq=1, Nk=1, seed=0, **_):
    """q, k, v, do and the scale. kind: (size of q and k, scale), scale 0 the
    default one; or the exponent of the scores' unit, when these are whole
    numbers of it and exact in fp32."""
    q, k, v, do = C.exact_inputs(B, H, Hkv, Nq, Nk, d, dtype, seed, 1.0)
    if isinstance(kind, tuple):
        size, scale = kind
        return (q * size).to(dtype), (k * size).to(dtype), v, do, scale
    a = max(-60, min(kind // 2, 50))
    scale = 2.0 ** (kind - 2 * a)
    q, k = ((4 * x).round().clamp(-8, 8) * 2.0 ** a for x in (q, k))
    return q.to(dtype), k.to(dtype), v, do, scale


def one_hot(q, k, scale, causal, exact):
    """Of one head in 64 bits: visible keys that a row's weights can go to,
    the largest score and what it can be off by in fp32."""
    n, m = len(q), len(k)
    i, j = np.arange(n)[:, None], np.arange(m)[None]
    vis = (j <= i + m - n) if causal else (j >= 0) & (i >= 0)
    s = np.where(vis, scale * (q @ k.T), -np.inf)
    top = s.max(1, keepdims=True)
    d = q.shape[1]
    off = (2 if exact else d + 6) * C.U32 * np.where(
        vis, scale * (np.abs(q) @ np.abs(k).T), 0.0).max(1, keepdims=True)
    # a key whose score is more than 100 below, whatever is rounded, has a
    # weight of e^-100 at most
    return vis & (s >= top - 2 * off - 100.0), top[:, 0], off[:, 0]


def check_forward(q, k, v, o, lse, scale, causal, exact):
    """Returns the rows whose weights go to one key, and that key."""
    held, top, off = one_hot(C.f64(q), C.f64(k), scale, causal, exact)
    V = C.f64(v)
    u = C.half_step(q.dtype)
    o, lse = C.f64(o), C.f64(lse)
    seen = held.any(1)
    assert np.isfinite(o).all() and np.isfinite(lse[seen]).all()
    alone = held.sum(1) == 1
    key = held.argmax(1)
    # the weight rounded for its product, the result
    want = V[key]
    bad = np.abs(o - want) > (2.1 * u + 16 * C.U32) * np.abs(want)
    assert not bad[alone].any(), np.argwhere(bad[alone])[:4].tolist()
    # among several: between their values
    for i in np.flatnonzero(seen & ~alone):
        lo, hi = V[held[i]].min(0), V[held[i]].max(0)
        room = 2.0 ** -7 * np.abs(V[held[i]]).max(0)
        assert (o[i] >= lo - room).all() and (o[i] <= hi + room).all(), i
    n = np.maximum(held.sum(1), 1)
    tol = off + 8 * C.U32 * np.abs(top) + np.log(n) + 1e-5
    assert (np.abs(lse - top)[seen] <= tol[seen]).all()
    return alone, key


SIZES = [(1e5, 0.0), (1e6, 0.0), (1.0, 1e10), (1e12, 1e8),
         16, 20, 24, 27, 31, 33, 60, 100, 112]


@pytest.mark.parametrize("dtype,impl", KINDS)
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", SIZES)
def test_large_scores(kind, shape, d, dtype, impl):
    B, H, Hkv = (shape.get(n, 1) for n in ("B", "H", "Hkv"))
    Nq, Nk, causal = shape["Nq"], shape["Nk"], shape.get("causal", False)
    q, k, v, do, scale = large(d, dtype, kind, **shape)
    ql, kl = shape.get("ql", [Nq] * B), shape.get("kl", [Nk] * B)
    ex = E.make_exact(B, H, Hkv, Nq, Nk, d, dtype=NAME[dtype], causal=causal,
                      scale=scale, impl=impl)
    kw = {}
    if "ql" in shape:
        kw = dict(q_len=torch.tensor(ql, dtype=torch.int32, device="cuda"),
                  k_len=torch.tensor(kl, dtype=torch.int32, device="cuda"))
    x = [t.cuda() for t in (q, k, v)]
    o = torch.zeros_like(x[0])
    lse = torch.zeros((B, H, Nq), device="cuda")
    E.elsaa_exact_forward(ex, *x, o=o, lse=lse, **kw)
    sc = scale or 1 / math.sqrt(d)
    G, exact, some = H // Hkv, not isinstance(kind, tuple), 0
    for b in range(B):
        n, m = ql[b], kl[b]
        for h in range(H):
            alone, _ = check_forward(q[b, h, :n], k[b, h // G, :m],
                                     v[b, h // G, :m], o[b, h, :n],
                                     lse[b, h, :n], sc, causal, exact)
            some += alone.sum()
    # most rows say which key it is
    assert some > 0.5 * sum(ql) * H


@pytest.mark.parametrize("dtype,impl", KINDS)
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores_rise_from_tile_to_tile(sign, dtype, impl):
    """Every tile's scores are far above the last one's, or far below 0 all."""
    q, k, v, _ = C.exact_inputs(1, 1, 1, 130, 1500, 64, dtype)
    q, k = torch.zeros_like(q), torch.zeros_like(k)
    q[..., 0] = 2.0 ** 20
    j = torch.arange(1500)
    # bf16 has 8 bits: two channels make the number
    k[0, 0, :, 0] = (j // 128).to(dtype) * 128 - (2048 if sign < 0 else 0)
    q[..., 1], k[0, 0, :, 1] = 2.0 ** 20, (j % 128).to(dtype)
    ex = E.make_exact(1, 1, 1, 130, 1500, 64, dtype=NAME[dtype], causal=True,
                      scale=64.0, impl=impl)
    lse = torch.empty((1, 1, 130), device="cuda")
    o = E.elsaa_exact_forward(ex, q.cuda(), k.cuda(), v.cuda(), lse=lse)
    alone, key = check_forward(q[0, 0], k[0, 0], v[0, 0], o[0, 0], lse[0, 0],
                               64.0, True, True)
    assert alone.all() and (key == np.arange(130) + 1370).all()


@pytest.mark.parametrize("dtype,impl", KINDS)
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", SIZES)
def test_gradients_of_large_scores(kind, shape, d, dtype, impl):
    """Rows whose weights go to one key: dV gets d_o whole, dS is what the
    rounding of o leaves. (The others' d_o is 0: whether a tie is one is more
    than lse holds.)"""
    B, H, Hkv = (shape.get(n, 1) for n in ("B", "H", "Hkv"))
    Nq, Nk, causal = shape["Nq"], shape["Nk"], shape.get("causal", False)
    q, k, v, do, scale = large(d, dtype, kind, **shape)
    ql, kl = shape.get("ql", [Nq] * B), shape.get("kl", [Nk] * B)
    ex = E.make_exact(B, H, Hkv, Nq, Nk, d, dtype=NAME[dtype], causal=causal,
                      scale=scale, impl=impl)
    kw = {}
    if "ql" in shape:
        kw = dict(q_len=torch.tensor(ql, dtype=torch.int32, device="cuda"),
                  k_len=torch.tensor(kl, dtype=torch.int32, device="cuda"))
    x = [t.cuda() for t in (q, k, v)]
    o = torch.zeros_like(x[0])
    lse = torch.zeros((B, H, Nq), device="cuda")
    E.elsaa_exact_forward(ex, *x, o=o, lse=lse, **kw)
    sc = scale or 1 / math.sqrt(d)
    G, exact = H // Hkv, not isinstance(kind, tuple)
    rows = {}
    for b in range(B):
        for h in range(H):
            rows[b, h] = check_forward(
                q[b, h, :ql[b]], k[b, h // G, :kl[b]], v[b, h // G, :kl[b]],
                o[b, h, :ql[b]], lse[b, h, :ql[b]], sc, causal, exact)
            do[b, h, :ql[b]][torch.tensor(~rows[b, h][0])] = 0
    got = E.elsaa_exact_backward(ex, *x, o, lse, do.cuda(), **kw)
    u = C.half_step(dtype)
    rnd = 2.0 ** -8 if dtype == BF and impl == 0 else 0.0
    for b in range(B):
        n, m = ql[b], kl[b]
        for j in range(Hkv):
            K, V = C.f64(k[b, j, :m]), C.f64(v[b, j, :m])
            dk, dv, dkt, dvt = (np.zeros((m, d)) for _ in range(4))
            for h in range(j * G, j * G + G):
                alone, key = rows[b, h]
                Q, DO, O = (C.f64(t[b, h, :n]) for t in (q, do, o))
                # P is 1, or within 0.01 of it where lse is below 2^16, and
                # rounded; dS = <d_o, v - o>
                p = alone * 1.0
                ds = p * (DO * (V[key] - O)).sum(1)
                mag = (np.abs(DO) * (np.abs(V[key]) + np.abs(O))).sum(1)
                off = p * ((d + 8) * C.U32 * mag) + (rnd + 0.02) * np.abs(ds)
                dq = sc * ds[:, None] * K[key]
                tol = sc * off[:, None] * np.abs(K[key]) + 2 * u * np.abs(dq)
                C.close(got[0][b, h, :n], dq, tol, ("dq", b, h))
                np.add.at(dk, key, sc * ds[:, None] * Q)
                np.add.at(dkt, key, sc * (off + n * G * C.U32 * np.abs(ds))[
                    :, None] * np.abs(Q))
                np.add.at(dv, key, p[:, None] * DO)
                np.add.at(dvt, key, (0.02 + n * G * C.U32) *
                          p[:, None] * np.abs(DO))
            C.close(got[1][b, j, :m], dk, dkt + 2 * u * np.abs(dk), "dk")
            C.close(got[2][b, j, :m], dv, dvt + 2 * u * np.abs(dv), "dv")
