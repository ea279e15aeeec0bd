"""Inputs, oracle values and derived tolerances of the tests of rows and heads
and of exact attention (not a test module)."""
import numpy as np
import torch

from oracle import layer

U32 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return t.detach().double().cpu().numpy()


# ---------------------------------------------------------------- exact

def exact_inputs(B, H, Hkv, Nq, Nk, d, dtype, seed=0, spread=1.5):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    q = (r(B, H, Nq, d) * spread).to(dtype)
    k = (r(B, Hkv, Nk, d) * spread).to(dtype)
    v, do = r(B, Hkv, Nk, d).to(dtype), r(B, H, Nq, d).to(dtype)
    return q, k, v, do


def weight_error(d, s_mag):
    """Relative error of a weight exp(s - lse) in fp32: of s (a sum of d
    products in any order, scaled, its reference subtracted: d + 4 roundings
    of numbers up to s_mag), and of the exponential (2^-22)."""
    return 1.1 * ((d + 4) * U32 * (s_mag + 1.0) * 2 + 2.0 ** -22)


def exact_forward_ref(q, k, v, scale, causal, ql, kl, tensor):
    """Oracle o, lse of every head and the tolerances. tensor: weights are
    rounded to bf16 for the product with V."""
    B, H, Nq, d = q.shape
    G = H // k.shape[1]
    out = {}
    u = half_step(q.dtype)
    for b in range(B):
        for h in range(H):
            n, m = ql[b], kl[b]
            r = layer.attend(f64(q[b, h, :n]), f64(k[b, h // G, :m]),
                             f64(v[b, h // G, :m]), scale, causal)
            e = weight_error(d, r["s_mag"])
            # both the weights and their sum; sums of m terms in fp32
            w = 2 * e + (m + 8) * U32 + (2.0 ** -8 if tensor else 0.0)
            r["o_tol"] = w * r["o_mag"] * 1.01 + u * np.abs(r["o"])
            lse = np.where(np.isfinite(r["lse"]), np.abs(r["lse"]), 0.0)
            r["lse_tol"] = e[:, 0] + (m + 4) * U32 + 4 * U32 * lse
            out[b, h] = r
    return out


def exact_backward_ref(q, k, v, o, lse, do, scale, causal, ql, kl, tensor):
    """Oracle dq [B, H], dk, dv [B, Hkv] with tolerances."""
    B, H, Nq, d = q.shape
    Hkv = k.shape[1]
    G = H // Hkv
    u = half_step(q.dtype)
    rnd = 2.0 ** -8 if tensor else 0.0
    out = dict(dq={}, dk={}, dv={})
    for b in range(B):
        n, m = ql[b], kl[b]
        for j in range(Hkv):
            K, V = f64(k[b, j, :m]), f64(v[b, j, :m])
            dk, dv = np.zeros_like(K), np.zeros_like(V)
            dkt, dvt = np.zeros_like(K), np.zeros_like(V)
            for h in range(j * G, j * G + G):
                Q, DO = f64(q[b, h, :n]), f64(do[b, h, :n])
                r = layer.attend_backward(Q, K, V, f64(o[b, h, :n]),
                                          f64(lse[b, h, :n]), DO, scale,
                                          causal)
                # lse itself is rounded to fp32; it is an input here
                ep = weight_error(d, r["s_mag"])
                eds = r["p"] * ((ep + 3 * U32) * r["dp_mag"] +
                                (d + 4) * U32 * r["dp_mag"])
                eds = 1.02 * eds + (rnd + U32) * np.abs(r["ds"])
                n32 = (max(n * G, m) + 8) * U32
                dqt = scale * (eds @ np.abs(K) +
                               n32 * (np.abs(r["ds"]) @ np.abs(K)))
                out["dq"][b, h] = (r["dq"], dqt + u * np.abs(r["dq"]))
                dk += r["dk"]
                dv += r["dv"]
                dkt += scale * (eds.T @ np.abs(Q) +
                                n32 * (np.abs(r["ds"]).T @ np.abs(Q)))
                dvt += ((ep + rnd + n32) * r["p"]).T @ np.abs(DO)
            out["dk"][b, j] = (dk, dkt + u * np.abs(dk))
            out["dv"][b, j] = (dv, dvt + u * np.abs(dv))
    return out


def close(got, ref, tol, what):
    got = f64(got)
    with np.errstate(invalid="ignore"):
        same = (got == ref) | (np.isnan(got) & np.isnan(ref))
        off = np.where(same, 0.0, np.abs(got - ref))
    bad = ~(off <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(),
                           float(np.nanmax(off)), got[bad][:4], ref[bad][:4])


# ---------------------------------------------------------------- heads

def heads_ref(x, heads, kinds, pos, new, w, backward=None):
    """Oracle of one tensor of rows x [B, N, heads, d] (fp32 or bf16).

    heads: the elsaa_heads; pos [axes, B, N] ints; new: rows per sequence; w:
    weights or None; kinds: whether it is normed and rotated, copies.
    Without backward: {(b, h): (out, tol)}. With backward = gradients
    [B, heads * copies, N, d]: ({(b, h): (dx, tol)}, dw, dw_tol).
    """
    turned, copies = kinds
    r = heads.rotary
    n_pairs = r.dim // 2
    turns, axis = list(r.turns)[:n_pairs], list(r.axis)[:n_pairs]
    d = heads.d_h
    W = np.ones(d) if w is None else f64(w)
    norm = bool(heads.norm) and turned
    u = half_step(x.dtype)
    out, dw, dwt = {}, np.zeros(d), np.zeros(d)
    terms = 0
    for b in range(x.shape[0]):
        n = new[b]
        ang = layer.angles(turns, axis, pos[:, b, :n])
        if not turned:
            ang = np.zeros((n, 0))
        for h in range(x.shape[2]):
            X = f64(x[b, :n, h])
            if backward is None:
                y, mag = layer.head_forward(X, ang, r.interleaved, norm, W,
                                            heads.eps)
                # the sum of squares (8 in a row, 5 levels), the root, the
                # angle (2^-25 of half a turn and 2 ulp), products: below 32
                # roundings of |lo| + |hi|
                out[b, h] = (y, u * np.abs(y) + (32 * U32 * mag if turned
                                                 else 0.0))
                continue
            g = f64(backward[b, h * copies:(h + 1) * copies, :n])
            e = layer.head_backward(g, X, ang, r.interleaved, norm, W,
                                    heads.eps)
            few = (48 + copies) * U32
            out[b, h] = (e["dx"], u * np.abs(e["dx"]) +
                         (few * e["dx_mag"] if turned or copies > 1 else 0.0))
            if norm:
                dw += e["dw"]
                dwt += e["dw_mag"]
                terms += n
    if backward is None:
        return out
    return out, dw, dwt * (terms + 64) * U32
