"""Gradients of exact attention with scales of the caller's and with scores
that leave a row to a few keys, on every way through the backward pass: whole
walks, walks that are divided and added up, a padded batch."""
import numpy as np
import pytest
import torch

import layer_cases as C
from paper_2607_20214_gb300 import elsaa as E
from test_exact_gpu import run_case

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def with_small_weights(q, k, v, o, lse, do, scale, causal, ql, kl, tensor,
                       reference=C.exact_backward_ref):
    """The reference, its tolerances for numbers below fp32's normal ones too:
    a weight below 2^-126 may be 0 (the exponential gives no smaller ones), and
    so may dS and a result. With |dP - D| <= m and n rows, such weights leave
    out 2^-126 sum |d_o| of dV, and 2^-126 (m + 1) scale sum |q| of dK, |k| of
    dQ."""
    out = reference(q, k, v, o, lse, do, scale, causal, ql, kl, tensor)
    tiny = 2.0 ** -126
    B, H = q.shape[:2]
    G = H // k.shape[1]

    def add(name, at, more):
        val, tol = out[name][at]
        out[name][at] = val, tol + more + tiny
    for b in range(B):
        n, m = ql[b], kl[b]
        for j in range(k.shape[1]):
            K, V = (C.f64(x[b, j, :m]) for x in (k, v))
            Q, DO, O = (np.abs(C.f64(x[b, j * G:j * G + G, :n])) for x in
                        (q, do, o))
            if n == 0 or m == 0:
                continue
            most = (DO.sum(-1).max() * (np.abs(V).max() + O.max()) + 1) * tiny
            for h in range(j * G, j * G + G):
                add("dq", (b, h), scale * most * np.abs(K).sum(0))
            add("dk", (b, j), scale * most * Q.sum((0, 1)))
            add("dv", (b, j), tiny * DO.sum((0, 1)))
    return out


@pytest.mark.parametrize("dtype,impl", [(BF, 0), (BF, E.ELSAA_IMPL_SIMT),
                                        (F32, 0)])
@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,d,causal,ql,kl", [
    (1, 2, 1, 150, 150, 64, 1, None, None),
    (1, 4, 1, 260, 1100, 64, 0, None, None),
    (1, 2, 1, 200, 1030, 128, 1, None, None),
    (2, 4, 2, 190, 333, 32, 1, [190, 77], [333, 60])])
@pytest.mark.parametrize("spread,scale", [(1.5, 0.05), (1.0, 0.4), (1.5, 4.0),
                                          (12.0, 0.0), (0.0, 3.0)])
def test_scales_and_peaked_scores(spread, scale, B, H, Hkv, Nq, Nk, d, causal,
                                  ql, kl, dtype, impl, monkeypatch):
    monkeypatch.setattr(C, "exact_backward_ref", with_small_weights)
    run_case(B, H, Hkv, Nq, Nk, d, dtype, causal, ql=ql, kl=kl, impl=impl,
             spread=spread, scale=scale, seed=11)
