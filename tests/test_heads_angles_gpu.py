"""Sines and cosines of 16-bit heads (include/elsaa_heads.h: 2^-20 off at
most), as exact as they leave the library."""
import math

import numpy as np
import pytest
import torch

import layer_cases as C
from paper_2607_20214_gb300 import elsaa as E

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("il", [False, True])
def test_angles_of_16_bit_heads(il):
    """Sine and cosine as they leave in dw, the one fp32 result of bf16 heads:
    of one token and head whose row is ones and whose gradient is (1, 0) in
    every pair, dw is (cos a, -sin a) / sqrt(1 + eps). Angles of all sizes,
    whole quarters and their neighbours among them."""
    d, n = 128, 64
    g = np.random.default_rng(0)
    angles = g.integers(0, 2 ** 64, (200, n), dtype=np.uint64)
    near = np.arange(-8, 8, dtype=np.int64) * 2 ** 30
    for i in range(4):  # quarter turns, from below and above
        angles[i] = (np.uint64(i << 62) + np.tile(near, 4).astype(np.uint64))
    # angles that a float of half turns rounds to a whole one, tiny ones
    angles[4] = 2 ** 63 - np.arange(n, dtype=np.uint64) * np.uint64(2 ** 33)
    angles[5] = np.arange(n, dtype=np.uint64) * np.uint64(2 ** 32)
    lo = np.arange(0, d, 2) if il else np.arange(n)
    hi = lo + (1 if il else n)
    x = torch.ones(1, 1, 1, d, dtype=BF, device="cuda")
    grad = torch.zeros(1, 1, 1, d, device="cuda")
    grad[..., torch.tensor(lo)] = 1.0
    pos = torch.ones(1, 1, dtype=torch.int32, device="cuda")
    worst = 0.0
    for turns in angles:
        rot = E.make_rotary(d, interleaved=il)
        for p in range(n):
            rot.turns[p] = int(turns[p])
        h = E.make_heads(1, 1, 1, 1, d, rotary=rot, grad_fp32=True)
        dw = E.elsaa_heads_backward(h, grad, q=x, positions=pos,
                                    w_q=torch.ones(d, device="cuda"))[3]
        dw = C.f64(dw) * math.sqrt(1 + h.eps)
        a = turns.astype(np.int64) / 2.0 ** 63 * math.pi
        worst = max(worst, np.abs(dw[lo] - np.cos(a)).max(),
                    np.abs(dw[hi] + np.sin(a)).max())
    # the argument, up to pi: its half turns rounded to fp32 and cut at 2^-32
    # of a turn, pi as fp32, their product rounded; the hardware's sine and
    # cosine, 2^-21.41 and 2^-21.19 off; the norm's root and dw's product
    arg = math.pi * (2.0 ** -25 + 2.0 ** -31) + 8.8e-8 + 2.0 ** -23
    assert worst <= arg + 2.0 ** -21.19 + 4 * C.U32, worst
    assert arg + 2.0 ** -21.19 <= 2.0 ** -20
