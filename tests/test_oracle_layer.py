"""The oracle of rows and heads and of exact attention, pinned by independent
statements (no GPU)."""
import math

import numpy as np
import pytest

from oracle import layer
from paper_2607_20214_gb300 import elsaa as E


@pytest.mark.parametrize("interleaved", [0, 1])
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(0)
    x, ang = rng.normal(size=(5, 12)), rng.normal(size=(5, 4))
    y, _ = layer.rotate(x, ang, interleaved)
    lo, hi = ((slice(0, 8, 2), slice(1, 8, 2)) if interleaved else
              (slice(0, 4), slice(4, 8)))
    z = (x[:, lo] + 1j * x[:, hi]) * np.exp(1j * ang)
    assert np.allclose(y[:, lo], z.real) and np.allclose(y[:, hi], z.imag)
    assert np.array_equal(y[:, 8:], x[:, 8:])


def test_products_depend_on_the_distance_only():
    rng = np.random.default_rng(1)
    r = E.make_rotary(16)
    turns, axis = list(r.turns)[:8], list(r.axis)[:8]
    q, k = rng.normal(size=(1, 16)), rng.normal(size=(1, 16))

    def dot(m, n):
        a, b = (layer.rotate(x, layer.angles(turns, axis, np.array([[p]])),
                             0)[0] for x, p in ((q, m), (k, n)))
        return float((a @ b.T)[0, 0])
    for far in (0, 1000, 2 ** 31 - 100):
        assert abs(dot(far + 7, far + 3) - dot(7, 3)) < 1e-12


@pytest.mark.parametrize("frequency", [1.0, 10000.0 ** -0.5, 3e-5, -0.25, 7.0])
def test_turns_are_the_frequency(frequency):
    t = E._turns(frequency)
    for pos in (1, -3, 12345):
        a = layer.angles([t], [0], np.array([[pos]]))[0, 0]
        assert abs(math.remainder(a - pos * frequency, 2 * math.pi)) < 1e-11


def test_axes_in_blocks_and_in_turn():
    r = E.make_rotary(20, interleaved=True, sections=[4, 3, 3])
    assert list(r.axis)[:10] == [0] * 4 + [1] * 3 + [2] * 3
    r = E.make_rotary(20, interleaved=True, sections=[5, 2, 3], in_turn=True)
    assert list(r.axis)[:10] == [0, 1, 2, 0, 1, 2, 0, 2, 0, 0]
    for bad in ([4, 3], [5, 5, 0, 0, 0], [11, -1]):
        with pytest.raises(ValueError):
            E.make_rotary(20, sections=bad)
    with pytest.raises(ValueError):
        E.make_rotary(15)
    with pytest.raises(ValueError):
        E.make_rotary(16, frequencies=[1.0] * 7)


@pytest.mark.parametrize("norm", [0, 1])
def test_head_gradients_against_differences(norm):
    rng = np.random.default_rng(2)
    x, w, ang = (rng.normal(size=s) for s in ((3, 8), (8,), (3, 3)))
    g = rng.normal(size=(2, 3, 8))

    def loss(x, w):
        return float((layer.head_forward(x, ang, 0, norm, w, 0.1)[0] *
                      g.sum(0)).sum())
    r = layer.head_backward(g, x, ang, 0, norm, w, 0.1)
    step = 1e-6
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = step
        num = (loss(x + d, w) - loss(x - d, w)) / (2 * step)
        assert abs(num - r["dx"][i]) < 1e-7
    if norm:
        for i in range(8):
            d = np.zeros(8)
            d[i] = step
            num = (loss(x, w + d) - loss(x, w - d)) / (2 * step)
            assert abs(num - r["dw"][i]) < 1e-7


@pytest.mark.parametrize("nq,nk,causal", [(5, 5, 1), (3, 7, 1), (7, 3, 1),
                                          (4, 6, 0), (1, 1, 1), (3, 0, 1)])
def test_attention_against_loops_and_differences(nq, nk, causal):
    rng = np.random.default_rng(3)
    q, k, v = (rng.normal(size=(n, 4)) for n in (nq, nk, nk))
    do = rng.normal(size=(nq, 4))
    r = layer.attend(q, k, v, 0.7, causal)
    for i in range(nq):
        seen = [j for j in range(nk) if not causal or j <= i + nk - nq]
        e = [math.exp(0.7 * float(q[i] @ k[j])) for j in seen]
        if not seen:
            assert r["lse"][i] == -math.inf and not r["o"][i].any()
            continue
        assert abs(r["lse"][i] - math.log(sum(e))) < 1e-12
        want = sum(w * v[j] for w, j in zip(e, seen)) / sum(e)
        assert np.allclose(r["o"][i], want)
    b = layer.attend_backward(q, k, v, r["o"], r["lse"], do, 0.7, causal)
    step = 1e-6
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        for i in np.ndindex(x.shape):
            was = x[i]
            f = []
            for s in (step, -step):
                x[i] = was + s
                f.append(float((layer.attend(q, k, v, 0.7, causal)["o"] *
                                do).sum()))
            x[i] = was
            assert abs((f[0] - f[1]) / (2 * step) - b[name][i]) < 1e-7
