"""The cache oracle (oracle/cache.py) against independent definitions, on the
CPU."""
import numpy as np
import torch

from oracle import cache as oc


def test_codes_are_those_of_float8_e4m3fn():
    """Values of all codes; nearest codes of numbers around all of them."""
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(oc.E4M3, want, equal_nan=True)
    pos = np.sort(want[:127]).astype(np.float64)
    mid = (pos[1:] + pos[:-1]) / 2
    x = np.concatenate([pos, mid, mid * (1 + 2.0 ** -20),
                        mid * (1 - 2.0 ** -20), [447.0, 1e-9]])
    x = np.concatenate([x, -x])
    want = torch.tensor(x).float().to(torch.float8_e4m3fn).view(torch.uint8)
    assert np.array_equal(oc.encode(x), want.numpy())
    assert oc.encode([1e9, -1e9]).tolist() == [0x7E, 0xFE]


def empty(pages, ps, d, table, lengths):
    return dict(k=np.zeros((pages, 1, ps, d), np.uint8),
                v=np.zeros((pages, 1, ps, d), np.uint8),
                k_scale=np.ones((pages, 1), np.float32),
                v_scale=np.ones((pages, 1), np.float32),
                bounds=np.zeros((pages, 1, 2, d), np.int8),
                table=np.array(table, np.int32),
                lengths=np.array(lengths, np.int32))


def test_exponents_and_bounds_of_a_page_by_hand():
    """448 2^e holds the largest; bounds are the extreme codes over 4, rounded
    outwards; a channel of NaN may hold anything; a page that grows rescales."""
    c = empty(1, 4, 3, [[0]], [2])
    k = np.array([[9.0, -3.0, np.nan], [448.0, -64.0, np.nan]])[None, None]
    oc.append(c, k, k, [2])
    assert c["k_scale"][0, 0] == 1.0
    assert c["bounds"][0, 0].tolist() == [[112, 0, 112], [2, -16, -112]]
    assert oc.E4M3[c["k"][0, 0, :2]][:, :2].tolist() == [[9, -3], [448, -64]]
    c["lengths"][:] = 3
    k = np.array([[449.0, 5.0, 8.0]])[None, None]
    oc.append(c, k, k, [1])
    assert c["k_scale"][0, 0] == 2.0
    # halves of the older bounds and of the codes, 224 of 449 / 2
    assert c["bounds"][0, 0].tolist() == [[56, 1, 56], [1, -8, -56]]
    assert oc.E4M3[c["k"][0, 0, :3]][:, :2].tolist() == [
        [4.5, -1.5], [224, -32], [224, 2.5]]


def test_attention_is_softmax_over_the_rows_seen():
    g = np.random.default_rng(0)
    c = empty(3, 4, 8, [[2, 0, 1]], [10])
    x = g.standard_normal((1, 1, 10, 8))
    oc.append(c, x, 2 * x[:, :, ::-1], [10])
    k = np.concatenate([oc.E4M3[c["k"][i, 0]] * c["k_scale"][i, 0]
                        for i in (2, 0, 1)])[:10]
    v = np.concatenate([oc.E4M3[c["v"][i, 0]] * c["v_scale"][i, 0]
                        for i in (2, 0, 1)])[:10]
    q = g.standard_normal((1, 2, 2, 8))
    o, lse, w, _, _ = oc.attention(c, q, [2], 0.3)
    total = np.zeros(10)
    for h in range(2):
        for t in range(2):
            n = 9 + t
            s = torch.tensor(k[:n] @ q[0, h, t] * 0.3)
            p = torch.softmax(s, 0).numpy()
            total[:n] += p
            assert np.allclose(o[0, h, t], p @ v[:n], rtol=1e-12, atol=1e-14)
            assert np.isclose(lse[0, h, t], float(torch.logsumexp(s, 0)))
    assert np.allclose(w[0, 0, :10], total) and (w[0, 0, 10:] == 0).all()
    # listed pages: rows 4..7 of the sequence alone
    o, lse, w, _, _ = oc.attention(c, q, [2], 0.3, np.array([[[1, -1]]]))
    p = torch.softmax(torch.tensor(k[4:8] @ q[0, 0, 0] * 0.3), 0).numpy()
    assert np.allclose(o[0, 0, 0], p @ v[4:8])
    assert np.isclose(w.sum(), 4) and np.isclose(w[0, 0, 4:8].sum(), 4)


def test_selection_takes_the_best_box_and_eviction_the_heaviest():
    c = empty(5, 2, 2, [[0, 1, 2, 3]], [8])
    rows = np.array([[0, 0], [0, 0], [4, -8], [4, -8], [40, 40], [0, 0],
                     [8, 0], [-8, 0]], float)[None, None]
    oc.append(c, rows, rows, [8])
    q = np.array([[[[1.0, -1.0]]]])
    # box maxima of q: 0, 12, 40 (from the corner (40, 0)), 8
    assert oc.select(c, q, [1], 2, 0, 0)[0, 0].tolist() == [1, 2]
    assert oc.select(c, q, [1], 1, 0, 0)[0, 0].tolist() == [2]
    assert oc.select(c, q, [1], 3, 1, 1)[0, 0].tolist() == [0, 2, 3]
    assert oc.select(c, q, [0], 3, 1, 1)[0, 0].tolist() == [-1, -1, -1]
    w = np.array([[[1, 5, 5, 0, np.nan, 5, 2, 0]]], np.float32)
    out = np.zeros((1, 1, 4))
    n, kept = oc.evict(c, w, 3, 1, np.array([[4, 3]]), out)
    assert n.tolist() == [3] and kept[0, 0].tolist() == [1, 2, 7]
    assert out[0, 0].tolist() == [5, 5, 0, 0]
