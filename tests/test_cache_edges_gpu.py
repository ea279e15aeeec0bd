"""The cache operators on the GPU at the edges of their definitions, against
the 64-bit oracle (oracle/cache.py).

Bounds of O and lse. A score is a sum of d fp32 products and a few more
roundings: at most (d + 8) 2^-24 of sum_i |q_i k_i| scale off, with 2^-21 for
the power of two and its argument; a weight is off by that share e. A sum over
the tokens, of values or of weights, has at most `depth` additions one after
the other: in the CUDA-core kernel a lane adds 16 tokens of a tile of 128 at
most, then come the warp's rows (5 steps at most), four warps and the item's
pieces, no more than tiles; in the tensor-core kernel a tile's 128 tokens and
a few more. So O, a mean of values, is off by (2 e + 2 depth 2^-24) max|v| and
half a step of its type, lse by e + depth 2^-24 + 2^-22 |lse|. Only the
tensor-core kernel rounds a weight to fp16: 2^-11 of it, and 2^-18 in all for
the pieces.
"""
import numpy as np
import pytest
import torch

from cache_cases import NAN, Case, int_tensor
from oracle import cache as oc
from paper_2607_20214_gb300 import build
from paper_2607_20214_gb300 import elsaa as E

pytestmark = pytest.mark.gpu

IMPL = [pytest.param(0, id="auto"), pytest.param(1, id="simt")]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    E.load_library()


def on_tensor_cores(case, impl):
    return impl == 0 and case.dtype == "bf16" and case.d in (64, 128)


def bounds_of(case, ref, impl):
    """(bound of O without its type's rounding, bound of lse, of a weight)."""
    size, vmax = ref[3], ref[4]
    e = (case.d + 8) * 2.0 ** -24 * size + 2.0 ** -21
    tiles = -(-case.c["lengths"].astype(np.int64) // 128)
    tc = on_tensor_cores(case, impl)
    depth = (130 if tc else 17) * tiles[:, None, None] + 10
    depth = depth * 2.0 ** -24
    tol = (2 * e + 2 * depth) * vmax
    if tc:
        tol = tol + (2.0 ** -11 + 2.0 ** -18) * vmax
    return tol, e + depth, e.max() + 2 * depth.max()


def check(case, o, lse, ref, new, impl=0):
    half = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}[case.dtype]
    tol, el, _ = bounds_of(case, ref, impl)
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(case.B):
        n = new[b]
        ro, rl = ref[0][b, :, :n], ref[1][b, :, :n]
        empty = np.isneginf(rl)
        assert np.array_equal(np.isneginf(lse[b, :, :n]), empty)
        assert np.all(o[b, :, :n][empty] == 0)
        lim = tol[b, :, :n, None] + half * np.abs(ro)
        assert np.all(np.abs(o[b, :, :n] - ro) <= lim), b
        some = ~empty
        lim = (el[b, :, :n] + 2.0 ** -22 * np.abs(rl))[some]
        assert np.all(np.abs(lse[b, :, :n][some] - rl[some]) <= lim), b


def attend(case, q, qd, new, impl, pages=None, scale=0.0, weights=False):
    """Runs the call and checks all that it writes."""
    T = qd.shape[2]
    cache = case.device(E, impl, scale=scale)
    o = torch.full_like(qd, 7.0)
    lse = torch.full((case.B, case.H, T), 7.0, device="cuda")
    win = wout = None
    if weights:
        slots = case.max_pages * case.ps
        win = torch.rand((case.B, case.hkv, slots), device="cuda")
        wout = torch.full_like(win, -3.0)
    ws = torch.full((E.elsaa_cache_workspace_size(cache, T, weights),), 0xC7,
                    dtype=torch.uint8, device="cuda")
    E.elsaa_cache_attention(
        cache, qd, pages=None if pages is None else int_tensor(pages), o=o,
        lse=lse, weight_in=win, weight_out=wout, new_len=int_tensor(new),
        workspace=ws)
    E.elsaa_check_status(cache.tensors["status"])
    ref = oc.attention(case.c, q, new, scale or case.d ** -0.5, pages)
    check(case, o, lse, ref, new, impl)
    for b, n in enumerate(new):
        assert (o[b, :, n:] == 7).all() and (lse[b, :, n:] == 7).all()
    if weights:
        e = bounds_of(case, ref, impl)[2]
        GT = case.H // case.hkv * T
        got, w0 = wout.double().cpu().numpy(), win.double().cpu().numpy()
        for b, n in enumerate(case.c["lengths"]):
            want = (w0[b] + ref[2][b])[:, :n]
            lim = 2 * e * ref[2][b][:, :n] + (GT + 1) * 2.0 ** -24 * want
            assert np.all(np.abs(got[b][:, :n] - want) <= lim), b
            assert np.all(got[b][:, n:] == -3.0)


def table_case(pool, ps, d, lengths, max_pages, H, hkv, dtype, seed):
    """A cache whose table names the pool's pages many times over (reading a
    page for several places is allowed)."""
    case = Case([pool * ps], H, hkv, d, ps, dtype, seed=seed, extra_pages=0)
    case.B, case.max_pages = len(lengths), max_pages
    case.c["table"] = case.rng.integers(
        0, pool, (case.B, max_pages)).astype(np.int32)
    case.c["lengths"] = np.array(lengths, np.int32)
    return case


@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("T,G", [(1, 1), (3, 2), (5, 4)])
def test_queries_of_zeros_at_the_smallest_scales(impl, weights, T, G):
    """Every key counts the same for a query of zeros, whatever the scale;
    rows behind new_len, which are taken as zeros, reach no weight."""
    for scale in (1e-30, 1e-45, 1e-3):
        case = Case([300, 40, 5, 0, 128], 2 * G, 2, 64, 16, seed=T)
        q, qd = case.rows(2 * G, T)
        q[0], q[1, 0], q[2, :, T - 1] = 0, 0, 0
        qd.copy_(torch.tensor(q))
        new = [T, max(T - 1, 1), min(T, 2), 0, 1]
        attend(case, q, qd, new, impl, scale=scale, weights=weights)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("ps", [16, 32, 128])
def test_channels_that_hold_no_number_count_as_the_widest(dtype, d, ps):
    """Pages whose keys are all NaN in some channels, in a channel of
    infinities, everywhere; they grow, are selected from and evicted from."""
    case = Case([30 * ps, 9 * ps], 4, 2, d, ps, dtype, seed=d + ps,
                spread=0.3, extra_pages=12)
    k = case.rng.standard_normal((2, 2, 30 * ps, d))
    for p in range(0, 30, 3):
        k[:, :, p * ps:(p + 1) * ps, case.rng.permutation(d)[:d // 3]] = np.nan
    k[0, 0, 5 * ps:6 * ps] = np.nan
    k[0, 1, 7 * ps:8 * ps, :5] = -np.inf
    k[0, 1, 7 * ps:8 * ps, 5:9] = np.inf
    k[0, 1, 7 * ps:8 * ps:2, 3:7] = np.nan
    cache = case.device(E)
    kd = torch.tensor(k).cuda().to(cache.torch_dtype)
    k = kd.double().cpu().numpy()
    # the last page in two parts, then whole
    for end in (30 * ps - ps // 2, 30 * ps - 1, 30 * ps):
        n = [30 * ps - ps // 2 if end < 30 * ps - 1 else
             end - (30 * ps - ps // 2) if end < 30 * ps else 1, 0]
        t0 = end - n[0]
        if t0 == 0:
            n[1] = 9 * ps
        rows = max(n)
        part = np.zeros((2, 2, rows, d))
        part[0, :, :n[0]] = k[0, :, t0:end]
        part[1, :, :n[1]] = k[1, :, :n[1]]
        case.c["lengths"][0] = end
        cache.tensors["lengths"][0] = end
        pd = torch.tensor(part).cuda().to(cache.torch_dtype)
        E.elsaa_cache_append(cache, pd, pd, new_len=int_tensor(n))
        oc.append(case.c, part, part, n)
        assert case.same_bytes(cache) == []
    assert (case.c["bounds"][:, :, 0] >= case.c["bounds"][:, :, 1]).all()
    q, qd = case.rows(4, 1)
    for n_sel, first, last in ((8, 0, 0), (13, 1, 1)):
        got = E.elsaa_cache_select(cache, qd, n_sel, first, last)
        assert np.array_equal(got.cpu().numpy(),
                              oc.select(case.c, q, [1, 1], n_sel, first, last))
    keep = 3 * ps + 1
    w = np.zeros((2, 2, case.max_pages * ps), np.float32)
    w[:, :, :ps], w[:, :, 5 * ps:6 * ps], w[:, :, 7 * ps:8 * ps] = 3, 2, 1
    dst = case.free[:8].reshape(2, 4).astype(np.int32)
    E.elsaa_cache_evict(cache, torch.tensor(w).cuda(), keep, 1,
                        int_tensor(dst))
    oc.evict(case.c, w, keep, 1, dst, np.zeros((2, 2, 4 * ps)))
    assert case.same_bytes(cache) == []


def test_select_with_large_queries_and_small_keys():
    """The score fits fp32 where the query's part of it does not."""
    case = Case([600], 2, 1, 64, 16, seed=31)
    case.c["k_scale"][:] = 2.0 ** case.rng.integers(
        -60, -50, case.c["k_scale"].shape)
    q, qd = case.rows(2, 1, size=2.0 ** 125)
    got = E.elsaa_cache_select(case.device(E), qd, 9, 0, 0)
    ref = oc.select(case.c, q, [1], 9, 0, 0)
    assert np.array_equal(got.cpu().numpy(), ref)


def test_select_scores_beyond_fp32_tie():
    case = Case([600], 1, 1, 64, 16, seed=32)
    case.c["bounds"][:, :, 0], case.c["bounds"][:, :, 1] = 100, -100
    case.c["k_scale"][:] = 2.0 ** 119
    case.c["k_scale"][case.c["table"][0, 20]] = 2.0 ** 120
    qd = torch.full((1, 1, 1, 64), 2.0 ** 100, device="cuda",
                    dtype=torch.bfloat16)
    got = E.elsaa_cache_select(case.device(E), qd, 5, 0, 0)
    assert got[0, 0].tolist() == [0, 1, 2, 3, 4]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64),
                                     ("bf16", 32)])
@pytest.mark.parametrize("B,max_pages", [(5, 257), (5, 1024), (3, 5000),
                                         (2, 16384), (40, 1024), (76, 300)])
def test_select_by_clusters(dtype, d, B, max_pages):
    """Several CTAs score the pages of a sequence and head and leave the keys
    with the first: all of them with pages, some without, several rounds
    each; sequences full, empty and in between; clusters smaller than the
    pages ask for."""
    lengths = [max_pages * 16, 0, 16 * 255 + 3, 1, 16 * 256 + 1] + 71 * [70]
    case = table_case(50, 16, d, [min(n, max_pages * 16) for n in lengths[:B]],
                      max_pages, 4, 2, dtype, seed=max_pages)
    new = ([1, 1, 2, 1, 2] + 71 * [1])[:B]
    q, qd = case.rows(4, 2)
    cache = case.device(E)
    for n_sel, first, last in ((40, 1, 1), (300, 0, 3)):
        got = E.elsaa_cache_select(cache, qd, n_sel, first, last,
                                   new_len=int_tensor(new))
        E.elsaa_check_status(cache.tensors["status"])
        ref = oc.select(case.c, q, new, n_sel, first, last)
        assert np.array_equal(got.cpu().numpy(), ref), (n_sel, first, last)


def test_select_passes_over_pages_outside_the_pool():
    """They rank behind every page, and are recorded."""
    case = Case([600, 300], 2, 2, 64, 16, seed=33, extra_pages=4)
    q, qd = case.rows(2, 1)
    cache = case.device(E)
    num = len(case.c["k"])
    for b, p, bad in ((0, 3, num), (0, 36, -7), (1, 0, 2 ** 31 - 1)):
        cache.tensors["page_table"][b, p] = bad
        case.c["table"][b, p] = case.free[0]
    # in the oracle: a page of score -inf
    i = case.free[0]
    case.c["k_scale"][i] = -np.inf
    case.c["bounds"][i, :, 0], case.c["bounds"][i, :, 1] = 1, -1
    for n_sel, first, last in ((9, 0, 0), (35, 0, 1), (60, 1, 1)):
        got = E.elsaa_cache_select(cache, qd, n_sel, first, last)
        ref = oc.select(case.c, q, [1, 1], n_sel, first, last)
        assert np.array_equal(got.cpu().numpy(), ref)
    with pytest.raises(E.ElsaaError, match="status 5"):
        E.elsaa_check_status(cache.tensors["status"])


@pytest.mark.parametrize("d,ps", [(64, 16), (128, 128), (32, 32)])
def test_evict_with_pages_outside_the_pool(d, ps):
    """Tokens kept from such a page become zeros, pages that should go to
    one are not written, and the first is recorded."""
    lengths = [20 * ps + 3, 7 * ps]
    keep = 3 * ps
    case = Case(lengths, 2, 2, d, ps, seed=34, extra_pages=9)
    w = np.exp(case.rng.standard_normal((2, 2, case.max_pages * ps)))
    w = w.astype(np.float32)
    w[0, :, 5 * ps:5 * ps + 9] = 1e9
    w[1, 1, 2 * ps:3 * ps:2] = 1e9
    dst = case.free[:6].reshape(2, 3).astype(np.int32)
    cache = case.device(E)
    num = len(case.c["k"])
    zero = case.free[6]
    for b, p, bad in ((0, 5, num), (0, 20, -1), (1, 2, 2 ** 31 - 1)):
        cache.tensors["page_table"][b, p] = bad
        case.c["table"][b, p] = zero
    for x in "kv":  # in the oracle: a page of zeros
        case.c[x][zero] = 0
        case.c[x + "_scale"][zero] = 2.0 ** -64
    on_device = dst.copy()
    on_device[1, 1] = num + 5
    spare = dst[1, 1]
    was = {x: case.c[x][[zero, spare]].copy() for x in
           ("k", "v", "k_scale", "v_scale", "bounds")}
    for x in ("k", "v"):  # the device's page was not touched above
        was[x][0] = NAN
        was[x + "_scale"][0] = np.nan
    kept = torch.empty((2, 2, keep), dtype=torch.int32, device="cuda")
    wout = torch.zeros((2, 2, 3 * ps), device="cuda")
    _, lens = E.elsaa_cache_evict(cache, torch.tensor(w).cuda(), keep, 5,
                                  int_tensor(on_device), weight_out=wout,
                                  kept=kept)
    with pytest.raises(E.ElsaaError, match="status 5"):
        E.elsaa_check_status(cache.tensors["status"])
    ref_w = np.zeros((2, 2, 3 * ps))
    ref_len, ref_kept = oc.evict(case.c, w, keep, 5, dst, ref_w)
    assert np.array_equal(lens.cpu().numpy(), ref_len)
    assert np.array_equal(kept.cpu().numpy(), ref_kept)
    assert np.array_equal(wout.double().cpu().numpy(), ref_w)
    for x in was:
        case.c[x][[zero, spare]] = was[x]
    assert case.same_bytes(cache) == []


@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("weights", [False, True])
def test_lists_in_any_order_with_others_behind(impl, weights):
    """Pages in any order, entries outside the sequence's behind them, lists
    longer than the sequence has pages or the table entries."""
    case = Case([700, 40, 0, 300], 6, 3, 64, 32, seed=35)
    pages = np.resize(np.array([99, -3, 2 ** 31 - 1, -2 ** 31, 26, 22, -1],
                               np.int32), (4, 3, 40))
    for b, n in enumerate([700, 40, 0, 300]):
        p = case.rng.permutation(-(-n // 32))
        for h in range(3):
            take = p[:max(0, len(p) - h)]
            pages[b, h, :len(take)] = take
    q, qd = case.rows(6, 3)
    attend(case, q, qd, [3, 2, 1, 3], impl, pages=pages, weights=weights)


@pytest.mark.parametrize("dtype,d,impl", [
    ("fp32", 32, 0), ("fp32", 64, 0), ("fp32", 128, 0), ("bf16", 32, 0),
    ("bf16", 64, 1), ("bf16", 128, 1), ("bf16", 64, 0), ("bf16", 128, 0)])
@pytest.mark.parametrize("T,G,ps", [(1, 1, 16), (1, 4, 64), (2, 3, 32),
                                    (5, 4, 16), (7, 1, 128), (16, 8, 32)])
@pytest.mark.parametrize("weights", [False, True])
def test_attention_within_its_kernels_own_bound(dtype, d, impl, T, G, ps,
                                                weights):
    """Every type and head size with several tokens and weights; short
    sequences, where a weight in half precision would show, and longer."""
    case = Case([9, 130, 0, 1000, 128, 1, 16], 2 * G, 2, d, ps, dtype,
                seed=d + T)
    q, qd = case.rows(2 * G, T)
    new = [T, max(T - 1, 1), min(T, 2), T, T, 1, 0]
    attend(case, q, qd, new, impl, weights=weights)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("fp32", 64),
                                     ("fp32", 128), ("bf16", 32)])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 6), (4, 2)])
@pytest.mark.parametrize("weights", [False, True])
def test_listed_pages_on_cuda_cores(dtype, d, T, G, weights):
    case = Case([700, 40, 0, 300], 3 * G, 3, d, 32, dtype, seed=36)
    pages = np.full((4, 3, 9), -1, np.int32)
    for b, n in enumerate([700, 40, 0, 300]):
        for h in range(3):
            take = sorted(case.rng.permutation(-(-n // 32))[:9 - h])
            pages[b, h, :len(take)] = take
    q, qd = case.rows(3 * G, T)
    attend(case, q, qd, [T, 1, 0, T], 0, pages=pages, weights=weights)


@pytest.mark.parametrize("impl", IMPL)
def test_lengths_outside_the_table_are_clipped(impl):
    """A negative length is none, one beyond the table is the table's, whose
    entries behind the last page are skipped; the others are as ever."""
    case = Case([100, 90], 4, 2, 64, 16, seed=37)
    q, qd = case.rows(4, 1)
    for bad in (-1, -2 ** 31, 10 ** 6, 2 ** 31 - 1):
        cache = case.device(E, impl)
        cache.tensors["lengths"][1] = bad
        # six pages of the second sequence are whole but for 6 rows, which
        # hold NaN: numbers, so that the clipped length can be compared
        k = {x: case.c[x].copy() for x in "kv"}
        last = case.c["table"][1, 5]
        for x in "kv":
            case.c[x][last, :, 10:] = 0x30
            cache.tensors[x].copy_(torch.tensor(case.c[x]))
        lse = torch.empty((2, 4, 1), device="cuda")
        o = E.elsaa_cache_attention(cache, qd, lse=lse)
        with pytest.raises(E.ElsaaError, match="status"):
            E.elsaa_check_status(cache.tensors["status"])
        was = case.c["lengths"].copy()
        case.c["lengths"][1] = 0 if bad < 0 else 96
        ref = oc.attention(case.c, q, [1, 1], 0.125)
        check(case, o, lse, ref, [1, 1], impl)
        case.c["lengths"][:] = was
        case.c.update(k)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_decoding_step_by_step(dtype, d):
    """Append, select, attend over the selected pages with weights, in every
    step all that is written against the oracle, lse too."""
    case = Case([200, 33, 94], 4, 2, d, 32, dtype, seed=38, extra_pages=20,
                spare=3)
    for b in range(3):
        t = case.c["table"][b]
        gaps = np.flatnonzero(t < 0)
        t[gaps] = case.free[3 * b:3 * b + len(gaps)]
    cache = case.device(E)
    w = torch.zeros((3, 2, case.max_pages * 32), device="cuda")
    total = 0.0
    for step in range(6):
        case.c["lengths"] += 1
        cache.tensors["lengths"] += 1
        (k, kd), (v, vd) = case.rows(2, 1), case.rows(2, 1)
        q, qd = case.rows(4, 1)
        E.elsaa_cache_append(cache, kd, vd)
        oc.append(case.c, k, v, [1] * 3)
        pages = E.elsaa_cache_select(cache, qd, 5)
        ref = oc.select(case.c, q, [1] * 3, 5, 1, 1)
        assert np.array_equal(pages.cpu().numpy(), ref)
        lse = torch.full((3, 4, 1), 7.0, device="cuda")
        o = E.elsaa_cache_attention(cache, qd, pages=pages, lse=lse,
                                    weight_in=w, weight_out=w)
        ref = oc.attention(case.c, q, [1] * 3, d ** -0.5, ref)
        check(case, o, lse, ref, [1] * 3)
        total = total + ref[2]
    E.elsaa_check_status(cache.tensors["status"])
    assert case.same_bytes(cache) == []
    assert np.abs(w.double().cpu().numpy() - total).max() <= 6 * 2.0 ** -17


@pytest.mark.parametrize("impl", IMPL)
def test_attention_with_the_most_heads(impl):
    """2^26 items, one key each: their number times the CTAs that may share
    one does not fit in 32 bits. O is the key's value."""
    B, H, d, ps = 4096, 16384, 64, 16
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    cache = E.new_cache(B, H, H, d, ps, 1, 1, impl=impl)
    t = cache.tensors
    gen = torch.Generator(device="cuda").manual_seed(40)
    t["page_table"].zero_()
    t["lengths"].fill_(1)
    v = torch.randn((1, H, ps, d), generator=gen, device="cuda")
    t["v"].copy_(v)
    t["k"].copy_(v)
    t["v_scale"].fill_(0.25)
    q = torch.empty((B, H, 1, d), dtype=torch.bfloat16, device="cuda")
    q.normal_(generator=gen)
    o = torch.full_like(q, 7.0)
    lse = torch.full((B, H, 1), 7.0, device="cuda")
    E.elsaa_cache_attention(cache, q, o=o, lse=lse)
    E.elsaa_check_status(t["status"])
    want = (t["v"][0, :, :1].float() * 0.25).to(torch.bfloat16)  # [H, 1, d]
    key = t["k"][0, :, 0].float()
    for b in range(0, B, 256):
        assert (o[b:b + 256] == want).all()
        x = q[b:b + 256, :, 0].float() * key
        s, size = x.sum(2) / 8, x.abs().sum(2) / 8
        assert ((lse[b:b + 256, :, 0] - s).abs() <=
                3 * (d + 8) * 2.0 ** -24 * size + 2.0 ** -21).all()
