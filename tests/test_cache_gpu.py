"""The cache operators on the GPU against the 64-bit oracle (oracle/cache.py).

Bounds of the floating results. A score is a sum of d fp32 products (the
tensor cores' operands are exact, too): at most (d + 8) 2^-24 of
sum_i |q_i k_i| scale off, with 2^-21 for the power of two and its argument.
A weight is then off by that share e; O, a mean of values with these weights,
by 2 e max|v|, by 2^-11 max|v| for a weight rounded to fp16 (half a step is
2^-11 of it; three pieces of 4 bits hold its 11 bits, and below 2^-18 of the
largest of its 256 tokens the error is at most 2^-26 of that, 2^-18 in all),
and by half a step of the type in the end; lse by e + 2^-22 |lse|.
"""
import numpy as np
import pytest
import torch

from cache_cases import NAN, Case, int_tensor
from oracle import cache as oc
from paper_2607_20214_gb300 import build
from paper_2607_20214_gb300 import elsaa as E

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    E.load_library()


def check_attention(case, o, lse, ref, new_len, base=None):
    ro, rl, _, size, vmax = ref
    half = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}[case.dtype]
    e = (case.d + 8) * 2.0 ** -24 * size + 2.0 ** -21
    tol = (2 * e + 2.0 ** -11 + 2.0 ** -18) * vmax
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(case.B):
        n = new_len[b]
        empty = np.isneginf(rl[b, :, :n])
        assert np.array_equal(np.isneginf(lse[b, :, :n]), empty)
        assert np.all(o[b, :, :n][empty] == 0)
        err = np.abs(o[b, :, :n] - ro[b, :, :n])
        lim = tol[b, :, :n, None] + half * np.abs(ro[b, :, :n])
        assert np.all(err <= lim), (b, float((err / np.maximum(lim, 1e-30)).max()))
        with np.errstate(invalid="ignore"):
            el = np.abs(lse[b, :, :n] - rl[b, :, :n])[~empty]
        ll = (e[b, :, :n] + 2.0 ** -22 * np.abs(rl[b, :, :n]))[~empty]
        assert np.all(el <= ll), (b, float((el / ll).max()))
        if base is not None:  # rows behind the last new token
            assert np.all(o[b, :, n:] == base)
            assert np.all(lse[b, :, n:] == base)


def run_attention(case, T=1, new_len=None, impl=0, pages=None, weights=False,
                  q_size=1.0, scale=0.0, alias=False):
    q, qd = case.rows(case.H, T, q_size)
    n = [T] * case.B if new_len is None else new_len
    cache = case.device(E, impl, scale=scale)
    o = torch.full_like(qd, 7.0)
    lse = torch.full((case.B, case.H, T), 7.0, device="cuda")
    slots = case.max_pages * case.ps
    win = wout = None
    if weights:
        win = torch.rand((case.B, case.hkv, slots), device="cuda")
        wout = win if alias else torch.full_like(win, -3.0)
        w0 = win.double().cpu().numpy()
    ws = torch.full((E.elsaa_cache_workspace_size(cache, T, weights),), 0xC7,
                    dtype=torch.uint8, device="cuda")
    pd = None if pages is None else int_tensor(pages)
    E.elsaa_cache_attention(
        cache, qd, pages=pd, o=o, lse=lse, weight_in=win, weight_out=wout,
        new_len=None if new_len is None else int_tensor(n), workspace=ws)
    E.elsaa_check_status(cache.tensors["status"])
    sc = scale or case.d ** -0.5
    ref = oc.attention(case.c, q, n, sc, pages)
    check_attention(case, o, lse, ref, n, base=7.0)
    if weights:
        e = (case.d + 8) * 2.0 ** -24 * ref[3].max() + 2.0 ** -21
        G = case.H // case.hkv
        got = wout.double().cpu().numpy()
        for b in range(case.B):
            m = case.c["lengths"][b]
            want = w0[b] + ref[2][b]
            lim = 2 * e * ref[2][b] + (G * T + 1) * 2.0 ** -24 * want
            assert np.all(np.abs(got[b] - want)[:, :m] <= lim[:, :m])
            if not alias:
                assert np.all(got[b][:, m:] == -3.0)
    return cache


IMPL = [pytest.param(0, id="auto"), pytest.param(1, id="simt")]


@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,ps,H,hkv", [
    (32, 16, 2, 2), (64, 16, 4, 4), (64, 64, 8, 2), (128, 32, 3, 3),
    (128, 128, 16, 2), (128, 16, 10, 2), (64, 128, 32, 1)])
def test_attention_one_token(impl, dtype, d, ps, H, hkv):
    """Lengths of zero, one, around pages and tiles; ragged, odd groups."""
    case = Case([1, 0, 127, 128, 129, 300, 16, 1000], H, hkv, d, ps, dtype,
                seed=d + ps + H)
    run_attention(case, impl=impl)


@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,G", [(2, 1), (5, 4), (3, 8), (17, 1), (8, 16),
                                 (64, 2)])
def test_attention_several_tokens(impl, d, T, G):
    """Each new token sees the ones before it; fewer tokens in some
    sequences, none in one, more than the sequence holds in another."""
    case = Case([130, 70, 5, 257, 1, 0, 33], 2 * G, 2, d, 32, seed=T)
    new = [T, 1, min(T, 3), max(T - 1, 1), T, 0, 0]
    run_attention(case, T=T, new_len=new, impl=impl)


@pytest.mark.parametrize("impl", IMPL)
def test_attention_without_new_len(impl):
    run_attention(Case([200, 3, 64], 4, 2, 128, 64), T=6, impl=impl)


@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("q_size,k_size", [(40.0, 1.0), (1e-3, 1e-4),
                                           (3e4, 2e-3), (1.0, 1e30)])
def test_attention_sizes_of_scores(impl, q_size, k_size):
    """One key takes all; none matters; large and small operands."""
    case = Case([400, 129], 8, 2, 128, 16, seed=3, k_size=k_size)
    run_attention(case, impl=impl, q_size=q_size,
                  scale=0.0 if k_size < 1e10 else 1e-30)


@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("d,ps", [(64, 16), (128, 64)])
def test_attention_weights(impl, d, ps):
    case = Case([500, 0, 1, 77], 8, 2, d, ps, seed=4)
    run_attention(case, T=3, new_len=[3, 0, 1, 2], impl=impl, weights=True)
    run_attention(case, impl=impl, weights=True, alias=True)


@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("d,ps", [(64, 32), (128, 16), (128, 128)])
def test_attention_listed_pages(impl, weights, d, ps):
    """Lists that end in -1, name the open page, name one page only."""
    case = Case([700, 40, 0, 300], 6, 3, d, ps, seed=5)
    pages = np.full((4, 3, 9), -1, np.int32)
    for b, n in enumerate([700, 40, 0, 300]):
        np_ = -(-n // ps)
        for h in range(3):
            take = sorted(case.rng.permutation(np_)[:max(1, min(9, np_ - h))])
            pages[b, h, :len(take)] = take
    pages[3, 0] = [-(-300 // ps) - 1] + [-1] * 8
    run_attention(case, impl=impl, pages=pages, weights=weights)
    run_attention(case, T=2, new_len=[2, 1, 0, 2], impl=impl, pages=pages,
                  weights=weights)


@pytest.mark.parametrize("impl", IMPL)
def test_long_sequence_is_shared_by_many_ctas(impl):
    run_attention(Case([40000], 4, 1, 64, 128, seed=6), impl=impl,
                  weights=True)
    run_attention(Case([9000, 1, 20, 5000], 1, 1, 128, 64, seed=7), impl=impl)


@pytest.mark.parametrize("impl", IMPL)
def test_attention_is_reproducible(impl):
    case = Case([5000, 300, 900], 8, 2, 128, 64, seed=8)
    cache = case.device(E, impl)
    _, q = case.rows(8, 2)
    w = torch.zeros((3, 2, case.max_pages * 64), device="cuda")
    runs = []
    for _ in range(3):
        lse = torch.empty((3, 8, 2), device="cuda")
        out = torch.empty_like(w)
        runs.append((E.elsaa_cache_attention(cache, q, lse=lse, weight_in=w,
                                             weight_out=out).clone(), lse,
                     out[0, :, :5000].clone()))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


@pytest.mark.parametrize("impl", IMPL)
def test_bad_pages_and_lengths_are_skipped_and_reported(impl):
    """A page outside the pool counts as absent, a length outside the table
    is clipped; the status word names the first."""
    case = Case([100, 90], 4, 2, 64, 16, seed=9)
    q, qd = case.rows(4, 1)
    for bad in (-5, len(case.c["k"]), 2 ** 31 - 1):
        cache = case.device(E, impl)
        cache.tensors["page_table"][0, 2] = bad
        lse = torch.empty((2, 4, 1), device="cuda")
        o = E.elsaa_cache_attention(cache, qd, lse=lse)
        with pytest.raises(E.ElsaaError, match="status 5"):
            E.elsaa_check_status(cache.tensors["status"])
        ref = oc.attention(case.c, q, [1, 1], 0.125,
                           skip=[case.c["table"][0, 2]])
        check_attention(case, o, lse, ref, [1, 1])
    for bad in (-1, 10 ** 6):
        cache = case.device(E, impl)
        cache.tensors["lengths"][1] = bad
        o = E.elsaa_cache_attention(cache, qd)
        with pytest.raises(E.ElsaaError, match="status"):
            E.elsaa_check_status(cache.tensors["status"])
        ref = oc.attention(case.c, q, [1, 1], 0.125)
        assert torch.isfinite(o[0]).all()
        if bad < 0:
            assert (o[1] == 0).all()


@pytest.mark.parametrize("impl", IMPL)
def test_nan_stays_in_its_row(impl):
    """A NaN key or value reaches the queries that see it and no other."""
    case = Case([100, 100], 4, 2, 128, 32, seed=10)
    case.c["v"][case.c["table"][0, 1], 0, 3, 5] = NAN
    case.c["k"][case.c["table"][1, 0], 1, 2, 7] = NAN
    _, q = case.rows(4, 1)
    o = E.elsaa_cache_attention(case.device(E, impl), q)
    nan = torch.isnan(o[:, :, 0])
    assert nan[0, :2, 5].all() and nan[0].sum() == 2
    assert nan[1, 2:].all() and not nan[1, :2].any()


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,ps", [(32, 16), (64, 128), (128, 32),
                                  (128, 128)])
@pytest.mark.parametrize("T", [1, 2, 45, 300])
def test_append(dtype, d, ps, T):
    """Into empty pages, behind older rows, over several pages; rows that
    raise a page's exponent by much, and by nothing; fewer rows than T."""
    old = [0, 1, ps - 1, ps, ps + 5, 3, 2 * ps - 1, 7]
    new = [T, T, T, T, max(T - 1, 1), min(T, 3), T, 0]
    case = Case([a + b for a, b in zip(old, new)], 2, 2, d, ps, dtype,
                seed=T + d)
    # what the pages hold behind the older rows does not matter and stays
    for b, n in enumerate(old):
        for p in range(case.max_pages - 2):
            i = case.c["table"][b, p]
            if i >= 0 and n < (p + 1) * ps:
                for x in "kv":
                    case.c[x][i, :, max(0, n - p * ps):] = 0x21
    k, kd = case.rows(2, T)
    v, vd = case.rows(2, T)
    grow = torch.tensor([1.0, 1e-3, 30.0, 1.0, 0.01, 1e4, 1.0, 1.0])
    grow = grow.to(kd.dtype).view(8, 1, 1, 1)
    kd, vd = kd * grow.cuda(), vd * grow.cuda()
    k, v = kd.double().cpu().numpy(), vd.double().cpu().numpy()
    cache = case.device(E)
    E.elsaa_cache_append(cache, kd, vd, new_len=int_tensor(new))
    E.elsaa_check_status(cache.tensors["status"])
    oc.append(case.c, k, v, new)
    assert case.same_bytes(cache) == []


def test_append_extremes():
    """Zeros, subnormals, infinities, NaN, the largest numbers."""
    for dtype, size in (("fp32", 1e-42), ("bf16", 0.0), ("fp32", 3.4e38),
                        ("bf16", 3.3e38), ("fp32", 448.0 * 2 ** 7),
                        ("fp32", float("inf"))):
        case = Case([20, 5], 2, 2, 64, 16, dtype, seed=11)
        x = torch.full((2, 2, 5, 64), size)
        x[..., 1::2] *= -1
        x[0, 0, 1, 3] = float("nan")
        if size == 448.0 * 2 ** 7:  # just above a step of the exponent
            x[1, 0, 0, 0] = float(np.nextafter(np.float32(size), np.float32(1e9)))
        xd = x.cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        cache = case.device(E)
        E.elsaa_cache_append(cache, xd, xd)
        E.elsaa_check_status(cache.tensors["status"])
        v = xd.double().cpu().numpy()
        oc.append(case.c, v, v, [5, 5])
        assert case.same_bytes(cache) == [], (dtype, size)


def test_append_token_by_token_equals_the_oracle():
    case = Case([0, 17], 2, 2, 128, 32, seed=12, extra_pages=12, spare=4)
    tab = case.c["table"]
    tab[0, :3], tab[1, 1:4] = case.free[:3], case.free[3:6]
    cache = case.device(E)
    for i in range(40):
        case.c["lengths"] += 1
        cache.tensors["lengths"] += 1
        k, kd = case.rows(2, 1, size=float(np.exp(case.rng.normal())))
        v, vd = case.rows(2, 1)
        E.elsaa_cache_append(cache, kd, vd)
        oc.append(case.c, k, v, [1, 1])
    assert case.same_bytes(cache) == []


def test_append_bad_entries_write_nothing():
    case = Case([40, 40], 2, 2, 64, 16, seed=13)
    _, x = case.rows(2, 40)
    cache = case.device(E)
    cache.tensors["page_table"][:] = len(case.c["k"])
    cache.tensors["lengths"][1] = 10 ** 9
    E.elsaa_cache_append(cache, x, x)
    with pytest.raises(E.ElsaaError, match="status"):
        E.elsaa_check_status(cache.tensors["status"])
    assert case.same_bytes(cache) == []


# ------------------------------------------------------------------ select

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,ps,H,hkv,T", [
    (64, 16, 4, 4, 1), (128, 32, 8, 2, 1), (32, 16, 2, 1, 3),
    (128, 16, 32, 2, 4), (64, 128, 3, 3, 2)])
def test_select(dtype, d, ps, H, hkv, T):
    lengths = [1000, 0, 1, ps, 5 * ps + 1, 2500]
    case = Case(lengths, H, hkv, d, ps, dtype, seed=d + T, spread=0.3)
    new = [T, 0, 1, max(1, T - 1), T, T]
    q, qd = case.rows(H, T)
    cache = case.device(E)
    for n_sel, first, last in ((4, 1, 1), (7, 0, 2), (1, 0, 0), (200, 2, 2),
                               (3, 3, 0)):
        got = E.elsaa_cache_select(cache, qd, n_sel, first, last,
                                   new_len=int_tensor(new))
        E.elsaa_check_status(cache.tensors["status"])
        ref = oc.select(case.c, q, new, n_sel, first, last)
        assert np.array_equal(got.cpu().numpy(), ref), (n_sel, first, last)


def test_select_ties_go_to_the_lower_page():
    """Equal boxes; a zero query, whose every score is 0; queries with
    infinities and NaN."""
    case = Case([900, 900], 2, 2, 64, 16, seed=14)
    case.c["bounds"][:, :, 0] = 5
    case.c["bounds"][:, :, 1] = -7
    case.c["k_scale"][:] = 0.5
    q, qd = case.rows(2, 1)
    qd[0] = 0
    qd[1, 0, 0, 3] = float("inf")
    qd[1, 1, 0, 4] = float("nan")
    q = qd.double().cpu().numpy()
    got = E.elsaa_cache_select(case.device(E), qd, 9, 0, 1)
    ref = oc.select(case.c, q, [1, 1], 9, 0, 1)
    assert np.array_equal(got.cpu().numpy(), ref)
    assert ref[0, 0].tolist() == list(range(8)) + [56]


def test_selected_pages_hold_the_best_keys():
    """All pages that matter are selected: attention over the list equals
    attention over everything when one page holds keys along the query."""
    case = Case([2000], 2, 1, 128, 32, seed=15)
    q, qd = case.rows(2, 1)
    want = 23
    i = case.c["table"][0, want]
    x = q[0, :, 0].sum(0)
    x = np.tile(x / np.abs(x).max() * 400, (32, 1))
    case.c["k"][i, 0] = oc.encode(x)
    case.c["k_scale"][i, 0] = 1.0
    hi, lo = oc._extremes(case.c["k"][i, 0])
    case.c["bounds"][i, 0] = np.stack([hi, lo])
    got = E.elsaa_cache_select(case.device(E), qd, 2, 0, 1)
    assert got[0, 0].tolist() == [want, 62]


# ------------------------------------------------------------------- evict

@pytest.mark.parametrize("d,ps,keep,recent", [
    (64, 16, 100, 10), (128, 128, 130, 0), (32, 32, 64, 64),
    (128, 16, 1, 1), (64, 64, 5000, 3), (128, 64, 777, 100)])
def test_evict(d, ps, keep, recent):
    lengths = [1500, 0, 1, keep, keep + 1, 90, 4000]
    lengths = [min(n, 5000) for n in lengths]
    need = sum(-(-min(n, keep) // ps) for n in lengths)
    case = Case(lengths, 2, 2, d, ps, seed=keep, extra_pages=need + 2)
    g = case.rng
    slots = case.max_pages * ps
    w = np.exp(2 * g.standard_normal((7, 2, slots))).astype(np.float32)
    w[g.random(w.shape) < 0.4] = 0.0
    w[g.random(w.shape) < 0.1] = 1.0
    w[0, 1, 5], w[0, 1, 9] = np.nan, np.inf
    w[4, 0, :keep // 2] = -1.0
    width = -(-keep // ps) + 1
    dst = np.full((7, width), -1, np.int32)
    at = 0
    for b, n in enumerate(lengths):
        m = -(-min(n, keep) // ps)
        dst[b, :m] = case.free[at:at + m]
        at += m
    cache = case.device(E)
    wout = torch.full((7, 2, width * ps), -3.0, device="cuda")
    kept = torch.empty((7, 2, keep), dtype=torch.int32, device="cuda")
    _, out_len = E.elsaa_cache_evict(
        cache, torch.tensor(w).cuda(), keep, recent, int_tensor(dst),
        weight_out=wout, kept=kept)
    E.elsaa_check_status(cache.tensors["status"])
    ref_w = np.full((7, 2, width * ps), -3.0)
    ref_len, ref_kept = oc.evict(case.c, w, keep, recent, dst, ref_w)
    assert np.array_equal(out_len.cpu().numpy(), ref_len)
    assert np.array_equal(kept.cpu().numpy(), ref_kept)
    assert np.array_equal(wout.double().cpu().numpy(), ref_w, equal_nan=True)
    assert case.same_bytes(cache) == []
    # without the optional output, lengths in place
    cache = case.device(E)
    E.elsaa_cache_evict(cache, torch.tensor(w).cuda(), keep, recent,
                        int_tensor(dst), lengths_out=cache.tensors["lengths"])
    assert np.array_equal(cache.tensors["lengths"].cpu().numpy(), ref_len)


# ---------------------------------------------------------------- together

def decode_loop(case, cache, steps, pages_of=None, graph=False, ws=None):
    """Steps of a decoding model: append, select, attend over the selected
    pages with weights; eager, or one captured step replayed."""
    B, H, d = case.B, case.H, case.d
    dt = cache.torch_dtype
    k = torch.empty((B, case.hkv, 1, d), dtype=dt, device="cuda")
    v, q = torch.empty_like(k), torch.empty((B, H, 1, d), dtype=dt,
                                            device="cuda")
    o = torch.empty_like(q)
    w = torch.zeros((B, case.hkv, case.max_pages * case.ps), device="cuda")
    ws = E.new_cache_workspace(cache, 1, True)
    pages = torch.empty((B, case.hkv, 6), dtype=torch.int32, device="cuda")

    def step():
        cache.tensors["lengths"] += 1
        E.elsaa_cache_append(cache, k, v)
        E.elsaa_cache_select(cache, q, 6, 1, 1, pages=pages, workspace=ws)
        E.elsaa_cache_attention(cache, q, pages=pages, weight_in=w,
                                weight_out=w, o=o, workspace=ws)

    g = None
    if graph:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                step()
        torch.cuda.current_stream().wait_stream(s)
    outs = []
    for i in range(steps):
        gen = torch.Generator(device="cuda").manual_seed(100 + i)
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        g.replay() if graph else step()
        outs.append((o.clone(), pages.clone()))
    E.elsaa_check_status(cache.tensors["status"])
    return outs, w


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
def test_decoding_against_the_oracle_and_replayed(dtype, d):
    """Append, select, attend with weights for some steps across a page
    boundary, then evict and go on; captured and replayed steps give the same
    bits as eager ones."""
    def fresh():
        return Case([200, 33, 94], 4, 2, d, 32, dtype, seed=16,
                    extra_pages=20, spare=3)
    case, other = fresh(), fresh()
    for c in (case, other):
        for b in range(3):
            t = c.c["table"][b]
            gaps = np.flatnonzero(t < 0)
            t[gaps] = c.free[3 * b:3 * b + len(gaps)]
    cache, again = case.device(E), other.device(E)
    steps = 5
    outs, w = decode_loop(case, cache, steps)
    outs2, w2 = decode_loop(other, again, steps, graph=True)
    for a, b in zip(outs, outs2):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    for b, n in enumerate((205, 38, 99)):  # rows behind are not written
        assert torch.equal(w[b, :, :n], w2[b, :, :n])
    total = np.zeros(w.shape)
    for i in range(steps):
        gen = torch.Generator(device="cuda").manual_seed(100 + i)
        x = []
        for heads in (2, 2, 4):
            r = torch.randn((3, heads, 1, d), generator=gen, device="cuda")
            x.append(r.to(cache.torch_dtype).double().cpu().numpy())
        case.c["lengths"] += 1
        oc.append(case.c, x[0], x[1], [1] * 3)
        pages = oc.select(case.c, x[2], [1] * 3, 6, 1, 1)
        assert np.array_equal(outs[i][1].cpu().numpy(), pages)
        ref = oc.attention(case.c, x[2], [1] * 3, d ** -0.5, pages)
        total += ref[2]
        o, lse = outs[i][0], torch.tensor(ref[1])
        check_attention(case, o, lse, ref, [1] * 3)
    assert case.same_bytes(cache) == []
    assert np.abs(w.double().cpu().numpy() - total).max() <= steps * 2.0 ** -16
    # evict by the device's weights and attend again
    keep = 50
    dst = np.full((3, 2), -1, np.int32)
    dst[0], dst[1], dst[2] = case.free[9:11], case.free[11:13], case.free[13:15]
    hw = w.cpu().numpy()
    w3, _ = E.elsaa_cache_evict(cache, w, keep, 8, int_tensor(dst),
                                lengths_out=cache.tensors["lengths"])
    ref_w = np.zeros((3, 2, 64))
    ref_len, _ = oc.evict(case.c, hw, keep, 8, dst, ref_w)
    assert np.array_equal(w3.double().cpu().numpy(), ref_w)
    t = cache.tensors
    small = E.make_cache(t["k"], t["v"], t["k_scale"], t["v_scale"],
                         t["bounds"], int_tensor(dst), t["lengths"], H=4,
                         dtype=dtype)
    case.c["table"], case.c["lengths"] = dst, ref_len
    q, qd = case.rows(4, 1)
    lse = torch.empty((3, 4, 1), device="cuda")
    o = E.elsaa_cache_attention(small, qd, lse=lse)
    check_attention(case, o, lse, oc.attention(case.c, q, [1] * 3, d ** -0.5),
                    [1] * 3)


def test_prompt_then_decode_matches_dense_attention():
    """A prompt appended in one call and a first token after it: attention
    over the cache is attention over the prompt, up to the 8-bit rows."""
    B, H, N, d = 2, 4, 384, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((B, H, N, d), generator=gen, device="cuda")
            .to(torch.bfloat16) for _ in "kv")
    q = torch.randn((B, H, 1, d), generator=gen, device="cuda").to(
        torch.bfloat16)
    cache = E.new_cache(B, H, H, d, 64, 2 * B * N // 64, N // 64)
    cache.tensors["page_table"].copy_(
        torch.arange(B * N // 64, dtype=torch.int32).view(B, -1))
    cache.tensors["lengths"].fill_(N)
    E.elsaa_cache_append(cache, k, v)
    o = E.elsaa_cache_attention(cache, q)
    s = (q.double() @ k.double().transpose(2, 3)) * d ** -0.5
    ref = torch.softmax(s, 3) @ v.double()
    # a row's rounding is 2^-4 of each element at most: the score moves by
    # sum |q k| 2^-4 / sqrt(d) at most, about 2^-4 |q| |k| / sqrt(d) / 3 in
    # fact; values move by 2^-4
    rel = float((o.double() - ref).norm() / ref.norm())
    assert rel < 2.0 ** -3


def test_other_stream_and_offsets_past_32_bits():
    """Pages far into a pool of more than 4 GB, work on a stream of its own."""
    num, hkv, ps, d = 300000, 1, 128, 128
    free = torch.cuda.mem_get_info()[0]
    if free < 3 * num * hkv * ps * d:
        pytest.skip("not enough memory")
    pools = [torch.zeros((num, hkv, ps, d), dtype=torch.uint8, device="cuda")
             for _ in "kv"]
    scales = [torch.ones((num, hkv), device="cuda") for _ in "kv"]
    bounds = torch.zeros((num, hkv, 2, d), dtype=torch.int8, device="cuda")
    table = int_tensor([[num - 1, num - 2, 5], [num // 2, num - 3, num - 4]])
    cache = E.make_cache(pools[0], pools[1], scales[0], scales[1], bounds,
                         table, int_tensor([300, 260]), H=2)
    s = torch.cuda.Stream()
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn((2, 1, 300, d), generator=gen, device="cuda")
            .to(torch.bfloat16) for _ in "kv")
    q = torch.randn((2, 2, 1, d), generator=gen, device="cuda").to(
        torch.bfloat16)
    torch.cuda.synchronize()
    w = torch.zeros((2, 1, 384), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        E.elsaa_cache_append(cache, k, v, new_len=int_tensor([300, 260]))
        lse = torch.empty((2, 2, 1), device="cuda")
        o = E.elsaa_cache_attention(cache, q, lse=lse, weight_in=w,
                                    weight_out=w)
        dst = int_tensor([[num - 10], [num - 11]])
        E.elsaa_cache_evict(cache, w, 100, 10, dst)
    s.synchronize()
    E.elsaa_check_status(cache.tensors["status"])
    idx = torch.tensor([[num - 1, num - 2, 5], [num // 2, num - 3, num - 4],
                        [num - 10, num - 11, 0]])
    c = dict(table=np.arange(6, dtype=np.int32).reshape(2, 3),
             lengths=np.array([300, 260], np.int32))
    at = idx.flatten().cuda()
    for x, p, sc in zip("kv", pools, scales):
        c[x] = p[at].cpu().numpy()
        c[x + "_scale"] = sc[at].cpu().numpy()
    c["bounds"] = bounds[at].cpu().numpy()
    got = {x: c[x].copy() for x in c}
    zero = {x: (np.ones_like(c[x]) if "scale" in x else
                np.zeros_like(c[x])) for x in ("k", "v", "k_scale", "v_scale",
                                               "bounds")}
    zero.update(table=c["table"], lengths=c["lengths"])
    oc.append(zero, k.double().cpu().numpy(), v.double().cpu().numpy(),
              [300, 260])
    for x in "kv":
        assert np.array_equal(oc.E4M3[got[x][:6]], oc.E4M3[zero[x][:6]])
    case = Case([1], 2, 1, d, ps)
    case.B = 2
    ref = oc.attention(zero, q.double().cpu().numpy(), [1, 1], d ** -0.5)
    check_attention(case, o, lse, ref, [1, 1])
    dst6 = np.array([[6], [7]], np.int32)
    wz = np.zeros((2, 1, 128))
    oc.evict(zero, w.cpu().numpy(), 100, 10, dst6, wz)
    for x in "kv":
        assert np.array_equal(oc.E4M3[got[x][6:8]], oc.E4M3[zero[x][6:8]])


# ---------------------------------------------------- the rules' other sides

@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("B", [32, 33, 300, 700])
def test_attention_many_sequences(impl, B):
    """The division with a sequence a lane, a sequence a thread, several a
    thread; most sequences short or empty, a few long."""
    g = np.random.default_rng(B)
    lengths = g.choice([0, 1, 2, 15, 40], B)
    lengths[g.integers(0, B, 3)] = 900
    new = np.minimum(lengths, 1)
    run_attention(Case([int(x) for x in lengths], 2, 1, 64, 16, seed=B),
                  new_len=[int(x) for x in new], impl=impl)


@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("H,hkv,T", [(1, 1, 1), (16, 1, 1), (4, 4, 1),
                                     (20, 2, 2)])
def test_attention_one_sequence_shared_by_the_most_ctas(impl, H, hkv, T):
    run_attention(Case([9000], H, hkv, 128, 128, seed=H), T=T, impl=impl)


@pytest.mark.parametrize("impl", IMPL)
def test_queries_that_are_no_numbers_stay_alone(impl):
    """NaN and infinities in one query reach no other query's row."""
    case = Case([300, 40], 8, 2, 64, 32, seed=17)
    _, q = case.rows(8, 2)
    clean = E.elsaa_cache_attention(case.device(E, impl), q)
    q[0, 1, 0, 5] = float("nan")
    q[1, 6, 1, 0] = float("inf")
    o = E.elsaa_cache_attention(case.device(E, impl), q)
    bad = torch.isnan(o).any(3)
    assert bad[0, 1, 0] and bad[1, 6, 1] and bad.sum() == 2
    assert torch.equal(o[~bad], clean[~bad])


def big_cache(pages_of_pool, ps, d, lengths, max_pages, H, hkv, seed):
    """A cache whose table names the pool's pages many times over (reading a
    page for several places is allowed)."""
    case = Case([pages_of_pool * ps], H, hkv, d, ps, seed=seed, extra_pages=0)
    c = case.c
    B = len(lengths)
    c["table"] = case.rng.integers(0, pages_of_pool, (B, max_pages)).astype(
        np.int32)
    c["lengths"] = np.array(lengths, np.int32)
    case.B, case.max_pages = B, max_pages
    return case


def test_select_from_more_pages_than_shared_memory_holds():
    case = big_cache(40, 16, 32, [20011 * 16 - 3, 700], 20011, 2, 1, 18)
    # scores that differ: every place has its own page, of 40 boxes; ties go
    # to the lower place
    q, qd = case.rows(2, 1)
    got = E.elsaa_cache_select(case.device(E), qd, 600, 2, 3)
    ref = oc.select(case.c, q, [1, 1], 600, 2, 3)
    assert np.array_equal(got.cpu().numpy(), ref)


@pytest.mark.parametrize("n", [16385, 60000, 400000])
def test_evict_long_rows(n):
    """Rows of one CTA, of a cluster, and of a cluster without room for their
    keys."""
    pages = -(-n // 16)
    case = big_cache(60, 16, 32, [n, 100], pages, 1, 1, 19)
    keep = 1000
    width = -(-keep // 16)
    num = len(case.c["k"])
    for x in ("k", "v", "k_scale", "v_scale", "bounds"):  # room for the kept
        a = case.c[x]
        case.c[x] = np.concatenate([a, np.zeros((2 * width,) + a.shape[1:],
                                                a.dtype)])
    dst = (num + np.arange(2 * width, dtype=np.int32)).reshape(2, width)
    w = np.exp(2 * case.rng.standard_normal((2, 1, pages * 16))).astype(
        np.float32)
    w[case.rng.random(w.shape) < 0.3] = 0.25
    cache = case.device(E)
    kept = torch.empty((2, 1, keep), dtype=torch.int32, device="cuda")
    wout = torch.zeros((2, 1, width * 16), device="cuda")
    _, lens = E.elsaa_cache_evict(cache, torch.tensor(w).cuda(), keep, 17,
                                  int_tensor(dst), weight_out=wout, kept=kept)
    ref_w = np.zeros((2, 1, width * 16))
    ref_len, ref_kept = oc.evict(case.c, w, keep, 17, dst, ref_w)
    assert np.array_equal(kept.cpu().numpy(), ref_kept)
    assert np.array_equal(lens.cpu().numpy(), ref_len)
    assert np.array_equal(wout.double().cpu().numpy(), ref_w)
    assert case.same_bytes(cache) == []


def test_two_graphs_share_a_workspace_and_two_streams_do_not():
    """Graphs of different sizes replayed in turn over one workspace; two
    calls at once on streams and workspaces of their own."""
    a, b = Case([3000, 10], 8, 2, 128, 64, seed=20), Case([70, 900, 5], 4, 4,
                                                        64, 16, seed=21)
    ca, cb = a.device(E), b.device(E)
    _, qa = a.rows(8, 1)
    _, qb = b.rows(4, 3)
    want = [E.elsaa_cache_attention(ca, qa), E.elsaa_cache_attention(cb, qb)]
    n = max(E.elsaa_cache_workspace_size(ca, 1),
            E.elsaa_cache_workspace_size(cb, 3))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(qa), torch.zeros_like(qb)]
    graphs = []
    side = torch.cuda.Stream()
    for c, q, o in ((ca, qa, outs[0]), (cb, qb, outs[1])):
        g = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            E.elsaa_cache_attention(c, q, o=o, workspace=ws)
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0, 0):
        outs[i].zero_()
        graphs[i].replay()
        assert torch.equal(outs[i], want[i])
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    w1 = E.new_cache_workspace(ca, 1)
    w2 = E.new_cache_workspace(cb, 3)
    torch.cuda.synchronize()
    for _ in range(20):
        outs[0].zero_(), outs[1].zero_()
        torch.cuda.synchronize()
        E.elsaa_cache_attention(ca, qa, o=outs[0], workspace=w1, stream=s1)
        E.elsaa_cache_attention(cb, qb, o=outs[1], workspace=w2, stream=s2)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_the_timing_tool_names_the_cache_kernels():
    case = Case([2000], 4, 2, 64, 32, seed=22)
    cache = case.device(E)
    _, q = case.rows(4, 1)
    _, k = case.rows(2, 1)
    w = torch.zeros((1, 2, case.max_pages * 32), device="cuda")
    E.elsaa_profile_start()
    E.elsaa_cache_append(cache, k, k)
    pages = E.elsaa_cache_select(cache, q, 40)
    E.elsaa_cache_attention(cache, q, pages=pages, weight_out=w)
    E.elsaa_cache_evict(cache, w, 32, 1, int_tensor([[case.free[0]]]))
    got = E.elsaa_profile_stop()
    assert {"cache_append", "cache_select", "cache_attn_tc", "cache_merge",
            "cache_weights", "cache_keep", "cache_compact"} <= set(got)


@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("d,ps,T,G", [(64, 16, 5, 1), (128, 128, 5, 2),
                                      (64, 64, 6, 16), (128, 16, 3, 4)])
def test_nan_of_a_later_token_stays_unseen(impl, d, ps, T, G):
    """A value or a key that is no number reaches the new tokens from its own
    on, its own channel, and no other; the new tokens lie in two tiles."""
    case = Case([130, 66, 258], 2 * G, 2, d, ps, seed=23)
    _, q = case.rows(2 * G, T)
    clean = E.elsaa_cache_attention(case.device(E, impl), q)
    want = torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
    for b, h, t, ch in ((0, 0, 1, 5), (0, 0, 2, d - 1), (0, 1, T - 1, 0),
                        (1, 0, 0, d // 2), (2, 1, 2, 7), (2, 1, 1, 7)):
        pos = int(case.c["lengths"][b]) - T + t
        case.c["v"][case.c["table"][b, pos // ps], h, pos % ps, ch] = NAN
        want[b, h * G:(h + 1) * G, t:, ch] = True
    pos = 258 - 2
    case.c["k"][case.c["table"][2, pos // ps], 0, pos % ps, 1] = NAN
    want[2, :G, T - 2:] = True
    o = E.elsaa_cache_attention(case.device(E, impl), q)
    assert torch.equal(torch.isnan(o), want)
    assert torch.equal(o[~want], clean[~want])


@pytest.mark.parametrize("impl", IMPL)
@pytest.mark.parametrize("d", [64, 128])
def test_nan_values_of_the_least_weights_are_seen(impl, d):
    """A weight too small for a float is not zero."""
    case = Case([500], 4, 2, d, 32, seed=24)
    _, q = case.rows(4, 1, 60.0)
    for h in range(2):
        for p in range(0, 500, 37):
            case.c["v"][case.c["table"][0, p // 32], h, p % 32, p % d] = NAN
    want = torch.zeros(d, dtype=torch.bool, device="cuda")
    want[[p % d for p in range(0, 500, 37)]] = True
    o = E.elsaa_cache_attention(case.device(E, impl), q)
    assert torch.equal(torch.isnan(o), want.expand(1, 4, 1, d))


@pytest.mark.parametrize("raw", [False, True])
def test_what_a_call_allocates_belongs_to_its_stream(monkeypatch, raw):
    """Not to the current one, which could give it out again meanwhile."""
    case = Case([200, 30], 4, 2, 64, 32, seed=25)
    cache = case.device(E)
    _, q = case.rows(4, 1)
    made = []
    new = E.new_cache_workspace
    monkeypatch.setattr(E, "new_cache_workspace", lambda *a: made.append(
        torch.cuda.current_stream().cuda_stream) or new(*a))
    want = E.elsaa_cache_attention(cache, q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    st = side.cuda_stream if raw else side
    pages = E.elsaa_cache_select(cache, q, 8, stream=st)
    o = E.elsaa_cache_attention(cache, q, pages=pages, stream=st)
    w = torch.ones((2, 2, case.max_pages * 32), device="cuda")
    dst = int_tensor([[case.free[0]], [case.free[1]]])
    torch.cuda.synchronize()
    wout, _ = E.elsaa_cache_evict(cache, w, 20, 4, dst, stream=st)
    side.synchronize()
    assert made == [0] + 3 * [side.cuda_stream]
    assert torch.equal(o, want)
    assert (wout.cpu()[:, :, :20] == 1).all() and wout.sum() == 80


def test_a_cache_of_another_device_is_refused(monkeypatch):
    case = Case([20], 4, 2, 64, 32, seed=26)
    cache = case.device(E)
    _, q = case.rows(4, 1)
    _, k = case.rows(2, 1)
    w = torch.zeros((1, 2, case.max_pages * 32), device="cuda")
    dst = int_tensor([[case.free[0]]])
    ws = E.new_cache_workspace(cache, 1, True, 8)
    out = torch.zeros((1, 2, 32), device="cuda"), int_tensor([0])
    pages = int_tensor([[[0, 0]]] * 2).reshape(1, 2, 2)
    monkeypatch.setattr(E, "_current_device", lambda: 1)
    for call in (lambda: E.elsaa_cache_append(cache, k, k),
                 lambda: E.elsaa_cache_select(cache, q, 2, pages=pages,
                                              workspace=ws),
                 lambda: E.elsaa_cache_attention(cache, q, o=q,
                                                 workspace=ws),
                 lambda: E.elsaa_cache_evict(cache, w, 8, 1, dst, *out,
                                             workspace=ws)):
        with pytest.raises(ValueError, match="current device"):
            call()


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("T,G,ps", [(5, 4, 16), (17, 1, 64), (6, 4, 128),
                                    (9, 2, 32)])
@pytest.mark.parametrize("lengths", [[700, 90, 0], [6000, 33]])
def test_attention_in_three_groups_of_columns(T, G, ps, lengths, weights):
    """17 to 24 queries a head, in whole items and in shared ones."""
    run_attention(Case(lengths, 2 * G, 2, 128, ps, seed=T), T=T,
                  weights=weights)


@pytest.mark.parametrize("B,H,hkv,n", [(32, 9, 9, 500), (32, 10, 10, 500),
                                       (31, 2, 2, 2040), (2, 1, 1, 900),
                                       (2, 1, 1, 500), (33, 4, 2, 500)])
def test_attention_on_both_sides_of_whole_items(B, H, hkv, n):
    """A CTA an item; more items than CTAs; items too long; more sequences
    than a warp has lanes."""
    g = np.random.default_rng(n + B)
    lengths = [n] + [int(x) for x in g.integers(0, n, B - 1)]
    run_attention(Case(lengths, H, hkv, 64, 64, seed=B, spare=0))
