"""Exact attention and its backward pass against the 64-bit oracle."""
import math

import numpy as np
import pytest
import torch

import layer_cases as C
from paper_2607_20214_gb300 import elsaa as E

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "fp32"}
SIMT = E.ELSAA_IMPL_SIMT


def lens(x, B, dev="cuda"):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def run_case(B, H, Hkv, Nq, Nk, d, dtype=BF, causal=True, ql=None, kl=None,
             impl=0, scale=0.0, seed=0, spread=1.5, backward=True):
    """Forward and backward of one case against the oracle; behind the lengths
    the inputs hold NaN, and what the outputs held stays."""
    q, k, v, do = C.exact_inputs(B, H, Hkv, Nq, Nk, d, dtype, seed, spread)
    qn, kn = ql or [Nq] * B, kl or [Nk] * B
    tensor = dtype == BF and impl != SIMT
    sc = scale or 1.0 / math.sqrt(d)
    ref = C.exact_forward_ref(q, k, v, sc, causal, qn, kn, tensor)
    for b in range(B):
        q[b, :, qn[b]:] = math.nan
        do[b, :, qn[b]:] = math.nan
        k[b, :, kn[b]:] = math.nan
        v[b, :, kn[b]:] = math.nan
    ex = E.make_exact(B, H, Hkv, Nq, Nk, d, dtype=NAME[dtype], causal=causal,
                      scale=scale, impl=impl)
    qg, kg, vg, dog = (x.cuda() for x in (q, k, v, do))
    o = torch.full_like(qg, 7.0)
    lse = torch.full((B, H, Nq), 7.0, device="cuda")
    ws = E.new_exact_workspace(ex, qg.device, backward=True)
    kw = dict(q_len=lens(ql, B) if ql else None,
              k_len=lens(kl, B) if kl else None, workspace=ws)
    E.elsaa_exact_forward(ex, qg, kg, vg, o=o, lse=lse, **kw)
    E.elsaa_check_status(ws)
    for (b, h), r in ref.items():
        n = qn[b]
        C.close(o[b, h, :n], r["o"], r["o_tol"], ("o", b, h))
        C.close(lse[b, h, :n], r["lse"], r["lse_tol"], ("lse", b, h))
        assert (o[b, h, n:] == 7).all() and (lse[b, h, n:] == 7).all()
    if not backward:
        return
    oo, ll = o.clone(), lse.clone()
    for b in range(B):
        oo[b, :, qn[b]:] = math.nan
        ll[b, :, qn[b]:] = math.nan
    back = C.exact_backward_ref(q, k, v, o, lse, do, sc, causal, qn, kn,
                                tensor)
    grads = [torch.full_like(x, 7.0) for x in (qg, kg, vg)]

    def go():
        E.elsaa_exact_backward(ex, qg, kg, vg, oo, ll, dog, dq=grads[0],
                               dk=grads[1], dv=grads[2], **kw)
        E.elsaa_check_status(ws)
    go()
    for name, g, rows in zip(("dq", "dk", "dv"), grads, (qn, kn, kn)):
        for (b, h), (val, tol) in back[name].items():
            C.close(g[b, h, :rows[b]], val, tol, (name, b, h))
            assert (g[b, h, rows[b]:] == 7).all(), (name, b, h)
    first = [g.clone() for g in grads]
    go()
    for g, f in zip(grads, first):
        assert torch.equal(g, f)  # the same bits again


KINDS = [(BF, 0), (BF, SIMT), (F32, 0)]


@pytest.mark.parametrize("dtype,impl", KINDS)
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("N", [1, 2, 127, 128, 129, 300])
def test_lengths(N, causal, d, dtype, impl):
    run_case(1, 2, 1, N, N, d, dtype, causal, impl=impl)


@pytest.mark.parametrize("dtype,impl", KINDS)
@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,causal", [
    (2, 8, 2, 1, 700, 1), (1, 4, 4, 1, 1, 0), (1, 6, 2, 3, 257, 1),
    (2, 3, 1, 130, 500, 1), (1, 2, 2, 300, 70, 1), (1, 5, 1, 200, 33, 0),
    (3, 4, 2, 65, 64, 1), (1, 16, 1, 100, 129, 0)])
def test_groups_and_unequal_lengths(B, H, Hkv, Nq, Nk, causal, dtype, impl):
    run_case(B, H, Hkv, Nq, Nk, 64, dtype, causal, impl=impl)


@pytest.mark.parametrize("dtype,impl", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [0, 1])
def test_padded_batches(causal, d, dtype, impl):
    run_case(6, 4, 2, 190, 333, d, dtype, causal,
             ql=[190, 0, 1, 129, 64, 190], kl=[333, 200, 1, 0, 128, 100],
             impl=impl)


@pytest.mark.parametrize("dtype,impl", KINDS)
def test_lengths_outside_are_clipped(dtype, impl):
    q, k, v, _ = (x.cuda() for x in C.exact_inputs(2, 2, 1, 40, 50, 64, dtype))
    ex = E.make_exact(2, 2, 1, 40, 50, 64, dtype=NAME[dtype], causal=True,
                      impl=impl)
    o = torch.zeros_like(q)
    E.elsaa_exact_forward(ex, q, k, v, q_len=lens([100, -5], 2),
                          k_len=lens([1000, 50], 2), o=o)
    want = E.elsaa_exact_forward(ex, q, k, v)
    assert torch.equal(o[0], want[0]) and not o[1].any()


@pytest.mark.parametrize("dtype,impl", KINDS)
@pytest.mark.parametrize("spread,scale", [(0.0, 0.0), (1e-20, 0.0),
                                          (12.0, 0.0), (1.5, 4.0)])
def test_flat_and_peaked_scores(spread, scale, dtype, impl):
    run_case(1, 2, 1, 150, 150, 64, dtype, 1, impl=impl, spread=spread,
             scale=scale, backward=spread < 2 and scale == 0)


@pytest.mark.parametrize("dtype,impl", KINDS)
def test_rising_scores(dtype, impl):
    """The maximum grows from tile to tile, by more than fp32's exponents hold
    in a weight."""
    q, k, v, _ = C.exact_inputs(1, 1, 1, 70, 600, 64, dtype)
    q[..., 0], k[..., 0] = 8.0, torch.linspace(-200, 200, 600).to(dtype)
    ref = C.exact_forward_ref(q, k, v, 0.125, 0, [70], [600],
                              dtype == BF and impl == 0)[0, 0]
    ex = E.make_exact(1, 1, 1, 70, 600, 64, dtype=NAME[dtype], impl=impl)
    lse = torch.empty((1, 1, 70), device="cuda")
    o = E.elsaa_exact_forward(ex, q.cuda(), k.cuda(), v.cuda(), lse=lse)
    C.close(o[0, 0], ref["o"], ref["o_tol"], "o")
    C.close(lse[0, 0], ref["lse"], ref["lse_tol"], "lse")


@pytest.mark.parametrize("dtype,impl", KINDS)
def test_scores_of_minus_infinity_are_no_weight(dtype, impl):
    """A key whose scores are -inf counts for nothing; a query that has none
    other is one that sees nothing."""
    q, k, v, _ = C.exact_inputs(1, 1, 1, 64, 200, 64, dtype)
    q[..., 0] = q[..., 0].abs() + 1
    k[0, 0, ::3, 0] = -math.inf
    ex = E.make_exact(1, 1, 1, 64, 200, 64, dtype=NAME[dtype], impl=impl)
    keep = [j for j in range(200) if j % 3]
    ref = C.exact_forward_ref(q, k[:, :, keep], v[:, :, keep], 0.125, 0, [64],
                              [len(keep)], dtype == BF and impl == 0)[0, 0]
    lse = torch.empty((1, 1, 64), device="cuda")
    o = E.elsaa_exact_forward(ex, q.cuda(), k.cuda(), v.cuda(), lse=lse)
    C.close(o[0, 0], ref["o"], ref["o_tol"], "o")
    C.close(lse[0, 0], ref["lse"], ref["lse_tol"], "lse")
    k[0, 0, :, 0] = -math.inf
    o = E.elsaa_exact_forward(ex, q.cuda(), k.cuda(), v.cuda(), lse=lse)
    assert not o.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("G,Nq", [(2, 300), (1, 1000), (3, 129)])
def test_many_padded_sequences(G, Nq):
    """More items than are divided into shares, of sequences that need fewer
    tiles than the batch: every row is written, some sequences against the
    oracle, and nothing behind the lengths."""
    B, Hkv, d, Nk = 90, 8, 32, 260
    q, k, v, _ = C.exact_inputs(B, Hkv * G, Hkv, Nq, Nk, d, BF)
    ql = [(b * 37) % (Nq + 1) for b in range(B)]
    kl = [(b * 101) % (Nk + 1) for b in range(B)]
    ql[1], ql[2], kl[3] = 128, Nq, Nk
    ex = E.make_exact(B, Hkv * G, Hkv, Nq, Nk, d, causal=True)
    o = torch.full(q.shape, 7.0, dtype=BF, device="cuda")
    lse = torch.full(q.shape[:3], math.nan, device="cuda")
    E.elsaa_exact_forward(ex, q.cuda(), k.cuda(), v.cuda(), o=o, lse=lse,
                          q_len=lens(ql, B), k_len=lens(kl, B))
    for b in range(B):
        n = ql[b]
        assert not lse[b, :, :n].isnan().any()
        assert lse[b, :, n:].isnan().all() and (o[b, :, n:] == 7).all()
    for b in (1, 2, 3, 40):
        one = [x[b:b + 1] for x in (q, k, v)]
        ref = C.exact_forward_ref(*one, 1 / math.sqrt(d), True, [ql[b]],
                                  [kl[b]], True)
        for (_, h), r in ref.items():
            C.close(o[b, h, :ql[b]], r["o"], r["o_tol"], ("o", b, h))
            C.close(lse[b, h, :ql[b]], r["lse"], r["lse_tol"], ("lse", b, h))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("dtype,impl", KINDS)
def test_gradients_where_finite_rows_score_minus_infinity(dtype, impl, d,
                                                          causal):
    """A query whose scores with every key overflow has no weights: its
    gradient is 0, and the others' are those without it (in the same order,
    so the same bits)."""
    q, k, v, do = C.exact_inputs(1, 2, 1, 70, 150, d, dtype)
    q[..., 0] = 0
    k[..., 0] = -1e20
    ex = E.make_exact(1, 2, 1, 70, 150, d, dtype=NAME[dtype], causal=causal,
                      impl=impl)

    def run(q, do):
        x = [t.cuda() for t in (q, k, v)]
        lse = torch.empty((1, 2, 70), device="cuda")
        o = E.elsaa_exact_forward(ex, *x, lse=lse)
        return o, lse, E.elsaa_exact_backward(ex, *x, o, lse, do.cuda())
    q1 = q.clone()
    q1[0, 1, 5, 0] = 1e20
    o, lse, got = run(q1, do)
    assert not o[0, 1, 5].any() and lse[0, 1, 5] == -math.inf
    do[0, 1, 5] = 0
    o0, lse0, want = run(q, do)
    assert lse0[0, 1, 5] > -math.inf
    assert not got[0][0, 1, 5].any()
    want[0][0, 1, 5] = 0
    for x, y in zip(got, want):
        assert torch.equal(x, y) and x.isfinite().all()


def test_infinite_scores_do_not_reach_other_rows():
    q, k, v, _ = (x.cuda() for x in C.exact_inputs(1, 2, 1, 200, 200, 64, BF))
    ex = E.make_exact(1, 2, 1, 200, 200, 64)
    want = E.elsaa_exact_forward(ex, q, k, v)
    q[0, 1, 77] = math.nan
    got = E.elsaa_exact_forward(ex, q, k, v)
    assert got[0, 1, 77].isnan().all()
    got[0, 1, 77] = want[0, 1, 77]
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_streams_graphs_and_two_calls_at_once(dtype):
    ins = [C.exact_inputs(1, 4, 2, 260, 260, 64, dtype, s) for s in (0, 1)]
    ins = [[x.cuda() for x in i] for i in ins]
    ex = E.make_exact(1, 4, 2, 260, 260, 64, dtype=NAME[dtype], causal=True)

    def step(x, out, ws, stream=None):
        q, k, v, do = x
        o, lse, dq, dk, dv = out
        E.elsaa_exact_forward(ex, q, k, v, o=o, lse=lse, workspace=ws,
                              stream=stream)
        E.elsaa_exact_backward(ex, q, k, v, o, lse, do, dq=dq, dk=dk, dv=dv,
                               workspace=ws, stream=stream)

    def buffers(x):
        return [torch.zeros_like(x[0]),
                torch.zeros(x[0].shape[:3], device="cuda")] + [
                    torch.zeros_like(t) for t in x[:3]]
    want = [buffers(x) for x in ins]
    ws = [E.new_exact_workspace(ex, "cuda", backward=True) for _ in ins]
    for x, w in zip(ins, want):
        step(x, w, ws[0])
    torch.cuda.synchronize()
    # two streams at once, a workspace each
    got = [buffers(x) for x in ins]
    streams = [torch.cuda.Stream() for _ in ins]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for x, g, w, s in zip(ins, got, ws, streams):
            step(x, g, w, s)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))
    # captured over one workspace, replayed on other contents
    got = [buffers(x) for x in ins]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x, g in zip(ins, got):
            step(x, g, ws[0])
    for a, b in zip(ins[0], ins[1]):
        t = a.clone()
        a.copy_(b)
        b.copy_(t)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for g, w in zip(got, want[::-1]):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_lengths_are_read_when_the_graph_runs():
    q, k, v, _ = (x.cuda() for x in C.exact_inputs(2, 2, 2, 150, 150, 64, BF))
    ex = E.make_exact(2, 2, 2, 150, 150, 64, causal=True)
    ws = E.new_exact_workspace(ex, "cuda")
    n = lens([150, 150], 2)
    o = torch.zeros_like(q)
    E.elsaa_exact_forward(ex, q, k, v, q_len=n, k_len=n, o=o, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        E.elsaa_exact_forward(ex, q, k, v, q_len=n, k_len=n, o=o, workspace=ws)
    n.copy_(lens([20, 140], 2))
    o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    full = E.elsaa_exact_forward(ex, q, k, v)
    assert torch.equal(o[0, :, :20], full[0, :, :20])
    assert torch.equal(o[1, :, :140], full[1, :, :140])
    assert not o[0, :, 20:].any() and not o[1, :, 140:].any()


def test_causal_forward_agrees_with_the_causal_base():
    """elsaa_forward's causal variant with one base segment and lambda = 0 is
    this operator up to its denominator's eps."""
    from paper_2607_20214_gb300.workloads import Workload
    wl = Workload("one_segment", B=1, H=2, N=512, d_h=64, dtype="bf16",
                  block=64, race_tables=4, recipe="plain", temperature=2.0,
                  seed=5, plane_seed=1005, causal=1, causal_base_len=512,
                  lam=0.0)
    from paper_2607_20214_gb300.workloads import make_inputs
    x = {k: t.cuda() for k, t in make_inputs(wl).items()}
    p = E.params_for(wl)
    p.fusion_mode = 1
    gates = torch.zeros((1, 2, 512, 2), device="cuda")
    gates[..., 0] = 1.0
    o = E.elsaa_forward(p, x["q"], x["k"], x["v"], x["w_sort"], x["w_race"],
                        gates=gates)
    ex = E.make_exact(1, 2, 2, 512, 512, 64, causal=True, scale=p.scale)
    got = E.elsaa_exact_forward(ex, x["q"], x["k"], x["v"])
    # either rounds weights (2^-8 of sum P |v|) and the result
    ref = C.exact_forward_ref(*(x[n].cpu() for n in "qkv"),
                              p.scale or 0.125, 1, [512], [512], True)
    for h in range(2):
        r = ref[0, h]
        C.close(o[0, h], C.f64(got[0, h]),
                2 * (r["o_tol"] + 1e-5 * r["o_mag"]), h)


def test_many_heads_and_rows():
    run_case(3, 40, 5, 33, 200, 32, BF, 1, backward=True)
    run_case(2, 2, 2, 700, 900, 128, BF, 1)


def test_argument_checks():
    q, k, v, _ = (x.cuda() for x in C.exact_inputs(1, 2, 1, 8, 8, 64, BF))
    ex = E.make_exact(1, 2, 1, 8, 8, 64)
    with pytest.raises(ValueError):
        E.elsaa_exact_forward(ex, q[:, :1], k, v)
    with pytest.raises(ValueError):
        E.elsaa_exact_forward(ex, q.float(), k, v)
    with pytest.raises(ValueError):
        E.elsaa_exact_forward(ex, q, k.cpu(), v)
    with pytest.raises(ValueError):
        E.elsaa_exact_forward(ex, q.transpose(1, 2).contiguous()
                              .transpose(1, 2), k, v)
    with pytest.raises(ValueError):
        E.elsaa_exact_forward(ex, q, k, v, lse=torch.zeros(1, 2, 9,
                                                           device="cuda"))
    with pytest.raises(E.ElsaaError):
        E.elsaa_exact_backward(ex, q, k, v, q, torch.zeros(1, 2, 8,
                                                           device="cuda"), q,
                               workspace=E.new_exact_workspace(ex, "cuda")[
                                   :128])
    with pytest.raises(TypeError):
        E.elsaa_exact_forward(ex, None, k, v)


@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,d,causal,kl", [
    (1, 1, 1, 1, 5000, 64, 1, None), (2, 8, 2, 2, 3000, 128, 1, [2999, 700]),
    (1, 1, 1, 700, 2100, 64, 1, None), (1, 2, 1, 300, 1300, 32, 0, [1]),
    (3, 2, 2, 1100, 1100, 64, 1, [1100, 513, 0])])
def test_keys_in_chunks(B, H, Hkv, Nq, Nk, d, causal, kl):
    """Few items: the keys of a row are split and joined."""
    ql = None if kl is None else [Nq] + [max(1, Nq // 2)] * (B - 1)
    run_case(B, H, Hkv, Nq, Nk, d, BF, causal, ql=ql, kl=kl, backward=False)
    run_case(B, H, Hkv, Nq, Nk, d, F32, causal, ql=ql, kl=kl, backward=False)


def test_long_rows_in_chunks():
    """Rows of more keys than a chunk beside rows of few, chunks whose keys
    none of a tile's rows sees, peaks in one chunk."""
    q, k, v, _ = C.exact_inputs(1, 1, 1, 1600, 1600, 64, BF, 4)
    k[0, 0, 777] *= 9.0
    ref = C.exact_forward_ref(q, k, v, 0.125, 1, [1600], [1600], True)[0, 0]
    ex = E.make_exact(1, 1, 1, 1600, 1600, 64, causal=True)
    lse = torch.empty((1, 1, 1600), device="cuda")
    o = E.elsaa_exact_forward(ex, q.cuda(), k.cuda(), v.cuda(), lse=lse)
    C.close(o[0, 0], ref["o"], ref["o_tol"], "o")
    C.close(lse[0, 0], ref["lse"], ref["lse_tol"], "lse")


def test_many_short_sequences():
    """More items than a grid's first CTAs, single tokens of grouped heads."""
    run_case(200, 8, 2, 1, 40, 64, BF, 1, backward=False)
    run_case(100, 4, 2, 3, 5, 32, BF, 1)


@pytest.mark.parametrize("dtype,impl", KINDS)
@pytest.mark.parametrize("causal", [0, 1])
def test_padded_groups_of_few_rows(causal, dtype, impl):
    """Tiles that hold several heads with padding between them."""
    run_case(5, 12, 2, 5, 70, 64, dtype, causal, ql=[3, 5, 0, 1, 4],
             kl=[70, 2, 9, 69, 0], impl=impl)
    run_case(2, 9, 3, 50, 300, 64, dtype, causal, ql=[20, 50], kl=[300, 41],
             impl=impl)


@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,kl", [
    (1, 1, 1, 1, 9000, [9000]), (4, 4, 4, 3, 4000, [4000, 0, 1, 2600]),
    (7, 2, 1, 300, 1100, [1100, 0, 0, 700, 3, 0, 0]),
    (256, 1, 1, 2, 1030, [1030 - 4 * i for i in range(256)]),
    (257, 1, 1, 2, 1030, [1030 - 4 * i for i in range(257)])])
def test_shares(B, H, Hkv, Nq, Nk, kl):
    """Rows divided among CTAs: few rows of many keys, sequences without any,
    as many sequences as a share can be of."""
    run_case(B, H, Hkv, Nq, Nk, 64, BF, 1, ql=[Nq] * B, kl=kl, backward=False)
    run_case(B, H, Hkv, Nq, Nk, 64, BF, 0, ql=[(i % 2) * Nq for i in range(B)],
             kl=kl, backward=False)


def test_offsets_past_32_bits():
    """K and V of more than 2^31 elements each: the last head's rows."""
    Hkv, Nk, d = 16, 1_060_000, 128
    k = torch.zeros((1, Hkv, Nk, d), dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(0)
    at = torch.randint(0, Nk, (3000,), generator=g, device="cuda").unique()
    k[0, -1, at] = torch.randn(len(at), d, generator=g, device="cuda").to(BF)
    v[0, -1, at] = torch.randn(len(at), d, generator=g, device="cuda").to(BF)
    q = (4 * torch.randn(1, Hkv, 2, d, generator=g, device="cuda")).to(BF)
    ex = E.make_exact(1, Hkv, Hkv, 2, Nk, d)
    lse = torch.empty((1, Hkv, 2), device="cuda")
    o = E.elsaa_exact_forward(ex, q, k, v, lse=lse)
    s = (q[0, -1].double() @ k[0, -1, at].double().t()) / math.sqrt(d)
    e = torch.exp(s)
    total = e.sum(1) + Nk - len(at)  # the other scores are 0
    want = (e @ v[0, -1, at].double()) / total[:, None]
    mag = (e @ v[0, -1, at].double().abs()) / total[:, None]
    # weights and result rounded to bf16, sums over a million terms in fp32 of
    # which each CTA adds at most a few thousand in a row
    tol = 2.0 ** -8 * (mag + want.abs()) + 2.0 ** -10 * mag
    assert bool(((o[0, -1].double() - want).abs() <= tol).all())
    assert bool(((lse[0, -1].double() - torch.log(total)).abs() < 1e-3).all())
    assert not o[0, :-1].any()


def test_another_current_device_is_refused(monkeypatch):
    q, k, v, _ = (x.cuda() for x in C.exact_inputs(1, 1, 1, 8, 8, 64, BF))
    ex = E.make_exact(1, 1, 1, 8, 8, 64)
    monkeypatch.setattr(E, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        E.elsaa_exact_forward(ex, q, k, v)


def test_backward_of_one_leaf_in_a_graph_beside_an_eager_one():
    """torch's graph of the leaves lives while the calls are captured."""
    q, k, v, do = (x.cuda() for x in C.exact_inputs(1, 2, 1, 96, 96, 64, BF))
    leaf = q.clone().requires_grad_()
    eager = (leaf.float() ** 2).sum()
    ex = E.make_exact(1, 2, 1, 96, 96, 64, causal=True)
    ws = E.new_exact_workspace(ex, "cuda", backward=True)
    lse = torch.empty((1, 2, 96), device="cuda")
    x = leaf.detach()
    o = E.elsaa_exact_forward(ex, x, k, v, lse=lse, workspace=ws)
    want = E.elsaa_exact_backward(ex, x, k, v, o, lse, do, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = E.elsaa_exact_backward(ex, x, k, v, o, lse, do, workspace=ws)
    graph.replay()
    eager.backward()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(leaf.grad, (2 * q.float()).to(BF))


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,causal,ql,kl", [
    (1, 8, 1, 260, 1300, 0, None, None), (1, 8, 1, 600, 600, 1, None, None),
    (2, 4, 2, 333, 1100, 1, [333, 200], [1100, 900]),
    (3, 6, 1, 300, 1024, 0, [300, 0, 129], [1, 1024, 0])])
def test_divided_walks(B, H, Hkv, Nq, Nk, causal, ql, kl, d):
    """Few items: the sums of the backward pass are divided and added up."""
    run_case(B, H, Hkv, Nq, Nk, d, BF, causal, ql=ql, kl=kl)


@pytest.mark.parametrize("H,Hkv,Nq,Nk,d", [
    (75, 1, 129, 4100, 128), (70, 1, 129, 4100, 128), (150, 1, 129, 2100, 64),
    (20, 5, 257, 1100, 64)])
@pytest.mark.parametrize("padded", [False, True])
def test_the_workspace_is_large_enough(H, Hkv, Nq, Nk, d, padded):
    """Its size does not know of q_len, with which rows lie on more tiles: what
    lies behind it stays."""
    q, k, v, do = (x.cuda() for x in C.exact_inputs(1, H, Hkv, Nq, Nk, d, BF))
    ex = E.make_exact(1, H, Hkv, Nq, Nk, d)
    size = E.elsaa_exact_workspace_size(ex, True)
    room = torch.full((size + (1 << 26),), 77, dtype=torch.uint8,
                      device="cuda")
    ws = room[:size]
    n = lens([Nq], 1) if padded else None
    lse = torch.zeros((1, H, Nq), device="cuda")
    o = E.elsaa_exact_forward(ex, q, k, v, q_len=n, lse=lse, workspace=ws)
    g = E.elsaa_exact_backward(ex, q, k, v, o, lse, do, q_len=n, workspace=ws)
    E.elsaa_check_status(ws)
    assert (room[size:] == 77).all()
    s = (q.double().view(1, Hkv, -1, d) @ k.double().transpose(2, 3)) * d ** -.5
    p = torch.softmax(s, -1)
    dv = p.transpose(2, 3) @ do.double().view(1, Hkv, -1, d)
    # weights of 2^-8 and sums of thousands of terms, in fp32 or bf16
    scale = (p.transpose(2, 3) @ do.double().abs().view(1, Hkv, -1, d))
    assert bool(((g[2].double() - dv).abs() <= 2.0 ** -6 * scale).all())


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,causal,ql,kl", [
    (1, 4, 1, 200, 600, 1, None, None), (2, 6, 2, 150, 400, 0, [150, 40],
                                         [1, 400])])
def test_divided_walks_on_the_cuda_cores(B, H, Hkv, Nq, Nk, causal, ql, kl, d):
    run_case(B, H, Hkv, Nq, Nk, d, F32, causal, ql=ql, kl=kl)
