"""Rows to heads and back (norm, rotation, layout) against the 64-bit oracle,
and a run of the calls together."""
import math

import numpy as np
import pytest
import torch

import layer_cases as C
from paper_2607_20214_gb300 import elsaa as E

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "fp32"}


def inputs(h, dtype, seed=0):
    """One projection's output [B, N, H + 2 Hkv, d], views, weights."""
    g = torch.Generator().manual_seed(seed)
    H, Hkv, d = h.H, h.H_kv, h.d_h
    x = torch.randn(h.B, h.N, H + 2 * Hkv, d, generator=g).to(dtype).cuda()
    w = [(1 + 0.3 * torch.randn(d, generator=g)).cuda() for _ in range(2)]
    return x, (x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]), w


def run_case(B, H, Hkv, N, d, dtype=BF, norm=True, dim=None, il=False,
             sections=None, turn=False, expand=False, g32=True, new=None,
             held=None, positions=None, weights=True, seed=0):
    rot = E.make_rotary(d if dim is None else dim, interleaved=il,
                        sections=sections, in_turn=turn)
    h = E.make_heads(B, H, Hkv, N, d, dtype=NAME[dtype], norm=norm,
                     rotary=rot, expand=expand, grad_fp32=g32)
    x, (q, k, v), w = inputs(h, dtype, seed)
    n_new = new or [N] * B
    for b in range(B):
        x[b, n_new[b]:] = math.nan
    i32 = dict(dtype=torch.int32, device="cuda")
    wq, wk = w if norm and weights else (None, None)
    kw = dict(w_q=wq, w_k=wk, positions=None, lengths=None,
              new_len=torch.tensor(new, **i32) if new else None)
    pos = np.tile(np.arange(N), (rot.axes, B, 1))
    if held:
        kw["lengths"] = torch.tensor(held, **i32)
        pos = np.stack([np.arange(N) + held[b] - n_new[b]
                        for b in range(B)])[None]
    if positions is not None:
        kw["positions"] = positions.to(**i32)
        pos = positions.numpy().reshape(rot.axes, B, N)
    kv = H if expand else Hkv
    copies = H // Hkv if expand else 1
    outs = [torch.full((B, n, N, d), 7.0, dtype=dtype, device="cuda")
            for n in (H, kv, kv)]
    E.elsaa_heads_forward(h, q, k, v, q_out=outs[0], k_out=outs[1],
                          v_out=outs[2], **kw)
    for name, t, o, wt, turned, cp in (
            ("q", q, outs[0], wq, True, 1), ("k", k, outs[1], wk, True, copies),
            ("v", v, outs[2], None, False, copies)):
        ref = C.heads_ref(t, h, (turned, cp), pos, n_new, wt)
        for (b, i), (val, tol) in ref.items():
            for c in range(cp):
                got = o[b, i * cp + c]
                C.close(got[:n_new[b]], val, tol, (name, b, i, c))
                assert (got[n_new[b]:] == 7).all()
    # backward
    g = torch.Generator().manual_seed(seed + 1)
    gt = F32 if g32 or dtype == F32 else dtype
    grads = [torch.randn(B, n, N, d, generator=g).to(gt).cuda()
             for n in (H, kv, kv)]
    for t in grads:
        for b in range(B):
            t[b, :, n_new[b]:] = math.nan
    dx = torch.full_like(x, 7.0)
    views = dx[:, :, :H], dx[:, :, H:H + Hkv], dx[:, :, H + Hkv:]
    ws = E.new_heads_workspace(h, "cuda")
    dws = [torch.full((d,), 7.0, device="cuda") if norm else None
           for _ in range(2)]

    def back():
        E.elsaa_heads_backward(h, *grads, q=q, k=k, dq_rows=views[0],
                               dk_rows=views[1], dv_rows=views[2],
                               dw_q=dws[0], dw_k=dws[1], workspace=ws, **kw)
    back()
    for name, t, dt, gr, wt, turned, cp, dw in (
            ("q", q, views[0], grads[0], wq, True, 1, dws[0]),
            ("k", k, views[1], grads[1], wk, True, copies, dws[1]),
            ("v", v, views[2], grads[2], None, False, copies, None)):
        ref, rw, tw = C.heads_ref(t, h, (turned, cp), pos, n_new, wt, gr)
        for (b, i), (val, tol) in ref.items():
            C.close(dt[b, :n_new[b], i], val, tol, ("d" + name, b, i))
            assert (dt[b, n_new[b]:, i] == 7).all()
        if dw is not None:
            C.close(dw, rw, tw, "dw_" + name)
    first = [dx.clone()] + [t.clone() for t in dws if t is not None]
    back()
    again = [dx] + [t for t in dws if t is not None]
    assert all(torch.equal(a, b) for a, b in zip(first, again))


KINDS = [(BF, True), (BF, False), (F32, False)]


@pytest.mark.parametrize("dtype,g32", KINDS)
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("il", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_types_and_pairings(norm, il, d, dtype, g32):
    run_case(2, 4, 2, 37, d, dtype, norm, il=il, g32=g32)


@pytest.mark.parametrize("d,dim,il", [
    (128, 64, False), (128, 16, False), (64, 48, False), (32, 16, False),
    (128, 96, True), (64, 2, True), (32, 30, True), (64, 0, False)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_part_of_the_channels(d, dim, il, dtype):
    run_case(1, 3, 3, 20, d, dtype, True, dim=dim, il=il)


@pytest.mark.parametrize("expand", [False, True])
@pytest.mark.parametrize("B,H,Hkv,N", [(1, 1, 1, 1), (5, 8, 2, 1),
                                       (2, 7, 1, 3), (1, 12, 4, 9)])
def test_heads_and_tokens(B, H, Hkv, N, expand):
    run_case(B, H, Hkv, N, 64, expand=expand)
    run_case(B, H, Hkv, N, 128, F32, expand=expand)


@pytest.mark.parametrize("turn", [False, True])
@pytest.mark.parametrize("axes", [2, 3, 4])
def test_axes(axes, turn):
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (axes, 2, 30), generator=g)
    n = 32
    sec = [n // axes + (i < n % axes) for i in range(axes)]
    run_case(2, 2, 1, 30, 64, sections=sec, turn=turn, positions=pos,
             expand=True)


def test_far_positions_and_padded_batches():
    run_case(4, 4, 2, 9, 64, F32, new=[9, 0, 1, 5],
             held=[2 ** 31 - 1, 7, 1, 100000])
    run_case(3, 4, 1, 40, 128, new=[40, 3, 0], expand=True, g32=False)
    pos = torch.arange(40).repeat(2, 1) * 50000000
    run_case(2, 2, 2, 40, 32, positions=pos[:, :40])


def test_without_weights_and_large_rows():
    run_case(1, 2, 2, 5, 64, weights=False)
    h = E.make_heads(1, 1, 1, 3, 64, dtype="fp32")
    q = torch.zeros(1, 3, 1, 64, device="cuda")
    q[0, 1] = 1e18
    q[0, 2, 0, 5] = math.inf
    o = E.elsaa_heads_forward(h, q)[0]
    assert not o[0, 0, 0].any()
    assert torch.allclose(o[0, 0, 1], torch.ones(64, device="cuda"))
    assert o[0, 0, 2, 5].isnan()


def test_an_infinity_stays_in_its_pair():
    h = E.make_heads(1, 1, 1, 2, 64, norm=False, rotary=E.make_rotary(32))
    q = torch.ones(1, 2, 1, 64, dtype=BF, device="cuda")
    q[0, :, 0, 3] = math.inf
    q[0, :, 0, 50] = -math.inf
    o = E.elsaa_heads_forward(h, q)[0][0, 0, 1]
    where = (~o.isfinite()).nonzero().flatten().tolist()
    assert where == [3, 19, 50] and o[50] == -math.inf


def test_some_of_the_heads_and_other_strides():
    h = E.make_heads(2, 4, 2, 6, 64, rotary=E.make_rotary(64))
    x, (q, k, v), (wq, wk) = inputs(h, BF)
    want = E.elsaa_heads_forward(h, q, k, v, w_q=wq, w_k=wk)
    only = E.elsaa_heads_forward(h, k=k, w_k=wk)
    assert only[0] is None and only[2] is None
    assert torch.equal(only[1], want[1])
    # token-major rows, an expanded batch
    qt = q.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3)
    assert torch.equal(E.elsaa_heads_forward(h, qt, w_q=wq)[0], want[0])
    qe = q[:1].expand(2, -1, -1, -1)
    got = E.elsaa_heads_forward(h, qe, w_q=wq)[0]
    assert torch.equal(got[0], want[0][0]) and torch.equal(got[1], got[0])
    dq = torch.randn(2, 4, 6, 64, device="cuda").to(BF)
    a = E.elsaa_heads_backward(h, dq, q=q, w_q=wq)
    assert a[1] is None and a[2] is None and a[4] is None
    b = E.elsaa_heads_backward(h, dq, q=qt, w_q=wq,
                               dq_rows=torch.empty_like(qt))
    assert torch.equal(a[0], b[0]) and torch.equal(a[3], b[3])
    with pytest.raises(E.ElsaaError):
        E.elsaa_heads_backward(h, dq, q=qe, w_q=wq, dq_rows=qe)


def test_many_tokens():
    """More tokens than the backward kernel has warps, against the kernel on
    parts of them."""
    h = E.make_heads(2, 2, 1, 9001, 64, rotary=E.make_rotary(64),
                     grad_fp32=True)
    x, (q, k, v), (wq, wk) = inputs(h, BF)
    o = E.elsaa_heads_forward(h, q, k, v, w_q=wq, w_k=wk)
    dq = torch.randn(2, 2, 9001, 64, device="cuda")
    full = E.elsaa_heads_backward(h, dq, q=q, w_q=wq)
    total = torch.zeros(64, dtype=torch.float64, device="cuda")
    size = 0.0
    for at in range(0, 9001, 1000):
        n = min(1000, 9001 - at)
        p = E.make_heads(2, 2, 1, n, 64, rotary=E.make_rotary(64),
                         grad_fp32=True)
        pos = torch.arange(at, at + n, dtype=torch.int32,
                           device="cuda").repeat(2, 1)
        qs = q[:, at:at + n]
        assert torch.equal(E.elsaa_heads_forward(p, qs, w_q=wq,
                                                 positions=pos)[0],
                           o[0][:, :, at:at + n])
        g = E.elsaa_heads_backward(p, dq[:, :, at:at + n].contiguous(), q=qs,
                                   w_q=wq, positions=pos)
        assert torch.equal(g[0], full[0][:, at:at + n])
        total += g[3].double()
        size += g[3].abs().max().item()
    # 36004 terms of size about 1 in partial sums: 2^-24 times the root of
    # their number, times the sums' size, with a factor of 16
    assert (total - full[3].double()).abs().max() <= 16 * 2.0 ** -24 * 36004


def test_together_with_attention():
    """Rows -> heads -> attention -> back, as a layer does it, against torch in
    64 bits with derivatives by torch; and as a captured graph."""
    B, H, Hkv, N, d = 2, 4, 2, 70, 64
    rot = E.make_rotary(d)
    h = E.make_heads(B, H, Hkv, N, d, dtype="fp32", rotary=rot,
                     grad_fp32=True)
    ex = E.make_exact(B, H, Hkv, N, N, d, dtype="fp32", causal=True)
    x, (q, k, v), (wq, wk) = inputs(h, F32)
    do = torch.randn(B, H, N, d, device="cuda")
    ws = E.new_exact_workspace(ex, "cuda", backward=True)
    hw = E.new_heads_workspace(h, "cuda")

    def layer(x):
        q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
        qh, kh, vh = E.elsaa_heads_forward(h, q, k, v, w_q=wq, w_k=wk)
        lse = torch.empty(B, H, N, device="cuda")
        o = E.elsaa_exact_forward(ex, qh, kh, vh, lse=lse, workspace=ws)
        dq, dk, dv = E.elsaa_exact_backward(ex, qh, kh, vh, o, lse, do,
                                            workspace=ws)
        dx = torch.empty_like(x)
        r = E.elsaa_heads_backward(
            h, dq, dk, dv, q=q, k=k, w_q=wq, w_k=wk, dq_rows=dx[:, :, :H],
            dk_rows=dx[:, :, H:H + Hkv], dv_rows=dx[:, :, H + Hkv:],
            workspace=hw)
        return o, dx, r[3], r[4]
    got = layer(x)
    X = x.double().requires_grad_()
    W = [w.double().requires_grad_() for w in (wq, wk)]
    ang = torch.arange(N, device="cuda").double()[:, None] * torch.tensor(
        [10000.0 ** (-i / 32) for i in range(32)], dtype=torch.float64,
        device="cuda")

    def head(t, w):
        t = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + h.eps) * w
        c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        a, b = t[..., :32], t[..., 32:]
        return torch.cat([a * c - b * s, b * c + a * s], -1).transpose(1, 2)
    Q, K = head(X[:, :, :H], W[0]), head(X[:, :, H:H + Hkv], W[1])
    V = X[:, :, H + Hkv:].transpose(1, 2)
    K, V = (t.repeat_interleave(H // Hkv, 1) for t in (K, V))
    S = (Q @ K.transpose(2, 3)) / 8
    S = S.masked_fill(torch.ones(N, N, device="cuda").triu(1) > 0, -math.inf)
    O = torch.softmax(S, -1) @ V
    O.backward(do.double())
    for name, g, r in zip(("o", "dx", "dw_q", "dw_k"), got,
                          (O, X.grad, W[0].grad, W[1].grad)):
        # fp32 throughout: chains of below 2^9 roundings of numbers that add
        # up to at most 2^4 times the largest result
        tol = 2.0 ** (9 + 4 - 24) * float(r.detach().abs().max())
        assert float((g.double() - r.detach()).abs().max()) <= tol, name
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = layer(x)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_into_the_cache():
    """New tokens' rows to heads at the cache's positions, into the cache, and
    attention over it."""
    B, H, Hkv, d, ps = 2, 4, 2, 64, 16
    cache = E.new_cache(B, H, Hkv, d, ps, 8, 4)
    cache.tensors["page_table"].copy_(torch.arange(8).view(2, 4))
    lengths = cache.tensors["lengths"]
    rot = E.make_rotary(d)
    g = torch.Generator().manual_seed(0)
    rows = torch.randn(B, 30, H + 2 * Hkv, d, generator=g).to(BF).cuda()
    one = E.make_heads(B, H, Hkv, 1, d, rotary=rot)
    everything = E.make_heads(B, H, Hkv, 30, d, rotary=rot)
    parts = lambda x: (x[:, :, :H], x[:, :, H:H + Hkv],  # noqa: E731
                       x[:, :, H + Hkv:])
    qs, ks, vs = E.elsaa_heads_forward(everything, *parts(rows))
    for t in range(30):
        lengths.add_(1)
        q, k, v = E.elsaa_heads_forward(one, *parts(rows[:, t:t + 1]),
                                        lengths=lengths)
        assert torch.equal(q[:, :, 0], qs[:, :, t])
        assert torch.equal(k[:, :, 0], ks[:, :, t])
        E.elsaa_cache_append(cache, k, v)
    o = E.elsaa_cache_attention(cache, q)
    ex = E.make_exact(B, H, Hkv, 1, 30, d, causal=True)
    want = E.elsaa_exact_forward(ex, q, ks, vs)
    # keys and values in e4m3 with a page's scale: 2^-4 of each, and 2^-9 of
    # the scale's step below; scores of norm-8 rows move by 2^-4 |q||k| / 8
    bound = vs.float().abs().max() * (2.0 ** -4 + 2.0 ** -4 * 8)
    assert float((o.float() - want.float()).abs().max()) <= float(bound)


def test_streams():
    h = E.make_heads(2, 4, 2, 300, 64, rotary=E.make_rotary(64))
    x, (q, k, v), (wq, wk) = inputs(h, BF)
    want = E.elsaa_heads_forward(h, q, k, v, w_q=wq, w_k=wk)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = E.elsaa_heads_forward(h, q, k, v, w_q=wq, w_k=wk, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_argument_checks():
    h = E.make_heads(1, 2, 1, 8, 64, rotary=E.make_rotary(64))
    x, (q, k, v), (wq, wk) = inputs(h, BF)
    for bad in (dict(q=q.float()), dict(q=q[:, :4]), dict(q=q.cpu()),
                dict(q=q, w_q=wq[:32]), dict(q=q, w_q=wq.to(BF)),
                dict(q=q.transpose(1, 3).contiguous().transpose(1, 3)),
                dict(q=q, positions=torch.zeros(1, 8, device="cuda")),
                dict(q=q, q_out=torch.zeros(1, 2, 9, 64, device="cuda",
                                            dtype=BF))):
        with pytest.raises(ValueError):
            E.elsaa_heads_forward(h, **bad)
    with pytest.raises(TypeError):
        E.elsaa_heads_forward(h)
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    p = torch.zeros(1, 8, dtype=torch.int32, device="cuda")
    with pytest.raises(E.ElsaaError):
        E.elsaa_heads_forward(h, q, positions=p, lengths=n)
    with pytest.raises(E.ElsaaError):
        E.elsaa_heads_backward(h, torch.zeros(1, 2, 8, 64, device="cuda",
                                              dtype=BF))


def test_offsets_past_32_bits():
    """Rows of more than 2^31 elements: the last tokens against a call of
    their own."""
    H, N, d = 256, 66_000, 128
    h = E.make_heads(1, H, H, N, d, rotary=E.make_rotary(d))
    g = torch.Generator(device="cuda").manual_seed(0)
    q = torch.randint(-100, 100, (1, N, H, d), generator=g, device="cuda",
                      dtype=torch.int8).to(BF)
    assert q.numel() > 2 ** 31
    o = E.elsaa_heads_forward(h, q)[0]
    few = E.make_heads(1, H, H, 5, d, rotary=E.make_rotary(d))
    pos = torch.arange(N - 5, N, dtype=torch.int32, device="cuda")[None]
    want = E.elsaa_heads_forward(few, q[:, -5:], positions=pos)[0]
    assert torch.equal(o[:, :, -5:], want)
    rows = E.elsaa_heads_backward(h, o, q=q)[0]
    part = E.elsaa_heads_backward(few, want, q=q[:, -5:], positions=pos)[0]
    assert torch.equal(rows[:, -5:], part)
