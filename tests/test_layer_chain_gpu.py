"""Rows and heads with the operators of the library that they stand beside:
rows -> heads -> elsaa_forward -> elsaa_backward -> rows, and new tokens' rows
into the cache and attention over it, each stage against its oracle on what
the stage before it left."""
import numpy as np
import pytest
import torch

import layer_cases as C
from oracle import cache as oc
from paper_2607_20214_gb300 import elsaa as E
from paper_2607_20214_gb300.workloads import Workload, make_inputs
from test_backward_gpu import compare
from test_cache_gpu import check_attention
from test_parity_gpu import TOL_O, run_oracle

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_through_elsaa_and_back(dtype):
    """K and V heads copied for elsaa_forward, elsaa_backward's fp32 gradients
    added up over the copies."""
    B, H, Hkv, N, d = 2, 4, 2, 384, 64
    wl = Workload("chain", B=B, H=H, N=N, d_h=d, dtype=dtype, block=64,
                  race_tables=4, recipe="plain", temperature=2.0, seed=21,
                  plane_seed=1021, backward=True)
    x = make_inputs(wl)
    dt = BF if dtype == "bf16" else F32
    g = torch.Generator().manual_seed(5)
    rows = (torch.randn(B, N, H + 2 * Hkv, d, generator=g) * 1.5).to(dt).cuda()
    q, k, v = rows[:, :, :H], rows[:, :, H:H + Hkv], rows[:, :, H + Hkv:]
    wq, wk = (1.2 + 0.3 * torch.randn(d, generator=g)
              for _ in "qk")
    wq, wk = wq.cuda(), wk.cuda()
    heads = E.make_heads(B, H, Hkv, N, d, dtype=dtype,
                         rotary=E.make_rotary(d), expand=True,
                         grad_fp32=True)
    p = E.params_for(wl)
    planes = [x[n].cuda() for n in ("w_sort", "w_race")]
    do = x["do"].cuda()
    hw = E.new_heads_workspace(heads, "cuda")
    fw = E.new_workspace(p, "cuda")
    perm = [torch.empty((B, H, N), dtype=torch.int32, device="cuda")
            for _ in "qk"]

    def layer():
        qh, kh, vh = E.elsaa_heads_forward(heads, q, k, v, w_q=wq, w_k=wk)
        o = E.elsaa_forward(p, qh, kh, vh, *planes, perm_q=perm[0],
                            perm_k=perm[1], workspace=fw)
        dg = torch.empty((B, H, N, 2), device="cuda")
        dl = torch.empty((B, H, N), device="cuda")
        dq, dk, dv = E.elsaa_backward(p, qh, kh, vh, *planes, do, *perm,
                                      d_gates=dg, d_lambda=dl)
        drows = torch.empty_like(rows)
        _, _, _, dwq, dwk = E.elsaa_heads_backward(
            heads, dq, dk, dv, q=q, k=k, w_q=wq, w_k=wk,
            dq_rows=drows[:, :, :H], dk_rows=drows[:, :, H:H + Hkv],
            dv_rows=drows[:, :, H + Hkv:], workspace=hw)
        return qh, kh, vh, o, dq, dk, dv, drows, dwq, dwk, dg, dl
    E.elsaa_profile_start()
    got = layer()
    tc = "bwd_block_tc" in E.elsaa_profile_stop()
    qh, kh, vh, o, dq, dk, dv, drows, dwq, dwk, dg, dl = got
    pos = np.tile(np.arange(N), (1, B, 1))
    G = H // Hkv
    for x_, out, w, turned, cp in ((q, qh, wq, True, 1), (k, kh, wk, True, G),
                                   (v, vh, None, False, G)):
        for (b, i), (val, tol) in C.heads_ref(x_, heads, (turned, cp), pos,
                                              [N] * B, w).items():
            for c in range(cp):
                C.close(out[b, i * cp + c], val, tol, (b, i, c))
    # ELSAA on these heads
    x.update(q=qh.cpu(), k=kh.cpu(), v=vh.cpu())
    for (b, h), r in run_oracle(wl, x).items():
        assert np.abs(C.f64(o[b, h]) - r["O"]).max() <= TOL_O[dtype]
    compare(wl, dict(dQ=dq.cpu(), dK=dk.cpu(), dV=dv.cpu(),
                     dgates=dg.cpu(), dlam=dl.cpu(), perm_q=perm[0].cpu(),
                     perm_k=perm[1].cpu(), tc=tc), x,
            [(0, 0), (1, 3)])
    # and from its gradients
    for x_, g_, at, w, turned, cp, dw in (
            (q, dq, 0, wq, True, 1, dwq), (k, dk, H, wk, True, G, dwk),
            (v, dv, H + Hkv, None, False, G, None)):
        ref, rw, tw = C.heads_ref(x_, heads, (turned, cp), pos, [N] * B, w, g_)
        for (b, i), (val, tol) in ref.items():
            C.close(drows[b, :, at + i], val, tol, ("d", b, i))
        if dw is not None:
            C.close(dw, rw, tw, "dw")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = layer()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("d", [64, 128])
def test_rows_into_the_cache_and_attention(d):
    """What heads of new tokens leave in the cache, byte for byte, and the
    attention over these bytes: a result of zeros, of values in another order
    or of another token's would be far outside the bound."""
    B, H, Hkv, ps, N = 2, 4, 2, 16, 30
    cache = E.new_cache(B, H, Hkv, d, ps, 8, 4)
    cache.tensors["page_table"].copy_(torch.arange(8).view(2, 4))
    lengths = cache.tensors["lengths"]
    lengths.copy_(torch.tensor([0, 0]))
    c = {n: t.cpu().view(torch.uint8).numpy().copy() if n in "kv"
         else t.cpu().numpy().copy() for n, t in cache.tensors.items()
         if n != "status"}
    c["table"] = c.pop("page_table")
    rot = E.make_rotary(d)
    one = E.make_heads(B, H, Hkv, 1, d, rotary=rot)
    g = torch.Generator().manual_seed(0)
    rows = (2 * torch.randn(B, N, H + 2 * Hkv, d, generator=g)).to(BF).cuda()
    w = (1.5 + 0.3 * torch.randn(d, generator=g)).cuda()

    class Like:  # what check_attention reads
        dtype = "bf16"
    Like.d, Like.B = d, B
    for t in range(N):
        lengths.add_(1)
        x = rows[:, t:t + 1]
        parts = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
        q, k, v = E.elsaa_heads_forward(one, *parts, w_q=w, w_k=w,
                                        lengths=lengths)
        pos = np.full((1, B, 1), t)
        for r, out, wt, turned in zip(parts, (q, k, v), (w, w, None),
                                      (True, True, False)):
            for (b, i), (val, tol) in C.heads_ref(r, one, (turned, 1), pos,
                                                  [1] * B, wt).items():
                C.close(out[b, i], val, tol, (t, b, i))
        E.elsaa_cache_append(cache, k, v)
        c["lengths"] += 1
        oc.append(c, C.f64(k), C.f64(v), [1] * B)
        if t not in (0, 15, 16, 29):
            continue
        lse = torch.empty((B, H, 1), device="cuda")
        o = E.elsaa_cache_attention(cache, q, lse=lse)
        ref = oc.attention(c, C.f64(q), [1] * B, d ** -0.5)
        check_attention(Like, o, lse, ref, [1] * B)
        wrong = [torch.zeros_like(o), o.roll(1, 1), o.flip(3), o.flip(0)]
        for bad in wrong:
            with pytest.raises(AssertionError):
                check_attention(Like, bad, lse, ref, [1] * B)
    for n in "kv":
        a = oc.E4M3[cache.tensors[n].cpu().view(torch.uint8).numpy()]
        assert np.array_equal(a, oc.E4M3[c[n]], equal_nan=True)
        n += "_scale"
        assert np.array_equal(cache.tensors[n].cpu().numpy(), c[n])
