"""How far a NaN reaches in exact attention with causal = 1."""
import math

import pytest
import torch

import layer_cases as C
from paper_2607_20214_gb300 import elsaa as E

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "fp32"}
KINDS = [(BF, 0), (BF, E.ELSAA_IMPL_SIMT), (F32, 0)]


def causal(N):
    return torch.ones(N, N).tril() > 0


def tiles_that_meet(sees):
    """[G N, N] of [N, N]: query rows of G heads, one behind the other, in one
    tile of 128 with a row that sees one of the same 128 keys."""
    rows, keys = sees.shape
    out = torch.zeros_like(sees)
    for r in range(0, rows, 128):
        for c in range(0, keys, 128):
            out[r:r + 128, c:c + 128] = sees[r:r + 128, c:c + 128].any()
    return out


@pytest.mark.parametrize("dtype,impl", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,at", [(200, 199), (200, 0), (300, 260),
                                  (130, 129)])
def test_a_nan_stays_within_its_tiles(N, at, d, dtype, impl):
    G = 3
    q, k, v, do = (x.cuda() for x in C.exact_inputs(1, G, 1, N, N, d, dtype))
    ex = E.make_exact(1, G, 1, N, N, d, dtype=NAME[dtype], causal=True,
                      impl=impl)

    def run(q, k, v, do):
        lse = torch.zeros((1, G, N), device="cuda")
        o = E.elsaa_exact_forward(ex, q, k, v, lse=lse)
        return o, lse
    o, lse = run(q, k, v, do)
    clean = E.elsaa_exact_backward(ex, q, k, v, o, lse, do)
    sees = causal(N).repeat(G, 1)
    meet = tiles_that_meet(sees)[:, at].view(G, N).cuda()
    seen = sees[:, at].view(G, N).cuda()

    def check(got, want, may, must, what):
        nan = got[0].isnan().any(-1)
        assert not (nan & ~may).any(), what
        assert nan[must].all(), what
        assert torch.equal(got[0][~nan], want[0][~nan]), what

    # a value: rows that see it, and rows of a tile with one that does
    v1 = v.clone()
    v1[0, 0, at] = math.nan
    check(run(q, k, v1, do)[0], o, meet, seen, "o")
    # a key in the backward pass: dq likewise, dk and dv its own row
    k1 = k.clone()
    k1[0, 0, at] = math.nan
    own = torch.zeros(1, N, dtype=torch.bool, device="cuda")
    own[0, at] = True
    dq, dk, dv = E.elsaa_exact_backward(ex, q, k1, v, o, lse, do)
    check(dq, clean[0], meet, seen, "dq")
    check(dk, clean[1], own, own, "dk")
    check(dv, clean[2], own, own, "dv")
    # a query row, or its d_o: its own dq, and keys of the 128 with one it sees
    keys = causal(N)[at]
    may = torch.zeros(1, N, dtype=torch.bool, device="cuda")
    for c in range(0, N, 128):
        may[0, c:c + 128] = bool(keys[c:c + 128].any())
    must = keys.cuda()[None]
    own = torch.zeros(G, N, dtype=torch.bool, device="cuda")
    own[1, at] = True
    for name in ("q", "do"):
        x = dict(q=q, do=do)
        x[name] = x[name].clone()
        x[name][0, 1, at] = math.nan
        dq, dk, dv = E.elsaa_exact_backward(ex, x["q"], k, v, o, lse, x["do"])
        check(dq, clean[0], own, own, name)
        check(dk, clean[1], may, must, name)
        check(dv, clean[2], may, must, name)
