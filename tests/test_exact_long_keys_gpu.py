"""Exact attention over keys of which one CTA walks millions of tiles."""
import math

import pytest
import torch

from paper_2607_20214_gb300 import elsaa as E

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_one_row_over_hundreds_of_millions_of_keys():
    """More key tiles than are divided among CTAs: one walks three million of
    them for half of its row slots, the other half waits for it."""
    Nk, d = 3 << 27, 32
    k = torch.zeros((1, 1, Nk, d), dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    # whole blocks of 32 keys of weight 2^7: every sum is a multiple of 32 and
    # below 2^29, which fp32 holds
    g = torch.Generator(device="cuda").manual_seed(0)
    block = torch.randint(0, Nk // 128, (4000,), generator=g,
                          device="cuda").unique()
    block[-1] = Nk // 128 - 1
    at = (block[:, None] * 128 + 96 +
          torch.arange(32, device="cuda")).flatten()
    k[0, 0, at, 0] = 7.0
    v[0, 0, at, 1] = 1.0
    q = torch.zeros((1, 1, 1, d), dtype=BF, device="cuda")
    q[..., 0] = 1.0
    ex = E.make_exact(1, 1, 1, 1, Nk, d, scale=math.log(2.0))
    ws = E.new_exact_workspace(ex, "cuda")
    lse = torch.empty((1, 1, 1), device="cuda")
    o = E.elsaa_exact_forward(ex, q, k, v, lse=lse, workspace=ws)
    E.elsaa_check_status(ws)
    total = Nk + 127.0 * len(at)
    # the exponential and scale * log2 e are 2^-22 off, the result is rounded
    want = 128.0 * len(at) / total
    assert abs(float(o[0, 0, 0, 1]) - want) <= (2.0 ** -9 + 1e-5) * want
    assert abs(float(lse) - math.log(total)) <= 1e-5 + 2.0 ** -20
    assert not o[..., 0].any() and not o[..., 2:].any()
