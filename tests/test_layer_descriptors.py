"""What the calls of rows and heads and of exact attention check their tensors
by, and hand on, is what the structure's fields say at the call: of a copy, of
an edited one, of one whose memory was written (no GPU needed: the library is
one that notes what it is given)."""
import copy
import ctypes
import pickle

import pytest
import torch

from paper_2607_20214_gb300 import build
from paper_2607_20214_gb300 import elsaa as E

BF, F32 = torch.bfloat16, torch.float32
# a ValueError; the second where its text would name the device, which the
# CPU's number here is none of
REFUSED = ValueError, RuntimeError


class Library:
    """Notes the fields of the structures it is given; no call does anything."""

    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        def call(x, *args):
            assert isinstance(x, ctypes.Structure)
            self.seen.append({f[0]: getattr(x, f[0]) for f in x._fields_})
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(E, "load_library", lambda: lib)
    # tensors of the CPU stand for those of the current device
    monkeypatch.setattr(E, "_current_device", lambda: -1)
    monkeypatch.setattr(E, "_raw", lambda stream, index: None)
    return lib


WS = torch.empty(512, dtype=torch.uint8)


def rows(e, dtype=BF, **over):
    f = {n: over.get(n, getattr(e, n)) for n in ("B", "H", "H_kv", "N_q",
                                                 "N_k", "d_h")}
    q = torch.zeros(f["B"], f["H"], f["N_q"], f["d_h"], dtype=dtype)
    k = torch.zeros(f["B"], f["H_kv"], f["N_k"], f["d_h"], dtype=dtype)
    return q, k, k.clone()


def forward(e, x):
    return E.elsaa_exact_forward(e, *x, o=torch.zeros_like(x[0]),
                                 lse=torch.zeros(x[0].shape[:3]),
                                 workspace=WS)


def backward(e, x):
    q, k, v = x
    return E.elsaa_exact_backward(
        e, q, k, v, q, torch.zeros(q.shape[:3]), q, dq=torch.zeros_like(q),
        dk=torch.zeros_like(k), dv=torch.zeros_like(v), workspace=WS)


EDITS = [dict(B=3), dict(H=8), dict(H_kv=4), dict(N_q=11), dict(N_k=4000),
         dict(d_h=32)]
CALLS = [forward, backward]


def exact():
    return E.make_exact(2, 4, 2, 10, 20, 64, causal=True)


def copies(x):
    y = type(x).from_buffer_copy(x)  # without the attributes of the object
    return copy.copy(x), copy.deepcopy(x), pickle.loads(pickle.dumps(x)), y


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("edit", EDITS)
def test_edited_sizes_are_those_of_the_call(library, call, edit):
    e = exact()
    old = rows(e)
    call(e, old)
    for n, x in edit.items():
        setattr(e, n, x)
    with pytest.raises(REFUSED):
        call(e, old)
    call(e, rows(e))
    assert len(library.seen) == 2
    assert all(library.seen[1][n] == x for n, x in edit.items())


@pytest.mark.parametrize("call", CALLS)
def test_an_edited_type_is_that_of_the_call(library, call):
    e = exact()
    old = rows(e)
    call(e, old)
    e.dtype = E.ELSAA_FP32
    with pytest.raises(REFUSED):
        call(e, old)
    call(e, rows(e, F32))


@pytest.mark.parametrize("call", CALLS)
def test_a_copy_is_its_own(library, call):
    e = exact()
    call(e, rows(e))  # (what is kept from it goes into the copies)
    for f in copies(e):
        f.causal, f.N_k = 0, 24
        call(f, rows(f))
        got = library.seen[-1]
        assert (got["causal"], got["N_k"]) == (0, 24)
        with pytest.raises(REFUSED):
            call(f, rows(e))
        call(e, rows(e))
        got = library.seen[-1]
        assert (got["causal"], got["N_k"]) == (1, 20)


def test_memory_written_in_another_way(library):
    e = exact()
    old = rows(e)
    forward(e, old)
    ctypes.pointer(e).contents.N_q = 12
    with pytest.raises(REFUSED):
        forward(e, old)
    forward(e, rows(e, N_q=12))
    e.N_q = 10
    forward(e, old)


def test_what_a_call_allocates_follows_the_fields(library, monkeypatch):
    monkeypatch.setattr(E, "_On", lambda index: type(
        "On", (), dict(index=index, device=torch.device("cpu"))))
    e = exact()
    x = rows(e)
    assert E.elsaa_exact_forward(e, *x, workspace=WS).shape == x[0].shape
    f = copy.copy(e)
    f.N_q, f.d_h = 7, 32
    x = rows(f)
    o = E.elsaa_exact_forward(f, *x, workspace=WS)
    assert o.shape == x[0].shape


def test_a_copy_has_its_own_workspace_size():
    build.build()
    e = E.make_exact(1, 16, 4, 65536, 65536, 64, causal=True)
    for f in copies(e):
        f.N_q, f.N_k, f.H, f.H_kv = 10, 1100, 1, 1
        fresh = E.make_exact(1, 1, 1, 10, 1100, 64, causal=True)
        for back in (False, True):
            assert (E.elsaa_exact_workspace_size(f, back) ==
                    E.elsaa_exact_workspace_size(fresh, back) !=
                    E.elsaa_exact_workspace_size(e, back))
    h = E.make_heads(1, 2, 2, 5, 64)
    for f in copies(h):
        f.d_h = 128
        assert (E.elsaa_heads_workspace_size(f) ==
                2 * E.elsaa_heads_workspace_size(h))


# ---------------------------------------------------------------- heads

def heads():
    return E.make_heads(2, 4, 2, 6, 64, rotary=E.make_rotary(64))


def parts(h, dtype=BF):
    x = torch.zeros(h.B, h.N, h.H + 2 * h.H_kv, h.d_h, dtype=dtype)
    return x[:, :, :h.H], x[:, :, h.H:h.H + h.H_kv], x[:, :, h.H + h.H_kv:]


def outs(h, dtype=BF):
    kv = h.H if h.expand else h.H_kv
    return [torch.zeros(h.B, n, h.N, h.d_h, dtype=dtype)
            for n in (h.H, kv, kv)]


def heads_forward(h, x, o, **kw):
    return E.elsaa_heads_forward(h, *x, q_out=o[0], k_out=o[1], v_out=o[2],
                                 **kw)


def heads_backward(h, x, o, **kw):
    return E.elsaa_heads_backward(h, *o, q=x[0], k=x[1], dq_rows=x[0],
                                  dk_rows=x[1], dv_rows=x[2], **kw)


@pytest.mark.parametrize("call", [heads_forward, heads_backward])
@pytest.mark.parametrize("edit", [
    dict(B=3), dict(H=8), dict(H_kv=4), dict(N=7), dict(d_h=128),
    dict(dtype=1), dict(expand=1)])
def test_edited_heads(library, call, edit):
    h = heads()
    x, o = parts(h), outs(h)
    call(h, x, o)
    for f in (h,) + copies(h):
        for n, v in edit.items():
            setattr(f, n, v)
        dt = F32 if f.dtype else BF
        with pytest.raises(REFUSED):
            call(f, x, o)
        call(f, parts(f, dt), outs(f, dt))
        assert all(library.seen[-1][n] == v for n, v in edit.items())


def test_an_edited_type_of_the_gradients(library):
    h = heads()
    x, o = parts(h), outs(h)
    heads_backward(h, x, o)
    h.grad_fp32 = 1
    with pytest.raises(REFUSED):
        heads_backward(h, x, o)
    heads_backward(h, x, outs(h, F32))


@pytest.mark.parametrize("call", [heads_forward, heads_backward])
def test_edited_axes(library, call):
    h = heads()
    x, o = parts(h), outs(h)
    pos = torch.zeros(1, h.B, h.N, dtype=torch.int32)
    call(h, x, o, positions=pos)
    call(h, x, o, positions=pos[0])
    h.rotary.axes = 2
    for bad in (pos, pos[0]):
        with pytest.raises(REFUSED):
            call(h, x, o, positions=bad)
    call(h, x, o, positions=pos.repeat(2, 1, 1))


def test_a_rotation_is_copied():
    r = E.make_rotary(64)
    h = E.make_heads(1, 1, 1, 1, 64, rotary=r)
    r.axes = 3
    assert h.rotary.axes == 1 and h.facts()[-1] == (1, 1, 1)
