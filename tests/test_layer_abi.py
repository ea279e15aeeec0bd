"""The C ABI of rows and heads and of exact attention: struct layouts, and what
is refused on the host before any launch (no GPU needed)."""
import ctypes
import os
import re

import pytest

from paper_2607_20214_gb300 import build
from paper_2607_20214_gb300 import elsaa as E

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INV, UNS, WS = (E.ELSAA_ERR_INVALID_ARG, E.ELSAA_ERR_UNSUPPORTED,
                E.ELSAA_ERR_WORKSPACE)
P = 0x10000  # a pointer that nothing follows
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    build.build()
    return E.load_library()


@pytest.mark.parametrize("header,name", [
    ("elsaa_heads.h", "elsaa_rotary"), ("elsaa_heads.h", "elsaa_heads"),
    ("elsaa_heads.h", "elsaa_rows"), ("elsaa_exact.h", "elsaa_exact")])
def test_struct_matches_header(header, name):
    src = open(os.path.join(ROOT, "include", header)).read()
    body = src[src.index("typedef struct %s {" % name):]
    body = body[body.index("{") + 1:body.index("} %s;" % name)]
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    types = {"int": ctypes.c_int, "float": ctypes.c_float,
             "int64_t": ctypes.c_int64, "void": ctypes.c_void_p,
             "uint64_t": ctypes.c_uint64 * 64, "uint8_t": ctypes.c_uint8 * 64,
             "elsaa_rotary": E.elsaa_rotary}
    fields = []
    for decl in filter(None, (x.strip() for x in body.split(";"))):
        typ, rest = decl.split(None, 1)
        for n in rest.split(","):
            n = re.sub(r"\[.*\]", "", n.strip().lstrip("*"))
            fields.append((n, types[typ]))
    assert fields == list(getattr(E, name)._fields_)


def exact(**over):
    kw = dict(B=2, H=4, H_kv=2, N_q=10, N_k=20, d_h=64, dtype=0, causal=1,
              scale=0.0, impl=0)
    kw.update(over)
    return E.elsaa_exact(**kw)


EXACT_BAD = [
    (dict(B=0), INV, "positive"), (dict(N_q=0), INV, "positive"),
    (dict(N_k=-1), INV, "positive"), (dict(H=3), INV, "multiple"),
    (dict(H_kv=0), INV, "positive"), (dict(dtype=2), INV, "dtype"),
    (dict(causal=2), INV, "causal"), (dict(impl=3), INV, "impl"),
    (dict(scale=-1.0), INV, "scale"),
    (dict(scale=float("inf")), INV, "scale"),
    (dict(scale=float("nan")), INV, "scale"),
    (dict(scale=2e38), INV, "scale"), (dict(d_h=96), UNS, "d_h"),
    (dict(N_q=1 << 29), UNS, "2^30"), (dict(N_k=1 << 30), UNS, "2^30"),
    (dict(B=1 << 30, H=1 << 15, H_kv=1 << 15), UNS, "2^30"),
    (dict(H=1 << 16, H_kv=1 << 16), UNS, "65535"),
]


def exact_calls(lib, e, **over):
    r, n = ctypes.byref(e), ctypes.c_size_t()
    a = dict.fromkeys("q k v o do dq dk dv ws".split(), P)
    a.update(lse=P, bytes=BIG)
    a.update(over)
    return {
        "size": lambda: lib.elsaa_exact_workspace_size(r, 1, ctypes.byref(n)),
        "forward": lambda: lib.elsaa_exact_forward(
            r, a["q"], a["k"], a["v"], None, None, a["o"], a["lse"], a["ws"],
            a["bytes"], None),
        "backward": lambda: lib.elsaa_exact_backward(
            r, a["q"], a["k"], a["v"], a["o"], a["lse"], a["do"], None, None,
            a["dq"], a["dk"], a["dv"], a["ws"], a["bytes"], None),
    }


@pytest.mark.parametrize("over,code,text", EXACT_BAD)
def test_bad_exact_is_refused_everywhere(lib, over, code, text):
    for name, call in exact_calls(lib, exact(**over)).items():
        assert call() == code, name
        assert text in E.elsaa_last_error(), name


@pytest.mark.parametrize("over,code,text,names", [
    (dict(q=None), INV, "non-NULL", ("forward", "backward")),
    (dict(o=None), INV, "non-NULL", ("forward", "backward")),
    (dict(lse=None), INV, "non-NULL", ("backward",)),
    (dict(do=None), INV, "non-NULL", ("backward",)),
    (dict(dv=None), INV, "non-NULL", ("backward",)),
    (dict(k=P + 8), INV, "aligned", ("forward", "backward")),
    (dict(lse=P + 4), INV, "aligned", ("forward", "backward")),
    (dict(dk=P + 2), INV, "aligned", ("backward",)),
    (dict(ws=None), WS, "NULL", ("forward", "backward")),
    (dict(ws=P + 16), WS, "aligned", ("forward", "backward")),
    (dict(bytes=128), WS, "too small", ("forward", "backward"))])
def test_bad_exact_arguments(lib, over, code, text, names):
    calls = exact_calls(lib, exact(), **over)
    for name in names:
        assert calls[name]() == code, name
        assert text in E.elsaa_last_error(), name


def test_null_structs(lib):
    n = ctypes.c_size_t()
    assert lib.elsaa_exact_workspace_size(None, 0, ctypes.byref(n)) == INV
    assert lib.elsaa_exact_workspace_size(ctypes.byref(exact()), 0,
                                          None) == INV
    assert lib.elsaa_heads_workspace_size(None, ctypes.byref(n)) == INV
    assert lib.elsaa_heads_workspace_size(heads().ref, None) == INV


def heads(**over):
    rot = over.pop("rotary", None)
    kw = dict(B=2, H=4, H_kv=2, N=10, d_h=64)
    kw.update({k: v for k, v in over.items() if k in kw})
    h = E.make_heads(rotary=rot or E.make_rotary(64), **kw)
    for k, v in over.items():
        if k not in kw:
            setattr(h, k, v)
    return h


def rotary(**over):
    r = E.make_rotary(64)
    for k, v in over.items():
        setattr(r, k, v)
    return r


def far_axis():
    r = E.make_rotary(64)
    r.axis[31] = 1
    return r


HEADS_BAD = [
    (dict(B=0), INV, "positive"), (dict(N=0), INV, "positive"),
    (dict(H=5), INV, "multiple"), (dict(dtype=7), INV, "dtype"),
    (dict(norm=2), INV, "0 or 1"), (dict(expand=-1), INV, "0 or 1"),
    (dict(grad_fp32=3), INV, "0 or 1"), (dict(eps=0.0), INV, "eps"),
    (dict(eps=float("nan")), INV, "eps"), (dict(d_h=48), UNS, "d_h"),
    (dict(H=1 << 16, H_kv=1), UNS, "65535"),
    (dict(B=1 << 16, N=1 << 16), UNS, "2^30"),
    (dict(rotary=rotary(dim=66)), INV, "dim"),
    (dict(rotary=rotary(dim=-2)), INV, "dim"),
    (dict(rotary=rotary(dim=40)), UNS, "multiple of 16"),
    (dict(rotary=rotary(dim=63, interleaved=1)), UNS, "multiple"),
    (dict(rotary=rotary(interleaved=2)), INV, "interleaved"),
    (dict(rotary=rotary(axes=0)), INV, "axes"),
    (dict(rotary=rotary(axes=5)), INV, "axes"),
    (dict(rotary=far_axis()), INV, "below"),
]


def row(data=P, batch=640, row=64, head=6400):
    return ctypes.byref(E.elsaa_rows(data, batch, row, head))


def heads_calls(lib, h, **over):
    n = ctypes.c_size_t()
    a = dict(q=row(), k=row(), v=row(), wq=P, wk=P, pos=None, lens=None, new=None,
             qo=P, ko=P, vo=P, dq=P, dk=P, dv=P, qr=row(batch=64 * 4000),
             kr=row(batch=64 * 4000), vr=row(batch=64 * 4000), dwq=P, dwk=P,
             ws=P, bytes=BIG)
    a.update(over)
    return {
        "size": lambda: lib.elsaa_heads_workspace_size(h.ref, ctypes.byref(n)),
        "forward": lambda: lib.elsaa_heads_forward(
            h.ref, a["q"], a["k"], a["v"], a["wq"], a["wk"], a["pos"],
            a["lens"], a["new"], a["qo"], a["ko"], a["vo"], None),
        "backward": lambda: lib.elsaa_heads_backward(
            h.ref, a["dq"], a["dk"], a["dv"], a["q"], a["k"], a["wq"],
            a["wk"], a["pos"], a["lens"], a["new"], a["qr"], a["kr"], a["vr"],
            a["dwq"], a["dwk"], a["ws"], a["bytes"], None),
    }


@pytest.mark.parametrize("over,code,text", HEADS_BAD)
def test_bad_heads_are_refused_everywhere(lib, over, code, text):
    for name, call in heads_calls(lib, heads(**over)).items():
        assert call() == code, name
        assert text in E.elsaa_last_error(), name


BOTH = ("forward", "backward")


@pytest.mark.parametrize("over,code,text,names", [
    (dict(pos=P, lens=P), INV, "exclude", BOTH),
    (dict(q=None), INV, "together", ("forward",)),
    (dict(vo=None), INV, "together", ("forward",)),
    (dict(dk=None), INV, "together", ("backward",)),
    (dict(q=None, k=None, v=None, qo=None, ko=None, vo=None), INV, "one of",
     ("forward",)),
    (dict(dq=None, dk=None, dv=None, qr=None, kr=None, vr=None, dwq=None,
          dwk=None), INV, "one of", ("backward",)),
    (dict(q=row(data=None)), INV, "without data", BOTH),
    (dict(q=row(data=P + 8)), INV, "aligned", BOTH),
    (dict(k=row(row=60)), INV, "multiples of 16 bytes", BOTH),
    (dict(k=row(batch=1 << 60)), INV, "2^50", BOTH),
    (dict(qo=P + 8), INV, "aligned", ("forward",)),
    (dict(dq=P + 8), INV, "aligned", ("backward",)),
    (dict(qr=row(batch=632)), INV, "overlap", ("backward",)),
    (dict(qr=row(head=0, batch=64 * 4000)), INV, "overlap", ("backward",)),
    (dict(kr=row(row=-56, batch=64 * 4000)), INV, "overlap", ("backward",)),
    (dict(q=None), INV, "needs the rows", ("backward",)),
    (dict(ws=None), WS, "NULL", ("backward",)),
    (dict(ws=P + 128), WS, "aligned", ("backward",)),
    (dict(bytes=100), WS, "too small", ("backward",))])
def test_bad_heads_arguments(lib, over, code, text, names):
    calls = heads_calls(lib, heads(), **over)
    for name in names:
        assert calls[name]() == code, name
        assert text in E.elsaa_last_error(), name


def test_weights_need_the_norm(lib):
    h = heads(norm=0)
    for name, call in heads_calls(lib, h).items():
        if name != "size":
            assert call() == INV and "norm = 1" in E.elsaa_last_error()
    call = heads_calls(lib, h, wq=None, wk=None)["backward"]
    assert call() == INV and "norm = 1" in E.elsaa_last_error()
