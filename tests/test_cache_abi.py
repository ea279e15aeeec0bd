"""The cache operators' C ABI: struct layout, and what is refused on the host
before any launch (no GPU needed)."""
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


@pytest.fixture(scope="module")
def lib():
    build.build()
    return E.load_library()


def cache(**over):
    kw = dict(B=2, H=8, H_kv=2, d_h=64, dtype=E.ELSAA_BF16, page_size=32,
              num_pages=10, max_pages=4, scale=0.0, impl=0, k=P, v=P,
              k_scale=P, v_scale=P, bounds=P, page_table=P, lengths=P,
              status=P)
    kw.update(over)
    return E.elsaa_cache(**kw)


def test_struct_matches_header():
    src = open(os.path.join(ROOT, "include", "elsaa_cache.h")).read()
    body = src[src.index("typedef struct elsaa_cache"):]
    body = body[body.index("{") + 1:body.index("} elsaa_cache;")]
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = []
    for decl in filter(None, (x.strip() for x in body.split(";"))):
        names = decl.split(",")
        first = names[0].split()
        typ = " ".join(first[:-1])
        for name in [first[-1]] + [x.strip() for x in names[1:]]:
            ptr = name.startswith("*")
            fields.append((ctypes.c_void_p if ptr else
                           {"int": ctypes.c_int,
                            "float": ctypes.c_float}[typ], name.lstrip("*")))
    assert [(n, t) for t, n in fields] == list(E.elsaa_cache._fields_)


BAD = [
    (dict(B=0), INV, "positive"), (dict(H=7), INV, "multiple"),
    (dict(H_kv=0), INV, "positive"), (dict(num_pages=0), INV, "positive"),
    (dict(max_pages=-1), INV, "positive"), (dict(dtype=2), INV, "dtype"),
    (dict(impl=2), INV, "impl"), (dict(scale=-1.0), INV, "scale"),
    (dict(scale=float("nan")), INV, "scale"),
    (dict(d_h=96), UNS, "d_h"), (dict(page_size=48), UNS, "page_size"),
    (dict(page_size=256), UNS, "page_size"), (dict(B=5000), UNS, "B must"),
    (dict(max_pages=1 << 27), UNS, "max_pages"),
    (dict(num_pages=1 << 27), UNS, "num_pages"),
    (dict(k=None), INV, "non-NULL"), (dict(bounds=None), INV, "non-NULL"),
    (dict(lengths=None), INV, "non-NULL"), (dict(v=P + 8), INV, "aligned"),
    (dict(bounds=P + 4), INV, "aligned"), (dict(status=P + 4), INV, "aligned"),
]


def calls(lib, c, **over):
    """The return codes of every entry point with valid other arguments."""
    n = ctypes.c_size_t()
    r = ctypes.byref(c)
    big = 1 << 40
    a = dict(T=1, keep=64, recent=1, n_sel=3, first=1, last=1, ws=P, bytes=big,
             q=P, o=P, pages=P, weight=P, weight_out=P + 256, dst=P,
             dst_pages=2, lengths_out=P, win=None, wout=None, k=P, v=P)
    a.update(over)
    return {
        "size": lambda: lib.elsaa_cache_workspace_size(r, a["T"], 0, a["keep"],
                                                       ctypes.byref(n)),
        "append": lambda: lib.elsaa_cache_append(r, a["T"], a["k"], a["v"],
                                                 None, None),
        "select": lambda: lib.elsaa_cache_select(
            r, a["T"], a["q"], None, a["n_sel"], a["first"], a["last"],
            a["pages"], a["ws"], a["bytes"], None),
        "attention": lambda: lib.elsaa_cache_attention(
            r, a["T"], a["q"], None, a["pages"], a["n_sel"], a["win"],
            a["wout"], a["o"], None, a["ws"], a["bytes"], None),
        "evict": lambda: lib.elsaa_cache_evict(
            r, a["weight"], a["keep"], a["recent"], a["dst"], a["dst_pages"],
            a["weight_out"], a["lengths_out"], None, a["ws"], a["bytes"],
            None),
    }


@pytest.mark.parametrize("over,code,text", BAD)
def test_bad_caches_are_refused_everywhere(lib, over, code, text):
    for name, call in calls(lib, cache(**over)).items():
        assert call() == code, name
        assert text in E.elsaa_last_error(), name


@pytest.mark.parametrize("name,over,code,text", [
    ("size", dict(T=0), INV, "T"), ("size", dict(T=65), UNS, "T"),
    ("size", dict(T=33), UNS, "128"), ("size", dict(keep=-1), INV, "keep"),
    ("append", dict(T=0), INV, "T"), ("append", dict(k=None), INV, "non-NULL"),
    ("append", dict(v=P + 2), INV, "aligned"),
    ("select", dict(q=None), INV, "non-NULL"),
    ("select", dict(q=P + 8), INV, "aligned"),
    ("select", dict(pages=None), INV, "non-NULL"),
    ("select", dict(n_sel=0), INV, "n_sel"),
    ("select", dict(first=-1), INV, "first"),
    ("select", dict(first=2, last=2), INV, "first"),
    ("select", dict(last=2 ** 31 - 1), INV, "first"),
    ("select", dict(ws=None), WS, "NULL"),
    ("select", dict(ws=P + 16), WS, "aligned"),
    ("select", dict(bytes=8), WS, "small"),
    ("select", dict(T=65), UNS, "T"),
    ("attention", dict(T=-3), INV, "T"), ("attention", dict(T=40), UNS, "128"),
    ("attention", dict(o=None), INV, "non-NULL"),
    ("attention", dict(q=P + 4), INV, "aligned"),
    ("attention", dict(win=P), INV, "weight_out"),
    ("attention", dict(wout=P + 4), INV, "aligned"),
    ("attention", dict(win=P + 8, wout=P), INV, "aligned"),
    ("attention", dict(n_sel=0), INV, "n_sel"),
    ("attention", dict(n_sel=1 << 28), INV, "n_sel"),
    ("attention", dict(bytes=0), WS, "small"),
    ("attention", dict(ws=None), WS, "NULL"),
    ("evict", dict(weight=None), INV, "non-NULL"),
    ("evict", dict(lengths_out=None), INV, "non-NULL"),
    ("evict", dict(weight_out=P), INV, "weight"),
    ("evict", dict(keep=0), INV, "keep"),
    ("evict", dict(recent=65), INV, "recent"),
    ("evict", dict(recent=-1), INV, "recent"),
    ("evict", dict(dst_pages=1), INV, "dst_pages"),
    ("evict", dict(ws=None), WS, "NULL"),
    ("evict", dict(bytes=64), WS, "small"),
])
def test_bad_arguments_are_refused(lib, name, over, code, text):
    assert calls(lib, cache(), **over)[name]() == code
    assert text in E.elsaa_last_error()


def test_workspace_size_grows_with_what_it_serves(lib):
    base = E.elsaa_cache_workspace_size(cache())
    assert base > 0 and base % 256 == 0
    assert E.elsaa_cache_workspace_size(cache(), T=4) > base
    w = E.elsaa_cache_workspace_size(cache(), weights=True)
    assert w >= base + 4 * 2 * 8 * 4 * 32
    assert E.elsaa_cache_workspace_size(cache(), keep=1 << 24) >= \
        4 * 2 * 2 * (1 << 24)
    assert lib.elsaa_cache_workspace_size(ctypes.byref(cache()), 1, 0, 0,
                                          None) == INV


def test_binding_checks_shapes():
    import torch
    with pytest.raises(ValueError, match="CUDA"):
        E.make_cache(*[torch.zeros((2, 1, 16, 32), dtype=torch.uint8)] * 2,
                     None, None, None, torch.zeros((1, 1)), None)


@pytest.mark.parametrize("impl", [0, 1])
@pytest.mark.parametrize("B,H,H_kv,max_pages", [
    (1, 1, 1, 1), (1, 4, 1, 7), (2, 8, 2, 40), (8, 8, 8, 3), (40, 16, 8, 64),
    (3, 24, 3, 2000), (9, 20, 4, 1), (33, 12, 12, 2)])
def test_a_workspace_serves_fewer_tokens_too(lib, impl, B, H, H_kv,
                                             max_pages):
    """Whatever groups the columns of a smaller call come in."""
    for d in (64, 128):
        for weights in (False, True):
            sizes = [E.elsaa_cache_workspace_size(
                cache(B=B, H=H, H_kv=H_kv, max_pages=max_pages, d_h=d,
                      impl=impl), T, weights)
                for T in range(1, min(64, 128 * H_kv // H) + 1)]
            assert sizes == sorted(sizes)
