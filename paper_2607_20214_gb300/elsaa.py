"""Python binding of the libelsaa C ABI (include/elsaa.h, elsaa_cache.h,
elsaa_heads.h, elsaa_exact.h).

Argument marshalling only: every step of the operator runs in the CUDA
kernels of libelsaa.so. PyTorch provides device memory and streams. The
functions keep the C names. If the library has not been built, every call
raises RuntimeError; there is no fallback implementation.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

import torch

from .build import LIB

ELSAA_OK = 0
ELSAA_ERR_INVALID_ARG = 1
ELSAA_ERR_UNSUPPORTED = 2
ELSAA_ERR_WORKSPACE = 3
ELSAA_ERR_CUDA = 4
ELSAA_ERR_DEVICE = 5
ELSAA_BF16 = 0
ELSAA_FP32 = 1
ELSAA_IMPL_AUTO = 0
ELSAA_IMPL_SIMT = 1

SYMBOLS = ("elsaa_workspace_size", "elsaa_forward", "elsaa_check_status",
           "elsaa_last_error", "elsaa_abi_version", "elsaa_profile_start",
           "elsaa_profile_stop", "elsaa_forward_noalloc",
           "elsaa_backward_workspace_size", "elsaa_backward",
           "elsaa_gates_workspace_size", "elsaa_gates",
           "elsaa_selftest_wait_timeout", "elsaa_forward_race_summaries",
           "elsaa_check_status_noalloc",
           "elsaa_selftest_wait_timeout_noalloc", "elsaa_causal_levels",
           "elsaa_causal_index_lists", "elsaa_forward_selected_keys",
           "elsaa_forward_gated_workspace_size", "elsaa_forward_gated",
           "elsaa_cache_workspace_size", "elsaa_cache_append",
           "elsaa_cache_select", "elsaa_cache_attention",
           "elsaa_cache_evict", "elsaa_heads_workspace_size",
           "elsaa_heads_forward", "elsaa_heads_backward",
           "elsaa_exact_workspace_size", "elsaa_exact_forward",
           "elsaa_exact_backward")
# Size of the fixed scratch array behind elsaa_forward_noalloc.
ELSAA_STATIC_WORKSPACE_BYTES = 64 << 20


class elsaa_params(ctypes.Structure):
    """Mirror of struct elsaa_params (field order and types must match)."""
    _fields_ = [
        ("B", ctypes.c_int), ("H", ctypes.c_int), ("N", ctypes.c_int),
        ("d_h", ctypes.c_int), ("dtype", ctypes.c_int),
        ("causal", ctypes.c_int), ("block_size", ctypes.c_int),
        ("sort_bits", ctypes.c_int), ("gray_order", ctypes.c_int),
        ("race_tables", ctypes.c_int), ("race_bits", ctypes.c_int),
        ("beta", ctypes.c_float), ("eps", ctypes.c_float),
        ("scale", ctypes.c_float), ("lam", ctypes.c_float),
        ("fusion_mode", ctypes.c_int), ("impl", ctypes.c_int),
        ("neighbor_blocks", ctypes.c_int), ("causal_chunk", ctypes.c_int),
        ("causal_base_len", ctypes.c_int), ("out_fp32", ctypes.c_int),
        ("selector", ctypes.c_int), ("topk", ctypes.c_int),
        ("topk_blocks", ctypes.c_int),
    ]


class elsaa_gate_mlp(ctypes.Structure):
    """Mirror of struct elsaa_gate_mlp (device pointers as integers)."""
    _fields_ = [
        ("hidden", ctypes.c_int), ("w1", ctypes.c_void_p),
        ("b1", ctypes.c_void_p), ("w2", ctypes.c_void_p),
        ("b2", ctypes.c_void_p), ("w_lambda", ctypes.c_void_p),
        ("b_lambda", ctypes.c_void_p), ("c_lambda", ctypes.c_void_p),
        ("lambda_min", ctypes.c_float),
    ]


class elsaa_kernel_stat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int),
                ("total_ms", ctypes.c_double)]


class elsaa_cache(ctypes.Structure):
    """Mirror of struct elsaa_cache (include/elsaa_cache.h). make_cache fills
    it from tensors and keeps them alive in `tensors`."""
    _fields_ = [
        ("B", ctypes.c_int), ("H", ctypes.c_int), ("H_kv", ctypes.c_int),
        ("d_h", ctypes.c_int), ("dtype", ctypes.c_int),
        ("page_size", ctypes.c_int), ("num_pages", ctypes.c_int),
        ("max_pages", ctypes.c_int), ("scale", ctypes.c_float),
        ("impl", ctypes.c_int), ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p), ("bounds", ctypes.c_void_p),
        ("page_table", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
        ("status", ctypes.c_void_p),
    ]


class elsaa_rotary(ctypes.Structure):
    """Mirror of struct elsaa_rotary; make_rotary fills it."""
    _fields_ = [
        ("dim", ctypes.c_int), ("interleaved", ctypes.c_int),
        ("axes", ctypes.c_int), ("reserved", ctypes.c_int),
        ("turns", ctypes.c_uint64 * 64), ("axis", ctypes.c_uint8 * 64),
    ]


class _Described(ctypes.Structure):
    """A structure whose fields say all that a call checks its tensors by.

    _of works that out; it is kept beside the bytes that it came from, and
    looked up by them, so that a copy or a structure with an edited field (or
    whose memory was written in another way) is what its fields say. ref is
    the structure's own address, a copy's that of the copy. (The calls hand on
    the structure itself: ctypes takes its address in 0.1 us less.)
    """
    _known = (None, None)

    @property
    def ref(self):
        return ctypes.byref(self)

    def facts(self):
        now = bytes(self)
        known, facts = self._known
        if known != now:
            facts = self._of()
            self._known = now, facts
        return facts


class elsaa_heads(_Described):
    """Mirror of struct elsaa_heads; make_heads fills it."""
    _fields_ = [
        ("B", ctypes.c_int), ("H", ctypes.c_int), ("H_kv", ctypes.c_int),
        ("N", ctypes.c_int), ("d_h", ctypes.c_int), ("dtype", ctypes.c_int),
        ("norm", ctypes.c_int), ("expand", ctypes.c_int),
        ("grad_fp32", ctypes.c_int), ("eps", ctypes.c_float),
        ("rotary", elsaa_rotary),
    ]

    def _of(self):
        """Types of rows and heads and of the heads' gradients; shapes of the
        rows of q and of k and v, of their heads, of weights, lengths and
        positions."""
        dt = _torch_dtype(self.dtype)
        B, H, N, d = self.B, self.H, self.N, self.d_h
        kv = H if self.expand else self.H_kv
        return (dt, torch.float32 if self.grad_fp32 else dt,
                (B, N, H, d), (B, N, self.H_kv, d), (B, H, N, d),
                (B, kv, N, d), (d,), (B,), (self.rotary.axes, B, N))


class elsaa_rows(ctypes.Structure):
    """Mirror of struct elsaa_rows (strides in elements)."""
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64),
                ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class elsaa_exact(_Described):
    """Mirror of struct elsaa_exact; make_exact fills it."""
    _fields_ = [
        ("B", ctypes.c_int), ("H", ctypes.c_int), ("H_kv", ctypes.c_int),
        ("N_q", ctypes.c_int), ("N_k", ctypes.c_int), ("d_h", ctypes.c_int),
        ("dtype", ctypes.c_int), ("causal", ctypes.c_int),
        ("scale", ctypes.c_float), ("impl", ctypes.c_int),
    ]

    def _of(self):
        """Type of the tensors; shapes of q, of k and v, of lse, of lengths."""
        B, H, Nq = self.B, self.H, self.N_q
        return (_torch_dtype(self.dtype), (B, H, Nq, self.d_h),
                (B, self.H_kv, self.N_k, self.d_h), (B, H, Nq), (B,))


class ElsaaError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("libelsaa error %d: %s" % (code, msg))
        self.code = code


_lib = None


def load_library(path: str = LIB) -> ctypes.CDLL:
    """Load libelsaa.so (built in-tree by build.build())."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(
            "libelsaa.so is not built (%s); run "
            "`python -c 'import __graft_entry__ as g; g.build()'`" % path)
    L = ctypes.CDLL(path)
    vp = ctypes.c_void_p
    L.elsaa_workspace_size.argtypes = [ctypes.POINTER(elsaa_params),
                                       ctypes.POINTER(ctypes.c_size_t)]
    L.elsaa_workspace_size.restype = ctypes.c_int
    L.elsaa_forward.argtypes = [ctypes.POINTER(elsaa_params)] + [vp] * 14 + [
        ctypes.c_size_t, vp]
    L.elsaa_forward.restype = ctypes.c_int
    L.elsaa_check_status.argtypes = [vp, vp]
    L.elsaa_check_status.restype = ctypes.c_int
    L.elsaa_last_error.argtypes = []
    L.elsaa_last_error.restype = ctypes.c_char_p
    L.elsaa_abi_version.argtypes = []
    L.elsaa_abi_version.restype = ctypes.c_int
    L.elsaa_forward_noalloc.argtypes = [ctypes.POINTER(elsaa_params)] + [
        vp] * 13 + [vp]
    L.elsaa_forward_noalloc.restype = ctypes.c_int
    L.elsaa_profile_start.argtypes = []
    L.elsaa_profile_start.restype = ctypes.c_int
    L.elsaa_profile_stop.argtypes = [ctypes.POINTER(elsaa_kernel_stat),
                                     ctypes.c_int,
                                     ctypes.POINTER(ctypes.c_int)]
    L.elsaa_profile_stop.restype = ctypes.c_int
    L.elsaa_backward_workspace_size.argtypes = [
        ctypes.POINTER(elsaa_params), ctypes.POINTER(ctypes.c_size_t)]
    L.elsaa_backward_workspace_size.restype = ctypes.c_int
    L.elsaa_backward.argtypes = [ctypes.POINTER(elsaa_params)] + [vp] * 18 + [
        ctypes.c_size_t, vp]
    L.elsaa_forward_race_summaries.argtypes = [
        ctypes.POINTER(elsaa_params), vp, ctypes.c_size_t, vp, vp, vp]
    L.elsaa_forward_race_summaries.restype = ctypes.c_int
    L.elsaa_backward.restype = ctypes.c_int
    L.elsaa_gates_workspace_size.argtypes = [
        ctypes.POINTER(elsaa_params), ctypes.POINTER(elsaa_gate_mlp),
        ctypes.POINTER(ctypes.c_size_t)]
    L.elsaa_gates_workspace_size.restype = ctypes.c_int
    L.elsaa_gates.argtypes = [ctypes.POINTER(elsaa_params),
                              ctypes.POINTER(elsaa_gate_mlp)] + [vp] * 4 + [
        ctypes.c_size_t, vp]
    L.elsaa_gates.restype = ctypes.c_int
    L.elsaa_selftest_wait_timeout.argtypes = [vp, ctypes.c_size_t,
                                              ctypes.c_int, vp]
    L.elsaa_selftest_wait_timeout.restype = ctypes.c_int
    L.elsaa_causal_levels.argtypes = [ctypes.POINTER(elsaa_params),
                                      ctypes.POINTER(ctypes.c_int)]
    L.elsaa_causal_levels.restype = ctypes.c_int
    L.elsaa_causal_index_lists.argtypes = [ctypes.POINTER(elsaa_params), vp,
                                           ctypes.c_size_t, vp, vp]
    L.elsaa_causal_index_lists.restype = ctypes.c_int
    L.elsaa_forward_gated_workspace_size.argtypes = [
        ctypes.POINTER(elsaa_params), ctypes.POINTER(elsaa_gate_mlp),
        ctypes.POINTER(ctypes.c_size_t)]
    L.elsaa_forward_gated_workspace_size.restype = ctypes.c_int
    L.elsaa_forward_gated.argtypes = [
        ctypes.POINTER(elsaa_params), ctypes.POINTER(elsaa_gate_mlp)] + [
        vp] * 14 + [ctypes.c_size_t, vp]
    L.elsaa_forward_gated.restype = ctypes.c_int
    L.elsaa_forward_selected_keys.argtypes = [
        ctypes.POINTER(elsaa_params), vp, ctypes.c_size_t, vp, vp]
    L.elsaa_forward_selected_keys.restype = ctypes.c_int
    L.elsaa_check_status_noalloc.argtypes = [vp]
    L.elsaa_check_status_noalloc.restype = ctypes.c_int
    L.elsaa_selftest_wait_timeout_noalloc.argtypes = [ctypes.c_int, vp]
    L.elsaa_selftest_wait_timeout_noalloc.restype = ctypes.c_int
    pc, ci, sz = ctypes.POINTER(elsaa_cache), ctypes.c_int, ctypes.c_size_t
    L.elsaa_cache_workspace_size.argtypes = [pc, ci, ci, ci,
                                             ctypes.POINTER(sz)]
    L.elsaa_cache_append.argtypes = [pc, ci, vp, vp, vp, vp]
    L.elsaa_cache_select.argtypes = [pc, ci, vp, vp, ci, ci, ci, vp, vp, sz,
                                     vp]
    L.elsaa_cache_attention.argtypes = [pc, ci, vp, vp, vp, ci, vp, vp, vp,
                                        vp, vp, sz, vp]
    L.elsaa_cache_evict.argtypes = [pc, vp, ci, ci, vp, ci, vp, vp, vp, vp,
                                    sz, vp]
    for name in ("workspace_size", "append", "select", "attention", "evict"):
        getattr(L, "elsaa_cache_" + name).restype = ci
    ph, pr = ctypes.POINTER(elsaa_heads), ctypes.POINTER(elsaa_rows)
    pe = ctypes.POINTER(elsaa_exact)
    L.elsaa_heads_workspace_size.argtypes = [ph, ctypes.POINTER(sz)]
    L.elsaa_heads_forward.argtypes = [ph] + [pr] * 3 + [vp] * 9
    L.elsaa_heads_backward.argtypes = [ph] + [vp] * 3 + [pr] * 2 + [
        vp] * 5 + [pr] * 3 + [vp] * 3 + [sz, vp]
    L.elsaa_exact_workspace_size.argtypes = [pe, ci, ctypes.POINTER(sz)]
    L.elsaa_exact_forward.argtypes = [pe] + [vp] * 8 + [sz, vp]
    L.elsaa_exact_backward.argtypes = [pe] + [vp] * 12 + [sz, vp]
    for name in ("heads_workspace_size", "heads_forward", "heads_backward",
                 "exact_workspace_size", "exact_forward", "exact_backward"):
        getattr(L, "elsaa_" + name).restype = ci
    _lib = L
    return L


def elsaa_last_error() -> str:
    return load_library().elsaa_last_error().decode()


def elsaa_abi_version() -> int:
    return load_library().elsaa_abi_version()


def _check(rc: int):
    if rc != ELSAA_OK:
        raise ElsaaError(rc, elsaa_last_error())


def make_params(B, H, N, d_h, dtype="bf16", block_size=64, sort_bits=5,
                gray_order=1, race_tables=4, race_bits=4, beta=1.0, eps=1e-6,
                scale=0.0, lam=1.0, fusion_mode=0, causal=0,
                impl=ELSAA_IMPL_AUTO, neighbor_blocks=0, causal_chunk=128,
                causal_base_len=4096, out_fp32=0, selector=0, topk=0,
                topk_blocks=1) -> elsaa_params:
    dt = {"bf16": ELSAA_BF16, "fp32": ELSAA_FP32}[dtype] if isinstance(
        dtype, str) else int(dtype)
    return elsaa_params(B, H, N, d_h, dt, causal, block_size, sort_bits,
                        gray_order, race_tables, race_bits, beta, eps, scale,
                        lam, fusion_mode, impl, neighbor_blocks, causal_chunk,
                        causal_base_len, out_fp32, selector, topk,
                        topk_blocks)


def params_for(wl, **over) -> elsaa_params:
    """Parameters of a Workload (paper_2607_20214_gb300.workloads)."""
    kw = dict(B=wl.B, H=wl.H, N=wl.N, d_h=wl.d_h, dtype=wl.dtype,
              block_size=wl.block, sort_bits=wl.sort_bits,
              gray_order=wl.gray_order, race_tables=wl.race_tables,
              race_bits=wl.race_bits, beta=wl.beta, eps=wl.eps,
              lam=wl.lam, fusion_mode=wl.fusion_mode, causal=wl.causal,
              neighbor_blocks=wl.neighbor_blocks,
              causal_chunk=wl.causal_chunk,
              causal_base_len=wl.causal_base_len,
              selector=wl.selector, topk=wl.topk,
              topk_blocks=wl.topk_blocks)
    kw.update(over)
    return make_params(**kw)


def elsaa_workspace_size(params: elsaa_params) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().elsaa_workspace_size(ctypes.byref(params),
                                               ctypes.byref(n)))
    return n.value


def _ptr(t, name, dtype=None, numel=None, device=None):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if device is not None and t.device != device:
        raise ValueError("%s must be on %s (got %s)" % (name, device,
                                                        t.device))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must be %s (got %s)" % (name, dtype, t.dtype))
    if numel is not None and t.numel() != numel:
        raise ValueError("%s must have %d elements (got %d)" % (
            name, numel, t.numel()))
    return t.data_ptr()


# torch.cuda.current_stream builds a Stream object (2 us, as much as a kernel
# launch); the raw handle is all that is needed
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice",
                          torch.cuda.current_device)


def _stream_of(stream, dev):
    """cudaStream_t of `stream`, by default torch's current one on dev."""
    if stream is None:
        if _raw_stream is not None and dev.index is not None:
            return _raw_stream(dev.index)
        stream = torch.cuda.current_stream(dev)
    return getattr(stream, "cuda_stream", stream)


def new_workspace(params: elsaa_params, device) -> torch.Tensor:
    """Caller-owned scratch of elsaa_workspace_size bytes (256-aligned)."""
    n = elsaa_workspace_size(params)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def elsaa_forward(params: elsaa_params, q, k, v, w_sort, w_race,
                  lambda_tok=None, gates=None, o=None, log_d_sparse=None,
                  d_lr=None, m_sparse=None, perm_q=None, perm_k=None,
                  workspace=None, stream=None):
    """Enqueue elsaa_forward on `stream` (default: torch's current stream).

    Tensors are device tensors laid out as in include/elsaa.h. Returns o
    (allocated here when not given). Raises ElsaaError on a non-zero return.
    """
    lib = load_library()
    dev = q.device
    if dev.type != "cuda":
        raise ValueError("q must be a CUDA tensor")
    tdt = torch.float32 if params.dtype == ELSAA_FP32 else torch.bfloat16
    odt = torch.float32 if params.out_fp32 else tdt
    BHN = params.B * params.H * params.N
    nqkv = BHN * params.d_h
    if o is None:
        o = torch.empty(q.shape, dtype=odt, device=dev)
    if workspace is None:
        workspace = new_workspace(params, dev)
    sp = _stream_of(stream, dev)
    args = [
        _ptr(q, "q", tdt, nqkv, dev), _ptr(k, "k", tdt, nqkv, dev),
        _ptr(v, "v", tdt, nqkv, dev),
        _ptr(w_sort, "w_sort", torch.float32,
             params.H * params.sort_bits * params.d_h, dev)
        if params.sort_bits > 0 else None,
        _ptr(w_race, "w_race", torch.float32,
             params.H * params.race_tables * params.race_bits * params.d_h,
             dev),
        _ptr(lambda_tok, "lambda_tok", torch.float32, BHN, dev),
        _ptr(gates, "gates", torch.float32, 2 * BHN, dev),
        _ptr(o, "o", odt, nqkv, dev),
        _ptr(log_d_sparse, "log_d_sparse", torch.float32, BHN, dev),
        _ptr(d_lr, "d_lr", torch.float32, BHN, dev),
        _ptr(m_sparse, "m_sparse", torch.float32, BHN, dev),
        _ptr(perm_q, "perm_q", torch.int32, BHN, dev),
        _ptr(perm_k, "perm_k", torch.int32, BHN, dev),
        _ptr(workspace, "workspace", None, None, dev),
    ]
    rc = lib.elsaa_forward(ctypes.byref(params), *args,
                           workspace.numel() * workspace.element_size(), sp)
    _check(rc)
    return o


def elsaa_backward_workspace_size(params: elsaa_params) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().elsaa_backward_workspace_size(ctypes.byref(params),
                                                        ctypes.byref(n)))
    return n.value


def elsaa_forward_race_summaries(params: elsaa_params, workspace,
                                 race_A=None, race_B=None, stream=None):
    """Copy the RACE summaries A [B, H, r], B [B, H, r, d_h] (fp32) of the
    last elsaa_forward on `workspace` into race_A, race_B (allocated here
    when not given); returns (race_A, race_B)."""
    lib = load_library()
    dev = workspace.device
    r = params.race_tables << params.race_bits
    BH = params.B * params.H
    if race_A is None:
        race_A = torch.empty((params.B, params.H, r), dtype=torch.float32,
                             device=dev)
    if race_B is None:
        race_B = torch.empty((params.B, params.H, r, params.d_h),
                             dtype=torch.float32, device=dev)
    sp = _stream_of(stream, dev)
    rc = lib.elsaa_forward_race_summaries(
        ctypes.byref(params), _ptr(workspace, "workspace", None, None, dev),
        workspace.numel() * workspace.element_size(),
        _ptr(race_A, "race_A", torch.float32, BH * r, dev),
        _ptr(race_B, "race_B", torch.float32, BH * r * params.d_h, dev), sp)
    _check(rc)
    return race_A, race_B


def elsaa_backward(params: elsaa_params, q, k, v, w_sort, w_race, d_o,
                   perm_q, perm_k, lambda_tok=None, gates=None, dq=None,
                   dk=None, dv=None, d_gates=None, d_lambda=None,
                   race_A=None, race_B=None, workspace=None, stream=None):
    """Enqueue elsaa_backward on `stream`; returns (dq, dk, dv) (fp32,
    allocated here when not given). perm_q, perm_k come from elsaa_forward
    on the same inputs; race_A, race_B (optional) from
    elsaa_forward_race_summaries."""
    lib = load_library()
    dev = q.device
    if dev.type != "cuda":
        raise ValueError("q must be a CUDA tensor")
    tdt = torch.float32 if params.dtype == ELSAA_FP32 else torch.bfloat16
    BHN = params.B * params.H * params.N
    nqkv = BHN * params.d_h
    r = params.race_tables << params.race_bits
    shape = tuple(q.shape)
    dq = torch.empty(shape, dtype=torch.float32, device=dev) if dq is None else dq
    dk = torch.empty(shape, dtype=torch.float32, device=dev) if dk is None else dk
    dv = torch.empty(shape, dtype=torch.float32, device=dev) if dv is None else dv
    if workspace is None:
        n = elsaa_backward_workspace_size(params)
        workspace = torch.empty(max(n, 256), dtype=torch.uint8, device=dev)
    sp = _stream_of(stream, dev)
    args = [
        _ptr(q, "q", tdt, nqkv, dev), _ptr(k, "k", tdt, nqkv, dev),
        _ptr(v, "v", tdt, nqkv, dev),
        _ptr(w_sort, "w_sort", torch.float32, None, dev)
        if w_sort is not None else None,
        _ptr(w_race, "w_race", torch.float32,
             params.H * params.race_tables * params.race_bits * params.d_h,
             dev),
        _ptr(lambda_tok, "lambda_tok", torch.float32, BHN, dev),
        _ptr(gates, "gates", torch.float32, 2 * BHN, dev),
        _ptr(d_o, "d_o", tdt, nqkv, dev),
        _ptr(perm_q, "perm_q", torch.int32, BHN, dev),
        _ptr(perm_k, "perm_k", torch.int32, BHN, dev),
        _ptr(dq, "dq", torch.float32, nqkv, dev),
        _ptr(dk, "dk", torch.float32, nqkv, dev),
        _ptr(dv, "dv", torch.float32, nqkv, dev),
        _ptr(d_gates, "d_gates", torch.float32, 2 * BHN, dev),
        _ptr(d_lambda, "d_lambda", torch.float32, BHN, dev),
        _ptr(race_A, "race_A", torch.float32, params.B * params.H * r, dev),
        _ptr(race_B, "race_B", torch.float32,
             params.B * params.H * r * params.d_h, dev),
        _ptr(workspace, "workspace", None, None, dev),
    ]
    rc = lib.elsaa_backward(ctypes.byref(params), *args,
                            workspace.numel() * workspace.element_size(), sp)
    _check(rc)
    return dq, dk, dv


def _gate_struct(params: elsaa_params, mlp: dict, dev) -> elsaa_gate_mlp:
    H, d, g = params.H, params.d_h, int(mlp["hidden"])
    has_l = mlp.get("w_lambda") is not None
    f32 = torch.float32
    return elsaa_gate_mlp(
        g, _ptr(mlp["w1"], "w1", f32, H * g * d, dev),
        _ptr(mlp["b1"], "b1", f32, H * g, dev),
        _ptr(mlp["w2"], "w2", f32, H * 2 * g, dev),
        _ptr(mlp["b2"], "b2", f32, H * 2, dev),
        _ptr(mlp["w_lambda"], "w_lambda", f32, H * d, dev) if has_l else None,
        _ptr(mlp["b_lambda"], "b_lambda", f32, H, dev) if has_l else None,
        _ptr(mlp["c_lambda"], "c_lambda", f32, H, dev) if has_l else None,
        float(mlp.get("lambda_min", 1e-6)))


def elsaa_gates_workspace_size(params: elsaa_params, mlp: dict,
                               device=None) -> int:
    dev = mlp["w1"].device if device is None else device
    m = _gate_struct(params, mlp, dev)
    n = ctypes.c_size_t(0)
    _check(load_library().elsaa_gates_workspace_size(
        ctypes.byref(params), ctypes.byref(m), ctypes.byref(n)))
    return n.value


def elsaa_gates(params: elsaa_params, mlp: dict, q, gates=None,
                lambda_tok=None, workspace=None, stream=None):
    """Enqueue elsaa_gates on `stream`: per-token (g_sparse, g_lr) and,
    when mlp["w_lambda"] is given, lambda_i. `mlp` holds device tensors
    w1, b1, w2, b2 (and w_lambda, b_lambda, c_lambda, lambda_min) as in
    include/elsaa.h. Returns (gates [B, H, N, 2], lambda_tok [B, H, N] or
    None), allocated here when not given."""
    lib = load_library()
    dev = q.device
    if dev.type != "cuda":
        raise ValueError("q must be a CUDA tensor")
    tdt = torch.float32 if params.dtype == ELSAA_FP32 else torch.bfloat16
    BHN = params.B * params.H * params.N
    shape = (params.B, params.H, params.N)
    m = _gate_struct(params, mlp, dev)
    if gates is None:
        gates = torch.empty(shape + (2,), dtype=torch.float32, device=dev)
    if lambda_tok is None and mlp.get("w_lambda") is not None:
        lambda_tok = torch.empty(shape, dtype=torch.float32, device=dev)
    if workspace is None:
        n = elsaa_gates_workspace_size(params, mlp, dev)
        workspace = torch.empty(max(n, 256), dtype=torch.uint8, device=dev)
    sp = _stream_of(stream, dev)
    rc = lib.elsaa_gates(
        ctypes.byref(params), ctypes.byref(m),
        _ptr(q, "q", tdt, BHN * params.d_h, dev),
        _ptr(gates, "gates", torch.float32, 2 * BHN, dev),
        _ptr(lambda_tok, "lambda_tok", torch.float32, BHN, dev),
        _ptr(workspace, "workspace", None, None, dev),
        workspace.numel() * workspace.element_size(), sp)
    _check(rc)
    return gates, lambda_tok


def elsaa_selftest_wait_timeout(workspace: torch.Tensor, limit_ms=100,
                                stream=None):
    """Enqueue the bounded-wait self-test: one wait that nothing satisfies
    runs out after limit_ms and records a timeout in the status word."""
    lib = load_library()
    if stream is None:
        stream = torch.cuda.current_stream(workspace.device)
    sp = stream.cuda_stream if hasattr(stream, "cuda_stream") else stream
    _check(lib.elsaa_selftest_wait_timeout(
        workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        int(limit_ms), sp))


def elsaa_check_status(workspace: torch.Tensor, stream=None):
    """Synchronise and raise ElsaaError if a kernel recorded a fault."""
    lib = load_library()
    if stream is None:
        stream = torch.cuda.current_stream(workspace.device)
    sp = stream.cuda_stream if hasattr(stream, "cuda_stream") else stream
    _check(lib.elsaa_check_status(workspace.data_ptr(), sp))


def elsaa_profile_start():
    _check(load_library().elsaa_profile_start())


def elsaa_profile_stop() -> dict:
    """{kernel name: (launches, summed device ms)} since profile_start."""
    arr = (elsaa_kernel_stat * 64)()
    n = ctypes.c_int(0)
    _check(load_library().elsaa_profile_stop(arr, 64, ctypes.byref(n)))
    return {arr[i].name.decode(): (arr[i].launches, arr[i].total_ms)
            for i in range(n.value)}


def elsaa_forward_noalloc(params: elsaa_params, q, k, v, w_sort, w_race,
                          lambda_tok=None, gates=None, o=None,
                          log_d_sparse=None, d_lr=None, m_sparse=None,
                          perm_q=None, perm_k=None, stream=None):
    """elsaa_forward without a workspace, for callers that cannot allocate
    device memory (a host application that owns every buffer, or a path
    that must not risk the device-wide synchronisation of cudaMalloc).

    Scratch comes from the library's fixed ELSAA_STATIC_WORKSPACE_BYTES
    array, shared by all calls: order overlapping calls on one stream. The
    first call on a device may load the library's module there and should
    precede any stream capture. `o` must be given (nothing is allocated here
    either). elsaa_check_status_noalloc reads the call's status word.
    """
    lib = load_library()
    if o is None:
        raise ValueError("o must be given: elsaa_forward_noalloc allocates "
                         "nothing")
    dev = q.device
    tdt = torch.float32 if params.dtype == ELSAA_FP32 else torch.bfloat16
    odt = torch.float32 if params.out_fp32 else tdt
    BHN = params.B * params.H * params.N
    nqkv = BHN * params.d_h
    sp = _stream_of(stream, dev)
    args = [
        _ptr(q, "q", tdt, nqkv, dev), _ptr(k, "k", tdt, nqkv, dev),
        _ptr(v, "v", tdt, nqkv, dev),
        _ptr(w_sort, "w_sort", torch.float32,
             params.H * params.sort_bits * params.d_h, dev)
        if params.sort_bits > 0 else None,
        _ptr(w_race, "w_race", torch.float32,
             params.H * params.race_tables * params.race_bits * params.d_h,
             dev),
        _ptr(lambda_tok, "lambda_tok", torch.float32, BHN, dev),
        _ptr(gates, "gates", torch.float32, 2 * BHN, dev),
        _ptr(o, "o", odt, nqkv, dev),
        _ptr(log_d_sparse, "log_d_sparse", torch.float32, BHN, dev),
        _ptr(d_lr, "d_lr", torch.float32, BHN, dev),
        _ptr(m_sparse, "m_sparse", torch.float32, BHN, dev),
        _ptr(perm_q, "perm_q", torch.int32, BHN, dev),
        _ptr(perm_k, "perm_k", torch.int32, BHN, dev),
    ]
    _check(lib.elsaa_forward_noalloc(ctypes.byref(params), *args, sp))
    return o


def _stream_ptr(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def elsaa_check_status_noalloc(stream=None):
    """elsaa_check_status for elsaa_forward_noalloc: synchronise and raise
    ElsaaError if a kernel recorded a fault in the static array's status
    word."""
    _check(load_library().elsaa_check_status_noalloc(_stream_ptr(stream)))


def elsaa_selftest_wait_timeout_noalloc(limit_ms=100, stream=None):
    """The bounded-wait self-test on the static array's status word."""
    _check(load_library().elsaa_selftest_wait_timeout_noalloc(
        int(limit_ms), _stream_ptr(stream)))


def elsaa_causal_levels(params: elsaa_params) -> int:
    """Halving levels Lv of the causal sparse branch for params."""
    n = ctypes.c_int(0)
    _check(load_library().elsaa_causal_levels(ctypes.byref(params),
                                              ctypes.byref(n)))
    return n.value


def elsaa_causal_index_lists(params: elsaa_params, workspace, lists=None,
                             stream=None):
    """Sorted orders of every SortLSH call of the last causal forward on
    `workspace`: int32 [Lv, 2, B, H, N / 2] (allocated here when not
    given; None when Lv = 0). See include/elsaa.h for the layout."""
    lv = elsaa_causal_levels(params)
    if lv == 0:
        return None
    dev = workspace.device
    shape = (lv, 2, params.B, params.H, params.N // 2)
    if lists is None:
        lists = torch.empty(shape, dtype=torch.int32, device=dev)
    n = lv * params.B * params.H * params.N
    _check(load_library().elsaa_causal_index_lists(
        ctypes.byref(params), _ptr(workspace, "workspace", None, None, dev),
        workspace.numel() * workspace.element_size(),
        _ptr(lists, "lists", torch.int32, n, dev), _stream_ptr(stream)))
    return lists


def elsaa_forward_selected_keys(params: elsaa_params, workspace, keys=None,
                                stream=None):
    """The key sets of the last top-k forward (selector = 1) on `workspace`:
    int32 [B, H, N, topk], each row's original key indices increasing
    (allocated here when not given)."""
    dev = workspace.device
    shape = (params.B, params.H, params.N, params.topk)
    if keys is None:
        keys = torch.empty(shape, dtype=torch.int32, device=dev)
    n = params.B * params.H * params.N * params.topk
    _check(load_library().elsaa_forward_selected_keys(
        ctypes.byref(params), _ptr(workspace, "workspace", None, None, dev),
        workspace.numel() * workspace.element_size(),
        _ptr(keys, "keys", torch.int32, n, dev), _stream_ptr(stream)))
    return keys


def elsaa_forward_gated_workspace_size(params: elsaa_params, mlp: dict,
                                       device=None) -> int:
    dev = mlp["w1"].device if device is None else device
    m = _gate_struct(params, mlp, dev)
    n = ctypes.c_size_t(0)
    _check(load_library().elsaa_forward_gated_workspace_size(
        ctypes.byref(params), ctypes.byref(m), ctypes.byref(n)))
    return n.value


def elsaa_forward_gated(params: elsaa_params, mlp: dict, q, k, v, w_sort,
                        w_race, o=None, log_d_sparse=None, d_lr=None,
                        m_sparse=None, perm_q=None, perm_k=None,
                        gates_out=None, lambda_out=None, workspace=None,
                        stream=None):
    """Enqueue elsaa_forward_gated: the forward with the gates and lambda
    of the gate MLP `mlp` (as for elsaa_gates) computed in the same call.
    Returns o (allocated here when not given)."""
    lib = load_library()
    dev = q.device
    tdt = torch.float32 if params.dtype == ELSAA_FP32 else torch.bfloat16
    odt = torch.float32 if params.out_fp32 else tdt
    BHN = params.B * params.H * params.N
    nqkv = BHN * params.d_h
    m = _gate_struct(params, mlp, dev)
    if o is None:
        o = torch.empty(q.shape, dtype=odt, device=dev)
    if workspace is None:
        n = elsaa_forward_gated_workspace_size(params, mlp, dev)
        workspace = torch.empty(max(n, 256), dtype=torch.uint8, device=dev)
    args = [
        _ptr(q, "q", tdt, nqkv, dev), _ptr(k, "k", tdt, nqkv, dev),
        _ptr(v, "v", tdt, nqkv, dev),
        _ptr(w_sort, "w_sort", torch.float32,
             params.H * params.sort_bits * params.d_h, dev)
        if params.sort_bits > 0 else None,
        _ptr(w_race, "w_race", torch.float32,
             params.H * params.race_tables * params.race_bits * params.d_h,
             dev),
        _ptr(o, "o", odt, nqkv, dev),
        _ptr(log_d_sparse, "log_d_sparse", torch.float32, BHN, dev),
        _ptr(d_lr, "d_lr", torch.float32, BHN, dev),
        _ptr(m_sparse, "m_sparse", torch.float32, BHN, dev),
        _ptr(perm_q, "perm_q", torch.int32, BHN, dev),
        _ptr(perm_k, "perm_k", torch.int32, BHN, dev),
        _ptr(gates_out, "gates_out", torch.float32, 2 * BHN, dev),
        _ptr(lambda_out, "lambda_out", torch.float32, BHN, dev),
        _ptr(workspace, "workspace", None, None, dev),
    ]
    _check(lib.elsaa_forward_gated(
        ctypes.byref(params), ctypes.byref(m), *args,
        workspace.numel() * workspace.element_size(), _stream_ptr(stream)))
    return o


# ------------------------------------------------ the cache (elsaa_cache.h)

_CODES = (torch.float8_e4m3fn, torch.uint8)


def make_cache(k, v, k_scale, v_scale, bounds, page_table, lengths, H=None,
               dtype="bf16", scale=0.0, impl=ELSAA_IMPL_AUTO,
               status=None) -> elsaa_cache:
    """The cache over these device tensors (layouts: include/elsaa_cache.h).

    k, v [num_pages, H_kv, page_size, d_h] float8_e4m3fn (or its bytes);
    k_scale, v_scale [num_pages, H_kv] fp32; bounds [num_pages, H_kv, 2, d_h]
    int8; page_table [B, max_pages] and lengths [B] int32; H query heads
    (default H_kv); status [4] int32 zeros (default: made here).
    """
    dev = k.device
    if dev.type != "cuda":
        raise ValueError("k must be a CUDA tensor")
    if k.dim() != 4 or page_table.dim() != 2:
        raise ValueError("k must have 4 dimensions and page_table 2")
    num, hkv, ps, d = k.shape
    B, width = page_table.shape
    if k.dtype not in _CODES or v.dtype not in _CODES:
        raise ValueError("k and v must be float8_e4m3fn or uint8")
    if status is None:
        status = torch.zeros(4, dtype=torch.int32, device=dev)
    dt = {"bf16": ELSAA_BF16, "fp32": ELSAA_FP32}[dtype] if isinstance(
        dtype, str) else int(dtype)
    f32, i32 = torch.float32, torch.int32
    c = elsaa_cache(
        B, hkv if H is None else H, hkv, d, dt, ps, num, width, scale, impl,
        _ptr(k, "k", None, k.numel(), dev), _ptr(v, "v", None, k.numel(), dev),
        _ptr(k_scale, "k_scale", f32, num * hkv, dev),
        _ptr(v_scale, "v_scale", f32, num * hkv, dev),
        _ptr(bounds, "bounds", torch.int8, num * hkv * 2 * d, dev),
        _ptr(page_table, "page_table", i32, B * width, dev),
        _ptr(lengths, "lengths", i32, B, dev),
        _ptr(status, "status", i32, 4, dev))
    c.tensors = dict(k=k, v=v, k_scale=k_scale, v_scale=v_scale,
                     bounds=bounds, page_table=page_table, lengths=lengths,
                     status=status)
    c.device = dev
    c.torch_dtype = f32 if dt == ELSAA_FP32 else torch.bfloat16
    c.ref = ctypes.byref(c)
    c.index = k.get_device()
    c.slots = B * hkv * width * ps
    return c


def new_cache(B, H, H_kv, d_h, page_size, num_pages, max_pages,
              dtype="bf16", scale=0.0, impl=ELSAA_IMPL_AUTO,
              device="cuda") -> elsaa_cache:
    """An empty cache: pools of num_pages pages, a page table of -1 and
    lengths of 0 (in `tensors`, for the caller to fill)."""
    def zeros(shape, dt):
        return torch.zeros(shape, dtype=dt, device=device)
    pool = (num_pages, H_kv, page_size, d_h)
    return make_cache(
        zeros(pool, torch.uint8).view(torch.float8_e4m3fn),
        zeros(pool, torch.uint8).view(torch.float8_e4m3fn),
        torch.ones((num_pages, H_kv), device=device),
        torch.ones((num_pages, H_kv), device=device),
        zeros((num_pages, H_kv, 2, d_h), torch.int8),
        torch.full((B, max_pages), -1, dtype=torch.int32, device=device),
        zeros((B,), torch.int32), H, dtype, scale, impl)


def elsaa_cache_workspace_size(cache: elsaa_cache, T=1, weights=False,
                               keep=0) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().elsaa_cache_workspace_size(
        ctypes.byref(cache), int(T), int(bool(weights)), int(keep),
        ctypes.byref(n)))
    return n.value


def new_cache_workspace(cache: elsaa_cache, T=1, weights=False,
                        keep=0) -> torch.Tensor:
    """Scratch for the cache calls of up to T tokens a sequence (weights:
    elsaa_cache_attention with weight_out; keep: elsaa_cache_evict)."""
    n = elsaa_cache_workspace_size(cache, T, weights, keep)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=cache.device)


def _cptr(t, name, dtype, numel, cache):
    """_ptr for the cache's device; the checks that pass cost least (a step
    of decoding makes a dozen of them)."""
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.dtype is dtype and \
            t.get_device() == cache.index and t.numel() == numel and \
            t.is_contiguous():
        return t.data_ptr()
    return _ptr(t, name, dtype, numel, cache.device)


def _rows(t, name, cache, heads):
    """(pointer, T) of [B, heads, T, d_h] rows."""
    s = t.shape
    if len(s) != 4 or (s[0], s[1], s[3]) != (cache.B, heads, cache.d_h):
        raise ValueError("%s must be [%d, %d, T, %d] (got %s)" % (
            name, cache.B, heads, cache.d_h, tuple(s)))
    return _cptr(t, name, cache.torch_dtype, t.numel(), cache), s[2]


def _own(stream, cache):
    """Memory that a call makes for itself belongs to the call's stream, or it
    could be given out again while the call still runs there."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(_stream_of(stream, None),
                                           cache.device)
    return torch.cuda.stream(stream)


def _stream_for(stream, cache):
    """_stream_of, for a cache on the current device: on another one the
    kernels would follow pointers that are not its own."""
    if _current_device() != cache.index:
        raise ValueError("the cache is on %s, which is not the current "
                         "device" % cache.device)
    return _stream_of(stream, cache.device)


def _scratch(workspace, cache):
    """(pointer, bytes) of a workspace."""
    if workspace.get_device() != cache.index or \
            not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous, on %s" % cache.device)
    return workspace.data_ptr(), workspace.nbytes


def elsaa_cache_append(cache: elsaa_cache, k, v, new_len=None, stream=None):
    """Enqueue elsaa_cache_append: rows k, v [B, H_kv, T, d_h] become the
    newest tokens (lengths count them already)."""
    kp, T = _rows(k, "k", cache, cache.H_kv)
    _check(load_library().elsaa_cache_append(
        cache.ref, T, kp, _cptr(v, "v", cache.torch_dtype, k.numel(), cache),
        _cptr(new_len, "new_len", torch.int32, cache.B, cache),
        _stream_for(stream, cache)))


def elsaa_cache_select(cache: elsaa_cache, q, n_sel, first=1, last=1,
                       new_len=None, pages=None, workspace=None,
                       stream=None):
    """Enqueue elsaa_cache_select for queries q [B, H, T, d_h]; returns pages
    [B, H_kv, n_sel] int32 (allocated here when not given)."""
    qp, T = _rows(q, "q", cache, cache.H)
    if pages is None or workspace is None:
        with _own(stream, cache):
            if pages is None:
                pages = torch.empty((cache.B, cache.H_kv, n_sel),
                                    dtype=torch.int32, device=cache.device)
            if workspace is None:
                workspace = new_cache_workspace(cache, T)
    ws, nbytes = _scratch(workspace, cache)
    _check(load_library().elsaa_cache_select(
        cache.ref, T, qp, _cptr(new_len, "new_len", torch.int32, cache.B,
                                cache), n_sel, first, last,
        _cptr(pages, "pages", torch.int32, cache.B * cache.H_kv * n_sel,
              cache), ws, nbytes, _stream_for(stream, cache)))
    return pages


def elsaa_cache_attention(cache: elsaa_cache, q, pages=None, new_len=None,
                          weight_in=None, weight_out=None, o=None, lse=None,
                          workspace=None, stream=None):
    """Enqueue elsaa_cache_attention for queries q [B, H, T, d_h]; returns o
    (allocated here when not given, rows behind new_len then undefined).
    pages: as elsaa_cache_select returns them, or None for all."""
    qp, T = _rows(q, "q", cache, cache.H)
    if o is None or workspace is None:
        with _own(stream, cache):
            if o is None:
                o = torch.empty_like(q)
            if workspace is None:
                workspace = new_cache_workspace(cache, T,
                                                weight_out is not None)
    f32, i32, B = torch.float32, torch.int32, cache.B
    n_sel = 0 if pages is None else pages.shape[-1]
    ws, nbytes = _scratch(workspace, cache)
    _check(load_library().elsaa_cache_attention(
        cache.ref, T, qp, _cptr(new_len, "new_len", i32, B, cache),
        _cptr(pages, "pages", i32, B * cache.H_kv * n_sel, cache), n_sel,
        _cptr(weight_in, "weight_in", f32, cache.slots, cache),
        _cptr(weight_out, "weight_out", f32, cache.slots, cache),
        _cptr(o, "o", cache.torch_dtype, q.numel(), cache),
        _cptr(lse, "lse", f32, B * cache.H * T, cache), ws, nbytes,
        _stream_for(stream, cache)))
    return o


def elsaa_cache_evict(cache: elsaa_cache, weight, keep, recent, dst_table,
                      weight_out=None, lengths_out=None, kept=None,
                      workspace=None, stream=None):
    """Enqueue elsaa_cache_evict; returns (weight_out, lengths_out), allocated
    here when not given. The kept tokens are in the pages of dst_table
    [B, dst_pages] afterwards."""
    i32, f32, B = torch.int32, torch.float32, cache.B
    width, ps, bh = dst_table.shape[-1], cache.page_size, B * cache.H_kv
    if weight_out is None or lengths_out is None or workspace is None:
        with _own(stream, cache):
            if weight_out is None:
                weight_out = torch.zeros((B, cache.H_kv, width * ps),
                                         device=cache.device)
            if lengths_out is None:
                lengths_out = torch.empty((B,), dtype=i32,
                                          device=cache.device)
            if workspace is None:
                workspace = new_cache_workspace(cache, 1, False, keep)
    ws, nbytes = _scratch(workspace, cache)
    _check(load_library().elsaa_cache_evict(
        cache.ref, _cptr(weight, "weight", f32, cache.slots, cache), keep,
        recent, _cptr(dst_table, "dst_table", i32, B * width, cache), width,
        _cptr(weight_out, "weight_out", f32, bh * width * ps, cache),
        _cptr(lengths_out, "lengths_out", i32, B, cache),
        _cptr(kept, "kept", i32, bh * keep, cache), ws, nbytes,
        _stream_for(stream, cache)))
    return weight_out, lengths_out


# --------------------------- rows and heads (elsaa_heads.h), exact attention
# (elsaa_exact.h)

_DTYPES = {"bf16": ELSAA_BF16, "fp32": ELSAA_FP32}


def _dtype_code(dtype):
    return _DTYPES[dtype] if isinstance(dtype, str) else int(dtype)


def _torch_dtype(code):
    return torch.float32 if code == ELSAA_FP32 else torch.bfloat16


def _turns(radians):
    """A frequency (a double, radians per position) as turns * 2^64."""
    import decimal
    with decimal.localcontext() as ctx:
        ctx.prec = 60
        two_pi = decimal.Decimal("6.28318530717958647692528676655900576839433"
                                 "879875021")
        x = decimal.Decimal(float(radians)) / two_pi * (1 << 64)
        return int(x.to_integral_value()) % (1 << 64)


def make_rotary(dim, base=10000.0, interleaved=False, sections=None,
                in_turn=False, frequencies=None) -> elsaa_rotary:
    """The rotation of a head's first `dim` channels.

    frequencies: radians per position of the dim / 2 pairs (default:
    base^(-2 i / dim)). sections: pairs of every position axis (default: one
    axis); in_turn=False gives the first pairs to the first axis, the next to
    the second; True deals them out in turn while an axis has any left.
    """
    n = dim // 2
    if dim < 0 or dim > 128 or dim % 2:
        raise ValueError("dim must be even, 0 to 128")
    if frequencies is None:
        frequencies = [float(base) ** (-i / n) for i in range(n)]
    if len(frequencies) != n:
        raise ValueError("frequencies must have dim / 2 = %d entries" % n)
    left = [n] if sections is None else [int(x) for x in sections]
    if not 1 <= len(left) <= 4 or min(left) < 0 or sum(left) != n:
        raise ValueError("sections must be 1 to 4 counts that add up to "
                         "dim / 2 = %d" % n)
    axes, axis = len(left), []
    if in_turn:
        while sum(left):
            for i in range(axes):
                if left[i]:
                    left[i] -= 1
                    axis.append(i)
    else:
        axis = [i for i, x in enumerate(left) for _ in range(x)]
    r = elsaa_rotary(dim, int(bool(interleaved)), axes, 0)
    for i in range(n):
        r.turns[i] = _turns(frequencies[i])
        r.axis[i] = axis[i]
    return r


def make_heads(B, H, H_kv, N, d_h, dtype="bf16", norm=True, rotary=None,
               expand=False, grad_fp32=False, eps=1e-6) -> elsaa_heads:
    """What elsaa_heads_forward and elsaa_heads_backward are about (fields:
    include/elsaa_heads.h; a call goes by what they are then). rotary: as
    make_rotary returns it (copied), or None."""
    return elsaa_heads(B, H, H_kv, N, d_h, _dtype_code(dtype),
                       int(bool(norm)), int(bool(expand)),
                       int(bool(grad_fp32)), eps,
                       make_rotary(0) if rotary is None else rotary)


def elsaa_heads_workspace_size(heads: elsaa_heads) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().elsaa_heads_workspace_size(heads,
                                                     ctypes.byref(n)))
    return n.value


def new_heads_workspace(heads: elsaa_heads, device) -> torch.Tensor:
    """Scratch for elsaa_heads_backward."""
    return torch.empty(max(elsaa_heads_workspace_size(heads), 256),
                       dtype=torch.uint8, device=device)


def _index(t, name):
    """The device of a call's tensors, which must be the current one."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    index = t.get_device()
    if index != _current_device():
        if index < 0:
            raise ValueError("%s must be a CUDA tensor" % name)
        raise ValueError("%s is on %s, which is not the current device"
                         % (name, t.device))
    return index


class _On:
    """A device, as _own wants it."""

    def __init__(self, index):
        self.index, self.device = index, torch.device("cuda", index)


def _whole(t, name, dtype, shape, index):
    """Pointer of a contiguous tensor of this type and shape; None stays. (The
    checks that pass cost least: a small call makes a dozen of them.)"""
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.dtype is dtype and \
            t.shape == shape and t.get_device() == index and \
            t.is_contiguous():
        return t.data_ptr()
    n = 1
    for x in shape:
        n *= x
    _ptr(t, name, dtype, n, torch.device("cuda", index))
    raise ValueError("%s must be %s (got %s)" % (name, list(shape),
                                                 list(t.shape)))


def _strided(t, name, dtype, shape, index):
    """elsaa_rows of [B, N, heads, d_h], whose channels lie side by side."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype is dtype and t.shape == shape and t.get_device() == index:
        sb, sn, sh, sd = t.stride()
        if sd == 1:
            return elsaa_rows(t.data_ptr(), sb, sn, sh)
        raise ValueError("%s must have its channels side by side" % name)
    if t.get_device() != index:
        raise ValueError("%s must be on cuda:%d (got %s)" % (name, index,
                                                            t.device))
    raise ValueError("%s must be %s %s (got %s %s)" % (
        name, dtype, list(shape), t.dtype, list(t.shape)))


def _raw(stream, index):
    """cudaStream_t of `stream`, by default torch's current one."""
    if stream is None and _raw_stream is not None:
        return _raw_stream(index)
    return _stream_of(stream, torch.device("cuda", index))


def _space(workspace, index):
    """(pointer, bytes) of a workspace."""
    if workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous, on cuda:%d" % index)
    return workspace.data_ptr(), workspace.nbytes


def _positions(positions, shape, index):
    if positions is None:
        return None
    if shape[0] == 1 and positions.dim() == 2:
        shape = shape[1:]
    return _whole(positions, "positions", torch.int32, shape, index)


def elsaa_heads_forward(heads: elsaa_heads, q=None, k=None, v=None, w_q=None,
                        w_k=None, positions=None, lengths=None, new_len=None,
                        q_out=None, k_out=None, v_out=None, stream=None):
    """Enqueue elsaa_heads_forward: rows q [B, N, H, d_h] and k, v
    [B, N, H_kv, d_h] (strided views of a projection's output; None: not
    wanted) to normed and rotated heads. Returns (q_out, k_out, v_out),
    allocated here when not given (rows behind new_len then undefined)."""
    on = _index(q if q is not None else k if k is not None else v, "q")
    f32, i32 = torch.float32, torch.int32
    dt, _, rq, rk, oq, ok, w, B, at = heads.facts()
    rows_q = _strided(q, "q", dt, rq, on)
    rows_k = _strided(k, "k", dt, rk, on)
    rows_v = _strided(v, "v", dt, rk, on)
    if (q is not None and q_out is None) or (
            k is not None and k_out is None) or (
            v is not None and v_out is None):
        with _own(stream, _On(on)):
            def new(x, out, shape):
                if x is None or out is not None:
                    return out
                return torch.empty(shape, dtype=dt, device=x.device)
            q_out, k_out, v_out = (new(q, q_out, oq), new(k, k_out, ok),
                                   new(v, v_out, ok))
    _check(load_library().elsaa_heads_forward(
        heads, rows_q, rows_k, rows_v, _whole(w_q, "w_q", f32, w, on),
        _whole(w_k, "w_k", f32, w, on), _positions(positions, at, on),
        _whole(lengths, "lengths", i32, B, on),
        _whole(new_len, "new_len", i32, B, on),
        _whole(q_out, "q_out", dt, oq, on), _whole(k_out, "k_out", dt, ok, on),
        _whole(v_out, "v_out", dt, ok, on), _raw(stream, on)))
    return q_out, k_out, v_out


def elsaa_heads_backward(heads: elsaa_heads, dq=None, dk=None, dv=None,
                         q=None, k=None, w_q=None, w_k=None, positions=None,
                         lengths=None, new_len=None, dq_rows=None,
                         dk_rows=None, dv_rows=None, dw_q=None, dw_k=None,
                         workspace=None, stream=None):
    """Enqueue elsaa_heads_backward: gradients of the heads to those of the
    rows and of the norm's weights. Returns (dq_rows, dk_rows, dv_rows, dw_q,
    dw_k): the rows of the gradients given, allocated here when not given
    (rows behind new_len then undefined); dw_q and dw_k likewise where the
    weights are given."""
    on = _index(dq if dq is not None else dk if dk is not None else dv, "dq")
    f32, i32 = torch.float32, torch.int32
    dt, gt, rq, rk, oq, ok, w, B, at = heads.facts()
    if w_q is not None and dw_q is None and dq is not None or \
            w_k is not None and dw_k is None and dk is not None or \
            dq is not None and dq_rows is None or \
            dk is not None and dk_rows is None or \
            dv is not None and dv_rows is None or \
            workspace is None and not (dw_q is None and dw_k is None):
        own = _On(on)
        with _own(stream, own):
            def new(x, out, shape, t):
                if x is None or out is not None:
                    return out
                return torch.empty(shape, dtype=t, device=own.device)
            dq_rows, dk_rows, dv_rows = (
                new(dq, dq_rows, rq, dt), new(dk, dk_rows, rk, dt),
                new(dv, dv_rows, rk, dt))
            if dq is not None:
                dw_q = new(w_q, dw_q, w, f32)
            if dk is not None:
                dw_k = new(w_k, dw_k, w, f32)
            if workspace is None:
                workspace = new_heads_workspace(heads, own.device)
    ws, nbytes = (None, 0) if workspace is None else _space(workspace, on)
    _check(load_library().elsaa_heads_backward(
        heads, _whole(dq, "dq", gt, oq, on), _whole(dk, "dk", gt, ok, on),
        _whole(dv, "dv", gt, ok, on), _strided(q, "q", dt, rq, on),
        _strided(k, "k", dt, rk, on), _whole(w_q, "w_q", f32, w, on),
        _whole(w_k, "w_k", f32, w, on), _positions(positions, at, on),
        _whole(lengths, "lengths", i32, B, on),
        _whole(new_len, "new_len", i32, B, on),
        _strided(dq_rows, "dq_rows", dt, rq, on),
        _strided(dk_rows, "dk_rows", dt, rk, on),
        _strided(dv_rows, "dv_rows", dt, rk, on),
        _whole(dw_q, "dw_q", f32, w, on), _whole(dw_k, "dw_k", f32, w, on),
        ws, nbytes, _raw(stream, on)))
    return dq_rows, dk_rows, dv_rows, dw_q, dw_k


def make_exact(B, H, H_kv, N_q, N_k, d_h, dtype="bf16", causal=False,
               scale=0.0, impl=ELSAA_IMPL_AUTO) -> elsaa_exact:
    """What elsaa_exact_forward and elsaa_exact_backward are about (fields:
    include/elsaa_exact.h; a call goes by what they are then)."""
    return elsaa_exact(B, H, H_kv, N_q, N_k, d_h, _dtype_code(dtype),
                       int(bool(causal)), scale, impl)


def elsaa_exact_workspace_size(exact: elsaa_exact, backward=False) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().elsaa_exact_workspace_size(
        exact, int(bool(backward)), ctypes.byref(n)))
    return n.value


def new_exact_workspace(exact: elsaa_exact, device,
                        backward=False) -> torch.Tensor:
    """Scratch for elsaa_exact_forward (backward: for both calls).
    elsaa_check_status(workspace) reads the status of the last call on it."""
    return torch.empty(max(elsaa_exact_workspace_size(exact, backward), 256),
                       dtype=torch.uint8, device=device)


def elsaa_exact_forward(exact: elsaa_exact, q, k, v, q_len=None, k_len=None,
                        o=None, lse=None, workspace=None, stream=None):
    """Enqueue elsaa_exact_forward: q [B, H, N_q, d_h] over k, v
    [B, H_kv, N_k, d_h]. Returns o (allocated here when not given, rows behind
    q_len then undefined); lse [B, H, N_q] fp32 is written when given."""
    on = _index(q, "q")
    i32 = torch.int32
    dt, rows, kv, row, B = exact.facts()
    if o is None or workspace is None:
        own = _On(on)
        with _own(stream, own):
            if o is None:
                o = torch.empty(rows, dtype=dt, device=own.device)
            if workspace is None:
                workspace = new_exact_workspace(exact, own.device)
    ws, nbytes = _space(workspace, on)
    _check(load_library().elsaa_exact_forward(
        exact, _whole(q, "q", dt, rows, on),
        _whole(k, "k", dt, kv, on), _whole(v, "v", dt, kv, on),
        _whole(q_len, "q_len", i32, B, on), _whole(k_len, "k_len", i32, B, on),
        _whole(o, "o", dt, rows, on),
        _whole(lse, "lse", torch.float32, row, on), ws, nbytes,
        _raw(stream, on)))
    return o


def elsaa_exact_backward(exact: elsaa_exact, q, k, v, o, lse, d_o, q_len=None,
                         k_len=None, dq=None, dk=None, dv=None,
                         workspace=None, stream=None):
    """Enqueue elsaa_exact_backward: the gradients of q, k and v from d_o, with
    o and lse of elsaa_exact_forward. Returns (dq, dk, dv), allocated here when
    not given (rows behind q_len and k_len then undefined)."""
    on = _index(q, "q")
    i32 = torch.int32
    dt, rows, kv, row, B = exact.facts()
    if dq is None or dk is None or dv is None or workspace is None:
        own = _On(on)
        with _own(stream, own):
            def new(out, shape):
                return out if out is not None else torch.empty(
                    shape, dtype=dt, device=own.device)
            dq, dk, dv = new(dq, rows), new(dk, kv), new(dv, kv)
            if workspace is None:
                workspace = new_exact_workspace(exact, own.device, True)
    ws, nbytes = _space(workspace, on)
    _check(load_library().elsaa_exact_backward(
        exact, _whole(q, "q", dt, rows, on),
        _whole(k, "k", dt, kv, on), _whole(v, "v", dt, kv, on),
        _whole(o, "o", dt, rows, on),
        _whole(lse, "lse", torch.float32, row, on),
        _whole(d_o, "d_o", dt, rows, on),
        _whole(q_len, "q_len", i32, B, on), _whole(k_len, "k_len", i32, B, on),
        _whole(dq, "dq", dt, rows, on), _whole(dk, "dk", dt, kv, on),
        _whole(dv, "dv", dt, kv, on), ws, nbytes,
        _raw(stream, on)))
    return dq, dk, dv
