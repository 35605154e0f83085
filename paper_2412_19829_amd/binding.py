"""Thin ctypes binding of libgformer_attn.so (see include/gformer.h).

Argument marshalling only (a decode step's and the packed and paged calls' in an extension module,
_decode_call.so, where that loads): every step of the attention forward runs in the HIP kernels behind the C ABI.  torch is used by callers for device memory and
streams; this module only reads `data_ptr()` / shapes / strides from tensors.
There is no CPU fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgformer_attn.so")
CALL_PATH = os.path.join(HERE, "_decode_call.so")

GF_OK, GF_ERR_INVALID_ARG, GF_ERR_UNSUPPORTED, GF_ERR_WORKSPACE, GF_ERR_DEVICE = range(5)
GF_F32, GF_BF16 = 0, 1
GF_PHI_ELU1, GF_PHI_IDENTITY = 0, 1
GF_FLOPS_PAPER, GF_FLOPS_PER_HEAD = 0, 1
GF_IMPL_AUTO, GF_IMPL_SCALAR, GF_IMPL_MFMA, GF_IMPL_MFMA_BLOCKED, GF_IMPL_MFMA_STREAM = 0, 1, 2, 3, 4
GF_IMPL_MFMA_CHUNK = 5
GF_LAUNCH_WINDOWED, GF_LAUNCH_LINEAR_STATE, GF_LAUNCH_LINEAR_MAIN = 1, 2, 4

EXPORTS = ("gformer_params_init", "gformer_attn_workspace_bytes", "gformer_attn_plan",
           "gformer_attn_fwd", "gformer_attn_fwd_noalloc", "gformer_attn_prefill", "gformer_attn_decode",
           "gformer_attn_bwd_workspace_bytes", "gformer_attn_bwd",
           "gformer_feature_params_init",
           "gformer_random_features",
           "gformer_packed_params_init", "gformer_packed_attn_fwd", "gformer_packed_attn_bwd_workspace_bytes",
           "gformer_packed_attn_bwd", "gformer_paged_params_init", "gformer_paged_decode_workspace_bytes",
           "gformer_paged_decode", "gformer_paged_fill", "gformer_pages_copy",
           "gformer_partition_balance", "gformer_partition_heads",
           "gformer_status_string", "gformer_version")


class GformerParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("phi", ctypes.c_int32), ("n_sparse_heads", ctypes.c_int32),
                ("chunk", ctypes.c_int32), ("segment_len", ctypes.c_int32),
                ("impl", ctypes.c_int32), ("launch_mask", ctypes.c_int32),
                ("overlap", ctypes.c_int32), ("bidirectional", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("eps", ctypes.c_float),
                ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3)]


class GformerPlan(ctypes.Structure):
    _fields_ = [("impl", ctypes.c_int32), ("chunk", ctypes.c_int32),
                ("segment_len", ctypes.c_int32), ("n_segments", ctypes.c_int32),
                ("windowed_blocks", ctypes.c_int32), ("windowed_threads", ctypes.c_int32),
                ("linear_blocks", ctypes.c_int32), ("linear_threads", ctypes.c_int32),
                ("state_blocks", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("workspace_bytes", ctypes.c_uint64)]

    def as_dict(self) -> dict:
        return {n: int(getattr(self, n)) for n, _ in self._fields_ if n != "reserved"}


class GformerFeatureParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("head_begin", ctypes.c_int32), ("head_end", ctypes.c_int32),
                ("impl", ctypes.c_int32), ("reserved0", ctypes.c_int32),
                ("x_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3)]


class GformerPackedParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("zero_tail", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float),
                *((f"{x}_stride", ctypes.c_int64 * 2) for x in ("q", "k", "v", "o", "do", "dq", "dk", "dv"))]


class GformerPagedParams(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float),
                *((f"{x}_stride", ctypes.c_int64 * 2) for x in ("q", "o", "k", "v")),
                *((f"{x}_stride", ctypes.c_int64 * 3) for x in ("kpage", "vpage"))]


class GformerPartitionInputs(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("reserved0", ctypes.c_int32),
                ("p", ctypes.c_double), ("size", ctypes.c_double),
                ("flops_per0", ctypes.c_double), ("flops_per1", ctypes.c_double),
                ("perf0", ctypes.c_double), ("perf1", ctypes.c_double)]


class GformerError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"gformer status {status}: {message}")
        self.status = status


_Int64x2 = ctypes.c_int64 * 2
_Int64x3 = ctypes.c_int64 * 3
_lib = None


def lib():
    """Load the shared library (built by paper_2412_19829_amd/build.py).  Fails loudly."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: run `python -m paper_2412_19829_amd.build` "
                "(or __graft_entry__.build()) first; there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER(GformerParams)
        L.gformer_params_init.restype = None
        L.gformer_params_init.argtypes = [P]
        L.gformer_attn_workspace_bytes.restype = ctypes.c_size_t
        L.gformer_attn_workspace_bytes.argtypes = [ctypes.c_int] * 5 + [P]
        L.gformer_attn_plan.restype = ctypes.c_int
        L.gformer_attn_plan.argtypes = [ctypes.c_int] * 5 + [P, ctypes.POINTER(GformerPlan)]
        L.gformer_attn_fwd.restype = ctypes.c_int
        L.gformer_attn_fwd.argtypes = [ctypes.c_void_p] * 4 + [ctypes.c_int] * 5 + \
            [P, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.gformer_attn_fwd_noalloc.restype = ctypes.c_int
        L.gformer_attn_fwd_noalloc.argtypes = [ctypes.c_void_p] * 4 + [ctypes.c_int] * 5 + \
            [P, ctypes.c_void_p]
        L.gformer_attn_prefill.restype = ctypes.c_int
        L.gformer_attn_prefill.argtypes = [ctypes.c_void_p] * 7 + [ctypes.c_int] * 5 + \
            [P, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.gformer_attn_bwd_workspace_bytes.restype = ctypes.c_size_t
        L.gformer_attn_bwd_workspace_bytes.argtypes = [ctypes.c_int] * 5 + [P]
        L.gformer_attn_bwd.restype = ctypes.c_int
        L.gformer_attn_bwd.argtypes = [ctypes.c_void_p] * 7 + [ctypes.c_int] * 5 + \
            [P, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.gformer_attn_decode.restype = ctypes.c_int
        L.gformer_attn_decode.argtypes = [ctypes.c_void_p] * 7 + [ctypes.c_int] * 4 + \
            [ctypes.c_int64, P, ctypes.c_void_p]
        FP = ctypes.POINTER(GformerFeatureParams)
        L.gformer_feature_params_init.restype = None
        L.gformer_feature_params_init.argtypes = [FP]
        L.gformer_random_features.restype = ctypes.c_int
        L.gformer_random_features.argtypes = [ctypes.c_void_p] * 3 + [ctypes.c_int] * 5 + \
            [FP, ctypes.c_void_p]
        PP, GP = ctypes.POINTER(GformerPackedParams), ctypes.POINTER(GformerPagedParams)
        for name, init in (("packed", PP), ("paged", GP)):
            getattr(L, f"gformer_{name}_params_init").restype = None
            getattr(L, f"gformer_{name}_params_init").argtypes = [init]
        L.gformer_packed_attn_fwd.restype = ctypes.c_int
        L.gformer_packed_attn_fwd.argtypes = [ctypes.c_void_p] * 8 + [ctypes.c_int] * 6 + [PP, ctypes.c_void_p]
        L.gformer_packed_attn_bwd_workspace_bytes.restype = ctypes.c_size_t
        L.gformer_packed_attn_bwd_workspace_bytes.argtypes = [ctypes.c_int] * 6 + [PP]
        L.gformer_packed_attn_bwd.restype = ctypes.c_int
        L.gformer_packed_attn_bwd.argtypes = [ctypes.c_void_p] * 12 + [ctypes.c_int] * 6 + \
            [PP, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.gformer_paged_decode_workspace_bytes.restype = ctypes.c_size_t
        L.gformer_paged_decode_workspace_bytes.argtypes = [ctypes.c_int] * 6 + [GP]
        L.gformer_paged_decode.restype = ctypes.c_int
        L.gformer_paged_decode.argtypes = [ctypes.c_void_p] * 8 + [ctypes.c_int] * 7 + \
            [GP, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.gformer_paged_fill.restype = ctypes.c_int
        L.gformer_paged_fill.argtypes = [ctypes.c_void_p] * 7 + [ctypes.c_int] * 6 + [GP, ctypes.c_void_p]
        L.gformer_pages_copy.restype = ctypes.c_int
        L.gformer_pages_copy.argtypes = [ctypes.c_void_p] * 4 + [ctypes.c_int] * 4 + [GP, ctypes.c_void_p]
        L.gformer_partition_balance.restype = ctypes.c_int
        L.gformer_partition_balance.argtypes = [ctypes.POINTER(GformerPartitionInputs),
                                                ctypes.POINTER(ctypes.c_double),
                                                ctypes.POINTER(ctypes.c_double)]
        L.gformer_partition_heads.restype = ctypes.c_int
        L.gformer_partition_heads.argtypes = [ctypes.c_int] * 5 + [ctypes.c_double] * 2 + \
            [ctypes.c_int, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_double)]
        L.gformer_status_string.restype = ctypes.c_char_p
        L.gformer_status_string.argtypes = [ctypes.c_int]
        L.gformer_version.restype = ctypes.c_int
        L.gformer_version.argtypes = []
        L.decode_address = ctypes.cast(L.gformer_attn_decode, ctypes.c_void_p).value
        L.address = {name: ctypes.cast(getattr(L, f"gformer_{name}"), ctypes.c_void_p).value for name in _NATIVE}
        _lib = L
    return _lib


_native = None
_module = None   # the extension module, or None where there is none
_NATIVE = ("packed_attn_fwd", "packed_attn_bwd", "packed_attn_bwd_workspace_bytes", "paged_fill", "paged_decode",
           "paged_decode_workspace_bytes", "pages_copy")


def _decode_call():
    """The extension module with the host side of a decode step (host/decode_call.cpp).  Without it every step goes through
    this file's own code, which costs the host 4 us more: a warning says so, once."""
    global _native, _module
    if _native is None:
        import importlib.util

        import torch  # noqa: F401  (its libraries are what the module links to)
        try:
            spec = importlib.util.spec_from_file_location("_decode_call", CALL_PATH)
            mod = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(mod)
            _native = mod.decode
            _module = mod
        except ImportError as e:
            warnings.warn(f"decode steps are marshalled in Python ({e}); `python -m paper_2412_19829_amd.build` builds the "
                          "module", RuntimeWarning, stacklevel=3)
            _native = lambda *_: None
    return _native


def gformer_params_init() -> GformerParams:
    p = GformerParams()
    lib().gformer_params_init(ctypes.byref(p))
    return p


def make_params(dtype=GF_BF16, n_sparse_heads=0, phi=GF_PHI_ELU1, chunk=0, segment_len=0,
                impl=GF_IMPL_AUTO, launch_mask=0, overlap=0, bidirectional=0, softmax_scale=1.0,
                eps=0.0, q_stride=None, k_stride=None, v_stride=None, o_stride=None) -> GformerParams:
    p = GformerParams(ctypes.sizeof(GformerParams), int(dtype), int(phi), int(n_sparse_heads), int(chunk),
                      int(segment_len), int(impl), int(launch_mask), int(overlap), int(bidirectional),
                      float(softmax_scale), float(eps))
    for name, val in (("q_stride", q_stride), ("k_stride", k_stride),
                      ("v_stride", v_stride), ("o_stride", o_stride)):
        if val is not None:
            setattr(p, name, _Int64x3(*map(int, val)))
    return p


def gformer_status_string(status: int) -> str:
    return lib().gformer_status_string(int(status)).decode()


def gformer_version() -> int:
    return int(lib().gformer_version())


def gformer_attn_workspace_bytes(B, H, N, d, window, params: GformerParams) -> int:
    return int(lib().gformer_attn_workspace_bytes(B, H, N, d, window, ctypes.byref(params)))


def gformer_attn_plan(B, H, N, d, window, params: GformerParams):
    """Returns (status, GformerPlan)."""
    plan = GformerPlan()
    st = lib().gformer_attn_plan(B, H, N, d, window, ctypes.byref(params), ctypes.byref(plan))
    return int(st), plan


def gformer_attn_fwd_raw(q_ptr, k_ptr, v_ptr, out_ptr, B, H, N, d, window, params: GformerParams,
                         workspace_ptr=0, workspace_bytes=0, stream=0) -> int:
    """Direct call with integer device addresses; returns the gf_status."""
    return lib().gformer_attn_fwd(q_ptr, k_ptr, v_ptr, out_ptr, int(B), int(H), int(N), int(d), int(window),
                                  ctypes.byref(params), workspace_ptr, int(workspace_bytes), stream)


GFORMER_NOALLOC_SCRATCH_BYTES = 72 << 20


def gformer_attn_fwd_noalloc_raw(q_ptr, k_ptr, v_ptr, out_ptr, B, H, N, d, window,
                                 params: GformerParams, stream=0) -> int:
    """Direct call with integer device addresses; returns the gf_status."""
    return lib().gformer_attn_fwd_noalloc(q_ptr, k_ptr, v_ptr, out_ptr, int(B), int(H), int(N), int(d), int(window),
                                          ctypes.byref(params), stream)


def _strides3(t):
    s = t.stride()
    if s[3] != 1 and t.shape[3] > 1:
        raise ValueError("last dimension must be contiguous")
    return (s[0], s[1], s[2])


def _current_stream(t) -> int:
    """Raw handle of torch's current stream on `t`'s device (0.1 us through the raw getter against
    1.9 us for building a torch.cuda.Stream, of the 12 us a decode step's call took on the host)."""
    import torch

    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(t.get_device()) if raw is not None else torch.cuda.current_stream(t.device).cuda_stream


def _workspace(nbytes: int, t, stream: int):
    """Workspace of a call on a stream that the caller names.  It is that stream's memory, so that the allocator,
    which has it back before the call has run, gives it to nothing that runs beside the call."""
    import torch

    if stream == _current_stream(t):
        return torch.empty(nbytes, dtype=torch.uint8, device=t.device)
    theirs = torch.cuda.ExternalStream(stream, device=t.device) if stream else torch.cuda.default_stream(t.device)
    with torch.cuda.stream(theirs):
        return torch.empty(nbytes, dtype=torch.uint8, device=t.device)


def gformer_attn_fwd(q, k, v, out, window: int, n_sparse_heads: int, *, phi=GF_PHI_ELU1,
                     chunk=0, segment_len=0, impl=GF_IMPL_AUTO, launch_mask=0, overlap=0,
                     bidirectional=0, softmax_scale=1.0, eps=0.0, workspace=None,
                     stream: Optional[int] = None):
    """GFormer attention forward on torch device tensors shaped [B, H, N, d] (any strides with
    a contiguous last dimension, e.g. a permuted [B, N, H, d] buffer).

    `out` is written in place and returned.  `workspace` is an optional uint8 device tensor
    of at least gformer_attn_workspace_bytes(...) bytes; when omitted and one is needed it is
    allocated with torch.empty, for that stream (plumbing: the library itself never allocates).  The call is
    asynchronous on `stream` (a raw hipStream_t; default: torch's current stream)."""
    import torch

    if not (q.is_cuda and k.is_cuda and v.is_cuda and out.is_cuda):
        raise ValueError("q, k, v, out must be device tensors: there is no CPU path")
    if not (q.dtype == k.dtype == v.dtype == out.dtype):
        raise ValueError("q, k, v, out must share one dtype")
    if q.dtype == torch.bfloat16:
        dtype = GF_BF16
    elif q.dtype == torch.float32:
        dtype = GF_F32
    else:
        raise ValueError(f"unsupported dtype {q.dtype}")
    if not (q.shape == k.shape == v.shape == out.shape) or q.dim() != 4:
        raise ValueError("q, k, v, out must all be [B, H, N, d]")
    B, H, N, d = (int(x) for x in q.shape)
    params = make_params(dtype=dtype, n_sparse_heads=n_sparse_heads, phi=phi, chunk=chunk,
                         segment_len=segment_len, impl=impl, launch_mask=launch_mask,
                         overlap=overlap, bidirectional=bidirectional,
                         softmax_scale=softmax_scale, eps=eps,
                         q_stride=_strides3(q), k_stride=_strides3(k),
                         v_stride=_strides3(v), o_stride=_strides3(out))
    need = gformer_attn_workspace_bytes(B, H, N, d, window, params)
    ws_ptr, ws_bytes = 0, 0
    if need > 0:
        if workspace is None:
            workspace = (torch.empty(need, dtype=torch.uint8, device=q.device) if stream is None
                         else _workspace(need, q, stream))
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if stream is None:
        stream = _current_stream(q)
    st = gformer_attn_fwd_raw(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                              B, H, N, d, window, params, ws_ptr, ws_bytes, stream)
    if st != GF_OK:
        raise GformerError(st, gformer_status_string(st))
    return out


def gformer_feature_params_init() -> GformerFeatureParams:
    p = GformerFeatureParams()
    lib().gformer_feature_params_init(ctypes.byref(p))
    return p


def make_feature_params(dtype=GF_BF16, head_begin=0, head_end=0, impl=GF_IMPL_AUTO,
                        x_stride=None, o_stride=None) -> GformerFeatureParams:
    p = gformer_feature_params_init()
    p.dtype, p.head_begin, p.head_end, p.impl = int(dtype), int(head_begin), int(head_end), int(impl)
    for name, val in (("x_stride", x_stride), ("o_stride", o_stride)):
        if val is not None:
            setattr(p, name, _Int64x3(*map(int, val)))
    return p


def gformer_random_features_raw(x_ptr, w_ptr, out_ptr, B, H, N, d, m, params: GformerFeatureParams,
                                stream=0) -> int:
    """Direct call with integer device addresses; returns the gf_status."""
    return lib().gformer_random_features(x_ptr, w_ptr, out_ptr, int(B), int(H), int(N), int(d), int(m),
                                         ctypes.byref(params), stream)


def gformer_random_features(x, w, out, head_begin: int, head_end: int, *, impl=GF_IMPL_AUTO,
                            stream: Optional[int] = None):
    """Positive random features of heads [head_begin, head_end) of x ([B,H,N,d] device tensor)
    under the projection w ([d,d], dense), written to the same heads of `out` (may be x itself)."""
    import torch

    if not (x.is_cuda and w.is_cuda and out.is_cuda):
        raise ValueError("x, w, out must be device tensors: there is no CPU path")
    if not (x.dtype == w.dtype == out.dtype):
        raise ValueError("x, w, out must share one dtype")
    if x.dtype == torch.bfloat16:
        dtype = GF_BF16
    elif x.dtype == torch.float32:
        dtype = GF_F32
    else:
        raise ValueError(f"unsupported dtype {x.dtype}")
    if x.dim() != 4 or out.shape != x.shape or w.dim() != 2 or not w.is_contiguous():
        raise ValueError("x, out must be [B, H, N, d] and w a dense [m, d] matrix")
    B, H, N, d = (int(v) for v in x.shape)
    params = make_feature_params(dtype=dtype, head_begin=head_begin, head_end=head_end, impl=impl,
                                 x_stride=_strides3(x), o_stride=_strides3(out))
    if stream is None:
        stream = _current_stream(x)
    st = gformer_random_features_raw(x.data_ptr(), w.data_ptr(), out.data_ptr(), B, H, N, d,
                                     int(w.shape[0]), params, stream)
    if st != GF_OK:
        raise GformerError(st, gformer_status_string(st))
    return out


def gformer_attn_decode_raw(q_ptr, k_ptr, v_ptr, out_ptr, kcache_ptr, vcache_ptr, state_ptr, B, H, d,
                            window, t, params: GformerParams, stream=0) -> int:
    """Direct call with integer device addresses; returns the gf_status."""
    return lib().gformer_attn_decode(q_ptr, k_ptr, v_ptr, out_ptr, kcache_ptr, vcache_ptr, state_ptr, int(B),
                                     int(H), int(d), int(window), int(t), ctypes.byref(params), stream)


def gformer_attn_decode(q, k, v, out, kcache, vcache, state, window: int, n_sparse_heads: int, t: int,
                        *, phi=GF_PHI_ELU1, softmax_scale=1.0, eps=0.0, stream: Optional[int] = None):
    """One decode step on dense device tensors: q, k, v, out [B, H, d]; kcache, vcache
    [B, H0, window, d] (or None when H0 == 0); state fp32 [B, H - H0, d*d + d] (or None)."""
    st = (_native or _decode_call())((_lib or lib()).decode_address, q, k, v, out, kcache, vcache, state, window,
                                     n_sparse_heads, t, phi, softmax_scale, eps, stream)
    if st is not None:
        if st != GF_OK:
            raise GformerError(st, gformer_status_string(st))
        return out
    # not the plain call (the module above says which those are): checked and called from here
    import torch

    for x in (q, k, v, out, kcache, vcache, state):
        if x is not None and not (x.is_cuda and x.is_contiguous()):
            raise ValueError("decode tensors must be dense device tensors: there is no CPU path")
    tdt, shape = q.dtype, q.shape
    if tdt == torch.bfloat16:
        dtype = GF_BF16
    elif tdt == torch.float32:
        dtype = GF_F32
    else:
        raise ValueError(f"unsupported dtype {tdt}")
    B, H, d = shape
    for x in (k, v, out):
        if x.shape != shape or x.dtype != tdt:
            raise ValueError("q, k, v, out must all be [B, H, d] of one dtype")
    H0 = int(n_sparse_heads)
    if H0 > 0 and (kcache is None or vcache is None or kcache.dtype != tdt
                   or kcache.shape != (B, H0, window, d) or vcache.shape != kcache.shape):
        raise ValueError("kcache, vcache must be [B, H0, window, d] of the same dtype")
    if H0 < H and (state is None or state.dtype != torch.float32
                   or state.shape != (B, H - H0, d * d + d)):
        raise ValueError("state must be fp32 [B, H - H0, d*d + d]")
    params = make_params(dtype=dtype, n_sparse_heads=H0, phi=phi, softmax_scale=softmax_scale, eps=eps)
    if stream is None:
        stream = _current_stream(q)
    ptr = lambda x: 0 if x is None else x.data_ptr()
    st = gformer_attn_decode_raw(ptr(q), ptr(k), ptr(v), ptr(out), ptr(kcache), ptr(vcache), ptr(state),
                                 B, H, d, window, t, params, stream)
    if st != GF_OK:
        raise GformerError(st, gformer_status_string(st))
    return out


def gformer_attn_prefill_raw(q_ptr, k_ptr, v_ptr, out_ptr, kcache_ptr, vcache_ptr, state_ptr, B, H, N, d,
                             window, params: GformerParams, workspace_ptr=0, workspace_bytes=0,
                             stream=0) -> int:
    """Direct call with integer device addresses; returns the gf_status."""
    return lib().gformer_attn_prefill(q_ptr, k_ptr, v_ptr, out_ptr, kcache_ptr, vcache_ptr, state_ptr, int(B),
                                      int(H), int(N), int(d), int(window), ctypes.byref(params), workspace_ptr,
                                      int(workspace_bytes), stream)


def gformer_attn_prefill(q, k, v, out, kcache, vcache, state, window: int, n_sparse_heads: int, *,
                         phi=GF_PHI_ELU1, impl=GF_IMPL_AUTO, softmax_scale=1.0, eps=0.0,
                         workspace=None, stream: Optional[int] = None):
    """The causal layer on [B, H, N, d] device tensors that also fills the decode step's rings
    (kcache, vcache: dense [B, H0, window, d]) and carried states (fp32 [B, H - H0, d*d + d])."""
    import torch

    if not all(x.is_cuda for x in (q, k, v, out)):
        raise ValueError("q, k, v, out must be device tensors: there is no CPU path")
    dtype = GF_BF16 if q.dtype == torch.bfloat16 else GF_F32
    B, H, N, d = (int(x) for x in q.shape)
    for x in (kcache, vcache, state):
        if x is not None and not (x.is_cuda and x.is_contiguous()):
            raise ValueError("rings and states must be dense device tensors")
    params = make_params(dtype=dtype, n_sparse_heads=n_sparse_heads, phi=phi, impl=impl,
                         softmax_scale=softmax_scale, eps=eps, q_stride=_strides3(q),
                         k_stride=_strides3(k), v_stride=_strides3(v), o_stride=_strides3(out))
    need = gformer_attn_workspace_bytes(B, H, N, d, window, params)
    ws_ptr, ws_bytes = 0, 0
    if need > 0:
        if workspace is None:
            workspace = (torch.empty(need, dtype=torch.uint8, device=q.device) if stream is None
                         else _workspace(need, q, stream))
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if stream is None:
        stream = _current_stream(q)
    ptr = lambda x: 0 if x is None else x.data_ptr()
    st = gformer_attn_prefill_raw(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ptr(kcache),
                                  ptr(vcache), ptr(state), B, H, N, d, window, params, ws_ptr, ws_bytes,
                                  stream)
    if st != GF_OK:
        raise GformerError(st, gformer_status_string(st))
    return out


def gformer_attn_bwd_workspace_bytes(B, H, N, d, window, params: GformerParams) -> int:
    return int(lib().gformer_attn_bwd_workspace_bytes(B, H, N, d, window, ctypes.byref(params)))


def gformer_attn_bwd_raw(q_ptr, k_ptr, v_ptr, dout_ptr, dq_ptr, dk_ptr, dv_ptr, B, H, N, d, window,
                         params: GformerParams, workspace_ptr=0, workspace_bytes=0, stream=0) -> int:
    """Direct call with integer device addresses; returns the gf_status."""
    return lib().gformer_attn_bwd(q_ptr, k_ptr, v_ptr, dout_ptr, dq_ptr, dk_ptr, dv_ptr, int(B), int(H), int(N),
                                  int(d), int(window), ctypes.byref(params), workspace_ptr,
                                  int(workspace_bytes), stream)


def gformer_attn_bwd(q, k, v, dout, dq, dk, dv, window: int, n_sparse_heads: int, *,
                     phi=GF_PHI_ELU1, impl=GF_IMPL_AUTO, softmax_scale=1.0, eps=0.0, overlap=0,
                     bidirectional=0, workspace=None, stream: Optional[int] = None):
    """Backward of the layer (causal or bidirectional) on [B, H, N, d] device tensors: fills dq,
    dk, dv (laid out like q, k, v) from `dout`, the gradient with respect to the layer's output."""
    import torch

    if not all(x.is_cuda for x in (q, k, v, dout, dq, dk, dv)):
        raise ValueError("all tensors must be device tensors: there is no CPU path")
    if _strides3(dq) != _strides3(q) or _strides3(dk) != _strides3(k) or _strides3(dv) != _strides3(v):
        raise ValueError("dq, dk, dv must be laid out like q, k, v")
    dtype = GF_BF16 if q.dtype == torch.bfloat16 else GF_F32
    B, H, N, d = (int(x) for x in q.shape)
    params = make_params(dtype=dtype, n_sparse_heads=n_sparse_heads, phi=phi, impl=impl,
                         softmax_scale=softmax_scale, eps=eps, overlap=overlap,
                         bidirectional=bidirectional, q_stride=_strides3(q),
                         k_stride=_strides3(k), v_stride=_strides3(v), o_stride=_strides3(dout))
    need = gformer_attn_bwd_workspace_bytes(B, H, N, d, window, params)
    ws_ptr, ws_bytes = 0, 0
    if need > 0:
        if workspace is None:
            workspace = (torch.empty(need, dtype=torch.uint8, device=q.device) if stream is None
                         else _workspace(need, q, stream))
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if stream is None:
        stream = _current_stream(q)
    st = gformer_attn_bwd_raw(q.data_ptr(), k.data_ptr(), v.data_ptr(), dout.data_ptr(),
                              dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, N, d, window, params,
                              ws_ptr, ws_bytes, stream)
    if st != GF_OK:
        raise GformerError(st, gformer_status_string(st))
    return dq, dk, dv


# ---- packed sequences and the paged cache ------------------------------------------------------

def _row_strides(name, t):
    """Strides of a [rows, heads, d] or [pages, heads, tokens, d] tensor without the last; those of single
    rows, which say nothing, as if it were dense."""
    shape, s = t.shape, t.stride()
    if s[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    out, dense = [], shape[-1]
    for n, x in zip(reversed(shape[:-1]), reversed(s[:-1])):
        if n > 1 and x == 0:
            raise ValueError(f"{name}: broadcast dimensions (stride 0) are not supported")
        out.append(x if n > 1 else dense)
        dense *= max(n, 1)
    return out[::-1]


def _sizes(**sizes):
    """Numbers that the library takes as int: ctypes would hand over what is left of larger ones."""
    for name, n in sizes.items():
        if not -1 << 31 <= n < 1 << 31:
            raise ValueError(f"{name}: {n} does not fit 32 bits")


def _tensors(like, n_dims, **tensors):
    """Device tensors of one type, one device and `n_dims` dimensions."""
    import torch

    if like.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"unsupported dtype {like.dtype}")
    for name, t in tensors.items():
        _sizes(**{name: max(t.shape, default=0)})
        if not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor: there is no CPU path")
        if t.dtype != like.dtype or t.device != like.device:
            raise ValueError(f"{name} must have the type and device of the others")
        if t.dim() != n_dims:
            raise ValueError(f"{name} must have {n_dims} dimensions")
    return GF_BF16 if like.dtype == torch.bfloat16 else GF_F32


def _numbers(like, shape, **tensors):
    """Dense int32 tensors on the device of `like`; a None in `shape` fits any size."""
    import torch

    for name, t in tensors.items():
        _sizes(**{name: max(t.shape, default=0)})
        if not t.is_cuda or t.device != like.device or t.dtype != torch.int32 or not t.is_contiguous():
            raise ValueError(f"{name} must be a dense int32 tensor on the device of the others")
        if t.dim() != len(shape) or any(n is not None and n != x for n, x in zip(shape, t.shape)):
            raise ValueError(f"{name} must be of shape {list(shape)}")


def _packed_shapes(q, k, v, cu_q, cu_k, **like_q):
    for name, t in like_q.items():
        if t.shape != q.shape:
            raise ValueError(f"{name} must be of q's shape")
    if k.shape != v.shape or k.shape[2] != q.shape[2]:
        raise ValueError("q must be [total_q, H, d], k and v [total_k, Hkv, d]")
    if cu_q.numel() < 1:
        raise ValueError("cu_q must hold n_seqs + 1 offsets")
    _numbers(q, (None,), cu_q=cu_q)
    if cu_k is not None:
        _numbers(q, cu_q.shape, cu_k=cu_k)
    elif k.shape[0] != q.shape[0]:
        raise ValueError("cu_k may be left out only where q and k have the same rows")


def _call(entry, like, stream, *args):
    """entry(*args, stream) with the tensors' device current."""
    import torch

    if stream is None:
        stream = _current_stream(like)
    if torch.cuda.current_device() == like.get_device():
        st = entry(*args, stream)
    else:
        with torch.cuda.device(like.device):
            st = entry(*args, stream)
    if st != GF_OK:
        raise GformerError(st, gformer_status_string(st))


def _scratch(need, workspace, like, stream):
    """(address, bytes) of the caller's workspace, or of one for this call."""
    import torch

    if workspace is None:
        if need == 0:
            return None, 0, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=like.device) if stream is None else _workspace(need, like, stream)
    elif not workspace.is_cuda or workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a dense tensor on the device of the others")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _quick(function, entries, *args):
    """Whether the extension module has made the call (host/packed_call.cpp says which ones it makes)."""
    if _native is None:
        _decode_call()
    if _module is None:
        return False
    address = (_lib or lib()).address
    st = getattr(_module, function)(*(address[e] for e in entries), *args)
    if st is None:
        return False
    if st != GF_OK:
        raise GformerError(st, gformer_status_string(st))
    return True


def packed_attention_node(q, k, v, cu_q, cu_k, softmax_scale):
    """Packed attention with its node in torch's graph from the extension module (host/packed_grad.cpp), or None for what
    is not its plain call."""
    if _native is None:
        _decode_call()
    if _module is None:
        return None
    address = (_lib or lib()).address
    out = _module.packed_attention(address["packed_attn_fwd"], address["packed_attn_bwd"], address["packed_attn_bwd_workspace_bytes"],
                                   q, k, v, cu_q, cu_k, softmax_scale)
    if isinstance(out, int):
        raise GformerError(out, gformer_status_string(out))
    return out


def make_packed_params(dtype=GF_BF16, softmax_scale=1.0, zero_tail=0, **strides) -> GformerPackedParams:
    """strides: q_stride=, k_stride=, ... as (row, head)."""
    p = GformerPackedParams(ctypes.sizeof(GformerPackedParams), int(dtype), int(zero_tail), float(softmax_scale))
    for name, val in strides.items():
        setattr(p, name, _Int64x2(*val))
    return p


def make_paged_params(dtype=GF_BF16, page_size=64, softmax_scale=1.0, **strides) -> GformerPagedParams:
    """strides: q_stride=, ... as (sequence or row, head), kpage_stride=, vpage_stride= as (page, head, token)."""
    p = GformerPagedParams(ctypes.sizeof(GformerPagedParams), int(dtype), int(page_size), float(softmax_scale))
    for name, val in strides.items():
        setattr(p, name, (_Int64x2 if len(val) == 2 else _Int64x3)(*val))
    return p


def _rest(out, rest):
    """Address of the tensor that holds what rounding took from `out`."""
    if rest is None:
        return None
    if rest.dtype != out.dtype or rest.device != out.device or rest.shape != out.shape or rest.stride() != out.stride():
        raise ValueError("out_rest must be laid out like out")
    return rest.data_ptr()


def gformer_packed_attn_fwd(q, k, v, out, cu_q, cu_k=None, *, lse=None, out_rest=None, softmax_scale=1.0, zero_tail=0,
                            stream: Optional[int] = None):
    """Causal attention over packed sequences on device tensors: q, out [total_q, H, d], k, v [total_k, Hkv, d]
    (any strides with a contiguous last dimension); cu_q, cu_k int32 [n_seqs + 1] offsets (cu_k=None: the same
    sequences).  Optional and written, for the backward pass: lse, dense fp32 [H, total_q], and (bf16 only) out_rest, laid
    out like out, what rounding took from it."""
    if _quick("packed_fwd", ("packed_attn_fwd",), q, k, v, out, cu_q, cu_k, lse, out_rest, softmax_scale, zero_tail, stream):
        return out
    import torch

    dtype = _tensors(q, 3, q=q, k=k, v=v, out=out)
    _packed_shapes(q, k, v, cu_q, cu_k, out=out)
    T, H, d = q.shape
    if lse is not None and (lse.device != q.device or lse.dtype != torch.float32 or lse.shape != (H, T) or not lse.is_contiguous()):
        raise ValueError("lse must be dense fp32 [H, total_q]")
    p = make_packed_params(dtype, softmax_scale, zero_tail, q_stride=_row_strides("q", q), k_stride=_row_strides("k", k),
                           v_stride=_row_strides("v", v), o_stride=_row_strides("out", out))
    _call(lib().gformer_packed_attn_fwd, q, stream, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
          _rest(out, out_rest), None if lse is None else lse.data_ptr(), cu_q.data_ptr(), None if cu_k is None else cu_k.data_ptr(),
          cu_q.numel() - 1, T, k.shape[0], H, k.shape[1], d, ctypes.byref(p))
    return out


def gformer_packed_attn_bwd_workspace_bytes(total_q, total_k, n_seqs, H, Hkv, d, params=None) -> int:
    _sizes(total_q=total_q, total_k=total_k, n_seqs=n_seqs, H=H, Hkv=Hkv, d=d)
    return int(lib().gformer_packed_attn_bwd_workspace_bytes(total_q, total_k, n_seqs, H, Hkv, d,
                                                             ctypes.byref(params or make_packed_params())))


def gformer_packed_attn_bwd(q, k, v, out, lse, dout, dq, dk, dv, cu_q, cu_k=None, *, out_rest=None, softmax_scale=1.0,
                            zero_tail=0, workspace=None, stream: Optional[int] = None):
    """Gradients of gformer_packed_attn_fwd from what it wrote (out, lse, out_rest) and the gradient dout of
    out."""
    if _quick("packed_bwd", ("packed_attn_bwd", "packed_attn_bwd_workspace_bytes"), q, k, v, out, cu_q, cu_k, lse, dout, dq, dk, dv,
              out_rest, softmax_scale, zero_tail, workspace, stream):
        return dq, dk, dv
    import torch

    dtype = _tensors(q, 3, q=q, k=k, v=v, out=out, dout=dout, dq=dq, dk=dk, dv=dv)
    _packed_shapes(q, k, v, cu_q, cu_k, out=out, dout=dout, dq=dq)
    if dk.shape != k.shape or dv.shape != v.shape:
        raise ValueError("dk and dv must be of k's shape")
    T, H, d = q.shape
    if lse.device != q.device or lse.dtype != torch.float32 or lse.shape != (H, T) or not lse.is_contiguous():
        raise ValueError("lse must be dense fp32 [H, total_q]")
    p = make_packed_params(dtype, softmax_scale, zero_tail, q_stride=_row_strides("q", q), k_stride=_row_strides("k", k),
                           v_stride=_row_strides("v", v), o_stride=_row_strides("out", out), do_stride=_row_strides("dout", dout),
                           dq_stride=_row_strides("dq", dq), dk_stride=_row_strides("dk", dk), dv_stride=_row_strides("dv", dv))
    sizes = (cu_q.numel() - 1, T, k.shape[0], H, k.shape[1], d)
    need = gformer_packed_attn_bwd_workspace_bytes(T, k.shape[0], *sizes[:1], *sizes[3:], p)
    workspace, at, held = _scratch(need, workspace, q, stream)
    _call(lib().gformer_packed_attn_bwd, q, stream, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), _rest(out, out_rest),
          lse.data_ptr(), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), cu_q.data_ptr(),
          None if cu_k is None else cu_k.data_ptr(), *sizes, ctypes.byref(p), at, held)
    return dq, dk, dv


def gformer_paged_decode_workspace_bytes(B, H, Hkv, d, max_len, params=None, table_width=None) -> int:
    """For sequences of up to max_len tokens, the new one included (0: what a table of table_width pages holds)."""
    p = params or make_paged_params()
    if table_width is None:
        table_width = -(-max_len // p.page_size)
    _sizes(B=B, H=H, Hkv=Hkv, d=d, max_len=max_len, table_width=table_width)
    return int(lib().gformer_paged_decode_workspace_bytes(B, H, Hkv, d, table_width, max_len, ctypes.byref(p)))


def _paged(like, kpages, vpages, Hkv, d):
    _tensors(like, 4, kpages=kpages, vpages=vpages)
    if kpages.shape != vpages.shape or kpages.shape[1] != Hkv or kpages.shape[3] != d:
        raise ValueError("kpages and vpages must be [n_pages, Hkv, page_size, d]")
    return {"page_size": kpages.shape[2], "kpage_stride": _row_strides("kpages", kpages),
            "vpage_stride": _row_strides("vpages", vpages)}


def gformer_paged_decode(q, k, v, out, kpages, vpages, table, lens, *, max_len=0, softmax_scale=1.0, workspace=None,
                         stream: Optional[int] = None):
    """One new token of every sequence over a paged cache, on device tensors: q, out [B, H, d]; k, v [B, Hkv, d], the new
    keys and values, which go to their slots (both None: they are there already); kpages, vpages
    [n_pages, Hkv, page_size, d] (any strides with a contiguous last dimension); table int32 [B, table_width]; lens int32
    [B], the tokens in the cache before the call (negative: an idle row).  max_len bounds the longest
    sequence's tokens, the new one included (0: what the table holds)."""
    if _quick("paged_decode", ("paged_decode", "paged_decode_workspace_bytes"), q, k, v, out, kpages, vpages, table, lens, max_len,
              softmax_scale, workspace, stream):
        return out
    if (k is None) != (v is None):
        raise ValueError("k and v come together, or neither")
    new = {} if k is None else {"k": k, "v": v}
    dtype = _tensors(q, 3, q=q, out=out, **new)
    B, H, d = q.shape
    Hkv = kpages.shape[1] if kpages.dim() == 4 else 0
    if out.shape != q.shape or any(x.shape != (B, Hkv, d) for x in new.values()):
        raise ValueError("q and out must be [B, H, d], k and v [B, Hkv, d]")
    _numbers(q, (B, None), table=table)
    _numbers(q, (B,), lens=lens)
    strides = {f"{n}_stride": _row_strides(n, t) for n, t in {"q": q, **new}.items()}
    p = make_paged_params(dtype, softmax_scale=softmax_scale, o_stride=_row_strides("out", out), **strides,
                          **_paged(q, kpages, vpages, Hkv, d))
    width = table.shape[1]
    need = gformer_paged_decode_workspace_bytes(B, H, Hkv, d, max_len, p, width)
    workspace, at, held = _scratch(need, workspace, q, stream)
    _call(lib().gformer_paged_decode, q, stream, q.data_ptr(), None if k is None else k.data_ptr(),
          None if v is None else v.data_ptr(), out.data_ptr(), kpages.data_ptr(), vpages.data_ptr(), table.data_ptr(),
          lens.data_ptr(), B, H, Hkv, d, kpages.shape[0], width, int(max_len), ctypes.byref(p), at, held)
    return out


def gformer_paged_fill(k, v, kpages, vpages, table, start, cu, *, stream: Optional[int] = None):
    """Packed keys and values [total, Hkv, d] into a paged cache: row i of sequence s becomes its token start[s] + i.
    table int32 [n_seqs, table_width], start int32 [n_seqs], cu int32 [n_seqs + 1]."""
    if _quick("paged_fill", ("paged_fill",), k, v, kpages, vpages, table, start, cu, stream):
        return
    dtype = _tensors(k, 3, k=k, v=v)
    if k.shape != v.shape or cu.numel() < 1:
        raise ValueError("k and v must be [total, Hkv, d], cu [n_seqs + 1]")
    T, Hkv, d = k.shape
    n = cu.numel() - 1
    _numbers(k, (n + 1,), cu=cu)
    _numbers(k, (n, None), table=table)
    _numbers(k, (n,), start=start)
    p = make_paged_params(dtype, k_stride=_row_strides("k", k), v_stride=_row_strides("v", v), **_paged(k, kpages, vpages, Hkv, d))
    _call(lib().gformer_paged_fill, k, stream, k.data_ptr(), v.data_ptr(), kpages.data_ptr(), vpages.data_ptr(), table.data_ptr(),
          start.data_ptr(), cu.data_ptr(), n, T, Hkv, d, kpages.shape[0], table.shape[1], ctypes.byref(p))


def gformer_pages_copy(kpages, vpages, src, dst, *, stream: Optional[int] = None):
    """Pages src[i] -> dst[i] of a paged cache (int32 device tensors), whole, keys and values; no destination may be another
    one or another's source."""
    if _quick("pages_copy", ("pages_copy",), kpages, vpages, src, dst, stream):
        return
    dtype = _tensors(kpages, 4, kpages=kpages, vpages=vpages)
    P, Hkv, _, d = kpages.shape
    _numbers(kpages, (None,), src=src)
    _numbers(kpages, (src.numel(),), dst=dst)
    p = make_paged_params(dtype, **_paged(kpages, kpages, vpages, Hkv, d))
    _call(lib().gformer_pages_copy, kpages, stream, kpages.data_ptr(), vpages.data_ptr(), src.data_ptr(), dst.data_ptr(),
          src.numel(), Hkv, d, P, ctypes.byref(p))


def gformer_partition_balance(p, size, flops_per0, flops_per1, perf0, perf1):
    """Algorithm 2 through the C ABI (host arithmetic).  Returns (p', [latency0(p), latency1(p),
    latency0(p'), latency1(p')])."""
    inp = GformerPartitionInputs(ctypes.sizeof(GformerPartitionInputs), 0, p, size, flops_per0,
                                 flops_per1, perf0, perf1)
    pp = ctypes.c_double()
    lat = (ctypes.c_double * 4)()
    st = int(lib().gformer_partition_balance(ctypes.byref(inp), ctypes.byref(pp), lat))
    if st != GF_OK:
        raise GformerError(st, gformer_status_string(st))
    return pp.value, list(lat)


def gformer_partition_heads(B, H, N, E, W, perf_sparse, perf_linear, flop_model=GF_FLOPS_PAPER):
    """The balance of Section III-D over whole heads.  Returns (H0, [windowed latency, linear
    latency])."""
    h0 = ctypes.c_int()
    lat = (ctypes.c_double * 2)()
    st = int(lib().gformer_partition_heads(int(B), int(H), int(N), int(E), int(W), float(perf_sparse),
                                           float(perf_linear), int(flop_model), ctypes.byref(h0), lat))
    if st != GF_OK:
        raise GformerError(st, gformer_status_string(st))
    return h0.value, list(lat)
