"""Thin ctypes binding of libtsa.so: same names as the C ABI (include/tsa.h), argument
marshalling only.  Tensors are torch CUDA tensors used purely as device memory; every step
runs in the library's HIP kernels.  There is no fallback: if the library is missing or a
call fails, an exception is raised."""
from __future__ import annotations

import ctypes
import math
import os

import torch

from . import build as _build

TSA_OK, TSA_ERR_ARG, TSA_ERR_UNSUPPORTED, TSA_ERR_WORKSPACE, TSA_ERR_HIP = 0, 1, 2, 3, 4

EXPORTS = ("tsa_version", "tsa_last_error", "tsa_keep_count", "tsa_workspace_bytes", "tsa_score", "tsa_coverage_budget",
           "tsa_score_queries_workspace_bytes", "tsa_score_queries", "tsa_gather_queries", "tsa_pool_queries_workspace_bytes", "tsa_pool_queries",
           "tsa_select", "tsa_compress", "tsa_attend_workspace_bytes", "tsa_attend", "tsa_decompress", "tsa_compress_v_tiles", "tsa_attend_fused", "tsa_forward",
           "tsa_forward_dynamic_workspace_bytes", "tsa_forward_dynamic",
           "tsa_layer_drift_workspace_bytes", "tsa_layer_drift", "tsa_sparse_layers", "tsa_mfma_probe", "tsa_mix_probe", "tsa_read_probe", "tsa_copy_probe", "tsa_bench_set_attend_form",
           "tsa_select_static", "tsa_select_static_capacity", "tsa_rotary", "tsa_rotary_frequencies",
           "tsa_cache_write", "tsa_cache_read", "tsa_attend_cache_workspace_bytes", "tsa_attend_cache")

TSA_ROTARY_MAX_FREQS = 64
TSA_ROTARY_PLAIN, TSA_ROTARY_LINEAR, TSA_ROTARY_BASE, TSA_ROTARY_PARTS, TSA_ROTARY_WAVELENGTH = 0, 1, 2, 3, 4


class TsaError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("libtsa error %d: %s" % (code, msg))
        self.code = code


class tsa_desc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("L", ctypes.c_int32),
                ("d", ctypes.c_int32), ("last_q", ctypes.c_int32), ("pool_w", ctypes.c_int32),
                ("group_mode", ctypes.c_int32), ("force_first", ctypes.c_int32), ("force_last", ctypes.c_int32),
                ("scale", ctypes.c_float), ("block_list_per_head", ctypes.c_int32), ("q_stride_b", ctypes.c_int64), ("q_stride_h", ctypes.c_int64), ("q_stride_l", ctypes.c_int64),
                ("kv_stride_b", ctypes.c_int64), ("kv_stride_h", ctypes.c_int64), ("kv_stride_l", ctypes.c_int64),
                ("o_stride_b", ctypes.c_int64), ("o_stride_h", ctypes.c_int64), ("o_stride_l", ctypes.c_int64)]


def make_desc(B, Hq, Hkv, L, d, last_q=64, pool_w=1, group_mode=0, force_first=0, force_last=0, scale=0.0,
              block_list_per_head=0, q_strides=(0, 0, 0), kv_strides=(0, 0, 0), o_strides=(0, 0, 0)):
    """*_strides = (stride_b, stride_h, stride_l) in elements of Q, of K and V, of O; zeros = contiguous [B,H,L,d]."""
    return tsa_desc(B, Hq, Hkv, L, d, last_q, pool_w, group_mode, force_first, force_last, scale, block_list_per_head,
                    *q_strides, *kv_strides, *o_strides)


def blhd_strides(H, L, d):
    """Strides of a [B,L,H,d] tensor addressed as (b, h, t)."""
    return (L * H * d, d, H * d)


class tsa_rotary_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hq", "Hkv", "L", "d", "rot", "interleaved", "start")] + \
               [("gain", ctypes.c_float), ("reserved", ctypes.c_int32)] + \
               [("%s_stride_%s" % (t, a), ctypes.c_int64) for t in ("q", "k", "q_out", "k_out") for a in "bhl"] + \
               [("freq", ctypes.c_double * TSA_ROTARY_MAX_FREQS)]


def make_rotary_desc(B, Hq, Hkv, L, d, freq, interleaved=0, start=0, gain=1.0, q_strides=(0, 0, 0), k_strides=(0, 0, 0),
                     q_out_strides=(0, 0, 0), k_out_strides=(0, 0, 0)):
    """freq: radians per position of every pair (rot = 2 len(freq) columns are rotated); strides as in make_desc."""
    if len(freq) > TSA_ROTARY_MAX_FREQS:
        raise TsaError(TSA_ERR_ARG, "at most %d frequencies" % TSA_ROTARY_MAX_FREQS)
    return tsa_rotary_desc(B, Hq, Hkv, L, d, 2 * len(freq), interleaved, start, gain, 0, *q_strides, *k_strides, *q_out_strides,
                           *k_out_strides, (ctypes.c_double * TSA_ROTARY_MAX_FREQS)(*[float(f) for f in freq]))


TSA_CACHE_BF16, TSA_CACHE_E4M3 = 0, 1


class tsa_cache_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seqs", "n_tokens", "max_q", "Hq", "Hkv", "d", "page_size", "n_pages", "max_pages", "format",
                                              "window")] + [("scale", ctypes.c_float)] + \
               [("%s_stride_%s" % (t, a), ctypes.c_int64) for t in "qkvo" for a in "th"]


def make_cache_desc(n_seqs, n_tokens, Hq, Hkv, d, page_size, n_pages, max_pages, format=TSA_CACHE_BF16, max_q=0, window=0, scale=0.0,
                    q_strides=(0, 0), k_strides=(0, 0), v_strides=(0, 0), o_strides=(0, 0)):
    """*_strides = (stride of a token, stride of a head) in elements of the packed tensors; zeros = contiguous [n_tokens, heads, d].
    max_q: most new tokens of a sequence; 0 (not known) is right for any, and prepares the attention and its workspace for prompts."""
    return tsa_cache_desc(n_seqs, n_tokens, max_q, Hq, Hkv, d, page_size, n_pages, max_pages, format, window, scale,
                          *q_strides, *k_strides, *v_strides, *o_strides)


_lib = None


def load_library(build_if_missing: bool = True) -> ctypes.CDLL:
    """Loads the in-tree libtsa.so; builds it first only if it does not exist."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB_PATH
    if not os.path.exists(path):
        if not build_if_missing:
            raise ImportError("libtsa.so is not built (%s)" % path)
        _build.build_library()
    lib = ctypes.CDLL(path)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    dp = ctypes.POINTER(tsa_desc)
    lib.tsa_version.restype = ctypes.c_int
    lib.tsa_version.argtypes = []
    lib.tsa_last_error.restype = ctypes.c_char_p
    lib.tsa_last_error.argtypes = []
    lib.tsa_keep_count.restype = i32
    lib.tsa_keep_count.argtypes = [i32, ctypes.c_double]
    lib.tsa_workspace_bytes.restype = sz
    lib.tsa_workspace_bytes.argtypes = [dp, i32]
    lib.tsa_score.restype = ctypes.c_int
    lib.tsa_score.argtypes = [dp, vp, vp, vp, vp, sz, vp]
    ip = ctypes.POINTER(i32)
    lib.tsa_score_queries.restype = ctypes.c_int
    lib.tsa_score_queries.argtypes = [dp, vp, ip, i32, vp, vp, vp, sz, vp]
    lib.tsa_score_queries_workspace_bytes.restype = sz
    lib.tsa_score_queries_workspace_bytes.argtypes = [dp, i32]
    lib.tsa_bench_set_attend_form.restype = ctypes.c_int
    lib.tsa_bench_set_attend_form.argtypes = [i32]
    lib.tsa_copy_probe.restype = ctypes.c_int
    lib.tsa_copy_probe.argtypes = [vp, vp, sz, vp]
    lib.tsa_read_probe.restype = ctypes.c_int
    lib.tsa_read_probe.argtypes = [vp, sz, vp, vp]
    lib.tsa_mix_probe.restype = ctypes.c_int
    lib.tsa_mix_probe.argtypes = [i32, vp, i32, i32, vp, ctypes.POINTER(ctypes.c_double), vp]
    lib.tsa_gather_queries.restype = ctypes.c_int
    lib.tsa_gather_queries.argtypes = [dp, vp, ip, i32, vp, vp]
    lib.tsa_pool_queries_workspace_bytes.restype = sz
    lib.tsa_pool_queries_workspace_bytes.argtypes = [dp, i32]
    lib.tsa_pool_queries.restype = ctypes.c_int
    lib.tsa_pool_queries.argtypes = [dp, vp, i32, vp, ip, vp, sz, vp]
    lib.tsa_coverage_budget.restype = ctypes.c_int
    lib.tsa_coverage_budget.argtypes = [dp, vp, ctypes.c_double, vp, vp, sz, vp]
    lib.tsa_select.restype = ctypes.c_int
    lib.tsa_select.argtypes = [dp, vp, i32, vp, vp, vp, sz, vp]
    lib.tsa_select_static.restype = ctypes.c_int
    lib.tsa_select_static.argtypes = [dp, vp, i32, vp, vp, vp]
    lib.tsa_select_static_capacity.restype = sz
    lib.tsa_select_static_capacity.argtypes = []
    lib.tsa_compress.restype = ctypes.c_int
    lib.tsa_compress.argtypes = [dp, vp, vp, vp, vp, i32, vp, vp, vp, vp]
    lib.tsa_attend.restype = ctypes.c_int
    lib.tsa_attend.argtypes = [dp, vp, vp, vp, i32, i32, vp, i32, i32, vp, vp, vp, sz, vp]
    lib.tsa_compress_v_tiles.restype = ctypes.c_int
    lib.tsa_compress_v_tiles.argtypes = [dp, vp, vp, i32, vp, sz, vp]
    lib.tsa_attend_fused.restype = ctypes.c_int
    lib.tsa_attend_fused.argtypes = [dp, vp, vp, vp, vp, vp, i32, vp, i32, i32, vp, vp, vp, vp]
    lib.tsa_mfma_probe.restype = ctypes.c_int
    lib.tsa_mfma_probe.argtypes = [vp, i32, i32, vp, vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i32), vp]
    lib.tsa_attend_workspace_bytes.restype = sz
    lib.tsa_attend_workspace_bytes.argtypes = [dp, i32, i32]
    lib.tsa_decompress.restype = ctypes.c_int
    lib.tsa_decompress.argtypes = [dp, vp, vp, vp, i32, vp, vp, vp]
    lib.tsa_forward_dynamic_workspace_bytes.restype = sz
    lib.tsa_forward_dynamic_workspace_bytes.argtypes = [dp, i32]
    lib.tsa_forward_dynamic.restype = ctypes.c_int
    lib.tsa_forward_dynamic.argtypes = [dp, vp, vp, vp, ctypes.c_double, i32, vp, i32, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.tsa_forward.restype = ctypes.c_int
    lib.tsa_forward.argtypes = [dp, vp, vp, vp, i32, vp, i32, i32, vp, vp, vp, vp, sz, vp]
    lib.tsa_layer_drift_workspace_bytes.restype = sz
    lib.tsa_layer_drift_workspace_bytes.argtypes = [ctypes.c_int64]
    lib.tsa_layer_drift.restype = ctypes.c_int
    lib.tsa_layer_drift.argtypes = [vp, vp, ctypes.c_int64, i32, ctypes.c_float, vp, vp, sz, vp]
    lib.tsa_sparse_layers.restype = ctypes.c_int
    lib.tsa_sparse_layers.argtypes = [ctypes.POINTER(ctypes.c_float), i32, ctypes.c_double, ctypes.POINTER(i32)]
    lib.tsa_rotary.restype = ctypes.c_int
    lib.tsa_rotary.argtypes = [ctypes.POINTER(tsa_rotary_desc), vp, vp, vp, vp, vp, vp]
    dbl = ctypes.c_double
    lib.tsa_rotary_frequencies.restype = ctypes.c_int
    lib.tsa_rotary_frequencies.argtypes = [i32, i32, dbl, dbl, dbl, dbl, dbl, ctypes.POINTER(dbl), ctypes.POINTER(ctypes.c_float)]
    cp = ctypes.POINTER(tsa_cache_desc)
    lib.tsa_cache_write.restype = ctypes.c_int
    lib.tsa_cache_write.argtypes = [cp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.tsa_cache_read.restype = ctypes.c_int
    lib.tsa_cache_read.argtypes = [cp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp]
    lib.tsa_attend_cache_workspace_bytes.restype = sz
    lib.tsa_attend_cache_workspace_bytes.argtypes = [cp]
    lib.tsa_attend_cache.restype = ctypes.c_int
    lib.tsa_attend_cache.argtypes = [cp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    _lib = lib
    return lib


def _check(rc):
    if rc != TSA_OK:
        raise TsaError(rc, load_library().tsa_last_error().decode())


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise TsaError(TSA_ERR_ARG, "tensor is not on the GPU")
    if not t.is_contiguous():
        raise TsaError(TSA_ERR_ARG, "tensor is not contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ws(ws):
    if ws is None:
        return None, 0
    return _ptr(ws), ws.numel() * ws.element_size()


def tsa_version() -> int:
    return load_library().tsa_version()


def tsa_last_error() -> str:
    return load_library().tsa_last_error().decode()


def tsa_keep_count(L: int, tau: float) -> int:
    return load_library().tsa_keep_count(L, tau)


def tsa_workspace_bytes(desc: tsa_desc, k_keep: int) -> int:
    return load_library().tsa_workspace_bytes(ctypes.byref(desc), k_keep)


def tsa_score(desc, Q, K, scores, ws):
    p, n = _ws(ws)
    _check(load_library().tsa_score(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(scores), p, n, _stream()))


def _host_ints(values):
    return (ctypes.c_int32 * len(values))(*[int(v) for v in values])


def tsa_score_queries_workspace_bytes(desc, n) -> int:
    return int(load_library().tsa_score_queries_workspace_bytes(ctypes.byref(desc), n))


def tsa_score_queries(desc, Qsel, qpos, K, scores, ws=None):
    """qpos: sequence of host ints (ascending positions of the rows of Qsel)."""
    if ws is None:
        ws = torch.empty(max(256, tsa_score_queries_workspace_bytes(desc, len(qpos))), dtype=torch.uint8, device=K.device)
    p, n = _ws(ws)
    _check(load_library().tsa_score_queries(ctypes.byref(desc), _ptr(Qsel), _host_ints(qpos), len(qpos), _ptr(K),
                                            _ptr(scores), p, n, _stream()))


def tsa_gather_queries(desc, Q, qpos, Qsel):
    _check(load_library().tsa_gather_queries(ctypes.byref(desc), _ptr(Q), _host_ints(qpos), len(qpos), _ptr(Qsel), _stream()))


def tsa_pool_queries(desc, Q, n_pool, Qsel, ws=None):
    """Returns the positions (host list) of the pooled queries."""
    if ws is None:
        ws = torch.empty(max(256, load_library().tsa_pool_queries_workspace_bytes(ctypes.byref(desc), n_pool)),
                         dtype=torch.uint8, device=Q.device)
    p, n = _ws(ws)
    qpos = (ctypes.c_int32 * n_pool)()
    _check(load_library().tsa_pool_queries(ctypes.byref(desc), _ptr(Q), n_pool, _ptr(Qsel), qpos, p, n, _stream()))
    return list(qpos)


def tsa_coverage_budget(desc, scores, tau_cov, k_keep, ws):
    p, n = _ws(ws)
    _check(load_library().tsa_coverage_budget(ctypes.byref(desc), _ptr(scores), float(tau_cov), _ptr(k_keep), p, n, _stream()))


def tsa_select(desc, scores, k_keep, idx, inv, ws=None):
    p, n = _ws(ws)
    _check(load_library().tsa_select(ctypes.byref(desc), _ptr(scores), k_keep, _ptr(idx), _ptr(inv), p, n, _stream()))


def tsa_select_static(desc, scores, k_keep, idx, inv):
    _check(load_library().tsa_select_static(ctypes.byref(desc), _ptr(scores), k_keep, _ptr(idx), _ptr(inv), _stream()))


def tsa_compress(desc, Q, K, V, idx, k_keep, Qc, Kc, Vc):
    _check(load_library().tsa_compress(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(V), _ptr(idx), k_keep,
                                       _ptr(Qc), _ptr(Kc), _ptr(Vc), _stream()))


def tsa_attend_workspace_bytes(desc, Lc, kv_heads):
    return int(load_library().tsa_attend_workspace_bytes(ctypes.byref(desc), Lc, kv_heads))


def tsa_attend(desc, Qc, Kc, Vc, Lc, kv_heads, Oc, ws, lse=None, block_list=None, block_size=0, max_blocks_per_row=0):
    p, n = _ws(ws)
    _check(load_library().tsa_attend(ctypes.byref(desc), _ptr(Qc), _ptr(Kc), _ptr(Vc), Lc, kv_heads,
                                     _ptr(block_list), block_size, max_blocks_per_row, _ptr(Oc), _ptr(lse),
                                     p, n, _stream()))


def tsa_decompress(desc, Oc, idx, inv, k_keep, O=None, residual=None):
    _check(load_library().tsa_decompress(ctypes.byref(desc), _ptr(Oc), _ptr(idx), _ptr(inv), k_keep,
                                         _ptr(O), _ptr(residual), _stream()))


def tsa_compress_v_tiles(desc, V, idx, k_keep, Vt):
    p, n = _ws(Vt)
    _check(load_library().tsa_compress_v_tiles(ctypes.byref(desc), _ptr(V), _ptr(idx), k_keep, p, n, _stream()))


def tsa_attend_fused(desc, Q, K, Vt, idx, inv, k_keep, O=None, Oc=None, residual=None,
                     block_list=None, block_size=0, max_blocks_per_row=0):
    _check(load_library().tsa_attend_fused(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(Vt), _ptr(idx), _ptr(inv), k_keep,
                                           _ptr(block_list), block_size, max_blocks_per_row, _ptr(O), _ptr(Oc),
                                           _ptr(residual), _stream()))


def alloc_forward_dynamic_workspace(desc, k_max, device="cuda"):
    """Device buffer of tsa_forward_dynamic_workspace_bytes() bytes."""
    n = load_library().tsa_forward_dynamic_workspace_bytes(ctypes.byref(desc), k_max)
    if n == 0:
        raise TsaError(TSA_ERR_ARG, tsa_last_error())
    return torch.empty(n, dtype=torch.uint8, device=device)


def tsa_forward_dynamic(desc, Q, K, V, tau_cov, k_max, O, ws, residual=None, k_keep_out=None, idx_out=None,
                        block_list=None, block_size=0, max_blocks_per_row=0):
    p, n = _ws(ws)
    _check(load_library().tsa_forward_dynamic(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(V), float(tau_cov), k_max,
                                              _ptr(block_list), block_size, max_blocks_per_row,
                                              _ptr(O), _ptr(residual), _ptr(k_keep_out), _ptr(idx_out), p, n, _stream()))


def tsa_forward(desc, Q, K, V, k_keep, O, ws, residual=None, idx_out=None,
                block_list=None, block_size=0, max_blocks_per_row=0):
    p, n = _ws(ws)
    _check(load_library().tsa_forward(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(V), k_keep,
                                      _ptr(block_list), block_size, max_blocks_per_row,
                                      _ptr(O), _ptr(residual), _ptr(idx_out), p, n, _stream()))


def tsa_layer_drift(h_in, h_out, eps, drift_out, ws=None):
    """h_in, h_out [n_tokens, width] bf16 CUDA tensors; drift_out: 1-element fp32 CUDA tensor."""
    n_tokens, width = h_in.shape
    if ws is None:
        ws = torch.empty(load_library().tsa_layer_drift_workspace_bytes(n_tokens), dtype=torch.uint8, device=h_in.device)
    p, n = _ws(ws)
    _check(load_library().tsa_layer_drift(_ptr(h_in), _ptr(h_out), n_tokens, width, eps, _ptr(drift_out), p, n, _stream()))


def tsa_sparse_layers(drift, delta=0.5):
    """Eq. 2 on the host: list of 0/1 flags, 1 = layer is eligible for Token Sparse Attention."""
    n = len(drift)
    arr = (ctypes.c_float * n)(*[float(v) for v in drift])
    out = (ctypes.c_int32 * n)()
    _check(load_library().tsa_sparse_layers(arr, n, float(delta), out))
    return list(out)


# The handle of a device's current stream without the Python object around it, which costs 2.6 us of a call's 10.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _queue():
    """(handle of the current stream, current device)"""
    try:
        dev = torch.cuda.current_device()
        return _raw_stream(dev), dev
    except (RuntimeError, AssertionError) as e:             # no GPU
        raise TsaError(TSA_ERR_HIP, str(e)) from None


_BF16, _I32, _U8, _F32 = (torch.bfloat16,), (torch.int32,), (torch.uint8,), (torch.float32,)


def _view(t, dev, dtypes, shape, name, strides=None):
    """Address of a tensor that has to be on device `dev`, of one of these types and of this shape.  strides: element strides of all axes
    but the last, as the descriptor has them (None or zeros: contiguous); the tensor's own have to be the same."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise TsaError(TSA_ERR_ARG, "%s is not on the current GPU" % name)
    if t.dtype not in dtypes:
        raise TsaError(TSA_ERR_ARG, "%s is %s" % (name, t.dtype))
    if t.shape != shape:
        raise TsaError(TSA_ERR_ARG, "%s is %s, not %s" % (name, tuple(t.shape), shape))
    if strides is None or not any(strides):
        if not t.is_contiguous():
            raise TsaError(TSA_ERR_ARG, "%s is not contiguous" % name)
    elif t.stride() != (*strides, 1) and any(n > 1 and x != y for n, x, y in zip(shape, t.stride(), (*strides, 1))):
        raise TsaError(TSA_ERR_ARG, "%s has strides %s, the descriptor %s" % (name, t.stride(), tuple(strides)))
    return t.data_ptr()


def tsa_rotary_frequencies(kind, rot, base, factor=1.0, original=0.0, high=0.0, low=0.0):
    """(frequencies, gain) for make_rotary_desc."""
    freq, gain = (ctypes.c_double * max(1, rot // 2))(), ctypes.c_float()
    _check(load_library().tsa_rotary_frequencies(kind, rot, base, factor, original, high, low, freq, ctypes.byref(gain)))
    return list(freq), gain.value


def tsa_rotary(desc, Q, K, Q_out, K_out, positions=None):
    """Q [B,Hq,L,d], K [B,Hkv,L,d] and their outputs: bf16 tensors or views with the descriptor's strides; positions int32 [B,L]."""
    st, dev = _queue()
    B, L, d = desc.B, desc.L, desc.d
    q, k = (B, desc.Hq, L, d), (B, desc.Hkv, L, d)
    _check(load_library().tsa_rotary(
        ctypes.byref(desc), _view(Q, dev, _BF16, q, "Q", (desc.q_stride_b, desc.q_stride_h, desc.q_stride_l)),
        _view(K, dev, _BF16, k, "K", (desc.k_stride_b, desc.k_stride_h, desc.k_stride_l)), _view(positions, dev, _I32, (B, L), "positions"),
        _view(Q_out, dev, _BF16, q, "Q_out", (desc.q_out_stride_b, desc.q_out_stride_h, desc.q_out_stride_l)),
        _view(K_out, dev, _BF16, k, "K_out", (desc.k_out_stride_b, desc.k_out_stride_h, desc.k_out_stride_l)), st))


_POOL_TYPES = {TSA_CACHE_BF16: (torch.bfloat16,), TSA_CACHE_E4M3: (torch.uint8, torch.float8_e4m3fn)}


def _cache(desc, dev, k_pages, v_pages, k_scales, v_scales):
    shape = (desc.n_pages, desc.Hkv, desc.page_size, desc.d)
    kind = _POOL_TYPES.get(desc.format, ())
    return (_view(k_pages, dev, kind, shape, "k_pages"), _view(v_pages, dev, kind, shape, "v_pages"),
            _view(k_scales, dev, _U8, shape[:3], "k_scales"), _view(v_scales, dev, _U8, shape[:3], "v_scales"))


def _lengths(desc, dev, kv_len, page_table):
    n = desc.n_seqs
    return _view(kv_len, dev, _I32, (n,), "kv_len"), _view(page_table, dev, _I32, (n, desc.max_pages), "page_table")


def tsa_cache_write(desc, K, V, cu_q, kv_len, page_table, k_pages, v_pages, k_scales=None, v_scales=None):
    """K, V [n_tokens,Hkv,d] bf16 (views with the descriptor's strides); pools bf16, or uint8 / float8_e4m3fn with uint8 scales."""
    st, dev = _queue()
    rows = (desc.n_tokens, desc.Hkv, desc.d)
    _check(load_library().tsa_cache_write(
        ctypes.byref(desc), _view(K, dev, _BF16, rows, "K", (desc.k_stride_t, desc.k_stride_h)),
        _view(V, dev, _BF16, rows, "V", (desc.v_stride_t, desc.v_stride_h)), _view(cu_q, dev, _I32, (desc.n_seqs + 1,), "cu_q"),
        *_lengths(desc, dev, kv_len, page_table), *_cache(desc, dev, k_pages, v_pages, k_scales, v_scales), st))


def tsa_cache_read(desc, k_pages, v_pages, kv_len, page_table, L, K, V, k_scales=None, v_scales=None):
    """K, V [n_seqs,Hkv,L,d] bf16, contiguous: the first L positions of every sequence."""
    st, dev = _queue()
    shape = (desc.n_seqs, desc.Hkv, L, desc.d)
    _check(load_library().tsa_cache_read(ctypes.byref(desc), *_cache(desc, dev, k_pages, v_pages, k_scales, v_scales),
                                         *_lengths(desc, dev, kv_len, page_table), L, _view(K, dev, _BF16, shape, "K"),
                                         _view(V, dev, _BF16, shape, "V"), st))


def alloc_attend_cache_workspace(desc, device="cuda"):
    """Device buffer of tsa_attend_cache_workspace_bytes() bytes."""
    n = load_library().tsa_attend_cache_workspace_bytes(ctypes.byref(desc))
    if n == 0:
        raise TsaError(TSA_ERR_ARG, tsa_last_error())
    return torch.empty(n, dtype=torch.uint8, device=device)


def tsa_attend_cache(desc, Q, k_pages, v_pages, cu_q, kv_len, page_table, O, ws, lse=None, k_scales=None, v_scales=None):
    """Q, O [n_tokens,Hq,d] bf16 (views with the descriptor's strides), lse [n_tokens,Hq] fp32 or None; pools as in tsa_cache_write."""
    st, dev = _queue()
    rows = (desc.n_tokens, desc.Hq, desc.d)
    _check(load_library().tsa_attend_cache(
        ctypes.byref(desc), _view(Q, dev, _BF16, rows, "Q", (desc.q_stride_t, desc.q_stride_h)), *_cache(desc, dev, k_pages, v_pages, k_scales, v_scales),
        _view(cu_q, dev, _I32, (desc.n_seqs + 1,), "cu_q"), *_lengths(desc, dev, kv_len, page_table),
        _view(O, dev, _BF16, rows, "O", (desc.o_stride_t, desc.o_stride_h)), _view(lse, dev, _F32, rows[:2], "lse"),
        _view(ws, dev, _U8, ws.shape, "ws"), ws.numel(), st))


def tsa_mfma_probe(operands, iters, blocks, sink, clocks):
    """Queues the bare MFMA loop; returns (flops of the launch, wall clock rate in kHz)."""
    flops, khz = ctypes.c_double(0.0), ctypes.c_int32(0)
    _check(load_library().tsa_mfma_probe(_ptr(operands), iters, blocks, _ptr(sink), _ptr(clocks),
                                         ctypes.byref(flops), ctypes.byref(khz), _stream()))
    return flops.value, khz.value


def tsa_mix_probe(mix, operands, iters, blocks, sink):
    """Queues the instruction-mix loop `mix` (0..3); returns the flops of the launch's MFMAs."""
    flops = ctypes.c_double(0.0)
    _check(load_library().tsa_mix_probe(mix, _ptr(operands), iters, blocks, _ptr(sink), ctypes.byref(flops), _stream()))
    return flops.value


def tsa_read_probe(src, sink):
    """Queues the streaming read of src (byte size a multiple of 16); sink: a device tensor of at least 4 bytes."""
    _check(load_library().tsa_read_probe(_ptr(src), src.numel() * src.element_size(), _ptr(sink), _stream()))


def tsa_bench_set_attend_form(form: int):
    _check(load_library().tsa_bench_set_attend_form(form))


def tsa_copy_probe(src, dst):
    """Queues the streaming copy dst = src (same byte size, a multiple of 16)."""
    nbytes = src.numel() * src.element_size()
    if nbytes != dst.numel() * dst.element_size():
        raise TsaError(TSA_ERR_ARG, "src and dst differ in size")
    _check(load_library().tsa_copy_probe(_ptr(src), _ptr(dst), nbytes, _stream()))


def alloc_attend_workspace(desc, Lc, kv_heads, device="cuda"):
    n = tsa_attend_workspace_bytes(desc, Lc, kv_heads)
    if n == 0:
        raise TsaError(TSA_ERR_ARG, tsa_last_error())
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_workspace(desc, k_keep, device="cuda"):
    """Device buffer of tsa_workspace_bytes() bytes (torch allocations are 256-byte aligned)."""
    n = tsa_workspace_bytes(desc, k_keep)
    if n == 0:
        raise TsaError(TSA_ERR_ARG, tsa_last_error())
    return torch.empty(n, dtype=torch.uint8, device=device)
