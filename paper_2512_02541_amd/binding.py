"""ctypes binding of libagg.so: same names as the C ABI in ``include/agg.h``.

Argument marshalling only -- every step of the path runs in the library's HIP
kernels.  PyTorch supplies device memory (``tensor.data_ptr()``) and the HIP
stream.  A missing library is an error: there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
# AGG_LIBRARY_PATH points at another build of the same library (kernel development)
LIB_PATH = os.environ.get("AGG_LIBRARY_PATH") or os.path.join(_HERE, "libagg.so")

AGG_DIAG = 1
AGG_MEAN = 2
AGG_OK = 0
AGG_ERR_NULL, AGG_ERR_SHAPE, AGG_ERR_UNSUPPORTED, AGG_ERR_ALIGN = -1, -2, -3, -4
AGG_ERR_WORKSPACE, AGG_ERR_OVERFLOW, AGG_ERR_LAUNCH = -5, -6, -7


class AggError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, status_string(status), status))


class agg_shape(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("N", ctypes.c_int32),
        ("n_h", ctypes.c_int32), ("n_w", ctypes.c_int32),
        ("n_special", ctypes.c_int32),
        ("H", ctypes.c_int32), ("D", ctypes.c_int32),
        ("s_h", ctypes.c_int32), ("s_w", ctypes.c_int32),
        ("keep_first_frame", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
        ("scale", ctypes.c_float),
        ("mean_logit_bias", ctypes.c_float),
    ]

    @property
    def L(self) -> int:
        return self.n_special + self.n_h * self.n_w

    @property
    def NQ(self) -> int:
        return self.N * self.L


def make_shape(B, N, n_h, n_w, n_special, H, D, s_h, s_w, keep_first_frame=1,
               flags=AGG_DIAG | AGG_MEAN, scale=None, mean_logit_bias=0.0) -> agg_shape:
    if scale is None:
        scale = 1.0 / (D ** 0.5)
    return agg_shape(B, N, n_h, n_w, n_special, H, D, s_h, s_w, keep_first_frame, flags, scale,
                     mean_logit_bias)


_lib = None
_raw_stream = _initialized = _device = None

EXPORTS = [
    "agg_status_string", "agg_sigma_to_strides", "agg_kv_count", "agg_kv_indices_host",
    "agg_dropped_indices_host", "agg_kv_compact_bytes", "agg_kc_offset", "agg_vc_offset", "agg_workspace_bytes",
    "agg_kv_subsample", "agg_global_attn_fwd", "agg_global_attn_fwd_idx",
    "agg_dense_global_attn_fwd", "agg_frame_attn_fwd",
    "agg_block_workspace_bytes", "agg_global_block_fwd",
    "agg_select_kv_indices", "agg_list_compact_bytes", "agg_list_workspace_bytes",
    "agg_kv_subsample_list", "agg_global_attn_fwd_list", "agg_kv_pool",
    "agg_static_scratch_bytes", "agg_kv_subsample_static",
    "agg_rope_fwd", "agg_residual_norm_fwd",
    "agg_mx4_code_stride", "agg_mx4_scale_stride", "agg_mx4_quantize", "agg_mx4_dequantize",
    "agg_mx4_linear_fwd", "agg_block_ex_workspace_bytes", "agg_global_block_ex_fwd",
]

AGG_SELECT_FIRST = 0
AGG_SELECT_RANDOM = 1
AGG_SELECT_HIGH = 2
AGG_SELECT_LOW = 3

AGG_BLOCK_SGA = 0
AGG_BLOCK_FRAME = 1
AGG_BLOCK_DENSE = 2


class agg_block_weights(ctypes.Structure):
    _fields_ = [
        ("ln_gamma", ctypes.c_void_p), ("ln_beta", ctypes.c_void_p), ("ln_eps", ctypes.c_float),
        ("w_q", ctypes.c_void_p), ("w_k", ctypes.c_void_p), ("w_v", ctypes.c_void_p),
        ("w_o", ctypes.c_void_p),
        ("b_q", ctypes.c_void_p), ("b_k", ctypes.c_void_p), ("b_v", ctypes.c_void_p),
        ("b_o", ctypes.c_void_p),
    ]


def make_block_weights(ln_gamma, ln_beta, ln_eps, w_q, w_k, w_v, w_o, b_q=None, b_k=None,
                       b_v=None, b_o=None) -> agg_block_weights:
    """Packs device tensors (kept alive by the caller) into the C struct."""
    def p(t):
        return None if t is None else t.data_ptr()
    return agg_block_weights(p(ln_gamma), p(ln_beta), float(ln_eps), p(w_q), p(w_k), p(w_v),
                             p(w_o), p(b_q), p(b_k), p(b_v), p(b_o))


AGG_NORM_NONE = 0
AGG_NORM_LAYER = 1
AGG_NORM_RMS = 2

AGG_ROPE_SECTIONS = 0
AGG_ROPE_NEIGHBOURS = 1
AGG_ROPE_HEAD = 2


class agg_norm(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("eps", ctypes.c_float), ("gamma", ctypes.c_void_p),
                ("beta", ctypes.c_void_p)]


class agg_rope(ctypes.Structure):
    _fields_ = [("pairing", ctypes.c_int32), ("d_t", ctypes.c_int32), ("d_h", ctypes.c_int32),
                ("d_w", ctypes.c_int32), ("t0", ctypes.c_int32), ("patch0", ctypes.c_int32),
                ("base", ctypes.c_float)]


class agg_residual(ctypes.Structure):
    _fields_ = [("post", agg_norm), ("pre", agg_norm), ("scale", ctypes.c_void_p),
                ("gate", ctypes.c_void_p), ("gate_rows", ctypes.c_int64)]


class agg_mx4_matrix(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


class agg_mx4_linear(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int32), ("w", agg_mx4_matrix * 3), ("bias", ctypes.c_void_p * 3),
                ("y", ctypes.c_void_p * 3), ("residual", ctypes.c_void_p), ("res_scale", ctypes.c_void_p)]


class agg_block_options(ctypes.Structure):
    _fields_ = [("rope", ctypes.POINTER(agg_rope)), ("pos", ctypes.c_void_p), ("q_norm", agg_norm),
                ("k_norm", agg_norm), ("residual", agg_residual), ("first_done", ctypes.c_int32),
                ("x_norm", ctypes.c_void_p), ("mx", ctypes.POINTER(agg_mx4_matrix))]


# The structs below hold on to the tensors whose addresses they carry.
def make_norm(kind=AGG_NORM_NONE, eps=1e-5, gamma=None, beta=None) -> agg_norm:
    n = agg_norm(int(kind), float(eps), _ptr(gamma), _ptr(beta))
    n.keep = (gamma, beta)
    return n


def make_rope(pairing, d_t, d_h, d_w, base=100.0, t0=0, patch0=0) -> agg_rope:
    return agg_rope(int(pairing), int(d_t), int(d_h), int(d_w), int(t0), int(patch0), float(base))


def make_residual(post=None, pre=None, scale=None, gate=None, gate_rows=0) -> agg_residual:
    post, pre = post or agg_norm(), pre or agg_norm()
    r = agg_residual(post, pre, _ptr(scale), _ptr(gate), int(gate_rows))
    r.keep = (post, pre, scale, gate)
    return r


def make_mx4_linear(weights, outs, biases=None, residual=None, res_scale=None) -> agg_mx4_linear:
    """weights: one to three (codes, scales), outs as many tensors, biases as many (None: none)."""
    weights, outs = list(weights), list(outs)
    biases = list(biases) if biases is not None else [None] * len(weights)
    if not 1 <= len(weights) <= 3 or len(outs) != len(weights) or len(biases) != len(weights):
        raise ValueError("one to three weights, and as many outputs and biases")
    m = agg_mx4_linear()
    m.count = len(weights)
    for i, (codes, scales) in enumerate(weights):
        m.w[i] = agg_mx4_matrix(_ptr(codes), _ptr(scales))
        m.bias[i], m.y[i] = _ptr(biases[i]), _ptr(outs[i])
    m.residual, m.res_scale = _ptr(residual), _ptr(res_scale)
    m.keep = (weights, outs, biases, residual, res_scale)
    return m


def make_block_options(rope=None, pos=None, q_norm=None, k_norm=None, residual=None, x_norm=None,
                       mx=None) -> agg_block_options:
    """x_norm given: the first norm is done.  mx: (codes, scales) of the q, k, v and o matrices."""
    o = agg_block_options()
    if rope is not None:
        o.rope = ctypes.pointer(rope)
    o.pos = _ptr(pos)
    for name, value in (("q_norm", q_norm), ("k_norm", k_norm), ("residual", residual)):
        if value is not None:
            setattr(o, name, value)
    o.first_done, o.x_norm = int(x_norm is not None), _ptr(x_norm)
    if mx is not None:
        mx = list(mx)
        if len(mx) != 4:
            raise ValueError("four matrices: q, k, v, o")
        held = (agg_mx4_matrix * 4)(*[agg_mx4_matrix(_ptr(c), _ptr(s)) for c, s in mx])
        o.mx = ctypes.cast(held, ctypes.POINTER(agg_mx4_matrix))
    else:
        held = None
    o.keep = (rope, pos, q_norm, k_norm, residual, x_norm, mx, held)
    return o


def lib():
    """Opens libagg.so on first use; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "libagg.so is missing at %s -- build it with `python -m paper_2512_02541_amd.build`; "
            "there is no fallback path" % LIB_PATH)
    # PyTorch owns the device memory and streams handed to the library, so the library must
    # bind to the HIP runtime PyTorch ships: load torch (and with it that runtime) first.
    import torch  # noqa: F401

    L = ctypes.CDLL(LIB_PATH)
    vp, i32p, i64p = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int64)
    shp = ctypes.POINTER(agg_shape)
    L.agg_status_string.restype = ctypes.c_char_p
    L.agg_status_string.argtypes = [ctypes.c_int]
    L.agg_sigma_to_strides.argtypes = [ctypes.c_int, i32p, i32p]
    L.agg_kv_count.argtypes = [shp, i64p, i64p]
    L.agg_kv_indices_host.argtypes = [shp, vp]
    L.agg_dropped_indices_host.argtypes = [shp, vp]
    L.agg_kv_compact_bytes.argtypes = [shp, ctypes.POINTER(ctypes.c_size_t), i64p]
    L.agg_kc_offset.restype = ctypes.c_int64
    L.agg_kc_offset.argtypes = [ctypes.c_int64, ctypes.c_int32]
    L.agg_vc_offset.restype = ctypes.c_int64
    L.agg_vc_offset.argtypes = [ctypes.c_int64, ctypes.c_int32]
    L.agg_workspace_bytes.restype = ctypes.c_size_t
    L.agg_workspace_bytes.argtypes = [shp]
    L.agg_kv_subsample.argtypes = [shp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.agg_global_attn_fwd.argtypes = [shp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.agg_global_attn_fwd_idx.argtypes = [shp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.agg_dense_global_attn_fwd.argtypes = [shp, vp, vp, vp, vp, vp, vp]
    L.agg_frame_attn_fwd.argtypes = [shp, vp, vp, vp, vp, vp, vp]
    L.agg_block_workspace_bytes.restype = ctypes.c_size_t
    L.agg_block_workspace_bytes.argtypes = [shp, ctypes.c_int]
    L.agg_global_block_fwd.argtypes = [shp, ctypes.c_int, ctypes.POINTER(agg_block_weights), vp, vp,
                                       vp, ctypes.c_size_t, vp]
    L.agg_select_kv_indices.argtypes = [shp, ctypes.c_int, ctypes.c_uint64, vp, vp, vp]
    L.agg_list_compact_bytes.argtypes = [shp, ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t), i64p]
    L.agg_list_workspace_bytes.restype = ctypes.c_size_t
    L.agg_list_workspace_bytes.argtypes = [shp]
    L.agg_kv_subsample_list.argtypes = [shp, vp, ctypes.c_int64, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                        ctypes.c_size_t, vp]
    L.agg_global_attn_fwd_list.argtypes = [shp, ctypes.c_int64, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                           vp, vp, vp]
    L.agg_kv_pool.argtypes = [shp, vp, vp, vp, vp, vp]
    L.agg_static_scratch_bytes.restype = ctypes.c_size_t
    L.agg_static_scratch_bytes.argtypes = []
    L.agg_kv_subsample_static.argtypes = [shp, vp, vp, vp, vp, vp, vp, vp, vp]
    normp, i64 = ctypes.POINTER(agg_norm), ctypes.c_int64
    L.agg_rope_fwd.argtypes = [shp, ctypes.POINTER(agg_rope), normp, normp, vp, vp, i64, vp, i64, vp, vp, vp]
    L.agg_residual_norm_fwd.argtypes = [i64, ctypes.c_int32, ctypes.POINTER(agg_residual), vp, vp, vp, vp, vp]
    for fn in (L.agg_mx4_code_stride, L.agg_mx4_scale_stride):
        fn.restype, fn.argtypes = i64, [ctypes.c_int32]
    L.agg_mx4_quantize.argtypes = [i64, ctypes.c_int32, vp, i64, vp, vp, vp]
    L.agg_mx4_dequantize.argtypes = [i64, ctypes.c_int32, vp, vp, vp, vp]
    L.agg_mx4_linear_fwd.argtypes = [i64, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(agg_mx4_linear),
                                     vp, vp, vp]
    opts = ctypes.POINTER(agg_block_options)
    L.agg_block_ex_workspace_bytes.restype = ctypes.c_size_t
    L.agg_block_ex_workspace_bytes.argtypes = [shp, ctypes.c_int, opts]
    L.agg_global_block_ex_fwd.argtypes = [shp, ctypes.c_int, ctypes.POINTER(agg_block_weights), opts, vp, vp, vp,
                                          vp, ctypes.c_size_t, vp]
    global _raw_stream, _initialized, _device
    # the current stream's handle without building a Stream object for it (3 us a call)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _initialized = torch.cuda.is_initialized
    # (what torch.cuda.current_device asks once CUDA is initialised, which _stream sees to)
    _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _lib = L
    return L


def _check(status: int, where: str):
    if status != AGG_OK:
        raise AggError(status, where)


def _ptr(t):
    """Device (or host) address of a torch tensor / numpy array / raw int / None, as the plain
    number that the declared argument types take (a ctypes object per argument cost as much as the
    call itself)."""
    if t is None or isinstance(t, int):
        return t
    address = getattr(t, "data_ptr", None)
    return t.ctypes.data if address is None else address()


def _stream(stream):
    """Handle of `stream`, by default of the current device's current stream."""
    if stream is not None:
        return int(stream)
    if _raw_stream is not None and _initialized():
        return _raw_stream(_device())
    import torch

    return torch.cuda.current_stream().cuda_stream


def status_string(status: int) -> str:
    return lib().agg_status_string(int(status)).decode()


def agg_sigma_to_strides(sigma: int):
    sh, sw = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().agg_sigma_to_strides(int(sigma), ctypes.byref(sh), ctypes.byref(sw)),
           "agg_sigma_to_strides")
    return sh.value, sw.value


def agg_kv_count(shape: agg_shape):
    m, nd = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(lib().agg_kv_count(ctypes.byref(shape), ctypes.byref(m), ctypes.byref(nd)),
           "agg_kv_count")
    return m.value, nd.value


def agg_kv_indices_host(shape: agg_shape):
    import numpy as np

    m, _ = agg_kv_count(shape)
    idx = np.empty(m, dtype=np.int32)
    _check(lib().agg_kv_indices_host(ctypes.byref(shape), _ptr(idx)), "agg_kv_indices_host")
    return idx


def agg_dropped_indices_host(shape: agg_shape):
    import numpy as np

    _, nd = agg_kv_count(shape)
    idx = np.empty(nd, dtype=np.int32)
    _check(lib().agg_dropped_indices_host(ctypes.byref(shape), _ptr(idx)),
           "agg_dropped_indices_host")
    return idx


def agg_kv_compact_bytes(shape: agg_shape):
    nbytes, m_pad = ctypes.c_size_t(0), ctypes.c_int64(0)
    _check(lib().agg_kv_compact_bytes(ctypes.byref(shape), ctypes.byref(nbytes),
                                      ctypes.byref(m_pad)), "agg_kv_compact_bytes")
    return nbytes.value, m_pad.value


def agg_kc_offset(m: int, d: int) -> int:
    return int(lib().agg_kc_offset(int(m), int(d)))


def agg_vc_offset(m: int, d: int) -> int:
    return int(lib().agg_vc_offset(int(m), int(d)))


def agg_workspace_bytes(shape: agg_shape) -> int:
    return int(lib().agg_workspace_bytes(ctypes.byref(shape)))


def agg_kv_subsample(shape, K, V, Kc, Vc, idx, kmean, vmean, workspace, workspace_bytes,
                     stream=None):
    _check(lib().agg_kv_subsample(ctypes.byref(shape), _ptr(K), _ptr(V), _ptr(Kc), _ptr(Vc),
                                  _ptr(idx), _ptr(kmean), _ptr(vmean), _ptr(workspace),
                                  int(workspace_bytes), _stream(stream)), "agg_kv_subsample")


def agg_static_scratch_bytes() -> int:
    return int(lib().agg_static_scratch_bytes())


def agg_kv_subsample_static(shape, K, V, Kc, Vc, idx, kmean, vmean, stream=None):
    _check(lib().agg_kv_subsample_static(ctypes.byref(shape), _ptr(K), _ptr(V), _ptr(Kc), _ptr(Vc),
                                         _ptr(idx), _ptr(kmean), _ptr(vmean), _stream(stream)),
           "agg_kv_subsample_static")


def agg_global_attn_fwd(shape, Q, K, V, Kc, Vc, kmean, vmean, O, lse=None, stream=None):
    _check(lib().agg_global_attn_fwd(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), _ptr(Kc),
                                     _ptr(Vc), _ptr(kmean), _ptr(vmean), _ptr(O), _ptr(lse),
                                     _stream(stream)), "agg_global_attn_fwd")


def agg_global_attn_fwd_idx(shape, Q, K, V, idx, kmean, vmean, O, lse=None, stream=None):
    _check(lib().agg_global_attn_fwd_idx(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), _ptr(idx),
                                         _ptr(kmean), _ptr(vmean), _ptr(O), _ptr(lse),
                                         _stream(stream)), "agg_global_attn_fwd_idx")


def agg_dense_global_attn_fwd(shape, Q, K, V, O, lse=None, stream=None):
    _check(lib().agg_dense_global_attn_fwd(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), _ptr(O),
                                           _ptr(lse), _stream(stream)), "agg_dense_global_attn_fwd")


def agg_frame_attn_fwd(shape, Q, K, V, O, lse=None, stream=None):
    _check(lib().agg_frame_attn_fwd(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), _ptr(O),
                                    _ptr(lse), _stream(stream)), "agg_frame_attn_fwd")


def agg_block_workspace_bytes(shape: agg_shape, mode: int) -> int:
    return int(lib().agg_block_workspace_bytes(ctypes.byref(shape), int(mode)))


def agg_global_block_fwd(shape, mode, weights, x, y, workspace, workspace_bytes, stream=None):
    _check(lib().agg_global_block_fwd(ctypes.byref(shape), int(mode), ctypes.byref(weights),
                                      _ptr(x), _ptr(y), _ptr(workspace), int(workspace_bytes),
                                      _stream(stream)), "agg_global_block_fwd")


def agg_select_kv_indices(shape, rule, seed, K, list_out, stream=None):
    _check(lib().agg_select_kv_indices(ctypes.byref(shape), int(rule), int(seed), _ptr(K),
                                       _ptr(list_out), _stream(stream)), "agg_select_kv_indices")


def agg_list_compact_bytes(shape: agg_shape, M_list: int):
    nbytes, m_pad = ctypes.c_size_t(0), ctypes.c_int64(0)
    _check(lib().agg_list_compact_bytes(ctypes.byref(shape), int(M_list), ctypes.byref(nbytes),
                                        ctypes.byref(m_pad)), "agg_list_compact_bytes")
    return nbytes.value, m_pad.value


def agg_list_workspace_bytes(shape: agg_shape) -> int:
    return int(lib().agg_list_workspace_bytes(ctypes.byref(shape)))


def agg_kv_subsample_list(shape, list_in, M_list, K, V, Kc, Vc, kmean, vmean, kept_bits, n_dropped,
                          workspace, workspace_bytes, stream=None):
    _check(lib().agg_kv_subsample_list(ctypes.byref(shape), _ptr(list_in), int(M_list), _ptr(K),
                                       _ptr(V), _ptr(Kc), _ptr(Vc), _ptr(kmean), _ptr(vmean),
                                       _ptr(kept_bits), _ptr(n_dropped), _ptr(workspace),
                                       int(workspace_bytes), _stream(stream)),
           "agg_kv_subsample_list")


def agg_global_attn_fwd_list(shape, M_list, Q, K, V, Kc, Vc, kmean, vmean, kept_bits, n_dropped, O,
                             lse=None, stream=None):
    _check(lib().agg_global_attn_fwd_list(ctypes.byref(shape), int(M_list), _ptr(Q), _ptr(K),
                                          _ptr(V), _ptr(Kc), _ptr(Vc), _ptr(kmean), _ptr(vmean),
                                          _ptr(kept_bits), _ptr(n_dropped), _ptr(O), _ptr(lse),
                                          _stream(stream)), "agg_global_attn_fwd_list")


def agg_kv_pool(shape, K, V, Kc, Vc, stream=None):
    _check(lib().agg_kv_pool(ctypes.byref(shape), _ptr(K), _ptr(V), _ptr(Kc), _ptr(Vc),
                             _stream(stream)), "agg_kv_pool")


def _ref(struct):
    return None if struct is None else ctypes.byref(struct)


def agg_rope_fwd(shape, rope, q_norm, k_norm, pos, Q, q_stride, K, k_stride, Qr, Kr, stream=None):
    _check(lib().agg_rope_fwd(ctypes.byref(shape), _ref(rope), _ref(q_norm), _ref(k_norm), _ptr(pos),
                              _ptr(Q), int(q_stride), _ptr(K), int(k_stride), _ptr(Qr), _ptr(Kr),
                              _stream(stream)), "agg_rope_fwd")


def agg_residual_norm_fwd(rows, C, residual, x, branch, h, n, stream=None):
    _check(lib().agg_residual_norm_fwd(int(rows), int(C), ctypes.byref(residual), _ptr(x), _ptr(branch),
                                       _ptr(h), _ptr(n), _stream(stream)), "agg_residual_norm_fwd")


def agg_mx4_code_stride(K: int) -> int:
    return int(lib().agg_mx4_code_stride(int(K)))


def agg_mx4_scale_stride(K: int) -> int:
    return int(lib().agg_mx4_scale_stride(int(K)))


def agg_mx4_quantize(rows, K, x, x_stride, codes, scales, stream=None):
    _check(lib().agg_mx4_quantize(int(rows), int(K), _ptr(x), int(x_stride), _ptr(codes), _ptr(scales),
                                  _stream(stream)), "agg_mx4_quantize")


def agg_mx4_dequantize(rows, K, codes, scales, x, stream=None):
    _check(lib().agg_mx4_dequantize(int(rows), int(K), _ptr(codes), _ptr(scales), _ptr(x),
                                    _stream(stream)), "agg_mx4_dequantize")


def agg_mx4_linear_fwd(rows, N, K, linear, codes, scales, stream=None):
    _check(lib().agg_mx4_linear_fwd(int(rows), int(N), int(K), ctypes.byref(linear), _ptr(codes),
                                    _ptr(scales), _stream(stream)), "agg_mx4_linear_fwd")


def agg_block_ex_workspace_bytes(shape: agg_shape, mode: int, options: agg_block_options) -> int:
    return int(lib().agg_block_ex_workspace_bytes(ctypes.byref(shape), int(mode), ctypes.byref(options)))


def agg_global_block_ex_fwd(shape, mode, weights, options, x, y, n, workspace, workspace_bytes, stream=None):
    _check(lib().agg_global_block_ex_fwd(ctypes.byref(shape), int(mode), ctypes.byref(weights),
                                         ctypes.byref(options), _ptr(x), _ptr(y), _ptr(n), _ptr(workspace),
                                         int(workspace_bytes), _stream(stream)), "agg_global_block_ex_fwd")
