"""ctypes binding of include/quantpipe.h: same names, argument marshalling only.

torch is used for device memory and streams: tensors give `data_ptr()`, the current torch
stream gives the hipStream_t.  torch is imported before the library is loaded so that the
library binds to the HIP runtime already in the process.
"""
from __future__ import annotations

import ctypes as C
import os

import torch  # noqa: F401  (must precede CDLL: one HIP runtime per process)

__all__ = [
    "QP_OK", "QP_EINVAL", "QP_ENOSPC", "QP_EHIP", "QP_ENONFINITE", "QP_F32", "QP_BF16", "QP_LAPLACE", "QP_GAUSS", "QP_DIST_AUTO", "QP_WS_MODEL", "qp_model_fit_t", "qp_model_fit", "qp_model_fit_async", "qp_job_t", "qp_lane_t",
    "QP_SEARCH_CLIP_TO_DATA", "QP_SEARCH_COARSE_TO_FINE", "QP_SEARCH_LOW_BITS_ONLY",
    "QP_WS_STATS", "QP_WS_RESULT", "QP_WS_QPARAMS", "QP_WS_HIST", "QP_WS_CANDS", "QP_WS_SCORES",
    "qp_stats_t", "qp_qparams_t", "qp_search_cfg_t", "qp_search_result_t", "qp_controller_t", "QuantPipeError", "BITS",
    "lib", "qp_packed_bytes", "qp_workspace_bytes", "qp_ws_offset", "qp_default_search_cfg", "qp_stats",
    "qp_stats_async", "qp_aciq_alpha", "qp_aciq_constant", "qp_make_qparams", "qp_make_qparams_clipped", "qp_dsaciq_search",
    "qp_dsaciq_search_async", "qp_dsaciq_hist_search", "qp_dsaciq_hist_search_async", "qp_quant_pack", "qp_quant_pack_dev", "qp_unpack_dequant", "qp_unpack_dequant_dev",
    "qp_compress_async", "qp_compress_many_async", "qp_compress_noalloc", "qp_next_bits", "qp_controller_init", "qp_controller_update", "qp_strerror",
    "QP_KV_POOL_HEADER", "qp_kv_cache_t", "qp_kv_rows_t", "qp_kv_view_t", "qp_kv_attn_cfg_t", "kv_cache", "kv_rows", "alloc_kv_pages", "alloc_kv_pool", "alloc_kv_workspace",
    "qp_kv_page_bytes", "qp_kv_pool_bytes", "qp_kv_pool_init", "qp_kv_reserve", "qp_kv_fork", "qp_kv_free", "qp_kv_compact", "qp_kv_append", "qp_kv_read",
    "qp_kv_attention_workspace_bytes", "qp_kv_attention",
    "alloc_workspace", "alloc_packed", "dtype_of", "read_ws",
]

QP_OK, QP_EINVAL, QP_ENOSPC, QP_EHIP, QP_ENONFINITE = 0, -1, -2, -3, -4
QP_F32, QP_BF16 = 0, 1
QP_LAPLACE, QP_GAUSS, QP_DIST_AUTO = 0, 1, 2
QP_SEARCH_CLIP_TO_DATA, QP_SEARCH_COARSE_TO_FINE, QP_SEARCH_LOW_BITS_ONLY = 1, 2, 4
QP_WS_STATS, QP_WS_RESULT, QP_WS_QPARAMS, QP_WS_HIST, QP_WS_CANDS, QP_WS_SCORES, QP_WS_MODEL = range(7)
BITS = (2, 3, 4, 6, 8, 16)

QP_KV_POOL_HEADER = 16   # int32 words ahead of the reference counts in a pool record

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libquantpipe.so")


class qp_stats_t(C.Structure):
    _fields_ = [("n", C.c_uint64), ("n_nonfinite", C.c_uint64), ("mean", C.c_double), ("mad", C.c_double),
                ("abs_mean", C.c_double), ("var", C.c_double), ("min", C.c_double), ("max", C.c_double),
                ("nbins", C.c_uint32), ("peak_count", C.c_uint32), ("peak_density", C.c_double),
                ("b_r", C.c_double)]


class qp_qparams_t(C.Structure):
    _fields_ = [("bits", C.c_uint32), ("reserved", C.c_uint32), ("n", C.c_uint64), ("lo", C.c_float),
                ("hi", C.c_float), ("scale", C.c_float), ("inv_scale", C.c_float)]


class qp_search_cfg_t(C.Structure):
    _fields_ = [("t_steps", C.c_uint32), ("cands_per_round", C.c_uint32), ("nbins", C.c_uint32),
                ("dist", C.c_uint32), ("flags", C.c_uint32), ("coarse_stride", C.c_uint32)]


class qp_controller_t(C.Structure):
    _fields_ = [("window", C.c_uint32), ("count", C.c_uint32), ("bits_sum", C.c_double), ("seconds_sum", C.c_double),
                ("s_images", C.c_double), ("r_images_per_s", C.c_double), ("q_cur", C.c_uint32), ("decisions", C.c_uint32)]


class qp_search_result_t(C.Structure):
    _fields_ = [("b_e", C.c_double), ("b_r", C.c_double), ("b_star", C.c_double), ("alpha_star", C.c_double),
                ("mse_aciq", C.c_double), ("mse_star", C.c_double), ("j_star", C.c_uint32),
                ("t_steps", C.c_uint32)]


class qp_model_fit_t(C.Structure):
    _fields_ = [("fit_laplace", C.c_double), ("fit_gauss", C.c_double), ("dist", C.c_uint32), ("reserved", C.c_uint32)]


class qp_job_t(C.Structure):
    _fields_ = [("x_dev", C.c_void_p), ("n", C.c_uint64), ("dtype", C.c_uint32), ("bits", C.c_uint32),
                ("packed_dev", C.c_void_p), ("packed_bytes", C.c_uint64), ("qparams_out_dev", C.c_void_p)]


class qp_lane_t(C.Structure):
    _fields_ = [("ws_dev", C.c_void_p), ("ws_bytes", C.c_size_t), ("stream", C.c_void_p)]


class qp_kv_cache_t(C.Structure):
    _fields_ = [("pages_dev", C.c_void_p), ("pages_bytes", C.c_uint64), ("layers", C.c_uint32), ("n_pages", C.c_uint32),
                ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("page_tokens", C.c_uint32), ("reserved", C.c_uint32)]


class qp_kv_rows_t(C.Structure):
    _fields_ = [("table_dev", C.c_void_p), ("lengths_dev", C.c_void_p), ("rows", C.c_uint32), ("pages_per_row", C.c_uint32)]


class qp_kv_view_t(C.Structure):
    _fields_ = [("data_dev", C.c_void_p), ("dtype", C.c_uint32), ("reserved", C.c_uint32), ("token_stride", C.c_uint64),
                ("head_stride", C.c_uint64)]


class qp_kv_attn_cfg_t(C.Structure):
    _fields_ = [("scale", C.c_float), ("q_heads", C.c_uint32), ("causal", C.c_uint32), ("window", C.c_uint32)]


class QuantPipeError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {qp_strerror(status)} ({status})")


_lib = None


def lib():
    """The loaded C-ABI library.  Raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2211_04515_amd.build` "
                              "(or __graft_entry__.build()); there is no CPU fallback")
        L = C.CDLL(LIB_PATH)
        vp, u64, u32, sz, i32 = C.c_void_p, C.c_uint64, C.c_uint32, C.c_size_t, C.c_int
        sig = {
            "qp_packed_bytes": (sz, [u64, u32]),
            "qp_workspace_bytes": (sz, [u64, C.POINTER(qp_search_cfg_t)]),
            "qp_ws_offset": (sz, [i32]),
            "qp_default_search_cfg": (None, [C.POINTER(qp_search_cfg_t)]),
            "qp_stats": (i32, [vp, u64, i32, u32, vp, sz, vp, C.POINTER(qp_stats_t)]),
            "qp_stats_async": (i32, [vp, u64, i32, u32, vp, sz, vp]),
            "qp_aciq_alpha": (i32, [C.POINTER(qp_stats_t), u32, i32, C.POINTER(C.c_double)]),
            "qp_aciq_constant": (C.c_double, [u32, i32]),
            "qp_make_qparams": (i32, [C.c_double, C.c_double, u32, u64, C.POINTER(qp_qparams_t)]),
            "qp_make_qparams_clipped": (i32, [C.c_double, C.c_double, C.c_double, C.c_double, u32, u64,
                                              C.POINTER(qp_qparams_t)]),
            "qp_dsaciq_search": (i32, [vp, u64, i32, C.POINTER(qp_stats_t), u32, C.POINTER(qp_search_cfg_t), vp, sz,
                                       vp, C.POINTER(qp_search_result_t), C.POINTER(qp_qparams_t)]),
            "qp_dsaciq_search_async": (i32, [vp, u64, i32, u32, C.POINTER(qp_search_cfg_t), vp, sz, vp]),
            "qp_model_fit": (i32, [vp, sz, vp, C.POINTER(qp_model_fit_t)]),
            "qp_model_fit_async": (i32, [vp, sz, vp]),
            "qp_dsaciq_hist_search": (i32, [u32, C.POINTER(qp_search_cfg_t), vp, sz, vp, C.POINTER(qp_search_result_t),
                                            C.POINTER(qp_qparams_t)]),
            "qp_dsaciq_hist_search_async": (i32, [u32, C.POINTER(qp_search_cfg_t), vp, sz, vp]),
            "qp_quant_pack": (i32, [vp, u64, i32, C.POINTER(qp_qparams_t), vp, sz, vp]),
            "qp_quant_pack_dev": (i32, [vp, u64, i32, u32, vp, vp, sz, vp]),
            "qp_unpack_dequant": (i32, [vp, sz, C.POINTER(qp_qparams_t), vp, u64, vp]),
            "qp_unpack_dequant_dev": (i32, [vp, sz, u32, vp, vp, u64, vp]),
            "qp_compress_async": (i32, [vp, u64, i32, u32, C.POINTER(qp_search_cfg_t), vp, sz, vp, sz, vp, vp]),
            "qp_compress_noalloc": (i32, [vp, u64, i32, u32, C.POINTER(qp_search_cfg_t), vp, sz, vp, vp]),
            "qp_compress_many_async": (i32, [C.POINTER(qp_job_t), u32, C.POINTER(qp_search_cfg_t), C.POINTER(qp_lane_t), u32]),
            "qp_next_bits": (i32, [C.c_double, u32, C.c_double, C.c_double, C.c_double, C.POINTER(u32)]),
            "qp_controller_init": (i32, [C.POINTER(qp_controller_t), u32, C.c_double, C.c_double, u32]),
            "qp_controller_update": (i32, [C.POINTER(qp_controller_t), C.c_double, C.c_double, C.POINTER(u32)]),
            "qp_kv_page_bytes": (sz, [vp]),
            "qp_kv_pool_bytes": (sz, [u32]),
            "qp_kv_pool_init": (i32, [u32, vp, sz, vp]),
            "qp_kv_reserve": (i32, [vp, vp, vp, vp, sz, vp]),
            "qp_kv_fork": (i32, [vp, vp, vp, vp, sz, vp]),
            "qp_kv_free": (i32, [vp, vp, vp, vp, sz, vp]),
            "qp_kv_compact": (i32, [vp, vp, vp, sz, vp]),
            "qp_kv_append": (i32, [vp, vp, u32, vp, u64, vp, vp, vp]),
            "qp_kv_read": (i32, [vp, vp, u32, vp, vp, u64, vp, vp, vp]),
            "qp_kv_attention_workspace_bytes": (sz, [vp, vp, u64, u32]),
            "qp_kv_attention": (i32, [vp, vp, u32, vp, u64, vp, vp, vp, vp, sz, vp]),
            "qp_strerror": (C.c_char_p, [i32]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


EXPORTS = ("qp_packed_bytes", "qp_workspace_bytes", "qp_ws_offset", "qp_default_search_cfg", "qp_stats",
           "qp_stats_async", "qp_aciq_alpha", "qp_aciq_constant", "qp_make_qparams", "qp_make_qparams_clipped", "qp_dsaciq_search",
           "qp_dsaciq_search_async", "qp_model_fit", "qp_model_fit_async", "qp_dsaciq_hist_search", "qp_dsaciq_hist_search_async", "qp_quant_pack", "qp_quant_pack_dev", "qp_unpack_dequant",
           "qp_unpack_dequant_dev", "qp_compress_async", "qp_compress_many_async", "qp_compress_noalloc", "qp_next_bits", "qp_controller_init", "qp_controller_update",
           "qp_kv_page_bytes", "qp_kv_pool_bytes", "qp_kv_pool_init", "qp_kv_reserve", "qp_kv_fork", "qp_kv_free", "qp_kv_compact",
           "qp_kv_append", "qp_kv_read", "qp_kv_attention_workspace_bytes", "qp_kv_attention",
           "qp_strerror")


# ---- marshalling helpers ------------------------------------------------------------------

def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def dtype_of(t: "torch.Tensor") -> int:
    if t.dtype == torch.float32:
        return QP_F32
    if t.dtype == torch.bfloat16:
        return QP_BF16
    raise TypeError(f"unsupported tensor dtype {t.dtype}")


def _dev(t: "torch.Tensor"):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    return C.c_void_p(t.data_ptr())


def _cfgp(cfg):
    return C.byref(cfg) if cfg is not None else None


def _check(status: int, what: str, allow=()):
    if status != QP_OK and status not in allow:
        raise QuantPipeError(status, what)
    return status


def alloc_workspace(n: int, cfg=None, device="cuda") -> "torch.Tensor":
    nb = qp_workspace_bytes(n, cfg)
    if nb == 0:
        raise QuantPipeError(QP_EINVAL, "qp_workspace_bytes")
    return torch.empty(nb, dtype=torch.uint8, device=device)


def alloc_packed(n: int, bits: int, device="cuda") -> "torch.Tensor":
    nb = qp_packed_bytes(n, bits)
    if nb == 0:
        raise QuantPipeError(QP_EINVAL, "qp_packed_bytes")
    return torch.empty(nb, dtype=torch.uint8, device=device)


def read_ws(ws: "torch.Tensor", region: int, ctype):
    """Copy a fixed-size record out of the workspace (synchronises the current stream)."""
    off = qp_ws_offset(region)
    raw = ws[off:off + C.sizeof(ctype)].cpu().numpy().tobytes()
    return ctype.from_buffer_copy(raw)


# ---- the entry points, names as in quantpipe.h --------------------------------------------

def qp_strerror(status: int) -> str:
    return lib().qp_strerror(int(status)).decode()


def qp_packed_bytes(n: int, bits: int) -> int:
    return int(lib().qp_packed_bytes(int(n), int(bits)))


def qp_workspace_bytes(n: int, cfg=None) -> int:
    return int(lib().qp_workspace_bytes(int(n), _cfgp(cfg)))


def qp_ws_offset(region: int) -> int:
    return int(lib().qp_ws_offset(int(region)))


def qp_default_search_cfg() -> qp_search_cfg_t:
    cfg = qp_search_cfg_t()
    lib().qp_default_search_cfg(C.byref(cfg))
    return cfg


def qp_stats(x, ws, nbins: int = 2048, stream=None, allow_nonfinite: bool = False) -> qp_stats_t:
    out = qp_stats_t()
    st = lib().qp_stats(_dev(x), x.numel(), dtype_of(x), int(nbins), _dev(ws), ws.numel(), _stream(stream),
                        C.byref(out))
    _check(st, "qp_stats", allow=(QP_ENONFINITE,) if allow_nonfinite else ())
    return out


def qp_stats_async(x, ws, nbins: int = 2048, stream=None) -> None:
    _check(lib().qp_stats_async(_dev(x), x.numel(), dtype_of(x), int(nbins), _dev(ws), ws.numel(), _stream(stream)),
           "qp_stats_async")


def qp_aciq_alpha(stats: qp_stats_t, bits: int, dist: int = QP_LAPLACE) -> float:
    out = C.c_double()
    _check(lib().qp_aciq_alpha(C.byref(stats), int(bits), int(dist), C.byref(out)), "qp_aciq_alpha")
    return out.value


def qp_aciq_constant(bits: int, dist: int = QP_LAPLACE) -> float:
    return float(lib().qp_aciq_constant(int(bits), int(dist)))


def qp_make_qparams(center: float, alpha: float, bits: int, n: int) -> qp_qparams_t:
    q = qp_qparams_t()
    _check(lib().qp_make_qparams(float(center), float(alpha), int(bits), int(n), C.byref(q)), "qp_make_qparams")
    return q


def qp_make_qparams_clipped(center: float, alpha: float, data_min: float, data_max: float, bits: int, n: int) -> qp_qparams_t:
    q = qp_qparams_t()
    _check(lib().qp_make_qparams_clipped(float(center), float(alpha), float(data_min), float(data_max), int(bits), int(n),
                                         C.byref(q)), "qp_make_qparams_clipped")
    return q


def qp_dsaciq_search(x, stats: qp_stats_t, bits: int, ws, cfg=None, stream=None):
    """Returns (qp_search_result_t, qp_qparams_t of the winner)."""
    res, q = qp_search_result_t(), qp_qparams_t()
    _check(lib().qp_dsaciq_search(_dev(x), x.numel(), dtype_of(x), C.byref(stats), int(bits), _cfgp(cfg), _dev(ws),
                                  ws.numel(), _stream(stream), C.byref(res), C.byref(q)), "qp_dsaciq_search")
    return res, q


def qp_dsaciq_search_async(x, bits: int, ws, cfg=None, stream=None) -> None:
    _check(lib().qp_dsaciq_search_async(_dev(x), x.numel(), dtype_of(x), int(bits), _cfgp(cfg), _dev(ws), ws.numel(),
                                        _stream(stream)), "qp_dsaciq_search_async")


def qp_quant_pack(x, qparams: qp_qparams_t, packed, stream=None) -> None:
    _check(lib().qp_quant_pack(_dev(x), x.numel(), dtype_of(x), C.byref(qparams), _dev(packed),
                               packed.numel() * packed.element_size(), _stream(stream)), "qp_quant_pack")


def qp_quant_pack_dev(x, bits: int, qparams_dev_ptr: int, packed, stream=None) -> None:
    _check(lib().qp_quant_pack_dev(_dev(x), x.numel(), dtype_of(x), int(bits), C.c_void_p(qparams_dev_ptr),
                                   _dev(packed), packed.numel() * packed.element_size(), _stream(stream)),
           "qp_quant_pack_dev")


def qp_unpack_dequant(packed, qparams: qp_qparams_t, y, stream=None) -> None:
    if y.dtype != torch.float32:
        raise TypeError("y must be float32")
    _check(lib().qp_unpack_dequant(_dev(packed), packed.numel() * packed.element_size(), C.byref(qparams), _dev(y),
                                   y.numel(), _stream(stream)), "qp_unpack_dequant")


def qp_unpack_dequant_dev(packed, bits: int, qparams_dev_ptr: int, y, stream=None) -> None:
    if y.dtype != torch.float32:
        raise TypeError("y must be float32")
    _check(lib().qp_unpack_dequant_dev(_dev(packed), packed.numel() * packed.element_size(), int(bits),
                                       C.c_void_p(qparams_dev_ptr), _dev(y), y.numel(), _stream(stream)),
           "qp_unpack_dequant_dev")


def qp_compress_async(x, bits: int, ws, packed, qparams_out_dev_ptr: int = 0, cfg=None, stream=None) -> None:
    _check(lib().qp_compress_async(_dev(x), x.numel(), dtype_of(x), int(bits), _cfgp(cfg), _dev(ws), ws.numel(),
                                   _dev(packed), packed.numel() * packed.element_size(),
                                   C.c_void_p(qparams_out_dev_ptr) if qparams_out_dev_ptr else None,
                                   _stream(stream)), "qp_compress_async")


def qp_compress_many_async(jobs, lanes, cfg=None) -> None:
    """jobs: sequence of (x, bits, packed, qparams_out_dev_ptr or 0); lanes: sequence of (workspace, stream)."""
    ja = (qp_job_t * len(jobs))()
    for k, (x, bits, packed, qptr) in enumerate(jobs):
        ja[k] = qp_job_t(x.data_ptr(), x.numel(), dtype_of(x), int(bits), packed.data_ptr(),
                         packed.numel() * packed.element_size(), qptr or None)
    la = (qp_lane_t * len(lanes))()
    for k, (ws, stream) in enumerate(lanes):
        la[k] = qp_lane_t(ws.data_ptr(), ws.numel(), _stream(stream).value)
    _check(lib().qp_compress_many_async(ja, len(jobs), _cfgp(cfg), la, len(lanes)), "qp_compress_many_async")


def qp_compress_noalloc(x, bits: int, packed, qparams_out_dev_ptr: int, cfg=None, stream=None) -> None:
    _check(lib().qp_compress_noalloc(_dev(x), x.numel(), dtype_of(x), int(bits), _cfgp(cfg), _dev(packed),
                                     packed.numel() * packed.element_size(), C.c_void_p(qparams_out_dev_ptr),
                                     _stream(stream)), "qp_compress_noalloc")


def qp_next_bits(v_bits: float, q_cur: int, s_images: float, r_images_per_s: float, bandwidth_bits_per_s: float) -> int:
    out = C.c_uint32()
    _check(lib().qp_next_bits(float(v_bits), int(q_cur), float(s_images), float(r_images_per_s),
                              float(bandwidth_bits_per_s), C.byref(out)), "qp_next_bits")
    return out.value


def qp_controller_init(window: int, s_images: float, r_images_per_s: float, q_start: int = 32) -> qp_controller_t:
    c = qp_controller_t()
    _check(lib().qp_controller_init(C.byref(c), int(window), float(s_images), float(r_images_per_s), int(q_start)),
           "qp_controller_init")
    return c


def qp_controller_update(c: qp_controller_t, payload_bits: float, seconds: float) -> int:
    out = C.c_uint32()
    _check(lib().qp_controller_update(C.byref(c), float(payload_bits), float(seconds), C.byref(out)), "qp_controller_update")
    return out.value


def qp_model_fit(ws, stream=None) -> qp_model_fit_t:
    """Which model (Laplace or Gaussian) the statistics and histogram left in ws fit better."""
    out = qp_model_fit_t()
    _check(lib().qp_model_fit(_dev(ws), ws.numel(), _stream(stream), C.byref(out)), "qp_model_fit")
    return out


def qp_model_fit_async(ws, stream=None) -> None:
    _check(lib().qp_model_fit_async(_dev(ws), ws.numel(), _stream(stream)), "qp_model_fit_async")


def qp_dsaciq_hist_search(bits: int, ws, cfg=None, stream=None):
    """Histogram-fit reading of Eq. 1 on the statistics left in ws.  Returns (result, qparams)."""
    res, q = qp_search_result_t(), qp_qparams_t()
    _check(lib().qp_dsaciq_hist_search(int(bits), _cfgp(cfg), _dev(ws), ws.numel(), _stream(stream), C.byref(res),
                                       C.byref(q)), "qp_dsaciq_hist_search")
    return res, q


def qp_dsaciq_hist_search_async(bits: int, ws, cfg=None, stream=None) -> None:
    _check(lib().qp_dsaciq_hist_search_async(int(bits), _cfgp(cfg), _dev(ws), ws.numel(), _stream(stream)),
           "qp_dsaciq_hist_search_async")


# ---- the key/value cache in 4 bits ----------------------------------------------------------
# The structs hold device addresses; the tensors behind them are kept alive by the struct objects (`tensors`).  Tensors of a call
# lie on one device; a call goes to that device's current stream (or to `stream`, which must be one of its streams).

def kv_cache(pages, kv_heads: int, head_dim: int, page_tokens: int) -> qp_kv_cache_t:
    """The cache in `pages`: contiguous device bytes of shape [layers, n_pages, ...] (alloc_kv_pages makes them)."""
    if pages.dim() < 2 or pages.dtype != torch.uint8 or not pages.is_contiguous() or not pages.is_cuda:
        raise ValueError("pages: expected a contiguous uint8 device tensor [layers, n_pages, ...]")
    c = _sizes("kv_cache", pages.shape[0], pages.shape[1], kv_heads, head_dim, page_tokens)
    c.pages_dev, c.pages_bytes = pages.data_ptr(), pages.numel()
    c.tensors, c.device = (pages,), pages.get_device()
    return c


def kv_rows(table, lengths) -> qp_kv_rows_t:
    """Rows with their page table, int32 [rows, pages_per_row], and lengths, int32 [rows]."""
    if table.dim() != 2 or tuple(lengths.shape) != (table.shape[0],):
        raise ValueError("expected table [rows, pages_per_row] and lengths [rows]")
    device = table.get_device()
    r = qp_kv_rows_t(_ints(table, 0, device), _ints(lengths, 0, device), *table.shape)
    r.tensors, r.device = (table, lengths), device
    return r


def alloc_kv_pages(n_pages: int, kv_heads: int, head_dim: int, page_tokens: int, layers: int = 1, device="cuda") -> "torch.Tensor":
    """Room for a cache, not initialised: what was never written is never looked at."""
    c = _sizes("alloc_kv_pages", layers, n_pages, kv_heads, head_dim, page_tokens)
    if not (1 <= layers <= 65536 and 1 <= n_pages <= 1 << 24):
        raise QuantPipeError(QP_EINVAL, "alloc_kv_pages")
    return torch.empty((layers, n_pages, kv_heads, qp_kv_page_bytes(c) // kv_heads), dtype=torch.uint8, device=device)


def alloc_kv_pool(n_pages: int, device="cuda") -> "torch.Tensor":
    """A pool record with every page free: int32, the header, then the reference counts refs[n_pages], then room."""
    nb = qp_kv_pool_bytes(n_pages)
    if nb == 0:
        raise QuantPipeError(QP_EINVAL, "qp_kv_pool_bytes")
    pool = torch.empty(nb // 4, dtype=torch.int32, device=device)
    qp_kv_pool_init(n_pages, pool)
    return pool


def alloc_kv_workspace(cache: qp_kv_cache_t, rows: qp_kv_rows_t, tokens: int, q_heads: int) -> "torch.Tensor":
    nb = qp_kv_attention_workspace_bytes(cache, rows, tokens, q_heads)
    if nb == 0:
        raise QuantPipeError(QP_EINVAL, "qp_kv_attention_workspace_bytes")
    return torch.empty(nb, dtype=torch.uint8, device=cache.tensors[0].device)


# (A call's checks in Python are what the smallest calls cost: devices are compared as numbers, -1 is none, and a tensor's shape is asked for once.)
def _ints(t, count: int, device: int) -> int:
    if t.dtype != torch.int32 or t.numel() < count or not t.is_contiguous() or t.get_device() != device or device < 0:
        raise ValueError("expected a contiguous int32 tensor of at least %d entries on device %d" % (count, device))
    return t.data_ptr()


def _view(t, heads: int, dim: int, tokens: int, device: int) -> qp_kv_view_t:
    if t.shape != (tokens, heads, dim) or t.get_device() != device:
        raise ValueError("expected a tensor [%d, %d, %d] on device %d, got %s on %s" % (tokens, heads, dim, device, tuple(t.shape), t.device))
    a, b, c = t.stride()
    if c != 1:
        raise ValueError("the elements of a head must lie next to each other")
    # (an axis of one entry may carry any stride: it is never used)
    return qp_kv_view_t(t.data_ptr(), dtype_of(t), 0, a if tokens > 1 else 0, b if heads > 1 else 0)


def _kv_call(device: int, stream, what: str, *args) -> None:
    """The library's call on the device's own current stream, with that device current (kernels go to the current one)."""
    call = getattr(lib(), what)
    handle = torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream
    if device == torch.cuda.current_device():
        st = call(*args, handle)
    else:
        with torch.cuda.device(device):
            st = call(*args, handle)
    if st != QP_OK:
        raise QuantPipeError(st, what)


def _uint(v: int, what: str) -> int:
    """A number for a 32-bit field, which ctypes would cut down to its low bits."""
    if not 0 <= int(v) < 1 << 32:
        raise QuantPipeError(QP_EINVAL, what)
    return int(v)


def _sizes(what: str, *sizes) -> qp_kv_cache_t:
    """A cache of these sizes (layers, n_pages, kv_heads, head_dim, page_tokens), without its pages."""
    c = qp_kv_cache_t(None, 0, *(_uint(v, what) for v in sizes), 0)
    if qp_kv_page_bytes(c) == 0:
        raise QuantPipeError(QP_EINVAL, what)
    return c


def qp_kv_page_bytes(cache: qp_kv_cache_t) -> int:
    return int(lib().qp_kv_page_bytes(C.byref(cache)))


def qp_kv_pool_bytes(n_pages: int) -> int:
    return int(lib().qp_kv_pool_bytes(int(n_pages))) if 0 <= n_pages < 1 << 32 else 0


def qp_kv_attention_workspace_bytes(cache: qp_kv_cache_t, rows: qp_kv_rows_t, tokens: int, q_heads: int) -> int:
    if not (0 <= tokens < 1 << 32 and 0 <= q_heads < 1 << 32):
        return 0
    return int(lib().qp_kv_attention_workspace_bytes(C.byref(cache), C.byref(rows), int(tokens), int(q_heads)))


def qp_kv_pool_init(n_pages: int, pool, stream=None) -> None:
    if qp_kv_pool_bytes(n_pages) == 0:
        raise QuantPipeError(QP_EINVAL, "qp_kv_pool_init")
    d = pool.get_device()
    _kv_call(d, stream, "qp_kv_pool_init", int(n_pages), _ints(pool, 1, d), pool.numel() * 4)


def _same_device(cache, rows) -> int:
    if rows.device != cache.device:
        raise ValueError("the rows are on device %d, the pages on device %d" % (rows.device, cache.device))
    return cache.device


def _books(what: str, cache, rows, pool, per_row, stream) -> None:
    d = _same_device(cache, rows)
    _kv_call(d, stream, what, C.byref(cache), C.byref(rows), _ints(per_row, rows.rows, d), _ints(pool, 1, d), pool.numel() * 4)


def qp_kv_reserve(cache, rows, pool, want, stream=None) -> None:
    """want[r] more tokens for each row; words 0 and 1 of `pool` say afterwards whether it was done (both 0) or nothing was."""
    _books("qp_kv_reserve", cache, rows, pool, want, stream)


def qp_kv_fork(cache, rows, pool, parent, stream=None) -> None:
    """Row r becomes a copy of row parent[r] (negative: left alone) that shares its pages; word 2 of `pool` counts the rows refused so far."""
    _books("qp_kv_fork", cache, rows, pool, parent, stream)


def qp_kv_free(cache, rows, pool, keep, stream=None) -> None:
    """Row r keeps its first keep[r] tokens (negative: left alone) and gives up the pages behind them."""
    _books("qp_kv_free", cache, rows, pool, keep, stream)


def qp_kv_compact(cache, rows, pool, stream=None) -> None:
    """Moves the pages in use to the pool's low end; word 3 of `pool` says how many there are."""
    d = _same_device(cache, rows)
    _kv_call(d, stream, "qp_kv_compact", C.byref(cache), C.byref(rows), _ints(pool, 1, d), pool.numel() * 4)


def qp_kv_append(cache, rows, layer: int, token_begin, k, v, stream=None) -> None:
    """Quantizes k, v [tokens, kv_heads, head_dim] into the rows' last places."""
    d = _same_device(cache, rows)
    n = k.shape[0]
    kv, vv = _view(k, cache.kv_heads, cache.head_dim, n, d), _view(v, cache.kv_heads, cache.head_dim, n, d)
    _kv_call(d, stream, "qp_kv_append", C.byref(cache), C.byref(rows), _uint(layer, "qp_kv_append"), _ints(token_begin, rows.rows + 1, d), n, C.byref(kv), C.byref(vv))


def qp_kv_read(cache, rows, layer: int, token_begin, k, v, first=None, stream=None) -> None:
    """Writes the rows' tokens from first[r] (None: 0) on to k, v [tokens, kv_heads, head_dim]."""
    d = _same_device(cache, rows)
    n = k.shape[0]
    kv, vv = _view(k, cache.kv_heads, cache.head_dim, n, d), _view(v, cache.kv_heads, cache.head_dim, n, d)
    f = None if first is None else _ints(first, rows.rows, d)
    _kv_call(d, stream, "qp_kv_read", C.byref(cache), C.byref(rows), _uint(layer, "qp_kv_read"), _ints(token_begin, rows.rows + 1, d), f, n, C.byref(kv), C.byref(vv))


def qp_kv_attention(cache, rows, layer: int, token_begin, q, out, ws, scale: float = None, causal: bool = True, window: int = 0,
                    stream=None) -> None:
    """out = softmax(scale q K^T) V for the rows' last tokens; q, out [tokens, q_heads, head_dim]; scale None: 1 / sqrt(head_dim)."""
    d = _same_device(cache, rows)
    n, heads = q.shape[0], q.shape[1]
    qv, ov = _view(q, heads, cache.head_dim, n, d), _view(out, heads, cache.head_dim, n, d)
    if ws.get_device() != d or not ws.is_contiguous():
        raise ValueError("expected a contiguous workspace on device %d" % d)
    cfg = qp_kv_attn_cfg_t(cache.head_dim ** -0.5 if scale is None else scale, heads, 1 if causal else 0, _uint(window, "qp_kv_attention"))
    _kv_call(d, stream, "qp_kv_attention", C.byref(cache), C.byref(rows), _uint(layer, "qp_kv_attention"), _ints(token_begin, rows.rows + 1, d), n, C.byref(qv), C.byref(ov),
             C.byref(cfg), ws.data_ptr(), ws.numel() * ws.element_size())
