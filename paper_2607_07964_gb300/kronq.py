"""Thin Python binding of libkronq (include/kronq.h): the same entry points, taking torch
CUDA tensors. It only checks and marshals arguments (pointers, sizes, the current CUDA
stream); every step of the computation runs in the library's kernels. There is no CPU
or PyTorch fallback: if libkronq.so is missing or fails to load, every call raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# KQ_DEBUG=1 selects the debug build (bounds checks before the kernels' stores; see
# kq_debug_status), built with `python -m paper_2607_07964_gb300.build --debug`
LIB_PATH = os.path.join(_HERE, "libkronq_debug.so" if os.environ.get("KQ_DEBUG") == "1" else "libkronq.so")

KQ_OK, KQ_ERR_INVALID_ARG, KQ_ERR_UNSUPPORTED, KQ_ERR_NOT_PD = 0, 1, 2, 3
KQ_ERR_CUDA, KQ_ERR_TIMEOUT, KQ_ERR_WORKSPACE, KQ_ERR_NONFINITE = 4, 5, 6, 7
KQ_FWD, KQ_INV, KQ_FWD_SYM = 0, 1, 2
KQ_TRAIL_FP32, KQ_TRAIL_3XTF32 = 0, 1
KQ_SYRK_CHUNK_TOKENS = 512
KQ_BF16, KQ_F32 = 0, 1
KQ_LOGPROBS_MAX_TOP = 32

_lib = None


class KronqError(RuntimeError):
    def __init__(self, status: int, where: str, msg: str):
        super().__init__(f"{where}: {status_name(status)} ({msg})")
        self.status = status


def lib() -> ctypes.CDLL:
    """Load libkronq.so (built by paper_2607_07964_gb300.build); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2607_07964_gb300.build` (needs nvcc)")
        L = ctypes.CDLL(LIB_PATH)
        P, I64, I, F, SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        sig = {
            "kq_last_error": ([], ctypes.c_char_p),
            "kq_status_name": ([I], ctypes.c_char_p),
            "kq_version": ([], I),
            "kq_launch_count": ([], ctypes.c_uint64),
            "kq_graph_instantiate": ([P, I, P], I),
            "kq_graph_launch": ([P, P], I),
            "kq_graph_exec_destroy": ([P], I),
            "kq_check": ([P, I, P, P], I),
            "kq_selftest_timeout": ([P, I64, P], I),
            "kq_debug_build": ([], I),
            "kq_debug_status": ([P, P, I], I),
            "kq_selftest_bounds": ([P, I64, P], I),
            "kq_selftest_div": ([P, P, I64, P, P], I),
            "kq_accum_factor": ([P, I64, I64, I64, P, I, P, P, P], I),
            "kq_compute_scales": ([P, I64, I64, P, P, P, P, P], I),
            "kq_compute_scales_diag": ([P, I64, I64, P, P, P, P, P], I),
            "kq_compute_scales_exp": ([P, I64, I64, P, P, P, P, F, F, P], I),
            "kq_biip_stats_workspace": ([I64, I64], SZ),
            "kq_biip_stats": ([P, I64, I64, P, P, P, P, SZ, P], I),
            "kq_traces_diag": ([P, P, I64, P, P, I64, P, P], I),
            "kq_factor_diag_workspace": ([I64, I64], SZ),
            "kq_factor_diag": ([P, I64, I64, I64, P, P, P, SZ, P], I),
            "kq_traces": ([P, P, I64, P, P, I64, P, P], I),
            "kq_rotate_in": ([P, I64, I64, P, P, P, I, P], I),
            "kq_rotate_out": ([P, I64, I64, P, P, P, I, P], I),
            "kq_chol_inv_workspace": ([I64], SZ),
            "kq_chol_inv": ([P, I64, F, P, P, P, SZ, P], I),
            "kq_chol_inv_noalloc": ([P, I64, F, P, P, P], I),
            "kq_obs_quantize_workspace": ([I64, I64, I, I, I], SZ),
            "kq_obs_quantize": ([P, I64, I64, P, P, I, I, I, I, P, P, P, P, P, P, P, SZ, P], I),
            "kq_accum_drift_workspace": ([I64, I64], SZ),
            "kq_accum_drift": ([P, P, I64, I64, I64, P, I, P, P, SZ, P], I),
            "kq_packed_codes_bytes": ([I64, I64, I], SZ),
            "kq_pack_codes": ([P, I64, I64, I, P, P], I),
            "kq_infer_workspace": ([I64, I64, I64], SZ),
            "kq_infer": ([P, P, P, I64, I64, I, I, P, P, P, P, P, I64, P, P, P, SZ, P], I),
            "kq_gptaq_p_workspace": ([I64], SZ),
            "kq_gptaq_p": ([P, P, I64, F, P, P, P, SZ, P], I),
            "kq_dequant_revert": ([P, P, P, I64, I64, I, P, P, P, P, P, P], I),
            "kq_kv_append": ([P, P, P, I, I64, I64, I64, I64, I64, P, P, P, P, P, I64, P, P, P, P], I),
            "kq_kv_read": ([P, P, P, P, I, I64, P, P, P, P], I),
            "kq_kv_attend_workspace": ([I64, I64, I64, I64, I64], SZ),
            "kq_kv_attend": ([P, P, I, I64, I64, I64, I64, P, P, F, P, P, P, I64, P, P, SZ, P], I),
            "kq_kv_evict_workspace": ([I64, I64, I64, I64], SZ),
            "kq_kv_evict": ([P, P, P, P, P, I64, I64, I64, I64, P, P, P, P, P, SZ, P], I),
            "kq_token_logprobs": ([P, I, I64, I64, I64, P, I, P, P, P, P, P, P, P], I),
            "kq_token_logprobs_grad": ([P, I, I64, I64, I64, P, P, P, P, P, P, I64, P, P], I),
            "kq_proxy_loss_workspace": ([I64, I64], SZ),
            "kq_proxy_loss": ([P, P, I64, I64, P, P, P, P, SZ, P], I),
        }
        for name, (args, res) in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _lib = L
    return _lib


def status_name(s: int) -> str:
    return lib().kq_status_name(int(s)).decode()


def last_error() -> str:
    return lib().kq_last_error().decode()


def _ok(st: int, where: str) -> None:
    if st != KQ_OK:
        raise KronqError(st, where, last_error())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None and torch.cuda.is_initialized():   # the current stream's handle, without an object around it
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _need(t, name, dtype, shape=None, contiguous=True):
    if t is None or (t.is_cuda and t.dtype is dtype and (shape is None or t.shape == shape) and
                     (not contiguous or t.is_contiguous())):
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def version() -> int:
    return lib().kq_version()


def launch_count() -> int:
    """Kernels launched by libkronq so far in this process."""
    return int(lib().kq_launch_count())


def kq_check(info=None, reset: bool = True, stream=None) -> tuple[int, int]:
    """Synchronize the stream and read the device error word; returns (status, raw)."""
    raw = ctypes.c_int(0)
    st = lib().kq_check(_ptr(info), int(reset), ctypes.byref(raw), _stream(stream))
    return st, raw.value


def kq_debug_build() -> bool:
    return bool(lib().kq_debug_build())


DEBUG_UNITS = ("api", "syrk", "biip", "chol", "obs", "trail_tc", "gptaq", "infer", "check", "kv_store",
               "kv_attend", "kv_evict", "logprob")


def kq_debug_status(reset: bool = True) -> tuple[str | None, int]:
    """(source file, line) of the first failed bounds check of the debug build, or (None, 0)."""
    unit, line = ctypes.c_int(-1), ctypes.c_int(0)
    _ok(lib().kq_debug_status(ctypes.byref(unit), ctypes.byref(line), int(reset)), "kq_debug_status")
    return (DEBUG_UNITS[unit.value] if unit.value >= 0 else None), line.value


def kq_selftest_bounds(buf, n: int, stream=None) -> None:
    """buf: n + 1 float32 on the device; writes buf[i] = i for i <= n under a check against n."""
    _need(buf, "buf", torch.float32, (n + 1,))
    _ok(lib().kq_selftest_bounds(_ptr(buf), int(n), _stream(stream)), "kq_selftest_bounds")


def kq_selftest_timeout(info, limit_us: int, stream=None) -> None:
    """A kernel whose bounded wait runs out (nothing arrives); *info gets -KQ_ERR_TIMEOUT."""
    _need(info, "info", torch.int32)
    _ok(lib().kq_selftest_timeout(_ptr(info), int(limit_us), _stream(stream)), "kq_selftest_timeout")


def kq_graph_instantiate(graph: int, use_node_priority: bool = True) -> int:
    """cudaGraphExec_t (as an int) for the cudaGraph_t `graph`, honouring the captured
    per-node priorities when use_node_priority."""
    ex = ctypes.c_void_p()
    _ok(lib().kq_graph_instantiate(ctypes.c_void_p(graph), int(use_node_priority), ctypes.byref(ex)),
        "kq_graph_instantiate")
    return int(ex.value)


def kq_graph_launch(exec_: int, stream=None) -> None:
    _ok(lib().kq_graph_launch(ctypes.c_void_p(exec_), _stream(stream)), "kq_graph_launch")


def kq_graph_exec_destroy(exec_: int) -> None:
    _ok(lib().kq_graph_exec_destroy(ctypes.c_void_p(exec_)), "kq_graph_exec_destroy")


def kq_selftest_div(a, b, mismatches, stream=None) -> None:
    """mismatches (+)= the count of a[i] / b[i] where the sweep's division differs from IEEE
    round-to-nearest division in any bit; a, b fp32 of one shape, mismatches one int64."""
    _need(a, "a", torch.float32)
    _need(b, "b", torch.float32, tuple(a.shape))
    _need(mismatches, "mismatches", torch.int64, (1,))
    _ok(lib().kq_selftest_div(_ptr(a), _ptr(b), a.numel(), _ptr(mismatches), _stream(stream)), "kq_selftest_div")


def kq_accum_factor(A, H, accumulate: bool = False, trace=None, info=None, stream=None) -> None:
    """H (+)= A^T A; A [T, d] bf16 (row stride may exceed d), H [d, d] fp32."""
    if A.dim() != 2 or A.stride(1) != 1:
        raise ValueError("A must be 2-D with unit column stride")
    T, d = A.shape
    _need(A, "A", torch.bfloat16, contiguous=False)
    _need(H, "H", torch.float32, (d, d))
    _need(trace, "trace", torch.float64)
    _need(info, "info", torch.int32)
    _ok(lib().kq_accum_factor(_ptr(A), T, d, A.stride(0), _ptr(H), int(accumulate), _ptr(trace),
                              _ptr(info), _stream(stream)), "kq_accum_factor")


def kq_accum_drift_workspace(T: int, d: int) -> int:
    """Bytes for one pass over all T tokens (a smaller workspace makes token chunks)."""
    return int(lib().kq_accum_drift_workspace(T, d))


def kq_accum_drift(Xt, X, D, accumulate: bool = False, info=None, ws=None, stream=None) -> None:
    """D (+)= (X~ - X)^T X; Xt (X~) and X [T, d] bf16 with the same row stride, D [d, d] fp32."""
    if X.dim() != 2 or X.stride(1) != 1 or Xt.shape != X.shape or Xt.stride() != X.stride():
        raise ValueError("X~ and X must be 2-D, same shape and strides, unit column stride")
    T, d = X.shape
    _need(Xt, "Xt", torch.bfloat16, contiguous=False)
    _need(X, "X", torch.bfloat16, contiguous=False)
    _need(D, "D", torch.float32, (d, d))
    _need(info, "info", torch.int32)
    _need(ws, "ws", torch.uint8)
    _ok(lib().kq_accum_drift(_ptr(Xt), _ptr(X), T, d, X.stride(0), _ptr(D), int(accumulate), _ptr(info),
                             _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)), "kq_accum_drift")


def kq_gptaq_p_workspace(n: int) -> int:
    return int(lib().kq_gptaq_p_workspace(n))


def kq_gptaq_p(Dp, Lt, alpha: float, Pt, ws, info=None, stream=None) -> None:
    """Pt = P^T with P = alpha ((D' L) o M_U) L^T (Proposition 1, Algorithm 2)."""
    n = Lt.shape[0]
    _need(Dp, "Dp", torch.float32, (n, n))
    _need(Lt, "Lt", torch.float32, (n, n))
    _need(Pt, "Pt", torch.float32, (n, n))
    _need(ws, "ws", torch.uint8)
    _need(info, "info", torch.int32)
    _ok(lib().kq_gptaq_p(_ptr(Dp), _ptr(Lt), n, float(alpha), _ptr(Pt), _ptr(info), _ptr(ws),
                         0 if ws is None else ws.numel(), _stream(stream)), "kq_gptaq_p")


def kq_compute_scales(W, H_X, H_G, s_x, s_g, stream=None) -> None:
    """s_x and/or s_g (each side computed only if its output is given)."""
    d_out, d_in = W.shape
    _need(W, "W", torch.float32)
    _need(H_X, "H_X", torch.float32, (d_in, d_in))
    _need(H_G, "H_G", torch.float32, (d_out, d_out))
    _need(s_x, "s_x", torch.float32, (d_in,))
    _need(s_g, "s_g", torch.float32, (d_out,))
    _ok(lib().kq_compute_scales(_ptr(W), d_out, d_in, _ptr(H_X), _ptr(H_G), _ptr(s_x), _ptr(s_g),
                                _stream(stream)), "kq_compute_scales")


def kq_compute_scales_exp(W, H_X, H_G, s_x, s_g, ex: float, eg: float, stream=None) -> None:
    """Scales with the exponent as a parameter (1/4: kq_compute_scales)."""
    d_out, d_in = W.shape
    _need(W, "W", torch.float32)
    _need(H_X, "H_X", torch.float32, (d_in, d_in))
    _need(H_G, "H_G", torch.float32, (d_out, d_out))
    _need(s_x, "s_x", torch.float32, (d_in,))
    _need(s_g, "s_g", torch.float32, (d_out,))
    _ok(lib().kq_compute_scales_exp(_ptr(W), d_out, d_in, _ptr(H_X), _ptr(H_G), _ptr(s_x), _ptr(s_g), float(ex),
                                    float(eg), _stream(stream)), "kq_compute_scales_exp")


def kq_biip_stats_workspace(d_out: int, d_in: int) -> int:
    return int(lib().kq_biip_stats_workspace(d_out, d_in))


def kq_biip_stats(W, H_X, H_G, out, ws, stream=None) -> None:
    """out [4] float64 = [CV_in, CV_out, rho_in, rho_out] of W with the factors' diagonals."""
    d_out, d_in = W.shape
    _need(W, "W", torch.float32)
    _need(H_X, "H_X", torch.float32, (d_in, d_in))
    _need(H_G, "H_G", torch.float32, (d_out, d_out))
    _need(out, "out", torch.float64, (4,))
    _need(ws, "ws", torch.uint8)
    _ok(lib().kq_biip_stats(_ptr(W), d_out, d_in, _ptr(H_X), _ptr(H_G), _ptr(out), _ptr(ws),
                            0 if ws is None else ws.numel(), _stream(stream)), "kq_biip_stats")


def kq_traces(H_X, s_x, H_G, s_g, out, stream=None) -> None:
    """Sensitivity traces; either factor may be None (that side of `out` is kept)."""
    d_in = 0 if H_X is None else H_X.shape[0]
    d_out = 0 if H_G is None else H_G.shape[0]
    _need(H_X, "H_X", torch.float32, (d_in, d_in))
    _need(H_G, "H_G", torch.float32, (d_out, d_out))
    _need(s_x, "s_x", torch.float32, (d_in,))
    _need(s_g, "s_g", torch.float32, (d_out,))
    _need(out, "out", torch.float64, (6,))
    _ok(lib().kq_traces(_ptr(H_X), _ptr(s_x), d_in, _ptr(H_G), _ptr(s_g), d_out, _ptr(out),
                        _stream(stream)), "kq_traces")


def kq_factor_diag_workspace(T: int, d: int) -> int:
    return int(lib().kq_factor_diag_workspace(T, d))


def kq_factor_diag(A, diag, trace=None, ws=None, stream=None) -> None:
    """diag(A^T A) (fp64 sums, fp32 result) and optionally its total; A [T, d] bf16."""
    if A.dim() != 2 or A.stride(1) != 1:
        raise ValueError("A must be 2-D with unit column stride")
    T, d = A.shape
    _need(A, "A", torch.bfloat16, contiguous=False)
    _need(diag, "diag", torch.float32, (d,))
    _need(trace, "trace", torch.float64)
    _need(ws, "ws", torch.uint8)
    _ok(lib().kq_factor_diag(_ptr(A), T, d, A.stride(0), _ptr(diag), _ptr(trace), _ptr(ws),
                             0 if ws is None else ws.numel(), _stream(stream)), "kq_factor_diag")


def kq_compute_scales_diag(W, hx_diag, hg_diag, s_x, s_g, stream=None) -> None:
    d_out, d_in = W.shape
    _need(W, "W", torch.float32)
    _need(hx_diag, "hx_diag", torch.float32, (d_in,))
    _need(hg_diag, "hg_diag", torch.float32, (d_out,))
    _need(s_x, "s_x", torch.float32, (d_in,))
    _need(s_g, "s_g", torch.float32, (d_out,))
    _ok(lib().kq_compute_scales_diag(_ptr(W), d_out, d_in, _ptr(hx_diag), _ptr(hg_diag), _ptr(s_x), _ptr(s_g),
                                     _stream(stream)), "kq_compute_scales_diag")


def kq_traces_diag(hx_diag, s_x, hg_diag, s_g, out, stream=None) -> None:
    d_in = 0 if hx_diag is None else hx_diag.shape[0]
    d_out = 0 if hg_diag is None else hg_diag.shape[0]
    _need(hx_diag, "hx_diag", torch.float32, (d_in,))
    _need(hg_diag, "hg_diag", torch.float32, (d_out,))
    _need(s_x, "s_x", torch.float32, (d_in,))
    _need(s_g, "s_g", torch.float32, (d_out,))
    _need(out, "out", torch.float64, (6,))
    _ok(lib().kq_traces_diag(_ptr(hx_diag), _ptr(s_x), d_in, _ptr(hg_diag), _ptr(s_g), d_out, _ptr(out),
                             _stream(stream)), "kq_traces_diag")


def kq_rotate_in(W, H_X, s_x, sign_v, direction: int = KQ_FWD, stream=None, d_out: int = 0) -> None:
    """W may be None (then only H_X is transformed, forward direction)."""
    if W is not None:
        d_out, d_in = W.shape
    else:
        d_in = H_X.shape[0]
    _need(W, "W", torch.float32)
    _need(H_X, "H_X", torch.float32, (d_in, d_in))
    _need(s_x, "s_x", torch.float32, (d_in,))
    _need(sign_v, "sign_v", torch.int8, (d_in,))
    _ok(lib().kq_rotate_in(_ptr(W), d_out, d_in, _ptr(H_X), _ptr(s_x), _ptr(sign_v), int(direction),
                           _stream(stream)), "kq_rotate_in")


def kq_rotate_out(W, H_G, s_g, sign_u, direction: int = KQ_FWD, stream=None, d_in: int = 0) -> None:
    """W may be None (then only H_G is transformed, forward direction)."""
    if W is not None:
        d_out, d_in = W.shape
    else:
        d_out = H_G.shape[0]
    _need(W, "W", torch.float32)
    _need(H_G, "H_G", torch.float32, (d_out, d_out))
    _need(s_g, "s_g", torch.float32, (d_out,))
    _need(sign_u, "sign_u", torch.int8, (d_out,))
    _ok(lib().kq_rotate_out(_ptr(W), d_out, d_in, _ptr(H_G), _ptr(s_g), _ptr(sign_u), int(direction),
                            _stream(stream)), "kq_rotate_out")


def kq_chol_inv_workspace(n: int) -> int:
    return int(lib().kq_chol_inv_workspace(n))


def kq_chol_inv(H, damp_rel: float, Lt, info, ws, stream=None) -> None:
    n = H.shape[0]
    _need(H, "H", torch.float32, (n, n))
    _need(Lt, "Lt", torch.float32, (n, n))
    _need(info, "info", torch.int32)
    _need(ws, "ws", torch.uint8)
    _ok(lib().kq_chol_inv(_ptr(H), n, float(damp_rel), _ptr(Lt), _ptr(info), _ptr(ws),
                          0 if ws is None else ws.numel(), _stream(stream)), "kq_chol_inv")


KQ_CHOL_NOALLOC_MAX_N = 1024


def kq_chol_inv_noalloc(H, damp_rel: float, Lt, info=None, stream=None) -> None:
    """kq_chol_inv without a caller workspace (n <= KQ_CHOL_NOALLOC_MAX_N): the library's
    own fixed device array serves as scratch. Calls must not overlap on the GPU."""
    n = H.shape[0]
    _need(H, "H", torch.float32, (n, n))
    _need(Lt, "Lt", torch.float32, (n, n))
    _need(info, "info", torch.int32)
    _ok(lib().kq_chol_inv_noalloc(_ptr(H), n, float(damp_rel), _ptr(Lt), _ptr(info), _stream(stream)),
        "kq_chol_inv_noalloc")


def kq_obs_quantize_workspace(d_out: int, d_in: int, block: int = 128, mode: int = KQ_TRAIL_FP32,
                              with_p: bool = False) -> int:
    return int(lib().kq_obs_quantize_workspace(d_out, d_in, block, mode, int(with_p)))


def kq_obs_quantize(W, Lt, bits: int, group: int, block: int, codes, scale, zero, col_loss=None,
                    pre_q=None, ws=None, stream=None, mode: int = KQ_TRAIL_FP32, info=None, Pt=None) -> None:
    """mode: KQ_TRAIL_FP32 (fp32-ordered trailing update, bit-exact) or KQ_TRAIL_3XTF32.
    Pt: P^T from kq_gptaq_p for the GPTAQ drift correction, or None (GPTQ mode)."""
    d_out, d_in = W.shape
    ng = 1 if group == 0 else -(-d_in // group)
    _need(W, "W", torch.float32)
    _need(Lt, "Lt", torch.float32, (d_in, d_in))
    _need(Pt, "Pt", torch.float32, (d_in, d_in))
    _need(codes, "codes", torch.uint8, (d_out, d_in))
    _need(scale, "scale", torch.float32, (d_out, ng))
    _need(zero, "zero", torch.int32, (d_out, ng))
    _need(col_loss, "col_loss", torch.float32, (d_in,))
    _need(pre_q, "pre_q", torch.float32, (d_out, d_in))
    _need(ws, "ws", torch.uint8)
    _need(info, "info", torch.int32)
    _ok(lib().kq_obs_quantize(_ptr(W), d_out, d_in, _ptr(Lt), _ptr(Pt), bits, group, block, mode, _ptr(codes),
                              _ptr(scale), _ptr(zero), _ptr(col_loss), _ptr(pre_q), _ptr(info), _ptr(ws),
                              0 if ws is None else ws.numel(), _stream(stream)), "kq_obs_quantize")


def kq_packed_codes_bytes(d_out: int, d_in: int, bits: int) -> int:
    return int(lib().kq_packed_codes_bytes(d_out, d_in, bits))


def kq_pack_codes(codes, bits: int, packed, stream=None) -> None:
    """codes [d_out, d_in] uint8 -> packed words (int32 tensor of kq_packed_codes_bytes / 4)."""
    d_out, d_in = codes.shape
    _need(codes, "codes", torch.uint8)
    _need(packed, "packed", torch.int32, (kq_packed_codes_bytes(d_out, d_in, bits) // 4,))
    _ok(lib().kq_pack_codes(_ptr(codes), d_out, d_in, bits, _ptr(packed), _stream(stream)), "kq_pack_codes")


def kq_infer_workspace(B: int, d_in: int, d_out: int) -> int:
    return int(lib().kq_infer_workspace(B, d_in, d_out))


def kq_infer(packed, scale, zero, d_out: int, d_in: int, bits: int, group: int, s_x, s_g, sign_u, sign_v, x, y,
             ws, stream=None, info=None) -> None:
    """y [B, d_out] = W^ x for x [B, d_in]: the reverted quantized layer applied with online
    Hadamard transforms (Algorithm 2's revert, Sec. 3.2). info: optional int32 device word
    for a timed-out weight stream (read with kq_check)."""
    B = x.shape[0]
    _need(packed, "packed", torch.int32)
    _need(scale, "scale", torch.float32)
    _need(zero, "zero", torch.int32)
    _need(s_x, "s_x", torch.float32, (d_in,))
    _need(s_g, "s_g", torch.float32, (d_out,))
    _need(sign_u, "sign_u", torch.int8, (d_out,))
    _need(sign_v, "sign_v", torch.int8, (d_in,))
    _need(x, "x", torch.float32, (B, d_in))
    _need(y, "y", torch.float32, (B, d_out))
    _need(ws, "ws", torch.uint8)
    _need(info, "info", torch.int32)
    _ok(lib().kq_infer(_ptr(packed), _ptr(scale), _ptr(zero), d_out, d_in, bits, group, _ptr(s_x), _ptr(s_g),
                       _ptr(sign_u), _ptr(sign_v), _ptr(x), B, _ptr(y), _ptr(info), _ptr(ws),
                       0 if ws is None else ws.numel(), _stream(stream)), "kq_infer")


class _KvCache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("table", ctypes.c_void_p)] + [
        (n, ctypes.c_int64) for n in ("pages", "page", "kv_heads", "dim", "batch", "table_ld")]


def kq_kv_cache_bytes(page: int, dim: int) -> int:
    """Bytes of one page and head of the 4-bit cache: a cache is uint8 [pages, kv_heads, this]."""
    return page * (dim + 8)


def _cache(cache, table, dim: int) -> _KvCache:
    _need(cache, "cache", torch.uint8)
    _need(table, "table", torch.int32)
    if cache.dim() != 3 or table.dim() != 2:
        raise ValueError("cache must be [pages, kv_heads, page * (dim + 8)], table [batch, pages of a sequence]")
    pages, heads, size = cache.shape
    page, rest = divmod(size, dim + 8)
    if rest:
        raise ValueError(f"cache's last dimension must be page * (dim + 8) with dim = {dim}, got {size}")
    batch, table_ld = table.shape
    return _KvCache(cache.data_ptr(), table.data_ptr(), pages, page, heads, dim, batch, table_ld)


_DTYPES = {torch.bfloat16: KQ_BF16, torch.float32: KQ_F32}


def _dtype(t, name):
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return d


def _rows3(t, name, heads=None, dim=None):
    if t.dim() != 3 or (t.stride(2) != 1 and t.numel()):
        raise ValueError(f"{name} must be [tokens, heads, dim] with unit stride in dim")
    if (heads is not None and t.shape[1] != heads) or (dim is not None and t.shape[2] != dim):
        raise ValueError(f"{name} must have {heads} heads of {dim}, got {tuple(t.shape)}")


def kq_kv_append(k, v, start, lens, cache, table, lens_out=None, acc=None, pos=None, seen=None, seen_out=None, info=None,
                 stream=None) -> None:
    """k, v [T, kv_heads, dim] (bf16 or fp32, any token and head strides) into the 4-bit cache at the
    slots that follow lens [batch]; start [batch + 1] gives each sequence's tokens. acc, pos [batch,
    kv_heads, S]: weight 0 and position seen + index at the new slots."""
    dtype = _dtype(k, "k")
    _rows3(k, "k", cache.shape[1])
    _rows3(v, "v", cache.shape[1], k.shape[2])
    if v.dtype != k.dtype or v.shape != k.shape:
        raise ValueError("k and v must have one shape and type")
    _need(v, "v", k.dtype, contiguous=False)
    c = _cache(cache, table, k.shape[2])
    one, S = (c.batch,), 0
    _need(start, "start", torch.int32, (c.batch + 1,))
    _need(lens, "lens", torch.int32, one)
    if lens_out is not None:
        _need(lens_out, "lens_out", torch.int32, one)
    if seen is not None:
        _need(seen, "seen", torch.int32, one)
    if seen_out is not None:
        _need(seen_out, "seen_out", torch.int32, one)
    if acc is not None:
        S = acc.shape[-1]
        _need(acc, "acc", torch.float32, (c.batch, c.kv_heads, S))
    if pos is not None:
        if acc is not None and pos.shape != acc.shape:
            raise ValueError("acc and pos must have one shape")
        S = pos.shape[-1]
        _need(pos, "pos", torch.int32, (c.batch, c.kv_heads, S))
    if info is not None:
        _need(info, "info", torch.int32)
    k0, k1, _ = k.stride()
    v0, v1, _ = v.stride()
    _ok(lib().kq_kv_append(ctypes.byref(c), k.data_ptr(), v.data_ptr(), dtype, k.shape[0], k0, k1, v0, v1,
                           _ptr(start), _ptr(lens), _ptr(lens_out), _ptr(acc), _ptr(pos), S, _ptr(seen),
                           _ptr(seen_out), _ptr(info), _stream(stream)), "kq_kv_append")


def kq_kv_read(cache, table, start, first, lens, k, v, info=None, stream=None) -> None:
    """k, v [T, kv_heads, dim] (bf16 or fp32, contiguous) = the values of cached tokens: token i of
    sequence b is slot first[b] + i - start[b] (first None: 0); at or beyond lens[b] it reads 0."""
    dtype = _dtype(k, "k")
    _rows3(k, "k", cache.shape[1])
    _need(k, "k", k.dtype)
    _need(v, "v", k.dtype, tuple(k.shape))
    c = _cache(cache, table, k.shape[2])
    _need(start, "start", torch.int32, (c.batch + 1,))
    _need(first, "first", torch.int32, (c.batch,))
    _need(lens, "lens", torch.int32, (c.batch,))
    _need(info, "info", torch.int32)
    _ok(lib().kq_kv_read(ctypes.byref(c), _ptr(start), _ptr(first), _ptr(lens), dtype, k.shape[0], _ptr(k), _ptr(v),
                         _ptr(info), _stream(stream)), "kq_kv_read")


def kq_kv_attend_workspace(q, cache, table, acc=None) -> int:
    """Bytes of kq_kv_attend's workspace for these tensors."""
    return int(lib().kq_kv_attend_workspace(q.shape[0], q.shape[1], cache.shape[1], q.shape[2],
                                            0 if acc is None else acc.shape[-1]))


def kq_kv_attend(q, start, lens, cache, table, out, ws, scale: float, lse=None, acc=None, info=None, stream=None) -> None:
    """out [T, q_heads, dim] = attention of q over the cached slots of each token's sequence (the
    tokens' own keys are its last slots; token i sees what was cached up to itself). lse [T, q_heads]:
    the log-sums. acc [batch, kv_heads, S] += each slot's weight summed over heads and tokens."""
    dtype = _dtype(q, "q")
    _rows3(q, "q")
    T, heads, dim = q.shape
    c = _cache(cache, table, dim)
    _need(out, "out", q.dtype, (T, heads, dim))
    _need(lse, "lse", torch.float32, (T, heads))
    _need(start, "start", torch.int32, (c.batch + 1,))
    _need(lens, "lens", torch.int32, (c.batch,))
    S = 0
    if acc is not None:
        S = acc.shape[-1]
        _need(acc, "acc", torch.float32, (c.batch, c.kv_heads, S))
    _need(ws, "ws", torch.uint8)
    _need(info, "info", torch.int32)
    _ok(lib().kq_kv_attend(ctypes.byref(c), _ptr(q), dtype, T, heads, q.stride(0), q.stride(1), _ptr(start), _ptr(lens),
                           float(scale), _ptr(out), _ptr(lse), _ptr(acc), S, _ptr(info), _ptr(ws),
                           0 if ws is None else ws.numel(), _stream(stream)), "kq_kv_attend")


def kq_kv_evict_workspace(acc, budget: int) -> int:
    """Bytes of kq_kv_evict's workspace for weights acc [batch, kv_heads, S]."""
    return int(lib().kq_kv_evict_workspace(acc.shape[0], acc.shape[1], acc.shape[2], int(budget)))


def kq_kv_evict(cache, table, lens, acc, pos, seen, dim: int, budget: int, recent: int, sink: int, lens_out, acc_out,
                pos_out, ws, info=None, stream=None) -> None:
    """Cuts each sequence and head back to `budget` slots: the last `recent` and first `sink`
    positions and the slots of the largest acc stay; kept slots beyond the budget move into the
    freed ones. acc_out, pos_out may be acc, pos; lens_out = min(lens, budget) may not be lens."""
    c = _cache(cache, table, dim)
    S = acc.shape[-1]
    shape = (c.batch, c.kv_heads, S)
    for t, name, ty in ((acc, "acc", torch.float32), (pos, "pos", torch.int32), (acc_out, "acc_out", torch.float32),
                        (pos_out, "pos_out", torch.int32)):
        _need(t, name, ty, shape)
    for t, name in ((lens, "lens"), (seen, "seen"), (lens_out, "lens_out")):
        _need(t, name, torch.int32, (c.batch,))
    _need(ws, "ws", torch.uint8)
    _need(info, "info", torch.int32)
    _ok(lib().kq_kv_evict(ctypes.byref(c), _ptr(lens), _ptr(acc), _ptr(pos), _ptr(seen), S, int(budget), int(recent),
                          int(sink), _ptr(lens_out), _ptr(acc_out), _ptr(pos_out), _ptr(info), _ptr(ws),
                          0 if ws is None else ws.numel(), _stream(stream)), "kq_kv_evict")


def _logits(t, name):
    if t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1 and t.numel()):
        raise ValueError(f"{name} must be [T, V] with unit column stride")
    return _dtype(t, name)


def _row_stride(t):
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def kq_token_logprobs(logits, target, logp, entropy=None, lse=None, top_id=None, top_logp=None, info=None,
                      stream=None) -> None:
    """logp [T] of the target tokens [T] int64 (negative: not scored), with the entropy and log-sum
    of each row of logits [T, V] (bf16 or fp32) and its top_id.shape[1] most likely tokens."""
    dtype = _logits(logits, "logits")
    T, V = logits.shape
    top = 0 if top_id is None else top_id.shape[-1]
    _need(target, "target", torch.int64, (T,))
    for t, name in ((logp, "logp"), (entropy, "entropy"), (lse, "lse")):
        _need(t, name, torch.float32, (T,))
    _need(top_id, "top_id", torch.int32, (T, top))
    if (top_id is None) != (top_logp is None):
        raise ValueError("top_id and top_logp go together")
    _need(top_logp, "top_logp", torch.float32, (T, top))
    _need(info, "info", torch.int32)
    _ok(lib().kq_token_logprobs(_ptr(logits), dtype, T, V, _row_stride(logits), _ptr(target), top, _ptr(logp),
                                _ptr(entropy), _ptr(lse), _ptr(top_id), _ptr(top_logp), _ptr(info), _stream(stream)),
        "kq_token_logprobs")


def kq_token_logprobs_grad(logits, target, lse, g_logp, grad, entropy=None, g_entropy=None, info=None,
                           stream=None) -> None:
    """grad [T, V] = the gradient of sum(g_logp * logp + g_entropy * entropy) with respect to logits;
    lse and entropy from kq_token_logprobs. grad may be logits."""
    dtype = _logits(logits, "logits")
    T, V = logits.shape
    if _logits(grad, "grad") != dtype or grad.shape != logits.shape:
        raise ValueError("grad must have the shape and type of logits")
    _need(target, "target", torch.int64, (T,))
    for t, name in ((lse, "lse"), (g_logp, "g_logp"), (entropy, "entropy"), (g_entropy, "g_entropy")):
        _need(t, name, torch.float32, (T,))
    _need(info, "info", torch.int32)
    _ok(lib().kq_token_logprobs_grad(_ptr(logits), dtype, T, V, _row_stride(logits), _ptr(target), _ptr(lse),
                                     _ptr(entropy), _ptr(g_logp), _ptr(g_entropy), _ptr(grad), _row_stride(grad),
                                     _ptr(info), _stream(stream)), "kq_token_logprobs_grad")


def kq_dequant_revert(codes, scale, zero, group: int, s_x, s_g, sign_u, sign_v, W_hat, stream=None):
    d_out, d_in = codes.shape
    _need(codes, "codes", torch.uint8)
    _need(scale, "scale", torch.float32)
    _need(zero, "zero", torch.int32)
    _need(W_hat, "W_hat", torch.float32, (d_out, d_in))
    _ok(lib().kq_dequant_revert(_ptr(codes), _ptr(scale), _ptr(zero), d_out, d_in, group, _ptr(s_x),
                                _ptr(s_g), _ptr(sign_u), _ptr(sign_v), _ptr(W_hat), _stream(stream)),
        "kq_dequant_revert")


def kq_proxy_loss_workspace(d_out: int, d_in: int) -> int:
    return int(lib().kq_proxy_loss_workspace(d_out, d_in))


def kq_proxy_loss(W, W_hat, H_X, H_G, loss, ws, stream=None) -> None:
    d_out, d_in = W.shape
    _need(W, "W", torch.float32)
    _need(W_hat, "W_hat", torch.float32, (d_out, d_in))
    _need(H_X, "H_X", torch.float32, (d_in, d_in))
    _need(H_G, "H_G", torch.float32, (d_out, d_out))
    _need(loss, "loss", torch.float64, (1,))
    _need(ws, "ws", torch.uint8)
    _ok(lib().kq_proxy_loss(_ptr(W), _ptr(W_hat), d_out, d_in, _ptr(H_X), _ptr(H_G), _ptr(loss),
                            _ptr(ws), ws.numel(), _stream(stream)), "kq_proxy_loss")
