"""ctypes binding of libjab.so (include/jab.h). Argument marshalling only.

Each function has the name of its C entry point, takes torch tensors where the C function takes
device pointers, checks dtype / device / contiguity (the C side checks shapes, alignment and
workspace size), calls the library on the current CUDA stream (or the one given), and raises
JabError on a non-OK status.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

JAB_OK = 0
_STATUS_NAMES = {0: "JAB_OK", 1: "JAB_ERR_INVALID_ARG", 2: "JAB_ERR_UNSUPPORTED", 3: "JAB_ERR_CUDA",
                 4: "JAB_ERR_NONFINITE", 5: "JAB_ERR_RANGE", 6: "JAB_ERR_TIMEOUT",
                 7: "JAB_ERR_SCRATCH_LIMIT", 8: "JAB_ERR_INTERNAL", 9: "JAB_ERR_DEVICE_ASSERT"}

_HERE = os.path.dirname(os.path.abspath(__file__))


def lib_path() -> str:
    """libjab.so, or the checked build libjab_checked.so when the environment sets JAB_CHECKED=1."""
    name = "libjab_checked.so" if os.environ.get("JAB_CHECKED", "0") == "1" else "libjab.so"
    return os.path.join(_HERE, name)


class JabError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__(f"{where}: {_STATUS_NAMES.get(self.status, self.status)} "
                         f"({jab_status_string(self.status)})")


class BlockDesc(ctypes.Structure):
    """jab_block_desc: one attention block (Section 2.1; App. C)."""

    _fields_ = [("d_model", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("group_size", ctypes.c_int32), ("use_rope", ctypes.c_int32),
                ("rope_theta", ctypes.c_float), ("softmax_scale", ctypes.c_float)]

    def as_dict(self) -> dict:
        return {name: getattr(self, name) for name, _ in self._fields_}


def desc_from_shape(shape, group_size: int) -> BlockDesc:
    """BlockDesc from a workloads.BlockShape-like object (d_model, heads, head_dim, RoPE)."""
    return BlockDesc(shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, group_size,
                     1 if shape.use_rope else 0, float(shape.rope_theta), 0.0)


class _KvCacheDesc(ctypes.Structure):
    """jab_kv_cache"""

    _fields_ = [("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("bits", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("n_pages", ctypes.c_int64),
                ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p)]


_P = ctypes.c_void_p
_LIB = None


def lib() -> ctypes.CDLL:
    """Loads libjab.so; raises if it has not been built (there is no fallback)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2609_34866_gb300.build` "
                           "or __graft_entry__.build()")
    L = ctypes.CDLL(path)
    D = ctypes.POINTER(BlockDesc)
    i32, f32, sz = ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    L.jab_workspace_size.argtypes = [D, i32, i32, i32, i32]
    L.jab_workspace_size.restype = sz
    L.jab_reference_forward.argtypes = [D, i32, i32, _P, _P, _P, _P, _P, _P, sz, _P]
    L.jab_loss_forward.argtypes = [D, i32, i32, _P, _P, _P, i32, ctypes.POINTER(i32),
                                   ctypes.POINTER(_P), _P, _P, _P, sz, _P]
    L.jab_loss_forward_noalloc.argtypes = [D, i32, i32, _P, _P, _P, i32, ctypes.POINTER(i32),
                                           ctypes.POINTER(_P), _P, _P, _P]
    L.jab_loss_backward_scales.argtypes = [D, i32, i32, _P, _P, _P, i32, _P, f32, _P, _P, _P, sz, _P]
    L.jab_loss_backward_weights.argtypes = [D, i32, i32, _P, _P, _P, i32, _P, _P, _P, _P, _P, sz, _P]
    L.jab_prepare_x.argtypes = [D, i32, i32, _P, _P, sz, _P]
    L.jab_loss_backward_scales_prepared.argtypes = [D, i32, i32, _P, _P, _P, i32, _P, f32, _P, _P,
                                                    _P, sz, _P]
    L.jab_loss_backward_scales_kl.argtypes = [D, i32, i32, _P, _P, _P, _P, _P, i32, _P, f32, f32,
                                              _P, _P, _P, _P, sz, _P]
    L.jab_flip_rate.argtypes = [_P, _P, ctypes.c_int64, _P, _P]
    L.jab_reference_projection.argtypes = [D, i32, i32, _P, _P, _P, _P, sz, _P]
    L.jab_hutchinson_trace.argtypes = [D, i32, i32, _P, _P, _P, _P, i32, ctypes.c_uint64, _P, _P,
                                       _P, sz, _P]
    L.jab_rademacher_probes.argtypes = [ctypes.c_uint64, ctypes.c_int64, ctypes.c_int64, _P, _P]
    L.jab_omega_scores.argtypes = [D, _P, i32, ctypes.POINTER(i32), ctypes.POINTER(_P), _P, i32,
                                   _P, _P, _P, sz, _P]
    L.jab_loss_forward_kl.argtypes = [D, i32, i32, _P, _P, _P, _P, i32, ctypes.POINTER(i32),
                                      ctypes.POINTER(_P), f32, _P, _P, _P, _P, _P, sz, _P]
    L.jab_quantize.argtypes = [D, i32, _P, _P, _P, _P, _P]
    L.jab_allocate_bits.argtypes = [_P, _P, _P, i32, i32, ctypes.c_double, i32, _P]
    L.jab_init_scales.argtypes = [D, i32, i32, _P, _P, _P]
    L.jab_get_device_status.argtypes = [_P]
    L.jab_set_deterministic.argtypes = [i32]
    L.jab_selftest_bounds_check.argtypes = [_P, i32, _P]
    L.jab_selftest_wait_timeout.argtypes = [_P]
    L.jab_status_string.argtypes = [i32]
    L.jab_status_string.restype = ctypes.c_char_p
    L.jab_timing_enable.argtypes = [i32]
    L.jab_timing_collect.argtypes = []
    L.jab_timing_count.argtypes = []
    L.jab_timing_count.restype = i32
    L.jab_timing_get.argtypes = [i32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_double),
                                 ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]
    L.jab_timing_reset.argtypes = []
    KV = ctypes.POINTER(_KvCacheDesc)
    i64 = ctypes.c_int64
    L.jab_quantized_linear_workspace_size.argtypes = [i64, i32, i32]
    L.jab_quantized_linear_workspace_size.restype = sz
    L.jab_quantized_linear.argtypes = [i64, i32, i32, _P, i32, i64, _P, _P, _P, i32, i64, _P, sz, _P]
    L.jab_rope_table.argtypes = [i32, i32, f32, _P, _P, _P]
    L.jab_kv_write.argtypes = [KV, i64, i32, _P, i32, i64, _P, _P, _P, _P, i32, _P, _P]
    L.jab_kv_read.argtypes = [KV, i32, _P, i32, _P, _P, i32, _P, _P, i32, _P]
    L.jab_kv_attention_workspace_size.argtypes = [KV, i32, i64, i32, i32, i32, i32]
    L.jab_kv_attention_workspace_size.restype = sz
    L.jab_kv_attention.argtypes = [KV, i32, i64, i32, _P, i32, i64, _P, _P, i32, _P, i32, i32, i32, i32, f32,
                                   _P, i64, _P, _P, sz, _P]
    for fn in ("jab_reference_forward", "jab_loss_forward", "jab_loss_forward_noalloc",
               "jab_quantized_linear", "jab_rope_table", "jab_kv_write", "jab_kv_read", "jab_kv_attention",
               "jab_loss_backward_scales", "jab_loss_backward_weights", "jab_allocate_bits",
               "jab_prepare_x", "jab_loss_backward_scales_prepared", "jab_flip_rate",
               "jab_loss_backward_scales_kl",
               "jab_reference_projection", "jab_loss_forward_kl", "jab_hutchinson_trace",
               "jab_omega_scores", "jab_rademacher_probes",
               "jab_quantize", "jab_init_scales", "jab_get_device_status", "jab_timing_enable",
               "jab_selftest_wait_timeout", "jab_set_deterministic", "jab_selftest_bounds_check",
               "jab_timing_collect", "jab_timing_get", "jab_timing_reset"):
        getattr(L, fn).restype = i32
    _LIB = L
    return L


def jab_status_string(status: int) -> str:
    try:
        return lib().jab_status_string(int(status)).decode()
    except RuntimeError:
        return _STATUS_NAMES.get(int(status), "unknown")


def _ptr(t: Optional[torch.Tensor], dtype=None, name="tensor") -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


# The current stream's handle alone, where torch has it: building its stream object takes longer than a launch.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(status: int, where: str):
    if status != JAB_OK:
        raise JabError(status, where)


def jab_workspace_size(desc: BlockDesc, B: int, T: int, n_cand: int = 1, with_bwd: bool = True) -> int:
    return int(lib().jab_workspace_size(ctypes.byref(desc), B, T, n_cand, 1 if with_bwd else 0))


class Workspace:
    """A caller-owned device workspace (a uint8 torch tensor) sized by jab_workspace_size."""

    def __init__(self, desc: BlockDesc, B: int, T: int, n_cand: int = 1, with_bwd: bool = True,
                 device=None):
        self.nbytes = jab_workspace_size(desc, B, T, n_cand, with_bwd)
        if self.nbytes == 0:
            raise JabError(1, "jab_workspace_size")
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8,
                               device=device or torch.device("cuda", torch.cuda.current_device()))

    @property
    def ptr(self) -> int:
        return self.buf.data_ptr()


def jab_reference_forward(desc, B, T, X, W, A_ref, ws: Workspace, lse=None, a_sqnorm=None,
                          stream=None):
    st = lib().jab_reference_forward(
        ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), _ptr(W, torch.bfloat16, "W"),
        _ptr(A_ref, torch.float32, "A_ref"), _ptr(lse, torch.float32, "lse"),
        _ptr(a_sqnorm, torch.float64, "a_sqnorm"), ws.ptr, ws.nbytes, _stream(stream))
    _check(st, "jab_reference_forward")


def jab_loss_forward(desc, B, T, X, W, A_ref, bits: Sequence[int], scales: Sequence[torch.Tensor],
                     loss, ws: Workspace, sse_parts=None, stream=None):
    n = len(bits)
    if len(scales) != n:
        raise ValueError("bits and scales must have the same length")
    bits_arr = (ctypes.c_int32 * n)(*[int(b) for b in bits])
    sc_arr = (ctypes.c_void_p * n)(*[_ptr(s, torch.float32, "scales") for s in scales])
    st = lib().jab_loss_forward(
        ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), _ptr(W, torch.bfloat16, "W"),
        _ptr(A_ref, torch.float32, "A_ref"), n, bits_arr, sc_arr,
        _ptr(loss, torch.float64, "loss"), _ptr(sse_parts, torch.float64, "sse_parts"), ws.ptr,
        ws.nbytes, _stream(stream))
    _check(st, "jab_loss_forward")


def jab_reference_projection(desc, B, T, X, W, QKV_ref, ws: Workspace, stream=None):
    """Teacher [Q|K|V] (rotated, fp16 [B, T, D]) for the KL term."""
    st = lib().jab_reference_projection(
        ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), _ptr(W, torch.bfloat16, "W"),
        _ptr(QKV_ref, torch.float16, "QKV_ref"), ws.ptr, ws.nbytes, _stream(stream))
    _check(st, "jab_reference_projection")


def jab_loss_forward_kl(desc, B, T, X, W, A_ref, QKV_ref, bits: Sequence[int],
                        scales: Sequence[torch.Tensor], lambda_kl: float, loss, ws: Workspace,
                        mse=None, kl=None, kl_rows=None, stream=None):
    """Both terms of Eq. 3 per candidate: loss = mse + lambda_kl * kl (fp64 [n_cand] each)."""
    n = len(bits)
    if len(scales) != n:
        raise ValueError("bits and scales must have the same length")
    bits_arr = (ctypes.c_int32 * n)(*[int(b) for b in bits])
    sc_arr = (ctypes.c_void_p * n)(*[_ptr(s, torch.float32, "scales") for s in scales])
    st = lib().jab_loss_forward_kl(
        ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), _ptr(W, torch.bfloat16, "W"),
        _ptr(A_ref, torch.float32, "A_ref"), _ptr(QKV_ref, torch.float16, "QKV_ref"), n, bits_arr,
        sc_arr, float(lambda_kl), _ptr(loss, torch.float64, "loss"), _ptr(mse, torch.float64, "mse"),
        _ptr(kl, torch.float64, "kl"), _ptr(kl_rows, torch.float32, "kl_rows"), ws.ptr, ws.nbytes,
        _stream(stream))
    _check(st, "jab_loss_forward_kl")


def jab_hutchinson_trace(desc, B, T, X, W, A_ref, lse_ref, n_probes: int, seed: int, trace,
                         ws: Workspace, vhv=None, stream=None):
    """Tr(H) of L_JAB at the float weights from n_probes Rademacher probes (Section 2.4, Eq. 5)."""
    st = lib().jab_hutchinson_trace(
        ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), _ptr(W, torch.bfloat16, "W"),
        _ptr(A_ref, torch.float32, "A_ref"), _ptr(lse_ref, torch.float32, "lse_ref"), int(n_probes),
        int(seed) & ((1 << 64) - 1), _ptr(trace, torch.float64, "trace"),
        _ptr(vhv, torch.float64, "vhv"), ws.ptr, ws.nbytes, _stream(stream))
    _check(st, "jab_hutchinson_trace")


def jab_rademacher_probes(seed: int, first: int, out, stream=None):
    """Probe entries first .. first + out.numel() - 1 of jab_hutchinson_trace's sequence (fp16 +-1)."""
    st = lib().jab_rademacher_probes(int(seed) & ((1 << 64) - 1), int(first), int(out.numel()),
                                     _ptr(out, torch.float16, "out"), _stream(stream))
    _check(st, "jab_rademacher_probes")


def jab_omega_scores(desc, W, bits: Sequence[int], scales: Sequence[torch.Tensor], trace,
                     layers_after: int, c1, ws: Workspace, c2=None, stream=None):
    """Eq. 6: C1 = Tr(H) ||Q_b(W) - W||^2 per candidate (and C2 = layers_after * C1)."""
    n = len(bits)
    if len(scales) != n:
        raise ValueError("bits and scales must have the same length")
    bits_arr = (ctypes.c_int32 * n)(*[int(b) for b in bits])
    sc_arr = (ctypes.c_void_p * n)(*[_ptr(s, torch.float32, "scales") for s in scales])
    st = lib().jab_omega_scores(ctypes.byref(desc), _ptr(W, torch.bfloat16, "W"), n, bits_arr,
                                sc_arr, _ptr(trace, torch.float64, "trace"), int(layers_after),
                                _ptr(c1, torch.float64, "c1"), _ptr(c2, torch.float64, "c2"),
                                ws.ptr, ws.nbytes, _stream(stream))
    _check(st, "jab_omega_scores")


def jab_loss_forward_noalloc(desc, B, T, X, W, A_ref, bits: Sequence[int],
                             scales: Sequence[torch.Tensor], loss, sse_parts=None, stream=None):
    """jab_loss_forward on the library's fixed device scratch (no workspace argument): for callers
    that cannot allocate device memory. Raises JabError(JAB_ERR_SCRATCH_LIMIT) when the problem
    needs more scratch than JAB_NOALLOC_SCRATCH_BYTES."""
    n = len(bits)
    if len(scales) != n:
        raise ValueError("bits and scales must have the same length")
    bits_arr = (ctypes.c_int32 * n)(*[int(b) for b in bits])
    sc_arr = (ctypes.c_void_p * n)(*[_ptr(s, torch.float32, "scales") for s in scales])
    st = lib().jab_loss_forward_noalloc(
        ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), _ptr(W, torch.bfloat16, "W"),
        _ptr(A_ref, torch.float32, "A_ref"), n, bits_arr, sc_arr,
        _ptr(loss, torch.float64, "loss"), _ptr(sse_parts, torch.float64, "sse_parts"),
        _stream(stream))
    _check(st, "jab_loss_forward_noalloc")


def jab_loss_backward_scales(desc, B, T, X, W, A_ref, bits: int, scales, kappa: float, loss,
                             grad_scales, ws: Workspace, stream=None):
    st = lib().jab_loss_backward_scales(
        ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), _ptr(W, torch.bfloat16, "W"),
        _ptr(A_ref, torch.float32, "A_ref"), int(bits), _ptr(scales, torch.float32, "scales"),
        float(kappa), _ptr(loss, torch.float64, "loss"),
        _ptr(grad_scales, torch.float32, "grad_scales"), ws.ptr, ws.nbytes, _stream(stream))
    _check(st, "jab_loss_backward_scales")


def jab_prepare_x(desc, B, T, X, ws: Workspace, stream=None):
    """Converts X into the workspace's fp16 copy for jab_loss_backward_scales_prepared."""
    st = lib().jab_prepare_x(ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), ws.ptr,
                             ws.nbytes, _stream(stream))
    _check(st, "jab_prepare_x")


def jab_loss_backward_scales_prepared(desc, B, T, X, W, A_ref, bits: int, scales, kappa: float,
                                      loss, grad_scales, ws: Workspace, stream=None):
    """jab_loss_backward_scales on the fp16 X that jab_prepare_x left in `ws`."""
    st = lib().jab_loss_backward_scales_prepared(
        ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), _ptr(W, torch.bfloat16, "W"),
        _ptr(A_ref, torch.float32, "A_ref"), int(bits), _ptr(scales, torch.float32, "scales"),
        float(kappa), _ptr(loss, torch.float64, "loss"),
        _ptr(grad_scales, torch.float32, "grad_scales"), ws.ptr, ws.nbytes, _stream(stream))
    _check(st, "jab_loss_backward_scales_prepared")


def jab_loss_backward_scales_kl(desc, B, T, X, W, A_ref, QKV_ref, lse_ref, bits: int, scales,
                                kappa: float, lambda_kl: float, loss, grad_scales, ws: Workspace,
                                kl=None, stream=None):
    """Scale gradient of MSE + lambda_kl * KL (Eq. 3 with both terms); the teacher's projection and
    log-sum-exp from jab_reference_projection / jab_reference_forward."""
    st = lib().jab_loss_backward_scales_kl(
        ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), _ptr(W, torch.bfloat16, "W"),
        _ptr(A_ref, torch.float32, "A_ref"), _ptr(QKV_ref, torch.float16, "QKV_ref"),
        _ptr(lse_ref, torch.float32, "lse_ref"), int(bits), _ptr(scales, torch.float32, "scales"),
        float(kappa), float(lambda_kl), _ptr(loss, torch.float64, "loss"),
        _ptr(kl, torch.float64, "kl"), _ptr(grad_scales, torch.float32, "grad_scales"), ws.ptr,
        ws.nbytes, _stream(stream))
    _check(st, "jab_loss_backward_scales_kl")


def jab_flip_rate(codes_a, codes_b, count, stream=None):
    """Number of positions where two int8 code tensors differ (Eq. 15), into count (int64 [1])."""
    if codes_a.numel() != codes_b.numel():
        raise ValueError("code arrays differ in size")
    if codes_a.numel() == 0:
        codes_a = codes_b = None
    n = 0 if codes_a is None else int(codes_a.numel())
    st = lib().jab_flip_rate(_ptr(codes_a, torch.int8, "codes_a"), _ptr(codes_b, torch.int8, "codes_b"),
                             n, _ptr(count, torch.int64, "count"), _stream(stream))
    _check(st, "jab_flip_rate")


def jab_loss_backward_weights(desc, B, T, X, W, A_ref, bits: int, scales, loss, grad_w=None,
                              grad_sqnorm=None, ws: Workspace = None, stream=None):
    """Loss and the STE weight gradient dL/dw_hat (fp32 [D, d]) and/or its squared norm (fp64 [1])."""
    st = lib().jab_loss_backward_weights(
        ctypes.byref(desc), B, T, _ptr(X, torch.bfloat16, "X"), _ptr(W, torch.bfloat16, "W"),
        _ptr(A_ref, torch.float32, "A_ref"), int(bits), _ptr(scales, torch.float32, "scales"),
        _ptr(loss, torch.float64, "loss"), _ptr(grad_w, torch.float32, "grad_w"),
        _ptr(grad_sqnorm, torch.float64, "grad_sqnorm"), ws.ptr, ws.nbytes, _stream(stream))
    _check(st, "jab_loss_backward_weights")


def jab_allocate_bits(omega, widths, n_weights, avg_bits: float, method: str = "greedy"):
    """Width per layer minimising the summed score within avg_bits per weight (Eq. 7). Host only.

    omega: [L, K] scores (any array-like of floats); widths: K increasing ints; n_weights: L ints.
    method: "greedy" or "pareto". Returns a list of L widths."""
    import numpy as np
    om = np.ascontiguousarray(np.asarray(omega, dtype=np.float64))
    w = np.ascontiguousarray(np.asarray(widths, dtype=np.int32))
    n = np.ascontiguousarray(np.asarray(n_weights, dtype=np.int64))
    if om.ndim != 2 or om.shape != (n.size, w.size):
        raise ValueError("omega must be [len(n_weights), len(widths)]")
    out = np.zeros(n.size, dtype=np.int32)
    st = lib().jab_allocate_bits(om.ctypes.data, w.ctypes.data, n.ctypes.data, int(n.size),
                                 int(w.size), float(avg_bits), {"greedy": 0, "pareto": 1}[method],
                                 out.ctypes.data)
    _check(st, "jab_allocate_bits")
    return [int(b) for b in out]


def jab_quantize(desc, bits, W, scales, codes=None, w_hat=None, stream=None):
    st = lib().jab_quantize(ctypes.byref(desc), int(bits), _ptr(W, torch.bfloat16, "W"),
                            _ptr(scales, torch.float32, "scales"), _ptr(codes, torch.int8, "codes"),
                            _ptr(w_hat, torch.float32, "w_hat"), _stream(stream))
    _check(st, "jab_quantize")


def jab_init_scales(desc, bits, mode, W, scales, stream=None):
    st = lib().jab_init_scales(ctypes.byref(desc), int(bits), int(mode),
                               _ptr(W, torch.bfloat16, "W"), _ptr(scales, torch.float32, "scales"),
                               _stream(stream))
    _check(st, "jab_init_scales")


# ---------------------------------------------------------------- serving a fitted block
_DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}


def _dtype(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float16, bfloat16 or float32, got {t.dtype}")
    return _DTYPES[t.dtype]


def _rows(t: torch.Tensor, width: int, name: str, rows: Optional[int] = None):
    """(pointer, row pitch) of a CUDA tensor of rows of `width` contiguous elements: the first dimension
    may have any stride, the others are flattened."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    shape, strides, have = t.shape, t.stride(), 1
    for d in range(len(shape) - 1, 0, -1):
        if shape[d] != 1 and strides[d] != have:
            have = -1
            break
        have *= shape[d]
    if len(shape) < 2 or have != width:
        raise ValueError(f"{name} must have rows of {width} contiguous elements")
    if rows is not None and shape[0] != rows:
        raise ValueError(f"{name} must have {rows} rows")
    return t.data_ptr(), strides[0] if shape[0] > 1 else width


def _shaped(t: torch.Tensor, shape, dtype, name: str) -> int:
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    return _ptr(t, dtype, name)


def _held(i: int, name: str) -> property:
    """A tensor that a KvCache holds: it may be changed in place (cache.k_scales *= 2), not exchanged."""
    def put(self, t):
        if t is not self._tensors[i]:
            raise AttributeError(f"{name} cannot be exchanged: the calls go by its address; copy_ into it")

    return property(lambda self: self._tensors[i], put)


class KvCache:
    """A paged cache of quantised keys and values (jab_kv_cache): caller-owned tensors k_codes, v_codes
    (uint8 [n_pages, n_kv_heads, page_tokens, head_dim * bits / 8]) and k_scales, v_scales (float32
    [n_pages, n_kv_heads, page_tokens]), allocated here unless given. The calls go by the addresses that these tensors
    have now, so they are held for as long as the cache and cannot be exchanged (their contents can: copy_)."""

    def __init__(self, n_kv_heads: int, head_dim: int, bits: int, page_tokens: int, n_pages: int, device=None,
                 k_codes=None, v_codes=None, k_scales=None, v_scales=None):
        if bits not in (4, 8):
            raise ValueError("bits must be 4 or 8")
        device = device or torch.device("cuda", torch.cuda.current_device())
        lead = (n_pages, n_kv_heads, page_tokens)
        codes = lead + (head_dim * bits // 8,)

        def have(t, shape, dtype, name):
            t = torch.zeros(shape, dtype=dtype, device=device) if t is None else t
            _shaped(t, shape, dtype, name)
            return t

        self.n_kv_heads, self.head_dim, self.bits = int(n_kv_heads), int(head_dim), int(bits)
        self.page_tokens, self.n_pages = int(page_tokens), int(n_pages)
        self._tensors = (have(k_codes, codes, torch.uint8, "k_codes"), have(v_codes, codes, torch.uint8, "v_codes"),
                         have(k_scales, lead, torch.float32, "k_scales"), have(v_scales, lead, torch.float32, "v_scales"))
        self.desc = _KvCacheDesc(self.n_kv_heads, self.head_dim, self.bits, self.page_tokens, self.n_pages,
                                 self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.k_scales.data_ptr(),
                                 self.v_scales.data_ptr())
        self.ref = ctypes.byref(self.desc)

    k_codes, v_codes = _held(0, "k_codes"), _held(1, "v_codes")
    k_scales, v_scales = _held(2, "k_scales"), _held(3, "v_scales")


def jab_quantized_linear_workspace_size(M: int, N: int, K: int) -> int:
    return int(lib().jab_quantized_linear_workspace_size(M, N, K))


def jab_quantized_linear(x, codes, w_scales, y, ws, stream=None):
    """y[m, n] = s_m w_scales[n] sum_k q(x)[m, k] codes[n, k]: x fp16 / bf16 [M, K] quantised to 8 bits per row,
    codes int8 [N, K], the sum exact. y fp16 / bf16 / fp32 [M, N]; ws uint8, jab_quantized_linear_workspace_size
    bytes. Rows of x and y may have a pitch."""
    (M, K), N = x.shape, codes.shape[0]
    xp, ldx = _rows(x, K, "x")
    yp, ldy = _rows(y, N, "y", M)
    st = lib().jab_quantized_linear(M, N, K, xp, _dtype(x, "x"), ldx, _shaped(codes, (N, K), torch.int8, "codes"),
                                    _shaped(w_scales, (N,), torch.float32, "w_scales"), yp, _dtype(y, "y"), ldy,
                                    _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(stream))
    _check(st, "jab_quantized_linear")


def jab_rope_table(cos, sin, theta: float, stream=None):
    """cos and sin of position * theta^(-2j / head_dim) into fp32 [length, head_dim / 2] each."""
    st = lib().jab_rope_table(cos.shape[0], 2 * cos.shape[1], float(theta), _ptr(cos, torch.float32, "cos"),
                              _shaped(sin, cos.shape, torch.float32, "sin"), _stream(stream))
    _check(st, "jab_rope_table")


def jab_kv_write(cache: KvCache, qkv, n_q_heads: int, slots, q_out=None, positions=None, rope=None, stream=None):
    """Rows [Q | K | V] (fp16 / bf16 / fp32 [n_tokens, (n_q_heads + 2 n_kv_heads) * head_dim]): Q and K rotated at
    `positions` (int32 [n_tokens]) by the table rope = (cos, sin), as they are without a table, K and V quantised into the slots (int64
    [n_tokens]; < 0: padding), the rotated Q into q_out [n_tokens, n_q_heads * head_dim]."""
    n, dh = qkv.shape[0], cache.head_dim
    xp, ldx = _rows(qkv, (n_q_heads + 2 * cache.n_kv_heads) * dh, "qkv")
    if rope is not None and positions is None:
        raise ValueError("rope needs positions")
    cos = sin = pos = None
    length = 0
    if rope is not None:
        length = rope[0].shape[0]
        cos, sin = (_shaped(t, (length, dh // 2), torch.float32, "rope") for t in rope)
        pos = _shaped(positions, (n,), torch.int32, "positions")
    if q_out is not None:
        if q_out.numel() != n * n_q_heads * dh:
            raise ValueError("q_out must be [n_tokens, n_q_heads * head_dim] in qkv's type")
        q_out = _ptr(q_out, qkv.dtype, "q_out")
    st = lib().jab_kv_write(cache.ref, n, int(n_q_heads), xp, _dtype(qkv, "qkv"), ldx,
                            _shaped(slots, (n,), torch.int64, "slots"), pos, cos, sin, length, q_out,
                            _stream(stream))
    _check(st, "jab_kv_write")


def jab_kv_read(cache: KvCache, pages, counts, k, v, starts=None, stream=None):
    """Cached tokens starts[b] .. starts[b] + counts[b] - 1 of every sequence as numbers, into k and v (fp16 /
    bf16 / fp32 [n_seqs, T, n_kv_heads, head_dim]; 0 from counts[b] on). pages int32 [n_seqs, max_pages]."""
    B, T = k.shape[0], k.shape[1]
    shape = (B, T, cache.n_kv_heads, cache.head_dim)
    st = lib().jab_kv_read(cache.ref, B, _shaped(pages, (B, pages.shape[1]), torch.int32, "pages"),
                           pages.shape[1], None if starts is None else _shaped(starts, (B,), torch.int32, "starts"),
                           _shaped(counts, (B,), torch.int32, "counts"), T, _shaped(k, shape, k.dtype, "k"),
                           _shaped(v, shape, k.dtype, "v"), _dtype(k, "k"), _stream(stream))
    _check(st, "jab_kv_read")


def jab_kv_attention_workspace_size(cache: KvCache, n_seqs: int, n_tokens: int, n_q_heads: int, max_q_len: int,
                                    max_seq_len: int, shared_len: int = 0) -> int:
    return int(lib().jab_kv_attention_workspace_size(cache.ref, n_seqs, n_tokens, n_q_heads,
                                                     max_q_len, max_seq_len, shared_len))


def jab_kv_attention(cache: KvCache, q, q_start, pages, seq_lens, out, ws, max_q_len: int, max_seq_len: int,
                     shared_len: int = 0, window: int = 0, softmax_scale: float = 0.0, lse=None, stream=None):
    """Attention of the query rows q_start[b] .. q_start[b + 1] - 1 of q (fp16 / bf16 [n_tokens, n_q_heads,
    head_dim]) over the seq_lens[b] cached tokens of their sequence, the last of which are the queries' own:
    causal, within `window` keys if window > 0, the first shared_len keys read once for all sequences. out like
    q, lse fp32 [n_tokens, n_q_heads]; ws uint8, jab_kv_attention_workspace_size bytes."""
    n, B = q.shape[0], seq_lens.shape[0]
    dh = cache.head_dim
    if n == 0:
        return
    hq = q.numel() // (n * dh)
    qp, ldq = _rows(q, hq * dh, "q")
    op, ldo = _rows(out, hq * dh, "out", n)
    if out.dtype != q.dtype:
        raise ValueError("out must have q's type")
    st = lib().jab_kv_attention(
        cache.ref, B, n, hq, qp, _dtype(q, "q"), ldq, _shaped(q_start, (B + 1,), torch.int32, "q_start"),
        _shaped(pages, (B, pages.shape[1]), torch.int32, "pages"), pages.shape[1],
        _shaped(seq_lens, (B,), torch.int32, "seq_lens"), int(max_q_len), int(max_seq_len), int(shared_len),
        int(window), float(softmax_scale), op, ldo,
        None if lse is None else _shaped(lse, (n, hq), torch.float32, "lse"), _ptr(ws, torch.uint8, "ws"), ws.numel(),
        _stream(stream))
    _check(st, "jab_kv_attention")


def jab_selftest_wait_timeout(stream=None):
    """Launches the bounded-wait self-test kernel (its wait runs out after 2 s)."""
    _check(lib().jab_selftest_wait_timeout(_stream(stream)), "jab_selftest_wait_timeout")


def jab_set_deterministic(on: bool):
    """Deterministic-reduction mode, process-wide: every floating-point reduction in a fixed order
    (repeated calls bit-identical). Off by default: the STE weight gradient may then split its GEMM's
    token range and add the partial tiles with atomics."""
    _check(lib().jab_set_deterministic(int(on)), "jab_set_deterministic")


def jab_selftest_bounds_check(buf, n: int, stream=None) -> int:
    """Checked build only: writes buf[0..n] behind bounds checks against an n-element extent (the
    last write is skipped, JAB_ERR_DEVICE_ASSERT raised on the device). Returns the call's status
    (JAB_ERR_UNSUPPORTED from the normal build, which launches nothing)."""
    return int(lib().jab_selftest_bounds_check(_ptr(buf, torch.int32, "buf"), int(n), _stream(stream)))


def jab_get_device_status(stream=None) -> int:
    """Synchronises the stream and returns (and clears) the device-side status word."""
    return int(lib().jab_get_device_status(_stream(stream)))


def jab_timing_enable(on: bool = True):
    _check(lib().jab_timing_enable(1 if on else 0), "jab_timing_enable")


def jab_timing_reset():
    _check(lib().jab_timing_reset(), "jab_timing_reset")


def jab_timing_read() -> dict:
    """Synchronises the recorded events; returns {site: (total_ms, ranges, kernels)}."""
    L = lib()
    _check(L.jab_timing_collect(), "jab_timing_collect")
    out = {}
    for i in range(L.jab_timing_count()):
        name = ctypes.c_char_p()
        ms = ctypes.c_double()
        rng = ctypes.c_int64()
        nk = ctypes.c_int64()
        _check(L.jab_timing_get(i, ctypes.byref(name), ctypes.byref(ms), ctypes.byref(rng),
                                ctypes.byref(nk)), "jab_timing_get")
        out[name.value.decode()] = (ms.value, rng.value, nk.value)
    return out
