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


class _RopeScaling(ctypes.Structure):
    """jab_rope_scaling"""

    _fields_ = [("kind", ctypes.c_int32), ("factor", ctypes.c_float), ("original_length", ctypes.c_float),
                ("low_turns", ctypes.c_float), ("high_turns", ctypes.c_float), ("attention", ctypes.c_float)]


class _NormRope(ctypes.Structure):
    """jab_norm_rope"""

    _fields_ = [("norm", ctypes.c_int32), ("eps", ctypes.c_float), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("cos", ctypes.c_void_p),
                ("sin", ctypes.c_void_p), ("rope_len", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32)]


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
    H = ctypes.POINTER(_NormRope)
    L.jab_fp8_quantize.argtypes = [i64, i32, _P, i32, i64, i32, _P, _P, _P]
    L.jab_fp8_linear_workspace_size.argtypes = [i64, i32, i32]
    L.jab_fp8_linear_workspace_size.restype = sz
    L.jab_fp8_linear.argtypes = [i64, i32, i32, _P, i32, i64, _P, _P, i32, _P, i32, i64, _P, sz, _P]
    L.jab_rope_table_scaled.argtypes = [i32, i32, f32, ctypes.POINTER(_RopeScaling), _P, _P, _P]
    L.jab_kv_write_norm_rope.argtypes = [KV, i64, i32, _P, i32, i64, _P, H, _P, _P]
    L.jab_qk_norm_rope.argtypes = [i64, i32, i32, i32, _P, i32, i64, H, _P, i64, _P, i64, _P]
    L.jab_qk_norm_rope_backward_workspace_size.argtypes = [i64, i32, i32, i32]
    L.jab_qk_norm_rope_backward_workspace_size.restype = sz
    L.jab_qk_norm_rope_backward.argtypes = [i64, i32, i32, i32, _P, i32, i64, H, _P, i64, _P, i64, _P, i64, _P, _P, _P,
                                            sz, _P]
    L.jab_kv_release.argtypes = [KV, i32, _P, _P, _P, i32, i32, _P, i32, _P, _P, _P, _P]
    L.jab_kv_plan.argtypes = [KV, i32, i64, _P, _P, _P, i32, _P, i32, _P, _P, _P, _P, _P, _P, _P]
    for fn in ("jab_reference_forward", "jab_loss_forward", "jab_loss_forward_noalloc",
               "jab_quantized_linear", "jab_rope_table", "jab_kv_write", "jab_kv_read", "jab_kv_attention",
               "jab_fp8_quantize", "jab_fp8_linear", "jab_rope_table_scaled", "jab_kv_write_norm_rope",
               "jab_qk_norm_rope", "jab_qk_norm_rope_backward", "jab_kv_release", "jab_kv_plan",
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
    shape = t.shape
    if len(shape) == 2 and shape[1] == width and (rows is None or shape[0] == rows) and t.is_contiguous():
        return t.data_ptr(), width  # (the usual case, without the walk over the dimensions)
    strides, have = t.stride(), 1
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
    if t.dtype is dtype and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
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


_FP8 = torch.float8_e4m3fn


def _fp8_scales(t: torch.Tensor, rows: int, K: int, block_rows: int, name: str) -> int:
    if block_rows not in (1, 128):
        raise ValueError("block_rows must be 1 or 128")
    return _shaped(t, (-(-rows // block_rows), -(-K // 128)), torch.float32, name)


def jab_fp8_quantize(x, codes, scales, block_rows: int = 128, stream=None):
    """Rows x (fp16 / bf16 / fp32 [M, K], may have a pitch) as codes (float8_e4m3fn [M, K]) with a scale for every block of
    block_rows (1 or 128) rows x 128 columns: scales fp32 [ceil(M / block_rows), ceil(K / 128)]."""
    M, K = x.shape
    xp, ldx = _rows(x, K, "x")
    st = lib().jab_fp8_quantize(M, K, xp, _dtype(x, "x"), ldx, int(block_rows), _shaped(codes, (M, K), _FP8, "codes"),
                                _fp8_scales(scales, M, K, block_rows, "scales"), _stream(stream))
    _check(st, "jab_fp8_quantize")


def jab_fp8_linear_workspace_size(M: int, N: int, K: int) -> int:
    return int(lib().jab_fp8_linear_workspace_size(M, N, K))


def jab_fp8_linear(x, codes, w_scales, y, ws, block_rows: int = 128, stream=None):
    """y[m, n] = the product of x's rows, quantised to e4m3 with a scale for every 128 elements, with the weights that codes
    (float8_e4m3fn [N, K]) and w_scales (fp32 [ceil(N / block_rows), ceil(K / 128)]) stand for. x and y fp16 / bf16 /
    fp32 [M, K] and [M, N], rows may have a pitch; ws uint8, jab_fp8_linear_workspace_size bytes."""
    (M, K), N = x.shape, codes.shape[0]
    xp, ldx = _rows(x, K, "x")
    yp, ldy = _rows(y, N, "y", M)
    st = lib().jab_fp8_linear(M, N, K, xp, _dtype(x, "x"), ldx, _shaped(codes, (N, K), _FP8, "codes"),
                              _fp8_scales(w_scales, N, K, block_rows, "w_scales"), int(block_rows), yp, _dtype(y, "y"), ldy,
                              _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(stream))
    _check(st, "jab_fp8_linear")


_ROPE_KINDS = {"plain": 0, "linear": 1, "by_parts": 2}


def jab_rope_table_scaled(cos, sin, theta: float, kind: str = "plain", factor: float = 1.0, original_length: float = 0.0,
                          low_turns: float = 1.0, high_turns: float = 32.0, attention: float = 1.0, stream=None):
    """cos and sin of the angles position * f_j into fp32 [length, rotary_dim / 2] each, times `attention`. f_j = theta^(-2j /
    rotary_dim) ("plain"), divided by factor ("linear"), or that for pairs of low_turns and fewer in original_length
    tokens, unchanged for those of high_turns and more and in between in between ("by_parts")."""
    if kind not in _ROPE_KINDS:
        raise ValueError(f"kind must be one of {', '.join(_ROPE_KINDS)}, got {kind!r}")
    scaling = _RopeScaling(_ROPE_KINDS[kind], float(factor), float(original_length), float(low_turns), float(high_turns),
                           float(attention))
    st = lib().jab_rope_table_scaled(cos.shape[0], 2 * cos.shape[1], float(theta), ctypes.byref(scaling),
                                     _ptr(cos, torch.float32, "cos"), _shaped(sin, cos.shape, torch.float32, "sin"),
                                     _stream(stream))
    _check(st, "jab_rope_table_scaled")


def _norm_rope(n: int, dh: int, positions, rope, interleaved, norm_eps, q_weight, k_weight) -> _NormRope:
    qw = kw = pos = cos = sin = None
    length = half = 0
    f32 = torch.float32
    if norm_eps is not None:
        shape = (dh,)
        if q_weight is not None:
            qw = _shaped(q_weight, shape, f32, "q_weight")
        if k_weight is not None:
            kw = _shaped(k_weight, shape, f32, "k_weight")
    elif q_weight is not None or k_weight is not None:
        raise ValueError("weights of a norm need norm_eps")
    if rope is not None:
        if positions is None:
            raise ValueError("rope needs positions")
        cos_t, sin_t = rope
        shape = cos_t.shape
        length, half = shape
        cos, sin = _shaped(cos_t, shape, f32, "rope"), _shaped(sin_t, shape, f32, "rope")
        pos = _shaped(positions, (n,), torch.int32, "positions")
    return _NormRope(norm_eps is not None, norm_eps or 0.0, qw, kw, pos, cos, sin, length, 2 * half, bool(interleaved))


def jab_kv_write_norm_rope(cache: KvCache, qkv, n_q_heads: int, slots, q_out=None, positions=None, rope=None,
                           interleaved: bool = False, norm_eps: Optional[float] = None, q_weight=None, k_weight=None,
                           stream=None):
    """jab_kv_write with a norm for each head of Q and K (norm_eps; weights fp32 [head_dim], None: all 1) and then the
    rotation of their first elements: as many as the table rope = (cos, sin), fp32 [length, rotary_dim / 2] each, has
    angles for, in pairs (j, j + rotary_dim / 2) or, interleaved, (2j, 2j + 1)."""
    n, dh = qkv.shape[0], cache.head_dim
    xp, ldx = _rows(qkv, (n_q_heads + 2 * cache.n_kv_heads) * dh, "qkv")
    how = _norm_rope(n, dh, positions, rope, interleaved, norm_eps, q_weight, k_weight)
    if q_out is not None:
        if q_out.numel() != n * n_q_heads * dh:
            raise ValueError("q_out must be [n_tokens, n_q_heads * head_dim] in qkv's type")
        q_out = _ptr(q_out, qkv.dtype, "q_out")
    st = lib().jab_kv_write_norm_rope(cache.ref, n, int(n_q_heads), xp, _dtype(qkv, "qkv"), ldx,
                                      _shaped(slots, (n,), torch.int64, "slots"), ctypes.byref(how), q_out, _stream(stream))
    _check(st, "jab_kv_write_norm_rope")


def _heads(t, n: int, heads: int, dh: int, like, name: str):
    """(pointer, pitch) of rows of `heads` heads; no such heads: (None, 0)."""
    if heads == 0:
        return None, 0
    if t is None:
        raise ValueError(f"{name} is needed: there are {heads} heads of it")
    if t.dtype is not like.dtype:
        raise ValueError(f"{name} must have x's type")
    return _rows(t, heads * dh, name, n)


def _wide_rows(t, width: int, name: str, rows: int):
    """(pointer, pitch) of rows of `width` contiguous elements and more."""
    shape = t.shape
    if len(shape) == 2 and shape[0] == rows and shape[1] >= width and t.is_cuda:
        pitch, step = t.stride()
        if step == 1:
            return t.data_ptr(), pitch if rows > 1 else width
    raise ValueError(f"{name} must be a CUDA tensor of {rows} rows of at least {width} contiguous elements")


def jab_qk_norm_rope(x, n_q_heads: int, n_k_heads: int, head_dim: int, q, k, positions=None, rope=None,
                     interleaved: bool = False, norm_eps: Optional[float] = None, q_weight=None, k_weight=None, stream=None):
    """The norm and rotation of jab_kv_write_norm_rope on the heads of Q and K at the front of the rows x (fp16 / bf16 /
    fp32 [n_tokens, (n_q_heads + n_k_heads) * head_dim and more]), into q and k ([n_tokens, heads * head_dim], x's type, rows
    may have a pitch; views of x itself will do)."""
    n = x.shape[0]
    xp, ldx = _wide_rows(x, (n_q_heads + n_k_heads) * head_dim, "x", n)
    qp, ldq = _heads(q, n, n_q_heads, head_dim, x, "q")
    kp, ldk = _heads(k, n, n_k_heads, head_dim, x, "k")
    how = _norm_rope(n, head_dim, positions, rope, interleaved, norm_eps, q_weight, k_weight)
    st = lib().jab_qk_norm_rope(n, int(n_q_heads), int(n_k_heads), int(head_dim), xp, _dtype(x, "x"), ldx, ctypes.byref(how),
                                qp, ldq, kp, ldk, _stream(stream))
    _check(st, "jab_qk_norm_rope")


def jab_qk_norm_rope_backward_workspace_size(n_tokens: int, n_q_heads: int, n_k_heads: int, head_dim: int) -> int:
    return int(lib().jab_qk_norm_rope_backward_workspace_size(n_tokens, n_q_heads, n_k_heads, head_dim))


def jab_qk_norm_rope_backward(x, n_q_heads: int, n_k_heads: int, head_dim: int, dq, dk, dx, ws=None, positions=None, rope=None,
                              interleaved: bool = False, norm_eps: Optional[float] = None, q_weight=None, k_weight=None,
                              dq_weight=None, dk_weight=None, stream=None):
    """The gradient of jab_qk_norm_rope: from x as it was and the gradients dq and dk of its outputs, dx (the columns of Q and
    K) and, where they are given, dq_weight and dk_weight (fp32 [head_dim]). ws uint8 (with a weight's gradient only),
    jab_qk_norm_rope_backward_workspace_size bytes."""
    n = x.shape[0]
    width = (n_q_heads + n_k_heads) * head_dim
    xp, ldx = _wide_rows(x, width, "x", n)
    dxp, lddx = _wide_rows(dx, width, "dx", n)
    if dx.dtype is not x.dtype:
        raise ValueError("dx must have x's type")
    qp, ldq = _heads(dq, n, n_q_heads, head_dim, x, "dq")
    kp, ldk = _heads(dk, n, n_k_heads, head_dim, x, "dk")
    how = _norm_rope(n, head_dim, positions, rope, interleaved, norm_eps, q_weight, k_weight)
    wq = None if dq_weight is None else _shaped(dq_weight, (head_dim,), torch.float32, "dq_weight")
    wk = None if dk_weight is None else _shaped(dk_weight, (head_dim,), torch.float32, "dk_weight")
    st = lib().jab_qk_norm_rope_backward(n, int(n_q_heads), int(n_k_heads), int(head_dim), xp, _dtype(x, "x"), ldx,
                                         ctypes.byref(how), qp, ldq, kp, ldk, dxp, lddx, wq, wk, _ptr(ws, torch.uint8, "ws"),
                                         0 if ws is None else ws.numel(), _stream(stream))
    _check(st, "jab_qk_norm_rope_backward")


def _counters(n_free, new_free, lens, new_lens, B: int):
    """Pointers of (n_free, new_lens, new_free); what is not given is updated in place."""
    return (_shaped(n_free, (1,), torch.int32, "n_free"),
            _shaped(lens if new_lens is None else new_lens, (B,), torch.int32, "new_lens"),
            _shaped(n_free if new_free is None else new_free, (1,), torch.int32, "new_free"))


def jab_kv_release(cache: KvCache, seq_lens, ended, pages, free_pages, n_free, shared_len: int = 0, new_lens=None,
                   new_free=None, stream=None):
    """The pages of the sequences with ended[b] != 0 back onto the stack free_pages (int32 [capacity], n_free [1] of them
    free), but for those of the first shared_len tokens. seq_lens, ended int32 [n_seqs], pages int32 [n_seqs,
    max_pages]; the lengths and the stack's size afterwards go to new_lens and new_free, None: in place."""
    B = seq_lens.shape[0]
    nf, nl, nn = _counters(n_free, new_free, seq_lens, new_lens, B)
    st = lib().jab_kv_release(cache.ref, B, _shaped(seq_lens, (B,), torch.int32, "seq_lens"),
                              _shaped(ended, (B,), torch.int32, "ended"),
                              _shaped(pages, (B, pages.shape[1]), torch.int32, "pages"), pages.shape[1], int(shared_len),
                              _shaped(free_pages, (free_pages.numel(),), torch.int32, "free_pages"), free_pages.numel(), nf, nl,
                              nn, _stream(stream))
    _check(st, "jab_kv_release")


def jab_kv_plan(cache: KvCache, seq_lens, counts, pages, free_pages, n_free, q_start, slots, positions, new_lens=None,
                new_free=None, stream=None):
    """Places for the next counts[b] tokens of every sequence: pages from the top of the stack where one begins (into
    pages), q_start int32 [n_seqs + 1], and for every row slots (int64 [n_tokens], -1: padding behind the last sequence) and
    positions (int32 [n_tokens]). Other arguments as for jab_kv_release."""
    B, n = seq_lens.shape[0], slots.shape[0]
    nf, nl, nn = _counters(n_free, new_free, seq_lens, new_lens, B)
    st = lib().jab_kv_plan(cache.ref, B, n, _shaped(seq_lens, (B,), torch.int32, "seq_lens"),
                           _shaped(counts, (B,), torch.int32, "counts"),
                           _shaped(pages, (B, pages.shape[1]), torch.int32, "pages"), pages.shape[1],
                           _shaped(free_pages, (free_pages.numel(),), torch.int32, "free_pages"), free_pages.numel(), nf, nl, nn,
                           _shaped(q_start, (B + 1,), torch.int32, "q_start"), _shaped(slots, (n,), torch.int64, "slots"),
                           _shaped(positions, (n,), torch.int32, "positions"), _stream(stream))
    _check(st, "jab_kv_plan")


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
