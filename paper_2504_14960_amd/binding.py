"""ctypes binding of include/moe.h: argument marshalling only.

Functions take torch tensors that already live on the GPU, pass their device
pointers and the current stream to the C ABI and return nothing that was
computed on the host.  There is no fallback: if the HIP library is missing the
import of a symbol raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional

import torch

MOE_F32 = 0
MOE_BF16 = 1
MOE_SCORE_SOFTMAX = 0
MOE_SCORE_SIGMOID = 1
MOE_STATE_F32 = 0
MOE_STATE_MXFP8 = 1

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libmoe_hip.so")
_lib = None


class MoeError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"moe status {status}: {message}")
        self.status = status


class _GradTensor(C.Structure):      # moe_grad_tensor_t
    _fields_ = [("grad", C.c_void_p), ("n", C.c_int64), ("dt", C.c_int)]


class _AdamWTensor(C.Structure):     # moe_adamw_tensor_t
    _fields_ = [("param", C.c_void_p), ("master", C.c_void_p), ("grad", C.c_void_p), ("exp_avg", C.c_void_p),
                ("exp_avg_sq", C.c_void_p), ("exp_avg_scale", C.c_void_p), ("exp_avg_sq_scale", C.c_void_p),
                ("n", C.c_int64), ("weight_decay", C.c_float), ("lr_scale", C.c_float), ("param_dt", C.c_int),
                ("grad_dt", C.c_int), ("state", C.c_int)]


# the same in the host's own layout, padded to the alignment of a pointer
_GRAD_ROW, _ADAMW_ROW = struct.Struct("Pqi0P"), struct.Struct("7Pq2f3i0P")


def lib_path() -> str:
    return _LIB_PATH


def lib() -> C.CDLL:
    """Load libmoe_hip.so (built by ``python -m paper_2504_14960_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2504_14960_amd.build` "
            "(there is no non-HIP fallback)")
    L = C.CDLL(_LIB_PATH)
    vp, i, f, sz = C.c_void_p, C.c_int, C.c_double, C.c_size_t
    L.moe_last_error.restype = C.c_char_p
    L.moe_last_error.argtypes = []
    L.moe_version.restype = C.c_char_p
    L.moe_version.argtypes = []
    L.moe_capacity_from_factor.restype = i
    L.moe_capacity_from_factor.argtypes = [f, i, i, i]
    L.moe_max_rows.restype = i
    L.moe_max_rows.argtypes = [i, i, i, i]
    L.moe_permute_workspace_bytes.restype = sz
    L.moe_permute_workspace_bytes.argtypes = [i, i, i]
    L.moe_router_topk.restype = i
    L.moe_router_topk.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, vp, vp, vp]
    L.moe_permute.restype = i
    L.moe_permute.argtypes = [vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, sz, vp]
    L.moe_permute_noalloc.restype = i
    L.moe_permute_noalloc.argtypes = [vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp]
    L.moe_grouped_gemm_swiglu.restype = i
    L.moe_grouped_gemm_swiglu.argtypes = [vp, vp, i, i, i, i, vp, vp, vp, i, vp, vp, vp]
    L.moe_expert_gate_up.restype = i
    L.moe_expert_gate_up.argtypes = [vp, vp, i, i, i, i, vp, vp, i, vp, vp]
    L.moe_expert_down.restype = i
    L.moe_expert_down.argtypes = [vp, vp, i, i, i, i, vp, i, vp, vp]
    L.moe_unpermute_combine.restype = i
    L.moe_unpermute_combine.argtypes = [vp, vp, vp, vp, i, i, i, i, i, vp, vp]
    L.moe_unpermute_combine_backward.restype = i
    L.moe_unpermute_combine_backward.argtypes = [vp, vp, vp, vp, i, i, i, i, i, vp, vp, vp]
    L.moe_permute_backward.restype = i
    L.moe_permute_backward.argtypes = [vp, vp, vp, i, i, i, i, i, vp, vp]
    L.moe_router_backward_workspace_bytes.restype = sz
    L.moe_router_backward_workspace_bytes.argtypes = [i, i, i]
    L.moe_router_backward.restype = i
    L.moe_router_backward.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, sz, vp]
    L.moe_expert_backward_workspace_bytes.restype = sz
    L.moe_expert_backward_workspace_bytes.argtypes = [i, i, i, i]
    L.moe_expert_weights_transpose.restype = i
    L.moe_expert_weights_transpose.argtypes = [vp, vp, vp, i, i, i, vp, vp, vp]
    L.moe_grouped_gemm_swiglu_backward.restype = i
    L.moe_grouped_gemm_swiglu_backward.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.moe_permute_variant_workspace_bytes.restype = sz
    L.moe_permute_variant_workspace_bytes.argtypes = [i, i, i]
    L.moe_sort_chunks_workspace_bytes.restype = sz
    L.moe_sort_chunks_workspace_bytes.argtypes = [i]
    L.moe_sort_chunks.restype = i
    L.moe_sort_chunks.argtypes = [vp, i, vp, i, vp, i, i, i, i, vp, i, vp, vp, vp, sz, vp]
    L.moe_permute_variant.restype = i
    L.moe_permute_variant.argtypes = [vp, vp, vp, i, i, i, i, i, i, i, i, vp, vp, vp, vp, vp, i, vp, sz, vp]
    L.moe_layer_forward_train.restype = i
    L.moe_layer_forward_train.argtypes = [vp] * 6 + [i] * 7 + [vp, vp, vp, sz, vp]
    L.moe_layer_backward_workspace_bytes.restype = sz
    L.moe_layer_backward_workspace_bytes.argtypes = [i] * 6
    L.moe_layer_backward.restype = i
    L.moe_layer_backward.argtypes = [vp] * 7 + [i] * 7 + [vp] * 9 + [sz, vp]
    L.moe_probe_mfma_fp8.restype = i
    L.moe_probe_mfma_fp8.argtypes = [vp, i, i, vp, vp, vp]
    L.moe_probe_mfma_bf16.restype = i
    L.moe_probe_mfma_bf16.argtypes = [vp, i, i, vp, vp, vp]
    L.moe_expert_gate_up_saving.restype = i
    L.moe_expert_gate_up_saving.argtypes = [vp, vp, i, i, i, i, vp, vp, vp, vp, vp]
    L.moe_layer_workspace_bytes.restype = sz
    L.moe_layer_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    L.moe_workspace_bytes.restype = sz
    L.moe_workspace_bytes.argtypes = [i, i, i, i, i, i, i]
    L.moe_gemm_clock_sample.restype = i
    L.moe_gemm_clock_sample.argtypes = [vp]
    L.moe_layer_workspace_layout.restype = i
    L.moe_layer_workspace_layout.argtypes = [i, i, i, i, i, i, i, i, C.POINTER(sz), i]
    L.moe_layer_forward.restype = i
    L.moe_layer_forward.argtypes = [vp] * 9 + [i] * 9 + [vp, vp, sz, vp]
    L.moe_router_backward_addend.restype = i
    L.moe_router_backward_addend.argtypes = [vp] * 6 + [i] * 6 + [vp] * 5 + [sz, vp]
    L.moe_layer_backward_addend.restype = i
    L.moe_layer_backward_addend.argtypes = [vp] * 8 + [i] * 7 + [vp] * 9 + [sz, vp]
    L.moe_router_select.restype = i
    L.moe_router_select.argtypes = [vp] * 5 + [i] * 9 + [C.c_float, i] + [vp] * 3
    L.moe_router_select_backward.restype = i
    L.moe_router_select_backward.argtypes = [vp] * 6 + [i] * 6 + [C.c_float, i] + [vp] * 5 + [sz, vp]
    L.moe_router_bias_update_workspace_bytes.restype = sz
    L.moe_router_bias_update_workspace_bytes.argtypes = [i] * 2
    L.moe_router_bias_update.restype = i
    L.moe_router_bias_update.argtypes = [vp, i, i, C.c_float, vp, vp, sz, vp]
    L.moe_balance_loss_workspace_bytes.restype = sz
    L.moe_balance_loss_workspace_bytes.argtypes = [i] * 3
    L.moe_balance_loss.restype = i
    L.moe_balance_loss.argtypes = [vp] * 4 + [i] * 4 + [C.c_float] * 2 + [vp] * 5 + [sz, vp]
    L.moe_balance_loss_backward.restype = i
    L.moe_balance_loss_backward.argtypes = [vp] * 7 + [i] * 4 + [C.c_float] * 2 + [vp] * 2
    L.moe_grad_norm_workspace_bytes.restype = sz
    L.moe_grad_norm_workspace_bytes.argtypes = [i]
    L.moe_grad_norm.restype = i
    L.moe_grad_norm.argtypes = [vp, i, C.c_float, C.c_float, vp, vp, sz, vp]
    L.moe_adamw_step.restype = i
    L.moe_adamw_step.argtypes = [vp, i] + [f] * 4 + [C.c_int64, C.c_uint32, vp, vp]
    L.moe_set_option.restype = i
    L.moe_set_option.argtypes = [C.c_char_p, i]
    f = C.c_float
    L.moe_fp8_delayed_scale.restype = f
    L.moe_fp8_delayed_scale.argtypes = [C.POINTER(f), i, i]
    L.moe_fp8_quantize.restype = i
    L.moe_fp8_quantize.argtypes = [vp, i, sz, f, vp, vp, vp]
    L.moe_permute_fp8.restype = i
    L.moe_permute_fp8.argtypes = [vp, vp, i, i, i, i, i, f, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.moe_grouped_gemm_swiglu_fp8.restype = i
    L.moe_grouped_gemm_swiglu_fp8.argtypes = [vp, vp, i, i, i, i, vp, vp, vp, f, f, f, f, vp, vp, vp, vp]
    L.moe_expert_gate_up_fp8.restype = i
    L.moe_expert_gate_up_fp8.argtypes = [vp, vp, i, i, i, i, vp, vp, f, f, f, vp, vp, vp]
    L.moe_expert_down_fp8.restype = i
    L.moe_expert_down_fp8.argtypes = [vp, vp, i, i, i, i, vp, f, vp, vp]
    L.moe_fp8_block_scale_stride.restype = i
    L.moe_fp8_block_scale_stride.argtypes = [i]
    L.moe_fp8_block_quantize.restype = i
    L.moe_fp8_block_quantize.argtypes = [vp, i, i, i, vp, vp, vp]
    L.moe_expert_weights_fp8_block.restype = i
    L.moe_expert_weights_fp8_block.argtypes = [vp] * 3 + [i] * 4 + [vp] * 11
    L.moe_permute_fp8_block.restype = i
    L.moe_permute_fp8_block.argtypes = [vp, vp] + [i] * 5 + [vp] * 7 + [sz, vp]
    L.moe_grouped_gemm_swiglu_fp8_block.restype = i
    L.moe_grouped_gemm_swiglu_fp8_block.argtypes = [vp] * 3 + [i] * 4 + [vp] * 11
    L.moe_expert_gate_up_fp8_block.restype = i
    L.moe_expert_gate_up_fp8_block.argtypes = [vp] * 3 + [i] * 4 + [vp] * 8
    L.moe_expert_down_fp8_block.restype = i
    L.moe_expert_down_fp8_block.argtypes = [vp] * 3 + [i] * 4 + [vp] * 4
    L.moe_expert_backward_fp8_block_workspace_bytes.restype = sz
    L.moe_expert_backward_fp8_block_workspace_bytes.argtypes = [i] * 4
    L.moe_grouped_gemm_swiglu_fp8_block_backward.restype = i
    L.moe_grouped_gemm_swiglu_fp8_block_backward.argtypes = [vp] * 7 + [i] * 4 + [vp] * 9 + [sz, vp]
    _lib = L
    return L


def _check(status: int) -> None:
    if status != 0:
        raise MoeError(status, lib().moe_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("the MoE hot path takes device tensors only")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return MOE_BF16
    if t.dtype == torch.float32:
        return MOE_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream():
    # torch.cuda.current_stream().cuda_stream without the Stream object: 0.3 us instead of 2.8, a quarter of a small call.  Not part
    # of torch's public interface: a version without it takes the public way.
    try:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    except AttributeError:
        return torch.cuda.current_stream().cuda_stream


def version() -> str:
    return lib().moe_version().decode()


def set_option(name: str, value: int) -> None:
    _check(lib().moe_set_option(name.encode(), int(value)))


def capacity_from_factor(cf: float, T: int, K: int, E: int) -> int:
    return int(lib().moe_capacity_from_factor(float(cf), T, K, E))


def max_rows(T: int, K: int, E: int, capacity: int) -> int:
    return int(lib().moe_max_rows(T, K, E, capacity))


def permute_workspace_bytes(T: int, K: int, E: int) -> int:
    return int(lib().moe_permute_workspace_bytes(T, K, E))


def router_topk(x: Optional[torch.Tensor], w_router: Optional[torch.Tensor],
                logit_bias: Optional[torch.Tensor], logits: torch.Tensor, K: int, renormalize: bool,
                topk_idx: torch.Tensor, topk_gate: torch.Tensor, dtype: Optional[int] = None) -> None:
    T, E = logits.shape
    H = x.shape[1] if x is not None else 0
    dt = _dt(x) if x is not None else (MOE_BF16 if dtype is None else dtype)
    _check(lib().moe_router_topk(_ptr(x), _ptr(w_router), _ptr(logit_bias), _ptr(logits), T, H, E, K,
                                 int(bool(renormalize)), dt, _ptr(topk_idx), _ptr(topk_gate), _stream()))


def permute(x: Optional[torch.Tensor], topk_idx: torch.Tensor, E: int, capacity: int,
            x_perm: Optional[torch.Tensor], expert_counts: torch.Tensor, expert_offsets: torch.Tensor,
            row_of_assign: torch.Tensor, assign_of_row: torch.Tensor, workspace: torch.Tensor,
            H: Optional[int] = None, dtype: int = MOE_BF16) -> None:
    T, K = topk_idx.shape
    if x is not None:
        H, dtype = x.shape[1], _dt(x)
    elif H is None:
        H = 8
    _check(lib().moe_permute(_ptr(x), _ptr(topk_idx), T, H, E, K, int(capacity), dtype, _ptr(x_perm),
                             _ptr(expert_counts), _ptr(expert_offsets), _ptr(row_of_assign),
                             _ptr(assign_of_row), _ptr(workspace), workspace.numel() * workspace.element_size(),
                             _stream()))


def permute_noalloc(x: Optional[torch.Tensor], topk_idx: torch.Tensor, E: int, capacity: int,
                    x_perm: Optional[torch.Tensor], expert_counts: torch.Tensor, expert_offsets: torch.Tensor,
                    row_of_assign: torch.Tensor, assign_of_row: torch.Tensor, H: Optional[int] = None,
                    dtype: int = MOE_BF16) -> None:
    T, K = topk_idx.shape
    if x is not None:
        H, dtype = x.shape[1], _dt(x)
    elif H is None:
        H = 8
    _check(lib().moe_permute_noalloc(_ptr(x), _ptr(topk_idx), T, H, E, K, int(capacity), dtype, _ptr(x_perm),
                                     _ptr(expert_counts), _ptr(expert_offsets), _ptr(row_of_assign),
                                     _ptr(assign_of_row), _stream()))


def grouped_gemm_swiglu(x_perm: torch.Tensor, expert_offsets: torch.Tensor, w_gate: torch.Tensor,
                        w_up: torch.Tensor, w_down: torch.Tensor, h_workspace: torch.Tensor,
                        y_perm: torch.Tensor) -> None:
    R_max, H = x_perm.shape
    E, F, _ = w_gate.shape
    _check(lib().moe_grouped_gemm_swiglu(_ptr(x_perm), _ptr(expert_offsets), R_max, H, F, E, _ptr(w_gate),
                                         _ptr(w_up), _ptr(w_down), _dt(x_perm), _ptr(h_workspace),
                                         _ptr(y_perm), _stream()))


def expert_gate_up(x_perm: torch.Tensor, expert_offsets: torch.Tensor, w_gate: torch.Tensor,
                   w_up: torch.Tensor, h: torch.Tensor) -> None:
    R_max, H = x_perm.shape
    E, F, _ = w_gate.shape
    _check(lib().moe_expert_gate_up(_ptr(x_perm), _ptr(expert_offsets), R_max, H, F, E, _ptr(w_gate),
                                    _ptr(w_up), _dt(x_perm), _ptr(h), _stream()))


def expert_down(h: torch.Tensor, expert_offsets: torch.Tensor, w_down: torch.Tensor,
                y_perm: torch.Tensor) -> None:
    R_max, F = h.shape
    E, H, _ = w_down.shape
    _check(lib().moe_expert_down(_ptr(h), _ptr(expert_offsets), R_max, H, F, E, _ptr(w_down), _dt(h),
                                 _ptr(y_perm), _stream()))


def unpermute_combine(y_perm: torch.Tensor, row_of_assign: torch.Tensor, topk_gate: torch.Tensor,
                      addend: Optional[torch.Tensor], y: torch.Tensor) -> None:
    T, K = topk_gate.shape
    R_max, H = y_perm.shape
    _check(lib().moe_unpermute_combine(_ptr(y_perm), _ptr(row_of_assign), _ptr(topk_gate), _ptr(addend),
                                       T, H, K, R_max, _dt(y), _ptr(y), _stream()))


# ---- FP8 (E4M3) variant of the expert FFN; E4M3 tensors are torch.uint8 (codes) ----
def fp8_delayed_scale(amax_history, margin: int = 0) -> float:
    h = [float(v) for v in amax_history]
    arr = (C.c_float * max(len(h), 1))(*h)
    return float(lib().moe_fp8_delayed_scale(arr, len(h), int(margin)))


def fp8_quantize(src: torch.Tensor, scale: float, dst: torch.Tensor, amax: Optional[torch.Tensor] = None) -> None:
    if dst.dtype != torch.uint8 or dst.numel() != src.numel():
        raise ValueError("dst must be a uint8 tensor with as many elements as src")
    _check(lib().moe_fp8_quantize(_ptr(src), _dt(src), src.numel(), float(scale), _ptr(dst), _ptr(amax), _stream()))


def permute_fp8(x: torch.Tensor, topk_idx: torch.Tensor, E: int, capacity: int, scale: float,
                x_perm_fp8: torch.Tensor, expert_counts: torch.Tensor, expert_offsets: torch.Tensor,
                row_of_assign: torch.Tensor, assign_of_row: torch.Tensor, amax: Optional[torch.Tensor],
                workspace: torch.Tensor) -> None:
    T, K = topk_idx.shape
    if x.dtype != torch.bfloat16 or x_perm_fp8.dtype != torch.uint8:
        raise TypeError("permute_fp8 takes a bf16 x and writes uint8 E4M3 codes")
    _check(lib().moe_permute_fp8(_ptr(x), _ptr(topk_idx), T, x.shape[1], E, K, int(capacity), float(scale),
                                 _ptr(x_perm_fp8), _ptr(expert_counts), _ptr(expert_offsets), _ptr(row_of_assign),
                                 _ptr(assign_of_row), _ptr(amax), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream()))


def grouped_gemm_swiglu_fp8(x_perm: torch.Tensor, expert_offsets: torch.Tensor, w_gate: torch.Tensor,
                            w_up: torch.Tensor, w_down: torch.Tensor, dq_gate: float, dq_up: float,
                            scale_h: float, dq_down: float, h: torch.Tensor, amax_h: Optional[torch.Tensor],
                            y_perm: torch.Tensor) -> None:
    R_max, H = x_perm.shape
    E, F, _ = w_gate.shape
    _check(lib().moe_grouped_gemm_swiglu_fp8(_ptr(x_perm), _ptr(expert_offsets), R_max, H, F, E, _ptr(w_gate),
                                             _ptr(w_up), _ptr(w_down), float(dq_gate), float(dq_up), float(scale_h),
                                             float(dq_down), _ptr(h), _ptr(amax_h), _ptr(y_perm), _stream()))


def expert_gate_up_fp8(x_perm: torch.Tensor, expert_offsets: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor,
                       dq_gate: float, dq_up: float, scale_h: float, h: torch.Tensor,
                       amax_h: Optional[torch.Tensor]) -> None:
    R_max, H = x_perm.shape
    E, F, _ = w_gate.shape
    _check(lib().moe_expert_gate_up_fp8(_ptr(x_perm), _ptr(expert_offsets), R_max, H, F, E, _ptr(w_gate), _ptr(w_up),
                                        float(dq_gate), float(dq_up), float(scale_h), _ptr(h), _ptr(amax_h),
                                        _stream()))


def expert_down_fp8(h: torch.Tensor, expert_offsets: torch.Tensor, w_down: torch.Tensor, dq_down: float,
                    y_perm: torch.Tensor) -> None:
    R_max, F = h.shape
    E, H, _ = w_down.shape
    _check(lib().moe_expert_down_fp8(_ptr(h), _ptr(expert_offsets), R_max, H, F, E, _ptr(w_down), float(dq_down),
                                     _ptr(y_perm), _stream()))


# ---- E4M3 with a scale for every block of 128: codes as torch.uint8 or float8_e4m3fn, E8M0 scales as torch.uint8 or
# float8_e8m0fnu, in rows of fp8_block_scale_stride bytes ----
_CODES, _SCALES = (torch.uint8, torch.float8_e4m3fn), (torch.uint8, torch.float8_e8m0fnu)


def _blocks(name: str, codes: torch.Tensor, scales: torch.Tensor, shape, scale_rows: int):
    """The device pointers of codes of this shape and of their scales."""
    if tuple(codes.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(codes.shape)}")
    _is(name, codes, _CODES, codes.numel())
    _is(name + "_scales", scales, _SCALES, scale_rows * fp8_block_scale_stride(shape[-1]))
    return _ptr(codes), _ptr(scales)


def _bf16(name: str, t: torch.Tensor, numel: int):
    return _expect(name, t, torch.bfloat16, numel)


def fp8_block_scale_stride(C: int) -> int:
    return int(lib().moe_fp8_block_scale_stride(C))


def fp8_block_quantize(src: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor) -> None:
    """src [rows, C] (fp32 or bf16) to codes [rows, C] and scales [rows, fp8_block_scale_stride(C)]."""
    rows, C = src.shape
    c, s = _blocks("codes", codes, scales, (rows, C), rows)
    _check(lib().moe_fp8_block_quantize(_ptr(src), _dt(src), rows, C, c, s, _stream()))


def expert_weights_fp8_block(w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, gate: Optional[torch.Tensor],
                             gate_scales: Optional[torch.Tensor], up: Optional[torch.Tensor], up_scales: Optional[torch.Tensor],
                             down: Optional[torch.Tensor], down_scales: Optional[torch.Tensor],
                             wgu_t: Optional[torch.Tensor] = None, wgu_t_scales: Optional[torch.Tensor] = None,
                             wd_t: Optional[torch.Tensor] = None, wd_t_scales: Optional[torch.Tensor] = None) -> None:
    """A layer's weights (fp32 or bf16) as codes and scales of the forward (gate, up [E, F, H], down [E, H, F]) and of the
    backward (wgu_t [E, H, 2F], wd_t [E, F, H]); either set may be left out."""
    E, F, H = w_gate.shape
    for name, t, shape in (("w_up", w_up, (E, F, H)), ("w_down", w_down, (E, H, F))):
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} must have shape {shape}, not {tuple(t.shape)}")
        _is(name, t, (w_gate.dtype,), E * F * H)
    out = []
    for name, codes, scales, shape in (("gate", gate, gate_scales, (E, F, H)), ("up", up, up_scales, (E, F, H)),
                                       ("down", down, down_scales, (E, H, F)), ("wgu_t", wgu_t, wgu_t_scales, (E, H, 2 * F)),
                                       ("wd_t", wd_t, wd_t_scales, (E, F, H))):
        if (codes is None) != (scales is None):
            raise ValueError(f"{name} and {name}_scales are given together or left out together")
        out += (None, None) if codes is None else _blocks(name, codes, scales, shape, E * (shape[1] // 128))
    _check(lib().moe_expert_weights_fp8_block(_ptr(w_gate), _ptr(w_up), _ptr(w_down), _dt(w_gate), H, F, E, *out, _stream()))


def permute_fp8_block(x: torch.Tensor, topk_idx: torch.Tensor, E: int, capacity: int, x_perm: torch.Tensor,
                      x_scales: torch.Tensor, expert_counts: torch.Tensor, expert_offsets: torch.Tensor,
                      row_of_assign: torch.Tensor, assign_of_row: torch.Tensor, workspace: torch.Tensor) -> None:
    T, K = topk_idx.shape
    H, i32 = x.shape[1], torch.int32
    R = max_rows(T, K, E, int(capacity))
    c, s = _blocks("x_perm", x_perm, x_scales, (R, H), R)
    _check(lib().moe_permute_fp8_block(
        _bf16("x", x, T * H), _expect("topk_idx", topk_idx, i32, T * K), T, H, E, K, int(capacity), c, s,
        _expect("expert_counts", expert_counts, i32, E), _expect("expert_offsets", expert_offsets, i32, E + 1),
        _expect("row_of_assign", row_of_assign, i32, T * K), _expect("assign_of_row", assign_of_row, i32, R), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream()))


def grouped_gemm_swiglu_fp8_block(x_perm: torch.Tensor, x_scales: torch.Tensor, expert_offsets: torch.Tensor, w_gate: torch.Tensor,
                                  gate_scales: torch.Tensor, w_up: torch.Tensor, up_scales: torch.Tensor, w_down: torch.Tensor,
                                  down_scales: torch.Tensor, h: torch.Tensor, h_scales: torch.Tensor, gu: Optional[torch.Tensor],
                                  y_perm: torch.Tensor) -> None:
    """h (codes and scales) and y_perm (bf16) of x_perm's rows; gu [R, 2F] bf16: also g | u, for the backward."""
    R, H = x_perm.shape
    E, F, _ = w_gate.shape
    n = E * (F // 128)
    _check(lib().moe_grouped_gemm_swiglu_fp8_block(
        *_blocks("x_perm", x_perm, x_scales, (R, H), R), _expect("expert_offsets", expert_offsets, torch.int32, E + 1), R, H, F, E,
        *_blocks("w_gate", w_gate, gate_scales, (E, F, H), n), *_blocks("w_up", w_up, up_scales, (E, F, H), n),
        *_blocks("w_down", w_down, down_scales, (E, H, F), E * (H // 128)), *_blocks("h", h, h_scales, (R, F), R),
        None if gu is None else _bf16("gu", gu, R * 2 * F), _bf16("y_perm", y_perm, R * H), _stream()))


def expert_gate_up_fp8_block(x_perm: torch.Tensor, x_scales: torch.Tensor, expert_offsets: torch.Tensor, w_gate: torch.Tensor,
                             gate_scales: torch.Tensor, w_up: torch.Tensor, up_scales: torch.Tensor, h: torch.Tensor,
                             h_scales: torch.Tensor, gu: Optional[torch.Tensor] = None) -> None:
    R, H = x_perm.shape
    E, F, _ = w_gate.shape
    n = E * (F // 128)
    _check(lib().moe_expert_gate_up_fp8_block(
        *_blocks("x_perm", x_perm, x_scales, (R, H), R), _expect("expert_offsets", expert_offsets, torch.int32, E + 1), R, H, F, E,
        *_blocks("w_gate", w_gate, gate_scales, (E, F, H), n), *_blocks("w_up", w_up, up_scales, (E, F, H), n),
        *_blocks("h", h, h_scales, (R, F), R), None if gu is None else _bf16("gu", gu, R * 2 * F), _stream()))


def expert_down_fp8_block(h: torch.Tensor, h_scales: torch.Tensor, expert_offsets: torch.Tensor, w_down: torch.Tensor,
                          down_scales: torch.Tensor, y_perm: torch.Tensor) -> None:
    R, F = h.shape
    E, H, _ = w_down.shape
    _check(lib().moe_expert_down_fp8_block(
        *_blocks("h", h, h_scales, (R, F), R), _expect("expert_offsets", expert_offsets, torch.int32, E + 1), R, H, F, E,
        *_blocks("w_down", w_down, down_scales, (E, H, F), E * (H // 128)), _bf16("y_perm", y_perm, R * H), _stream()))


def expert_backward_fp8_block_workspace_bytes(R_max: int, H: int, F: int, E: int) -> int:
    return int(lib().moe_expert_backward_fp8_block_workspace_bytes(R_max, H, F, E))


def grouped_gemm_swiglu_fp8_block_backward(x_perm: torch.Tensor, x_scales: torch.Tensor, h: torch.Tensor, h_scales: torch.Tensor,
                                           gu: torch.Tensor, dy_perm: torch.Tensor, expert_offsets: torch.Tensor,
                                           wgu_t: torch.Tensor, wgu_t_scales: torch.Tensor, wd_t: torch.Tensor,
                                           wd_t_scales: torch.Tensor, dx_perm: torch.Tensor, dw_gate: torch.Tensor,
                                           dw_up: torch.Tensor, dw_down: torch.Tensor, workspace: torch.Tensor) -> None:
    R, H = x_perm.shape
    E, F, _ = wd_t.shape
    _check(lib().moe_grouped_gemm_swiglu_fp8_block_backward(
        *_blocks("x_perm", x_perm, x_scales, (R, H), R), *_blocks("h", h, h_scales, (R, F), R), _bf16("gu", gu, R * 2 * F),
        _bf16("dy_perm", dy_perm, R * H), _expect("expert_offsets", expert_offsets, torch.int32, E + 1), R, H, F, E,
        *_blocks("wgu_t", wgu_t, wgu_t_scales, (E, H, 2 * F), E * (H // 128)),
        *_blocks("wd_t", wd_t, wd_t_scales, (E, F, H), E * (F // 128)), _bf16("dx_perm", dx_perm, R * H),
        _bf16("dw_gate", dw_gate, E * F * H), _bf16("dw_up", dw_up, E * F * H), _bf16("dw_down", dw_down, E * F * H),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))


def router_backward_workspace_bytes(T: int, H: int, E: int) -> int:
    return int(lib().moe_router_backward_workspace_bytes(T, H, E))


def router_backward(x: torch.Tensor, w_router: torch.Tensor, logits: torch.Tensor, topk_idx: torch.Tensor,
                    dgate: torch.Tensor, renormalize: bool, dlogits: torch.Tensor, dx: Optional[torch.Tensor],
                    dw_router: Optional[torch.Tensor], dbias: Optional[torch.Tensor],
                    workspace: Optional[torch.Tensor], dlogits_addend: Optional[torch.Tensor] = None) -> None:
    T, E = logits.shape
    K = topk_idx.shape[1]
    H = x.shape[1]
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if dlogits_addend is not None:
        addend = _expect("dlogits_addend", dlogits_addend, torch.float32, T * E)
        _check(lib().moe_router_backward_addend(_ptr(x), _ptr(w_router), _ptr(logits), _ptr(topk_idx), _ptr(dgate), addend, T, H, E, K, int(bool(renormalize)), _dt(x),
                                                _ptr(dlogits), _ptr(dx), _ptr(dw_router), _ptr(dbias), _ptr(workspace),
                                                nbytes, _stream()))
        return
    _check(lib().moe_router_backward(_ptr(x), _ptr(w_router), _ptr(logits), _ptr(topk_idx), _ptr(dgate), T, H, E, K,
                                     int(bool(renormalize)), _dt(x), _ptr(dlogits), _ptr(dx), _ptr(dw_router),
                                     _ptr(dbias), _ptr(workspace), nbytes, _stream()))


# ---- what follows the gradients in a training step: balance loss, gradient norm, AdamW ----
def _is(name: str, t: torch.Tensor, dtypes, numel: int) -> None:
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(map(str, dtypes))}, not {t.dtype}")
    if t.numel() != numel:
        raise ValueError(f"{name} must have {numel} elements, not {t.numel()}")


def _expect(name: str, t: torch.Tensor, dtype, numel: int):
    """The device pointer of a tensor of this type and size."""
    if t.dtype is dtype and t.numel() == numel and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    _is(name, t, (dtype,), numel)
    return _ptr(t)


def _optional(name: str, t: Optional[torch.Tensor], dtype, numel: int):
    return None if t is None else _expect(name, t, dtype, numel)


# ---- routing by scores ----
def router_select(x: Optional[torch.Tensor], w_router: Optional[torch.Tensor], logit_bias: Optional[torch.Tensor],
                  logits: torch.Tensor, K: int, topk_idx: torch.Tensor, topk_gate: torch.Tensor, score: int = MOE_SCORE_SIGMOID,
                  select_bias: Optional[torch.Tensor] = None, n_groups: int = 1, topk_groups: int = 1, group_best: int = 2,
                  renormalize: bool = True, gate_scale: float = 1.0, dtype: Optional[int] = None) -> None:
    """topk_idx, topk_gate [T, K] from the scores of logits [T, E] (x given: computed first).  select_bias [E] chooses along
    and has no part in the gates; the experts come from the topk_groups best of n_groups groups.  -1: no expert was left."""
    T, E = logits.shape
    H = 0
    dt = MOE_BF16 if dtype is None else dtype
    if x is not None:
        H, dt = x.shape[1], _dt(x)
        _is("x", x, (x.dtype,), T * H)
        _is("w_router", w_router, (x.dtype,), E * H)
    f32 = torch.float32
    _check(lib().moe_router_select(
        _ptr(x), _ptr(w_router), _optional("logit_bias", logit_bias, f32, E), _expect("logits", logits, f32, T * E),
        _optional("select_bias", select_bias, f32, E), T, H, E, K, score, n_groups, topk_groups, group_best, int(bool(renormalize)),
        gate_scale, dt, _expect("topk_idx", topk_idx, torch.int32, T * K), _expect("topk_gate", topk_gate, f32, T * K), _stream()))


def router_select_backward(x: Optional[torch.Tensor], w_router: Optional[torch.Tensor], logits: torch.Tensor,
                           topk_idx: torch.Tensor, dgate: torch.Tensor, dlogits: torch.Tensor, dx: Optional[torch.Tensor],
                           dw_router: Optional[torch.Tensor], dbias: Optional[torch.Tensor], workspace: Optional[torch.Tensor],
                           score: int = MOE_SCORE_SIGMOID, renormalize: bool = True, gate_scale: float = 1.0,
                           dlogits_addend: Optional[torch.Tensor] = None) -> None:
    """dlogits [T, E] = gradient of dgate . topk_gate in the logits (+ dlogits_addend), and what follows from it: dx [T, H],
    dw_router [E, H] and dbias [E] where they are given (dx takes w_router, dw_router takes x and a workspace of
    router_backward_workspace_bytes)."""
    T, E = logits.shape
    K = topk_idx.shape[1]
    f32 = torch.float32
    ref = dx if dx is not None else x
    H, dt = (0, MOE_BF16) if ref is None else (ref.shape[1], _dt(ref))
    for name, t, numel in (("x", x, T * H), ("w_router", w_router, E * H), ("dx", dx, T * H)):
        if t is not None and ref is not None:
            _is(name, t, (ref.dtype,), numel)
    _check(lib().moe_router_select_backward(
        _ptr(x), _ptr(w_router), _expect("logits", logits, f32, T * E), _expect("topk_idx", topk_idx, torch.int32, T * K),
        _expect("dgate", dgate, f32, T * K), _optional("dlogits_addend", dlogits_addend, f32, T * E), T, H, E, K, score,
        int(bool(renormalize)), gate_scale, dt, _expect("dlogits", dlogits, f32, T * E), _ptr(dx),
        _optional("dw_router", dw_router, f32, E * H), _optional("dbias", dbias, f32, E), _ptr(workspace),
        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def router_bias_update_workspace_bytes(n_rows: int, E: int) -> int:
    return int(lib().moe_router_bias_update_workspace_bytes(n_rows, E))


def router_bias_update(counts: torch.Tensor, rate: float, select_bias: torch.Tensor,
                       workspace: Optional[torch.Tensor] = None) -> None:
    """One step of router_select's bias [E]: rate up for experts below the mean load, down above.  counts [n_rows, E] int32 (or
    [E]), e.g. balance_loss's."""
    E = select_bias.numel()
    rows = counts.numel() // E if E else 0
    _check(lib().moe_router_bias_update(
        _expect("counts", counts, torch.int32, rows * E), rows, E, rate, _expect("select_bias", select_bias, torch.float32, E),
        _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def _mask(token_mask: Optional[torch.Tensor], T: int):
    if token_mask is None:
        return None
    return _expect("token_mask", token_mask, torch.bool if token_mask.dtype == torch.bool else torch.uint8, T)


def _offsets(seq_offsets: Optional[torch.Tensor]):
    """Pointer and number of sequences."""
    if seq_offsets is None:
        return None, 1
    n = seq_offsets.numel()
    return _expect("seq_offsets", seq_offsets, torch.int32, max(2, n)), n - 1


def balance_loss_workspace_bytes(T: int, E: int, n_seq: int = 1) -> int:
    return int(lib().moe_balance_loss_workspace_bytes(T, E, n_seq))


def balance_loss(logits: torch.Tensor, topk_idx: torch.Tensor, balance_coef: float, z_coef: float, counts: torch.Tensor,
                 prob_sums: torch.Tensor, seq_tokens: torch.Tensor, losses: torch.Tensor, workspace: torch.Tensor,
                 token_mask: Optional[torch.Tensor] = None, seq_offsets: Optional[torch.Tensor] = None) -> None:
    """losses [2] = balance and z loss of a router's logits [T, E] and selection [T, K]; counts and prob_sums [n_seq, E],
    seq_tokens [n_seq + 1].  token_mask [T] (uint8 or bool): tokens that count; seq_offsets [n_seq + 1] int32."""
    T, E = logits.shape
    K = topk_idx.shape[1]
    offsets, n_seq = _offsets(seq_offsets)
    f32, i32 = torch.float32, torch.int32
    _check(lib().moe_balance_loss(
        _expect("logits", logits, f32, T * E), _expect("topk_idx", topk_idx, i32, T * K), _mask(token_mask, T), offsets, T, E, K,
        n_seq, balance_coef, z_coef, _expect("counts", counts, i32, n_seq * E),
        _expect("prob_sums", prob_sums, f32, n_seq * E), _expect("seq_tokens", seq_tokens, i32, n_seq + 1),
        _expect("losses", losses, f32, 2), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))


def balance_loss_backward(logits: torch.Tensor, counts: torch.Tensor, seq_tokens: torch.Tensor,
                          dlosses: Optional[torch.Tensor], K: int, balance_coef: float, z_coef: float,
                          dlogits: torch.Tensor, addend: Optional[torch.Tensor] = None,
                          token_mask: Optional[torch.Tensor] = None, seq_offsets: Optional[torch.Tensor] = None) -> None:
    """dlogits [T, E] = gradient of dlosses . losses in the logits, plus addend [T, E] (which may be dlogits)."""
    T, E = logits.shape
    offsets, n_seq = _offsets(seq_offsets)
    f32, i32 = torch.float32, torch.int32
    _check(lib().moe_balance_loss_backward(
        _expect("logits", logits, f32, T * E), _mask(token_mask, T), offsets, _expect("counts", counts, i32, n_seq * E),
        _expect("seq_tokens", seq_tokens, i32, n_seq + 1), None if dlosses is None else _expect("dlosses", dlosses, f32, 2),
        None if addend is None else _expect("addend", addend, f32, T * E), T, E, K, n_seq, balance_coef, z_coef,
        _expect("dlogits", dlogits, f32, T * E), _stream()))


class GradTensors:
    """A list of gradients (fp32 or bf16) that grad_norm goes over: built once, kept as long as the buffers are used."""

    def __init__(self, grads) -> None:
        self.grads = list(grads)
        self._list = _packed(_GradTensor, _GRAD_ROW, [(_ptr(g), g.numel(), _dt(g)) for g in self.grads])


def _packed(kind, row, rows):
    """A ctypes array of `kind` from tuples of its fields (a structure made one by one costs twice the time)."""
    return (kind * len(rows)).from_buffer_copy(b"".join(row.pack(*r) for r in rows))


def grad_norm_workspace_bytes(count: int) -> int:
    return int(lib().moe_grad_norm_workspace_bytes(count))


def grad_norm(tensors, out: torch.Tensor, workspace: torch.Tensor, max_norm: float = 0.0, multiplier: float = 1.0) -> None:
    """out [2] = norm of multiplier * the gradients of a GradTensors (or an AdamWTensors), and the factor that
    adamw_step takes as grad_scale: multiplier, clipped to max_norm (0: not), NaN where the norm is not finite."""
    grads = tensors.grads if isinstance(tensors, AdamWTensors) else tensors
    if not isinstance(grads, GradTensors):
        raise TypeError(f"tensors must be GradTensors or AdamWTensors, not {type(tensors).__name__}")
    _check(lib().moe_grad_norm(grads._list, len(grads._list), max_norm, multiplier, _expect("out", out, torch.float32, 2),
                               _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))


class AdamWTensors:
    """The tensors of an AdamW step: built once from the buffers a program trains with, and kept.

    params fp32 or bf16; masters: fp32 copies that are stepped in place of bf16 params (None, or None in places: bf16
    alone, rounded stochastically); grads fp32 or bf16; exp_avgs and exp_avg_sqs fp32, or uint8 E4M3 codes with
    uint8 E8M0 exp_avg_scales and exp_avg_sq_scales, one to every 32 elements (zeros are fresh states); or the same bytes as
    float8_e4m3fn and float8_e8m0fnu."""

    _CODES, _SCALES = (torch.uint8, torch.float8_e4m3fn), (torch.uint8, torch.float8_e8m0fnu)

    def __init__(self, params, grads, exp_avgs, exp_avg_sqs, masters=None, exp_avg_scales=None, exp_avg_sq_scales=None,
                 weight_decays=None, lr_scales=None) -> None:
        n = len(params)
        columns = [params, masters, grads, exp_avgs, exp_avg_sqs, exp_avg_scales, exp_avg_sq_scales]
        columns = [[None] * n if c is None else list(c) for c in columns]
        decays = [0.0] * n if weight_decays is None else list(weight_decays)
        scales = [1.0] * n if lr_scales is None else list(lr_scales)
        if any(len(c) != n for c in columns + [decays, scales]):
            raise ValueError("every list must have as many entries as params")
        self.tensors = list(zip(*columns))       # keeps the buffers alive
        self._list = _packed(_AdamWTensor, _ADAMW_ROW, [self._row(*r, d, s) for r, d, s in zip(self.tensors, decays, scales)])
        self.grads = GradTensors(columns[2])

    @classmethod
    def _row(cls, param, master, grad, m, v, m_scale, v_scale, decay, lr_scale):
        count = param.numel()
        small = m.dtype in cls._CODES
        _is("exp_avg", m, (torch.float32,) + cls._CODES, count)
        _is("exp_avg_sq", v, cls._CODES if small else (torch.float32,), count)
        _is("grad", grad, (grad.dtype,), count)
        if master is not None:
            _is("master", master, (torch.float32,), count)
        if small:
            for name, t in (("exp_avg_scale", m_scale), ("exp_avg_sq_scale", v_scale)):
                if t is None:
                    raise ValueError(f"8-bit states need {name}s")
                _is(name, t, cls._SCALES, (count + 31) // 32)
        elif m_scale is not None or v_scale is not None:
            raise ValueError("exp_avg_scales and exp_avg_sq_scales go with 8-bit states only")
        return (_ptr(param), _ptr(master) or 0, _ptr(grad), _ptr(m), _ptr(v), _ptr(m_scale) or 0, _ptr(v_scale) or 0, count,
                decay, lr_scale, _dt(param), _dt(grad), MOE_STATE_MXFP8 if small else MOE_STATE_F32)


def adamw_step(tensors: AdamWTensors, lr: float, beta1: float, beta2: float, eps: float, step: int, seed: int = 0,
               grad_scale: Optional[torch.Tensor] = None) -> None:
    """One AdamW step (the first has step = 1) over all tensors.  grad_scale [1] fp32 on the device multiplies every
    gradient; NaN in it leaves everything as it is.  seed: of stochastic rounding, another one in every step."""
    if not isinstance(tensors, AdamWTensors):        # the rows of a GradTensors are shorter than those the call reads
        raise TypeError(f"tensors must be AdamWTensors, not {type(tensors).__name__}")
    scale = None if grad_scale is None else _expect("grad_scale", grad_scale, torch.float32, 1)
    _check(lib().moe_adamw_step(tensors._list, len(tensors._list), lr, beta1, beta2, eps, step, seed & 0xffffffff, scale,
                                _stream()))


def expert_backward_workspace_bytes(R_max: int, H: int, F: int, E: int) -> int:
    return int(lib().moe_expert_backward_workspace_bytes(R_max, H, F, E))


def expert_weights_transpose(w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, wgu_t: torch.Tensor,
                             wd_t: torch.Tensor) -> None:
    E, F, H = w_gate.shape
    _check(lib().moe_expert_weights_transpose(_ptr(w_gate), _ptr(w_up), _ptr(w_down), H, F, E, _ptr(wgu_t), _ptr(wd_t),
                                              _stream()))


def expert_gate_up_saving(x_perm: torch.Tensor, expert_offsets: torch.Tensor, w_gate: torch.Tensor,
                          w_up: torch.Tensor, h: torch.Tensor, gu: torch.Tensor) -> None:
    R_max, H = x_perm.shape
    E, F, _ = w_gate.shape
    _check(lib().moe_expert_gate_up_saving(_ptr(x_perm), _ptr(expert_offsets), R_max, H, F, E, _ptr(w_gate),
                                           _ptr(w_up), _ptr(h), _ptr(gu), _stream()))


def grouped_gemm_swiglu_backward(x_perm: torch.Tensor, h: torch.Tensor, gu: Optional[torch.Tensor],
                                 dy_perm: torch.Tensor, expert_offsets: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor,
                                 wgu_t: torch.Tensor, wd_t: torch.Tensor, dx_perm: torch.Tensor, dw_gate: torch.Tensor,
                                 dw_up: torch.Tensor, dw_down: torch.Tensor, workspace: torch.Tensor) -> None:
    R_max, H = x_perm.shape
    E, F, _ = w_gate.shape
    _check(lib().moe_grouped_gemm_swiglu_backward(_ptr(x_perm), _ptr(h), _ptr(gu), _ptr(dy_perm), _ptr(expert_offsets), R_max, H,
                                                  F, E, _ptr(w_gate), _ptr(w_up), _ptr(wgu_t), _ptr(wd_t),
                                                  _ptr(dx_perm), _ptr(dw_gate), _ptr(dw_up), _ptr(dw_down),
                                                  _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                  _stream()))


def unpermute_combine_backward(dy: torch.Tensor, y_perm: torch.Tensor, row_of_assign: torch.Tensor,
                               topk_gate: torch.Tensor, dy_perm: torch.Tensor, dgate: torch.Tensor) -> None:
    T, K = topk_gate.shape
    R_max, H = y_perm.shape
    _check(lib().moe_unpermute_combine_backward(_ptr(dy), _ptr(y_perm), _ptr(row_of_assign), _ptr(topk_gate), T, H, K,
                                                R_max, _dt(dy), _ptr(dy_perm), _ptr(dgate), _stream()))


def permute_backward(dx_perm: torch.Tensor, row_of_assign: torch.Tensor, addend: Optional[torch.Tensor],
                     dx: torch.Tensor, K: int) -> None:
    T, H = dx.shape
    _check(lib().moe_permute_backward(_ptr(dx_perm), _ptr(row_of_assign), _ptr(addend), T, H, K, dx_perm.shape[0],
                                      _dt(dx), _ptr(dx), _stream()))


def permute_variant_workspace_bytes(T: int, K: int, E: int) -> int:
    return int(lib().moe_permute_variant_workspace_bytes(T, K, E))


def permute_variant(x: Optional[torch.Tensor], topk_idx: torch.Tensor, scores: Optional[torch.Tensor], E: int,
                    capacity: int, drop_by_score: bool, pad_to_capacity: bool, x_perm: Optional[torch.Tensor],
                    expert_counts: torch.Tensor, expert_offsets: torch.Tensor, row_of_assign: torch.Tensor,
                    assign_of_row: torch.Tensor, workspace: torch.Tensor, H: Optional[int] = None,
                    dtype: Optional[int] = None) -> None:
    T, K = topk_idx.shape
    if x is not None:
        H, dtype = x.shape[1], _dt(x)
    _check(lib().moe_permute_variant(_ptr(x), _ptr(topk_idx), _ptr(scores), T, H or 8, E, K, capacity,
                                     int(drop_by_score), int(pad_to_capacity), MOE_BF16 if dtype is None else dtype,
                                     _ptr(x_perm), _ptr(expert_counts), _ptr(expert_offsets), _ptr(row_of_assign),
                                     _ptr(assign_of_row), assign_of_row.numel(), _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream()))


def sort_chunks_workspace_bytes(n_dst: int) -> int:
    return int(lib().moe_sort_chunks_workspace_bytes(n_dst))


def sort_chunks(src: Optional[torch.Tensor], chunk_rows: torch.Tensor, order: torch.Tensor, group: int,
                dst: Optional[torch.Tensor], chunk_rows_out: Optional[torch.Tensor],
                group_offsets: Optional[torch.Tensor], workspace: torch.Tensor, H: Optional[int] = None,
                dtype: Optional[int] = None) -> None:
    ref = src if src is not None else dst
    if ref is not None:
        H, dtype = ref.shape[1], _dt(ref)
    _check(lib().moe_sort_chunks(_ptr(src), 0 if src is None else src.shape[0], _ptr(chunk_rows), chunk_rows.numel(),
                                 _ptr(order), order.numel(), group, H or 8, MOE_BF16 if dtype is None else dtype,
                                 _ptr(dst), 0 if dst is None else dst.shape[0], _ptr(chunk_rows_out),
                                 _ptr(group_offsets), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                 _stream()))


def probe_mfma_bf16(image: torch.Tensor, iters: int, workgroups: int, sink: torch.Tensor,
                    ticks: Optional[torch.Tensor]) -> None:
    assert image.numel() * image.element_size() == 65536 and sink.numel() >= workgroups * 256
    _check(lib().moe_probe_mfma_bf16(_ptr(image), iters, workgroups, _ptr(sink), _ptr(ticks), _stream()))


def layer_forward_train(x: torch.Tensor, w_router: torch.Tensor, logit_bias: Optional[torch.Tensor],
                        w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, K: int, renormalize: bool,
                        capacity: int, y: torch.Tensor, gu: torch.Tensor, workspace: torch.Tensor) -> None:
    T, H = x.shape
    E, F, _ = w_gate.shape
    _check(lib().moe_layer_forward_train(_ptr(x), _ptr(w_router), _ptr(logit_bias), _ptr(w_gate), _ptr(w_up),
                                         _ptr(w_down), T, H, E, K, F, int(renormalize), int(capacity), _ptr(y), _ptr(gu),
                                         _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))


def layer_backward_workspace_bytes(T: int, H: int, E: int, K: int, F: int, capacity: int) -> int:
    return int(lib().moe_layer_backward_workspace_bytes(T, H, E, K, F, capacity))


def layer_backward(x: torch.Tensor, w_router: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor,
                   wgu_t: torch.Tensor, wd_t: torch.Tensor, dy: torch.Tensor, K: int, renormalize: bool, capacity: int,
                   forward_workspace: torch.Tensor, gu: Optional[torch.Tensor], dx: torch.Tensor,
                   dw_router: Optional[torch.Tensor], dbias: Optional[torch.Tensor], dw_gate: torch.Tensor,
                   dw_up: torch.Tensor, dw_down: torch.Tensor, workspace: torch.Tensor,
                   dlogits_addend: Optional[torch.Tensor] = None) -> None:
    T, H = x.shape
    E, F, _ = w_gate.shape
    if dlogits_addend is not None:
        addend = _expect("dlogits_addend", dlogits_addend, torch.float32, T * E)
        _check(lib().moe_layer_backward_addend(_ptr(x), _ptr(w_router), _ptr(w_gate), _ptr(w_up), _ptr(wgu_t),
                                               _ptr(wd_t), _ptr(dy), addend, T, H, E, K, F,
                                               int(renormalize), int(capacity), _ptr(forward_workspace), _ptr(gu),
                                               _ptr(dx), _ptr(dw_router), _ptr(dbias), _ptr(dw_gate), _ptr(dw_up),
                                               _ptr(dw_down), _ptr(workspace),
                                               workspace.numel() * workspace.element_size(), _stream()))
        return
    _check(lib().moe_layer_backward(_ptr(x), _ptr(w_router), _ptr(w_gate), _ptr(w_up), _ptr(wgu_t), _ptr(wd_t),
                                    _ptr(dy), T, H, E, K, F, int(renormalize), int(capacity), _ptr(forward_workspace),
                                    _ptr(gu), _ptr(dx), _ptr(dw_router), _ptr(dbias), _ptr(dw_gate), _ptr(dw_up),
                                    _ptr(dw_down), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                    _stream()))


def probe_mfma_fp8(image: torch.Tensor, iters: int, workgroups: int, sink: torch.Tensor,
                   ticks: Optional[torch.Tensor]) -> None:
    assert image.numel() * image.element_size() == 65536 and sink.numel() >= workgroups * 256
    _check(lib().moe_probe_mfma_fp8(_ptr(image), iters, workgroups, _ptr(sink), _ptr(ticks), _stream()))


def layer_workspace_bytes(T: int, H: int, E: int, K: int, F: int, Fs: int, capacity: int, dtype: int) -> int:
    return int(lib().moe_layer_workspace_bytes(T, H, E, K, F, Fs, capacity, dtype))


def workspace_bytes(T: int, H: int, E: int, K: int, F: int, capacity: int, dtype: int) -> int:
    return int(lib().moe_workspace_bytes(T, H, E, K, F, capacity, dtype))


def gemm_clock_sample(ticks: Optional[torch.Tensor]) -> None:
    """ticks: int64 device tensor of 2 elements that the following grouped bf16 GEMM launches fill, or None."""
    if ticks is not None and (ticks.dtype != torch.int64 or ticks.numel() < 2):
        raise ValueError("ticks must be an int64 tensor with at least 2 elements")
    _check(lib().moe_gemm_clock_sample(_ptr(ticks)))


_LAYOUT_NAMES = ("logits", "topk_idx", "topk_gate", "expert_counts", "expert_offsets", "row_of_assign",
                 "assign_of_row", "x_perm", "h", "y_perm", "shared_y")


def layer_workspace_layout(T: int, H: int, E: int, K: int, F: int, Fs: int, capacity: int, dtype: int) -> dict:
    arr = (C.c_size_t * 11)()
    _check(lib().moe_layer_workspace_layout(T, H, E, K, F, Fs, capacity, dtype, arr, 11))
    return dict(zip(_LAYOUT_NAMES, (int(v) for v in arr)))


def layer_forward(x: torch.Tensor, w_router: torch.Tensor, logit_bias: Optional[torch.Tensor],
                  w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                  ws_gate: Optional[torch.Tensor], ws_up: Optional[torch.Tensor],
                  ws_down: Optional[torch.Tensor], K: int, renormalize: bool, capacity: int,
                  y: torch.Tensor, workspace: torch.Tensor) -> None:
    T, H = x.shape
    E, F, _ = w_gate.shape
    Fs = 0 if ws_gate is None else ws_gate.shape[0]
    _check(lib().moe_layer_forward(_ptr(x), _ptr(w_router), _ptr(logit_bias), _ptr(w_gate), _ptr(w_up),
                                   _ptr(w_down), _ptr(ws_gate), _ptr(ws_up), _ptr(ws_down), T, H, E, K, F,
                                   Fs, int(bool(renormalize)), int(capacity), _dt(x), _ptr(y),
                                   _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()))
