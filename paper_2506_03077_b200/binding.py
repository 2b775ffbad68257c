"""ctypes binding of libstreambp.so: the same entry points as include/streambp.h.

Only argument marshalling happens here (torch tensors -> device pointers, Python
dataclasses -> C structs); every step of the computation runs in the CUDA library.
There is no fallback: if the library is missing or cannot be loaded, importing
`lib()` raises.
"""
from __future__ import annotations

import ctypes as C
import os
from bisect import bisect_left
from dataclasses import dataclass
from typing import Dict, List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libstreambp.so")

STREAMBP_F32, STREAMBP_BF16 = 0, 1
OK = 0
E_NULL, E_SHAPE, E_ALIGN, E_WORKSPACE, E_DTYPE, E_CUDA, E_BAD_LABEL, E_NO_VALID_LABELS, E_DEVICE_TIMEOUT, \
    E_WORKSPACE_GUARD = range(-1, -11, -1)
OP_NT, OP_NN, OP_TN = 0, 1, 2

WEIGHT_FIELDS = ("g1", "wq", "bq", "wk", "bk", "wv", "bv", "wo", "g2", "w_gate", "w_up", "w_down")

EXPORTS = (
    "streambp_layer_workspace_bytes", "streambp_layer_backward",
    "streambp_lmhead_workspace_bytes", "streambp_lmhead_ce_backward",
    "streambp_model_workspace_bytes", "streambp_model_backward",
    "streambp_last_device_status", "streambp_status_string",
    "streambp_last_cuda_error", "streambp_last_launch_count", "streambp_gemm", "streambp_gemm_grouped", "streambp_gemm_swiglu",
    "streambp_layer_suggest_chunk", "streambp_lmhead_suggest_chunk",
    "streambp_profile_enable", "streambp_profile_read", "streambp_product_kernel",
    "streambp_attention_forward", "streambp_attention_backward", "streambp_attention_backward_static",
    "streambp_lmhead_rl_backward", "streambp_layer_backward_packed",
    "streambp_test_expire_wait", "streambp_test_per_device_value", "streambp_test_sort_cluster",
    "streambp_layer_workspace_bytes_grouped", "streambp_layer_backward_grouped", "streambp_test_workspace_guard",
    "streambp_lmhead_workspace_bytes_grouped", "streambp_lmhead_ce_backward_grouped",
    "streambp_lmhead_rl_backward_grouped",
    "streambp_adamw_step", "streambp_grad_norm_workspace_bytes", "streambp_grad_norm", "streambp_mx8_encode",
    "streambp_mx8_decode", "streambp_gemm_epilogue", "streambp_gemm_epilogue_workspace_bytes",
    "streambp_gemm_epilogue_backward", "streambp_attention_window_forward", "streambp_attention_window_workspace_bytes",
    "streambp_attention_window_backward",
    "streambp_token_logprobs_workspace_bytes", "streambp_token_logprobs", "streambp_token_logprobs_backward",
    "streambp_distill_topk_workspace_bytes", "streambp_distill_topk", "streambp_lmhead_logprobs_workspace_bytes",
    "streambp_lmhead_logprobs", "streambp_lmhead_distill_workspace_bytes", "streambp_lmhead_distill_backward",
    "streambp_layernorm_forward", "streambp_layernorm_workspace_bytes", "streambp_layernorm_backward",
    "streambp_embedding_workspace_bytes", "streambp_embedding_forward", "streambp_embedding_backward_workspace_bytes",
    "streambp_embedding_backward",
)


class LayerCfgC(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("d_ff", C.c_int32), ("qkv_bias", C.c_int32),
                ("rope_theta", C.c_float), ("rms_eps", C.c_float), ("dtype", C.c_int32)]


class LayerPtrsC(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in WEIGHT_FIELDS]


class HeadCfgC(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("vocab", C.c_int64), ("rms_eps", C.c_float),
                ("ignore_index", C.c_int64), ("dtype", C.c_int32)]


class RlCfgC(C.Structure):
    _fields_ = [("objective", C.c_int32), ("beta", C.c_float), ("clip_eps", C.c_float)]


class DistillCfgC(C.Structure):
    _fields_ = [("k", C.c_int32), ("tail", C.c_int32), ("temperature", C.c_float)]


class GemmProblemC(C.Structure):
    _fields_ = [("op", C.c_int32), ("n_segments", C.c_int32), ("M", C.c_int64), ("N", C.c_int64),
                ("A", C.c_void_p * 3), ("lda", C.c_int64 * 3), ("B", C.c_void_p * 3), ("ldb", C.c_int64 * 3),
                ("K", C.c_int64 * 3), ("C", C.c_void_p), ("ldc", C.c_int64), ("out_dtype", C.c_int32),
                ("accumulate", C.c_int32)]


class AdamWTensorC(C.Structure):
    _fields_ = [("param", C.c_void_p), ("master", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p),
                ("v", C.c_void_p), ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("count", C.c_int64),
                ("weight_decay", C.c_float)]


class AdamWCfgC(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("param_dtype", C.c_int32), ("state_dtype", C.c_int32), ("step", C.c_int64)]


class ModelCfgC(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("layer", LayerCfgC), ("head", HeadCfgC)]


class StreamBPError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: status {status} ({status_string(status)})")


_lib = None


def lib() -> C.CDLL:
    """Load libstreambp.so (built by paper_2506_03077_b200.build). Raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} not found: build it with `python -m paper_2506_03077_b200.build` "
            "(there is no CPU or PyTorch fallback)")
    L = C.CDLL(LIB_PATH)
    vp, i64, sz, i32 = C.c_void_p, C.c_int64, C.c_size_t, C.c_int32
    L.streambp_layer_workspace_bytes.restype = sz
    L.streambp_layer_workspace_bytes.argtypes = [C.POINTER(LayerCfgC), i64, i64]
    L.streambp_layer_backward.restype = C.c_int
    L.streambp_layer_backward.argtypes = [C.POINTER(LayerCfgC), C.POINTER(LayerPtrsC), vp, vp, i64, i64, i64, C.c_int,
                                          C.POINTER(LayerPtrsC), vp, vp, sz, vp]
    L.streambp_layer_backward_packed.restype = C.c_int
    L.streambp_layer_backward_packed.argtypes = [C.POINTER(LayerCfgC), C.POINTER(LayerPtrsC), vp, vp, i64, i64,
                                                 C.POINTER(i64), i32, i64, C.c_int, C.POINTER(LayerPtrsC), vp, vp, sz, vp]
    L.streambp_layer_workspace_bytes_grouped.restype = sz
    L.streambp_layer_workspace_bytes_grouped.argtypes = [C.POINTER(LayerCfgC), i64, i64, i32]
    L.streambp_layer_backward_grouped.restype = C.c_int
    L.streambp_layer_backward_grouped.argtypes = [C.POINTER(LayerCfgC), C.POINTER(LayerPtrsC), vp, vp, i64, i64, i32,
                                                  C.POINTER(i64), i32, i64, C.c_int, C.POINTER(LayerPtrsC), vp, vp, sz, vp]
    L.streambp_lmhead_workspace_bytes.restype = sz
    L.streambp_lmhead_workspace_bytes.argtypes = [C.POINTER(HeadCfgC), i64, i64]
    L.streambp_lmhead_ce_backward.restype = C.c_int
    L.streambp_lmhead_ce_backward.argtypes = [C.POINTER(HeadCfgC), vp, vp, vp, vp, i64, i64, C.c_int, vp, vp, vp, vp,
                                              vp, vp, sz, vp]
    L.streambp_lmhead_rl_backward.restype = C.c_int
    L.streambp_lmhead_rl_backward.argtypes = [C.POINTER(HeadCfgC), C.POINTER(RlCfgC), vp, vp, vp, vp, vp, vp, vp, vp,
                                              i64, i64, C.c_int, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.streambp_lmhead_workspace_bytes_grouped.restype = sz
    L.streambp_lmhead_workspace_bytes_grouped.argtypes = [C.POINTER(HeadCfgC), i64, i64, i32]
    L.streambp_lmhead_ce_backward_grouped.restype = C.c_int
    L.streambp_lmhead_ce_backward_grouped.argtypes = [C.POINTER(HeadCfgC), vp, vp, vp, vp, i64, i64, i32, C.c_int, vp,
                                                      vp, vp, vp, vp, vp, sz, vp]
    L.streambp_lmhead_rl_backward_grouped.restype = C.c_int
    L.streambp_lmhead_rl_backward_grouped.argtypes = [C.POINTER(HeadCfgC), C.POINTER(RlCfgC), vp, vp, vp, vp, vp, vp,
                                                      vp, vp, i64, i64, i32, C.c_int, vp, vp, vp, vp, vp, vp, vp, sz,
                                                      vp]
    L.streambp_model_workspace_bytes.restype = sz
    L.streambp_model_workspace_bytes.argtypes = [C.POINTER(ModelCfgC), i64, i64, i64]
    L.streambp_model_backward.restype = C.c_int
    L.streambp_model_backward.argtypes = [C.POINTER(ModelCfgC), vp, C.POINTER(LayerPtrsC), vp, vp, vp, vp, vp, i64,
                                          i64, i64, C.c_int, vp, vp, C.POINTER(LayerPtrsC), vp, vp, vp, vp, sz, vp]
    L.streambp_last_device_status.restype = C.c_int
    L.streambp_last_device_status.argtypes = [vp, vp]
    L.streambp_status_string.restype = C.c_char_p
    L.streambp_status_string.argtypes = [C.c_int]
    L.streambp_last_cuda_error.restype = C.c_int
    L.streambp_last_cuda_error.argtypes = []
    L.streambp_last_launch_count.restype = i64
    L.streambp_last_launch_count.argtypes = []
    L.streambp_layer_suggest_chunk.restype = i64
    L.streambp_layer_suggest_chunk.argtypes = [C.POINTER(LayerCfgC), i64, sz]
    L.streambp_lmhead_suggest_chunk.restype = i64
    L.streambp_lmhead_suggest_chunk.argtypes = [C.POINTER(HeadCfgC), i64, sz]
    L.streambp_gemm_grouped.restype = C.c_int
    L.streambp_gemm_grouped.argtypes = [C.POINTER(GemmProblemC), i32, vp, vp]
    L.streambp_gemm_swiglu.restype = C.c_int
    L.streambp_gemm_swiglu.argtypes = [vp, i64, vp, vp, i64, i64, i64, i64, vp, vp, vp, i32, vp]
    L.streambp_gemm.restype = C.c_int
    L.streambp_gemm.argtypes = [C.c_int, i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, i32, C.c_int, C.c_int, vp]
    L.streambp_attention_forward.restype = C.c_int
    L.streambp_attention_forward.argtypes = [vp, vp, vp, i64, i64, i32, i32, i32, i32, vp, vp, C.c_int, vp]
    L.streambp_attention_backward.restype = C.c_int
    L.streambp_attention_backward.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i32, i32, i32, i32, vp, vp, vp, vp,
                                              C.c_int, vp]
    L.streambp_attention_backward_static.restype = C.c_int
    L.streambp_attention_backward_static.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i32, i32, i32, i32, vp, vp, vp,
                                                     C.c_int, vp]
    L.streambp_product_kernel.restype = C.c_int
    L.streambp_product_kernel.argtypes = []
    L.streambp_profile_enable.restype = None
    L.streambp_profile_enable.argtypes = [C.c_int]
    L.streambp_profile_read.restype = C.c_int
    L.streambp_profile_read.argtypes = [C.c_int, C.POINTER(C.c_double), C.POINTER(i64), C.POINTER(C.c_double)]
    L.streambp_test_expire_wait.restype = C.c_int
    L.streambp_test_expire_wait.argtypes = [C.c_uint64, vp]
    L.streambp_test_workspace_guard.restype = C.c_int
    L.streambp_test_workspace_guard.argtypes = [vp, sz, i32, vp]
    L.streambp_test_per_device_value.restype = C.c_int
    L.streambp_test_per_device_value.argtypes = [C.c_int, C.c_int]
    L.streambp_test_sort_cluster.restype = C.c_int
    L.streambp_test_sort_cluster.argtypes = [C.c_int]
    L.streambp_gemm_epilogue.restype = C.c_int
    L.streambp_gemm_epilogue.argtypes = [vp, i64, vp, i64, i64, i64, i64, vp, i32, vp, i64, vp, i64, vp, i64, i32, vp]
    L.streambp_gemm_epilogue_workspace_bytes.restype = sz
    L.streambp_gemm_epilogue_workspace_bytes.argtypes = [i64, i64]
    L.streambp_gemm_epilogue_backward.restype = C.c_int
    L.streambp_gemm_epilogue_backward.argtypes = [vp, i64, vp, i64, i32, i64, i64, vp, i64, vp, C.c_int, i32, vp, sz, vp]
    L.streambp_attention_window_forward.restype = C.c_int
    L.streambp_attention_window_forward.argtypes = [vp, vp, vp, i64, i64, i32, i32, i32, i32, i64, i64, vp, vp, C.c_int, vp]
    L.streambp_attention_window_workspace_bytes.restype = sz
    L.streambp_attention_window_workspace_bytes.argtypes = [i64, i64, i32, i32, i32, i64, i64]
    L.streambp_attention_window_backward.restype = C.c_int
    L.streambp_attention_window_backward.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i32, i32, i32, i32, i64, i64, i32,
                                                     C.c_int, vp, vp, vp, vp, sz, C.c_int, vp]
    L.streambp_adamw_step.restype = C.c_int
    L.streambp_adamw_step.argtypes = [C.POINTER(AdamWCfgC), C.POINTER(AdamWTensorC), i32, vp, vp, vp]
    L.streambp_grad_norm_workspace_bytes.restype = sz
    L.streambp_grad_norm_workspace_bytes.argtypes = []
    L.streambp_grad_norm.restype = C.c_int
    L.streambp_grad_norm.argtypes = [C.POINTER(vp), C.POINTER(i64), i32, C.c_float, vp, vp, vp, sz, vp]
    L.streambp_mx8_encode.restype = C.c_int
    L.streambp_mx8_encode.argtypes = [vp, i64, i32, vp, vp, vp]
    L.streambp_mx8_decode.restype = C.c_int
    L.streambp_mx8_decode.argtypes = [vp, vp, i64, vp, i32, vp]
    f32 = C.c_float
    for name, restype, argtypes in (
            ("streambp_token_logprobs_workspace_bytes", sz, []),
            ("streambp_token_logprobs", C.c_int, [vp, i64, i64, i64, i32, vp, i64, f32, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
            ("streambp_token_logprobs_backward", C.c_int, [vp, i64, i64, i64, i32, vp, i64, f32, vp, vp, vp, vp, vp, vp, i64, vp]),
            ("streambp_distill_topk_workspace_bytes", sz, []),
            ("streambp_distill_topk", C.c_int, [C.POINTER(DistillCfgC), vp, i64, i64, i64, i32, vp, vp, vp, vp, vp, i64, vp, sz, vp]),
            ("streambp_lmhead_logprobs_workspace_bytes", sz, [C.POINTER(HeadCfgC), i64, i64]),
            ("streambp_lmhead_logprobs", C.c_int, [C.POINTER(HeadCfgC), vp, vp, vp, vp, i64, i64, f32, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
            ("streambp_lmhead_distill_workspace_bytes", sz, [C.POINTER(HeadCfgC), i64, i64, i32]),
            ("streambp_lmhead_distill_backward", C.c_int, [C.POINTER(HeadCfgC), C.POINTER(DistillCfgC), vp, vp, vp, vp, vp, vp, i64, i64,
                                                           i32, C.c_int, vp, vp, vp, vp, vp, vp, sz, vp]),
            ("streambp_layernorm_forward", C.c_int, [vp, i64, vp, vp, f32, i64, i64, i32, vp, i64, vp, vp, vp]),
            ("streambp_layernorm_workspace_bytes", sz, [i64, i64]),
            ("streambp_layernorm_backward", C.c_int, [vp, i64, vp, i64, vp, vp, vp, vp, i64, i64, i64, i32, vp, i64, vp, vp, C.c_int, vp,
                                                      sz, vp]),
            ("streambp_embedding_workspace_bytes", sz, []),
            ("streambp_embedding_forward", C.c_int, [vp, i64, vp, i64, i64, i64, i32, f32, i64, vp, i64, vp, sz, vp]),
            ("streambp_embedding_backward_workspace_bytes", sz, [i64, i64, i64]),
            ("streambp_embedding_backward", C.c_int, [vp, i64, vp, i64, i64, i64, i32, f32, i64, C.c_int, vp, vp, sz, vp])):
        fn = getattr(L, name)
        fn.restype, fn.argtypes = restype, argtypes
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().streambp_status_string(int(status)).decode()


def _check(status: int, what: str):
    if status != OK:
        extra = ""
        if status == E_CUDA:
            extra = f" [cuda error {lib().streambp_last_cuda_error()}]"
        raise StreamBPError(status, what + extra)


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.float32:
        return STREAMBP_F32
    if dt == torch.bfloat16:
        return STREAMBP_BF16
    raise TypeError(f"unsupported storage dtype {dt}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "tensors must be contiguous CUDA tensors"
    return t.data_ptr()


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _launch(what: str, device: int, stream: Optional[torch.cuda.Stream], fn, *args) -> int:
    """fn(*args, stream) with the tensors' device current (it need not be the caller's), on the given stream, which must
    belong to that device, or on that device's current stream."""
    if stream is not None and stream.device_index != device:
        raise ValueError(f"{what}: the stream belongs to cuda:{stream.device_index}, the tensors lie on cuda:{device}")
    raw = stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(device)
    if torch._C._cuda_getDevice() == device:
        return fn(*args, raw)
    with torch.cuda.device(device):
        return fn(*args, raw)


def _same(what: str, device: int, *tensors) -> None:
    """All tensors contiguous and on that CUDA device."""
    for t in tensors:
        if t.get_device() != device or device < 0 or not t.is_contiguous():
            raise ValueError(f"{what}: tensors must be contiguous CUDA tensors on one device")


def _want(ok: bool, what: str, rule: str) -> None:
    if not ok:
        raise ValueError(f"{what}: {rule}")


@dataclass
class LayerConfig:
    d_model: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    d_ff: int
    qkv_bias: bool
    rope_theta: float
    rms_eps: float = 1e-6
    dtype: torch.dtype = torch.bfloat16

    def c(self) -> LayerCfgC:
        return LayerCfgC(self.d_model, self.n_q_heads, self.n_kv_heads, self.head_dim, self.d_ff,
                         1 if self.qkv_bias else 0, self.rope_theta, self.rms_eps, _dtype_code(self.dtype))


@dataclass
class HeadConfig:
    d_model: int
    vocab: int
    rms_eps: float = 1e-6
    ignore_index: int = -100
    dtype: torch.dtype = torch.bfloat16

    def c(self) -> HeadCfgC:
        return HeadCfgC(self.d_model, self.vocab, self.rms_eps, self.ignore_index, _dtype_code(self.dtype))


def _ptr_struct(tensors: Dict[str, torch.Tensor]) -> LayerPtrsC:
    return LayerPtrsC(**{f: _ptr(tensors.get(f)) for f in WEIGHT_FIELDS})


def layer_grad_shapes(cfg: LayerConfig) -> Dict[str, tuple]:
    dq, dkv, d, I = cfg.n_q_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim, cfg.d_model, cfg.d_ff
    shp = {"g1": (d,), "wq": (dq, d), "wk": (dkv, d), "wv": (dkv, d), "wo": (d, dq), "g2": (d,),
           "w_gate": (I, d), "w_up": (I, d), "w_down": (d, I)}
    if cfg.qkv_bias:
        shp.update({"bq": (dq,), "bk": (dkv,), "bv": (dkv,)})
    return shp


def alloc_layer_grads(cfg: LayerConfig, device="cuda") -> Dict[str, torch.Tensor]:
    return {k: torch.zeros(s, dtype=torch.float32, device=device) for k, s in layer_grad_shapes(cfg).items()}


def layer_workspace_bytes(cfg: LayerConfig, T: int, chunk: int, wgrad_group: int = 1) -> int:
    c = cfg.c()
    if wgrad_group != 1:
        return int(lib().streambp_layer_workspace_bytes_grouped(C.byref(c), T, chunk, wgrad_group))
    return int(lib().streambp_layer_workspace_bytes(C.byref(c), T, chunk))


def layer_suggest_chunk(cfg: LayerConfig, T: int, budget_bytes: int) -> int:
    """Largest chunk (multiple of 128 rows, or T) whose layer workspace fits budget_bytes; 0 if none does."""
    c = cfg.c()
    return int(lib().streambp_layer_suggest_chunk(C.byref(c), T, budget_bytes))


def lmhead_suggest_chunk(cfg: HeadConfig, T: int, budget_bytes: int) -> int:
    c = cfg.c()
    return int(lib().streambp_lmhead_suggest_chunk(C.byref(c), T, budget_bytes))


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def layer_backward(cfg: LayerConfig, weights: Dict[str, torch.Tensor], X: torch.Tensor, dY: torch.Tensor,
                   chunk: int, grads: Dict[str, torch.Tensor], dX: torch.Tensor, workspace: torch.Tensor,
                   pos0: int = 0, accumulate: bool = False, stream=None, check: bool = True, wgrad_group: int = 1,
                   cu_seqlens: Optional[Sequence[int]] = None) -> int:
    """streambp_layer_backward (or streambp_layer_backward_grouped when wgrad_group != 1); returns the status
    (raises on error when check=True)."""
    c = cfg.c()
    w, g = _ptr_struct(weights), _ptr_struct(grads)
    if wgrad_group != 1:
        cu = (C.c_int64 * len(cu_seqlens))(*cu_seqlens) if cu_seqlens is not None else None
        st = lib().streambp_layer_backward_grouped(C.byref(c), C.byref(w), _ptr(X), _ptr(dY), X.shape[0], chunk,
                                                   wgrad_group, cu, len(cu_seqlens) - 1 if cu_seqlens is not None else 0,
                                                   pos0, 1 if accumulate else 0, C.byref(g), _ptr(dX), _ptr(workspace),
                                                   workspace.numel(), _stream_ptr(stream))
        if check:
            _check(st, "streambp_layer_backward_grouped")
        return st
    st = lib().streambp_layer_backward(C.byref(c), C.byref(w), _ptr(X), _ptr(dY), X.shape[0], chunk, pos0,
                                       1 if accumulate else 0, C.byref(g), _ptr(dX), _ptr(workspace),
                                       workspace.numel(), _stream_ptr(stream))
    if check:
        _check(st, "streambp_layer_backward")
    return st


class HostFedLayerBackward:
    """streambp_layer_backward for activations that live in pinned host memory (plumbing only: streams, events and
    copies; every step of the path still runs in the library's kernels).  Two sets of device buffers alternate:
    while the kernels of step k run on the compute stream, a copy stream brings in the X, dY of step k+1 and
    takes out the dX of step k-1, so a sequence's 3 T d storage-dtype values cross PCIe behind the compute of
    its neighbours instead of in front of its own."""

    def __init__(self, cfg: LayerConfig, weights, grads, T: int, chunk: int, workspace: torch.Tensor,
                 wgrad_group: int = 1):
        self.wgrad_group = wgrad_group
        self.cfg, self.weights, self.grads, self.chunk, self.ws = cfg, weights, grads, chunk, workspace
        dev = workspace.device
        mk = lambda: torch.empty(T, cfg.d_model, dtype=cfg.dtype, device=dev)
        self.X, self.dY, self.dX = [mk(), mk()], [mk(), mk()], [mk(), mk()]
        self.copy_stream = torch.cuda.Stream(device=dev)
        self.loaded = [torch.cuda.Event(), torch.cuda.Event()]      # inputs of buffer i are on the device
        self.computed = [torch.cuda.Event(), torch.cuda.Event()]    # the call on buffer i has finished
        self.n_prefetched = 0       # prefetch() calls so far; call k fills buffer pair k % 2
        self.n_run = 0              # step() calls so far; call k consumes buffer pair k % 2

    def prefetch(self, X_host: torch.Tensor, dY_host: torch.Tensor) -> None:
        """Starts the host-to-device copy of the inputs of the next step that has none yet (at most two ahead)."""
        assert self.n_prefetched - self.n_run < 2, "both buffer pairs hold inputs that have not been consumed"
        i = self.n_prefetched & 1
        cs = self.copy_stream
        if self.n_prefetched >= 2:
            cs.wait_event(self.computed[i])     # the previous user of these buffers is done with them
        with torch.cuda.stream(cs):
            self.X[i].copy_(X_host, non_blocking=True)
            self.dY[i].copy_(dY_host, non_blocking=True)
            self.loaded[i].record(cs)
        self.n_prefetched += 1

    def step(self, dX_host: torch.Tensor, accumulate: bool = False, stream=None) -> None:
        """Runs the backward on the oldest prefetched inputs and starts the copy of its dX to dX_host.  The copy
        stream is in order, so that copy also precedes the next prefetch into the same buffer pair."""
        assert self.n_run < self.n_prefetched, "prefetch() the inputs first"
        i = self.n_run & 1
        st = stream if stream is not None else torch.cuda.current_stream()
        st.wait_event(self.loaded[i])
        layer_backward(self.cfg, self.weights, self.X[i], self.dY[i], self.chunk, self.grads, self.dX[i], self.ws,
                       accumulate=accumulate, stream=st, wgrad_group=self.wgrad_group)
        self.computed[i].record(st)
        cs = self.copy_stream
        cs.wait_event(self.computed[i])
        with torch.cuda.stream(cs):
            dX_host.copy_(self.dX[i], non_blocking=True)
        self.n_run += 1

    def drain(self, stream=None) -> None:
        """Makes `stream` wait for the copies that are still in flight."""
        st = stream if stream is not None else torch.cuda.current_stream()
        st.wait_stream(self.copy_stream)


def layer_backward_packed(cfg: LayerConfig, weights, X, dY, chunk: int, cu_seqlens: Sequence[int], grads, dX, workspace,
                          pos0: int = 0, accumulate: bool = False, stream=None, check: bool = True) -> int:
    """streambp_layer_backward_packed: X, dY hold the sequences back to back; cu_seqlens = [0, ..., T] on the host."""
    c = cfg.c()
    w, g = _ptr_struct(weights), _ptr_struct(grads)
    n = len(cu_seqlens) - 1
    cu = (C.c_int64 * (n + 1))(*[int(v) for v in cu_seqlens])
    st = lib().streambp_layer_backward_packed(C.byref(c), C.byref(w), _ptr(X), _ptr(dY), X.shape[0], chunk, cu, n, pos0,
                                              1 if accumulate else 0, C.byref(g), _ptr(dX), _ptr(workspace),
                                              workspace.numel(), _stream_ptr(stream))
    if check:
        _check(st, "streambp_layer_backward_packed")
    return st


def lmhead_workspace_bytes(cfg: HeadConfig, T: int, chunk: int, wgrad_group: int = 1) -> int:
    c = cfg.c()
    if wgrad_group == 1:
        return int(lib().streambp_lmhead_workspace_bytes(C.byref(c), T, chunk))
    return int(lib().streambp_lmhead_workspace_bytes_grouped(C.byref(c), T, chunk, wgrad_group))


def lmhead_ce_backward(cfg: HeadConfig, g_final, w_vocab, H, labels, chunk: int, loss, n_valid, dH, d_w_vocab,
                       d_g_final, workspace, accumulate: bool = False, stream=None, check: bool = True,
                       wgrad_group: int = 1) -> int:
    """streambp_lmhead_ce_backward; wgrad_group != 1 goes through streambp_lmhead_ce_backward_grouped."""
    c = cfg.c()
    head = (C.byref(c), _ptr(g_final), _ptr(w_vocab), _ptr(H), _ptr(labels), H.shape[0], chunk)
    tail = (1 if accumulate else 0, _ptr(loss), _ptr(n_valid), _ptr(dH), _ptr(d_w_vocab), _ptr(d_g_final),
            _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if wgrad_group == 1:
        name, st = "streambp_lmhead_ce_backward", lib().streambp_lmhead_ce_backward(*head, *tail)
    else:
        name = "streambp_lmhead_ce_backward_grouped"
        st = lib().streambp_lmhead_ce_backward_grouped(*head, wgrad_group, *tail)
    if check:
        _check(st, name)
    return st


def _model_cfg(n_layers: int, layer: LayerConfig, head: HeadConfig) -> ModelCfgC:
    return ModelCfgC(n_layers, layer.c(), head.c())


def model_workspace_bytes(n_layers: int, layer: LayerConfig, head: HeadConfig, T: int, chunk_layer: int,
                          chunk_head: int) -> int:
    c = _model_cfg(n_layers, layer, head)
    return int(lib().streambp_model_workspace_bytes(C.byref(c), T, chunk_layer, chunk_head))


def model_backward(layer: LayerConfig, head: HeadConfig, layers: Sequence[Dict[str, torch.Tensor]], g_final, w_vocab,
                   labels, chunk_layer: int, chunk_head: int, loss, layer_grads: Sequence[Dict[str, torch.Tensor]],
                   d_g_final, d_w_vocab, workspace, embed=None, ids=None, X0=None, d_embed=None, dX0=None,
                   accumulate: bool = False, stream=None, check: bool = True) -> int:
    L = len(layers)
    c = _model_cfg(L, layer, head)
    W = (LayerPtrsC * L)(*[_ptr_struct(w) for w in layers])
    G = (LayerPtrsC * L)(*[_ptr_struct(g) for g in layer_grads])
    T = labels.shape[0]
    st = lib().streambp_model_backward(C.byref(c), _ptr(embed), W, _ptr(g_final), _ptr(w_vocab), _ptr(ids), _ptr(X0),
                                       _ptr(labels), T, chunk_layer, chunk_head, 1 if accumulate else 0, _ptr(loss),
                                       _ptr(d_embed), G, _ptr(d_g_final), _ptr(d_w_vocab), _ptr(dX0), _ptr(workspace),
                                       workspace.numel(), _stream_ptr(stream))
    if check:
        _check(st, "streambp_model_backward")
    return st


def last_device_status(workspace: torch.Tensor, stream=None) -> int:
    return int(lib().streambp_last_device_status(_ptr(workspace), _stream_ptr(stream)))


def last_launch_count() -> int:
    return int(lib().streambp_last_launch_count())


def gemm(op: int, A: torch.Tensor, B: torch.Tensor, C_out: torch.Tensor, accumulate: bool = False, engine: int = 0,
         stream=None, check: bool = True) -> int:
    """streambp_gemm on 2-D row-major tensors (leading dimension = stride(0))."""
    if op == OP_NT:
        M, K = A.shape
        N = B.shape[0]
    elif op == OP_NN:
        M, K = A.shape
        N = B.shape[1]
    else:
        K, M = A.shape
        N = B.shape[1]
    assert A.stride(1) == 1 and B.stride(1) == 1 and C_out.stride(1) == 1
    st = lib().streambp_gemm(op, M, N, K, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0), C_out.data_ptr(),
                             C_out.stride(0), _dtype_code(A.dtype), _dtype_code(C_out.dtype), 1 if accumulate else 0,
                             engine, _stream_ptr(stream))
    if check:
        _check(st, "streambp_gemm")
    return st


def gemm_grouped(problems, sched: Optional[torch.Tensor] = None, stream=None, check: bool = True) -> int:
    """streambp_gemm_grouped.  problems: list of (op, [(A, B), ...], C_out, accumulate) with 2-D row-major bf16
    operands; each problem sums its (A, B) segments.  sched: None or an int32 CUDA tensor of two zeros."""
    arr = (GemmProblemC * len(problems))()
    for i, (op, segs, C_out, acc) in enumerate(problems):
        g = arr[i]
        g.op, g.n_segments = op, len(segs)
        for s, (A, B) in enumerate(segs):
            assert A.stride(1) == 1 and B.stride(1) == 1
            if op == OP_NT:
                M, K, N = A.shape[0], A.shape[1], B.shape[0]
            elif op == OP_NN:
                M, K, N = A.shape[0], A.shape[1], B.shape[1]
            else:
                K, M, N = A.shape[0], A.shape[1], B.shape[1]
            g.A[s], g.lda[s], g.B[s], g.ldb[s], g.K[s] = A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0), K
        g.M, g.N = M, N
        assert C_out.stride(1) == 1 and tuple(C_out.shape) == (M, N)
        g.C, g.ldc, g.out_dtype, g.accumulate = C_out.data_ptr(), C_out.stride(0), _dtype_code(C_out.dtype), 1 if acc else 0
    st = lib().streambp_gemm_grouped(arr, len(problems), _ptr(sched), _stream_ptr(stream))
    if check:
        _check(st, "streambp_gemm_grouped")
    return st


def gemm_swiglu(A, w_gate, w_up, g, u, m, stream=None, check: bool = True) -> int:
    """streambp_gemm_swiglu: g = A w_gate^T, u = A w_up^T, m = silu(g) * u; A [M, K], weights [N, K], outputs [M, N] dense."""
    M, K = A.shape
    N = w_gate.shape[0]
    assert A.stride(1) == 1 and w_gate.stride(1) == 1 and w_up.stride(1) == 1 and w_gate.stride(0) == w_up.stride(0)
    for t in (g, u, m):
        assert t.is_contiguous() and tuple(t.shape) == (M, N)
    st = lib().streambp_gemm_swiglu(_ptr(A), A.stride(0), _ptr(w_gate), _ptr(w_up), w_gate.stride(0), M, N, K, _ptr(g),
                                    _ptr(u), _ptr(m), _dtype_code(A.dtype), _stream_ptr(stream))
    if check:
        _check(st, "streambp_gemm_swiglu")
    return st


ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


def _rows(what: str, dev: int, dtype: torch.dtype, shape: tuple, t: Optional[torch.Tensor]) -> tuple:
    """(address, leading dimension) of a matrix whose rows are contiguous; (None, 0) for None."""
    if t is None:
        return None, 0
    if t.get_device() != dev or t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{what}: expected a {dtype} tensor {shape} on cuda:{dev}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    rows, cols = t.stride()
    if (cols != 1 and shape[1] > 1) or (rows < shape[1] and shape[0] > 1):
        raise ValueError(f"{what}: rows must be contiguous and must not overlap (strides {t.stride()})")
    return t.data_ptr(), max(rows, shape[1])


def gemm_epilogue(A, W, C_out, bias=None, activation: str = "none", residual=None, pre=None, stream=None,
                  check: bool = True) -> int:
    """streambp_gemm_epilogue: C = act(A W^T + bias) + residual, the sum before act in `pre` if given.  A [M, K],
    W [N, K], the others [M, N]; rows contiguous, any leading dimension; residual may be C_out."""
    what, dev, dt = "gemm_epilogue", A.get_device(), A.dtype
    _want(A.is_cuda and A.dim() == 2 and W.dim() == 2, what, "A and W are CUDA matrices")
    (M, K), N = A.shape, W.shape[0]
    a, w = _rows(what, dev, dt, (M, K), A), _rows(what, dev, dt, (N, K), W)
    c, r, z = (_rows(what, dev, dt, (M, N), t) for t in (C_out, residual, pre))
    if bias is not None and (bias.get_device() != dev or bias.dtype != dt or tuple(bias.shape) != (N,) or not bias.is_contiguous()):
        raise ValueError(f"{what}: bias is a contiguous {dt} vector of {N} on cuda:{dev}")
    st = _launch(what, dev, stream, lib().streambp_gemm_epilogue, a[0], a[1], w[0], w[1], M, N, K,
                 None if bias is None else bias.data_ptr(), ACTIVATIONS[activation], r[0], r[1], c[0], c[1], z[0], z[1],
                 _dtype_code(dt))
    if check:
        _check(st, "streambp_gemm_epilogue")
    return st


def gemm_epilogue_workspace_bytes(M: int, N: int) -> int:
    return int(lib().streambp_gemm_epilogue_workspace_bytes(M, N))


def gemm_epilogue_backward(dC, pre, activation: str, dZ=None, dbias=None, workspace=None, accumulate: bool = False,
                           stream=None, check: bool = True) -> int:
    """streambp_gemm_epilogue_backward: dZ = dC act'(pre), dbias (fp32 [N]) = or += column sums of dZ."""
    what, dev, dt = "gemm_epilogue_backward", dC.get_device(), dC.dtype
    _want(dC.is_cuda and dC.dim() == 2, what, "dC is a CUDA matrix")
    M, N = dC.shape
    d, z, g = (_rows(what, dev, dt, (M, N), t) for t in (dC, pre, dZ))
    if dbias is not None and (dbias.get_device() != dev or dbias.dtype != torch.float32 or tuple(dbias.shape) != (N,) or
                              not dbias.is_contiguous()):
        raise ValueError(f"{what}: dbias is a contiguous fp32 vector of {N} on cuda:{dev}")
    if workspace is not None and (workspace.get_device() != dev or not workspace.is_contiguous()):
        raise ValueError(f"{what}: workspace is contiguous, on cuda:{dev}")
    st = _launch(what, dev, stream, lib().streambp_gemm_epilogue_backward, d[0], d[1], z[0], z[1], ACTIVATIONS[activation], M, N,
                 g[0], g[1], None if dbias is None else dbias.data_ptr(), 1 if accumulate else 0, _dtype_code(dt),
                 None if workspace is None else workspace.data_ptr(),
                 0 if workspace is None else workspace.numel() * workspace.element_size())
    if check:
        _check(st, "streambp_gemm_epilogue_backward")
    return st


KERNEL_CLASSES = {"gemm": 0, "attention_fwd": 1, "attention_bwd": 2}


def test_expire_wait(limit_ns: int, stream=None) -> int:
    """Test hook: one tiny kernel whose bounded wait runs out after `limit_ns` (see streambp.h)."""
    return lib().streambp_test_expire_wait(int(limit_ns), _stream_ptr(stream))


test_expire_wait.__test__ = False     # a library call, not a pytest test


def product_kernel() -> str:
    """Which tcgen05 product kernel runs bf16 products on the current device."""
    return {2: "cta_pair", 1: "single_cta", 0: "none"}[lib().streambp_product_kernel()]


def profile_enable(on: bool) -> None:
    lib().streambp_profile_enable(1 if on else 0)


def profile_read(kernel_class: str):
    """(milliseconds, launches, algorithmic FLOPs) recorded for one kernel class."""
    ms, n, fl = C.c_double(), C.c_int64(), C.c_double()
    _check(lib().streambp_profile_read(KERNEL_CLASSES[kernel_class], C.byref(ms), C.byref(n), C.byref(fl)),
           "streambp_profile_read")
    return ms.value, n.value, fl.value


def attention_forward(q, k, v, q0: int, o, lse, engine: int = 0, stream=None, check: bool = True) -> int:
    """streambp_attention_forward; q, o: [n, Hq, dh], k, v: [q0+n, Hkv, dh], lse: [Hq, n] fp32."""
    n, Hq, dh = q.shape
    st = lib().streambp_attention_forward(_ptr(q), _ptr(k), _ptr(v), n, q0, Hq, k.shape[1], dh, _dtype_code(q.dtype),
                                          _ptr(o), _ptr(lse), engine, _stream_ptr(stream))
    if check:
        _check(st, "streambp_attention_forward")
    return st


def attention_backward(q, k, v, o, d_o, lse, q0: int, dq, dk, dv, engine: int = 0, stream=None,
                       check: bool = True) -> int:
    """streambp_attention_backward; dq fp32 overwritten, dk / dv fp32 accumulated."""
    n, Hq, dh = q.shape
    delta = torch.empty(Hq, n, dtype=torch.float32, device=q.device)
    st = lib().streambp_attention_backward(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse), n, q0, Hq,
                                           k.shape[1], dh, _dtype_code(q.dtype), _ptr(delta), _ptr(dq), _ptr(dk),
                                           _ptr(dv), engine, _stream_ptr(stream))
    if check:
        _check(st, "streambp_attention_backward")
    return st


STATIC_DELTA_MAX_FLOATS = 1 << 20


def attention_backward_static(q, k, v, o, d_o, lse, q0: int, dq, dk, dv, engine: int = 0, stream=None,
                              check: bool = True) -> int:
    """streambp_attention_backward_static: like attention_backward, but the row-sum scratch is the
    library's fixed 4 MiB array, so neither this wrapper nor the library allocates device memory.
    For callers that cannot allocate at call time.  Requires n * Hq <= STATIC_DELTA_MAX_FLOATS;
    calls that overlap on the GPU race on the shared array."""
    n, Hq, dh = q.shape
    st = lib().streambp_attention_backward_static(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse), n, q0, Hq,
                                                  k.shape[1], dh, _dtype_code(q.dtype), _ptr(dq), _ptr(dk), _ptr(dv),
                                                  engine, _stream_ptr(stream))
    if check:
        _check(st, "streambp_attention_backward_static")
    return st


def _window_args(what: str, q, k, v, q0: int) -> tuple:
    """Sizes of a windowed call: q [n, Hq, dh], k and v [q0 + n, Hkv, dh]."""
    if q.dim() != 3 or k.dim() != 3 or q0 < 0:
        raise ValueError(f"{what}: q is [n, Hq, dh], k and v are [q0 + n, Hkv, dh], q0 >= 0")
    shape, (n, Hq, dh), kv = q.shape, q.shape, k.shape
    if kv[0] != q0 + n or kv[2] != dh or v.shape != kv:
        raise ValueError(f"{what}: k and v are [{q0 + n}, Hkv, {dh}], got {tuple(kv)} and {tuple(v.shape)}")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError(f"{what}: q, k and v share a type")
    return n, Hq, kv[1], dh, shape, kv


def attention_window_forward(q, k, v, q0: int, window: int, sinks: int, o, lse, engine: int = 0, stream=None,
                             check: bool = True) -> int:
    """streambp_attention_window_forward; q, o: [n, Hq, dh], k, v: [q0+n, Hkv, dh], lse: [Hq, n] fp32."""
    what = "attention_window_forward"
    n, Hq, Hkv, dh, shape, _ = _window_args(what, q, k, v, q0)
    if o.shape != shape or o.dtype != q.dtype or lse.shape != (Hq, n) or lse.dtype != torch.float32:
        raise ValueError(f"{what}: o is like q, lse is fp32 [{Hq}, {n}]")
    dev = q.get_device()
    _same(what, dev, q, k, v, o, lse)
    st = _launch(what, dev, stream, lib().streambp_attention_window_forward, q.data_ptr(), k.data_ptr(), v.data_ptr(), n, q0, Hq,
                 Hkv, dh, _dtype_code(q.dtype), window, sinks, o.data_ptr(), lse.data_ptr(), engine)
    if check:
        _check(st, "streambp_attention_window_forward")
    return st


def attention_window_workspace_bytes(n: int, q0: int, n_q_heads: int, n_kv_heads: int, head_dim: int, window: int,
                                     sinks: int) -> int:
    return int(lib().streambp_attention_window_workspace_bytes(n, q0, n_q_heads, n_kv_heads, head_dim, window, sinks))


def attention_window_backward(q, k, v, o, d_o, lse, q0: int, window: int, sinks: int, dq, dk, dv, workspace,
                              accumulate: bool = False, engine: int = 0, stream=None, check: bool = True) -> int:
    """streambp_attention_window_backward; dq, dk, dv share a type (fp32, or bf16 for bf16 storage): overwritten, or with
    accumulate=True (fp32) dk and dv are added to."""
    what = "attention_window_backward"
    n, Hq, Hkv, dh, shape, kv = _window_args(what, q, k, v, q0)
    if (o.shape != shape or d_o.shape != shape or o.dtype != q.dtype or d_o.dtype != q.dtype or lse.shape != (Hq, n) or
            lse.dtype != torch.float32):
        raise ValueError(f"{what}: o and d_o are like q, lse is fp32 [{Hq}, {n}]")
    grad = dq.dtype
    if dq.shape != shape or dk.shape != kv or dv.shape != kv or dk.dtype != grad or dv.dtype != grad:
        raise ValueError(f"{what}: dq, dk and dv have the shapes of q, k and v and share a type")
    dev = q.get_device()
    _same(what, dev, q, k, v, o, d_o, lse, dq, dk, dv, workspace)
    st = _launch(what, dev, stream, lib().streambp_attention_window_backward, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                 o.data_ptr(), d_o.data_ptr(), lse.data_ptr(), n, q0, Hq, Hkv, dh, _dtype_code(q.dtype), window, sinks,
                 _dtype_code(grad), 1 if accumulate else 0, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(),
                 workspace.numel() * workspace.element_size(), engine)
    if check:
        _check(st, "streambp_attention_window_backward")
    return st


OBJ_GRPO, OBJ_DPO = 1, 2


def lmhead_rl_backward(cfg: HeadConfig, objective: int, beta: float, clip_eps: float, g_final, w_vocab, H, tokens,
                       logp_old, logp_ref, advantage, weight, chunk: int, loss, dH, d_w_vocab, d_g_final, workspace,
                       logp=None, ell=None, accumulate: bool = False, stream=None, check: bool = True,
                       wgrad_group: int = 1) -> int:
    """streambp_lmhead_rl_backward (GRPO / DPO objectives of the streamed LM head); wgrad_group != 1 goes through
    streambp_lmhead_rl_backward_grouped."""
    c = cfg.c()
    rl = RlCfgC(objective, beta, clip_eps)
    head = (C.byref(c), C.byref(rl), _ptr(g_final), _ptr(w_vocab), _ptr(H), _ptr(tokens), _ptr(logp_old),
            _ptr(logp_ref), _ptr(advantage), _ptr(weight), H.shape[0], chunk)
    tail = (1 if accumulate else 0, _ptr(loss), _ptr(logp), _ptr(ell), _ptr(dH), _ptr(d_w_vocab), _ptr(d_g_final),
            _ptr(workspace), workspace.numel(), _stream_ptr(stream))
    if wgrad_group == 1:
        name, st = "streambp_lmhead_rl_backward", lib().streambp_lmhead_rl_backward(*head, *tail)
    else:
        name = "streambp_lmhead_rl_backward_grouped"
        st = lib().streambp_lmhead_rl_backward_grouped(*head, wgrad_group, *tail)
    if check:
        _check(st, name)
    return st


# ---- AdamW ------------------------------------------------------------------------------------------------------
MX8_BLOCK = 32
STATE_F32, STATE_MX8 = 0, 1


class AdamWPlan:
    """The tensors of an AdamW step, checked once and laid out for the calls (host memory only; the tensors are kept
    alive).  Each entry is a dict: param (fp32 or bf16), grad (fp32), m, v, optional master (fp32, bf16 parameters
    only), optional weight_decay (0).  m and v are fp32, or uint8 codes with m_scale and v_scale (uint8, one per 32
    elements).  All entries share the parameter's and the moments' types and one device; tensors that a step writes
    must not overlap one another or a gradient."""

    def __init__(self, tensors: Sequence[Dict]):
        what = "AdamWPlan"
        _want(len(tensors) > 0, what, "needs at least one tensor")
        self.tensors = [dict(t) for t in tensors]
        p0, m0 = self.tensors[0]["param"], self.tensors[0]["m"]
        _same(what, p0.get_device(), p0)
        self.device = p0.device
        self.param_dtype, index, f32 = _dtype_code(p0.dtype), p0.get_device(), torch.float32
        _want(m0.dtype in (f32, torch.uint8), what, "m is fp32 or uint8 codes")
        mx8 = m0.dtype == torch.uint8
        self.state_dtype = STATE_MX8 if mx8 else STATE_F32
        n, size_p, size_m = len(self.tensors), p0.element_size(), m0.element_size()
        self.c = (AdamWTensorC * n)()
        self.grads, self.counts = (C.c_void_p * n)(), (C.c_int64 * n)()
        written = []
        for i, t in enumerate(self.tensors):
            p, g, m, v, ma, ms, vs = (t.get(k) for k in ("param", "grad", "m", "v", "master", "m_scale", "v_scale"))
            count, c = p.numel(), self.c[i]
            for x in (p, g, m, v) if ma is None else (p, g, m, v, ma):
                if x.get_device() != index or not x.is_contiguous() or x.numel() != count:
                    raise ValueError(f"{what}: tensors of an entry are contiguous, of one size and on one CUDA device")
            if p.dtype != p0.dtype or m.dtype != m0.dtype or v.dtype != m0.dtype or g.dtype != f32:
                raise ValueError(f"{what}: grad is fp32; parameters share a type, moments share a type")
            if ma is not None:
                _want(p.dtype == torch.bfloat16 and ma.dtype == f32, what, "master is fp32 and goes with bf16 parameters")
                c.master = a = ma.data_ptr()
                written.append((a, a + 4 * count))
            if mx8:
                blocks = (count + MX8_BLOCK - 1) // MX8_BLOCK
                for x in (ms, vs):
                    if x is None or x.dtype != torch.uint8 or x.numel() != blocks or x.get_device() != index or not x.is_contiguous():
                        raise ValueError(f"{what}: m_scale and v_scale are contiguous uint8, one per 32 elements")
                c.m_scale, c.v_scale = ms.data_ptr(), vs.data_ptr()
                written += [(c.m_scale or 0, (c.m_scale or 0) + blocks), (c.v_scale or 0, (c.v_scale or 0) + blocks)]
            elif ms is not None or vs is not None:
                raise ValueError(f"{what}: scales go with 8-bit moments")
            c.param, c.m, c.v, c.count = pa, ma_, va, _ = p.data_ptr(), m.data_ptr(), v.data_ptr(), count
            c.weight_decay = t.get("weight_decay", 0.0)
            c.grad = self.grads[i] = g.data_ptr()
            self.counts[i] = count
            written += [(pa, pa + size_p * count), (ma_, ma_ + size_m * count), (va, va + size_m * count)]
        written = sorted(x for x in written if x[0] < x[1])
        _want(all(x[1] <= y[0] for x, y in zip(written, written[1:])), what, "tensors that a step writes overlap")
        starts = [x[0] for x in written]
        for a, count in zip(self.grads, self.counts):                 # the written tensor that starts last before a gradient's end
            at = bisect_left(starts, a + 4 * count) - 1 if count else -1
            _want(at < 0 or written[at][1] <= a, what, "a gradient overlaps a tensor that the step writes")

    def __len__(self) -> int:
        return len(self.tensors)


def adamw_step(plan: AdamWPlan, lr: float, beta1: float, beta2: float, eps: float, step, grad_scale=None, stream=None,
               check: bool = True) -> int:
    """streambp_adamw_step.  step: an int >= 1, or an int64 CUDA tensor of one value that the kernel reads;
    grad_scale: None or an fp32 CUDA tensor of one value (see grad_norm)."""
    on_device = isinstance(step, torch.Tensor)
    if on_device:
        _want(step.dtype == torch.int64 and step.numel() == 1 and step.device == plan.device, "adamw_step",
              "step is an int or one int64 on the tensors' device")
    if grad_scale is not None:
        _want(grad_scale.dtype == torch.float32 and grad_scale.numel() == 1 and grad_scale.device == plan.device,
              "adamw_step", "grad_scale is one fp32 value on the tensors' device")
    c = AdamWCfgC(lr, beta1, beta2, eps, plan.param_dtype, plan.state_dtype, 0 if on_device else int(step))
    st = _launch("adamw_step", plan.device.index, stream, lib().streambp_adamw_step, C.byref(c), plan.c, len(plan),
                 None if grad_scale is None else grad_scale.data_ptr(), step.data_ptr() if on_device else None)
    if check:
        _check(st, "streambp_adamw_step")
    return st


def grad_norm_workspace_bytes() -> int:
    return int(lib().streambp_grad_norm_workspace_bytes())


def grad_norm(plan: AdamWPlan, max_norm: float, norm: torch.Tensor, scale: Optional[torch.Tensor],
              workspace: torch.Tensor, stream=None, check: bool = True) -> int:
    """streambp_grad_norm over the gradients of a plan: norm and scale (or None) are fp32 CUDA tensors of one value."""
    for t in (norm, scale):
        _want(t is None or (t.dtype == torch.float32 and t.numel() == 1), "grad_norm", "norm and scale are one fp32 value each")
    _same("grad_norm", plan.device.index, *((norm, workspace) if scale is None else (norm, workspace, scale)))
    st = _launch("grad_norm", plan.device.index, stream, lib().streambp_grad_norm, plan.grads, plan.counts, len(plan), max_norm,
                 norm.data_ptr(), None if scale is None else scale.data_ptr(), workspace.data_ptr(),
                 workspace.numel() * workspace.element_size())
    if check:
        _check(st, "streambp_grad_norm")
    return st


def mx8_encode(values: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, keep_nonzero: bool = False, stream=None,
               check: bool = True) -> int:
    """streambp_mx8_encode: fp32 values -> uint8 codes and one scale byte per 32 of them."""
    n = values.numel()
    _want(values.dtype == torch.float32 and codes.dtype == torch.uint8 and scales.dtype == torch.uint8 and
          codes.numel() == n and scales.numel() == (n + MX8_BLOCK - 1) // MX8_BLOCK, "mx8_encode",
          "fp32 values, uint8 codes of the same size, one uint8 scale per 32")
    _same("mx8_encode", values.get_device(), values, codes, scales)
    st = _launch("mx8_encode", values.get_device(), stream, lib().streambp_mx8_encode, values.data_ptr(), n,
                 1 if keep_nonzero else 0, codes.data_ptr(), scales.data_ptr())
    if check:
        _check(st, "streambp_mx8_encode")
    return st


def mx8_decode(codes: torch.Tensor, scales: torch.Tensor, out: torch.Tensor, stream=None, check: bool = True) -> int:
    """streambp_mx8_decode: the values (fp32 or bf16) that the codes stand for."""
    n = codes.numel()
    _want(codes.dtype == torch.uint8 and scales.dtype == torch.uint8 and out.numel() == n and
          scales.numel() == (n + MX8_BLOCK - 1) // MX8_BLOCK, "mx8_decode",
          "uint8 codes, one uint8 scale per 32, as many values out")
    _same("mx8_decode", codes.get_device(), codes, scales, out)
    st = _launch("mx8_decode", codes.get_device(), stream, lib().streambp_mx8_decode, codes.data_ptr(), scales.data_ptr(), n,
                 out.data_ptr(), _dtype_code(out.dtype))
    if check:
        _check(st, "streambp_mx8_decode")
    return st


# ---- the ends of a model ------------------------------------------------------------------------------------------
TOP_MAX = 128
DISTILL_MAX_VOCAB = 1 << 22


def _vectors(what: str, dev: int, shape: tuple, **tensors) -> list:
    """Addresses of optional contiguous tensors of one shape: name=(tensor, dtype)."""
    out = []
    for name, (t, dtype) in tensors.items():
        if t is None:
            out.append(None)
        elif t.get_device() == dev and t.dtype == dtype and t.shape == shape and t.is_contiguous():
            out.append(t.data_ptr())
        else:
            raise ValueError(f"{what}: {name} is a contiguous {dtype} tensor {shape} on cuda:{dev}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return out


def _space(what: str, dev: int, workspace: Optional[torch.Tensor]) -> tuple:
    """(address, bytes) of a workspace, (None, 0) for None."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"{what}: workspace is contiguous, on cuda:{dev}")
    return workspace.data_ptr(), workspace.nbytes


def _matrix(what: str, name: str, t: torch.Tensor) -> int:
    """The device of a CUDA matrix."""
    _want(t.is_cuda and t.dim() == 2, what, f"{name} is a CUDA matrix")
    return t.get_device()


def token_logprobs_workspace_bytes() -> int:
    return int(lib().streambp_token_logprobs_workspace_bytes())


def _score_outputs(what: str, dev: int, n: int, tokens, logp, lse, entropy, top_logp, top_ids) -> tuple:
    f, i = torch.float32, torch.int64
    rows = _vectors(what, dev, (n,), tokens=(tokens, i), logp=(logp, f), lse=(lse, f), entropy=(entropy, f))
    lists = top_logp if top_logp is not None else top_ids
    if lists is None:
        return rows, 0, (None, None)
    _want(lists.dim() == 2, what, "top_logp and top_ids are [rows, k]")
    k = lists.shape[1]
    return rows, k, _vectors(what, dev, (n, k), top_logp=(top_logp, f), top_ids=(top_ids, i))


def token_logprobs(logits, tokens, workspace, logp=None, lse=None, entropy=None, top_logp=None, top_ids=None,
                   temperature: float = 1.0, ignore_index: int = -100, stream=None, check: bool = True) -> int:
    """streambp_token_logprobs; logits [rows, vocab] fp32 or bf16 with contiguous rows, tokens int64 [rows] or None, logp, lse,
    entropy fp32 [rows], top_logp fp32 and top_ids int64 [rows, k]; outputs that are None are not formed."""
    what, dev = "token_logprobs", _matrix("token_logprobs", "logits", logits)
    n, V = logits.shape
    z = _rows(what, dev, logits.dtype, (n, V), logits)
    rows, k, lists = _score_outputs(what, dev, n, tokens, logp, lse, entropy, top_logp, top_ids)
    st = _launch(what, dev, stream, lib().streambp_token_logprobs, z[0], z[1], n, V, _dtype_code(logits.dtype), rows[0], ignore_index,
                 temperature, k, *rows[1:], *lists, *_space(what, dev, workspace))
    if check:
        _check(st, "streambp_token_logprobs")
    return st


def token_logprobs_backward(logits, tokens, lse, entropy, d_logits, d_logp=None, d_lse=None, d_entropy=None,
                            temperature: float = 1.0, ignore_index: int = -100, stream=None, check: bool = True) -> int:
    """streambp_token_logprobs_backward; lse and entropy (None without d_entropy) of the forward call, d_logits like logits
    (or logits itself)."""
    what, dev = "token_logprobs_backward", _matrix("token_logprobs_backward", "logits", logits)
    n, V = logits.shape
    z = _rows(what, dev, logits.dtype, (n, V), logits)
    d = z if d_logits is logits else _rows(what, dev, logits.dtype, (n, V), d_logits)
    f = torch.float32
    v = _vectors(what, dev, (n,), tokens=(tokens, torch.int64), lse=(lse, f), entropy=(entropy, f), d_logp=(d_logp, f), d_lse=(d_lse, f),
                 d_entropy=(d_entropy, f))
    st = _launch(what, dev, stream, lib().streambp_token_logprobs_backward, z[0], z[1], n, V, _dtype_code(logits.dtype), v[0],
                 ignore_index, temperature, *v[1:], d[0], d[1])
    if check:
        _check(st, "streambp_token_logprobs_backward")
    return st


def distill_topk_workspace_bytes() -> int:
    return int(lib().streambp_distill_topk_workspace_bytes())


def _entries(what: str, dev: int, n: int, ids, values) -> tuple:
    _want(ids.dim() == 2, what, "ids and values are [rows, k]")
    k = ids.shape[1]
    return k, _vectors(what, dev, (n, k), ids=(ids, torch.int64), values=(values, torch.float32))


def distill_topk(logits, ids, values, row_loss, workspace, d_logits=None, weight=None, temperature: float = 1.0,
                 tail: bool = False, stream=None, check: bool = True) -> int:
    """streambp_distill_topk; logits [rows, vocab] fp32 or bf16 with contiguous rows, ids int64 and values fp32 [rows, k], weight
    and row_loss fp32 [rows] (optional), d_logits like logits (or logits itself, or None)."""
    what, dev = "distill_topk", _matrix("distill_topk", "logits", logits)
    n, V = logits.shape
    z = _rows(what, dev, logits.dtype, (n, V), logits)
    d = z if d_logits is logits else _rows(what, dev, logits.dtype, (n, V), d_logits)
    k, entries = _entries(what, dev, n, ids, values)
    w = _vectors(what, dev, (n,), weight=(weight, torch.float32), row_loss=(row_loss, torch.float32))
    cfg = DistillCfgC(k, 1 if tail else 0, temperature)
    st = _launch(what, dev, stream, lib().streambp_distill_topk, C.byref(cfg), z[0], z[1], n, V, _dtype_code(logits.dtype), *entries, *w,
                 d[0], d[1], *_space(what, dev, workspace))
    if check:
        _check(st, "streambp_distill_topk")
    return st


def _head_args(what: str, cfg: HeadConfig, g_final, w_vocab, H) -> int:
    """Checks what a head reads and returns the device."""
    dev = _matrix(what, "H", H)
    d, V = cfg.d_model, cfg.vocab
    for name, t, shape in (("H", H, (H.shape[0], d)), ("g_final", g_final, (d,)), ("w_vocab", w_vocab, (V, d))):
        if t.get_device() != dev or t.dtype != cfg.dtype or tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError(f"{what}: {name} is a contiguous {cfg.dtype} tensor {shape} on cuda:{dev}")
    return dev


def lmhead_logprobs_workspace_bytes(cfg: HeadConfig, T: int, chunk: int) -> int:
    c = cfg.c()
    return int(lib().streambp_lmhead_logprobs_workspace_bytes(C.byref(c), T, chunk))


def lmhead_logprobs(cfg: HeadConfig, g_final, w_vocab, H, tokens, chunk: int, workspace, logp=None, lse=None, entropy=None,
                    top_logp=None, top_ids=None, temperature: float = 1.0, stream=None, check: bool = True) -> int:
    """streambp_lmhead_logprobs: token_logprobs of the head's logits, which exist for one chunk of H [T, d_model] at a time."""
    what = "lmhead_logprobs"
    dev = _head_args(what, cfg, g_final, w_vocab, H)
    T = H.shape[0]
    rows, k, lists = _score_outputs(what, dev, T, tokens, logp, lse, entropy, top_logp, top_ids)
    c = cfg.c()
    st = _launch(what, dev, stream, lib().streambp_lmhead_logprobs, C.byref(c), g_final.data_ptr(), w_vocab.data_ptr(), H.data_ptr(),
                 rows[0], T, chunk, temperature, k, *rows[1:], *lists, *_space(what, dev, workspace))
    if check:
        _check(st, "streambp_lmhead_logprobs")
    return st


def lmhead_distill_workspace_bytes(cfg: HeadConfig, T: int, chunk: int, wgrad_group: int = 1) -> int:
    c = cfg.c()
    return int(lib().streambp_lmhead_distill_workspace_bytes(C.byref(c), T, chunk, wgrad_group))


def lmhead_distill_backward(cfg: HeadConfig, g_final, w_vocab, H, ids, values, weight, chunk: int, loss, dH, d_w_vocab, d_g_final,
                            workspace, row_loss=None, temperature: float = 1.0, tail: bool = False, accumulate: bool = False,
                            stream=None, check: bool = True, wgrad_group: int = 1) -> int:
    """streambp_lmhead_distill_backward: the streamed head under distill_topk's loss; weight fp32 [T]."""
    what = "lmhead_distill_backward"
    dev = _head_args(what, cfg, g_final, w_vocab, H)
    T, d, V = H.shape[0], cfg.d_model, cfg.vocab
    k, entries = _entries(what, dev, T, ids, values)
    f = torch.float32
    w = _vectors(what, dev, (T,), weight=(weight, f), row_loss=(row_loss, f))
    for name, t, dtype, shape in (("loss", loss, f, (1,)), ("dH", dH, cfg.dtype, (T, d)), ("d_w_vocab", d_w_vocab, f, (V, d)),
                                  ("d_g_final", d_g_final, f, (d,))):
        _vectors(what, dev, shape, **{name: (t, dtype)})
    c, dc = cfg.c(), DistillCfgC(k, 1 if tail else 0, temperature)
    st = _launch(what, dev, stream, lib().streambp_lmhead_distill_backward, C.byref(c), C.byref(dc), g_final.data_ptr(), w_vocab.data_ptr(),
                 H.data_ptr(), *entries, w[0], T, chunk, wgrad_group, 1 if accumulate else 0, loss.data_ptr(), w[1], dH.data_ptr(),
                 d_w_vocab.data_ptr(), d_g_final.data_ptr(), *_space(what, dev, workspace))
    if check:
        _check(st, "streambp_lmhead_distill_backward")
    return st


def layernorm_forward(x, gain, bias, eps: float, y, mean=None, rstd=None, stream=None, check: bool = True) -> int:
    """streambp_layernorm_forward; x, y [rows, d] with contiguous rows (y may be x), gain and bias [d] of the same type or None,
    mean and rstd fp32 [rows] or None."""
    what, dev, dt = "layernorm_forward", _matrix("layernorm_forward", "x", x), x.dtype
    n, d = x.shape
    a, o = (_rows(what, dev, dt, (n, d), t) for t in (x, y))
    g = _vectors(what, dev, (d,), gain=(gain, dt), bias=(bias, dt))
    s = _vectors(what, dev, (n,), mean=(mean, torch.float32), rstd=(rstd, torch.float32))
    st = _launch(what, dev, stream, lib().streambp_layernorm_forward, a[0], a[1], *g, eps, n, d, _dtype_code(dt), o[0], o[1], *s)
    if check:
        _check(st, "streambp_layernorm_forward")
    return st


def layernorm_workspace_bytes(rows: int, d: int) -> int:
    return int(lib().streambp_layernorm_workspace_bytes(rows, d))


def layernorm_backward(dy, x, gain, mean, rstd, dx=None, d_gain=None, d_bias=None, add=None, workspace=None,
                       accumulate: bool = False, stream=None, check: bool = True) -> int:
    """streambp_layernorm_backward; dy, x, add, dx [rows, d], d_gain and d_bias fp32 [d] (overwritten, or added to)."""
    what, dev, dt = "layernorm_backward", _matrix("layernorm_backward", "x", x), x.dtype
    n, d = x.shape
    nd = (n, d)
    g, a, r, o = _rows(what, dev, dt, nd, dy), _rows(what, dev, dt, nd, x), _rows(what, dev, dt, nd, add), _rows(what, dev, dt, nd, dx)
    w = _vectors(what, dev, (d,), gain=(gain, dt), d_gain=(d_gain, torch.float32), d_bias=(d_bias, torch.float32))
    s = _vectors(what, dev, (n,), mean=(mean, torch.float32), rstd=(rstd, torch.float32))
    st = _launch(what, dev, stream, lib().streambp_layernorm_backward, g[0], g[1], a[0], a[1], w[0], *s, r[0], r[1], n, d,
                 _dtype_code(dt), o[0], o[1], w[1], w[2], 1 if accumulate else 0, *_space(what, dev, workspace))
    if check:
        _check(st, "streambp_layernorm_backward")
    return st


def embedding_workspace_bytes() -> int:
    return int(lib().streambp_embedding_workspace_bytes())


def embedding_forward(table, ids, out, workspace, scale: float = 1.0, padding_id: int = -1, stream=None, check: bool = True) -> int:
    """streambp_embedding_forward; table [vocab, d], ids int64 [n], out [n, d] of the table's type, rows contiguous."""
    what, dev, dt = "embedding_forward", _matrix("embedding_forward", "table", table), table.dtype
    (V, d), n = table.shape, ids.numel()
    t, o = _rows(what, dev, dt, (V, d), table), _rows(what, dev, dt, (n, d), out)
    i = _vectors(what, dev, (n,), ids=(ids, torch.int64))
    st = _launch(what, dev, stream, lib().streambp_embedding_forward, t[0], t[1], i[0], n, V, d, _dtype_code(dt), scale, padding_id, o[0],
                 o[1], *_space(what, dev, workspace))
    if check:
        _check(st, "streambp_embedding_forward")
    return st


def embedding_backward_workspace_bytes(n: int, vocab: int, d: int) -> int:
    return int(lib().streambp_embedding_backward_workspace_bytes(n, vocab, d))


def embedding_backward(d_out, ids, d_table, workspace, scale: float = 1.0, padding_id: int = -1, accumulate: bool = False,
                       stream=None, check: bool = True) -> int:
    """streambp_embedding_backward; d_out [n, d] with contiguous rows, d_table contiguous fp32 [vocab, d] on 16 bytes
    (overwritten, or added to)."""
    what, dev, dt = "embedding_backward", _matrix("embedding_backward", "d_out", d_out), d_out.dtype
    n, d = d_out.shape
    _want(d_table.dim() == 2 and d_table.shape[1] == d, what, "d_table is [vocab, d]")
    V = d_table.shape[0]
    g = _rows(what, dev, dt, (n, d), d_out)
    i = _vectors(what, dev, (n,), ids=(ids, torch.int64)) + _vectors(what, dev, (V, d), d_table=(d_table, torch.float32))
    st = _launch(what, dev, stream, lib().streambp_embedding_backward, g[0], g[1], i[0], n, V, d, _dtype_code(dt), scale, padding_id,
                 1 if accumulate else 0, i[1], *_space(what, dev, workspace))
    if check:
        _check(st, "streambp_embedding_backward")
    return st
