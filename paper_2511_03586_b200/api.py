"""Thin ctypes binding of ``libpd.so``: argument marshalling only.

Every function mirrors one entry point of ``include/pd.h`` under the same name,
takes CUDA ``torch.Tensor`` arguments (torch supplies device memory and the
stream, nothing else), and raises :class:`PdError` on a non-zero status.  There
is no fallback: if the library is missing or cannot be loaded, importing this
module fails.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libpd.so")

PD_OK = 0
PD_BF16, PD_F32 = 0, 1

EXPORTS = (
    "pd_status_string", "pd_last_cuda_error", "pd_get_device_status", "pd_clear_device_status",
    "pd_softmax", "pd_layernorm", "pd_rmsnorm", "pd_bias_gelu_residual", "pd_gemm_bf16", "pd_set_gemm_tile_mode", "pd_attention_fwd",
    "pd_encoder_layer_workspace_bytes", "pd_encoder_layer_workspace_layout", "pd_encoder_layer_fwd", "pd_encoder_layer_stage_count",
    "pd_encoder_layer_stage_name", "pd_encoder_layer_fwd_profiled", "pd_encoder_layer_static_scratch_bytes",
    "pd_encoder_layer_fwd_static", "pd_kv_cache_append", "pd_attention_paged_workspace_bytes",
    "pd_attention_paged_fwd", "pd_norm_gate_residual_norm", "pd_sample",
)


class PdError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        name = _lib.pd_status_string(status).decode()
        extra = f" (cudaError {_lib.pd_last_cuda_error()})" if name == "PD_ERR_CUDA" else ""
        super().__init__(f"{where}: {name}{extra}")


class EncoderLayerDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("seq", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("ffn", ctypes.c_int32), ("ln_eps", ctypes.c_float)]


class EncoderLayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "w_qkv", "w_o", "w_ffn1", "w_ffn2", "b_qkv", "b_o", "b_ffn1", "b_ffn2",
        "ln1_gamma", "ln1_beta", "ln2_gamma", "ln2_beta")]


class PagedAttentionDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "tokens", "heads_q", "heads_kv", "head_dim", "num_pages", "page_size", "max_pages", "max_q_len",
        "max_kv_len", "window", "sinks")] + [("scale", ctypes.c_float)] + [(n, ctypes.c_int64) for n in (
            "ld_q", "ld_out", "page_stride", "slot_stride", "head_stride")]


class NormGateResidualDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "cols", "gate_rows")] + [
        (n, ctypes.c_int32) for n in ("x_dtype", "y_dtype", "post_norm", "pre_norm")] + [
            (n, ctypes.c_float) for n in ("alpha", "eps")]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2511_03586_b200.build` (needs nvcc)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, st = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    lib.pd_status_string.argtypes = [st]; lib.pd_status_string.restype = ctypes.c_char_p
    lib.pd_last_cuda_error.argtypes = []; lib.pd_last_cuda_error.restype = ctypes.c_int
    lib.pd_get_device_status.argtypes = [ctypes.POINTER(ctypes.c_int)]; lib.pd_get_device_status.restype = st
    lib.pd_clear_device_status.argtypes = []; lib.pd_clear_device_status.restype = st
    lib.pd_debug_set_wait_limit_ns.argtypes = [ctypes.c_uint64]; lib.pd_debug_set_wait_limit_ns.restype = st
    lib.pd_debug_withhold_loads.argtypes = [ctypes.c_int]; lib.pd_debug_withhold_loads.restype = st
    lib.pd_softmax.argtypes = [vp, vp, i64, i64, vp]; lib.pd_softmax.restype = st
    lib.pd_layernorm.argtypes = [vp, vp, vp, vp, i64, i64, ctypes.c_float, vp]; lib.pd_layernorm.restype = st
    lib.pd_rmsnorm.argtypes = [vp, vp, vp, i64, i64, ctypes.c_float, vp]; lib.pd_rmsnorm.restype = st
    lib.pd_reducemean.argtypes = [vp, vp, i64, i64, vp]; lib.pd_reducemean.restype = st
    lib.pd_bias_gelu_residual.argtypes = [vp, vp, vp, vp, i64, i64, vp]; lib.pd_bias_gelu_residual.restype = st
    lib.pd_gemm_bf16.argtypes = [vp, vp, vp, i64, i64, i64, i64, i64, i64, ctypes.c_int, ctypes.c_int,
                                 i64, i64, i64, i64, vp]
    lib.pd_gemm_bf16.restype = st
    lib.pd_set_gemm_tile_mode.argtypes = [ctypes.c_int]; lib.pd_set_gemm_tile_mode.restype = st
    lib.pd_gemm_bias_act.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ctypes.c_int, ctypes.c_int, vp]
    lib.pd_gemm_bias_act.restype = st
    lib.pd_swiglu_gemm.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp]; lib.pd_swiglu_gemm.restype = st
    lib.pd_set_gemm_split_k.argtypes = [ctypes.c_int]; lib.pd_set_gemm_split_k.restype = st
    lib.pd_set_layernorm_fusion.argtypes = [ctypes.c_int]; lib.pd_set_layernorm_fusion.restype = st
    lib.pd_gemm_bias_residual_layernorm.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, ctypes.c_float, vp]
    lib.pd_gemm_bias_residual_layernorm.restype = st
    lib.pd_attention_fwd.argtypes = [vp, vp, i64, i64, i64, vp]; lib.pd_attention_fwd.restype = st
    lib.pd_encoder_layer_workspace_bytes.argtypes = [ctypes.POINTER(EncoderLayerDesc)]
    lib.pd_encoder_layer_workspace_bytes.restype = ctypes.c_size_t
    lib.pd_encoder_layer_workspace_layout.argtypes = [ctypes.POINTER(EncoderLayerDesc),
                                                      ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t)]
    lib.pd_encoder_layer_workspace_layout.restype = st
    lib.pd_encoder_layer_fwd.argtypes = [ctypes.POINTER(EncoderLayerDesc), ctypes.POINTER(EncoderLayerWeights),
                                         vp, vp, vp, ctypes.c_size_t, vp]
    lib.pd_encoder_layer_fwd.restype = st
    lib.pd_encoder_stack_workspace_bytes.argtypes = [ctypes.POINTER(EncoderLayerDesc), ctypes.c_int]
    lib.pd_encoder_stack_workspace_bytes.restype = ctypes.c_size_t
    lib.pd_encoder_stack_fwd.argtypes = [ctypes.POINTER(EncoderLayerDesc), ctypes.POINTER(EncoderLayerWeights),
                                         ctypes.c_int, vp, vp, vp, ctypes.c_size_t, vp]
    lib.pd_encoder_stack_fwd.restype = st
    lib.pd_encoder_layer_static_scratch_bytes.argtypes = []
    lib.pd_encoder_layer_static_scratch_bytes.restype = ctypes.c_size_t
    lib.pd_encoder_layer_fwd_static.argtypes = [ctypes.POINTER(EncoderLayerDesc), ctypes.POINTER(EncoderLayerWeights),
                                                vp, vp, vp]
    lib.pd_encoder_layer_fwd_static.restype = st
    lib.pd_encoder_layer_kernel_count.argtypes = [ctypes.POINTER(EncoderLayerDesc)]
    lib.pd_encoder_layer_kernel_count.restype = ctypes.c_int
    lib.pd_encoder_layer_stage_count.argtypes = []; lib.pd_encoder_layer_stage_count.restype = ctypes.c_int
    lib.pd_encoder_layer_stage_name.argtypes = [ctypes.c_int]
    lib.pd_encoder_layer_stage_name.restype = ctypes.c_char_p
    lib.pd_encoder_layer_fwd_profiled.argtypes = lib.pd_encoder_layer_fwd.argtypes + [ctypes.POINTER(ctypes.c_float)]
    lib.pd_encoder_layer_fwd_profiled.restype = st
    # (the descs as plain addresses: the bindings below hand over packed bytes)
    lib.pd_kv_cache_append.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, vp, vp]; lib.pd_kv_cache_append.restype = st
    lib.pd_attention_paged_workspace_bytes.argtypes = [vp]
    lib.pd_attention_paged_workspace_bytes.restype = ctypes.c_size_t
    lib.pd_attention_paged_fwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.pd_attention_paged_fwd.restype = st
    lib.pd_norm_gate_residual_norm.argtypes = [vp] * 11
    lib.pd_norm_gate_residual_norm.restype = st
    lib.pd_sample.argtypes = [vp, ctypes.c_int, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.pd_sample.restype = st
    return lib


_lib = _load()


def _check(status: int, where: str):
    if status != PD_OK:
        raise PdError(status, where)


def _stream(stream) -> int:
    return (stream if stream is not None else torch.cuda.current_stream()).cuda_stream


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def pd_softmax(x: torch.Tensor, y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    rows, cols = x.shape
    if y is None:
        y = torch.empty_like(x)
    _check(_lib.pd_softmax(_dev(x, torch.float32, "x"), _dev(y, torch.float32, "y"), rows, cols, _stream(stream)),
           "pd_softmax")
    return y


def pd_layernorm(x, gamma, beta, eps: float, y=None, stream=None) -> torch.Tensor:
    rows, cols = x.shape
    if y is None:
        y = torch.empty_like(x)
    _check(_lib.pd_layernorm(_dev(x, torch.float32, "x"), _dev(gamma, torch.float32, "gamma"),
                             _dev(beta, torch.float32, "beta"), _dev(y, torch.float32, "y"), rows, cols,
                             float(eps), _stream(stream)), "pd_layernorm")
    return y


def pd_rmsnorm(x, gamma, eps: float, y=None, stream=None) -> torch.Tensor:
    rows, cols = x.shape
    if y is None:
        y = torch.empty_like(x)
    _check(_lib.pd_rmsnorm(_dev(x, torch.float32, "x"), _dev(gamma, torch.float32, "gamma"),
                           _dev(y, torch.float32, "y"), rows, cols, float(eps), _stream(stream)), "pd_rmsnorm")
    return y


def pd_reducemean(x, y=None, stream=None) -> torch.Tensor:
    rows, cols = x.shape
    if y is None:
        y = torch.empty(rows, dtype=torch.float32, device=x.device)
    _check(_lib.pd_reducemean(_dev(x, torch.float32, "x"), _dev(y, torch.float32, "y"), rows, cols, _stream(stream)),
           "pd_reducemean")
    return y


def pd_bias_gelu_residual(x, bias, r=None, out=None, stream=None) -> torch.Tensor:
    rows, cols = x.shape
    if out is None:
        out = torch.empty_like(x)
    rp = None if r is None else _dev(r, torch.float32, "r")
    _check(_lib.pd_bias_gelu_residual(_dev(x, torch.float32, "x"), _dev(bias, torch.float32, "bias"), rp,
                                      _dev(out, torch.float32, "out"), rows, cols, _stream(stream)),
           "pd_bias_gelu_residual")
    return out


def pd_gemm_bf16(a: torch.Tensor, b: torch.Tensor, c: torch.Tensor | None = None, *, b_is_nk: bool = False,
                 c_dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """C = A @ B for bf16 A [M,K] (or [batch,M,K]) and B [K,N] (or [N,K] when
    ``b_is_nk``; batched likewise).  Inputs must be dense."""
    batched = a.dim() == 3
    if batched:
        batch, M, K = a.shape
    else:
        (M, K), batch = a.shape, 1
    N = b.shape[-2] if b_is_nk else b.shape[-1]
    if c is None:
        c = torch.empty(((batch, M, N) if batched else (M, N)), dtype=c_dtype, device=a.device)
    ldb = b.shape[-1]
    _check(_lib.pd_gemm_bf16(_dev(a, torch.bfloat16, "a"), _dev(b, torch.bfloat16, "b"), _dev(c, c.dtype, "c"),
                             M, N, K, K, ldb, N, int(b_is_nk), PD_F32 if c.dtype == torch.float32 else PD_BF16,
                             batch, M * K, b.shape[-2] * b.shape[-1], M * N, _stream(stream)), "pd_gemm_bf16")
    return c


def pd_set_gemm_tile_mode(mode: int) -> None:
    """0: automatic; 1: single-CTA tiles only; 2: CTA-pair (cta_group::2) tiles for every shape."""
    _check(_lib.pd_set_gemm_tile_mode(int(mode)), "pd_set_gemm_tile_mode")


def pd_gemm_bf16_raw(a_ptr, b_ptr, c_ptr, M, N, K, lda, ldb, ldc, b_is_nk, c_dtype, batch, strideA, strideB,
                     strideC, stream=None) -> int:
    """Direct call with explicit pointers and strides; returns the status instead of raising."""
    return _lib.pd_gemm_bf16(a_ptr, b_ptr, c_ptr, M, N, K, lda, ldb, ldc, int(b_is_nk), int(c_dtype), batch,
                             strideA, strideB, strideC, _stream(stream))


ACT_NONE, ACT_GELU, ACT_RELU = 0, 1, 2


def pd_gemm_bias_act(a, b, bias=None, residual=None, *, act: int = ACT_NONE, c_dtype=torch.bfloat16, c=None,
                     stream=None) -> torch.Tensor:
    """C = act(A @ B + bias) + residual for bf16 A [M,K], B [K,N], residual [M,N]; fp32 bias [N]."""
    M, K = a.shape
    N = b.shape[1]
    if c is None:
        c = torch.empty(M, N, dtype=c_dtype, device=a.device)
    _check(_lib.pd_gemm_bias_act(_dev(a, torch.bfloat16, "a"), _dev(b, torch.bfloat16, "b"),
                                 None if bias is None else _dev(bias, torch.float32, "bias"),
                                 None if residual is None else _dev(residual, torch.bfloat16, "residual"),
                                 _dev(c, c.dtype, "c"), M, N, K, int(act),
                                 PD_F32 if c.dtype == torch.float32 else PD_BF16, _stream(stream)), "pd_gemm_bias_act")
    return c


def pd_swiglu_gemm(x, wg, wu, y=None, stream=None) -> torch.Tensor:
    """Y = SiLU(X @ Wg) * (X @ Wu) for bf16 X [M,K], Wg, Wu [K,N]; bf16 Y."""
    M, K = x.shape
    N = wg.shape[1]
    if y is None:
        y = torch.empty(M, N, dtype=torch.bfloat16, device=x.device)
    _check(_lib.pd_swiglu_gemm(_dev(x, torch.bfloat16, "x"), _dev(wg, torch.bfloat16, "wg"),
                               _dev(wu, torch.bfloat16, "wu"), _dev(y, torch.bfloat16, "y"), M, N, K,
                               _stream(stream)), "pd_swiglu_gemm")
    return y


def pd_set_gemm_split_k(mode: int) -> None:
    """0: split K over a thread-block cluster when a contraction has few output tiles; 1: never."""
    _check(_lib.pd_set_gemm_split_k(int(mode)), "pd_set_gemm_split_k")


def pd_set_layernorm_fusion(mode: int) -> None:
    """0: LayerNorm inside the feeding contraction's epilogue where the shape allows; 1: separate row kernel."""
    _check(_lib.pd_set_layernorm_fusion(int(mode)), "pd_set_layernorm_fusion")


def pd_gemm_bias_residual_layernorm(a, b, bias, residual, gamma, beta, eps: float, y=None, stream=None) -> torch.Tensor:
    """Y = LayerNorm(A @ B + bias + residual) for bf16 A [M,K], B [K,N], residual [M,N] (or None),
    fp32 bias (or None), gamma, beta [N]; bf16 Y."""
    M, K = a.shape
    N = b.shape[1]
    if y is None:
        y = torch.empty(M, N, dtype=torch.bfloat16, device=a.device)
    _check(_lib.pd_gemm_bias_residual_layernorm(
        _dev(a, torch.bfloat16, "a"), _dev(b, torch.bfloat16, "b"),
        None if bias is None else _dev(bias, torch.float32, "bias"),
        None if residual is None else _dev(residual, torch.bfloat16, "residual"),
        _dev(gamma, torch.float32, "gamma"), _dev(beta, torch.float32, "beta"), _dev(y, torch.bfloat16, "y"),
        M, N, K, float(eps), _stream(stream)), "pd_gemm_bias_residual_layernorm")
    return y


def pd_attention_fwd(qkv: torch.Tensor, *, batch: int, seq: int, heads: int, ctx: torch.Tensor | None = None,
                     stream=None) -> torch.Tensor:
    """qkv bf16 [batch*seq, 3*heads*64] -> ctx bf16 [batch*seq, heads*64]."""
    if tuple(qkv.shape) != (batch * seq, 3 * heads * 64):
        raise ValueError("qkv must be [batch*seq, 3*heads*64]")
    if ctx is None:
        ctx = torch.empty(batch * seq, heads * 64, dtype=torch.bfloat16, device=qkv.device)
    _check(_lib.pd_attention_fwd(_dev(qkv, torch.bfloat16, "qkv"), _dev(ctx, torch.bfloat16, "ctx"), batch, seq,
                                 heads, _stream(stream)), "pd_attention_fwd")
    return ctx


@dataclass
class EncoderLayerParams:
    """Device tensors of one layer (bf16 matrices [in, out], fp32 vectors)."""
    w_qkv: torch.Tensor
    w_o: torch.Tensor
    w_ffn1: torch.Tensor
    w_ffn2: torch.Tensor
    b_qkv: torch.Tensor
    b_o: torch.Tensor
    b_ffn1: torch.Tensor
    b_ffn2: torch.Tensor
    ln1_gamma: torch.Tensor
    ln1_beta: torch.Tensor
    ln2_gamma: torch.Tensor
    ln2_beta: torch.Tensor

    def as_struct(self) -> EncoderLayerWeights:
        s = EncoderLayerWeights()
        for name in ("w_qkv", "w_o", "w_ffn1", "w_ffn2"):
            setattr(s, name, _dev(getattr(self, name), torch.bfloat16, name))
        for name in ("b_qkv", "b_o", "b_ffn1", "b_ffn2", "ln1_gamma", "ln1_beta", "ln2_gamma", "ln2_beta"):
            setattr(s, name, _dev(getattr(self, name), torch.float32, name))
        return s


def pd_encoder_layer_workspace_bytes(batch: int, seq: int, hidden: int, heads: int, ffn: int,
                                     ln_eps: float = 1e-5) -> int:
    d = EncoderLayerDesc(batch, seq, hidden, heads, ffn, ln_eps)
    return int(_lib.pd_encoder_layer_workspace_bytes(ctypes.byref(d)))


LAYER_BUFFERS = ("qkv", "scores", "probs", "ctx", "pre", "h1", "mid")


def pd_encoder_layer_workspace_layout(batch: int, seq: int, hidden: int, heads: int, ffn: int,
                                      ln_eps: float = 1e-5) -> dict:
    """{buffer name: (byte offset, byte size)} of the layer's intermediates inside its workspace."""
    d = EncoderLayerDesc(batch, seq, hidden, heads, ffn, ln_eps)
    n = len(LAYER_BUFFERS)
    off, size = (ctypes.c_size_t * n)(), (ctypes.c_size_t * n)()
    _check(_lib.pd_encoder_layer_workspace_layout(ctypes.byref(d), off, size), "pd_encoder_layer_workspace_layout")
    return {name: (int(off[i]), int(size[i])) for i, name in enumerate(LAYER_BUFFERS)}


def pd_encoder_layer_fwd(params: EncoderLayerParams, x: torch.Tensor, *, batch: int, seq: int, heads: int,
                         ln_eps: float = 1e-5, y: torch.Tensor | None = None,
                         workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    T, hidden = x.shape
    if T != batch * seq:
        raise ValueError("x must be [batch*seq, hidden]")
    ffn = params.w_ffn1.shape[1]
    d = EncoderLayerDesc(batch, seq, hidden, heads, ffn, ln_eps)
    if y is None:
        y = torch.empty_like(x)
    if workspace is None:
        nbytes = int(_lib.pd_encoder_layer_workspace_bytes(ctypes.byref(d)))
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=x.device)
    w = params.as_struct()
    _check(_lib.pd_encoder_layer_fwd(ctypes.byref(d), ctypes.byref(w), _dev(x, torch.bfloat16, "x"),
                                     _dev(y, torch.bfloat16, "y"), workspace.data_ptr(), workspace.numel(),
                                     _stream(stream)), "pd_encoder_layer_fwd")
    return y


def pd_encoder_stack_fwd(layers, x: torch.Tensor, *, batch: int, seq: int, heads: int, ln_eps: float = 1e-5,
                         y: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """Runs ``layers`` (a list of EncoderLayerParams of one shape) one after the other on x [batch*seq, hidden]."""
    T, hidden = x.shape
    if T != batch * seq:
        raise ValueError("x must be [batch*seq, hidden]")
    d = EncoderLayerDesc(batch, seq, hidden, heads, layers[0].w_ffn1.shape[1], ln_eps)
    if y is None:
        y = torch.empty_like(x)
    if workspace is None:
        nbytes = int(_lib.pd_encoder_stack_workspace_bytes(ctypes.byref(d), len(layers)))
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=x.device)
    w = (EncoderLayerWeights * len(layers))(*[p.as_struct() for p in layers])
    _check(_lib.pd_encoder_stack_fwd(ctypes.byref(d), w, len(layers), _dev(x, torch.bfloat16, "x"),
                                     _dev(y, torch.bfloat16, "y"), workspace.data_ptr(), workspace.numel(),
                                     _stream(stream)), "pd_encoder_stack_fwd")
    return y


def pd_encoder_layer_static_scratch_bytes() -> int:
    return int(_lib.pd_encoder_layer_static_scratch_bytes())


def pd_encoder_layer_fwd_static(params: EncoderLayerParams, x: torch.Tensor, y: torch.Tensor, *, batch: int,
                                seq: int, heads: int, ln_eps: float = 1e-5, stream=None) -> torch.Tensor:
    """The layer for callers that cannot allocate: intermediates live in the
    library's fixed 32 MiB device array, and the caller passes the output tensor
    too, so neither this binding nor the library allocates anything."""
    T, hidden = x.shape
    if T != batch * seq:
        raise ValueError("x must be [batch*seq, hidden]")
    d = EncoderLayerDesc(batch, seq, hidden, heads, params.w_ffn1.shape[1], ln_eps)
    w = params.as_struct()
    _check(_lib.pd_encoder_layer_fwd_static(ctypes.byref(d), ctypes.byref(w), _dev(x, torch.bfloat16, "x"),
                                            _dev(y, torch.bfloat16, "y"), _stream(stream)),
           "pd_encoder_layer_fwd_static")
    return y


def pd_encoder_layer_kernel_count(batch: int, seq: int, hidden: int, heads: int, ffn: int) -> int:
    d = EncoderLayerDesc(batch, seq, hidden, heads, ffn, 1e-5)
    return int(_lib.pd_encoder_layer_kernel_count(ctypes.byref(d)))


def pd_encoder_layer_stage_names() -> list[str]:
    return [_lib.pd_encoder_layer_stage_name(i).decode() for i in range(_lib.pd_encoder_layer_stage_count())]


def pd_encoder_layer_fwd_profiled(params: EncoderLayerParams, x: torch.Tensor, *, batch: int, seq: int, heads: int,
                                  ln_eps: float = 1e-5, y: torch.Tensor | None = None,
                                  workspace: torch.Tensor | None = None, stream=None):
    """Runs the layer with per-stage CUDA events; returns (y, {stage name: ms})."""
    T, hidden = x.shape
    if T != batch * seq:
        raise ValueError("x must be [batch*seq, hidden]")
    d = EncoderLayerDesc(batch, seq, hidden, heads, params.w_ffn1.shape[1], ln_eps)
    if y is None:
        y = torch.empty_like(x)
    if workspace is None:
        nbytes = int(_lib.pd_encoder_layer_workspace_bytes(ctypes.byref(d)))
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=x.device)
    w = params.as_struct()
    n = _lib.pd_encoder_layer_stage_count()
    ms = (ctypes.c_float * n)()
    _check(_lib.pd_encoder_layer_fwd_profiled(ctypes.byref(d), ctypes.byref(w), _dev(x, torch.bfloat16, "x"),
                                              _dev(y, torch.bfloat16, "y"), workspace.data_ptr(),
                                              workspace.numel(), _stream(stream), ms), "pd_encoder_layer_fwd_profiled")
    return y, dict(zip(pd_encoder_layer_stage_names(), [float(v) for v in ms]))


def pd_get_device_status() -> int:
    code = ctypes.c_int(0)
    st = _lib.pd_get_device_status(ctypes.byref(code))
    if st not in (PD_OK, 7):
        raise PdError(st, "pd_get_device_status")
    return code.value


def pd_clear_device_status() -> None:
    _check(_lib.pd_clear_device_status(), "pd_clear_device_status")


def pd_debug_set_wait_limit_ns(limit_ns: int) -> None:
    """Time after which a wait inside the contraction, paged attention and row-prefetching norm kernels gives up (default 2 s)."""
    _check(_lib.pd_debug_set_wait_limit_ns(int(limit_ns)), "pd_debug_set_wait_limit_ns")


def pd_debug_withhold_loads(on: bool) -> None:
    """Test switch: the producers of the same kernels issue no load, so a bounded wait runs out."""
    _check(_lib.pd_debug_withhold_loads(int(bool(on))), "pd_debug_withhold_loads")


# ---- a paged key/value cache and the operators of a decoder that reads it ----------------------------------------
# These bindings run on the device of their first tensor, whichever is current, and on that device's current stream
# unless one is given; every tensor has to live there.  A decode step calls them with little work each, so the checks
# are kept to attribute reads: device indices instead of device objects, raw stream handles, no context manager unless
# the device has to be switched, descriptors packed in one go (the host side of a call went from 19-32 us to 9-16).

def _device(t, name: str) -> int:
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError(f"{name} must be a CUDA tensor")
    return t.get_device()


def _on(device: int, t, dtype, name: str, dense: bool = True) -> int | None:
    """Address of ``t`` (None for None) after checking its device, type and, unless told otherwise, density."""
    if t is None:
        return None
    try:
        if t.get_device() == device and t.dtype is dtype and (not dense or t.is_contiguous()):
            return t.data_ptr()
    except AttributeError:
        pass
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        raise TypeError(f"{name} must be a tensor on cuda:{device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    raise ValueError(f"{name} must be contiguous")


def _call(fn, device: int, stream, *args) -> None:
    """fn(*args, stream) with ``device`` current."""
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(device)
    elif stream.device_index != device:
        raise ValueError(f"stream must belong to cuda:{device}")
    else:
        handle = stream.cuda_stream
    if torch._C._cuda_getDevice() == device:
        status = fn(*args, handle)
    else:
        with torch.cuda.device(device):
            status = fn(*args, handle)
    if status != PD_OK:
        raise PdError(status, fn.__name__)


def _new(like, stream, n: int | None = None, dtype=None) -> torch.Tensor:
    """A dense tensor for a call on ``stream``: like ``like``, or of ``n`` elements of ``dtype``.  From that stream's memory,
    since what the current stream has freed it may still be writing.  The caller may use it on the current stream, which is
    recorded, so that the memory is not handed out again before both are through with it.  (A shape handed over as a tuple
    costs 0.7 us more.)"""
    if stream is None:
        return torch.empty_like(like, memory_format=_DENSE) if n is None else like.new_empty(n, dtype=dtype)
    with torch.cuda.stream(stream):
        t = _new(like, None, n, dtype)
    t.record_stream(torch.cuda.current_stream(like.device))
    return t


_DENSE = torch.contiguous_format
_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32

# The descs' fields, packed as C lays them out (half the time of filling a structure, and values beyond a field's 32 bits
# raise instead of losing their upper half).
_PAGED_DESC, _NORM_DESC = struct.Struct("@12if5q"), struct.Struct("@3q4i2f")
assert _PAGED_DESC.size == ctypes.sizeof(PagedAttentionDesc) and _NORM_DESC.size == ctypes.sizeof(NormGateResidualDesc)


def _pack(layout: struct.Struct, *values) -> bytes:
    try:
        return layout.pack(*values)
    except (struct.error, OverflowError) as e:
        raise ValueError(f"an argument does not fit its field: {e}") from None


def _token_stride(t: torch.Tensor, name: str) -> int:
    """Elements from token to token of [tokens, heads, head_dim] whose heads lie side by side."""
    if t.dim() != 3:
        raise ValueError(f"{name} must be [tokens, heads, head_dim]")
    tokens, heads, d = t.shape
    token_stride, head_stride, stride = t.stride()
    if (d > 1 and stride != 1) or (heads > 1 and head_stride != d):
        raise ValueError(f"{name}: the heads of a token must lie side by side")
    return token_stride if tokens > 1 else heads * d


def _paged_cache(device: int, k_cache, v_cache, block_table, cu_q, kv_len):
    """The cache's extents (as the desc has them), its strides, and the addresses of the five tensors."""
    kc, vc = _on(device, k_cache, _BF16, "k_cache", False), _on(device, v_cache, _BF16, "v_cache", False)
    table, cu, lens = _on(device, block_table, _I32, "block_table"), _on(device, cu_q, _I32, "cu_q"), _on(device, kv_len, _I32, "kv_len")
    shape, strides, other = k_cache.shape, k_cache.stride(), v_cache.stride()
    if len(shape) != 4 or v_cache.shape != shape:
        raise ValueError("k_cache and v_cache must be [pages, page_size, heads, head_dim] with the same strides")
    num_pages, page_size, heads, head_dim = shape
    if strides != other and any(n > 1 and a != b for n, a, b in zip(shape, strides, other)):
        raise ValueError("k_cache and v_cache must be [pages, page_size, heads, head_dim] with the same strides")
    if head_dim > 1 and strides[3] != 1:
        raise ValueError("the elements of a cached head must be contiguous")
    if block_table.dim() != 2 or cu_q.dim() != 1 or kv_len.dim() != 1:
        raise ValueError("block_table must be [batch, max_pages], cu_q [batch + 1], kv_len [batch]")
    batch, max_pages = block_table.shape
    if kv_len.numel() != batch or cu_q.numel() != batch + 1:
        raise ValueError("block_table must be [batch, max_pages], cu_q [batch + 1], kv_len [batch]")
    # strides of extents of one are never used; the library still asks for legal ones
    strides = (strides[0] if num_pages > 1 else page_size * heads * head_dim,
               strides[1] if page_size > 1 else heads * head_dim, strides[2] if heads > 1 else head_dim)
    return (batch, heads, head_dim, num_pages, page_size, max_pages), strides, (kc, vc, table, cu, lens)


def pd_kv_cache_append(k_new, v_new, k_cache, v_cache, block_table, cu_q, kv_len, stream=None) -> None:
    """Writes the new tokens' keys and values (bf16 [tokens, heads_kv, head_dim], column blocks of a packed projection
    will do) to their slots of the caches (bf16 [pages, page_size, heads_kv, head_dim], any page, slot and head
    strides).  ``kv_len`` counts the new tokens already."""
    device = _device(k_new, "k_new")
    (batch, heads, head_dim, *pages), strides, (kc, vc, table, cu, lens) = _paged_cache(
        device, k_cache, v_cache, block_table, cu_q, kv_len)
    k, v = _on(device, k_new, _BF16, "k_new", False), _on(device, v_new, _BF16, "v_new", False)
    ld = _token_stride(k_new, "k_new")
    tokens, new_heads, d = k_new.shape
    if new_heads != heads or d != head_dim or v_new.shape != k_new.shape:
        raise ValueError("k_new and v_new must be [tokens, heads_kv, head_dim]")
    if v_new.stride() != k_new.stride() and ld != _token_stride(v_new, "v_new"):
        raise ValueError("k_new and v_new must have the same token stride")
    desc = _pack(_PAGED_DESC, batch, tokens, 0, heads, head_dim, *pages, 0, 0, 0, 0, 0.0, 0, 0, *strides)
    _call(_lib.pd_kv_cache_append, device, stream, desc, k, v, ld, kc, vc, table, cu, lens)


def pd_attention_paged_workspace_bytes(desc: PagedAttentionDesc) -> int:
    return int(_lib.pd_attention_paged_workspace_bytes(ctypes.byref(desc)))


def pd_attention_paged_fwd(q, k_cache, v_cache, block_table, cu_q, kv_len, *, max_q_len: int, max_kv_len: int,
                           window: int = 0, sinks: int = 0, scale: float | None = None, out=None, workspace=None,
                           stream=None) -> torch.Tensor:
    """Causal attention of the packed new tokens q (bf16 [tokens, heads_q, head_dim]) over the paged caches, which hold
    their keys and values already; ``window`` > 0 limits a query to that many last keys, plus the first ``sinks``.
    ``scale`` defaults to head_dim ** -0.5.  Rows of q behind the last sequence are left as they are in ``out``."""
    device = _device(q, "q")
    (batch, heads_kv, head_dim, *pages), strides, (kc, vc, table, cu, lens) = _paged_cache(
        device, k_cache, v_cache, block_table, cu_q, kv_len)
    qp, ld_q = _on(device, q, _BF16, "q", False), _token_stride(q, "q")
    tokens, heads_q, d = q.shape
    if d != head_dim:
        raise ValueError("q and the caches must have the same head_dim")
    if out is None:
        out = _new(q, stream)
        op, ld_out = out.data_ptr(), heads_q * head_dim
    else:
        op, ld_out = _on(device, out, torch.bfloat16, "out", False), _token_stride(out, "out")
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    desc = _pack(_PAGED_DESC, batch, tokens, heads_q, heads_kv, head_dim, *pages, max_q_len, max_kv_len, window, sinks,
                 head_dim ** -0.5 if scale is None else scale, ld_q, ld_out, *strides)
    if workspace is None:
        ws_bytes = _lib.pd_attention_paged_workspace_bytes(desc)
        workspace = _new(q, stream, ws_bytes, torch.uint8) if ws_bytes else None
        ws = workspace.data_ptr() if ws_bytes else None
    else:
        ws, ws_bytes = _on(device, workspace, torch.uint8, "workspace"), workspace.numel()
    _call(_lib.pd_attention_paged_fwd, device, stream, desc, qp, kc, vc, table, cu, lens, op, ws, ws_bytes)
    return out


_NORMS = {"none": 0, "rms": 1, "layer": 2}
_PD_DTYPES = {torch.bfloat16: PD_BF16, torch.float32: PD_F32}


def _vector(device: int, t, cols: int, name: str) -> int | None:
    if t is None:
        return None
    ptr = _on(device, t, _F32, name)
    if t.numel() != cols:
        raise ValueError(f"{name} must have {cols} elements")
    return ptr


def _float_type(t, name: str) -> int:
    code = _PD_DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be torch.bfloat16 or torch.float32, got {t.dtype}")
    return code


def pd_norm_gate_residual_norm(y, x, *, gate=None, gate_rows: int | None = None, alpha: float = 1.0, eps: float = 1e-5,
                               post_norm: str = "rms", post_gamma=None, post_beta=None, pre_norm: str = "rms",
                               pre_gamma=None, pre_beta=None, h=None, n=None, stream=None):
    """h = alpha * x + gate * post_norm(y), n = pre_norm(h); returns (h, n).

    y, n: bf16 or fp32 [rows, cols] (the block's output, the next block's input); x, h: bf16 or fp32 (the residual
    stream).  Norms: "none", "rms", "layer"; gamma and beta fp32 [cols] or None.  gate: y's type, [groups, cols] (or
    [cols]), one row for every ``gate_rows`` rows (default: rows / groups rounded up)."""
    device = _device(y, "y")
    if post_norm not in _NORMS or pre_norm not in _NORMS:
        raise ValueError(f"norms must be among {tuple(_NORMS)}")
    if not isinstance(x, torch.Tensor):
        raise TypeError("x must be a tensor")
    y_code, x_code = _float_type(y, "y"), _float_type(x, "x")
    yp, xp = _on(device, y, y.dtype, "y"), _on(device, x, x.dtype, "x")
    if y.dim() != 2 or x.shape != y.shape:
        raise ValueError("y and x must be [rows, cols]")
    rows, cols = y.shape
    vectors = (_vector(device, post_gamma, cols, "post_gamma"), _vector(device, post_beta, cols, "post_beta"),
               _vector(device, pre_gamma, cols, "pre_gamma"), _vector(device, pre_beta, cols, "pre_beta"))
    gp = _on(device, gate, y.dtype, "gate")
    if gate is not None:
        if gate.dim() not in (1, 2) or gate.shape[-1] != cols:
            raise ValueError("gate must be [groups, cols] or [cols]")
        groups = gate.shape[0] if gate.dim() == 2 else 1
        if gate_rows is None:
            gate_rows = max(1, -(-rows // max(groups, 1)))
        if gate_rows < 1 or -(-rows // gate_rows) > groups:
            raise ValueError("gate has too few rows")
    if h is None:
        h = _new(x, stream)
        hp = h.data_ptr()
    elif h.shape != x.shape:
        raise ValueError("h must be [rows, cols]")
    else:
        hp = _on(device, h, x.dtype, "h")
    if n is None:
        n = _new(y, stream)
        np_ = n.data_ptr()
    elif n.shape != y.shape:
        raise ValueError("n must be [rows, cols]")
    else:
        np_ = _on(device, n, y.dtype, "n")
    d = _pack(_NORM_DESC, rows, cols, gate_rows or 1, x_code, y_code, _NORMS[post_norm], _NORMS[pre_norm], alpha, eps)
    _call(_lib.pd_norm_gate_residual_norm, device, stream, d, yp, xp, gp, *vectors, hp, np_)
    return h, n


def pd_sample(logits, u, *, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None, probs=None, stream=None):
    """Draws a token per row of logits (bf16 or fp32 [rows, vocab], rows of any stride) with the random numbers u
    (fp32 [rows] in [0, 1)); temperature, top_p, min_p: fp32 [rows], top_k: int32 [rows], None for no such filter.
    Returns (tokens int32 [rows], probs fp32 [rows])."""
    device = _device(logits, "logits")
    code, lp = _float_type(logits, "logits"), logits.data_ptr()
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [rows, vocab] with contiguous rows")
    rows, vocab = logits.shape
    if u is None:
        raise TypeError("u must be a tensor")
    if tokens is None:
        tokens = _new(logits, stream, rows, torch.int32)
    if probs is None:
        probs = _new(logits, stream, rows, torch.float32)
    ptrs = []
    for name, t, dtype in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32),
                           ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32), ("u", u, torch.float32),
                           ("tokens", tokens, torch.int32), ("probs", probs, torch.float32)):
        ptrs.append(_on(device, t, dtype, name))
        if t is not None and t.numel() != rows:
            raise ValueError(f"{name} must have one value per row")
    _call(_lib.pd_sample, device, stream, lp, code, rows, vocab, logits.stride(0) if rows > 1 else vocab, *ptrs)
    return tokens, probs
