"""MI355X (gfx950) fused BitLinear: Python binding of ``libmmf.so``.

The forward pass of the BitLinear layer of "Scalable MatMul-free Language
Modeling" (arXiv 2406.02528; Algorithm 1 with bias 0): RMSNorm, per-token
absmax int8 quantisation, ternary accumulation with int32 sums and
dequantisation.  Every step runs in the HIP kernels of ``libmmf.so``; this
module only checks tensor shapes, dtypes and devices and passes raw pointers
and the current HIP stream through the C ABI declared in ``include/mmf.h``.
PyTorch is used for device memory and streams only.

Also the GLU channel mixer's gated up-projection, the MLGRU token mixer
(input projections with gate activations, the recurrence, the whole mixer),
the training forward and backward of the layer, and what a block's training
step needs around it: the residual addition fused into the quantiser, the GLU
mixer's and the recurrence's training forms, and the global gradient norm with
clipping.  And linear attention with a decay per head (forward and backward), a
step of beam search (selection, reordering of states) and distillation from a
teacher's best tokens (loss and gradient).

Functions carry the names of the C entry points.  There is no fallback: if
the library is not built, importing this package raises ``ImportError``.
"""
from __future__ import annotations

import array
import ctypes
import itertools
import operator
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmmf.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'` "
        "(hipcc --offload-arch=gfx950); there is no CPU fallback")

_lib = ctypes.CDLL(LIB_PATH)

MMF_OK = 0
MMF_PATH_AUTO, MMF_PATH_GEMV, MMF_PATH_GEMM = 0, 1, 2

_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_SZ = ctypes.c_size_t

_SIGNATURES = {
    "mmf_status_string": ([ctypes.c_int], ctypes.c_char_p),
    "mmf_version": ([], ctypes.c_int),
    "mmf_packed_weight_bytes": ([_I64, _I64], _SZ),
    "mmf_ternarize_weights": ([_P, _I64, _I64, _P, _P, _P], ctypes.c_int),
    "mmf_act_quant": ([_P, _P, _P, _P, _I64, _I64, _P], ctypes.c_int),
    "mmf_act_quant_f32": ([_P, _P, _P, _P, _I64, _I64, _P], ctypes.c_int),
    "mmf_act_quant_ex": ([_P, ctypes.c_int, _P, _P, _P, _P, _I64, _I64, _P], ctypes.c_int),
    "mmf_add_act_quant": ([_P, ctypes.c_int, _P, ctypes.c_int, _P, _P, _P, _P, _P, _P, _I64, _I64, _P], ctypes.c_int),
    "mmf_add_act_quant_bwd_workspace_bytes": ([_I64, _I64], _SZ),
    "mmf_add_act_quant_bwd": ([_P, ctypes.c_int, _P, _P, ctypes.c_int, _P, _P, _P, _P, _P, _I64, _I64, _P, _SZ, _P],
                              ctypes.c_int),
    "mmf_bitlinear_fwd": ([_P, _P, _P, _P, _P, _I64, _I64, _I64, _P], ctypes.c_int),
    "mmf_bitlinear_fwd_f32": ([_P, _P, _P, _P, _P, _I64, _I64, _I64, _P], ctypes.c_int),
    "mmf_bitlinear_workspace_bytes": ([_I64, _I64], _SZ),
    "mmf_bitlinear_fwd_ws": ([_P, ctypes.c_int, _P, _P, _P, _P, _I64, _I64, _I64, _P, _SZ, _P],
                             ctypes.c_int),
    "mmf_bitlinear_noalloc_max_bytes": ([], _SZ),
    "mmf_bitlinear_fwd_noalloc": ([_P, ctypes.c_int, _P, _P, _P, _P, _I64, _I64, _I64, _P],
                                  ctypes.c_int),
    "mmf_ternary_gemm_dequant": ([_P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _P], ctypes.c_int),
    "mmf_ternary_gemm_i32": ([_P, _P, _P, _I64, _I64, _I64, _P], ctypes.c_int),
    "mmf_set_path": ([ctypes.c_int], ctypes.c_int),
    "mmf_prefill_tile_plan": ([ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_int],
                              ctypes.c_int),
    "mmf_glu_pack": ([_P, _P, _I64, _I64, _P, _P], ctypes.c_int),
    "mmf_glu_fwd": ([_P, _P, _P, _P, _P, _I64, _I64, _I64, _P], ctypes.c_int),
    "mmf_glu_fwd_f32": ([_P, _P, _P, _P, _P, _I64, _I64, _I64, _P], ctypes.c_int),
    "mmf_glu_fwd_ws": ([_P, ctypes.c_int, _P, _P, _P, _P, _I64, _I64, _I64, _P, _SZ, _P],
                       ctypes.c_int),
    "mmf_ternary_gemm_glu": ([_P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _P], ctypes.c_int),
    "mmf_bitlinear_fwd_bias": ([_P, ctypes.c_int, _P, _P, _P, _P, _P, _I64, _I64, _I64, _P],
                               ctypes.c_int),
    "mmf_mlgru_proj_workspace_bytes": ([_I64, _I64, _I64], _SZ),
    "mmf_mlgru_proj": ([_P, ctypes.c_int, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _P, _SZ, _P],
                       ctypes.c_int),
    "mmf_mlgru_proj_q": ([_P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _P], ctypes.c_int),
    "mmf_mlgru_scan_workspace_bytes": ([_I64, _I64, _I64], _SZ),
    "mmf_mlgru_scan": ([_P, _P, _P, _P, _I64, _I64, _I64, _P, _SZ, _P], ctypes.c_int),
    "mmf_mlgru_workspace_bytes": ([_I64, _I64, _I64], _SZ),
    "mmf_bitlinear_train_workspace_bytes": ([_I64, _I64, _I64], _SZ),
    "mmf_bitlinear_train_fwd": ([_P, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64,
                                 _I64, _P, _SZ, _P], ctypes.c_int),
    "mmf_bitlinear_bwd_workspace_bytes": ([_I64, _I64, _I64], _SZ),
    "mmf_bitlinear_bwd": ([_P, _P, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64,
                           _I64, _P, _SZ, _P], ctypes.c_int),
    "mmf_mlgru_train_states_bytes": ([_I64, _I64, _I64], _SZ),
    "mmf_mlgru_train_scan_workspace_bytes": ([_I64, _I64, _I64], _SZ),
    "mmf_mlgru_train_scan": ([_P, _P, _P, _P, _P, _P, _SZ, _I64, _I64, _I64, _P, _SZ, _P], ctypes.c_int),
    "mmf_mlgru_scan_bwd_workspace_bytes": ([_I64, _I64, _I64], _SZ),
    "mmf_mlgru_scan_bwd": ([_P, _P, _P, _SZ, _P, ctypes.c_int, _P, _P, _P, _P, _I64, _I64, _I64, _P, _SZ, _P],
                           ctypes.c_int),
    "mmf_glu_train_workspace_bytes": ([_I64, _I64, _I64], _SZ),
    "mmf_glu_train_fwd": ([_P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _P, _SZ, _P], ctypes.c_int),
    "mmf_glu_gate_bwd": ([_P, _P, _P, _P, _P, _P, ctypes.c_int, _P, _I64, _I64, _I64, _P], ctypes.c_int),
    "mmf_glu_bwd_workspace_bytes": ([_I64, _I64, _I64], _SZ),
    "mmf_glu_bwd": ([_P, ctypes.c_int, _P, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _P,
                     _SZ, _P], ctypes.c_int),
    "mmf_grad_norm_workspace_bytes": ([_P, _I64], _SZ),
    "mmf_grad_norm": ([_P, _P, _P, _I64, _P, _P, _SZ, _P], ctypes.c_int),
    "mmf_grad_clip": ([_P, _P, _P, _I64, _P, ctypes.c_float, _P, _P], ctypes.c_int),
    "mmf_linattn_workspace_bytes": ([_I64] * 5, _SZ),
    "mmf_linattn_fwd": ([_P, ctypes.c_int, _P, ctypes.c_float, _P, _P, _P, _I64, _I64, _I64, _I64, _I64, _P, _SZ, _P],
                        ctypes.c_int),
    "mmf_linattn_bwd_workspace_bytes": ([_I64] * 5, _SZ),
    "mmf_linattn_bwd": ([_P, ctypes.c_int, _P, ctypes.c_float, _P, _P, ctypes.c_int, _P, _P, _P, _I64, _I64, _I64, _I64,
                         _I64, _P, _SZ, _P], ctypes.c_int),
    "mmf_beam_select_workspace_bytes": ([_I64] * 4, _SZ),
    "mmf_beam_select": ([_P, ctypes.c_int, _P, _P, _I64, _P, _P, _P, _P, _I64, _I64, _I64, _I64, _P, _SZ, _P],
                        ctypes.c_int),
    "mmf_beam_reorder": ([_P, _P, _P, _I64, _P, _I64, _I64, _P], ctypes.c_int),
    "mmf_distill_fwd": ([_P, ctypes.c_int, _P, _P, ctypes.c_int, ctypes.c_float, _P, _I64, _I64, _I64, _P], ctypes.c_int),
    "mmf_distill_bwd": ([_P, ctypes.c_int, _P, _P, ctypes.c_int, ctypes.c_float, _P, _P, ctypes.c_int, _P, _I64, _I64,
                         _I64, _P], ctypes.c_int),
    "mmf_mlgru_fwd": ([_P, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                       _I64, _I64, _I64, _P, _SZ, _P], ctypes.c_int),
}
for _name, (_args, _res) in _SIGNATURES.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = _res


class MMFError(RuntimeError):
    pass


def _check(status: int) -> None:
    if status != MMF_OK:
        raise MMFError(_lib.mmf_status_string(status).decode())


# A call's checks and argument conversions are a large part of a small call (a
# one-token forward is one launch, 3.5 us from ctypes with plain integers), so
# they stay at attribute reads: torch.cuda.current_stream() alone builds a
# Stream object (3.0 us; the raw handle 0.3 us), a checked tensor went through
# str and tuple conversions (0.63 us; 0.3 us), and pointers are passed as
# integers.  The one-token forward took 12.4 us per call before, 7.2 us now.
def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


def _need(t: torch.Tensor, name: str, dtype, shape) -> None:
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.shape == shape and t.is_contiguous():
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on a HIP device")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


# The current device, asked once per call (0.13 us each), or one that no tensor
# is on where there is none.
def _here() -> int:
    try:
        return torch._C._cuda_getDevice()
    except RuntimeError:
        return -2


def _need_here(t: torch.Tensor, name: str, dtype, shape, here: int) -> None:
    """_need, and on the current device `here`: the call is enqueued there."""
    try:
        if t.dtype is dtype and t.get_device() == here and t.shape == shape and t.is_contiguous():
            return
    except AttributeError:  # not a tensor: the check below says so
        pass
    _need(t, name, dtype, shape)
    raise ValueError(f"{name} must be on the current device, cuda:{torch.cuda.current_device()}")


def _ws_here(workspace: torch.Tensor | None, here: int):
    if workspace is None:
        return None, 0
    n = workspace.numel()
    _need_here(workspace, "workspace", torch.uint8, (n,), here)
    return workspace.data_ptr(), n


def _stream_here(stream, here: int) -> int:
    return torch._C._cuda_getCurrentRawStream(here) if stream is None else _stream(stream)


def _x_kind(x: torch.Tensor) -> bool:
    """True for float32 activations, False for bfloat16."""
    if x.dtype == torch.float32:
        return True
    if x.dtype == torch.bfloat16:
        return False
    raise TypeError(f"x must be bfloat16 or float32, got {x.dtype}")


def _kind(t: torch.Tensor, name: str) -> bool:
    """_x_kind of a tensor with another name."""
    if t.dtype == torch.float32:
        return True
    if t.dtype == torch.bfloat16:
        return False
    raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")


def mmf_version() -> int:
    return int(_lib.mmf_version())


def mmf_status_string(status: int) -> str:
    return _lib.mmf_status_string(int(status)).decode()


def mmf_packed_weight_bytes(N: int, K: int) -> int:
    return int(_lib.mmf_packed_weight_bytes(N, K))


def mmf_set_path(path: int) -> int:
    prev = int(_lib.mmf_set_path(int(path)))
    if prev < 0:
        raise ValueError(f"unknown path {path}")
    return prev


MMF_EPILOGUE_DEQUANT, MMF_EPILOGUE_RAW_I32, MMF_EPILOGUE_GLU, MMF_EPILOGUE_AFFINE = 0, 1, 2, 3
TILE_PLANS = ("128x512", "128x256_paired", "64x512", "64x256", "256x256")


def mmf_prefill_tile_plan(M: int, K: int, N: int, epilogue: int = MMF_EPILOGUE_DEQUANT, cus: int = 256) -> str:
    """The prefill contraction's tile plan for M x K x N on `cus` compute
    units (host only), as a name from TILE_PLANS."""
    r = int(_lib.mmf_prefill_tile_plan(M, K, N, epilogue, cus))
    _check(-r if r < 0 else 0)
    return TILE_PLANS[r]


def mmf_ternarize_weights(W: torch.Tensor, Wpacked: torch.Tensor, w_scale: torch.Tensor,
                          stream=None) -> None:
    """W float32 [N][K] -> Wpacked int32 [K/16][N] (uint32 bit patterns), w_scale float32 [1]."""
    N, K = W.shape
    _need(W, "W", torch.float32, (N, K))
    _need(Wpacked, "Wpacked", torch.int32, (K // 16, N))
    _need(w_scale, "w_scale", torch.float32, (1,))
    _check(_lib.mmf_ternarize_weights(_ptr(W), N, K, _ptr(Wpacked), _ptr(w_scale), _stream(stream)))


def mmf_act_quant(x: torch.Tensor, gamma: torch.Tensor | None, q: torch.Tensor,
                  a_scale: torch.Tensor, q_rowsum: torch.Tensor | None = None,
                  stream=None) -> None:
    """x bf16/f32 [M][K], gamma f32 [K] or None -> q int8 [M][K], a_scale f32 [M], q_rowsum i32 [M]."""
    M, K = x.shape
    is_f32 = _x_kind(x)
    _need(x, "x", x.dtype, (M, K))
    if gamma is not None:
        _need(gamma, "gamma", torch.float32, (K,))
    _need(q, "q", torch.int8, (M, K))
    _need(a_scale, "a_scale", torch.float32, (M,))
    if q_rowsum is not None:
        _need(q_rowsum, "q_rowsum", torch.int32, (M,))
        _check(_lib.mmf_act_quant_ex(_ptr(x), int(is_f32), _ptr(gamma), _ptr(q), _ptr(a_scale),
                                     _ptr(q_rowsum), M, K, _stream(stream)))
        return
    fn = _lib.mmf_act_quant_f32 if is_f32 else _lib.mmf_act_quant
    _check(fn(_ptr(x), _ptr(gamma), _ptr(q), _ptr(a_scale), M, K, _stream(stream)))


def mmf_act_quant_ex(x: torch.Tensor, gamma: torch.Tensor | None, q: torch.Tensor,
                     a_scale: torch.Tensor, q_rowsum: torch.Tensor | None, stream=None) -> None:
    """mmf_act_quant with the row sums q_rowsum i32 [M] (None: not written)."""
    mmf_act_quant(x, gamma, q, a_scale, q_rowsum, stream)


def mmf_add_act_quant(x: torch.Tensor, branch: torch.Tensor | None, gamma: torch.Tensor | None,
                      s: torch.Tensor | None, q: torch.Tensor, a_scale: torch.Tensor,
                      q_rowsum: torch.Tensor | None = None, rstd: torch.Tensor | None = None,
                      stream=None) -> None:
    """s = x + branch (bf16/f32 [M][K], in the type of x; may be x) and its
    quantisation as mmf_act_quant gives it: q int8 [M][K], a_scale f32 [M],
    q_rowsum i32 [M], rstd f32 [M].  branch bf16/f32 [M][K], or None: s = x,
    which may be None."""
    here = _here()
    M, K = x.shape
    is_f32 = _x_kind(x)
    _need_here(x, "x", x.dtype, (M, K), here)
    branch_f32 = False
    if branch is not None:
        branch_f32 = _kind(branch, "branch")
        _need_here(branch, "branch", branch.dtype, (M, K), here)
    if gamma is not None:
        _need_here(gamma, "gamma", torch.float32, (K,), here)
    if s is not None or branch is not None:
        _need_here(s, "s", x.dtype, (M, K), here)
    _need_here(q, "q", torch.int8, (M, K), here)
    _need_here(a_scale, "a_scale", torch.float32, (M,), here)
    if q_rowsum is not None:
        _need_here(q_rowsum, "q_rowsum", torch.int32, (M,), here)
    if rstd is not None:
        _need_here(rstd, "rstd", torch.float32, (M,), here)
    _check(_lib.mmf_add_act_quant(_ptr(x), is_f32, _ptr(branch), branch_f32, _ptr(gamma), _ptr(s), _ptr(q),
                                  _ptr(a_scale), _ptr(q_rowsum), _ptr(rstd), M, K, _stream_here(stream, here)))


def mmf_add_act_quant_bwd_workspace_bytes(M: int, K: int) -> int:
    return int(_lib.mmf_add_act_quant_bwd_workspace_bytes(M, K))


def mmf_add_act_quant_bwd(dY: torch.Tensor, ds_out: torch.Tensor | None, s: torch.Tensor,
                          gamma: torch.Tensor | None, rstd: torch.Tensor, ds: torch.Tensor,
                          ds_bf16: torch.Tensor | None, dgamma: torch.Tensor | None,
                          workspace: torch.Tensor | None = None, stream=None) -> None:
    """Backward: ds f32 [M][K] (may be ds_out), the same in bf16 (or None) and
    dgamma f32 [K] (or None) from dY bf16/f32 [M][K], the residual stream's
    gradient ds_out f32 [M][K] (or None) and the forward's s and rstd."""
    here = _here()
    M, K = s.shape
    s_f32, dy_f32 = _kind(s, "s"), _kind(dY, "dY")
    _need_here(dY, "dY", dY.dtype, (M, K), here)
    if ds_out is not None:
        _need_here(ds_out, "ds_out", torch.float32, (M, K), here)
    _need_here(s, "s", s.dtype, (M, K), here)
    if gamma is not None:
        _need_here(gamma, "gamma", torch.float32, (K,), here)
    _need_here(rstd, "rstd", torch.float32, (M,), here)
    _need_here(ds, "ds", torch.float32, (M, K), here)
    if ds_bf16 is not None:
        _need_here(ds_bf16, "ds_bf16", torch.bfloat16, (M, K), here)
    if dgamma is not None:
        _need_here(dgamma, "dgamma", torch.float32, (K,), here)
    wp, wn = _ws_here(workspace, here)
    _check(_lib.mmf_add_act_quant_bwd(_ptr(dY), dy_f32, _ptr(ds_out), _ptr(s), s_f32, _ptr(gamma), _ptr(rstd),
                                      _ptr(ds), _ptr(ds_bf16), _ptr(dgamma), M, K, wp, wn, _stream_here(stream, here)))


def mmf_bitlinear_fwd(x: torch.Tensor, gamma: torch.Tensor | None, Wpacked: torch.Tensor,
                      w_scale: torch.Tensor, y: torch.Tensor, stream=None) -> None:
    """The fused forward: y f32 [M][N] from x bf16/f32 [M][K] and packed weights [K/16][N]."""
    M, K = x.shape
    N = Wpacked.shape[1]
    is_f32 = _x_kind(x)
    _need(x, "x", x.dtype, (M, K))
    if gamma is not None:
        _need(gamma, "gamma", torch.float32, (K,))
    _need(Wpacked, "Wpacked", torch.int32, (K // 16, N))
    _need(w_scale, "w_scale", torch.float32, (1,))
    _need(y, "y", torch.float32, (M, N))
    fn = _lib.mmf_bitlinear_fwd_f32 if is_f32 else _lib.mmf_bitlinear_fwd
    _check(fn(_ptr(x), _ptr(gamma), _ptr(Wpacked), _ptr(w_scale), _ptr(y), M, K, N,
              _stream(stream)))


def mmf_bitlinear_workspace_bytes(M: int, K: int) -> int:
    return int(_lib.mmf_bitlinear_workspace_bytes(M, K))


def mmf_bitlinear_fwd_ws(x: torch.Tensor, gamma: torch.Tensor | None, Wpacked: torch.Tensor,
                         w_scale: torch.Tensor, y: torch.Tensor, workspace: torch.Tensor,
                         stream=None) -> None:
    """The fused forward with caller scratch (a uint8 device tensor)."""
    M, K = x.shape
    N = Wpacked.shape[1]
    is_f32 = _x_kind(x)
    _need(x, "x", x.dtype, (M, K))
    if gamma is not None:
        _need(gamma, "gamma", torch.float32, (K,))
    _need(Wpacked, "Wpacked", torch.int32, (K // 16, N))
    _need(w_scale, "w_scale", torch.float32, (1,))
    _need(y, "y", torch.float32, (M, N))
    _need(workspace, "workspace", torch.uint8, (workspace.numel(),))
    _check(_lib.mmf_bitlinear_fwd_ws(_ptr(x), int(is_f32), _ptr(gamma), _ptr(Wpacked),
                                     _ptr(w_scale), _ptr(y), M, K, N, _ptr(workspace),
                                     workspace.numel(), _stream(stream)))


def mmf_bitlinear_noalloc_max_bytes() -> int:
    return int(_lib.mmf_bitlinear_noalloc_max_bytes())


def mmf_bitlinear_fwd_noalloc(x: torch.Tensor, gamma: torch.Tensor | None, Wpacked: torch.Tensor,
                              w_scale: torch.Tensor, y: torch.Tensor, stream=None) -> None:
    """The fused forward with the library's static device scratch (allocates nothing)."""
    M, K = x.shape
    N = Wpacked.shape[1]
    is_f32 = _x_kind(x)
    _need(x, "x", x.dtype, (M, K))
    if gamma is not None:
        _need(gamma, "gamma", torch.float32, (K,))
    _need(Wpacked, "Wpacked", torch.int32, (K // 16, N))
    _need(w_scale, "w_scale", torch.float32, (1,))
    _need(y, "y", torch.float32, (M, N))
    _check(_lib.mmf_bitlinear_fwd_noalloc(_ptr(x), int(is_f32), _ptr(gamma), _ptr(Wpacked),
                                          _ptr(w_scale), _ptr(y), M, K, N, _stream(stream)))


def mmf_ternary_gemm_dequant(q: torch.Tensor, a_scale: torch.Tensor, q_rowsum: torch.Tensor,
                             Wpacked: torch.Tensor, w_scale: torch.Tensor, y: torch.Tensor,
                             stream=None) -> None:
    """Contraction + dequant from quantised activations (the forward after act-quant)."""
    M, K = q.shape
    N = Wpacked.shape[1]
    _need(q, "q", torch.int8, (M, K))
    _need(a_scale, "a_scale", torch.float32, (M,))
    _need(q_rowsum, "q_rowsum", torch.int32, (M,))
    _need(Wpacked, "Wpacked", torch.int32, (K // 16, N))
    _need(w_scale, "w_scale", torch.float32, (1,))
    _need(y, "y", torch.float32, (M, N))
    _check(_lib.mmf_ternary_gemm_dequant(_ptr(q), _ptr(a_scale), _ptr(q_rowsum), _ptr(Wpacked),
                                         _ptr(w_scale), _ptr(y), M, K, N, _stream(stream)))


def mmf_ternary_gemm_i32(q: torch.Tensor, Wpacked: torch.Tensor, acc: torch.Tensor,
                         stream=None) -> None:
    """Raw int32 ternary sums acc [M][N] from q int8 [M][K] and packed weights."""
    M, K = q.shape
    N = Wpacked.shape[1]
    _need(q, "q", torch.int8, (M, K))
    _need(Wpacked, "Wpacked", torch.int32, (K // 16, N))
    _need(acc, "acc", torch.int32, (M, N))
    _check(_lib.mmf_ternary_gemm_i32(_ptr(q), _ptr(Wpacked), _ptr(acc), M, K, N, _stream(stream)))


def mmf_glu_pack(Wg_packed: torch.Tensor, Wu_packed: torch.Tensor, Wgu_packed: torch.Tensor,
                 stream=None) -> None:
    """Interleave the packed gate and up projections [K/16][L] into [K/16][2L]
    (16-column blocks of gate and up in turn); L % 16 == 0."""
    J, L = Wg_packed.shape
    _need(Wg_packed, "Wg_packed", torch.int32, (J, L))
    _need(Wu_packed, "Wu_packed", torch.int32, (J, L))
    _need(Wgu_packed, "Wgu_packed", torch.int32, (J, 2 * L))
    _check(_lib.mmf_glu_pack(_ptr(Wg_packed), _ptr(Wu_packed), L, 16 * J, _ptr(Wgu_packed),
                             _stream(stream)))


def _glu_args(x, gamma, Wgu_packed, w_scales, p):
    M, K = x.shape
    L = Wgu_packed.shape[1] // 2
    is_f32 = _x_kind(x)
    _need(x, "x", x.dtype, (M, K))
    if gamma is not None:
        _need(gamma, "gamma", torch.float32, (K,))
    _need(Wgu_packed, "Wgu_packed", torch.int32, (K // 16, 2 * L))
    _need(w_scales, "w_scales", torch.float32, (2,))
    _need(p, "p", torch.float32, (M, L))
    return M, K, L, is_f32


def mmf_glu_fwd(x: torch.Tensor, gamma: torch.Tensor | None, Wgu_packed: torch.Tensor,
                w_scales: torch.Tensor, p: torch.Tensor, stream=None) -> None:
    """GLU up-projections and gate: p f32 [M][L] = SiLU(g) * u from x bf16/f32
    [M][K], the interleaved packed weights [K/16][2L] and w_scales [gate, up]."""
    M, K, L, is_f32 = _glu_args(x, gamma, Wgu_packed, w_scales, p)
    fn = _lib.mmf_glu_fwd_f32 if is_f32 else _lib.mmf_glu_fwd
    _check(fn(_ptr(x), _ptr(gamma), _ptr(Wgu_packed), _ptr(w_scales), _ptr(p), M, K, L,
              _stream(stream)))


def mmf_glu_fwd_ws(x: torch.Tensor, gamma: torch.Tensor | None, Wgu_packed: torch.Tensor,
                   w_scales: torch.Tensor, p: torch.Tensor, workspace: torch.Tensor,
                   stream=None) -> None:
    """mmf_glu_fwd with caller scratch (uint8, mmf_bitlinear_workspace_bytes(M, K))."""
    M, K, L, is_f32 = _glu_args(x, gamma, Wgu_packed, w_scales, p)
    _need(workspace, "workspace", torch.uint8, (workspace.numel(),))
    _check(_lib.mmf_glu_fwd_ws(_ptr(x), int(is_f32), _ptr(gamma), _ptr(Wgu_packed),
                               _ptr(w_scales), _ptr(p), M, K, L, _ptr(workspace),
                               workspace.numel(), _stream(stream)))


def mmf_ternary_gemm_glu(q: torch.Tensor, a_scale: torch.Tensor, q_rowsum: torch.Tensor,
                         Wgu_packed: torch.Tensor, w_scales: torch.Tensor, p: torch.Tensor,
                         stream=None) -> None:
    """The GLU contraction and gate from quantised activations: p [M][L]."""
    M, K = q.shape
    L = Wgu_packed.shape[1] // 2
    _need(q, "q", torch.int8, (M, K))
    _need(a_scale, "a_scale", torch.float32, (M,))
    _need(q_rowsum, "q_rowsum", torch.int32, (M,))
    _need(Wgu_packed, "Wgu_packed", torch.int32, (K // 16, 2 * L))
    _need(w_scales, "w_scales", torch.float32, (2,))
    _need(p, "p", torch.float32, (M, L))
    _check(_lib.mmf_ternary_gemm_glu(_ptr(q), _ptr(a_scale), _ptr(q_rowsum), _ptr(Wgu_packed),
                                     _ptr(w_scales), _ptr(p), M, K, L, _stream(stream)))


def _ws_args(workspace: torch.Tensor | None):
    if workspace is None:
        return _ptr(None), 0
    _need(workspace, "workspace", torch.uint8, (workspace.numel(),))
    return _ptr(workspace), workspace.numel()


def mmf_bitlinear_fwd_bias(x: torch.Tensor, gamma: torch.Tensor | None, Wpacked: torch.Tensor,
                           w_scale: torch.Tensor, bias: torch.Tensor, y: torch.Tensor,
                           stream=None) -> None:
    """y f32 [M][N] = BitLinear(x) + bias [N] (N % 4 == 0)."""
    M, K = x.shape
    N = Wpacked.shape[1]
    is_f32 = _x_kind(x)
    _need(x, "x", x.dtype, (M, K))
    if gamma is not None:
        _need(gamma, "gamma", torch.float32, (K,))
    _need(Wpacked, "Wpacked", torch.int32, (K // 16, N))
    _need(w_scale, "w_scale", torch.float32, (1,))
    _need(bias, "bias", torch.float32, (N,))
    _need(y, "y", torch.float32, (M, N))
    _check(_lib.mmf_bitlinear_fwd_bias(_ptr(x), int(is_f32), _ptr(gamma), _ptr(Wpacked),
                                       _ptr(w_scale), _ptr(bias), _ptr(y), M, K, N,
                                       _stream(stream)))


def mmf_mlgru_proj_workspace_bytes(M: int, K: int, d: int) -> int:
    return int(_lib.mmf_mlgru_proj_workspace_bytes(M, K, d))


def mmf_mlgru_scan_workspace_bytes(B: int, T: int, d: int) -> int:
    return int(_lib.mmf_mlgru_scan_workspace_bytes(B, T, d))


def mmf_mlgru_workspace_bytes(B: int, T: int, d: int) -> int:
    return int(_lib.mmf_mlgru_workspace_bytes(B, T, d))


def mmf_mlgru_proj(x: torch.Tensor, gamma: torch.Tensor | None, Wfcg: torch.Tensor,
                   w_scales: torch.Tensor, bias: torch.Tensor | None, lb: torch.Tensor | None,
                   fcg: torch.Tensor, workspace: torch.Tensor | None = None, stream=None) -> None:
    """MLGRU input projections and gates: fcg f32 [M][3d] (f | c | g) from x
    bf16/f32 [M][K], Wfcg [K/16][3d], w_scales [3], bias [3d] or None, lb [d]
    or None."""
    M, K = x.shape
    d = Wfcg.shape[1] // 3
    is_f32 = _x_kind(x)
    _need(x, "x", x.dtype, (M, K))
    if gamma is not None:
        _need(gamma, "gamma", torch.float32, (K,))
    _need(Wfcg, "Wfcg", torch.int32, (K // 16, 3 * d))
    _need(w_scales, "w_scales", torch.float32, (3,))
    if bias is not None:
        _need(bias, "bias", torch.float32, (3 * d,))
    if lb is not None:
        _need(lb, "lb", torch.float32, (d,))
    _need(fcg, "fcg", torch.float32, (M, 3 * d))
    wp, wn = _ws_args(workspace)
    _check(_lib.mmf_mlgru_proj(_ptr(x), int(is_f32), _ptr(gamma), _ptr(Wfcg), _ptr(w_scales),
                               _ptr(bias), _ptr(lb), _ptr(fcg), M, K, d, wp, wn, _stream(stream)))


def mmf_mlgru_proj_q(q: torch.Tensor, a_scale: torch.Tensor, q_rowsum: torch.Tensor,
                     Wfcg: torch.Tensor, w_scales: torch.Tensor, bias: torch.Tensor | None,
                     lb: torch.Tensor | None, fcg: torch.Tensor, stream=None) -> None:
    """The MLGRU projection's contraction and gates from quantised activations."""
    M, K = q.shape
    d = Wfcg.shape[1] // 3
    _need(q, "q", torch.int8, (M, K))
    _need(a_scale, "a_scale", torch.float32, (M,))
    _need(q_rowsum, "q_rowsum", torch.int32, (M,))
    _need(Wfcg, "Wfcg", torch.int32, (K // 16, 3 * d))
    _need(w_scales, "w_scales", torch.float32, (3,))
    if bias is not None:
        _need(bias, "bias", torch.float32, (3 * d,))
    if lb is not None:
        _need(lb, "lb", torch.float32, (d,))
    _need(fcg, "fcg", torch.float32, (M, 3 * d))
    _check(_lib.mmf_mlgru_proj_q(_ptr(q), _ptr(a_scale), _ptr(q_rowsum), _ptr(Wfcg),
                                 _ptr(w_scales), _ptr(bias), _ptr(lb), _ptr(fcg), M, K, d,
                                 _stream(stream)))


def mmf_mlgru_scan(fcg: torch.Tensor, B: int, T: int, h0: torch.Tensor | None,
                   o_prime: torch.Tensor, h_last: torch.Tensor | None,
                   workspace: torch.Tensor | None = None, stream=None) -> None:
    """MLGRU recurrence and output gate over B sequences of T tokens (rows
    b*T + t): o_prime f32 [B*T][d], final state h_last [B][d] (may be h0)."""
    d = fcg.shape[1] // 3
    _need(fcg, "fcg", torch.float32, (B * T, 3 * d))
    if h0 is not None:
        _need(h0, "h0", torch.float32, (B, d))
    _need(o_prime, "o_prime", torch.float32, (B * T, d))
    if h_last is not None:
        _need(h_last, "h_last", torch.float32, (B, d))
    wp, wn = _ws_args(workspace)
    _check(_lib.mmf_mlgru_scan(_ptr(fcg), _ptr(h0), _ptr(o_prime), _ptr(h_last), B, T, d, wp, wn,
                               _stream(stream)))


def mmf_mlgru_fwd(x: torch.Tensor, B: int, T: int, gamma: torch.Tensor | None,
                  Wfcg: torch.Tensor, w_scales: torch.Tensor, bias: torch.Tensor | None,
                  lb: torch.Tensor | None, h0: torch.Tensor | None, h_last: torch.Tensor | None,
                  gamma_o: torch.Tensor | None, Wo: torch.Tensor, w_scale_o: torch.Tensor,
                  b_o: torch.Tensor | None, o: torch.Tensor,
                  workspace: torch.Tensor | None = None, stream=None) -> None:
    """The whole MLGRU token mixer: o f32 [B*T][d] from x bf16/f32 [B*T][d]."""
    d = Wo.shape[1]
    is_f32 = _x_kind(x)
    _need(x, "x", x.dtype, (B * T, d))
    for name, t, shape in (("gamma", gamma, (d,)), ("bias", bias, (3 * d,)), ("lb", lb, (d,)),
                           ("h0", h0, (B, d)), ("h_last", h_last, (B, d)),
                           ("gamma_o", gamma_o, (d,)), ("b_o", b_o, (d,))):
        if t is not None:
            _need(t, name, torch.float32, shape)
    _need(Wfcg, "Wfcg", torch.int32, (d // 16, 3 * d))
    _need(w_scales, "w_scales", torch.float32, (3,))
    _need(Wo, "Wo", torch.int32, (d // 16, d))
    _need(w_scale_o, "w_scale_o", torch.float32, (1,))
    _need(o, "o", torch.float32, (B * T, d))
    wp, wn = _ws_args(workspace)
    _check(_lib.mmf_mlgru_fwd(_ptr(x), int(is_f32), _ptr(gamma), _ptr(Wfcg), _ptr(w_scales),
                              _ptr(bias), _ptr(lb), _ptr(h0), _ptr(h_last), _ptr(gamma_o),
                              _ptr(Wo), _ptr(w_scale_o), _ptr(b_o), _ptr(o), B, T, d, wp, wn,
                              _stream(stream)))


def mmf_mlgru_train_states_bytes(B: int, T: int, d: int) -> int:
    return int(_lib.mmf_mlgru_train_states_bytes(B, T, d))


def mmf_mlgru_train_scan_workspace_bytes(B: int, T: int, d: int) -> int:
    return int(_lib.mmf_mlgru_train_scan_workspace_bytes(B, T, d))


def mmf_mlgru_scan_bwd_workspace_bytes(B: int, T: int, d: int) -> int:
    return int(_lib.mmf_mlgru_scan_bwd_workspace_bytes(B, T, d))


def mmf_mlgru_train_scan(z: torch.Tensor, B: int, T: int, lb: torch.Tensor | None, h0: torch.Tensor | None,
                         o_prime: torch.Tensor, h_last: torch.Tensor | None, states: torch.Tensor,
                         workspace: torch.Tensor | None = None, stream=None) -> None:
    """The recurrence in training form: o_prime f32 [B*T][d] and h_last f32
    [B][d] (or None; may be h0) from the gates' pre-activations z f32 [B*T][3d]
    (f | c | g), lb f32 [d] or None and h0 f32 [B][d] or None; states uint8
    (mmf_mlgru_train_states_bytes) keeps what mmf_mlgru_scan_bwd starts from."""
    here = _here()
    d = z.shape[1] // 3
    _need_here(z, "z", torch.float32, (B * T, 3 * d), here)
    if lb is not None:
        _need_here(lb, "lb", torch.float32, (d,), here)
    if h0 is not None:
        _need_here(h0, "h0", torch.float32, (B, d), here)
    _need_here(o_prime, "o_prime", torch.float32, (B * T, d), here)
    if h_last is not None:
        _need_here(h_last, "h_last", torch.float32, (B, d), here)
    _need_here(states, "states", torch.uint8, (states.numel(),), here)
    wp, wn = _ws_here(workspace, here)
    _check(_lib.mmf_mlgru_train_scan(_ptr(z), _ptr(lb), _ptr(h0), _ptr(o_prime), _ptr(h_last), _ptr(states),
                                     states.numel(), B, T, d, wp, wn, _stream_here(stream, here)))


def mmf_mlgru_scan_bwd(z: torch.Tensor, B: int, T: int, lb: torch.Tensor | None, states: torch.Tensor,
                       do_prime: torch.Tensor, dh_last: torch.Tensor | None, dz: torch.Tensor,
                       dh0: torch.Tensor | None, dlb: torch.Tensor | None,
                       workspace: torch.Tensor | None = None, stream=None) -> None:
    """Backward of mmf_mlgru_train_scan: dz bf16 [B*T][3d] (the dO of
    mmf_bitlinear_bwd), dh0 f32 [B][d] (or None; may be dh_last) and dlb f32
    [d] (or None) from do_prime bf16/f32 [B*T][d], dh_last f32 [B][d] (or None) and the forward's
    z, lb and states."""
    here = _here()
    d = z.shape[1] // 3
    do_f32 = _kind(do_prime, "do_prime")
    _need_here(z, "z", torch.float32, (B * T, 3 * d), here)
    if lb is not None:
        _need_here(lb, "lb", torch.float32, (d,), here)
    _need_here(states, "states", torch.uint8, (states.numel(),), here)
    _need_here(do_prime, "do_prime", do_prime.dtype, (B * T, d), here)
    if dh_last is not None:
        _need_here(dh_last, "dh_last", torch.float32, (B, d), here)
    _need_here(dz, "dz", torch.bfloat16, (B * T, 3 * d), here)
    if dh0 is not None:
        _need_here(dh0, "dh0", torch.float32, (B, d), here)
    if dlb is not None:
        _need_here(dlb, "dlb", torch.float32, (d,), here)
    wp, wn = _ws_here(workspace, here)
    _check(_lib.mmf_mlgru_scan_bwd(_ptr(z), _ptr(lb), _ptr(states), states.numel(), _ptr(do_prime), do_f32,
                                   _ptr(dh_last), _ptr(dz), _ptr(dh0), _ptr(dlb), B, T, d, wp, wn,
                                   _stream_here(stream, here)))


def mmf_glu_train_workspace_bytes(M: int, K: int, L: int) -> int:
    return int(_lib.mmf_glu_train_workspace_bytes(M, K, L))


def mmf_glu_bwd_workspace_bytes(M: int, K: int, L: int) -> int:
    return int(_lib.mmf_glu_bwd_workspace_bytes(M, K, L))


def mmf_glu_train_fwd(q: torch.Tensor, a_scale: torch.Tensor, q_rowsum: torch.Tensor, W: torch.Tensor,
                      p: torch.Tensor, Wpacked: torch.Tensor, w_scale: torch.Tensor,
                      workspace: torch.Tensor | None = None, stream=None) -> None:
    """Training forward of the GLU's gated up-projections from quantised
    activations and the stacked latent weights W f32 [2L][K] (gate, up): p f32
    [M][L], and Wpacked int32 [K/16][2L] and w_scale f32 [1] for the backward."""
    here = _here()
    M, K = q.shape
    L = W.shape[0] // 2
    _need_here(q, "q", torch.int8, (M, K), here)
    _need_here(a_scale, "a_scale", torch.float32, (M,), here)
    _need_here(q_rowsum, "q_rowsum", torch.int32, (M,), here)
    _need_here(W, "W", torch.float32, (2 * L, K), here)
    _need_here(p, "p", torch.float32, (M, L), here)
    _need_here(Wpacked, "Wpacked", torch.int32, (K // 16, 2 * L), here)
    _need_here(w_scale, "w_scale", torch.float32, (1,), here)
    wp, wn = _ws_here(workspace, here)
    _check(_lib.mmf_glu_train_fwd(_ptr(q), _ptr(a_scale), _ptr(q_rowsum), _ptr(W), _ptr(p), _ptr(Wpacked),
                                  _ptr(w_scale), M, K, L, wp, wn, _stream_here(stream, here)))


def mmf_glu_gate_bwd(q: torch.Tensor, a_scale: torch.Tensor, q_rowsum: torch.Tensor, Wgu_packed: torch.Tensor,
                     w_scales: torch.Tensor, dp: torch.Tensor, dgu: torch.Tensor, stream=None) -> None:
    """The GLU gate's gradients dgu bf16 [M][2L] (dg | du) from dp bf16/f32
    [M][L], the projections recomputed from the quantised activations and the
    interleaved packed weights [K/16][2L] with w_scales [gate, up]."""
    here = _here()
    M, K = q.shape
    L = Wgu_packed.shape[1] // 2
    dp_f32 = _kind(dp, "dp")
    _need_here(q, "q", torch.int8, (M, K), here)
    _need_here(a_scale, "a_scale", torch.float32, (M,), here)
    _need_here(q_rowsum, "q_rowsum", torch.int32, (M,), here)
    _need_here(Wgu_packed, "Wgu_packed", torch.int32, (K // 16, 2 * L), here)
    _need_here(w_scales, "w_scales", torch.float32, (2,), here)
    _need_here(dp, "dp", dp.dtype, (M, L), here)
    _need_here(dgu, "dgu", torch.bfloat16, (M, 2 * L), here)
    _check(_lib.mmf_glu_gate_bwd(_ptr(q), _ptr(a_scale), _ptr(q_rowsum), _ptr(Wgu_packed), _ptr(w_scales), _ptr(dp),
                                 dp_f32, _ptr(dgu), M, K, L, _stream_here(stream, here)))


def mmf_glu_bwd(dp: torch.Tensor, x: torch.Tensor, gamma: torch.Tensor | None, rstd: torch.Tensor, q: torch.Tensor,
                a_scale: torch.Tensor, q_rowsum: torch.Tensor, Wpacked: torch.Tensor, w_scale: torch.Tensor,
                dx: torch.Tensor, dW: torch.Tensor, dgamma: torch.Tensor | None,
                workspace: torch.Tensor | None = None, stream=None) -> None:
    """Backward of the GLU's gated up-projections: dx f32 [M][K], dW f32
    [2L][K] (gate, up) and dgamma f32 [K] (or None) from dp bf16/f32 [M][L], the
    input x bf16/f32 [M][K] with gamma, rstd, q, a_scale and q_rowsum, and
    mmf_glu_train_fwd's Wpacked and w_scale."""
    here = _here()
    M, K = x.shape
    L = Wpacked.shape[1] // 2
    is_f32, dp_f32 = _x_kind(x), _kind(dp, "dp")
    _need_here(dp, "dp", dp.dtype, (M, L), here)
    _need_here(x, "x", x.dtype, (M, K), here)
    if gamma is not None:
        _need_here(gamma, "gamma", torch.float32, (K,), here)
    _need_here(rstd, "rstd", torch.float32, (M,), here)
    _need_here(q, "q", torch.int8, (M, K), here)
    _need_here(a_scale, "a_scale", torch.float32, (M,), here)
    _need_here(q_rowsum, "q_rowsum", torch.int32, (M,), here)
    _need_here(Wpacked, "Wpacked", torch.int32, (K // 16, 2 * L), here)
    _need_here(w_scale, "w_scale", torch.float32, (1,), here)
    _need_here(dx, "dx", torch.float32, (M, K), here)
    _need_here(dW, "dW", torch.float32, (2 * L, K), here)
    if dgamma is not None:
        _need_here(dgamma, "dgamma", torch.float32, (K,), here)
    wp, wn = _ws_here(workspace, here)
    _check(_lib.mmf_glu_bwd(_ptr(dp), dp_f32, _ptr(x), is_f32, _ptr(gamma), _ptr(rstd), _ptr(q), _ptr(a_scale),
                            _ptr(q_rowsum), _ptr(Wpacked), _ptr(w_scale), _ptr(dx), _ptr(dW), _ptr(dgamma), M, K, L,
                            wp, wn, _stream_here(stream, here)))


# Lists of tensors: checked and converted by map over whole lists, and passed
# as arrays of integers (a loop with the same checks and ctypes arrays took 0.5
# us a tensor and call, this 0.25).
_T = torch.Tensor
_dtype_of = operator.attrgetter("dtype")


def _grad_ptrs(tensors, name, here):
    """Addresses of a list of contiguous bf16 or f32 tensors on the current device, and their types."""
    try:
        kinds = list(map(_dtype_of, tensors))
        if (all(map(_T.is_contiguous, tensors)) and set(map(_T.get_device, tensors)) <= {here}
                and kinds.count(torch.float32) + kinds.count(torch.bfloat16) == len(kinds)):
            return array.array("Q", list(map(_T.data_ptr, tensors))), kinds
    except (AttributeError, TypeError, RuntimeError):
        pass
    for i, t in enumerate(tensors):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name}[{i}] must be a torch.Tensor")
        _kind(t, f"{name}[{i}]")
        _need_here(t, f"{name}[{i}]", t.dtype, t.shape, here)
    raise ValueError(f"{name} must be tensors on the current device")


def _listed(tensors, name):
    """The tensors as a list or tuple (a generator could be passed over only once)."""
    if isinstance(tensors, torch.Tensor):
        raise TypeError(f"{name} must be a list of tensors")
    return tensors if isinstance(tensors, (list, tuple)) else list(tensors)


def _grad_set(tensors, here):
    """What the C calls take: arrays of addresses, kinds and sizes, and the types."""
    tensors = _listed(tensors, "grads")
    ptrs, types = _grad_ptrs(tensors, "grads", here)
    n, n32 = len(types), types.count(torch.float32)
    if n32 == n or n32 == 0:
        is_f32 = array.array("i", (n32 > 0,)) * n
    else:
        is_f32 = array.array("i", [k is torch.float32 for k in types])
    return ptrs, is_f32, array.array("q", list(map(_T.numel, tensors))), types


def _at(a: array.array) -> int:
    return a.buffer_info()[0]


def mmf_grad_norm_workspace_bytes(counts) -> int:
    c = array.array("q", counts)
    return int(_lib.mmf_grad_norm_workspace_bytes(_at(c), len(c)))


def mmf_grad_norm(grads, norm: torch.Tensor, workspace: torch.Tensor | None = None, stream=None) -> None:
    """norm f32 [1] = the 2-norm over all elements of the tensors of the list
    `grads` (each bf16 or f32, contiguous, of any shape, on 16 bytes)."""
    here = _here()
    _need_here(norm, "norm", torch.float32, (1,), here)
    ptrs, kinds, counts, _ = _grad_set(grads, here)
    wp, wn = _ws_here(workspace, here)
    _check(_lib.mmf_grad_norm(_at(ptrs), _at(kinds), _at(counts), len(ptrs), _ptr(norm), wp, wn,
                              _stream_here(stream, here)))


def mmf_grad_clip(grads, norm: torch.Tensor, max_norm: float, outs=None, stream=None) -> None:
    """outs[i] = grads[i] * min(max_norm / (norm + 1e-6), 1); outs None: in
    place; max_norm infinite: no limit.  outs[i] has the type and the number of
    elements of grads[i]; no two of them may overlap."""
    here = _here()
    _need_here(norm, "norm", torch.float32, (1,), here)
    ptrs, kinds, counts, types = _grad_set(grads, here)
    dst = ptrs
    if outs is not None:
        outs = _listed(outs, "outs")
        dst, otypes = _grad_ptrs(outs, "outs", here)
        if otypes != types or array.array("q", list(map(_T.numel, outs))) != counts:
            raise ValueError("outs must have the types and numbers of elements of grads")
    if len(set(dst)) != len(dst):  # empty tensors may share an address
        full = [p for p, c in zip(dst, counts) if c]
        if len(set(full)) != len(full):
            raise ValueError("a tensor to write is in the list twice")
    _check(_lib.mmf_grad_clip(_at(ptrs), _at(kinds), _at(counts), len(ptrs), _ptr(norm), max_norm, _at(dst),
                              _stream_here(stream, here)))


def mmf_linattn_workspace_bytes(B: int, T: int, H: int, dk: int, dv: int) -> int:
    return int(_lib.mmf_linattn_workspace_bytes(B, T, H, dk, dv))


def mmf_linattn_fwd(qkv: torch.Tensor, B: int, T: int, H: int, dk: int, dv: int, decay: torch.Tensor, scale: float,
                    s0: torch.Tensor | None, o: torch.Tensor, s_last: torch.Tensor | None,
                    workspace: torch.Tensor | None = None, stream=None) -> None:
    """Linear attention with a decay per head: o [B*T][H dv] in the type of qkv
    bf16/f32 [B*T][H (2 dk + dv)] (q | k | v) and the last state s_last f32
    [B][H][dk][dv] (or None; may be s0) from decay f32 [H] and the first state
    s0 (or None)."""
    here = _here()
    dt = torch.float32 if _kind(qkv, "qkv") else torch.bfloat16
    _need_here(qkv, "qkv", dt, (B * T, H * (2 * dk + dv)), here)
    _need_here(decay, "decay", torch.float32, (H,), here)
    if s0 is not None:
        _need_here(s0, "s0", torch.float32, (B, H, dk, dv), here)
    _need_here(o, "o", dt, (B * T, H * dv), here)
    if s_last is not None:
        _need_here(s_last, "s_last", torch.float32, (B, H, dk, dv), here)
    wp, wn = _ws_here(workspace, here)
    _check(_lib.mmf_linattn_fwd(_ptr(qkv), dt is torch.float32, _ptr(decay), scale, _ptr(s0), _ptr(o), _ptr(s_last),
                                B, T, H, dk, dv, wp, wn, _stream_here(stream, here)))


def mmf_linattn_bwd_workspace_bytes(B: int, T: int, H: int, dk: int, dv: int) -> int:
    return int(_lib.mmf_linattn_bwd_workspace_bytes(B, T, H, dk, dv))


def mmf_linattn_bwd(qkv: torch.Tensor, B: int, T: int, H: int, dk: int, dv: int, decay: torch.Tensor, scale: float,
                    s0: torch.Tensor | None, dout: torch.Tensor, ds_last: torch.Tensor | None, dqkv: torch.Tensor,
                    ds0: torch.Tensor | None, workspace: torch.Tensor | None = None, stream=None) -> None:
    """Backward of mmf_linattn_fwd: dqkv bf16 [B*T][H (2 dk + dv)] (the dO of
    mmf_bitlinear_bwd) and ds0 f32 [B][H][dk][dv] (or None; may be ds_last) from
    dout bf16/f32 [B*T][H dv], ds_last f32 [B][H][dk][dv] (or None) and the
    forward's inputs."""
    here = _here()
    qkv_f32, do_f32 = _kind(qkv, "qkv"), _kind(dout, "dout")
    rows, wide, state = B * T, H * (2 * dk + dv), (B, H, dk, dv)
    _need_here(qkv, "qkv", qkv.dtype, (rows, wide), here)
    _need_here(decay, "decay", torch.float32, (H,), here)
    if s0 is not None:
        _need_here(s0, "s0", torch.float32, state, here)
    _need_here(dout, "dout", dout.dtype, (rows, H * dv), here)
    if ds_last is not None:
        _need_here(ds_last, "ds_last", torch.float32, state, here)
    _need_here(dqkv, "dqkv", torch.bfloat16, (rows, wide), here)
    if ds0 is not None:
        _need_here(ds0, "ds0", torch.float32, state, here)
    wp, wn = _ws_here(workspace, here)
    _check(_lib.mmf_linattn_bwd(_ptr(qkv), qkv_f32, _ptr(decay), scale, _ptr(s0), _ptr(dout), do_f32, _ptr(ds_last),
                                _ptr(dqkv), _ptr(ds0), B, T, H, dk, dv, wp, wn, _stream_here(stream, here)))


def mmf_beam_select_workspace_bytes(B: int, W: int, V: int, n: int) -> int:
    return int(_lib.mmf_beam_select_workspace_bytes(B, W, V, n))


def mmf_beam_select(logits: torch.Tensor, scores: torch.Tensor, done: torch.Tensor | None, end: int, B: int, W: int,
                    n: int, new_scores: torch.Tensor, tokens: torch.Tensor, parents: torch.Tensor,
                    new_done: torch.Tensor | None, workspace: torch.Tensor | None = None, stream=None) -> None:
    """One step of beam search: new_scores f32, tokens i32 and parents i32 [B][n]
    (and new_done u8, or None) of the n best continuations, from logits bf16/f32
    [B*W][V], scores f32 [B][W], done u8 [B][W] (or None) and the token `end`
    (-1: none)."""
    here = _here()
    is_f32 = _kind(logits, "logits")
    V = logits.shape[-1] if logits.dim() else 0
    _need_here(logits, "logits", logits.dtype, (B * W, V), here)
    _need_here(scores, "scores", torch.float32, (B, W), here)
    if done is not None:
        _need_here(done, "done", torch.uint8, (B, W), here)
    _need_here(new_scores, "new_scores", torch.float32, (B, n), here)
    _need_here(tokens, "tokens", torch.int32, (B, n), here)
    _need_here(parents, "parents", torch.int32, (B, n), here)
    if new_done is not None:
        _need_here(new_done, "new_done", torch.uint8, (B, n), here)
    wp, wn = _ws_here(workspace, here)
    _check(_lib.mmf_beam_select(_ptr(logits), is_f32, _ptr(scores), _ptr(done), end, _ptr(new_scores), _ptr(tokens),
                                _ptr(parents), _ptr(new_done), B, W, V, n, wp, wn, _stream_here(stream, here)))


_nbytes_of = operator.attrgetter("nbytes")


def _state_ptrs(tensors, name, rows, here):
    """Addresses and row sizes of a list of contiguous tensors of `rows` rows on the current device."""
    try:
        if (all(map(_T.is_contiguous, tensors)) and set(map(_T.get_device, tensors)) <= {here}
                and set(map(_T.size, tensors, itertools.repeat(0))) <= {rows}):
            return (array.array("Q", list(map(_T.data_ptr, tensors))),
                    array.array("q", [n // rows if rows else 0 for n in map(_nbytes_of, tensors)]))
    except (AttributeError, IndexError, TypeError, RuntimeError):
        pass
    for i, t in enumerate(tensors):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name}[{i}] must be a torch.Tensor")
        if t.dim() < 1 or t.shape[0] != rows:
            raise ValueError(f"{name}[{i}] must have {rows} rows, got shape {tuple(t.shape)}")
        _need_here(t, f"{name}[{i}]", t.dtype, t.shape, here)
    raise ValueError(f"{name} must be tensors on the current device")


def mmf_beam_reorder(states, parents: torch.Tensor, B: int, W: int, outs=None, stream=None) -> None:
    """outs[i] row (b, j) = states[i] row (b, parents[b][j]) for a list of tensors
    [B*W][...] of any type (rows of a multiple of 16 bytes); outs None: in place.
    parents i32 [B][W].  outs[i] has the type and shape of states[i] and may be
    states[i]; no two of outs may overlap, nor one of them another's state."""
    here = _here()
    states = _listed(states, "states")
    _need_here(parents, "parents", torch.int32, (B, W), here)
    src, rows = _state_ptrs(states, "states", B * W, here)
    dst = src
    if outs is not None:
        outs = _listed(outs, "outs")
        dst, orows = _state_ptrs(outs, "outs", B * W, here)
        if orows != rows or [t.dtype for t in outs] != [t.dtype for t in states]:
            raise ValueError("outs must have the types and shapes of states")
    if len(set(dst)) != len(dst):  # empty tensors may share an address
        full = [p for p, r in zip(dst, rows) if r]
        if len(set(full)) != len(full):
            raise ValueError("a tensor to write is in the list twice")
    if outs is not None and not set(dst).isdisjoint(src):  # some in place, or one that another is read from
        full = [(p, q) for p, q, r in zip(src, dst, rows) if r]
        written = {q for _, q in full}
        if any(p in written for p, q in full if p != q):
            raise ValueError("a tensor to write is one that another reads")
    _check(_lib.mmf_beam_reorder(_at(src), _at(dst), _at(rows), len(src), _ptr(parents), B, W,
                                 _stream_here(stream, here)))


def _distill_args(z, idx, t, here):
    z_f32, t_f32 = _kind(z, "z"), _kind(t, "t")
    M, V = z.shape
    K = t.shape[-1] if t.dim() else 0
    _need_here(z, "z", z.dtype, (M, V), here)
    _need_here(idx, "idx", torch.int32, (M, K), here)
    _need_here(t, "t", t.dtype, (M, K), here)
    return M, V, K, z_f32, t_f32


def mmf_distill_fwd(z: torch.Tensor, idx: torch.Tensor, t: torch.Tensor, tau: float, loss: torch.Tensor,
                    stream=None) -> None:
    """loss f32 [M] of student logits z bf16/f32 [M][V] from a teacher's logits t
    bf16/f32 [M][K] of the tokens idx i32 [M][K] (outside [0, V): none)."""
    here = _here()
    M, V, K, z_f32, t_f32 = _distill_args(z, idx, t, here)
    _need_here(loss, "loss", torch.float32, (M,), here)
    _check(_lib.mmf_distill_fwd(_ptr(z), z_f32, _ptr(idx), _ptr(t), t_f32, tau, _ptr(loss), M, V, K,
                                _stream_here(stream, here)))


def mmf_distill_bwd(z: torch.Tensor, idx: torch.Tensor, t: torch.Tensor, tau: float, dloss: torch.Tensor,
                    dz: torch.Tensor, loss: torch.Tensor | None = None, stream=None) -> None:
    """dz bf16/f32 [M][V] (may be z) from dloss f32 [M], and the loss f32 [M] (or
    None), in one pass; z, idx, t and tau as in mmf_distill_fwd."""
    here = _here()
    M, V, K, z_f32, t_f32 = _distill_args(z, idx, t, here)
    dz_f32 = _kind(dz, "dz")
    _need_here(dloss, "dloss", torch.float32, (M,), here)
    _need_here(dz, "dz", dz.dtype, (M, V), here)
    if loss is not None:
        _need_here(loss, "loss", torch.float32, (M,), here)
    _check(_lib.mmf_distill_bwd(_ptr(z), z_f32, _ptr(idx), _ptr(t), t_f32, tau, _ptr(dloss), _ptr(dz), dz_f32, _ptr(loss),
                                M, V, K, _stream_here(stream, here)))


def mmf_bitlinear_train_workspace_bytes(M: int, K: int, N: int) -> int:
    return int(_lib.mmf_bitlinear_train_workspace_bytes(M, K, N))


def mmf_bitlinear_bwd_workspace_bytes(M: int, K: int, N: int) -> int:
    return int(_lib.mmf_bitlinear_bwd_workspace_bytes(M, K, N))


def mmf_bitlinear_train_fwd(x: torch.Tensor, gamma: torch.Tensor | None, W: torch.Tensor,
                            bias: torch.Tensor | None, y: torch.Tensor, Wpacked: torch.Tensor,
                            w_scale: torch.Tensor, q: torch.Tensor, a_scale: torch.Tensor,
                            rstd: torch.Tensor | None, workspace: torch.Tensor | None = None,
                            stream=None) -> None:
    """Training forward from latent float32 weights W [N][K]: y [M][N] and the
    state the backward needs (Wpacked, w_scale, q, a_scale, rstd)."""
    M, K = x.shape
    N = W.shape[0]
    is_f32 = _x_kind(x)
    _need(x, "x", x.dtype, (M, K))
    if gamma is not None:
        _need(gamma, "gamma", torch.float32, (K,))
    _need(W, "W", torch.float32, (N, K))
    if bias is not None:
        _need(bias, "bias", torch.float32, (N,))
    _need(y, "y", torch.float32, (M, N))
    _need(Wpacked, "Wpacked", torch.int32, (K // 16, N))
    _need(w_scale, "w_scale", torch.float32, (1,))
    _need(q, "q", torch.int8, (M, K))
    _need(a_scale, "a_scale", torch.float32, (M,))
    if rstd is not None:
        _need(rstd, "rstd", torch.float32, (M,))
    wp, wn = _ws_args(workspace)
    _check(_lib.mmf_bitlinear_train_fwd(_ptr(x), int(is_f32), _ptr(gamma), _ptr(W), _ptr(bias), _ptr(y),
                                        _ptr(Wpacked), _ptr(w_scale), _ptr(q), _ptr(a_scale), _ptr(rstd),
                                        M, K, N, wp, wn, _stream(stream)))


def mmf_bitlinear_bwd(dO: torch.Tensor, x: torch.Tensor, gamma: torch.Tensor | None,
                      rstd: torch.Tensor, q: torch.Tensor, a_scale: torch.Tensor,
                      Wpacked: torch.Tensor, w_scale: torch.Tensor, dx: torch.Tensor,
                      dW: torch.Tensor, db: torch.Tensor | None, dgamma: torch.Tensor | None,
                      workspace: torch.Tensor | None = None, stream=None) -> None:
    """Backward: dx [M][K], dW [N][K], db [N], dgamma [K] (float32) from dO
    bf16 [M][N] and the training forward's saved state."""
    M, K = x.shape
    N = dO.shape[1]
    is_f32 = _x_kind(x)
    _need(dO, "dO", torch.bfloat16, (M, N))
    _need(x, "x", x.dtype, (M, K))
    if gamma is not None:
        _need(gamma, "gamma", torch.float32, (K,))
    _need(rstd, "rstd", torch.float32, (M,))
    _need(q, "q", torch.int8, (M, K))
    _need(a_scale, "a_scale", torch.float32, (M,))
    _need(Wpacked, "Wpacked", torch.int32, (K // 16, N))
    _need(w_scale, "w_scale", torch.float32, (1,))
    _need(dx, "dx", torch.float32, (M, K))
    _need(dW, "dW", torch.float32, (N, K))
    if db is not None:
        _need(db, "db", torch.float32, (N,))
    if dgamma is not None:
        _need(dgamma, "dgamma", torch.float32, (K,))
    wp, wn = _ws_args(workspace)
    _check(_lib.mmf_bitlinear_bwd(_ptr(dO), _ptr(x), int(is_f32), _ptr(gamma), _ptr(rstd), _ptr(q),
                                  _ptr(a_scale), _ptr(Wpacked), _ptr(w_scale), _ptr(dx), _ptr(dW),
                                  _ptr(db), _ptr(dgamma), M, K, N, wp, wn, _stream(stream)))


# ---------------------------------------------------------------------------
# allocating conveniences (outputs allocated with torch on the inputs' device)
# ---------------------------------------------------------------------------

def ternarize(W: torch.Tensor, stream=None):
    """Returns (Wpacked int32 [K/16][N], w_scale float32 [1])."""
    N, K = W.shape
    Wp = torch.empty((K // 16, N), dtype=torch.int32, device=W.device)
    ws = torch.empty((1,), dtype=torch.float32, device=W.device)
    mmf_ternarize_weights(W, Wp, ws, stream)
    return Wp, ws


def bitlinear(x: torch.Tensor, gamma: torch.Tensor | None, Wpacked: torch.Tensor,
              w_scale: torch.Tensor, stream=None) -> torch.Tensor:
    """Returns y float32 [M][N]."""
    y = torch.empty((x.shape[0], Wpacked.shape[1]), dtype=torch.float32, device=x.device)
    mmf_bitlinear_fwd(x, gamma, Wpacked, w_scale, y, stream)
    return y


def add_act_quant(x: torch.Tensor, branch: torch.Tensor | None, gamma: torch.Tensor | None, stream=None):
    """Returns (s in the type of x [M][K], q int8 [M][K], a_scale float32 [M],
    q_rowsum int32 [M], rstd float32 [M])."""
    M, K = x.shape
    s, q = torch.empty_like(x), torch.empty((M, K), dtype=torch.int8, device=x.device)
    a_scale, rstd = (torch.empty((M,), dtype=torch.float32, device=x.device) for _ in range(2))
    q_rowsum = torch.empty((M,), dtype=torch.int32, device=x.device)
    mmf_add_act_quant(x, branch, gamma, s, q, a_scale, q_rowsum, rstd, stream)
    return s, q, a_scale, q_rowsum, rstd


def glu_pack(Wg_packed: torch.Tensor, Wu_packed: torch.Tensor, stream=None) -> torch.Tensor:
    """Returns the interleaved [K/16][2L] packed weights of a GLU."""
    J, L = Wg_packed.shape
    Wgu = torch.empty((J, 2 * L), dtype=torch.int32, device=Wg_packed.device)
    mmf_glu_pack(Wg_packed, Wu_packed, Wgu, stream)
    return Wgu


def glu(x: torch.Tensor, gamma: torch.Tensor | None, Wgu_packed: torch.Tensor,
        w_scales: torch.Tensor, stream=None) -> torch.Tensor:
    """Returns p float32 [M][L] = SiLU(g) * u."""
    p = torch.empty((x.shape[0], Wgu_packed.shape[1] // 2), dtype=torch.float32, device=x.device)
    mmf_glu_fwd(x, gamma, Wgu_packed, w_scales, p, stream)
    return p


def mlgru_proj(x: torch.Tensor, gamma: torch.Tensor | None, Wfcg: torch.Tensor,
               w_scales: torch.Tensor, bias: torch.Tensor | None = None,
               lb: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Returns fcg float32 [M][3d]."""
    fcg = torch.empty((x.shape[0], Wfcg.shape[1]), dtype=torch.float32, device=x.device)
    mmf_mlgru_proj(x, gamma, Wfcg, w_scales, bias, lb, fcg, None, stream)
    return fcg


def mlgru_scan(fcg: torch.Tensor, B: int, T: int, h0: torch.Tensor | None = None, stream=None):
    """Returns (o_prime float32 [B*T][d], h_last float32 [B][d])."""
    d = fcg.shape[1] // 3
    o = torch.empty((B * T, d), dtype=torch.float32, device=fcg.device)
    h = torch.empty((B, d), dtype=torch.float32, device=fcg.device)
    mmf_mlgru_scan(fcg, B, T, h0, o, h, None, stream)
    return o, h
