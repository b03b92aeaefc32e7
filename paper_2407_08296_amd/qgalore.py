"""ctypes binding of libqgalore.so: argument marshalling only.

Every function has the name and argument order of the C entry point it wraps
(see include/qgalore.h) minus the `qg_` prefix.  Tensors are torch CUDA(HIP)
tensors used purely as device-memory handles; all arithmetic happens in the
library's kernels.  There is no CPU fallback: if the shared library has not
been built, importing a symbol from it raises.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("QGALORE_LIB") or os.path.join(_HERE, "libqgalore.so")   # QGALORE_LIB: another build of the library
GROUP = 256

EXPORTS = [
    "qg_status_string", "qg_last_hip_error", "qg_quant_int8", "qg_quant_int4", "qg_dequant_int8", "qg_dequant_int4",
    "qg_project", "qg_lowrank_adam", "qg_backproject_update_sr", "qg_cossim_workspace_bytes", "qg_subspace_cossim",
    "qg_policy_update", "qg_workspace_bytes", "qg_step", "qg_plan_bytes", "qg_plan_build", "qg_step_many",
    "qg_sr_uniform", "qg_project_many", "qg_lowrank_adam_many", "qg_backproject_update_sr_many",
    "qg_project_adam", "qg_project_adam_many", "qg_diag_clock_probe", "qg_diag_mfma_loop",
    "qg_diag_mfma_f64_loop",
    "qg_range_apply", "qg_orthonormalize_workspace_bytes", "qg_orthonormalize", "qg_refresh_workspace_bytes",
    "qg_subspace_refresh", "qg_subspace_refresh_many", "qg_int8_linear_forward", "qg_int8_linear_backward",
    "qg_int8_linear_t_forward", "qg_int8_linear_t_backward",
    "qg_quant_int8_zp", "qg_dequant_int8_zp", "qg_backproject_update_sr_zp", "qg_step_zp",
    "qg_int8_linear_zp_forward", "qg_int8_linear_zp_backward",
    "qg_int8_linear_t_zp_forward", "qg_int8_linear_t_zp_backward",
    "qg_state8_quant", "qg_state8_dequant", "qg_lowrank_adam8", "qg_step8",
    "qg_subspace_cossim_static", "qg_subspace_cossim_weighted", "qg_step_ld", "qg_subspace_refresh_many_ld",
    "qg_int8_linear_forward_ld", "qg_int8_linear_backward_ld",
    "qg_residual_norm_forward", "qg_residual_norm_workspace_bytes", "qg_residual_norm_backward",
    "qg_int8_linear_act_forward", "qg_int8_linear_act_workspace_bytes", "qg_int8_linear_act_backward", "qg_int8_gated_forward",
    "qg_int8_gated_backward", "qg_int8_gated_workspace_bytes", "qg_head_loss_workspace_bytes", "qg_head_loss_forward", "qg_head_loss_backward",
    "qg_rope_frequencies", "qg_rope_forward", "qg_rope_backward", "qg_attention_forward_workspace_bytes", "qg_attention_backward_workspace_bytes", "qg_attention_forward",
    "qg_attention_backward", "qg_cache_append", "qg_attention_paged_workspace_bytes", "qg_attention_paged",
]


class QGError(RuntimeError):
    pass


class HParams(C.Structure):
    _fields_ = [("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float), ("lr", C.c_float),
                ("alpha", C.c_float)]


class Policy(C.Structure):
    _fields_ = [("interval", C.c_int), ("streak", C.c_int), ("k", C.c_int), ("next_refresh", C.c_int),
                ("threshold", C.c_float), ("last_cos", C.c_float)]


class MatrixDesc(C.Structure):
    _fields_ = [("m", C.c_int64), ("n", C.c_int64), ("r", C.c_int64),
                ("Pq", C.c_void_p), ("Ps", C.c_void_p), ("G", C.c_void_p), ("Wq", C.c_void_p), ("Ws", C.c_void_p),
                ("M", C.c_void_p), ("V", C.c_void_p), ("R", C.c_void_p), ("N", C.c_void_p), ("ld", C.c_int64),
                ("Wz", C.c_void_p)]


class RefreshDesc(C.Structure):
    _fields_ = [("Pq", C.c_void_p), ("Ps", C.c_void_p), ("G", C.c_void_p), ("Pq_new", C.c_void_p),
                ("Ps_new", C.c_void_p)]


# qg_heads, qg_attention and qg_cache as bytes, the fields in the header's order and alignment (packed in 0.2 us where a ctypes structure and its
# pointer take 0.9 of the 10 us of a small call, which has up to nine of them)
_pack_heads = struct.Struct("@Pqq").pack
_pack_attention = struct.Struct("@qqiiiiPPPPffiq").pack
_pack_cache = struct.Struct("@PPPqiiiii").pack


_lib = None


def lib() -> C.CDLL:
    """Load libqgalore.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise QGError(f"{LIB_PATH} is missing: build it with `python -m paper_2407_08296_amd.build` "
                          "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        i64, vp, i32, u64, f32, sz = C.c_int64, C.c_void_p, C.c_int, C.c_uint64, C.c_float, C.c_size_t
        L.qg_status_string.restype = C.c_char_p
        L.qg_status_string.argtypes = [i32]
        L.qg_last_hip_error.restype = i32
        L.qg_quant_int8.argtypes = [vp, i64, i64, i32, vp, vp, vp]
        L.qg_quant_int4.argtypes = [vp, i64, i64, i32, vp, vp, vp]
        L.qg_dequant_int8.argtypes = [vp, vp, i64, i64, i32, vp, vp]
        L.qg_dequant_int4.argtypes = [vp, vp, i64, i64, i32, vp, vp]
        L.qg_project.argtypes = [vp, vp, vp, i64, i64, i64, i32, vp, vp, sz, vp]
        L.qg_lowrank_adam.argtypes = [vp, vp, vp, vp, i64, i64, C.POINTER(HParams), vp]
        L.qg_backproject_update_sr.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i32, f32, f32, u64, i64, vp, vp]
        L.qg_quant_int8_zp.argtypes = [vp, i64, i64, i32, vp, vp, vp, vp]
        L.qg_dequant_int8_zp.argtypes = [vp, vp, vp, i64, i64, i32, vp, vp]
        L.qg_backproject_update_sr_zp.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, f32, f32, u64, i64, vp]
        L.qg_step_zp.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, C.POINTER(HParams), u64,
                                 i64, vp]
        L.qg_int8_linear_zp_forward.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i32, vp, vp]
        L.qg_int8_linear_zp_backward.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i32, vp, vp, vp]
        L.qg_int8_linear_t_zp_forward.argtypes = L.qg_int8_linear_zp_forward.argtypes
        L.qg_int8_linear_t_zp_backward.argtypes = L.qg_int8_linear_zp_backward.argtypes
        L.qg_cossim_workspace_bytes.restype = sz
        L.qg_cossim_workspace_bytes.argtypes = [i64, i64]
        L.qg_subspace_cossim.argtypes = [vp, vp, vp, vp, i64, i64, i32, vp, vp, sz, vp]
        L.qg_subspace_cossim_static.argtypes = [vp, vp, vp, vp, i64, i64, i32, vp, vp]
        L.qg_subspace_cossim_weighted.argtypes = [vp, vp, vp, vp, vp, i64, i64, i32, vp, vp, sz, vp]
        L.qg_step_ld.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i32, C.POINTER(HParams), u64, i64,
                                 vp]
        L.qg_policy_update.argtypes = [C.POINTER(Policy), f32]
        L.qg_workspace_bytes.restype = sz
        L.qg_workspace_bytes.argtypes = [i64, i64, i64]
        L.qg_step.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, C.POINTER(HParams), u64, i64,
                              vp, sz, vp]
        L.qg_plan_bytes.restype = sz
        L.qg_plan_bytes.argtypes = [i32, C.POINTER(MatrixDesc)]
        L.qg_plan_build.argtypes = [i32, C.POINTER(MatrixDesc), vp, sz]
        L.qg_step_many.argtypes = [i32, vp, vp, sz, C.POINTER(HParams), u64, i64, vp]
        L.qg_sr_uniform.argtypes = [u64, i64, u64, i64, vp, vp]
        L.qg_project_many.argtypes = [i32, vp, vp, sz, vp]
        L.qg_lowrank_adam_many.argtypes = [i32, vp, vp, sz, C.POINTER(HParams), i64, vp]
        L.qg_backproject_update_sr_many.argtypes = [i32, vp, vp, sz, C.POINTER(HParams), u64, i64, vp]
        L.qg_project_adam.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, i64, C.POINTER(HParams), vp]
        L.qg_project_adam_many.argtypes = [i32, vp, vp, sz, C.POINTER(HParams), i64, i32, vp]
        L.qg_diag_clock_probe.argtypes = [i64, vp, vp]
        L.qg_diag_mfma_loop.argtypes = [i64, i32, vp, vp]
        L.qg_diag_mfma_f64_loop.argtypes = [i64, i32, vp, vp]
        L.qg_range_apply.argtypes = [vp, vp, i64, i64, i64, vp, vp]
        L.qg_orthonormalize_workspace_bytes.restype = sz
        L.qg_orthonormalize_workspace_bytes.argtypes = [i64, i64]
        L.qg_orthonormalize.argtypes = [vp, i64, i64, vp, vp, vp, sz, vp]
        L.qg_refresh_workspace_bytes.restype = sz
        L.qg_refresh_workspace_bytes.argtypes = [i32, i64, i64, i64]
        L.qg_subspace_refresh.argtypes = [vp, vp, vp, i64, i64, i64, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.qg_state8_quant.argtypes = [vp, i64, i32, vp, vp, vp]
        L.qg_state8_dequant.argtypes = [vp, vp, i64, i32, vp, vp]
        L.qg_lowrank_adam8.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, C.POINTER(HParams), vp]
        L.qg_step8.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, C.POINTER(HParams), u64, i64, vp]
        L.qg_int8_linear_forward.argtypes = [vp, vp, vp, vp, i64, i64, i64, i32, vp, vp]
        L.qg_int8_linear_backward.argtypes = [vp, vp, vp, vp, i64, i64, i64, i32, vp, vp, vp]
        L.qg_int8_linear_forward_ld.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i32, vp, vp]
        L.qg_int8_linear_backward_ld.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i32, vp, vp, vp]
        L.qg_int8_linear_t_forward.argtypes = L.qg_int8_linear_forward.argtypes
        L.qg_int8_linear_t_backward.argtypes = L.qg_int8_linear_backward.argtypes
        L.qg_subspace_refresh_many.argtypes = [i32, C.POINTER(RefreshDesc), i64, i64, i64, i32, i32, vp, vp, vp, sz, vp]
        L.qg_subspace_refresh_many_ld.argtypes = [i32, C.POINTER(RefreshDesc), i64, i64, i64, i64, i32, i32, vp, vp, vp, sz,
                                                  vp]
        L.qg_residual_norm_forward.argtypes = [vp, vp, vp, vp, i32, vp, f32, f32, i64, i64, i64, i32, vp, vp, vp]
        L.qg_residual_norm_workspace_bytes.restype = sz
        L.qg_residual_norm_workspace_bytes.argtypes = [i64, i64]
        L.qg_residual_norm_backward.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp, f32, f32, i64, i64, i64, i32, vp, vp, vp, vp, vp,
                                                vp, sz, vp]
        L.qg_int8_linear_act_forward.argtypes = [vp] * 5 + [i32, i64, i64, i64, i64, i64, i32, vp, vp, vp]
        L.qg_int8_linear_act_workspace_bytes.restype = sz
        L.qg_int8_linear_act_workspace_bytes.argtypes = [i64, i64, i64]
        L.qg_int8_linear_act_backward.argtypes = [vp] * 5 + [i32, i64, i64, i64, i64, i64, i32, vp, vp, vp, vp, sz, vp]
        L.qg_int8_gated_forward.argtypes = [vp] * 5 + [i32, i64, i64, i64, i64, i64, i32, vp, vp, vp, vp]
        L.qg_int8_gated_workspace_bytes.restype = sz
        L.qg_int8_gated_workspace_bytes.argtypes = [i64, i64, i64]
        L.qg_int8_gated_backward.argtypes = [vp] * 8 + [i32, i64, i64, i64, i64, i64, i32, vp, vp, vp, vp, sz, vp]
        L.qg_head_loss_workspace_bytes.restype = sz
        L.qg_head_loss_workspace_bytes.argtypes = [i64, i64, i64]
        L.qg_head_loss_forward.argtypes = [vp, vp, vp, i64, i64, i64, i64, vp, vp, vp, sz, vp]
        L.qg_head_loss_backward.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, vp, vp, vp, sz, vp]
        heads = attention = cache = vp          # their bytes
        f64 = C.c_double
        L.qg_rope_frequencies.argtypes = [i32, f64, f64, f64, f64, f64, vp]
        L.qg_rope_forward.argtypes = [heads, i32, heads, i32, vp, vp, i64, i32, i32, i32, f32, heads, heads, vp]
        L.qg_rope_backward.argtypes = L.qg_rope_forward.argtypes
        for f in (L.qg_attention_forward_workspace_bytes, L.qg_attention_backward_workspace_bytes):
            f.restype, f.argtypes = sz, [attention]
        L.qg_attention_forward.argtypes = [attention, heads, heads, heads, heads, vp, vp, sz, vp]
        L.qg_attention_backward.argtypes = [attention] + [heads] * 5 + [vp] + [heads] * 3 + [vp, sz, vp]
        L.qg_cache_append.argtypes = [cache, heads, i32, heads, heads, vp, vp, i64, vp, i32, i32, f32, heads, vp]
        L.qg_attention_paged_workspace_bytes.restype = sz
        L.qg_attention_paged_workspace_bytes.argtypes = [cache, i32]
        L.qg_attention_paged.argtypes = [cache, vp, heads, i32, f32, f32, i64, vp, heads, vp, sz, vp]
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != 0:
        L = lib()
        msg = L.qg_status_string(status).decode()
        if status == 6:
            msg += f" (hipError {L.qg_last_hip_error()})"
        raise QGError(f"libqgalore: {msg}")


def _ptr(t: torch.Tensor | None, dtypes=None) -> int | None:
    if t is None:
        return None
    if not t.is_cuda:
        raise QGError("device tensor expected")
    if not t.is_contiguous():
        raise QGError("contiguous tensor expected")
    if dtypes is not None and t.dtype not in dtypes:
        raise QGError(f"dtype {t.dtype} not in {dtypes}")
    return t.data_ptr()


def _stream() -> int:
    # (without the Stream object of torch.cuda.current_stream(): 0.3 us instead of 2.8 of the 10 a small call takes)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


_BF16 = (torch.bfloat16, torch.int16, torch.uint16)
_F32 = (torch.float32,)


def _bf16_rows(like: torch.Tensor, rows: int, cols: int) -> torch.Tensor:
    """A new bf16 [rows][cols] where `like` is.  (us on a host where the call of a small layer takes 8: sizes as a tuple 3.9, as
    arguments 2.0, new_empty 1.3, which gives a subclass's type for a subclass.)"""
    if like.dtype is torch.bfloat16 and type(like) is torch.Tensor:
        return like.new_empty(rows, cols)
    return torch.empty(rows, cols, dtype=torch.bfloat16, device=like.device)


def _expect(t: torch.Tensor | None, *shape: int) -> None:
    """Refuses a tensor of another shape than the sizes handed to the library say: its kernels would read past the end."""
    if t is not None and t.shape != shape:
        raise QGError(f"shape {tuple(t.shape)}, expected {shape}")


def hparams(beta1=0.9, beta2=0.999, eps=1e-8, lr=1e-3, alpha=0.25) -> HParams:
    return HParams(beta1, beta2, eps, lr, alpha)


# ---------------------------------------------------------------- quantizers
def quant_int8(x: torch.Tensor):
    rows, cols = x.shape
    q = torch.empty(rows, cols, dtype=torch.int8, device=x.device)
    s = torch.empty((rows, (cols + GROUP - 1) // GROUP), dtype=torch.float32, device=x.device)
    _check(lib().qg_quant_int8(_ptr(x, (torch.float32,)), rows, cols, GROUP, _ptr(q), _ptr(s), _stream()))
    return q, s


def quant_int4(x: torch.Tensor):
    rows, cols = x.shape
    total = rows * cols
    q = torch.empty(((total + 1) // 2,), dtype=torch.uint8, device=x.device)
    s = torch.empty(((total + GROUP - 1) // GROUP,), dtype=torch.float32, device=x.device)
    _check(lib().qg_quant_int4(_ptr(x, (torch.float32,)), rows, cols, GROUP, _ptr(q), _ptr(s), _stream()))
    return q, s


def dequant_int8(q: torch.Tensor, s: torch.Tensor) -> torch.Tensor:
    rows, cols = q.shape
    x = torch.empty(rows, cols, dtype=torch.float32, device=q.device)
    _check(lib().qg_dequant_int8(_ptr(q, (torch.int8,)), _ptr(s, (torch.float32,)), rows, cols, GROUP, _ptr(x),
                                 _stream()))
    return x


def dequant_int4(q: torch.Tensor, s: torch.Tensor, rows: int, cols: int) -> torch.Tensor:
    x = torch.empty(rows, cols, dtype=torch.float32, device=q.device)
    _check(lib().qg_dequant_int4(_ptr(q, (torch.uint8,)), _ptr(s, (torch.float32,)), rows, cols, GROUP, _ptr(x),
                                 _stream()))
    return x


# ---------------------------------------------------------------- step pieces
def project(Pq, Ps, G, m: int, n: int, r: int, R: torch.Tensor | None = None) -> torch.Tensor:
    if R is None:
        R = torch.empty(r, n, dtype=torch.float32, device=G.device)
    _check(lib().qg_project(_ptr(Pq, (torch.uint8,)), _ptr(Ps, (torch.float32,)), _ptr(G, _BF16), m, n, r, GROUP,
                            _ptr(R, (torch.float32,)), None, 0, _stream()))
    return R


def lowrank_adam(R, M, V, N, step: int, hp: HParams) -> None:
    _check(lib().qg_lowrank_adam(_ptr(R, (torch.float32,)), _ptr(M, (torch.float32,)), _ptr(V, (torch.float32,)),
                                 _ptr(N, _BF16), R.numel(), step, C.byref(hp), _stream()))


def project_adam(Pq, Ps, G, R, M, V, N, m: int, n: int, r: int, step: int, hp: HParams) -> None:
    _check(lib().qg_project_adam(_ptr(Pq, (torch.uint8,)), _ptr(Ps, (torch.float32,)), _ptr(G, _BF16),
                                 _ptr(R, (torch.float32,)), _ptr(M, (torch.float32,)), _ptr(V, (torch.float32,)),
                                 _ptr(N, _BF16), m, n, r, GROUP, step, C.byref(hp), _stream()))


def backproject_update_sr(Pq, Ps, N, Wq, Ws, m: int, n: int, r: int, alpha: float, lr: float, seed: int, step: int,
                          U_debug: torch.Tensor | None = None) -> None:
    _check(lib().qg_backproject_update_sr(_ptr(Pq, (torch.uint8,)), _ptr(Ps, (torch.float32,)), _ptr(N, _BF16),
                                          _ptr(Wq, (torch.int8,)), _ptr(Ws, (torch.float32,)), m, n, r, GROUP,
                                          alpha, lr, seed, step, _ptr(U_debug, (torch.float32,)), _stream()))


def subspace_cossim(PqA, PsA, PqB, PsB, m: int, r: int, weights: torch.Tensor | None = None) -> torch.Tensor:
    """qg_subspace_cossim, or qg_subspace_cossim_weighted when `weights` (fp32 [r]) is given."""
    nbytes = lib().qg_cossim_workspace_bytes(m, r)
    ws = torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=PqA.device)
    out = torch.empty(1, dtype=torch.float32, device=PqA.device)
    if weights is None:
        _check(lib().qg_subspace_cossim(_ptr(PqA, (torch.uint8,)), _ptr(PsA, (torch.float32,)), _ptr(PqB, (torch.uint8,)),
                                        _ptr(PsB, (torch.float32,)), m, r, GROUP, _ptr(out), _ptr(ws), nbytes, _stream()))
    else:
        _check(lib().qg_subspace_cossim_weighted(_ptr(PqA, (torch.uint8,)), _ptr(PsA, (torch.float32,)),
                                                 _ptr(PqB, (torch.uint8,)), _ptr(PsB, (torch.float32,)),
                                                 _ptr(weights, (torch.float32,)), m, r, GROUP, _ptr(out), _ptr(ws),
                                                 nbytes, _stream()))
    return out


def subspace_cossim_static(PqA, PsA, PqB, PsB, m: int, r: int, out: torch.Tensor) -> None:
    """qg_subspace_cossim_static: no workspace; `out` is the caller's one-float device tensor."""
    _check(lib().qg_subspace_cossim_static(_ptr(PqA, (torch.uint8,)), _ptr(PsA, (torch.float32,)),
                                           _ptr(PqB, (torch.uint8,)), _ptr(PsB, (torch.float32,)), m, r, GROUP,
                                           _ptr(out, (torch.float32,)), _stream()))


def policy_update(p: Policy, cos: float) -> bool:
    rc = lib().qg_policy_update(C.byref(p), cos)
    if rc < 0:
        raise QGError("libqgalore: null policy")
    return bool(rc)


def step(Pq, Ps, G, Wq, Ws, M, V, R, N, m: int, n: int, r: int, hp: HParams, seed: int, step: int) -> None:
    _check(lib().qg_step(_ptr(Pq, (torch.uint8,)), _ptr(Ps, (torch.float32,)), _ptr(G, _BF16),
                         _ptr(Wq, (torch.int8,)), _ptr(Ws, (torch.float32,)), _ptr(M, (torch.float32,)),
                         _ptr(V, (torch.float32,)), _ptr(R, (torch.float32,)), _ptr(N, _BF16), m, n, r, GROUP,
                         C.byref(hp), seed, step, None, 0, _stream()))


def step_ld(Pq, Ps, G, Wq, Ws, M, V, R, N, m: int, n: int, ld: int, r: int, hp: HParams, seed: int, step: int) -> None:
    """qg_step_ld: every n-wide array is stored with rows ld elements apart."""
    _check(lib().qg_step_ld(_ptr(Pq, (torch.uint8,)), _ptr(Ps, (torch.float32,)), _ptr(G, _BF16),
                            _ptr(Wq, (torch.int8,)), _ptr(Ws, (torch.float32,)), _ptr(M, (torch.float32,)),
                            _ptr(V, (torch.float32,)), _ptr(R, (torch.float32,)), _ptr(N, _BF16), m, n, ld, r, GROUP,
                            C.byref(hp), seed, step, _stream()))


@dataclass
class MatrixState:
    """Device tensors of one weight matrix, as passed to qg_step / qg_step_many."""
    m: int
    n: int
    r: int
    Pq: torch.Tensor
    Ps: torch.Tensor
    G: torch.Tensor
    Wq: torch.Tensor
    Ws: torch.Tensor
    M: torch.Tensor
    V: torch.Tensor
    R: torch.Tensor | None
    N: torch.Tensor
    ld: int = 0   # row pitch in elements of G, Wq, M, V, R, N; 0 = n
    Wz: torch.Tensor | None = None   # zero points of W (all matrices of a plan, or none)


class StepPlan:
    """Host + device copies of the grouped-launch plan of qg_step_many."""

    def __init__(self, mats: list[MatrixState]):
        self.count = len(mats)
        self.mats = mats
        descs = (MatrixDesc * self.count)()
        for d, s in zip(descs, mats):
            d.m, d.n, d.r = s.m, s.n, s.r
            d.Pq, d.Ps, d.G = _ptr(s.Pq, (torch.uint8,)), _ptr(s.Ps, (torch.float32,)), _ptr(s.G, _BF16)
            d.Wq, d.Ws = _ptr(s.Wq, (torch.int8,)), _ptr(s.Ws, (torch.float32,))
            d.M, d.V, d.R = _ptr(s.M, (torch.float32,)), _ptr(s.V, (torch.float32,)), _ptr(s.R, (torch.float32,))
            d.N = _ptr(s.N, _BF16)
            d.ld = s.ld
            d.Wz = _ptr(s.Wz, (torch.float32,))
        self.nbytes = lib().qg_plan_bytes(self.count, descs)
        self.host = torch.empty((self.nbytes,), dtype=torch.uint8).pin_memory()
        _check(lib().qg_plan_build(self.count, descs, self.host.data_ptr(), self.nbytes))
        self.dev = self.host.to(mats[0].Wq.device)


def step_many(plan: StepPlan, hp: HParams, seed: int, step: int) -> None:
    _check(lib().qg_step_many(plan.count, plan.host.data_ptr(), plan.dev.data_ptr(), plan.nbytes, C.byref(hp), seed,
                              step, _stream()))


def project_many(plan: StepPlan) -> None:
    _check(lib().qg_project_many(plan.count, plan.host.data_ptr(), plan.dev.data_ptr(), plan.nbytes, _stream()))


def lowrank_adam_many(plan: StepPlan, hp: HParams, step: int) -> None:
    _check(lib().qg_lowrank_adam_many(plan.count, plan.host.data_ptr(), plan.dev.data_ptr(), plan.nbytes,
                                      C.byref(hp), step, _stream()))


def project_adam_many(plan: StepPlan, hp: HParams, step: int, write_R: bool = False) -> None:
    _check(lib().qg_project_adam_many(plan.count, plan.host.data_ptr(), plan.dev.data_ptr(), plan.nbytes,
                                      C.byref(hp), step, int(write_R), _stream()))


def backproject_update_sr_many(plan: StepPlan, hp: HParams, seed: int, step: int) -> None:
    _check(lib().qg_backproject_update_sr_many(plan.count, plan.host.data_ptr(), plan.dev.data_ptr(), plan.nbytes,
                                               C.byref(hp), seed, step, _stream()))


# ---------------------------------------------------------------- zero-point (asymmetric) INT8 weights
def quant_int8_zp(x: torch.Tensor):
    rows, cols = x.shape
    q = torch.empty(rows, cols, dtype=torch.int8, device=x.device)
    s = torch.empty((rows, (cols + GROUP - 1) // GROUP), dtype=torch.float32, device=x.device)
    z = torch.empty_like(s)
    _check(lib().qg_quant_int8_zp(_ptr(x, (torch.float32,)), rows, cols, GROUP, _ptr(q), _ptr(s), _ptr(z), _stream()))
    return q, s, z


def dequant_int8_zp(q: torch.Tensor, s: torch.Tensor, z: torch.Tensor) -> torch.Tensor:
    rows, cols = q.shape
    x = torch.empty(rows, cols, dtype=torch.float32, device=q.device)
    _check(lib().qg_dequant_int8_zp(_ptr(q, (torch.int8,)), _ptr(s, (torch.float32,)), _ptr(z, (torch.float32,)), rows,
                                    cols, GROUP, _ptr(x), _stream()))
    return x


def backproject_update_sr_zp(Pq, Ps, N, Wq, Ws, Wz, m: int, n: int, r: int, alpha: float, lr: float, seed: int,
                             step: int) -> None:
    _check(lib().qg_backproject_update_sr_zp(_ptr(Pq, (torch.uint8,)), _ptr(Ps, (torch.float32,)), _ptr(N, _BF16),
                                             _ptr(Wq, (torch.int8,)), _ptr(Ws, (torch.float32,)),
                                             _ptr(Wz, (torch.float32,)), m, n, r, GROUP, alpha, lr, seed, step, _stream()))


def step_zp(Pq, Ps, G, Wq, Ws, Wz, M, V, R, N, m: int, n: int, r: int, hp: HParams, seed: int, step: int) -> None:
    _check(lib().qg_step_zp(_ptr(Pq, (torch.uint8,)), _ptr(Ps, (torch.float32,)), _ptr(G, _BF16),
                            _ptr(Wq, (torch.int8,)), _ptr(Ws, (torch.float32,)), _ptr(Wz, (torch.float32,)),
                            _ptr(M, (torch.float32,)), _ptr(V, (torch.float32,)), _ptr(R, (torch.float32,)),
                            _ptr(N, _BF16), m, n, r, GROUP, C.byref(hp), seed, step, _stream()))


def int8_linear_zp_forward(x: torch.Tensor, Wq: torch.Tensor, Ws: torch.Tensor, Wz: torch.Tensor,
                           bias: torch.Tensor | None = None):
    tokens, n = x.shape
    m = Wq.shape[0]
    y = _bf16_rows(x, tokens, m)
    _check(lib().qg_int8_linear_zp_forward(_ptr(x, _BF16), _ptr(Wq, (torch.int8,)), _ptr(Ws, (torch.float32,)),
                                           _ptr(Wz, (torch.float32,)), _ptr(bias, _BF16), tokens, m, n, GROUP,
                                           _ptr(y), _stream()))
    return y


def int8_linear_zp_backward(dy: torch.Tensor, x: torch.Tensor | None, Wq, Ws, Wz, m: int, n: int,
                            want_dx: bool = True, want_G: bool = True):
    tokens = dy.shape[0]
    dx = _bf16_rows(dy, tokens, n) if want_dx else None
    G = _bf16_rows(dy, m, n) if want_G else None
    _check(lib().qg_int8_linear_zp_backward(_ptr(dy, _BF16), _ptr(x, _BF16), _ptr(Wq, (torch.int8,)),
                                            _ptr(Ws, (torch.float32,)), _ptr(Wz, (torch.float32,)), tokens, m, n, GROUP,
                                            _ptr(dx), _ptr(G), _stream()))
    return dx, G


def int8_linear_t_zp_forward(x: torch.Tensor, Sq: torch.Tensor, Ss: torch.Tensor, Sz: torch.Tensor,
                             bias: torch.Tensor | None = None):
    """Zero-point weight stored transposed (Sq: [n][m])."""
    tokens, n = x.shape
    m = Sq.shape[1]
    y = _bf16_rows(x, tokens, m)
    _check(lib().qg_int8_linear_t_zp_forward(_ptr(x, _BF16), _ptr(Sq, (torch.int8,)), _ptr(Ss, (torch.float32,)),
                                             _ptr(Sz, (torch.float32,)), _ptr(bias, _BF16), tokens, m, n, GROUP,
                                             _ptr(y), _stream()))
    return y


def int8_linear_t_zp_backward(dy: torch.Tensor, x: torch.Tensor | None, Sq, Ss, Sz, m: int, n: int,
                              want_dx: bool = True, want_G: bool = True):
    tokens = dy.shape[0]
    dx = _bf16_rows(dy, tokens, n) if want_dx else None
    G = _bf16_rows(dy, n, m) if want_G else None
    _check(lib().qg_int8_linear_t_zp_backward(_ptr(dy, _BF16), _ptr(x, _BF16), _ptr(Sq, (torch.int8,)),
                                              _ptr(Ss, (torch.float32,)), _ptr(Sz, (torch.float32,)), tokens, m, n,
                                              GROUP, _ptr(dx), _ptr(G), _stream()))
    return dx, G


# ---------------------------------------------------------------- 8-bit Adam states
def state8_quant(x: torch.Tensor, signed: bool):
    count = x.numel()
    codes = torch.empty(count, dtype=torch.uint8, device=x.device)
    scales = torch.empty(((count + GROUP - 1) // GROUP,), dtype=torch.float32, device=x.device)
    _check(lib().qg_state8_quant(_ptr(x, (torch.float32,)), count, int(signed), _ptr(codes), _ptr(scales), _stream()))
    return codes, scales


def state8_dequant(codes: torch.Tensor, scales: torch.Tensor, signed: bool) -> torch.Tensor:
    x = torch.empty((codes.numel(),), dtype=torch.float32, device=codes.device)
    _check(lib().qg_state8_dequant(_ptr(codes, (torch.uint8,)), _ptr(scales, (torch.float32,)), codes.numel(),
                                   int(signed), _ptr(x), _stream()))
    return x


def lowrank_adam8(R, Mq, Ms, Vq, Vs, N, step: int, hp: HParams) -> None:
    _check(lib().qg_lowrank_adam8(_ptr(R, (torch.float32,)), _ptr(Mq, (torch.uint8,)), _ptr(Ms, (torch.float32,)),
                                  _ptr(Vq, (torch.uint8,)), _ptr(Vs, (torch.float32,)), _ptr(N, _BF16), R.numel(), step,
                                  C.byref(hp), _stream()))


def step8(Pq, Ps, G, Wq, Ws, Mq, Ms, Vq, Vs, R, N, m: int, n: int, r: int, hp: HParams, seed: int, step: int) -> None:
    _check(lib().qg_step8(_ptr(Pq, (torch.uint8,)), _ptr(Ps, (torch.float32,)), _ptr(G, _BF16), _ptr(Wq, (torch.int8,)),
                          _ptr(Ws, (torch.float32,)), _ptr(Mq, (torch.uint8,)), _ptr(Ms, (torch.float32,)),
                          _ptr(Vq, (torch.uint8,)), _ptr(Vs, (torch.float32,)), _ptr(R, (torch.float32,)), _ptr(N, _BF16),
                          m, n, r, GROUP, C.byref(hp), seed, step, _stream()))


# ---------------------------------------------------------------- INT8 linear layer
def int8_linear_forward(x: torch.Tensor, Wq: torch.Tensor, Ws: torch.Tensor, bias: torch.Tensor | None = None):
    tokens, n = x.shape
    m = Wq.shape[0]
    y = _bf16_rows(x, tokens, m)
    _check(lib().qg_int8_linear_forward(_ptr(x, _BF16), _ptr(Wq, (torch.int8,)), _ptr(Ws, (torch.float32,)),
                                        _ptr(bias, _BF16), tokens, m, n, GROUP, _ptr(y), _stream()))
    return y


def int8_linear_backward(dy: torch.Tensor, x: torch.Tensor | None, Wq: torch.Tensor | None, Ws: torch.Tensor | None,
                         m: int, n: int, want_dx: bool = True, want_G: bool = True):
    tokens = dy.shape[0]
    dx = _bf16_rows(dy, tokens, n) if want_dx else None
    G = _bf16_rows(dy, m, n) if want_G else None
    _check(lib().qg_int8_linear_backward(_ptr(dy, _BF16), _ptr(x, _BF16), _ptr(Wq, (torch.int8,)),
                                         _ptr(Ws, (torch.float32,)), tokens, m, n, GROUP, _ptr(dx), _ptr(G), _stream()))
    return dx, G


def int8_linear_forward_ld(x, Wq, Ws, bias, tokens: int, m: int, n: int, ld_n: int, ld_m: int, y: torch.Tensor) -> None:
    """qg_int8_linear_forward_ld: x [tokens][ld_n], Wq [m][ld_n], y [tokens][ld_m] (the caller's, padding untouched)."""
    _check(lib().qg_int8_linear_forward_ld(_ptr(x, _BF16), _ptr(Wq, (torch.int8,)), _ptr(Ws, (torch.float32,)),
                                           _ptr(bias, _BF16), tokens, m, n, ld_n, ld_m, GROUP, _ptr(y, _BF16), _stream()))


def int8_linear_backward_ld(dy, x, Wq, Ws, tokens: int, m: int, n: int, ld_n: int, ld_m: int, dx, G) -> None:
    """qg_int8_linear_backward_ld: dy [tokens][ld_m], x and dx [tokens][ld_n], Wq and G [m][ld_n]; dx or G may be None."""
    _check(lib().qg_int8_linear_backward_ld(_ptr(dy, _BF16), _ptr(x, _BF16), _ptr(Wq, (torch.int8,)),
                                            _ptr(Ws, (torch.float32,)), tokens, m, n, ld_n, ld_m, GROUP,
                                            _ptr(dx, _BF16), _ptr(G, _BF16), _stream()))


def int8_linear_t_forward(x: torch.Tensor, Sq: torch.Tensor, Ss: torch.Tensor, bias: torch.Tensor | None = None):
    """The layer on a weight stored transposed (Sq: [n][m])."""
    tokens, n = x.shape
    m = Sq.shape[1]
    y = _bf16_rows(x, tokens, m)
    _check(lib().qg_int8_linear_t_forward(_ptr(x, _BF16), _ptr(Sq, (torch.int8,)), _ptr(Ss, (torch.float32,)),
                                          _ptr(bias, _BF16), tokens, m, n, GROUP, _ptr(y), _stream()))
    return y


def int8_linear_t_backward(dy: torch.Tensor, x: torch.Tensor | None, Sq: torch.Tensor | None, Ss: torch.Tensor | None,
                           m: int, n: int, want_dx: bool = True, want_G: bool = True):
    """Returns (dx [tokens][n], G_S [n][m]) for a weight stored transposed."""
    tokens = dy.shape[0]
    dx = _bf16_rows(dy, tokens, n) if want_dx else None
    G = _bf16_rows(dy, n, m) if want_G else None
    _check(lib().qg_int8_linear_t_backward(_ptr(dy, _BF16), _ptr(x, _BF16), _ptr(Sq, (torch.int8,)),
                                           _ptr(Ss, (torch.float32,)), tokens, m, n, GROUP, _ptr(dx), _ptr(G), _stream()))
    return dx, G


# ---------------------------------------------------------------- INT8 linear layer with an epilogue
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
_I8 = (torch.int8,)


def _act(name: str) -> int:
    if name not in ACTIVATIONS:
        raise QGError(f"activation {name!r} is none of {sorted(ACTIVATIONS)}")
    return ACTIVATIONS[name]


def _weight(q: torch.Tensor | None, s: torch.Tensor | None, m: int, n: int):
    """Pointers to the codes and scales of an m x n weight."""
    _expect(q, m, n)
    _expect(s, m, (n + GROUP - 1) // GROUP)
    return _ptr(q, _I8), _ptr(s, _F32)


def int8_linear_act_forward(x: torch.Tensor, Wq: torch.Tensor, Ws: torch.Tensor, bias: torch.Tensor | None = None,
                            residual: torch.Tensor | None = None, act: str = "none", want_z: bool = False):
    """Returns (y, z): z = x W^T + bias, y = act(z) + residual; z is None unless want_z."""
    tokens, n = x.shape
    m = Wq.shape[0]
    _expect(bias, m)
    _expect(residual, tokens, m)
    w = _weight(Wq, Ws, m, n)
    y = _bf16_rows(x, tokens, m)
    z = _bf16_rows(x, tokens, m) if want_z else None
    _check(lib().qg_int8_linear_act_forward(_ptr(x, _BF16), *w, _ptr(bias, _BF16), _ptr(residual, _BF16), _act(act), tokens, m, n, n, m,
                                            GROUP, _ptr(z), _ptr(y), _stream()))
    return y, z


def _inputs_of(x: torch.Tensor | None, Wq: torch.Tensor | None) -> int:
    """n, from what a backward pass was given: x may be missing where no G is wanted, the weight where no dx is."""
    return x.shape[1] if x is not None else Wq.shape[1] if Wq is not None else 1


def int8_linear_act_backward(dy: torch.Tensor, z: torch.Tensor | None, x: torch.Tensor | None, Wq: torch.Tensor | None,
                             Ws: torch.Tensor | None, act: str = "none", want_dx: bool = True, want_G: bool = True,
                             want_dbias: bool = False):
    """Returns (dx, G, dbias) of int8_linear_act_forward (None where not wanted); the residual's gradient is dy itself.  z is not
    needed without an activation, x not without G, the weight not without dx."""
    tokens, m = dy.shape
    n = _inputs_of(x, Wq)
    kind = _act(act)
    _expect(x, tokens, n)
    _expect(z, tokens, m)
    w = _weight(Wq, Ws, m, n)
    dx = _bf16_rows(dy, tokens, n) if want_dx else None
    G = _bf16_rows(dy, m, n) if want_G else None
    dbias = dy.new_empty(m, dtype=torch.float32) if want_dbias else None
    ws = None
    nbytes = 0
    if want_dbias or kind:
        nbytes = lib().qg_int8_linear_act_workspace_bytes(tokens, m, n)
        ws = dy.new_empty(nbytes, dtype=torch.uint8)
    _check(lib().qg_int8_linear_act_backward(_ptr(dy, _BF16), _ptr(z, _BF16), _ptr(x, _BF16), *w, kind, tokens, m, n, n, m, GROUP,
                                             _ptr(dx), _ptr(G), _ptr(dbias), _ptr(ws), nbytes, _stream()))
    return dx, G, dbias


def int8_gated_forward(x: torch.Tensor, Wgq: torch.Tensor, Wgs: torch.Tensor, Wuq: torch.Tensor, Wus: torch.Tensor, act: str = "silu",
                       want_z: bool = False):
    """Returns (y, zg, zu): y = act(x Wg^T) * (x Wu^T); zg and zu, which the backward pass takes, are None unless want_z."""
    tokens, n = x.shape
    m = Wgq.shape[0]
    w = _weight(Wgq, Wgs, m, n) + _weight(Wuq, Wus, m, n)
    y = _bf16_rows(x, tokens, m)
    zg, zu = (_bf16_rows(x, tokens, m), _bf16_rows(x, tokens, m)) if want_z else (None, None)
    _check(lib().qg_int8_gated_forward(_ptr(x, _BF16), *w, _act(act), tokens, m, n, n, m, GROUP, _ptr(zg), _ptr(zu), _ptr(y), _stream()))
    return y, zg, zu


def int8_gated_backward(dy: torch.Tensor, zg: torch.Tensor, zu: torch.Tensor, x: torch.Tensor | None, Wgq: torch.Tensor | None,
                        Wgs: torch.Tensor | None, Wuq: torch.Tensor | None, Wus: torch.Tensor | None, act: str = "silu",
                        want_dx: bool = True, want_G: bool = True):
    """Returns (dx, Gg, Gu) of int8_gated_forward (None where not wanted).  x is not needed without Gg and Gu, the weights not
    without dx."""
    tokens, m = dy.shape
    n = _inputs_of(x, Wgq)
    _expect(x, tokens, n)
    for v in (zg, zu):
        _expect(v, tokens, m)
    w = _weight(Wgq, Wgs, m, n) + _weight(Wuq, Wus, m, n)
    dx = _bf16_rows(dy, tokens, n) if want_dx else None
    Gg, Gu = (_bf16_rows(dy, m, n), _bf16_rows(dy, m, n)) if want_G else (None, None)
    nbytes = lib().qg_int8_gated_workspace_bytes(tokens, m, n)
    ws = dy.new_empty(nbytes, dtype=torch.uint8)
    _check(lib().qg_int8_gated_backward(_ptr(dy, _BF16), _ptr(zg, _BF16), _ptr(zu, _BF16), _ptr(x, _BF16), *w, _act(act), tokens, m, n, n,
                                        m, GROUP, _ptr(dx), _ptr(Gg), _ptr(Gu), _ptr(ws), nbytes, _stream()))
    return dx, Gg, Gu


# ---------------------------------------------------------------- residual stream
GATE_NONE, GATE_CHANNEL, GATE_TOKEN = 0, 1, 2


def _gate(gate: torch.Tensor | None, tokens: int, d: int):
    """(pointer, kind) of a gate: None, fp32 [d] or bf16 [tokens][d]."""
    if gate is None:
        return None, GATE_NONE
    if gate.dim() == 1:
        _expect(gate, d)
        return _ptr(gate, _F32), GATE_CHANNEL
    _expect(gate, tokens, d)
    return _ptr(gate, _BF16), GATE_TOKEN


def _stream_type(h: torch.Tensor):
    if h.dtype is torch.float32:
        return _F32, 1
    return _BF16, 0


def residual_norm_forward(h: torch.Tensor, y: torch.Tensor | None = None, w_post: torch.Tensor | None = None,
                          gate: torch.Tensor | None = None, w_pre: torch.Tensor | None = None, scale: float = 1.0,
                          eps: float = 1e-6, out: torch.Tensor | None = None):
    """Returns (h', u): h' = h + scale * gate * norm(y; w_post), u = norm(h'; w_pre).  h: bf16 or fp32 [tokens][d], gate: None, fp32
    [d] or bf16 [tokens][d].  Without y, h' is h itself; without w_pre, u is None.  out: where h' is written (h itself: in place);
    without y nothing is, and another out than h is refused."""
    tokens, d = h.shape
    stype, fp32 = _stream_type(h)
    for v in (w_post, w_pre):
        _expect(v, d)
    _expect(y, tokens, d)
    g, kind = _gate(gate if y is not None else None, tokens, d)
    if y is None:
        if out is not None and out.data_ptr() != h.data_ptr():
            raise QGError("out without y: h' is h itself, and is not written anywhere else")
        out = None
    elif out is None:
        out = torch.empty_like(h)
    _expect(out, tokens, d)
    u = _bf16_rows(h if y is None else y, tokens, d) if w_pre is not None else None
    _check(lib().qg_residual_norm_forward(_ptr(h, stype), _ptr(y, _BF16), _ptr(w_post, _F32), g, kind, _ptr(w_pre, _F32), scale, eps,
                                          tokens, d, d, fp32, _ptr(out, (h.dtype,)), _ptr(u), _stream()))
    return (h if out is None else out), u


def residual_norm_backward(du: torch.Tensor | None, dh_next: torch.Tensor | None, h_next: torch.Tensor, y: torch.Tensor | None = None,
                           w_post: torch.Tensor | None = None, gate: torch.Tensor | None = None, w_pre: torch.Tensor | None = None,
                           scale: float = 1.0, eps: float = 1e-6, out: torch.Tensor | None = None):
    """Returns (dh, dy, dw_pre, dw_post, dgate), None for what has no input: the gradients of residual_norm_forward at its h' =
    h_next, from du and the stream's gradient dh_next (either may be None).  out: where dh is written (dh_next itself: in place)."""
    tokens, d = h_next.shape
    stype, fp32 = _stream_type(h_next)
    for v in (w_post, w_pre):
        _expect(v, d)
    for v in (du, dh_next, y, out):
        _expect(v, tokens, d)
    if y is None:
        w_post = gate = None
    g, kind = _gate(gate, tokens, d)
    dh = torch.empty_like(h_next) if out is None else out
    dy = _bf16_rows(y, tokens, d) if y is not None else None
    dw_pre = torch.empty_like(w_pre) if du is not None and w_pre is not None else None
    dw_post = torch.empty_like(w_post) if w_post is not None else None
    dgate = torch.empty_like(gate) if gate is not None else None
    nbytes = lib().qg_residual_norm_workspace_bytes(tokens, d)
    ws = h_next.new_empty(nbytes, dtype=torch.uint8)
    _check(lib().qg_residual_norm_backward(_ptr(du, _BF16), _ptr(dh_next, stype), _ptr(h_next, stype), _ptr(y, _BF16),
                                           _ptr(w_post, _F32), g, kind, _ptr(w_pre, _F32), scale, eps, tokens, d, d, fp32,
                                           _ptr(dh, stype), _ptr(dy), _ptr(dw_pre), _ptr(dw_post), _ptr(dgate), _ptr(ws), nbytes,
                                           _stream()))
    return dh, dy, dw_pre, dw_post, dgate


# ---------------------------------------------------------------- loss of a language model's head
def _head(x: torch.Tensor, W: torch.Tensor, labels: torch.Tensor, workspace: torch.Tensor | None):
    (tokens, h), vocab = x.shape, W.shape[0]
    _expect(W, vocab, h)
    _expect(labels, tokens)
    if workspace is None:
        nbytes = lib().qg_head_loss_workspace_bytes(tokens, h, vocab)
        if nbytes == 0:
            raise QGError("libqgalore: shape out of range")
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
    return tokens, h, vocab, workspace


def head_loss_forward(x: torch.Tensor, W: torch.Tensor, labels: torch.Tensor, workspace: torch.Tensor | None = None):
    """Returns (loss, lse), fp32 [tokens]: cross entropy of softmax(x W^T) against int64 labels; outside [0, vocab): no loss, 0.
    workspace: uint8, qg_head_loss_workspace_bytes(tokens, h, vocab) of them (allocated if None)."""
    tokens, h, vocab, ws = _head(x, W, labels, workspace)
    loss = torch.empty(tokens, dtype=torch.float32, device=x.device)
    lse = torch.empty(tokens, dtype=torch.float32, device=x.device)
    _check(lib().qg_head_loss_forward(_ptr(x, _BF16), _ptr(W, _BF16), _ptr(labels, (torch.int64,)), tokens, h, vocab, h, _ptr(loss),
                                      _ptr(lse), _ptr(ws, (torch.uint8,)), ws.numel(), _stream()))
    return loss, lse


def head_loss_backward(x: torch.Tensor, W: torch.Tensor, labels: torch.Tensor, lse: torch.Tensor, dloss: torch.Tensor,
                       want_dx: bool = True, want_dW: bool = True, workspace: torch.Tensor | None = None):
    """Returns (dx, dW) of sum_t dloss[t] loss[t] (None where not wanted), from the lse of head_loss_forward."""
    tokens, h, vocab, ws = _head(x, W, labels, workspace)
    _expect(lse, tokens)
    _expect(dloss, tokens)
    dx = _bf16_rows(x, tokens, h) if want_dx else None
    dW = _bf16_rows(x, vocab, h) if want_dW else None
    _check(lib().qg_head_loss_backward(_ptr(x, _BF16), _ptr(W, _BF16), _ptr(labels, (torch.int64,)), _ptr(lse, _F32), _ptr(dloss, _F32),
                                       tokens, h, vocab, h, _ptr(dx), _ptr(dW), _ptr(ws, (torch.uint8,)), ws.numel(), _stream()))
    return dx, dW


# ---------------------------------------------------------------- attention half of a decoder layer
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
_I32, _I64, _F64 = (torch.int32,), (torch.int64,), (torch.float64,)


def _heads(t: torch.Tensor | None):
    """A [tokens][heads][d] tensor of any token and head stride (a slice of a linear layer's output, heads outside)."""
    if t is None:
        return None
    st = t.stride()
    if not t.is_cuda or t.dtype is not torch.bfloat16 and t.dtype not in _BF16 or len(st) != 3 or st[2] != 1:
        if not t.is_cuda:
            raise QGError("device tensor expected")
        if t.dtype not in _BF16:
            raise QGError(f"dtype {t.dtype} not in {_BF16}")
        raise QGError(f"shape {tuple(t.shape)}, strides {st}: [tokens][heads][d] expected, elements of a head next to each other")
    return _pack_heads(t.data_ptr(), st[0], st[1])


def _written(t: torch.Tensor | None, like: torch.Tensor, what: str) -> torch.Tensor:
    """Where an output of like's shape goes: t, or a new tensor.  An expanded tensor has no place for every element, nor has a view whose heads overlap."""
    if t is None:
        return like.new_empty(*like.shape)      # (sizes as arguments: 1.5 us, as a torch.Size 2.6)
    T, H, d = shape = like.shape
    if t.shape != shape:
        raise QGError(f"shape {tuple(t.shape)}, expected {tuple(shape)}")
    ts, hs, _ = t.stride()
    if hs >= d and ts >= (H - 1) * hs + d:          # (any slice of a layer's output)
        return t
    if ts == 0 and T > 1 or hs == 0 and H > 1:
        raise QGError(f"{what}: an expanded tensor cannot be written")
    if not (hs >= (T - 1) * ts + d and ts >= d) and _meet(0, T, T, H, H, d, ts, hs, hs, itself=True):
        raise QGError(f"{what}: a tensor whose elements overlap cannot be written")
    return t


def _meet(D: int, T: int, U: int, H: int, K: int, d: int, ts: int, hs: int, ks: int, itself: bool = False) -> bool:
    """Whether some t ts + h hs and D + u ts + k ks, t < T, h < H, u < U, k < K, are less than d apart (itself: other than at t = u, h = k)."""
    heads = [(m * hs, m == 0) for m in range(1 - K, H)] if hs == ks else [(h * hs - k * ks, False) for h in range(H) for k in range(K)]
    for apart, same in heads:
        r = D - apart                           # (t - u) ts is to be nearer than d to this
        for n in (r // ts, r // ts + 1) if ts else (0,):
            if -U < n < T and abs(n * ts - r) < d and not (itself and same and n == 0):
                return True
    return False


def _span(t: torch.Tensor):
    """Where a [tokens][heads][d] tensor of 16-bit elements lies: begin and end in bytes, sizes, strides."""
    T, H, d = t.shape
    ts, hs, _ = t.stride()
    at = t.data_ptr()
    return at, at + 2 * ((T - 1) * ts + (H - 1) * hs + d), T, H, d, ts, hs


def _overlap(x, y) -> bool:
    """Whether two such places share an element.  Of arrays that lie in between each other: exact where they step from token to token alike, as slices of
    one layer's output do; where they do not, unless they keep to other columns of the rows that both step by, they are taken to."""
    if x[1] <= y[0] or y[1] <= x[0]:
        return False
    a, _, T, H, d, ts, hs = x
    b, _, U, K, _, us, ks = y
    alike = T == 1 or U == 1 or us == ts
    if T == 1:
        ts = us
    D = (b - a) // 2
    width, other = (H - 1) * hs + d, (K - 1) * ks + d      # of a token
    by = ts if alike else math.gcd(ts, us)
    if by >= width > 0 and D % by >= width and D % by + other <= by:
        return False
    return not alike or _meet(D, T, U, H, K, d, ts, hs, ks)


def _apart(outs, ins, places=()) -> None:
    """Refuses outputs that share memory with each other or with an input: workgroups read what others write.  An output may be the input beside it in `places`."""
    spans = [_span(t) for t in outs]
    for i in range(1, len(spans)):
        for j in range(i):
            if _overlap(spans[i], spans[j]):
                raise QGError("out: two outputs overlap")
    first, last = min([x[0] for x in spans]), max([x[1] for x in spans])
    for u in ins:
        if u is None or u.data_ptr() >= last:       # (most inputs need no more than that: 0.1 us, and what _span takes, 0.7, for those ahead of the outputs)
            continue
        y = _span(u)
        if y[1] <= first:
            continue
        for i, x in enumerate(spans):
            if _overlap(x, y) and not (places and u is places[i] and x[0] == y[0] and (x[5] == y[5] or x[2] == 1) and (x[6] == y[6] or x[3] == 1)):
                raise QGError("out: an output overlaps an input")


def _rope_layout(layout: str) -> int:
    if layout not in ROPE_LAYOUTS:
        raise QGError(f"layout {layout!r} not in {tuple(ROPE_LAYOUTS)}")
    return ROPE_LAYOUTS[layout]


def rope_frequencies(rot: int, base: float = 10000.0, factor: float = 1.0, context: float = 0, low: float = 1.0, high: float = 4.0,
                     device="cuda") -> torch.Tensor:
    """The rot/2 frequencies of rotary positions, float64 on `device`: base^(-2i/rot), with a factor stretched to longer contexts."""
    out = torch.empty(max(rot // 2, 1), dtype=torch.float64)
    _check(lib().qg_rope_frequencies(rot, base, factor, context, low, high, out.data_ptr()))
    return out.to(device)


def _rope(f, q, k, positions, freqs, layout, amplitude, out):
    tokens, heads_q, d = q.shape
    rot = 2 * freqs.shape[0]
    if k is not None:
        _expect(k, tokens, k.shape[1], d)
    _expect(positions, tokens)
    _expect(freqs, rot // 2)
    q_out = _written(None if out is None else out[0], q, "out")
    k_out = None if k is None else _written(None if out is None else out[1], k, "out")
    if out is not None:
        in_place = q_out is q and k_out is k
        _apart((q_out,) if k is None else (q_out, k_out), () if in_place else (q, k), (q, k))
    _check(f(_heads(q), heads_q, _heads(k), 0 if k is None else k.shape[1], _ptr(positions, _I64), _ptr(freqs, _F64), tokens, d, rot,
             _rope_layout(layout), amplitude, _heads(q_out), _heads(k_out), _stream()))
    return q_out, k_out


def rope_forward(q: torch.Tensor, k: torch.Tensor | None, positions: torch.Tensor, freqs: torch.Tensor, layout: str = "half",
                 amplitude: float = 1.0, out=None):
    """Returns (q', k'): the first 2 * len(freqs) elements of every head of q [tokens][heads][d] and k (None: only q) turned by
    positions[token] * freqs.  positions int64, freqs float64.  out: (q', k') to write into; the inputs themselves: in place, and nothing else that
    overlaps them or each other."""
    return _rope(lib().qg_rope_forward, q, k, positions, freqs, layout, amplitude, out)


def rope_backward(dq_out: torch.Tensor, dk_out: torch.Tensor | None, positions: torch.Tensor, freqs: torch.Tensor, layout: str = "half",
                  amplitude: float = 1.0, out=None):
    """Returns (dq, dk) of rope_forward, from the gradients of its outputs."""
    return _rope(lib().qg_rope_backward, dq_out, dk_out, positions, freqs, layout, amplitude, out)


def _attention(q, k, v, cu_q, cu_k, causal, scale, cap, slopes, window, prefix) -> bytes:
    tokens, heads, d = q.shape
    tokens_k, heads_k, _ = k.shape
    _expect(k, tokens_k, heads_k, d)
    _expect(v, tokens_k, heads_k, d)
    sequences = 1 if cu_q is None else cu_q.numel() - 1
    _expect(cu_q, sequences + 1)
    _expect(cu_k, sequences + 1)
    _expect(prefix, sequences)
    _expect(slopes, heads)
    try:
        return _pack_attention(tokens, tokens_k, heads, heads_k, d, sequences, _ptr(cu_q, _I32) or 0, _ptr(cu_k, _I32) or 0, _ptr(prefix, _I32) or 0,
                               _ptr(slopes, _F32) or 0, d ** -0.5 if scale is None else scale, cap, int(causal), window)
    except (OverflowError, struct.error) as e:
        raise QGError(f"libqgalore: {e}") from None


def _workspace(nbytes: int, like: torch.Tensor, given: torch.Tensor | None):
    """(pointer, bytes) of a call's workspace, and the tensor that holds it: the given one, or a new one if any is needed."""
    if given is None:
        if nbytes == 0:
            return None, None, 0
        given = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
    return given, _ptr(given, (torch.uint8,)), given.numel()


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor | None = None, cu_k: torch.Tensor | None = None,
                      causal: bool = True, scale: float | None = None, cap: float = 0.0, slopes: torch.Tensor | None = None,
                      window: int = 0, prefix: torch.Tensor | None = None, out: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None):
    """Returns (o, lse): attention of q [tokens][heads][d] over k and v [tokens_k][heads_k][d], o bf16 [tokens][heads][d], lse fp32
    [heads][tokens].  cu_q, cu_k: int32 [sequences + 1], boundaries of packed sequences (None: one sequence; cu_k None: as cu_q).
    scale: d^-0.5 if None; cap, slopes (fp32 [heads]), window, prefix (int32 [sequences]): as in qg_attention_forward.  out: where o is written, apart
    from the inputs."""
    a = _attention(q, k, v, cu_q, cu_k, causal, scale, cap, slopes, window, prefix)
    o = _written(out, q, "out")
    if out is not None:
        _apart((o,), (q, k, v))
    lse = torch.empty(q.shape[1], q.shape[0], dtype=torch.float32, device=q.device)
    ws, *at = _workspace(lib().qg_attention_forward_workspace_bytes(a), q, workspace)
    _check(lib().qg_attention_forward(a, _heads(q), _heads(k), _heads(v), _heads(o), _ptr(lse), *at, _stream()))
    return o, lse


def attention_backward(do: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
                       cu_q: torch.Tensor | None = None, cu_k: torch.Tensor | None = None, causal: bool = True,
                       scale: float | None = None, cap: float = 0.0, slopes: torch.Tensor | None = None, window: int = 0,
                       prefix: torch.Tensor | None = None, out=None, workspace: torch.Tensor | None = None):
    """Returns (dq, dk, dv) of attention_forward, from its inputs and results and do, the gradient of o.  out: (dq, dk, dv) to write into
    (slices of one gradient of the layer that gave q, k and v, say), apart from the inputs and each other."""
    a = _attention(q, k, v, cu_q, cu_k, causal, scale, cap, slopes, window, prefix)
    for t in (do, o):
        _expect(t, *q.shape)
    _expect(lse, q.shape[1], q.shape[0])
    dq, dk, dv = (_written(None if out is None else out[i], t, "out") for i, t in enumerate((q, k, v)))
    if out is not None:
        _apart((dq, dk, dv), (do, q, k, v, o))
    ws, *at = _workspace(lib().qg_attention_backward_workspace_bytes(a), q, workspace)
    _check(lib().qg_attention_backward(a, _heads(do), _heads(q), _heads(k), _heads(v), _heads(o), _ptr(lse, _F32), _heads(dq),
                                       _heads(dk), _heads(dv), *at, _stream()))
    return dq, dk, dv


def _cache(k_pages, v_pages, table) -> bytes:
    pages, page_size, heads, d = k_pages.shape
    _expect(v_pages, pages, page_size, heads, d)
    sequences, width = table.shape
    return _pack_cache(_ptr(k_pages, _BF16), _ptr(v_pages, _BF16), _ptr(table, _I32), pages, page_size, heads, d, sequences, width)


def cache_append(q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, k_pages: torch.Tensor,
                 v_pages: torch.Tensor, table: torch.Tensor, sequence: torch.Tensor | None = None, freqs: torch.Tensor | None = None,
                 layout: str = "half", amplitude: float = 1.0, out: torch.Tensor | None = None):
    """Puts k and v [tokens][heads_k][d] of new tokens into the pages [pages][page_size][heads_k][d] of a cache: token t to
    position positions[t] (int64) of sequence[t] (int32; None: t), whose pages table[sequence] (int32 [sequences][width]) lists.  k is turned on its
    way if freqs is given, and so is q, which is returned (None without q).  out: where q goes (q itself: in place), apart from all else.  k and v may be
    rows of the pages, if none of them is among those written."""
    c = _cache(k_pages, v_pages, table)
    tokens = k.shape[0]
    heads, d = k_pages.shape[2:]
    _expect(k, tokens, heads, d)
    _expect(v, tokens, heads, d)
    _expect(positions, tokens)
    _expect(sequence, tokens)
    rot = 0
    if freqs is not None:
        rot = 2 * freqs.shape[0]
        _expect(freqs, rot // 2)
    q_out = None
    if q is not None:
        _expect(q, tokens, q.shape[1], d)
        q_out = _written(out, q, "out")
        if out is not None:
            _apart((q_out,), (q, k, v, k_pages.flatten(0, 1), v_pages.flatten(0, 1)), (q,))
    if abs(k_pages.data_ptr() - v_pages.data_ptr()) < 2 * k_pages.numel():
        raise QGError("k_pages and v_pages overlap")
    _check(lib().qg_cache_append(c, _heads(q), 0 if q is None else q.shape[1], _heads(k), _heads(v), _ptr(positions, _I64),
                                 _ptr(sequence, _I32), tokens, _ptr(freqs, _F64), rot, _rope_layout(layout), amplitude, _heads(q_out), _stream()))
    return q_out


def attention_paged(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                    scale: float | None = None, cap: float = 0.0, slopes: torch.Tensor | None = None, window: int = 0,
                    out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of one new token per sequence, q [sequences][heads][d], over the first lengths[s] (int32) positions of its pages; the token is
    the last of them.  Returns o [sequences][heads][d].  out: where it is written (q itself, or apart from all inputs).  workspace: uint8, qg_attention_paged_workspace_bytes of them (allocated if None)."""
    c = _cache(k_pages, v_pages, table)
    sequences, heads, d = table.shape[0], q.shape[1], k_pages.shape[3]
    _expect(q, sequences, heads, d)
    _expect(lengths, sequences)
    _expect(slopes, heads)
    o = _written(out, q, "out")
    if out is not None:
        _apart((o,), (q, k_pages.flatten(0, 1), v_pages.flatten(0, 1)), (q,))
    ws, *at = _workspace(lib().qg_attention_paged_workspace_bytes(c, heads), q, workspace)
    _check(lib().qg_attention_paged(c, _ptr(lengths, _I32), _heads(q), heads, d ** -0.5 if scale is None else scale, cap, window,
                                    _ptr(slopes, _F32), _heads(o), *at, _stream()))
    return o


# ---------------------------------------------------------------- subspace refresh
def range_apply(G: torch.Tensor, Z: torch.Tensor, m: int, n: int, r: int) -> torch.Tensor:
    Y = torch.empty(m, r, dtype=torch.float32, device=G.device)
    _check(lib().qg_range_apply(_ptr(G, _BF16), _ptr(Z, _BF16), m, n, r, _ptr(Y), _stream()))
    return Y


def orthonormalize(Y: torch.Tensor):
    """Returns (Q, info): Q fp32 [m][r], info a device int32 (0 = every pivot positive)."""
    m, r = Y.shape
    nbytes = lib().qg_orthonormalize_workspace_bytes(m, r)
    if nbytes == 0:
        raise QGError("libqgalore: shape out of range")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=Y.device)
    Q = torch.empty_like(Y)
    info = torch.empty(1, dtype=torch.int32, device=Y.device)
    _check(lib().qg_orthonormalize(_ptr(Y, (torch.float32,)), m, r, _ptr(Q), _ptr(info), _ptr(ws), nbytes, _stream()))
    return Q, info


def subspace_refresh(Pq, Ps, G, m: int, n: int, r: int, passes: int = 1, workspace: torch.Tensor | None = None):
    """Returns (Pq_new, Ps_new, cos, info, workspace); cos and info are device tensors of one element."""
    nbytes = lib().qg_refresh_workspace_bytes(1, m, n, r)
    if nbytes == 0:
        raise QGError("libqgalore: shape out of range")
    if workspace is None:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=G.device)
    Pq_new, Ps_new = torch.empty_like(Pq), torch.empty_like(Ps)
    cos = torch.empty(1, dtype=torch.float32, device=G.device)
    info = torch.empty(1, dtype=torch.int32, device=G.device)
    _check(lib().qg_subspace_refresh(_ptr(Pq, (torch.uint8,)), _ptr(Ps, (torch.float32,)), _ptr(G, _BF16), m, n, r,
                                     GROUP, passes, _ptr(Pq_new), _ptr(Ps_new), _ptr(cos), _ptr(info),
                                     _ptr(workspace), workspace.numel(), _stream()))
    return Pq_new, Ps_new, cos, info, workspace


def subspace_refresh_many(Pqs, Pss, Gs, m: int, n: int, r: int, passes: int = 1,
                          workspace: torch.Tensor | None = None, out=None, ld: int = 0):
    """Refresh of several matrices of one shape.  Pqs, Pss, Gs: lists of device tensors.  `out`: optional
    (list of Pq_new, list of Ps_new) to write into.  ld: row pitch of the gradients (0: dense).
    Returns (Pq_news, Ps_news, cos[count], info[count], workspace)."""
    count = len(Gs)
    if count == 0 or len(Pqs) != count or len(Pss) != count:
        raise QGError("libqgalore: one Pq and one Ps per gradient expected")
    if workspace is None:
        nbytes = lib().qg_refresh_workspace_bytes(count, m, ld or n, r)
        if nbytes == 0:
            raise QGError("libqgalore: shape out of range")
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=Gs[0].device)
    if out is None:
        out = ([torch.empty_like(p) for p in Pqs], [torch.empty_like(p) for p in Pss])
    descs = (RefreshDesc * count)()
    for i in range(count):
        descs[i] = RefreshDesc(_ptr(Pqs[i], (torch.uint8,)), _ptr(Pss[i], (torch.float32,)), _ptr(Gs[i], _BF16),
                               _ptr(out[0][i], (torch.uint8,)), _ptr(out[1][i], (torch.float32,)))
    cos = torch.empty(count, dtype=torch.float32, device=Gs[0].device)
    info = torch.empty(count, dtype=torch.int32, device=Gs[0].device)
    _check(lib().qg_subspace_refresh_many_ld(count, descs, m, n, ld, r, GROUP, passes, _ptr(cos), _ptr(info),
                                             _ptr(workspace), workspace.numel(), _stream()))
    return out[0], out[1], cos, info, workspace


DIAG_MFMA_WORKGROUPS = 512


def diag_clock_probe(ticks_100mhz: int, out2: torch.Tensor) -> None:
    """Enqueue the clock probe on the current stream; out2 (2 x int64, device) receives {shader cycles, ticks}."""
    _check(lib().qg_diag_clock_probe(ticks_100mhz, _ptr(out2, (torch.int64,)), _stream()))


def diag_mfma_loop(iters: int, random_operands: bool, sink: torch.Tensor) -> float:
    """Enqueue the register-only MFMA loop; returns the flop it performs."""
    assert sink.numel() >= DIAG_MFMA_WORKGROUPS * 512
    _check(lib().qg_diag_mfma_loop(iters, int(random_operands), _ptr(sink, (torch.float32,)), _stream()))
    return DIAG_MFMA_WORKGROUPS * 8 * iters * 16 * 32768.0


def diag_mfma_f64_loop(iters: int, workgroups: int, sink: torch.Tensor) -> float:
    """Enqueue the register-only fp64 MFMA loop; returns the flop it performs."""
    assert sink.numel() >= workgroups * 256
    _check(lib().qg_diag_mfma_f64_loop(iters, workgroups, _ptr(sink, (torch.float32,)), _stream()))
    return workgroups * 4 * iters * 8 * 2048.0


def sr_uniform(seed: int, step: int, idx0: int, count: int, device="cuda") -> torch.Tensor:
    out = torch.empty(count, dtype=torch.float32, device=device)
    _check(lib().qg_sr_uniform(seed, step, idx0, count, _ptr(out), _stream()))
    return out
