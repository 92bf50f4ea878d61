"""ctypes binding of the C-ABI library declared in include/fw.h.

Argument marshalling only: every function here has the name and the meaning of
the C entry point it wraps, takes torch CUDA tensors (or raw device addresses)
where the C function takes device pointers, and raises FwError on a non-zero
status.  There is no computation and no fallback in this file: if libfw.so is
missing or cannot be loaded the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libfw.so")

FW_OK = 0
FW_ERR_INVALID_ARG, FW_ERR_SHAPE, FW_ERR_STATE, FW_ERR_WORKSPACE = 1, 2, 3, 4
FW_ERR_CUDA, FW_ERR_TIMEOUT, FW_ERR_UNSUPPORTED = 5, 6, 7
FW_WARN_NO_SUBSPACE, FW_WARN_NONFINITE = 64, 65
FW_F32, FW_BF16, FW_E4M3 = 0, 1, 2
FW_PREC_FP32, FW_PREC_TF32, FW_PREC_BF16 = 0, 1, 2
FW_INIT_ALIGN, FW_INIT_MAXCOL = 0, 1
FW_F_MU, FW_F_PHIX, FW_F_PHI_DIAG, FW_F_LAMBDA_BAR, FW_F_T, FW_F_Q, FW_F_QS, FW_F_PHIY, FW_F_ALIGN_W = range(9)
FW_MAX_GROUP = 64
FW_COV_COMMIT, FW_COV_ACCUMULATE = 0, 1

EXPORTS = [
    "fw_layer_desc_default", "fw_layer_workspace_bytes", "fw_layer_create", "fw_layer_destroy",
    "fw_layer_attach_params", "fw_cov_update", "fw_cond_reduce", "fw_grad_transform", "fw_step",
    "fw_group_cov_update", "fw_group_cond_reduce", "fw_group_grad_transform_step",
    "fw_layer_get", "fw_layer_set", "fw_layer_sync_status", "fw_status_string", "fw_version",
    "fw_profile_begin", "fw_profile_end", "fw_launch_count", "fw_cov_block_static",
    "fw_debug_wait_probe", "fw_recursion_on_chip", "fw_layer_reset",
    "fw_nhwc_scratch_bytes", "fw_cov_update_nhwc", "fw_group_cov_update_nhwc",
    "fw_whiten_forward", "fw_whiten_backward", "fw_step_momentum", "fw_whiteness",
    "fw_evd_scratch_bytes", "fw_evd_whiten", "fw_group_evd_whiten", "fw_spectrum",
    "fw_norm_desc_default", "fw_rmsnorm_scratch_bytes", "fw_rmsnorm_forward", "fw_rmsnorm_backward",
    "fw_distill_desc_default", "fw_distill_forward", "fw_distill_backward",
    "fw_gated_desc_default", "fw_gated_workspace_bytes", "fw_gated_create", "fw_gated_destroy", "fw_gated_forward",
    "fw_gated_backward", "fw_gated_sync_status",
    "fw_sandwich_desc_default", "fw_sandwich_scratch_bytes", "fw_sandwich_forward", "fw_sandwich_backward",
    "fw_logprob_desc_default", "fw_logprob_forward", "fw_logprob_backward", "fw_policy_desc_default", "fw_policy_forward",
    "fw_preference_desc_default", "fw_preference_loss",
    "fw_adamw_desc_default", "fw_adamw_workspace_bytes", "fw_adamw_create", "fw_adamw_destroy", "fw_adamw_step", "fw_adamw_state",
    "fw_adamw_sync_status",
]
FW_STATIC_MAX_M = 256
FW_ACT_SILU, FW_ACT_GELU, FW_ACT_GELU_TANH, FW_ACT_RELU = range(4)
FW_A_M, FW_A_V, FW_A_M_SCALE, FW_A_V_SCALE, FW_A_STEP = range(5)
FW_PROF_NAMES = ["pilot", "gram", "moments", "resync", "recur_mv", "recur_upd", "smooth", "gq", "misc", "recur_chip"]


class FwError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = _lib().fw_status_string(status).decode() if _LIB is not None else "?"
        super().__init__(f"{where}: fw_status {status} ({msg})")


class fw_layer_desc(C.Structure):
    _fields_ = [("M", C.c_int32), ("N", C.c_int32), ("x_dtype", C.c_int32), ("prec", C.c_int32),
                ("init", C.c_int32), ("alpha", C.c_float), ("beta", C.c_float), ("gamma", C.c_float),
                ("delta", C.c_float), ("eps", C.c_float), ("c_rel", C.c_float), ("c_abs", C.c_float)]


class fw_norm_desc(C.Structure):
    _fields_ = [("M", C.c_int32), ("dtype", C.c_int32), ("y_dtype", C.c_int32), ("eps", C.c_float)]


class fw_distill_desc(C.Structure):
    _fields_ = [("V", C.c_int32), ("K", C.c_int32), ("z_dtype", C.c_int32), ("t_dtype", C.c_int32),
                ("index_bits", C.c_int32), ("tau", C.c_float)]


class fw_gated_desc(C.Structure):
    _fields_ = [("M", C.c_int32), ("N", C.c_int32), ("x_dtype", C.c_int32), ("act", C.c_int32), ("grad", C.c_int32),
                ("max_rows", C.c_int64)]


class fw_sandwich_desc(C.Structure):
    _fields_ = [("M", C.c_int32), ("dtype", C.c_int32), ("y_dtype", C.c_int32), ("post", C.c_int32), ("eps", C.c_float), ("alpha", C.c_float)]


class fw_logprob_desc(C.Structure):
    _fields_ = [("V", C.c_int32), ("z_dtype", C.c_int32), ("index_bits", C.c_int32), ("tau", C.c_float)]


class fw_policy_desc(C.Structure):
    _fields_ = [("clip_low", C.c_float), ("clip_high", C.c_float), ("kl", C.c_float)]


class fw_preference_desc(C.Structure):
    _fields_ = [("beta", C.c_float), ("margin", C.c_float), ("smooth", C.c_float), ("mean", C.c_int32)]


class fw_adamw_desc(C.Structure):
    _fields_ = [("n", C.c_int32), ("state", C.c_int32), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_float), ("seed", C.c_uint32)]


_LIB = None


def _lib():
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} not found: build it with "
                          "`python -m paper_2010_01546_b200.build` (there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
    P = C.POINTER
    lib.fw_layer_desc_default.argtypes = [P(fw_layer_desc), i32, i32]; lib.fw_layer_desc_default.restype = None
    lib.fw_layer_workspace_bytes.argtypes = [P(fw_layer_desc)]; lib.fw_layer_workspace_bytes.restype = sz
    lib.fw_layer_create.argtypes = [P(fw_layer_desc), vp, sz, vp, P(vp)]; lib.fw_layer_create.restype = i32
    lib.fw_layer_destroy.argtypes = [vp]; lib.fw_layer_destroy.restype = i32
    lib.fw_layer_reset.argtypes = [vp]; lib.fw_layer_reset.restype = i32
    lib.fw_layer_attach_params.argtypes = [vp, vp, vp]; lib.fw_layer_attach_params.restype = i32
    lib.fw_cov_update.argtypes = [vp, vp, i64, i64, C.c_uint32]; lib.fw_cov_update.restype = i32
    lib.fw_nhwc_scratch_bytes.argtypes = [i32, i32, i32, i32, i32]; lib.fw_nhwc_scratch_bytes.restype = sz
    lib.fw_cov_update_nhwc.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp, sz, C.c_uint32]
    lib.fw_cov_update_nhwc.restype = i32
    lib.fw_group_cov_update_nhwc.argtypes = [P(vp), i32, P(vp), P(i32), P(i32), P(i32), P(i32), P(i32), P(vp), P(sz),
                                             C.c_uint32]
    lib.fw_group_cov_update_nhwc.restype = i32
    lib.fw_cond_reduce.argtypes = [vp, i32, i32, vp]; lib.fw_cond_reduce.restype = i32
    lib.fw_grad_transform.argtypes = [vp, vp, vp]; lib.fw_grad_transform.restype = i32
    lib.fw_step.argtypes = [vp, vp, vp, vp, vp, f32]; lib.fw_step.restype = i32
    lib.fw_step_momentum.argtypes = [vp, vp, vp, vp, vp, vp, vp, f32, f32, f32]; lib.fw_step_momentum.restype = i32
    lib.fw_whiteness.argtypes = [vp, vp]; lib.fw_whiteness.restype = i32
    lib.fw_evd_scratch_bytes.argtypes = [i32]; lib.fw_evd_scratch_bytes.restype = sz
    lib.fw_evd_whiten.argtypes = [vp, vp, sz, f32]; lib.fw_evd_whiten.restype = i32
    lib.fw_group_evd_whiten.argtypes = [P(vp), i32, P(vp), P(sz), f32]; lib.fw_group_evd_whiten.restype = i32
    lib.fw_spectrum.argtypes = [vp, i32, vp, sz, vp, vp]; lib.fw_spectrum.restype = i32
    lib.fw_whiten_forward.argtypes = [vp, vp, i64, vp]; lib.fw_whiten_forward.restype = i32
    lib.fw_whiten_backward.argtypes = [vp, vp, i64, vp]; lib.fw_whiten_backward.restype = i32
    lib.fw_group_cov_update.argtypes = [P(vp), i32, P(vp), P(i64), P(i64), C.c_uint32]
    lib.fw_group_cov_update.restype = i32
    lib.fw_group_cond_reduce.argtypes = [P(vp), i32, i32, i32, P(vp)]; lib.fw_group_cond_reduce.restype = i32
    lib.fw_group_grad_transform_step.argtypes = [P(vp), i32, P(vp), P(vp), P(vp), P(vp), f32]
    lib.fw_group_grad_transform_step.restype = i32
    lib.fw_layer_get.argtypes = [vp, i32, vp, sz]; lib.fw_layer_get.restype = i32
    lib.fw_layer_set.argtypes = [vp, i32, vp, sz]; lib.fw_layer_set.restype = i32
    lib.fw_layer_sync_status.argtypes = [vp]; lib.fw_layer_sync_status.restype = i32
    lib.fw_status_string.argtypes = [i32]; lib.fw_status_string.restype = C.c_char_p
    lib.fw_version.argtypes = []; lib.fw_version.restype = i32
    lib.fw_profile_begin.argtypes = []; lib.fw_profile_begin.restype = i32
    lib.fw_profile_end.argtypes = [P(f32), P(i64)]; lib.fw_profile_end.restype = i32
    lib.fw_launch_count.argtypes = []; lib.fw_launch_count.restype = i64
    lib.fw_cov_block_static.argtypes = [vp, i64, i64, i32, vp, vp, vp]; lib.fw_cov_block_static.restype = i32
    lib.fw_debug_wait_probe.argtypes = [vp, C.c_uint32]; lib.fw_debug_wait_probe.restype = i32
    lib.fw_recursion_on_chip.argtypes = [P(fw_layer_desc)]; lib.fw_recursion_on_chip.restype = i32
    lib.fw_norm_desc_default.argtypes = [P(fw_norm_desc), i32]; lib.fw_norm_desc_default.restype = None
    lib.fw_rmsnorm_scratch_bytes.argtypes = [P(fw_norm_desc)]; lib.fw_rmsnorm_scratch_bytes.restype = sz
    lib.fw_rmsnorm_forward.argtypes = [P(fw_norm_desc), i64, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp, vp]
    lib.fw_rmsnorm_forward.restype = i32
    lib.fw_rmsnorm_backward.argtypes = [P(fw_norm_desc), i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp, sz, vp]
    lib.fw_rmsnorm_backward.restype = i32
    lib.fw_distill_desc_default.argtypes = [P(fw_distill_desc), i32, i32]; lib.fw_distill_desc_default.restype = None
    lib.fw_distill_forward.argtypes = [P(fw_distill_desc), vp, i64, i64, vp, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.fw_distill_forward.restype = i32
    lib.fw_distill_backward.argtypes = [P(fw_distill_desc), vp, i64, i64, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.fw_distill_backward.restype = i32
    lib.fw_gated_desc_default.argtypes = [P(fw_gated_desc), i32, i32]; lib.fw_gated_desc_default.restype = None
    lib.fw_gated_workspace_bytes.argtypes = [P(fw_gated_desc)]; lib.fw_gated_workspace_bytes.restype = sz
    lib.fw_gated_create.argtypes = [P(fw_gated_desc), vp, sz, vp, P(vp)]; lib.fw_gated_create.restype = i32
    lib.fw_gated_destroy.argtypes = [vp]; lib.fw_gated_destroy.restype = i32
    lib.fw_gated_forward.argtypes = [vp, vp, i64, i64, vp, vp, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, i64]
    lib.fw_gated_forward.restype = i32
    lib.fw_gated_backward.argtypes = [vp, vp, i64, i64, vp, i64, vp, vp, i64, vp, vp, i64, vp, i64, vp, vp, i32, vp, vp]
    lib.fw_gated_backward.restype = i32
    lib.fw_gated_sync_status.argtypes = [vp]; lib.fw_gated_sync_status.restype = i32
    lib.fw_sandwich_desc_default.argtypes = [P(fw_sandwich_desc), i32]; lib.fw_sandwich_desc_default.restype = None
    lib.fw_sandwich_scratch_bytes.argtypes = [P(fw_sandwich_desc)]; lib.fw_sandwich_scratch_bytes.restype = sz
    lib.fw_sandwich_forward.argtypes = [P(fw_sandwich_desc), i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp]
    lib.fw_sandwich_forward.restype = i32
    lib.fw_sandwich_backward.argtypes = [P(fw_sandwich_desc), i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp,
                                         vp, sz, vp]
    lib.fw_sandwich_backward.restype = i32
    lib.fw_logprob_desc_default.argtypes = [P(fw_logprob_desc), i32]; lib.fw_logprob_desc_default.restype = None
    lib.fw_logprob_forward.argtypes = [P(fw_logprob_desc), vp, i64, i64, vp, vp, vp, vp]; lib.fw_logprob_forward.restype = i32
    lib.fw_logprob_backward.argtypes = [P(fw_logprob_desc), vp, i64, i64, vp, vp, vp, vp, i64, vp]; lib.fw_logprob_backward.restype = i32
    lib.fw_policy_desc_default.argtypes = [P(fw_policy_desc)]; lib.fw_policy_desc_default.restype = None
    lib.fw_policy_forward.argtypes = [P(fw_logprob_desc), P(fw_policy_desc), vp, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.fw_policy_forward.restype = i32
    lib.fw_preference_desc_default.argtypes = [P(fw_preference_desc)]; lib.fw_preference_desc_default.restype = None
    lib.fw_preference_loss.argtypes = [P(fw_logprob_desc), P(fw_preference_desc), vp, i64, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.fw_preference_loss.restype = i32
    lib.fw_adamw_desc_default.argtypes = [P(fw_adamw_desc), i32]; lib.fw_adamw_desc_default.restype = None
    lib.fw_adamw_workspace_bytes.argtypes = [P(fw_adamw_desc), P(i64)]; lib.fw_adamw_workspace_bytes.restype = sz
    lib.fw_adamw_create.argtypes = [P(fw_adamw_desc), P(i64), P(vp), P(vp), P(f32), vp, sz, vp, P(vp)]; lib.fw_adamw_create.restype = i32
    lib.fw_adamw_destroy.argtypes = [vp]; lib.fw_adamw_destroy.restype = i32
    lib.fw_adamw_step.argtypes = [vp, P(vp), P(i32), f32, vp, f32, vp]; lib.fw_adamw_step.restype = i32
    lib.fw_adamw_state.argtypes = [vp, i32, P(vp), P(sz)]; lib.fw_adamw_state.restype = i32
    lib.fw_adamw_sync_status.argtypes = [vp]; lib.fw_adamw_sync_status.restype = i32
    _LIB = lib
    return lib


def _ptr(t):
    """Device address of a torch tensor (or pass an int / None through)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _check(status: int, where: str, allow=()):
    if status != FW_OK and status not in allow:
        raise FwError(status, where)
    return status


def _vp_array(items):
    arr = (C.c_void_p * len(items))()
    for i, it in enumerate(items):
        arr[i] = _ptr(it)
    return arr


# ---- one function per C entry point ---------------------------------------
def fw_version() -> int:
    return _lib().fw_version()


def fw_status_string(status: int) -> str:
    return _lib().fw_status_string(status).decode()


def fw_layer_desc_default(M: int, N: int, **overrides) -> fw_layer_desc:
    d = fw_layer_desc()
    _lib().fw_layer_desc_default(C.byref(d), M, N)
    for k, v in overrides.items():
        setattr(d, k, v)
    return d


def fw_layer_workspace_bytes(desc: fw_layer_desc) -> int:
    return _lib().fw_layer_workspace_bytes(C.byref(desc))


def fw_layer_create(desc: fw_layer_desc, workspace, nbytes: int, stream: int = 0) -> int:
    out = C.c_void_p()
    _check(_lib().fw_layer_create(C.byref(desc), _ptr(workspace), nbytes, stream, C.byref(out)), "fw_layer_create")
    return out.value


def fw_layer_destroy(handle: int) -> None:
    _check(_lib().fw_layer_destroy(handle), "fw_layer_destroy")


def fw_layer_reset(handle) -> None:
    _check(_lib().fw_layer_reset(handle), "fw_layer_reset")


def fw_layer_attach_params(handle, W, b) -> None:
    _check(_lib().fw_layer_attach_params(handle, _ptr(W), _ptr(b)), "fw_layer_attach_params")


def fw_cov_update(handle, X, rows: int, ldx: int, flags: int = FW_COV_COMMIT) -> None:
    _check(_lib().fw_cov_update(handle, _ptr(X), rows, ldx, flags), "fw_cov_update")


def fw_nhwc_scratch_bytes(B: int, H: int, W: int, Cc: int, k: int) -> int:
    return int(_lib().fw_nhwc_scratch_bytes(B, H, W, Cc, k))


def fw_cov_update_nhwc(handle, A, B: int, H: int, W: int, Cc: int, k: int, scratch=None, scratch_bytes: int = 0,
                       flags: int = FW_COV_COMMIT) -> None:
    _check(_lib().fw_cov_update_nhwc(handle, _ptr(A), B, H, W, Cc, k, _ptr(scratch), scratch_bytes, flags),
           "fw_cov_update_nhwc")


def fw_group_cov_update_nhwc(handles, A, B, H, W, Cc, k, scratch, scratch_bytes, flags: int = FW_COV_COMMIT) -> None:
    n = len(handles)
    i32a = lambda v: (C.c_int32 * n)(*v)
    _check(_lib().fw_group_cov_update_nhwc(_vp_array(handles), n, _vp_array(A), i32a(B), i32a(H), i32a(W), i32a(Cc),
                                           i32a(k), _vp_array(scratch), (C.c_size_t * n)(*scratch_bytes), flags),
           "fw_group_cov_update_nhwc")


def fw_cond_reduce(handle, K: int, P: int, trace=None) -> None:
    _check(_lib().fw_cond_reduce(handle, K, P, _ptr(trace)), "fw_cond_reduce")


def fw_grad_transform(handle, G, G_out) -> None:
    _check(_lib().fw_grad_transform(handle, _ptr(G), _ptr(G_out)), "fw_grad_transform")


def fw_step_momentum(handle, W, b, G_t, g_b, vW, vb, lr: float, momentum: float, weight_decay: float) -> None:
    _check(_lib().fw_step_momentum(handle, _ptr(W), _ptr(b), _ptr(G_t), _ptr(g_b), _ptr(vW), _ptr(vb), lr, momentum,
                                   weight_decay), "fw_step_momentum")


def fw_whiteness(handle, rho_out) -> None:
    _check(_lib().fw_whiteness(handle, _ptr(rho_out)), "fw_whiteness")


def fw_evd_scratch_bytes(M: int) -> int:
    return int(_lib().fw_evd_scratch_bytes(M))


def fw_evd_whiten(handle, scratch, scratch_bytes: int, g_max: float = 0.0) -> None:
    _check(_lib().fw_evd_whiten(handle, _ptr(scratch), scratch_bytes, g_max), "fw_evd_whiten")


def fw_group_evd_whiten(handles, scratch, scratch_bytes, g_max: float = 0.0) -> None:
    n = len(handles)
    _check(_lib().fw_group_evd_whiten(_vp_array(handles), n, _vp_array(scratch),
                                      (C.c_size_t * n)(*scratch_bytes), g_max), "fw_group_evd_whiten")


def fw_spectrum(handle, which: int, scratch, scratch_bytes: int, lam_out=None, kappa_out=None) -> None:
    _check(_lib().fw_spectrum(handle, which, _ptr(scratch), scratch_bytes,
                              _ptr(lam_out) if lam_out is not None else None,
                              _ptr(kappa_out) if kappa_out is not None else None), "fw_spectrum")


def fw_whiten_forward(handle, X, rows: int, Y) -> None:
    _check(_lib().fw_whiten_forward(handle, _ptr(X), rows, _ptr(Y)), "fw_whiten_forward")


def fw_whiten_backward(handle, dY, rows: int, dX) -> None:
    _check(_lib().fw_whiten_backward(handle, _ptr(dY), rows, _ptr(dX)), "fw_whiten_backward")


def fw_step(handle, W, b, G_t, g_b, lr: float) -> None:
    _check(_lib().fw_step(handle, _ptr(W), _ptr(b), _ptr(G_t), _ptr(g_b), lr), "fw_step")


def fw_group_cov_update(handles, X, rows, ldx, flags: int = FW_COV_COMMIT) -> None:
    n = len(handles)
    _check(_lib().fw_group_cov_update(_vp_array(handles), n, _vp_array(X), (C.c_int64 * n)(*rows),
                                      (C.c_int64 * n)(*ldx), flags), "fw_group_cov_update")


def fw_group_cond_reduce(handles, K: int, P: int, traces=None) -> None:
    n = len(handles)
    tr = _vp_array(traces) if traces is not None else None
    _check(_lib().fw_group_cond_reduce(_vp_array(handles), n, K, P, tr), "fw_group_cond_reduce")


def fw_group_grad_transform_step(handles, G, W, b, g_b, lr: float) -> None:
    n = len(handles)
    _check(_lib().fw_group_grad_transform_step(_vp_array(handles), n, _vp_array(G), _vp_array(W),
                                               _vp_array(b) if b is not None else None,
                                               _vp_array(g_b) if g_b is not None else None, lr),
           "fw_group_grad_transform_step")


def fw_layer_get(handle, field: int, dst, nbytes: int) -> None:
    _check(_lib().fw_layer_get(handle, field, _ptr(dst), nbytes), "fw_layer_get")


def fw_layer_set(handle, field: int, src, nbytes: int) -> None:
    _check(_lib().fw_layer_set(handle, field, _ptr(src), nbytes), "fw_layer_set")


def fw_layer_sync_status(handle) -> int:
    """Returns FW_OK or one of the FW_WARN_* codes; raises on errors."""
    return _check(_lib().fw_layer_sync_status(handle), "fw_layer_sync_status",
                  allow=(FW_WARN_NO_SUBSPACE, FW_WARN_NONFINITE))


def fw_cov_block_static(X, rows: int, ldx: int, M: int, mu_out, phix_out, stream: int = 0) -> None:
    """Mean and covariance of one block with no workspace and no allocation
    (for callers that cannot allocate device memory); M <= FW_STATIC_MAX_M."""
    _check(_lib().fw_cov_block_static(_ptr(X), rows, ldx, M, _ptr(mu_out), _ptr(phix_out), stream),
           "fw_cov_block_static")


def fw_debug_wait_probe(handle, polls: int) -> None:
    _check(_lib().fw_debug_wait_probe(handle, polls), "fw_debug_wait_probe")


def fw_recursion_on_chip(desc: fw_layer_desc) -> bool:
    return bool(_lib().fw_recursion_on_chip(C.byref(desc)))


def fw_profile_begin() -> None:
    _check(_lib().fw_profile_begin(), "fw_profile_begin")


def fw_profile_end() -> dict:
    """{class name: (milliseconds, launches)} for the classes that ran."""
    n = len(FW_PROF_NAMES)
    ms = (C.c_float * n)()
    cnt = (C.c_int64 * n)()
    _check(_lib().fw_profile_end(ms, cnt), "fw_profile_end")
    return {FW_PROF_NAMES[i]: (float(ms[i]), int(cnt[i])) for i in range(n) if cnt[i]}


def fw_launch_count() -> int:
    return int(_lib().fw_launch_count())


# ---- operators around the layers: tensors in, with their sizes, strides and types looked at ----
_TYPES = _torch = None  # this library's types as torch has them, and torch (both with the first call)


def _here():
    """The device that the library launches on: the current one.  Tensors have to be there."""
    global _TYPES, _torch
    if _TYPES is None:
        import torch
        _torch = torch
        _TYPES = {FW_F32: torch.float32, FW_BF16: torch.bfloat16, FW_E4M3: torch.float8_e4m3fn, "int32": torch.int32,
                  "int64": torch.int64}
    if _torch.cuda.is_initialized():
        return _torch._C._cuda_getDevice()                 # what current_device() asks, without its checks (0.4 us a call)
    return _torch.cuda.current_device() if _torch.cuda.is_available() else None


def _refuse_device(t, dev, name):
    if not t.is_cuda:
        raise ValueError(f"{name}: not a CUDA tensor")
    raise ValueError(f"{name}: on cuda:{t.get_device()}, but the current device is cuda:{dev}")


def _matrix(t, rows, cols, dtype, name, dev):
    """(address, leading dimension) of a rows x cols tensor of one of this library's types, the elements of a row next to each
    other; (None, 0) for None."""
    if t is None:
        return None, 0
    if t.dtype is not _TYPES[dtype]:
        raise TypeError(f"{name}: {t.dtype} is not the type that its description says")
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or shape[0] != rows or shape[1] != cols:
        raise ValueError(f"{name}: expected {rows} x {cols}, got {tuple(shape)}")
    if stride[1] != 1 and cols > 1:
        raise ValueError(f"{name}: the elements of a row have to be next to each other")
    ld = stride[0]
    if ld < cols:
        if rows > 1:
            raise ValueError(f"{name}: rows overlap")
        ld = cols
    if t.get_device() != dev:
        _refuse_device(t, dev, name)
    return t.data_ptr(), ld


def _pair(a, b, rows, cols, dtype, name, dev):
    """Two matrices with one leading dimension."""
    pa, lda = _matrix(a, rows, cols, dtype, name, dev)
    pb, ldb = _matrix(b, rows, cols, dtype, name, dev)
    if a is not None and b is not None and lda != ldb:
        raise ValueError(f"{name}: their rows have to be equally far apart")
    return pa, pb, lda if a is not None else ldb


def _vector(t, n, name, dev, dtype=FW_F32):
    """Address of a contiguous tensor of n elements; None for None."""
    if t is None:
        return None
    if t.dtype is _TYPES[dtype] and t.numel() == n and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    if t.dtype is not _TYPES[dtype]:
        raise TypeError(f"{name}: {t.dtype} is not the type that is expected")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: expected {n} contiguous elements, got {tuple(t.shape)}")
    _refuse_device(t, dev, name)


def _override(d, overrides):
    """The description with some fields set; ctypes would take a misspelt one without a word."""
    for k, v in overrides.items():
        if not any(k == f[0] for f in d._fields_):
            raise TypeError(f"{type(d).__name__} has no field {k}")
        setattr(d, k, v)
    return d


def fw_norm_desc_default(M: int, **overrides) -> fw_norm_desc:
    d = fw_norm_desc()
    _lib().fw_norm_desc_default(C.byref(d), M)
    return _override(d, overrides)


def fw_rmsnorm_scratch_bytes(desc: fw_norm_desc) -> int:
    return int(_lib().fw_rmsnorm_scratch_bytes(C.byref(desc)))


def fw_rmsnorm_forward(desc: fw_norm_desc, x, w, y, res=None, sum_out=None, y_scale=None, rstd=None, stream: int = 0) -> None:
    rows, M, t, dev = x.shape[0], desc.M, desc.dtype, _here()
    px, ldx = _matrix(x, rows, M, t, "x", dev)
    pr, ldr = _matrix(res, rows, M, t, "res", dev)
    ps, lds = _matrix(sum_out, rows, M, t, "sum_out", dev)
    py, ldy = _matrix(y, rows, M, desc.y_dtype, "y", dev)
    _check(_lib().fw_rmsnorm_forward(C.byref(desc), rows, px, ldx, pr, ldr, _vector(w, M, "w", dev), ps, lds, py, ldy,
                                     _vector(y_scale, rows, "y_scale", dev), _vector(rstd, rows, "rstd", dev), stream), "fw_rmsnorm_forward")


def fw_rmsnorm_backward(desc: fw_norm_desc, dy, s, w, rstd, dx, dw=None, dsum=None, scratch=None, stream: int = 0) -> None:
    rows, M, t, dev = dy.shape[0], desc.M, desc.dtype, _here()
    if scratch is not None and not scratch.is_contiguous():
        raise ValueError("scratch: its bytes have to be contiguous")
    pdy, lddy = _matrix(dy, rows, M, t, "dy", dev)
    ps, lds = _matrix(s, rows, M, t, "s", dev)
    pds, ldds = _matrix(dsum, rows, M, t, "dsum", dev)
    pdx, lddx = _matrix(dx, rows, M, t, "dx", dev)
    n = 0
    if scratch is not None:
        if scratch.get_device() != dev:
            _refuse_device(scratch, dev, "scratch")
        n = scratch.numel() * scratch.element_size()
    _check(_lib().fw_rmsnorm_backward(C.byref(desc), rows, pdy, lddy, ps, lds, pds, ldds, _vector(w, M, "w", dev),
                                      _vector(rstd, rows, "rstd", dev), pdx, lddx, _vector(dw, M, "dw", dev), _ptr(scratch), n, stream),
           "fw_rmsnorm_backward")


def fw_distill_desc_default(V: int, K: int, **overrides) -> fw_distill_desc:
    d = fw_distill_desc()
    _lib().fw_distill_desc_default(C.byref(d), V, K)
    return _override(d, overrides)


def fw_distill_forward(desc: fw_distill_desc, Z, T, I, loss, stat=None, t_lse=None, weight=None, dZ=None, stream: int = 0) -> None:
    rows, V, K, dev = Z.shape[0], desc.V, desc.K, _here()
    pz, ldz = _matrix(Z, rows, V, desc.z_dtype, "Z", dev)
    pd, lddz = _matrix(dZ, rows, V, desc.z_dtype, "dZ", dev)
    _check(_lib().fw_distill_forward(C.byref(desc), pz, rows, ldz, _vector(T, rows * K, "T", dev, desc.t_dtype),
                                     _vector(I, rows * K, "I", dev, "int64" if desc.index_bits == 64 else "int32"),
                                     _vector(t_lse, rows, "t_lse", dev), _vector(weight, rows, "weight", dev), _vector(loss, rows, "loss", dev),
                                     _vector(stat, 2 * rows, "stat", dev), pd, lddz, stream), "fw_distill_forward")


def fw_distill_backward(desc: fw_distill_desc, Z, T, I, stat, dZ, t_lse=None, weight=None, stream: int = 0) -> None:
    rows, V, K, dev = Z.shape[0], desc.V, desc.K, _here()
    pz, ldz = _matrix(Z, rows, V, desc.z_dtype, "Z", dev)
    pd, lddz = _matrix(dZ, rows, V, desc.z_dtype, "dZ", dev)
    _check(_lib().fw_distill_backward(C.byref(desc), pz, rows, ldz, _vector(T, rows * K, "T", dev, desc.t_dtype),
                                      _vector(I, rows * K, "I", dev, "int64" if desc.index_bits == 64 else "int32"),
                                      _vector(t_lse, rows, "t_lse", dev), _vector(weight, rows, "weight", dev),
                                      _vector(stat, 2 * rows, "stat", dev), pd, lddz, stream), "fw_distill_backward")


def fw_sandwich_desc_default(M: int, **overrides) -> fw_sandwich_desc:
    d = fw_sandwich_desc()
    _lib().fw_sandwich_desc_default(C.byref(d), M)
    return _override(d, overrides)


def fw_sandwich_scratch_bytes(desc: fw_sandwich_desc) -> int:
    return int(_lib().fw_sandwich_scratch_bytes(C.byref(desc)))


def fw_sandwich_forward(desc: fw_sandwich_desc, o, x, w_pre, h, y, w_post=None, gate=None, y_scale=None, rstd=None, stream: int = 0) -> None:
    rows, M, t, dev = o.shape[0], desc.M, desc.dtype, _here()
    po, ldo = _matrix(o, rows, M, t, "o", dev)
    px, ldx = _matrix(x, rows, M, t, "x", dev)
    ph, ldh = _matrix(h, rows, M, t, "h", dev)
    py, ldy = _matrix(y, rows, M, desc.y_dtype, "y", dev)
    _check(_lib().fw_sandwich_forward(C.byref(desc), rows, po, ldo, px, ldx, _vector(w_post, M, "w_post", dev), _vector(gate, rows, "gate", dev),
                                      _vector(w_pre, M, "w_pre", dev), ph, ldh, py, ldy, _vector(y_scale, rows, "y_scale", dev),
                                      _vector(rstd, 2 * rows, "rstd", dev), stream), "fw_sandwich_forward")


def fw_sandwich_backward(desc: fw_sandwich_desc, dy, o, h, w_pre, rstd, dx, d_o, w_post=None, gate=None, dh=None, dw_post=None, dw_pre=None,
                         dgate=None, scratch=None, stream: int = 0) -> None:
    rows, M, t, dev = dy.shape[0], desc.M, desc.dtype, _here()
    if scratch is not None and not scratch.is_contiguous():
        raise ValueError("scratch: its bytes have to be contiguous")
    pdy, lddy = _matrix(dy, rows, M, t, "dy", dev)
    pdh, lddh = _matrix(dh, rows, M, t, "dh", dev)
    po, ldo = _matrix(o, rows, M, t, "o", dev)
    ph, ldh = _matrix(h, rows, M, t, "h", dev)
    pdx, lddx = _matrix(dx, rows, M, t, "dx", dev)
    pdo, lddo = _matrix(d_o, rows, M, t, "d_o", dev)
    n = 0
    if scratch is not None:
        if scratch.get_device() != dev:
            _refuse_device(scratch, dev, "scratch")
        n = scratch.numel() * scratch.element_size()
    _check(_lib().fw_sandwich_backward(C.byref(desc), rows, pdy, lddy, pdh, lddh, po, ldo, ph, ldh, _vector(w_post, M, "w_post", dev),
                                       _vector(gate, rows, "gate", dev), _vector(w_pre, M, "w_pre", dev), _vector(rstd, 2 * rows, "rstd", dev),
                                       pdx, lddx, pdo, lddo, _vector(dw_post, M, "dw_post", dev), _vector(dw_pre, M, "dw_pre", dev),
                                       _vector(dgate, rows, "dgate", dev), _ptr(scratch), n, stream), "fw_sandwich_backward")


def fw_logprob_desc_default(V: int, **overrides) -> fw_logprob_desc:
    d = fw_logprob_desc()
    _lib().fw_logprob_desc_default(C.byref(d), V)
    return _override(d, overrides)


def _classes(desc, id, rows, dev):
    return _vector(id, rows, "id", dev, "int64" if desc.index_bits == 64 else "int32")


def fw_logprob_forward(desc: fw_logprob_desc, Z, id, logp, stat=None, stream: int = 0) -> None:
    rows, dev = Z.shape[0], _here()
    pz, ldz = _matrix(Z, rows, desc.V, desc.z_dtype, "Z", dev)
    _check(_lib().fw_logprob_forward(C.byref(desc), pz, rows, ldz, _classes(desc, id, rows, dev), _vector(logp, rows, "logp", dev),
                                     _vector(stat, 2 * rows, "stat", dev), stream), "fw_logprob_forward")


def fw_logprob_backward(desc: fw_logprob_desc, Z, id, stat, dlogp, dZ, stream: int = 0) -> None:
    rows, dev = Z.shape[0], _here()
    pz, ldz = _matrix(Z, rows, desc.V, desc.z_dtype, "Z", dev)
    pd, lddz = _matrix(dZ, rows, desc.V, desc.z_dtype, "dZ", dev)
    _check(_lib().fw_logprob_backward(C.byref(desc), pz, rows, ldz, _classes(desc, id, rows, dev), _vector(stat, 2 * rows, "stat", dev),
                                      _vector(dlogp, rows, "dlogp", dev), pd, lddz, stream), "fw_logprob_backward")


def fw_policy_desc_default(**overrides) -> fw_policy_desc:
    p = fw_policy_desc()
    _lib().fw_policy_desc_default(C.byref(p))
    return _override(p, overrides)


def fw_policy_forward(desc: fw_logprob_desc, policy: fw_policy_desc, Z, id, logp_old, adv, loss, logp_ref=None, weight=None, logp=None,
                      stat=None, dlogp=None, dZ=None, stream: int = 0) -> None:
    rows, dev = Z.shape[0], _here()
    pz, ldz = _matrix(Z, rows, desc.V, desc.z_dtype, "Z", dev)
    pd, lddz = _matrix(dZ, rows, desc.V, desc.z_dtype, "dZ", dev)
    v = lambda t, name: _vector(t, rows, name, dev)  # noqa: E731
    _check(_lib().fw_policy_forward(C.byref(desc), C.byref(policy), pz, rows, ldz, _classes(desc, id, rows, dev), v(logp_old, "logp_old"),
                                    v(logp_ref, "logp_ref"), v(adv, "adv"), v(weight, "weight"), v(loss, "loss"), v(logp, "logp"),
                                    _vector(stat, 2 * rows, "stat", dev), v(dlogp, "dlogp"), pd, lddz, stream), "fw_policy_forward")


def fw_preference_desc_default(**overrides) -> fw_preference_desc:
    p = fw_preference_desc()
    _lib().fw_preference_desc_default(C.byref(p))
    return _override(p, overrides)


def fw_preference_loss(desc: fw_logprob_desc, preference: fw_preference_desc, logp, id, seq, loss, ref=None, weight=None, sums=None,
                       dlogp=None, stream: int = 0) -> None:
    rows, pairs, dev = logp.numel(), loss.numel(), _here()
    _check(_lib().fw_preference_loss(C.byref(desc), C.byref(preference), _vector(logp, rows, "logp", dev), rows,
                                     _classes(desc, id, rows, dev), _vector(seq, 2 * pairs + 1, "seq", dev, "int32"), pairs,
                                     _vector(ref, 2 * pairs, "ref", dev), _vector(weight, pairs, "weight", dev),
                                     _vector(loss, pairs, "loss", dev), _vector(sums, 2 * pairs, "sums", dev),
                                     _vector(dlogp, rows, "dlogp", dev), stream), "fw_preference_loss")


# ---- objects that own a workspace tensor ----
def _workspace(n: int, device, stream: int):
    """Memory for work on `stream`: taken from the allocator, and given back, as that stream's own.  Of the current stream's memory the
    owner before may have work pending, which would write over what this stream puts there."""
    import torch
    if torch.device(device).type != "cuda":
        return torch.empty(n, dtype=torch.uint8, device=device)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()):
        return torch.empty(n, dtype=torch.uint8, device=device)


# ---- convenience: a layer that owns its workspace tensor -------------------
class Layer:
    """Holds the torch workspace tensor (device memory plumbing) and the handle.
    Methods forward to the C entry points of the same name."""

    def __init__(self, M: int, N: int, device="cuda", stream: int = 0, **desc_overrides):
        self.desc = fw_layer_desc_default(M, N, **desc_overrides)
        self.M, self.N = M, N
        self.nbytes = fw_layer_workspace_bytes(self.desc)
        if self.nbytes == 0:
            raise FwError(FW_ERR_INVALID_ARG, "fw_layer_workspace_bytes")
        self.workspace = _workspace(self.nbytes + 256, device, stream)
        base = self.workspace.data_ptr()
        self._base = (base + 255) // 256 * 256
        self.handle = fw_layer_create(self.desc, self._base, self.nbytes, stream)
        self.device = device

    def close(self):
        if getattr(self, "handle", None):
            fw_layer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reset(self):
        fw_layer_reset(self.handle)

    def attach_params(self, W, b):
        fw_layer_attach_params(self.handle, W, b)

    def cov_update(self, X, flags: int = FW_COV_COMMIT):
        fw_cov_update(self.handle, X, X.shape[0], X.stride(0), flags)

    def cond_reduce(self, K, P, trace=None):
        fw_cond_reduce(self.handle, K, P, trace)

    def grad_transform(self, G, out=None):
        import torch
        out = torch.empty_like(G) if out is None else out
        fw_grad_transform(self.handle, G, out)
        return out

    def step(self, W, b, G_t, g_b, lr):
        fw_step(self.handle, W, b, G_t, g_b, lr)

    def get(self, field):
        import torch
        M = self.M
        n = 1 if field == FW_F_LAMBDA_BAR else (M if field in (FW_F_MU, FW_F_PHI_DIAG, FW_F_ALIGN_W) else M * M)
        out = torch.empty(n, dtype=torch.float32, device=self.device)
        fw_layer_get(self.handle, field, out, n * 4)
        return out.view(M, M) if n == M * M and M > 1 else out

    def set(self, field, t):
        t = t.contiguous()
        fw_layer_set(self.handle, field, t, t.numel() * 4)

    def sync_status(self):
        return fw_layer_sync_status(self.handle)


class Gated:
    """A gated feed-forward block over a workspace tensor of its own.  Methods take torch CUDA tensors, look at their sizes,
    strides and types, and forward to the C entry points fw_gated_*.  The stream outlives the block."""

    def __init__(self, M: int, N: int, max_rows: int = 0, device="cuda", stream: int = 0, **desc_overrides):
        self.desc = fw_gated_desc()
        _lib().fw_gated_desc_default(C.byref(self.desc), M, N)
        self.desc.max_rows = max_rows
        _override(self.desc, {k: int(v) for k, v in desc_overrides.items()})
        self.M, self.N = M, N
        self.nbytes = int(_lib().fw_gated_workspace_bytes(C.byref(self.desc)))
        if self.nbytes == 0:
            raise FwError(FW_ERR_INVALID_ARG, "fw_gated_workspace_bytes")
        dev = _here()
        self.workspace = _workspace(self.nbytes + 256, device, stream)
        if not self.workspace.is_cuda or self.workspace.get_device() != dev:
            _refuse_device(self.workspace, dev, "workspace")
        out = C.c_void_p()
        _check(_lib().fw_gated_create(C.byref(self.desc), (self.workspace.data_ptr() + 255) // 256 * 256, self.nbytes, stream,
                                      C.byref(out)), "fw_gated_create")
        self.handle = out.value

    def close(self):
        if getattr(self, "handle", None):
            _check(_lib().fw_gated_destroy(self.handle), "fw_gated_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def forward(self, X, Wg, Wu, H, Zg=None, Zu=None, x_scale=None, wg_scale=None, wu_scale=None, bg=None, bu=None):
        M, N, t, rows, dev = self.M, self.N, self.desc.x_dtype, X.shape[0], _here()
        px, ldx = _matrix(X, rows, M, t, "X", dev)
        pg, pu, ldw = _pair(Wg, Wu, N, M, t, "Wg, Wu", dev)
        ph, ldh = _matrix(H, rows, N, FW_BF16, "H", dev)
        zg, zu, ldz = _pair(Zg, Zu, rows, N, FW_BF16, "Zg, Zu", dev)
        _check(_lib().fw_gated_forward(self.handle, px, rows, ldx, _vector(x_scale, rows, "x_scale", dev), pg, pu, ldw,
                                       _vector(wg_scale, N, "wg_scale", dev), _vector(wu_scale, N, "wu_scale", dev), _vector(bg, N, "bg", dev),
                                       _vector(bu, N, "bu", dev), ph, ldh, zg, zu, ldz), "fw_gated_forward")

    def backward(self, dH, X, Wg, Wu, Zg, Zu, dX=None, dWg=None, dWu=None, dbg=None, dbu=None):
        M, N, rows, dev = self.M, self.N, dH.shape[0], _here()
        pd, lddh = _matrix(dH, rows, N, FW_BF16, "dH", dev)
        px, ldx = _matrix(X, rows, M, FW_BF16, "X", dev)
        pg, pu, ldw = _pair(Wg, Wu, N, M, FW_BF16, "Wg, Wu", dev)
        zg, zu, ldz = _pair(Zg, Zu, rows, N, FW_BF16, "Zg, Zu", dev)
        pdx, lddx = _matrix(dX, rows, M, FW_BF16, "dX", dev)
        kind = FW_F32
        if dWg is not None:
            import torch
            kind = FW_BF16 if dWg.dtype == torch.bfloat16 else FW_F32
        _check(_lib().fw_gated_backward(self.handle, pd, rows, lddh, px, ldx, pg, pu, ldw, zg, zu, ldz, pdx, lddx,
                                        _vector(dWg, N * M, "dWg", dev, kind), _vector(dWu, N * M, "dWu", dev, kind), kind,
                                        _vector(dbg, N, "dbg", dev), _vector(dbu, N, "dbu", dev)), "fw_gated_backward")

    def sync_status(self):
        return _check(_lib().fw_gated_sync_status(self.handle), "fw_gated_sync_status")


class _Grads:
    """Gradients that an AdamW has looked at: their addresses and types, and the tensors, which stay."""

    def __init__(self, owner, tensors, pointers, kinds):
        self.owner, self.tensors, self.pointers, self.kinds = owner, tensors, pointers, kinds


class AdamW:
    """AdamW over the fp32 tensors `params` of a network, over a workspace tensor of its own.  copies: None, or for each parameter
    a bf16 tensor of its shape or None; decay: weight decay of each (one number: of all).  Methods look at their tensors and forward
    to the C entry points fw_adamw_*.  Parameters and copies are kept; the stream outlives the object."""

    def __init__(self, params, copies=None, decay=None, stream: int = 0, **desc_overrides):
        params = list(params)
        n = len(params)
        copies = [None] * n if copies is None else list(copies)
        decay = [float(decay or 0.0)] * n if decay is None or isinstance(decay, (int, float)) else [float(x) for x in decay]
        if len(copies) != n or len(decay) != n:
            raise ValueError(f"copies, decay: expected one for each of {n} parameters")
        self.desc = fw_adamw_desc()
        _lib().fw_adamw_desc_default(C.byref(self.desc), n)
        _override(self.desc, desc_overrides)
        if self.desc.n != n:
            raise ValueError(f"n: {n} parameters are given")
        dev = _here()
        for i, (p, c) in enumerate(zip(params, copies)):
            _vector(p, p.numel(), f"params[{i}]", dev)
            if c is not None:
                _vector(c, p.numel(), f"copies[{i}]", dev, FW_BF16)
                if c.shape != p.shape:
                    raise ValueError(f"copies[{i}]: expected {tuple(p.shape)}, got {tuple(c.shape)}")
        self.params, self.copies = params, copies
        sizes = (C.c_int64 * max(n, 1))(*[p.numel() for p in params])
        self.nbytes = int(_lib().fw_adamw_workspace_bytes(C.byref(self.desc), sizes))
        if self.nbytes == 0:
            raise FwError(FW_ERR_INVALID_ARG, "fw_adamw_workspace_bytes")
        self.workspace = _workspace(self.nbytes + 256, "cuda", stream)
        out = C.c_void_p()
        _check(_lib().fw_adamw_create(C.byref(self.desc), sizes, _vp_array(params), _vp_array(copies), (C.c_float * n)(*decay),
                                      (self.workspace.data_ptr() + 255) // 256 * 256, self.nbytes, stream, C.byref(out)), "fw_adamw_create")
        self.handle = out.value

    def close(self):
        if getattr(self, "handle", None):
            _check(_lib().fw_adamw_destroy(self.handle), "fw_adamw_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def grads(self, tensors):
        """The gradients, one for each parameter, looked at once: buffers that are written again for every step need it once."""
        tensors = list(tensors)
        if len(tensors) != len(self.params):
            raise ValueError(f"grads: expected {len(self.params)}, got {len(tensors)}")
        dev, n = _here(), len(tensors)
        pointers, kinds = (C.c_void_p * n)(), (C.c_int32 * n)()
        half = _TYPES[FW_BF16]
        for i, (t, p) in enumerate(zip(tensors, self.params)):
            if t is None or t.shape != p.shape:
                raise ValueError(f"grads[{i}]: expected {tuple(p.shape)}, got {None if t is None else tuple(t.shape)}")
            kinds[i] = FW_BF16 if t.dtype is half else FW_F32
            pointers[i] = _vector(t, p.numel(), f"grads[{i}]", dev, kinds[i])
        return _Grads(self, tensors, pointers, kinds)

    def step(self, grads, lr: float, lr_factor=None, max_norm: float = 0.0, norm_out=None):
        """grads: a list of tensors, or what grads() gave for it."""
        if not isinstance(grads, _Grads):
            grads = self.grads(grads)
        elif grads.owner is not self:
            raise ValueError("grads: looked at by another AdamW")
        dev = _here()
        _check(_lib().fw_adamw_step(self.handle, grads.pointers, grads.kinds, lr, _vector(lr_factor, 1, "lr_factor", dev), max_norm,
                                    _vector(norm_out, 1, "norm_out", dev)), "fw_adamw_step")

    def state(self, field: int):
        """A part of the workspace as a tensor (FW_A_*), for checkpoints: read or written between steps, on this object's stream."""
        import torch
        at, n = C.c_void_p(), C.c_size_t()
        _check(_lib().fw_adamw_state(self.handle, field, C.byref(at), C.byref(n)), "fw_adamw_state")
        first = at.value - self.workspace.data_ptr()
        kind = (torch.int64 if field == FW_A_STEP else torch.float8_e8m0fnu if field in (FW_A_M_SCALE, FW_A_V_SCALE)
                else torch.float32 if self.desc.state == FW_F32 else torch.float8_e4m3fn)
        return self.workspace[first:first + n.value].view(kind)

    def sync_status(self) -> int:
        """FW_OK, or FW_WARN_NONFINITE where a step has been left out; raises on errors."""
        return _check(_lib().fw_adamw_sync_status(self.handle), "fw_adamw_sync_status", allow=(FW_WARN_NONFINITE,))
