"""ctypes binding of libaloco (include/aloco.h).

Argument marshalling only: every step of the round runs inside the
library's CUDA kernels.  If the compiled library is missing this module
raises on first use; there is no fallback path.
"""
from __future__ import annotations

import array
import ctypes
import functools
import operator
import os
import struct
from dataclasses import dataclass
from typing import NamedTuple, Optional, Sequence

MAX_WORKERS = 32
MAX_VOCAB = 262144
MAX_TOP = 32
MAX_NS_STEPS = 16
MAX_SIDE, MAX_LONG_SIDE = 16384, 1048576

F32, BF16 = 0, 1
SCHED_COSINE, SCHED_CONSTANT, SCHED_LINEAR = 0, 1, 2
CORR_FULL, CORR_MOMENTUM_ONLY, CORR_NONE = 0, 1, 2
PASS_AUTO, PASS_REGISTERS, PASS_BULK_COPY = 0, 1, 2
PASS_INT8_SPLIT, PASS_INT8_FUSED = 3, 4
PASS_TILE = 5
WAIT_SPIN, WAIT_BLOCK = 0, 1
MUON_ADAMW, MUON_ASPECT, MUON_UNIT = 0, 1, 2

OK = 0
ERR_ARG = -1
ERR_CUDA = -2
ERR_NONFINITE = -3
ERR_ALIAS = -4
ERR_NOMEM = -5

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)),
                         "libaloco.so")

# Names declared in include/aloco.h (checked by the ABI test).
EXPORTS = ("aloco_default_opts", "aloco_inner_lr_accum", "aloco_correction",
           "aloco_sync", "aloco_sync_ex", "aloco_sync_noalloc", "aloco_sync_host",
           "aloco_sync_shard", "aloco_sync_int8_shard", "aloco_combine_partials",
           "aloco_sync_int8", "aloco_int8_num_blocks", "aloco_int8_encode",
           "aloco_int8_decode", "aloco_adamw_default_cfg", "aloco_adamw_step",
           "aloco_adamw_step_normed",
           "aloco_muon_default_cfg", "aloco_muon_scratch_bytes", "aloco_muon_step",
           "aloco_orthogonalize_scratch_bytes", "aloco_orthogonalize",
           "aloco_token_scores", "aloco_token_scores_grad",
           "aloco_token_logprobs", "aloco_loss_scratch_bytes", "aloco_policy_loss",
           "aloco_preference_loss", "aloco_grads_create", "aloco_grads_destroy",
           "aloco_grad_norm", "aloco_clip_grads", "aloco_grads_scratch_bytes",
           "aloco_grad_norm_in", "aloco_clip_grads_in",
           "aloco_ctrl_default_cfg", "aloco_ctrl_init", "aloco_select_interval",
           "aloco_ctrl_state_bytes", "aloco_ctrl_save", "aloco_ctrl_load",
           "aloco_test_stall_tile", "aloco_last_error", "aloco_shutdown",
           "aloco_version")

CTRL_HISTORY = 16
ASSESS_NONE, ASSESS_SUPPORTED, ASSESS_CONSISTENT, ASSESS_MODERATE, \
    ASSESS_SEVERE, ASSESS_INVALID = range(6)
PHASE_WARMUP, PHASE_REFERENCE, PHASE_VARIABILITY, PHASE_MONITOR, \
    PHASE_CANDIDATE, PHASE_CONFIRM = range(6)


class Schedule(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("peak_lr", ctypes.c_double), ("final_lr", ctypes.c_double),
                ("warmup_steps", ctypes.c_int64),
                ("total_steps", ctypes.c_int64)]

    @classmethod
    def make(cls, kind=SCHED_COSINE, peak_lr=4e-4, final_lr=4e-5,
             warmup_steps=1000, total_steps=20000):
        return cls(kind, 0, peak_lr, final_lr, warmup_steps, total_steps)


class Opts(ctypes.Structure):
    _fields_ = [("mu_min", ctypes.c_double), ("mu_max", ctypes.c_double),
                ("kappa_max", ctypes.c_double), ("eps", ctypes.c_double),
                ("normalize", ctypes.c_int32), ("mode", ctypes.c_int32),
                ("time_kernel", ctypes.c_int32),
                ("blocks_per_sm", ctypes.c_int32),
                ("stream", ctypes.c_void_p), ("pass_", ctypes.c_int32),
                ("wait", ctypes.c_int32)]


class AdamwCfg(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double),
                ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double),
                ("max_grad_norm", ctypes.c_double), ("step", ctypes.c_int64)]


class AdamwStats(ctypes.Structure):
    _fields_ = [("grad_norm", ctypes.c_double * MAX_WORKERS),
                ("clip", ctypes.c_double * MAX_WORKERS),
                ("M", ctypes.c_int32), ("grid", ctypes.c_int32),
                ("kernel_ms", ctypes.c_float), ("reserved", ctypes.c_int32)]

    def as_dict(self):
        return {"grad_norm": list(self.grad_norm[:self.M]),
                "clip": list(self.clip[:self.M]), "M": self.M,
                "grid": self.grid, "kernel_ms": self.kernel_ms}


class Matrix(ctypes.Structure):
    _fields_ = [("offset", ctypes.c_int64), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


class MuonCfg(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("momentum", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("eps", ctypes.c_double),
                ("nesterov", ctypes.c_int32), ("scale", ctypes.c_int32),
                ("steps", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("coefficients", ctypes.c_double * 3 * MAX_NS_STEPS)]


class Tokens(ctypes.Structure):
    """aloco_tokens_t: logits and their tokens."""
    _fields_ = [("logits", ctypes.c_void_p), ("targets", ctypes.c_void_p),
                ("batch", ctypes.c_int64), ("rows", ctypes.c_int64),
                ("vocab", ctypes.c_int64), ("batch_stride", ctypes.c_int64),
                ("row_stride", ctypes.c_int64), ("temperature", ctypes.c_double),
                ("dtype", ctypes.c_int32), ("target_bytes", ctypes.c_int32)]


class LogitsGrad(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64),
                ("row_stride", ctypes.c_int64)]


class PolicyCfg(ctypes.Structure):
    _fields_ = [("clip_low", ctypes.c_double), ("clip_high", ctypes.c_double),
                ("kl_coef", ctypes.c_double)]


class PreferenceCfg(ctypes.Structure):
    _fields_ = [("beta", ctypes.c_double), ("label_smoothing", ctypes.c_double)]


class Correction(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in
                ("lam_sel", "lam_base", "rho_unc", "rho", "mu_t", "kappa_t",
                 "eta_out", "inv_norm")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class Stats(ctypes.Structure):
    _fields_ = [("D", ctypes.c_double), ("C", ctypes.c_double),
                ("mean_sq_norm", ctypes.c_double),
                ("drift", ctypes.c_double * MAX_WORKERS),
                ("corr", Correction), ("nonfinite", ctypes.c_int64),
                ("M", ctypes.c_int32), ("grid", ctypes.c_int32),
                ("kernel_ms", ctypes.c_float), ("pass_used", ctypes.c_int32)]

    def as_dict(self):
        # one unpack of the struct: reading the fields one by one through
        # ctypes costs several microseconds a call
        f = _STATS.unpack_from(self)
        M = f[_AT_M]
        return {"D": f[0], "C": f[1], "mean_sq_norm": f[2],
                "drift": list(f[3:3 + M]),
                "corr": dict(zip(_CORR_NAMES, f[3 + MAX_WORKERS:_AT_M - 1])),
                "nonfinite": f[_AT_M - 1], "M": M, "grid": f[_AT_M + 1],
                "kernel_ms": f[_AT_M + 2], "pass_used": f[_AT_M + 3]}


_CORR_NAMES = tuple(n for n, _ in Correction._fields_)
_STATS = struct.Struct("=%ddqiifi" % (3 + MAX_WORKERS + len(_CORR_NAMES)))
_AT_M = 3 + MAX_WORKERS + len(_CORR_NAMES) + 1  # index of M in the unpacked fields
assert _STATS.size == ctypes.sizeof(Stats)


class Partials(ctypes.Structure):
    """aloco_partials_t: one shard's partial sums of a round."""
    _fields_ = [("drift", ctypes.c_double * MAX_WORKERS),
                ("sum_sq", ctypes.c_double), ("sq_scale", ctypes.c_double),
                ("eps", ctypes.c_double), ("corr", Correction),
                ("nonfinite", ctypes.c_int64), ("n", ctypes.c_int64),
                ("M", ctypes.c_int32), ("pass_used", ctypes.c_int32),
                ("kernel_ms", ctypes.c_float), ("reserved", ctypes.c_int32)]

    def to_bytes(self) -> bytes:
        return ctypes.string_at(ctypes.addressof(self), ctypes.sizeof(self))

    @classmethod
    def from_bytes(cls, blob: bytes) -> "Partials":
        if len(blob) != ctypes.sizeof(cls):
            raise ValueError(f"partials blob of {len(blob)} bytes, want "
                             f"{ctypes.sizeof(cls)}")
        return cls.from_buffer_copy(blob)


_i64, _i32, _dbl = ctypes.c_int64, ctypes.c_int32, ctypes.c_double


class CtrlCfg(ctypes.Structure):
    _fields_ = [("H_base", _i64), ("H_min", _i64), ("H_max", _i64),
                ("q_H", _i64), ("warmup_steps", _i64), ("beta_tok", _dbl),
                ("thr_candidate", _dbl), ("thr_moderate", _dbl),
                ("thr_severe", _dbl), ("exposure_mult", _dbl),
                ("div_moderate", _dbl), ("div_severe", _dbl),
                ("retire_frac", _dbl), ("ref_ema", _dbl), ("mad_scale", _dbl),
                ("scale_floor", _dbl), ("eps", _dbl),
                ("mapper_bootstrap", _i32), ("ref_bootstrap", _i32),
                ("variability_intervals", _i32), ("severe_fallback", _i32)]


class CtrlState(ctypes.Structure):
    _fields_ = [("version", _i32), ("phase", _i32), ("intervals", _i64),
                ("H_acc", _i64), ("H_next", _i64), ("H_cand", _i64),
                ("bound", _i64), ("bound_lam", _dbl), ("phase_count", _i32),
                ("ref_needed", _i32), ("moderate_run", _i32),
                ("severe_run", _i32), ("log_D_ref", _dbl),
                ("log_C_ref", _dbl), ("lam_ref", _dbl), ("sum_log_D", _dbl),
                ("sum_log_C", _dbl), ("n_hist", _i32), ("head", _i32),
                ("hist_D", _dbl * CTRL_HISTORY),
                ("hist_C", _dbl * CTRL_HISTORY), ("mapper_n", _i32),
                ("calibrated", _i32), ("mapper_mass", _dbl * 8),
                ("M_base", _dbl), ("n_hat", _dbl), ("last_z", _dbl),
                ("last_r_D", _dbl), ("last_r_C", _dbl),
                ("last_assessment", _i32), ("referenced", _i32)]


class IntervalObs(ctypes.Structure):
    _fields_ = [("D", _dbl), ("C", _dbl), ("lam", _dbl), ("tokens", _dbl),
                ("H_step", _i64), ("step_end", _i64)]


class CtrlDecision(ctypes.Structure):
    _fields_ = [("H_tok", _i64), ("H_step", _i64), ("H_ref_step", _i64),
                ("assessment", _i32), ("phase", _i32), ("z", _dbl),
                ("r_D", _dbl), ("r_C", _dbl)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class AlocoError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"aloco status {status}: {message}")
        self.status = status


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load():
    """Load libaloco.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with "
            "`python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i64, i32, dbl = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, \
        ctypes.c_double
    lib.aloco_default_opts.argtypes = [ctypes.POINTER(Opts)]
    lib.aloco_default_opts.restype = None
    lib.aloco_inner_lr_accum.argtypes = [ctypes.POINTER(Schedule), i64, i64]
    lib.aloco_inner_lr_accum.restype = dbl
    lib.aloco_correction.argtypes = [ctypes.POINTER(Schedule), i64, i64, i64,
                                     dbl, dbl, ctypes.POINTER(Opts),
                                     ctypes.POINTER(Correction)]
    lib.aloco_correction.restype = i32
    sync_args = [vp, vp, ctypes.POINTER(vp), ctypes.c_size_t, i32, i32, i64,
                 i64, i64, ctypes.POINTER(Schedule), dbl, dbl]
    lib.aloco_sync.argtypes = sync_args + [ctypes.POINTER(Stats)]
    lib.aloco_sync.restype = i32
    lib.aloco_sync_ex.argtypes = sync_args + [ctypes.POINTER(Opts),
                                              ctypes.POINTER(Stats)]
    lib.aloco_sync_ex.restype = i32
    lib.aloco_sync_noalloc.argtypes = sync_args + [ctypes.POINTER(Opts),
                                                   ctypes.POINTER(Stats)]
    lib.aloco_sync_noalloc.restype = i32
    P = ctypes.POINTER
    lib.aloco_sync_int8.argtypes = sync_args + [vp, i32, P(Opts), P(Stats)]
    lib.aloco_sync_int8.restype = i32
    lib.aloco_adamw_default_cfg.argtypes = [P(AdamwCfg)]
    lib.aloco_adamw_default_cfg.restype = None
    lib.aloco_adamw_step.argtypes = [vp, vp, vp, vp, ctypes.c_size_t, i32,
                                     i32, i32, P(AdamwCfg), P(Opts),
                                     P(AdamwStats)]
    lib.aloco_adamw_step.restype = i32
    lib.aloco_adamw_step_normed.argtypes = [vp, vp, vp, vp, ctypes.c_size_t, i32,
                                            i32, i32, P(AdamwCfg), vp, P(Opts),
                                            P(AdamwStats)]
    lib.aloco_adamw_step_normed.restype = i32
    lib.aloco_token_logprobs.argtypes = [P(Tokens), vp, P(Opts)]
    lib.aloco_token_logprobs.restype = i32
    lib.aloco_loss_scratch_bytes.argtypes = [i64]
    lib.aloco_loss_scratch_bytes.restype = ctypes.c_size_t
    lib.aloco_policy_loss.argtypes = [P(Tokens), vp, vp, vp, vp, P(PolicyCfg), vp, vp,
                                      P(LogitsGrad), vp, ctypes.c_size_t, P(Opts)]
    lib.aloco_policy_loss.restype = i32
    lib.aloco_preference_loss.argtypes = [P(Tokens), vp, vp, ctypes.c_int32, i64,
                                          P(PreferenceCfg), vp, vp, vp, P(LogitsGrad), vp,
                                          ctypes.c_size_t, P(Opts)]
    lib.aloco_preference_loss.restype = i32
    lib.aloco_grads_create.argtypes = [vp, vp, vp, i64, P(vp)]
    lib.aloco_grads_create.restype = i32
    lib.aloco_grads_destroy.argtypes = [vp]
    lib.aloco_grads_destroy.restype = None
    lib.aloco_grad_norm.argtypes = [vp, vp, P(Opts)]
    lib.aloco_grad_norm.restype = i32
    lib.aloco_clip_grads.argtypes = [vp, dbl, vp, i32, vp, P(Opts)]
    lib.aloco_clip_grads.restype = i32
    lib.aloco_grads_scratch_bytes.argtypes = [vp]
    lib.aloco_grads_scratch_bytes.restype = ctypes.c_size_t
    lib.aloco_grad_norm_in.argtypes = [vp, vp, vp, ctypes.c_size_t, P(Opts)]
    lib.aloco_grad_norm_in.restype = i32
    lib.aloco_clip_grads_in.argtypes = [vp, dbl, vp, i32, vp, vp, ctypes.c_size_t, P(Opts)]
    lib.aloco_clip_grads_in.restype = i32
    lib.aloco_token_scores.argtypes = [P(Tokens), i32, vp, vp, vp, vp, vp, P(Opts)]
    lib.aloco_token_scores.restype = i32
    lib.aloco_token_scores_grad.argtypes = [P(Tokens), vp, vp, vp, vp, i32, vp, vp,
                                            P(LogitsGrad), P(Opts)]
    lib.aloco_token_scores_grad.restype = i32
    lib.aloco_muon_default_cfg.argtypes = [P(MuonCfg)]
    lib.aloco_muon_default_cfg.restype = None
    lib.aloco_muon_scratch_bytes.argtypes = [P(Matrix), i64, i32]
    lib.aloco_muon_scratch_bytes.restype = ctypes.c_size_t
    lib.aloco_muon_step.argtypes = [vp, vp, vp, ctypes.c_size_t, i32, i32, i32, P(Matrix), i64,
                                    P(MuonCfg), vp, ctypes.c_size_t, P(Opts)]
    lib.aloco_muon_step.restype = i32
    lib.aloco_orthogonalize_scratch_bytes.argtypes = [i64, i64, i64]
    lib.aloco_orthogonalize_scratch_bytes.restype = ctypes.c_size_t
    lib.aloco_orthogonalize.argtypes = [vp, i64, i64, i64, i64, i64, i32, vp, vp, i32, dbl, vp,
                                        ctypes.c_size_t, P(Opts)]
    lib.aloco_orthogonalize.restype = i32
    lib.aloco_sync_host.argtypes = sync_args + [ctypes.c_size_t, P(Opts), P(Stats)]
    lib.aloco_sync_host.restype = i32
    lib.aloco_sync_shard.argtypes = sync_args + [P(Opts), P(Partials)]
    lib.aloco_sync_shard.restype = i32
    lib.aloco_sync_int8_shard.argtypes = sync_args + [vp, i32, P(Opts), P(Partials)]
    lib.aloco_sync_int8_shard.restype = i32
    lib.aloco_combine_partials.argtypes = [vp, i32, P(Stats)]
    lib.aloco_combine_partials.restype = i32
    lib.aloco_test_stall_tile.argtypes = [i64]
    lib.aloco_test_stall_tile.restype = None
    lib.aloco_int8_num_blocks.argtypes = [vp, i32]
    lib.aloco_int8_num_blocks.restype = i64
    lib.aloco_int8_encode.argtypes = [vp, ctypes.c_size_t, vp, i32, vp, vp, vp,
                                      vp]
    lib.aloco_int8_encode.restype = i32
    lib.aloco_int8_decode.argtypes = [vp, vp, ctypes.c_size_t, vp, i32, vp, vp]
    lib.aloco_int8_decode.restype = i32
    lib.aloco_ctrl_default_cfg.argtypes = [P(CtrlCfg), i64, i64, i64, i64,
                                           i64]
    lib.aloco_ctrl_default_cfg.restype = None
    lib.aloco_ctrl_init.argtypes = [P(CtrlState), P(CtrlCfg),
                                    P(CtrlDecision)]
    lib.aloco_ctrl_init.restype = i32
    lib.aloco_select_interval.argtypes = [P(CtrlState), P(CtrlCfg),
                                          P(IntervalObs), P(Schedule),
                                          P(CtrlDecision)]
    lib.aloco_select_interval.restype = i32
    lib.aloco_ctrl_state_bytes.argtypes = []
    lib.aloco_ctrl_state_bytes.restype = ctypes.c_size_t
    lib.aloco_ctrl_save.argtypes = [P(CtrlState), vp, ctypes.c_size_t]
    lib.aloco_ctrl_save.restype = i32
    lib.aloco_ctrl_load.argtypes = [P(CtrlState), vp, ctypes.c_size_t]
    lib.aloco_ctrl_load.restype = i32
    lib.aloco_last_error.argtypes = []
    lib.aloco_last_error.restype = ctypes.c_char_p
    lib.aloco_shutdown.argtypes = []
    lib.aloco_shutdown.restype = None
    lib.aloco_version.argtypes = []
    lib.aloco_version.restype = i32
    _lib = lib
    return lib


def last_error() -> str:
    return load().aloco_last_error().decode()


def default_opts(**kw) -> Opts:
    o = Opts()
    load().aloco_default_opts(ctypes.byref(o))
    for k, val in kw.items():
        setattr(o, k, val)
    return o


def inner_lr_accum(schedule: Schedule, t0: int, H: int) -> float:
    return load().aloco_inner_lr_accum(ctypes.byref(schedule), t0, H)


def correction(schedule: Schedule, step: int, H_sel: int, H_base: int,
               outer_lr: float, outer_beta: float,
               opts: Optional[Opts] = None) -> Correction:
    out = Correction()
    rc = load().aloco_correction(ctypes.byref(schedule), step, H_sel, H_base,
                                 outer_lr, outer_beta,
                                 ctypes.byref(opts) if opts else None,
                                 ctypes.byref(out))
    if rc != OK:
        raise AlocoError(rc, last_error())
    return out


def _stream_of(stream, device) -> int:
    """The raw handle of `stream`, or of the device's current stream."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    if device.index is None:
        return torch.cuda.current_stream(device).cuda_stream
    return torch._C._cuda_getCurrentRawStream(device.index)


class _NoSwitch:
    def __enter__(self):
        pass

    def __exit__(self, *exc):
        return False


_NO_SWITCH = _NoSwitch()


def _on_device(device):
    """A context with `device` current; nothing to do where it already is."""
    import torch
    if torch.cuda.current_device() == device.index:
        return _NO_SWITCH
    return torch.cuda.device(device)


def _pointers(tensors):
    return (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


def sync_ptrs(g_ptr: int, v_ptr: int, x_ptrs: Sequence[int], N: int,
              dtype: int, H_sel: int, H_base: int, step: int,
              schedule: Schedule, outer_lr: float, outer_beta: float,
              opts: Optional[Opts] = None, raise_on_error: bool = True,
              noalloc: bool = False):
    """aloco_sync_ex (or, with noalloc=True, aloco_sync_noalloc) on raw
    device addresses.  Returns (status, Stats)."""
    M = len(x_ptrs)
    arr = (ctypes.c_void_p * max(M, 1))(*x_ptrs)
    st = Stats()
    fn = load().aloco_sync_noalloc if noalloc else load().aloco_sync_ex
    rc = fn(g_ptr, v_ptr, arr, N, M, dtype, H_sel, H_base,
                              step, ctypes.byref(schedule), outer_lr,
                              outer_beta,
                              ctypes.byref(opts) if opts is not None else None,
                              ctypes.byref(st))
    if raise_on_error and rc not in (OK, ERR_NONFINITE):
        raise AlocoError(rc, last_error())
    return rc, st


def sync(global_, momentum, locals_, *, H_sel: int, H_base: int, step: int,
         schedule: Schedule, outer_lr: float, outer_beta: float,
         opts: Optional[Opts] = None, stream=None, raise_on_error=True,
         noalloc: bool = False):
    """One outer synchronisation round on torch CUDA tensors, in place.

    global_, momentum: contiguous float32 [N]; locals_: M contiguous tensors
    [N] of float32 or bfloat16.  The round runs on `stream` (default: the
    current torch stream).  noalloc=True calls aloco_sync_noalloc, the entry
    point that allocates nothing (its scratch is a static device array)."""
    import torch
    N = global_.numel()
    rdt = locals_[0].dtype if locals_ else None
    if not (global_.dtype == momentum.dtype == torch.float32
            and momentum.numel() == N and rdt in (torch.float32, torch.bfloat16)
            and all([t.is_cuda and t.is_contiguous() for t in (global_, momentum)])
            and all([x.dtype == rdt and x.numel() == N and x.is_cuda
                     and x.is_contiguous() for x in locals_])):
        _refuse_round(global_, momentum, locals_)
    dtype = F32 if rdt == torch.float32 else BF16
    if opts is None:
        opts = default_opts()
    device = global_.device
    opts.stream = _stream_of(stream, device)
    with _on_device(device):
        rc, st = sync_ptrs(global_.data_ptr(), momentum.data_ptr(),
                           [x.data_ptr() for x in locals_], N, dtype, H_sel,
                           H_base, step, schedule, outer_lr, outer_beta, opts,
                           raise_on_error, noalloc)
    out = st.as_dict()
    out["status"] = rc
    return out


def _refuse_round(global_, momentum, locals_):
    """Raise what is wrong with sync()'s tensors."""
    import torch
    if global_.dtype != torch.float32 or momentum.dtype != torch.float32:
        raise TypeError("global and momentum must be float32")
    N = global_.numel()
    if momentum.numel() != N or any(x.numel() != N for x in locals_):
        raise ValueError("all buffers must have the same number of elements")
    if not locals_:
        raise ValueError("need at least one replica")
    rdt = locals_[0].dtype
    if any(x.dtype != rdt for x in locals_):
        raise TypeError("replicas must share one dtype")
    if rdt not in (torch.float32, torch.bfloat16):
        raise TypeError(f"unsupported replica dtype {rdt}")
    raise ValueError("buffers must be contiguous CUDA tensors")


def shutdown():
    if _lib is not None:
        _lib.aloco_shutdown()


# ------------------------------------------------------------ sharded rounds

def _replica_dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported replica dtype {t.dtype}")


def sync_shard(global_, momentum, locals_, *, H_sel: int, H_base: int,
               step: int, schedule: Schedule, outer_lr: float,
               outer_beta: float, opts: Optional[Opts] = None, stream=None,
               raise_on_error=True, parts=None, int8: bool = False):
    """One shard of a round on torch CUDA tensors (views of the shard's
    elements), in place: aloco_sync_shard, or aloco_sync_int8_shard with
    int8=True (parts: the shard's tensor parts).  Returns (status,
    Partials)."""
    N = global_.numel()
    if momentum.numel() != N or any([x.numel() != N for x in locals_]):
        raise ValueError("all buffers must have the same number of elements")
    for t in (global_, momentum, *locals_):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("buffers must be contiguous CUDA tensors")
    dtype = _replica_dtype_code(locals_[0])
    if opts is None:
        opts = default_opts()
    opts.stream = _stream_of(stream, global_.device)
    M = len(locals_)
    ptrs = _pointers(locals_)
    out = Partials()
    with _on_device(global_.device):
        if int8:
            arr, n = _parts_array(parts)
            rc = load().aloco_sync_int8_shard(
                global_.data_ptr(), momentum.data_ptr(), ptrs, N, M, dtype,
                H_sel, H_base, step, ctypes.byref(schedule), outer_lr,
                outer_beta, arr, n, ctypes.byref(opts), ctypes.byref(out))
        else:
            rc = load().aloco_sync_shard(
                global_.data_ptr(), momentum.data_ptr(), ptrs, N, M, dtype,
                H_sel, H_base, step, ctypes.byref(schedule), outer_lr,
                outer_beta, ctypes.byref(opts), ctypes.byref(out))
    if raise_on_error and rc not in (OK, ERR_NONFINITE):
        raise AlocoError(rc, last_error())
    return rc, out


def combine_partials(shards: Sequence[Partials], raise_on_error=True):
    """aloco_combine_partials over the shards in the given order (host
    only).  Returns the statistics dict with "status"."""
    n = len(shards)
    arr = (Partials * max(n, 1))(*shards)
    st = Stats()
    rc = load().aloco_combine_partials(arr if n else None, n,
                                       ctypes.byref(st))
    if raise_on_error and rc not in (OK, ERR_NONFINITE):
        raise AlocoError(rc, last_error())
    return st.as_dict() | {"status": rc}


class Controller:
    """The host interval controller (aloco_select_interval) with its state
    and settings."""

    def __init__(self, H_base: int, H_min: int, H_max: int, q_H: int,
                 warmup_steps: int, schedule: Schedule, **overrides):
        lib = load()
        self.cfg = CtrlCfg()
        lib.aloco_ctrl_default_cfg(ctypes.byref(self.cfg), H_base, H_min,
                                   H_max, q_H, warmup_steps)
        for k, val in overrides.items():
            setattr(self.cfg, k, val)
        self.schedule = schedule
        self.state = CtrlState()
        d = CtrlDecision()
        rc = lib.aloco_ctrl_init(ctypes.byref(self.state),
                                 ctypes.byref(self.cfg), ctypes.byref(d))
        if rc != OK:
            raise AlocoError(rc, last_error())
        self.decision = d

    def observe(self, D: float, C: float, lam: float, tokens: float,
                H_step: int, step_end: int) -> CtrlDecision:
        obs = IntervalObs(D, C, lam, tokens, H_step, step_end)
        d = CtrlDecision()
        rc = load().aloco_select_interval(
            ctypes.byref(self.state), ctypes.byref(self.cfg),
            ctypes.byref(obs), ctypes.byref(self.schedule), ctypes.byref(d))
        if rc != OK:
            raise AlocoError(rc, last_error())
        self.decision = d
        return d

    def save(self) -> bytes:
        n = load().aloco_ctrl_state_bytes()
        buf = ctypes.create_string_buffer(n)
        rc = load().aloco_ctrl_save(ctypes.byref(self.state), buf, n)
        if rc != OK:
            raise AlocoError(rc, last_error())
        return buf.raw

    def load_state(self, blob: bytes):
        buf = ctypes.create_string_buffer(blob, len(blob))
        rc = load().aloco_ctrl_load(ctypes.byref(self.state), buf, len(blob))
        if rc != OK:
            raise AlocoError(rc, last_error())


# ------------------------------------------------ INT8 communication (App. G.1)

def _parts_array(parts):
    if parts is None:
        return None, 0
    sizes = [int(p) for p in parts]
    try:
        arr = (ctypes.c_int64 * len(sizes)).from_buffer(array.array("q", sizes))
    except OverflowError:  # wraps, and the library refuses what comes of it
        arr = (ctypes.c_int64 * len(sizes))(*sizes)
    return arr, len(sizes)


def int8_num_blocks(parts) -> int:
    arr, n = _parts_array(parts)
    nb = load().aloco_int8_num_blocks(arr, n)
    if nb < 0:
        raise AlocoError(ERR_ARG, last_error())
    return nb


def int8_payload_bytes(parts) -> int:
    """Bytes one worker sends per sync: the codes plus one fp32 scale per
    block."""
    return int(sum(parts)) + 4 * int8_num_blocks(parts)


def int8_encode(x, parts=None, want_decoded=True, stream=None):
    """Blockwise INT8 codec of a contiguous float32 CUDA tensor; returns
    (codes int8, scales float32, decoded float32 or None)."""
    import torch
    if x.dtype != torch.float32 or not x.is_cuda or not x.is_contiguous():
        raise TypeError("x must be a contiguous float32 CUDA tensor")
    N = x.numel()
    nb = int8_num_blocks(parts if parts is not None else [N])
    codes = torch.empty(N, dtype=torch.int8, device=x.device)
    scales = torch.empty(nb, dtype=torch.float32, device=x.device)
    dec = torch.empty_like(x) if want_decoded else None
    arr, n = _parts_array(parts)
    with _on_device(x.device):
        rc = load().aloco_int8_encode(x.data_ptr(), N, arr, n,
                                      codes.data_ptr(), scales.data_ptr(),
                                      dec.data_ptr() if dec is not None
                                      else None, _stream_of(stream, x.device))
    if rc != OK:
        raise AlocoError(rc, last_error())
    return codes, scales, dec


def int8_decode(codes, scales, parts=None, stream=None):
    import torch
    N = codes.numel()
    out = torch.empty(N, dtype=torch.float32, device=codes.device)
    arr, n = _parts_array(parts)
    with _on_device(codes.device):
        rc = load().aloco_int8_decode(codes.data_ptr(), scales.data_ptr(), N,
                                      arr, n, out.data_ptr(),
                                      _stream_of(stream, codes.device))
    if rc != OK:
        raise AlocoError(rc, last_error())
    return out


def sync_host(global_, momentum, locals_, *, H_sel: int, H_base: int,
              step: int, schedule: Schedule, outer_lr: float,
              outer_beta: float, chunk_elems: int = 0,
              opts: Optional[Opts] = None, stream=None, raise_on_error=True):
    """aloco_sync_host on page-locked torch CPU tensors (theta, v updated in
    place; the replicas are read only)."""
    import torch
    N = global_.numel()
    dtype = F32 if locals_[0].dtype == torch.float32 else BF16
    if opts is None:
        opts = default_opts()
    s = stream if stream is not None else torch.cuda.current_stream()
    opts.stream = s.cuda_stream
    M = len(locals_)
    ptrs = (ctypes.c_void_p * M)(*[x.data_ptr() for x in locals_])
    st = Stats()
    rc = load().aloco_sync_host(global_.data_ptr(), momentum.data_ptr(), ptrs, N,
                                M, dtype, H_sel, H_base, step,
                                ctypes.byref(schedule), outer_lr, outer_beta,
                                chunk_elems, ctypes.byref(opts), ctypes.byref(st))
    if raise_on_error and rc not in (OK, ERR_NONFINITE):
        raise AlocoError(rc, last_error())
    return st.as_dict() | {"status": rc}


def sync_int8(global_, momentum, locals_, *, parts=None, H_sel: int,
              H_base: int, step: int, schedule: Schedule, outer_lr: float,
              outer_beta: float, opts: Optional[Opts] = None, stream=None,
              raise_on_error=True):
    """One outer round with INT8-communicated pseudo-gradients (in place on
    torch CUDA tensors, like sync())."""
    import torch
    N = global_.numel()
    rdt = locals_[0].dtype
    dtype = F32 if rdt == torch.float32 else BF16
    if opts is None:
        opts = default_opts()
    opts.stream = _stream_of(stream, global_.device)
    M = len(locals_)
    ptrs = _pointers(locals_)
    arr, n = _parts_array(parts)
    st = Stats()
    with _on_device(global_.device):
        rc = load().aloco_sync_int8(global_.data_ptr(), momentum.data_ptr(),
                                    ptrs, N, M, dtype, H_sel, H_base, step,
                                    ctypes.byref(schedule), outer_lr,
                                    outer_beta, arr, n, ctypes.byref(opts),
                                    ctypes.byref(st))
    if raise_on_error and rc not in (OK, ERR_NONFINITE):
        raise AlocoError(rc, last_error())
    out = st.as_dict()
    out["status"] = rc
    return out


# ----------------------------------------------------- inner AdamW (Sec. 2)

def adamw_cfg(**kw) -> AdamwCfg:
    """The library's default AdamW settings (C4 pre-training) with the given
    fields replaced."""
    c = AdamwCfg()
    load().aloco_adamw_default_cfg(ctypes.byref(c))
    for k, v in kw.items():
        if not hasattr(c, k):
            raise TypeError(f"unknown AdamW setting {k!r}")
        setattr(c, k, v)
    return c


def adamw_step(params, grads, exp_avg, exp_avg_sq, cfg: AdamwCfg,
               opts: Optional[Opts] = None, stream=None, want_stats=True,
               raise_on_error=True, grad_norms=None):
    """One AdamW step on every replica, in place (lists of torch CUDA tensors
    of one device: params and grads fp32 or bf16, moments fp32).  With
    grad_norms (M floats, the gradients' norms) the step takes them instead
    of computing them (aloco_adamw_step_normed).  Returns the per-replica
    gradient norms and clipping factors (want_stats), else None without
    waiting for the GPU."""
    import torch
    M = len(params)
    if not (len(grads) == len(exp_avg) == len(exp_avg_sq) == M):
        raise ValueError("params, grads and moments need one tensor per replica")
    N = params[0].numel()
    pdt = F32 if params[0].dtype == torch.float32 else BF16
    gdt = F32 if grads[0].dtype == torch.float32 else BF16
    if opts is None:
        opts = default_opts()
    opts.stream = _stream_of(stream, params[0].device)
    arr = _pointers
    st = AdamwStats() if want_stats else None
    with _on_device(params[0].device):
        if grad_norms is None:
            rc = load().aloco_adamw_step(arr(params), arr(grads), arr(exp_avg),
                                         arr(exp_avg_sq), N, M, pdt, gdt,
                                         ctypes.byref(cfg), ctypes.byref(opts),
                                         ctypes.byref(st) if st is not None else None)
        else:
            norms = (ctypes.c_double * M)(*[float(x) for x in grad_norms])
            rc = load().aloco_adamw_step_normed(
                arr(params), arr(grads), arr(exp_avg), arr(exp_avg_sq), N, M, pdt,
                gdt, ctypes.byref(cfg), norms, ctypes.byref(opts),
                ctypes.byref(st) if st is not None else None)
    if raise_on_error and rc != OK:
        raise AlocoError(rc, last_error())
    if st is None:
        return rc if not raise_on_error else None
    return st.as_dict() | {"status": rc}


# --------------------------------------------------- orthogonalised updates

# a, b, c of the steps X <- (a + b A + c A A) X, A = X X^T, that the default
# settings take five times.
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)


def muon_cfg(**kw) -> MuonCfg:
    """The library's default settings of muon_step with the given fields
    replaced; `coefficients` is a sequence of (a, b, c), one for every step of
    the orthogonal factor."""
    c = MuonCfg()
    load().aloco_muon_default_cfg(ctypes.byref(c))
    if "coefficients" in kw:
        steps = [tuple(float(x) for x in s) for s in kw.pop("coefficients")]
        if not 1 <= len(steps) <= MAX_NS_STEPS or any(len(s) != 3 for s in steps):
            raise ValueError(f"coefficients must be 1 to {MAX_NS_STEPS} triples")
        c.steps = len(steps)
        for i, s in enumerate(steps):
            c.coefficients[i][:] = s
    for k, v in kw.items():
        if not hasattr(c, k):
            raise TypeError(f"unknown muon setting {k!r}")
        setattr(c, k, v)
    return c


class Matrices:
    """The matrices of a replica's vector: (offset, rows, columns) of each, kept
    for muon_step step after step."""

    def __init__(self, parts):
        self.parts = [tuple(operator.index(x) for x in p) for p in parts]
        self.array = (Matrix * len(self.parts))(*self.parts)
        self._need = {}

    def scratch_bytes(self, workers: int) -> int:
        need = self._need.get(workers)
        if need is None:
            need = load().aloco_muon_scratch_bytes(self.array, len(self.parts), workers)
            self._need[workers] = need
        return need


def _scratch_of(need, device):
    """Device memory of a call, from the current stream's pool (whose blocks start
    on 512-byte boundaries)."""
    return _torch.empty(need, dtype=_torch.uint8, device=device)


def muon_step(params, grads, momentum, matrices, cfg: MuonCfg, stream=None):
    """One step of the matrices of every replica along the orthogonal factor of
    their momentum, in place (aloco_muon_step): lists of flat contiguous CUDA
    tensors of one device, params and grads fp32 or bf16, momentum fp32.
    `matrices`: a Matrices, or a sequence of (offset, rows, columns); what they do
    not cover is left alone.  Enqueues only; what it writes counts as written in
    place."""
    torch = _torch_module()
    M = len(params)
    if not M or not (len(grads) == len(momentum) == M):
        raise ValueError("params, grads and momentum need one tensor per replica")
    if not isinstance(matrices, Matrices):
        matrices = Matrices(matrices)
    device, N = params[0].device, params[0].numel()
    for name, ts, dtypes in (("params", params, (torch.float32, torch.bfloat16)),
                             ("grads", grads, (torch.float32, torch.bfloat16)),
                             ("momentum", momentum, (torch.float32,))):
        for t in ts:
            if t.dtype not in dtypes or t.dtype is not ts[0].dtype:
                raise TypeError(f"unsupported or mixed {name} dtype {t.dtype}")
            if t.device != device or not t.is_cuda or t.numel() != N or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous CUDA tensors of one size and device")
    ctx, handle = _on_stream(stream, device, (*params, *grads, *momentum))
    lib = load()
    with ctx:
        need = matrices.scratch_bytes(M)
        scratch = _scratch_of(need, device) if need else None
        rc = lib.aloco_muon_step(
            _pointers(params), _pointers(grads), _pointers(momentum), N, M,
            F32 if params[0].dtype is torch.float32 else BF16,
            F32 if grads[0].dtype is torch.float32 else BF16, matrices.array,
            len(matrices.parts), ctypes.byref(cfg), scratch.data_ptr() if need else None, need,
            ctypes.byref(Opts(stream=handle)))
    _finish(rc, ctx)
    _written([*params, *momentum])


@functools.lru_cache(maxsize=32)
def _steps(coefficients):
    """The C array of a tuple of tuples (a, b, c)."""
    if any(len(s) != 3 for s in coefficients):
        raise ValueError("coefficients must be triples")
    return (ctypes.c_double * (3 * len(coefficients)))(*[float(v) for s in coefficients for v in s])


def orthogonalize(x, *, coefficients=(NEWTON_SCHULZ,) * 5, eps: float = 1e-7, out=None,
                  stream=None):
    """Orthogonal factors of matrices [rows, columns] or [batch, rows, columns]
    (float32 or bfloat16 CUDA tensor with contiguous rows, any strides of the other
    dimensions) by Newton-Schulz steps, one for every (a, b, c) of `coefficients`
    (aloco_orthogonalize).  Returns bfloat16 of x's shape, or fills `out`, a
    contiguous one.  Enqueues only."""
    torch = _torch_module()
    if x.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"matrices must be float32 or bfloat16, not {x.dtype}")
    if x.dim() not in (2, 3):
        raise ValueError("need [rows, columns] or [batch, rows, columns]")
    if not x.is_cuda or (x.stride(-1) != 1 and x.shape[-1] > 1):
        raise ValueError("need a CUDA tensor with contiguous rows")
    steps = _steps(tuple(map(tuple, coefficients)))
    if out is not None and (out.dtype is not torch.bfloat16 or out.shape != x.shape or
                            out.device != x.device or not out.is_contiguous()):
        raise ValueError("out must be a contiguous bfloat16 tensor of x's shape and device")
    rows, cols = x.shape[-2:]
    batch = x.shape[0] if x.dim() == 3 else 1
    device = x.device
    ctx, handle = _on_stream(stream, device, (x, out))
    lib = load()
    with ctx:
        result = torch.empty(x.shape, dtype=torch.bfloat16, device=device) if out is None else out
        need = lib.aloco_orthogonalize_scratch_bytes(batch, rows, cols)
        scratch = _scratch_of(need, device) if need else None
        rc = lib.aloco_orthogonalize(
            x.data_ptr(), batch, rows, cols, x.stride(0) if x.dim() == 3 else 0, x.stride(-2),
            F32 if x.dtype is torch.float32 else BF16, result.data_ptr(),
            steps, len(steps) // 3, eps, scratch.data_ptr() if need else None, need,
            ctypes.byref(Opts(stream=handle)))
    _finish(rc, ctx, result)
    if out is not None:
        _written(out)
    return result


def test_stall_tile(tile: int):
    """Testing only: the next bulk-copy round (post-training loss, orthogonal
    factor or muon step) on this thread skips the copies of one tile, so that its
    bounded wait runs out; a tile below -1 makes a loss's first copy so many cycles
    late (aloco_test_stall_tile)."""
    load().aloco_test_stall_tile(int(tile))


# -------------------------------------------- post-training losses and gradients

class TokenScores(NamedTuple):
    """logp, entropy: float32, in targets' shape; top_ids: int32, and top_logp:
    float32, [..., top], the largest logits first and equal ones by their index
    (None for top = 0); stats: float32 [..., 2], what token_scores_grad needs of
    a row (its largest logit and sum)."""
    logp: object
    entropy: object
    top_ids: object
    top_logp: object
    stats: object


class PolicyLoss(NamedTuple):
    """terms: float32 [4] (the loss, its policy term, its KL term before the
    coefficient, the weight of the clipped rows); logp: float32, the tokens'
    log-probabilities; grad: the gradient by the logits, or None."""
    terms: object
    logp: object
    grad: object


class PreferenceLoss(NamedTuple):
    """loss: float32 scalar; log_ratios: float32 [2 pairs], the sequences' sums
    of logp - ref_logp; logp: float32, the tokens' log-probabilities; grad: the
    gradient by the logits, or None."""
    loss: object
    log_ratios: object
    logp: object
    grad: object


class _OtherStream:
    """The context of a call on a stream that is not the current one: what the
    call allocates belongs to that stream, and the memory of what it is given
    or returns is not handed out again before both are past it."""

    def __init__(self, stream, current, inputs):
        self.current = current
        self.stream = stream
        self.inner = _torch.cuda.stream(stream)
        self.inputs = inputs

    def __enter__(self):
        self.inner.__enter__()

    def __exit__(self, *exc):
        self.inner.__exit__(*exc)
        for t in self.inputs:
            if t is not None:
                t.record_stream(self.stream)
        return False


def _on_stream(stream, device, inputs):
    """(context, raw stream handle) of a call."""
    torch = _torch_module()
    if stream is not None:
        current = torch.cuda.current_stream(device)
        if stream != current:
            return _OtherStream(stream, current, inputs), stream.cuda_stream
    index = device.index
    handle = torch._C._cuda_getCurrentRawStream(index)
    if torch._C._cuda_getDevice() == index:
        return _NO_SWITCH, handle
    return torch.cuda.device(device), handle


def _finish(rc, ctx, *outputs):
    """Raise what a call reported; hand its outputs to the current stream."""
    if rc != OK:
        raise AlocoError(rc, last_error())
    if ctx.__class__ is _OtherStream:
        for t in outputs:
            if t is not None:
                t.record_stream(ctx.current)


def _written(tensors):
    """Tell autograd that a call has written into the caller's tensors (or
    tensor): a backward pass that saved one of them is refused then, as after an
    in-place operation of torch's own."""
    _torch.autograd.graph.increment_version(tensors)


_torch = None


def _torch_module():
    """torch, imported on first use (an import statement in every call costs
    more than the lookup)."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _tokens(logits, targets, temperature) -> Tokens:
    """The descriptor of [rows, V] or [batch, rows, V] logits and their targets."""
    torch = _torch_module()
    dtype = logits.dtype
    if dtype is torch.bfloat16:
        code = BF16
    elif dtype is torch.float32:
        code = F32
    else:
        raise TypeError(f"logits must be float32 or bfloat16, not {dtype}")
    shape, strides = logits.shape, logits.stride()
    if len(shape) == 3:
        batch, rows, vocab = shape
        batch_stride, row_stride, last = strides
    elif len(shape) == 2:
        (rows, vocab), batch = shape, 1
        batch_stride, (row_stride, last) = 0, strides
    else:
        raise ValueError("logits must be [rows, vocab] or [batch, rows, vocab]")
    if last != 1 and vocab > 1:
        raise ValueError("the logits of a row must be contiguous")
    if targets.dtype is torch.int64:
        size = 8
    elif targets.dtype is torch.int32:
        size = 4
    else:
        raise TypeError(f"targets must be int32 or int64, not {targets.dtype}")
    if targets.shape != shape[:-1] or not targets.is_contiguous():
        raise ValueError(f"targets must be contiguous of shape {tuple(shape[:-1])}")
    if not logits.is_cuda or targets.get_device() != logits.get_device():
        raise ValueError("logits and targets must be CUDA tensors of one device")
    return Tokens(logits.data_ptr(), targets.data_ptr(), batch, rows, vocab, batch_stride,
                  row_stride, temperature, code, size)


def _per_row(name, t, shape, index) -> int:
    """The address of a float32 tensor of one value per row, on device `index`."""
    if t.dtype is not _torch.float32 or t.shape != shape or t.get_device() != index or \
            not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor of shape "
                         f"{tuple(shape)} on the logits' device")
    return t.data_ptr()


def _logits_grad(logits, grad, want_grad):
    """(gradient tensor, its descriptor): `grad`, or a new one."""
    if grad is None:
        if not want_grad:
            return None, None
        grad = _torch.empty_like(logits)
    elif grad.dtype != logits.dtype or grad.shape != logits.shape or \
            grad.get_device() != logits.get_device() or \
            (grad.stride(-1) != 1 and grad.shape[-1] > 1):
        raise ValueError("grad must have the logits' shape, dtype and device, with "
                         "contiguous rows")
    st = grad.stride()
    return grad, ctypes.byref(LogitsGrad(grad.data_ptr(), st[0] if len(st) == 3 else 0, st[-2]))


def token_logprobs(logits, targets, *, temperature: float = 1.0, stream=None):
    """Log-probabilities of the tokens `targets` (int32 or int64, [rows] or
    [batch, rows]) under logits [..., V] / temperature (float32 or bfloat16 CUDA
    tensor with contiguous rows and any strides between them); 0 where a
    target is negative.  float32, in targets' shape."""
    tok = _tokens(logits, targets, temperature)
    device = logits.device
    ctx, handle = _on_stream(stream, device, (logits, targets))
    with ctx:
        logp = _torch.empty(targets.shape, dtype=_torch.float32, device=device)
        rc = load().aloco_token_logprobs(ctypes.byref(tok), logp.data_ptr(),
                                         ctypes.byref(Opts(stream=handle)))
    _finish(rc, ctx, logp)
    return logp


def token_scores(logits, targets, *, top: int = 0, temperature: float = 1.0,
                 stream=None) -> TokenScores:
    """Log-probabilities of the tokens `targets` with the entropy and the `top`
    (at most 32) best alternatives of every row (aloco_token_scores); logits and
    targets as token_logprobs takes them.  Enqueues only."""
    tok = _tokens(logits, targets, temperature)
    if not 0 <= top <= min(MAX_TOP, tok.vocab):
        raise ValueError(f"top = {top} outside [0, min(vocab, {MAX_TOP})]")
    device, shape = logits.device, targets.shape
    ctx, handle = _on_stream(stream, device, (logits, targets))
    with ctx:
        empty = _torch.empty
        logp = empty(shape, dtype=_torch.float32, device=device)
        entropy = empty(shape, dtype=_torch.float32, device=device)
        stats = empty((*shape, 2), dtype=_torch.float32, device=device)
        ids = best = None
        if top:
            ids = empty((*shape, top), dtype=_torch.int32, device=device)
            best = empty((*shape, top), dtype=_torch.float32, device=device)
        rc = load().aloco_token_scores(
            ctypes.byref(tok), top, logp.data_ptr(), entropy.data_ptr(),
            ids.data_ptr() if top else None, best.data_ptr() if top else None, stats.data_ptr(),
            ctypes.byref(Opts(stream=handle)))
    _finish(rc, ctx, logp, entropy, stats, ids, best)
    return TokenScores(logp, entropy, ids, best, stats)


def token_scores_grad(logits, targets, scores: TokenScores, *, d_logp=None, d_entropy=None,
                      d_top=None, temperature: float = 1.0, grad=None, stream=None):
    """Gradient by the logits of a loss over `scores` (token_scores' of the same
    logits, targets and temperature), from its gradients by their log-probabilities,
    entropies and alternatives' log-probabilities (float32 of their shapes; at
    least one is given).  `grad` (optional) receives it and may be `logits` itself;
    one that is given counts as written in place.  Enqueues only."""
    tok = _tokens(logits, targets, temperature)
    if d_logp is None and d_entropy is None and d_top is None:
        raise ValueError("need d_logp, d_entropy or d_top")
    device, shape, index = logits.device, targets.shape, logits.device.index
    stats = _per_row("scores.stats", scores.stats, (*shape, 2), index)
    by_logp = _per_row("d_logp", d_logp, shape, index) if d_logp is not None else None
    by_entropy = entropy = by_top = ids = None
    if d_entropy is not None:
        by_entropy = _per_row("d_entropy", d_entropy, shape, index)
        entropy = _per_row("scores.entropy", scores.entropy, shape, index)
    top = 0
    if d_top is not None:
        if scores.top_ids is None:
            raise ValueError("d_top needs scores with alternatives (top > 0)")
        top = scores.top_ids.shape[-1]
        by_top = _per_row("d_top", d_top, (*shape, top), index)
        t = scores.top_ids
        if t.dtype is not _torch.int32 or t.shape != (*shape, top) or \
                t.get_device() != index or not t.is_contiguous():
            raise ValueError("scores.top_ids must be contiguous int32 of shape "
                             f"{(*shape, top)} on the logits' device")
        ids = t.data_ptr()
    ctx, handle = _on_stream(stream, device, (logits, targets, *scores, d_logp, d_entropy, d_top,
                                              grad))
    with ctx:
        out, desc = _logits_grad(logits, grad, True)
        rc = load().aloco_token_scores_grad(
            ctypes.byref(tok), stats, entropy, by_logp, by_entropy, top, ids, by_top, desc,
            ctypes.byref(Opts(stream=handle)))
    _finish(rc, ctx, out)
    if grad is not None:
        _written(grad)
    return out


def policy_loss(logits, targets, advantages, old_logp, weights, *, ref_logp=None,
                clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                temperature: float = 1.0, grad=None, want_grad: bool = True,
                stream=None) -> PolicyLoss:
    """Clipped policy loss with a KL term over the rows of `logits`, and its
    gradient by them (aloco_policy_loss).  advantages, old_logp, weights and
    ref_logp are float32 of targets' shape; rows of weight 0 or a negative
    target take no part.  grad (optional) receives the gradient and may be
    `logits` itself; without it a new tensor does, unless want_grad is False.
    The terms are not part of an autograd graph: logits.backward(r.grad) goes on
    from the gradient.  (A grad that is given counts as written in place: a
    backward pass that needs what was there before is refused.)  Enqueues only."""
    tok = _tokens(logits, targets, temperature)
    device = logits.device
    shape, index = targets.shape, device.index
    adv = _per_row("advantages", advantages, shape, index)
    old = _per_row("old_logp", old_logp, shape, index)
    w = _per_row("weights", weights, shape, index)
    ref = _per_row("ref_logp", ref_logp, shape, index) if ref_logp is not None else None
    cfg = PolicyCfg(clip_low, clip_high, kl_coef)
    ctx, handle = _on_stream(stream, device, (logits, targets, advantages, old_logp, weights,
                                              ref_logp, grad))
    lib = load()
    with ctx:
        out, desc = _logits_grad(logits, grad, want_grad)
        logp = _torch.empty_like(old_logp)
        terms = _torch.empty(4, dtype=_torch.float32, device=device)
        need = lib.aloco_loss_scratch_bytes(tok.batch * tok.rows)
        scratch = _torch.empty(need, dtype=_torch.uint8, device=device)
        rc = lib.aloco_policy_loss(ctypes.byref(tok), adv, old, ref, w, ctypes.byref(cfg),
                                   terms.data_ptr(), logp.data_ptr(), desc, scratch.data_ptr(),
                                   need, ctypes.byref(Opts(stream=handle)))
    _finish(rc, ctx, terms, logp, out)
    if grad is not None:
        _written(grad)
    return PolicyLoss(terms, logp, out)


def preference_loss(logits, targets, cu_seqlens, ref_logp=None, *, beta: float = 0.1,
                    label_smoothing: float = 0.0, temperature: float = 1.0, grad=None,
                    want_grad: bool = True, stream=None) -> PreferenceLoss:
    """Preference loss of paired log ratios, and its gradient by the logits
    (aloco_preference_loss).  cu_seqlens (int32 or int64 CUDA tensor [2 pairs +
    1]) bounds the sequences among the rows taken in order, chosen and rejected
    answers in turn; rows with a negative target (prompts, padding) take no
    part.  ref_logp is float32 of targets' shape (None: no reference).  grad
    and want_grad as policy_loss, and so is the way on into a backward pass.
    Enqueues only."""
    tok = _tokens(logits, targets, temperature)
    device = logits.device
    ref = _per_row("ref_logp", ref_logp, targets.shape, device.index) \
        if ref_logp is not None else None
    if cu_seqlens.dtype is _torch.int32:
        cu_bytes = 4
    elif cu_seqlens.dtype is _torch.int64:
        cu_bytes = 8
    else:
        raise TypeError(f"cu_seqlens must be int32 or int64, not {cu_seqlens.dtype}")
    if cu_seqlens.dim() != 1 or cu_seqlens.numel() % 2 == 0 or \
            not cu_seqlens.is_contiguous() or cu_seqlens.get_device() != device.index:
        raise ValueError("cu_seqlens must be a contiguous vector of 2 pairs + 1 bounds on the "
                         "logits' device")
    pairs = cu_seqlens.numel() // 2
    cfg = PreferenceCfg(beta, label_smoothing)
    ctx, handle = _on_stream(stream, device, (logits, targets, cu_seqlens, ref_logp, grad))
    lib = load()
    with ctx:
        f32 = {"dtype": _torch.float32, "device": device}
        out, desc = _logits_grad(logits, grad, want_grad)
        loss = _torch.empty((), **f32)
        ratios = _torch.empty(2 * pairs, **f32)
        logp = _torch.empty(targets.shape, **f32)
        need = lib.aloco_loss_scratch_bytes(tok.batch * tok.rows)
        scratch = _torch.empty(need, dtype=_torch.uint8, device=device)
        rc = lib.aloco_preference_loss(
            ctypes.byref(tok), ref, cu_seqlens.data_ptr(), cu_bytes, pairs, ctypes.byref(cfg),
            loss.data_ptr(), ratios.data_ptr(), logp.data_ptr(), desc, scratch.data_ptr(), need,
            ctypes.byref(Opts(stream=handle)))
    _finish(rc, ctx, loss, ratios, logp, out)
    if grad is not None:
        _written(grad)
    return PreferenceLoss(loss, ratios, logp, out)


class _Owned:
    """Tensors that somebody holds besides Python, as a parameter holds its
    gradient (or a view its base), and whether one has lost its last such owner
    since the last call without having been written: its owner has another by
    then."""

    def __init__(self, tensors):
        self.seen = [(t, 0) for t in tensors if not t.is_inference()]
        self.take()

    def take(self):
        """Those that are owned now, with their versions."""
        self.seen = [(t, t._version) for t, _ in self.seen if t._use_count() > 1]

    def stale(self) -> bool:
        if not self.seen:
            return False
        if any(t._use_count() == 1 and t._version == v for t, v in self.seen):
            return True
        self.take()
        return False


# Handles of lists that are gone.  Freeing one waits for the device, which no
# stream that is being captured allows, and a list may be collected at any moment;
# they go when the next list is made, which waits for the device anyway.
_dropped_lists = []


class GradList:
    """The gradient tensors of one model (contiguous float32 or bfloat16 CUDA
    tensors of one device, in the order of the flat vector), kept for
    grad_norm and clip_grads step after step, on any stream.  It is a list of these tensors,
    which it holds, not of whatever takes their place: one whose memory has
    moved is refused, and so is one that its owner has let go of since the list
    was made or last used, if nothing has written to it since (zero_grad() drops
    a parameter's gradient, and the next backward pass makes another; with
    set_to_none=False it stays).  A graph that captured a call reads the
    tensors at every replay; they have to stay as for any captured call."""

    def __init__(self, tensors):
        import torch
        self._handle = None
        self._captured = False   # a graph reads the handle's table: it stays
        self.tensors = list(tensors)
        if not self.tensors:
            raise ValueError("need at least one gradient")
        self.device = self.tensors[0].device
        for t in self.tensors:
            if t.dtype not in (torch.float32, torch.bfloat16):
                raise TypeError(f"unsupported gradient dtype {t.dtype}")
            if not t.is_cuda or t.device != self.device or not t.is_contiguous():
                raise ValueError("gradients must be contiguous CUDA tensors of one device")
        n = len(self.tensors)
        self._pointers = [t.data_ptr for t in self.tensors]
        self._at = [p() for p in self._pointers]
        self._owned = _Owned(self.tensors)
        sizes = [t.numel() for t in self.tensors]
        self.numel = sum(sizes)
        handle = ctypes.c_void_p()
        with _on_device(self.device):
            while _dropped_lists:
                load().aloco_grads_destroy(_dropped_lists.pop())
            rc = load().aloco_grads_create(
                (ctypes.c_void_p * n)(*self._at), (ctypes.c_int64 * n)(*sizes),
                (ctypes.c_int32 * n)(*[_replica_dtype_code(t) for t in self.tensors]), n,
                ctypes.byref(handle))
        if rc != OK:
            raise AlocoError(rc, last_error())
        self._handle = handle
        self._need = load().aloco_grads_scratch_bytes(handle)
        self._kept = {}   # scratch by stream

    def _scratch(self, stream):
        """(tensor, address) of a call's scratch on `stream` (a raw handle, current):
        one for every stream, whose calls follow one another.  A captured call has
        its own, zeroed at every replay, which may run beside any other call."""
        capturing = _torch.cuda.is_current_stream_capturing()
        s = None if capturing else self._kept.get(stream)
        if s is None:
            t = _torch.zeros(self._need, dtype=_torch.uint8, device=self.device)
            s = t, t.data_ptr()
            if capturing:
                self._captured = True
            else:
                self._kept[stream] = s
        return s

    def _check(self):
        if [p() for p in self._pointers] != self._at:
            raise ValueError("a gradient's memory has moved since the GradList was made")
        if self._owned.stale():
            raise ValueError("a gradient has lost its owner and was not written since the last "
                             "call (zero_grad lets backward make gradients anew unless "
                             "set_to_none=False): make a new GradList")

    def __del__(self):
        if getattr(self, "_handle", None) is not None and _dropped_lists is not None:
            if not self._captured:
                _dropped_lists.append(self._handle)
            self._handle = None


def _grad_list(grads) -> GradList:
    if not isinstance(grads, GradList):
        return GradList(grads)
    grads._check()
    return grads


def grad_norm(grads, *, stream=None):
    """Global norm of a GradList: a float32 scalar tensor.  Enqueues only.  (A
    sequence of tensors does too, at the price of a list made for the call,
    which also waits for the GPU.)"""
    g = _grad_list(grads)
    ctx, handle = _on_stream(stream, g.device, g.tensors)
    with ctx:
        norm = _torch.empty((), dtype=_torch.float32, device=g.device)
        _scratch, at = g._scratch(handle)
        rc = load().aloco_grad_norm_in(g._handle, norm.data_ptr(), at, g._need,
                                       ctypes.byref(Opts(stream=handle)))
    _finish(rc, ctx, norm)
    return norm


def clip_grads(grads, max_norm: float, *, out=None, stream=None):
    """Scale the gradients by min(1, max_norm / (norm + 1e-6)): in place, or,
    with `out` (a contiguous float32 or bfloat16 vector of all their elements),
    into it, tensor after tensor, as adamw_step takes them.  Returns the norm
    before clipping, a float32 scalar tensor.  Enqueues only (grads as
    grad_norm takes them); what it writes counts as written in place."""
    g = _grad_list(grads)
    if out is not None and (out.numel() != g.numel or not out.is_contiguous() or
                            out.device != g.device):
        raise ValueError(f"out must be a contiguous vector of {g.numel} elements on the "
                         "gradients' device")
    dtype = _replica_dtype_code(out) if out is not None else F32
    ctx, handle = _on_stream(stream, g.device, g.tensors if out is None else [*g.tensors, out])
    with ctx:
        norm = _torch.empty((), dtype=_torch.float32, device=g.device)
        _scratch, at = g._scratch(handle)
        rc = load().aloco_clip_grads_in(g._handle, max_norm,
                                        out.data_ptr() if out is not None else None, dtype,
                                        norm.data_ptr(), at, g._need,
                                        ctypes.byref(Opts(stream=handle)))
    _finish(rc, ctx, norm)
    if out is not None:
        _written(out)
    else:
        _written(g.tensors)
        g._owned.take()
    return norm
