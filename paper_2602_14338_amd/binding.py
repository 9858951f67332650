"""ctypes binding of the C ABI: argument marshalling only, same names as the C entry points.

Tensors must live on the GPU; pointers are taken with ``data_ptr()`` and work is enqueued
on torch's current stream for that device.  Nothing here computes anything.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

AERO_F32, AERO_BF16, AERO_F16, AERO_F8E4M3 = 0, 1, 2, 3
AERO_ROW_PADDING, AERO_ROW_UNTOUCHED = -1, -2
AERO_DW_ACCUMULATE = 0x100
OP_GROUP_ADVANTAGE, OP_LOGPROB_FWD, OP_GRPO_LOSS_BWD, OP_LMHEAD_FUSED = 0, 1, 2, 3
OP_TOPK_LOGPROB, OP_DISTILL_LOSS_BWD, OP_VERIFY_DRAFT, OP_EMBEDDING_BWD = 4, 5, 6, 7
OP_PREFERENCE_LOSS, OP_PREFERENCE_LOSS_BWD, OP_GRAD_NORM = 8, 9, 10
AERO_TAIL_RENORM, AERO_TAIL_BUCKET = 0, 1
AERO_PAIR_LOGISTIC, AERO_PAIR_HINGE, AERO_PAIR_SQUARE = 0, 1, 2
AERO_MOMENT_BLOCK = 256
AERO_TOPK_MAX, AERO_DRAFT_MAX = 256, 63
AERO_LOGIT_LIMIT = 1.2e9   # of the calls around a drafter: masked at or below its negative, NaN at or above

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libaero_hip.so")


class AeroError(RuntimeError):
    pass


class _AdvParamsC(C.Structure):
    _fields_ = [("k_ratio", C.c_int32), ("s_rescue", C.c_int32), ("tau_num", C.c_int32),
                ("tau_den", C.c_int32), ("zero_keep", C.c_int32), ("reject_enable", C.c_int32),
                ("posterior_mode", C.c_int32), ("alpha0", C.c_float), ("beta0", C.c_float)]


@dataclass
class AdvParams:
    k_ratio: int = 1
    s_rescue: int = 0
    tau_num: int = 1
    tau_den: int = 2
    zero_keep: int = 4
    reject_enable: int = 0
    posterior_mode: int = 0
    alpha0: float = 1.0
    beta0: float = 1.0

    def to_c(self) -> _AdvParamsC:
        return _AdvParamsC(self.k_ratio, self.s_rescue, self.tau_num, self.tau_den, self.zero_keep,
                           self.reject_enable, self.posterior_mode, self.alpha0, self.beta0)


class _PreferenceParamsC(C.Structure):
    _fields_ = [("kind", C.c_int32), ("average", C.c_int32), ("beta", C.c_float), ("smoothing", C.c_float), ("margin", C.c_float)]


@dataclass
class PreferenceParams:
    kind: int = AERO_PAIR_LOGISTIC
    average: int = 0
    beta: float = 0.1
    smoothing: float = 0.0
    margin: float = 0.0

    def to_c(self) -> _PreferenceParamsC:
        return _PreferenceParamsC(self.kind, self.average, self.beta, self.smoothing, self.margin)


class _AdamWParamsC(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("seed", C.c_uint64), ("stochastic", C.c_int32)]


@dataclass
class AdamWParams:
    lr: float = 1e-3
    beta1: float = 0.9
    beta2: float = 0.999
    eps: float = 1e-8
    weight_decay: float = 0.01
    seed: int = 0
    stochastic: bool = False

    def to_c(self) -> _AdamWParamsC:
        return _AdamWParamsC(self.lr, self.beta1, self.beta2, self.eps, self.weight_decay, self.seed, int(bool(self.stochastic)))


class _TensorC(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("master", C.c_void_p), ("exp_avg", C.c_void_p), ("exp_avg_sq", C.c_void_p),
                ("exp_avg_scale", C.c_void_p), ("exp_avg_sq_scale", C.c_void_p), ("n", C.c_int64), ("param_dtype", C.c_int32),
                ("grad_dtype", C.c_int32), ("decay", C.c_float)]


def library_path() -> str:
    return _LIB_PATH


def _load() -> C.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise AeroError(f"{_LIB_PATH} is missing: build it with `python -m paper_2602_14338_amd.build` "
                        "(there is no fallback path)")
    lib = C.CDLL(_LIB_PATH)
    p, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
    lib.aero_status_string.restype = C.c_char_p
    lib.aero_status_string.argtypes = [i32]
    lib.aero_workspace_bytes.restype = sz
    lib.aero_workspace_bytes.argtypes = [i32, i64, i32, i32, i32, i32]
    lib.aero_group_advantage.restype = i32
    lib.aero_group_advantage.argtypes = [p, p, p, p, i32, i32, C.POINTER(_AdvParamsC)] + [p] * 7 + [p, p]
    lib.aero_logprob_fwd.restype = i32
    lib.aero_logprob_fwd.argtypes = [p, i32, i64, i32, i64, p, p, p, p, p, p, p]
    lib.aero_grpo_loss_bwd.restype = i32
    lib.aero_grpo_loss_bwd.argtypes = [p, i32, i64, i32, i64, p, p, p, p, p, p, p, i32, f32, f32, f32, f32, f32, p,
                                       p, p, p, p, p, p, p, p, sz, p]
    lib.aero_grpo_loss_bwd_noalloc.restype = i32
    lib.aero_grpo_loss_bwd_noalloc.argtypes = lib.aero_grpo_loss_bwd.argtypes[:-3] + [p]
    lib.aero_lmhead_logprob_fused.restype = i32
    lib.aero_lmhead_logprob_fused.argtypes = [p, p, i64, i32, i32, p, p, p, p, p, p, p, p, i32, f32, f32, f32, f32,
                                              f32, p, p, p, p, p, i32, p, p, sz, p]
    lib.aero_topk_logprob.restype = i32
    lib.aero_topk_logprob.argtypes = [p, i32, i64, i32, i64, p, i32, p, p, p, p, sz, p]
    lib.aero_distill_loss_bwd.restype = i32
    lib.aero_distill_loss_bwd.argtypes = [p, i32, i64, i32, i64, p, p, i32, p, i32, f32, p, p, p, p, p, sz, p]
    lib.aero_verify_draft.restype = i32
    lib.aero_verify_draft.argtypes = [p, p, i32, i32, i32, i32, i64, p, p, p, p, p, p, p, p, p, sz, p]
    lib.aero_embedding_fwd.restype = i32
    lib.aero_embedding_fwd.argtypes = [p, i32, i32, i32, p, i64, f32, p, i64, p, p]
    lib.aero_embedding_bwd.restype = i32
    lib.aero_embedding_bwd.argtypes = [p, i32, i64, i32, i64, p, i32, f32, p, i32, p, p, sz, p]
    lib.aero_preference_loss.restype = i32
    lib.aero_preference_loss.argtypes = [p, i64, p, p, i32, p, p, p, i32, C.POINTER(_PreferenceParamsC), p, p, p, p, p, p, sz, p]
    lib.aero_preference_loss_bwd.restype = i32
    lib.aero_preference_loss_bwd.argtypes = [p, i32, i64, i32, i64, p, p, p, i32, p, p, p, i32, C.POINTER(_PreferenceParamsC), f32, p, p, p,
                                             p, p, p, p, sz, p]
    lib.aero_tensor_table_bytes.restype = sz
    lib.aero_tensor_table_bytes.argtypes = [C.POINTER(_TensorC), i32]
    lib.aero_tensor_table.restype = i32
    lib.aero_tensor_table.argtypes = [C.POINTER(_TensorC), i32, p, sz]
    lib.aero_grad_norm.restype = i32
    lib.aero_grad_norm.argtypes = [p, p, f32, f32, p, p, p, sz, p]
    lib.aero_adamw_step.restype = i32
    lib.aero_adamw_step.argtypes = [p, p, C.POINTER(_AdamWParamsC), p, p, p, p]
    lib.aero_adamw_moments.restype = i32
    lib.aero_adamw_moments.argtypes = [p, p, i32, p, p, p]
    return lib


class _Lazy:
    """Loads the library on first use so that the package can be imported to build it."""
    _cdll = None

    def __getattr__(self, name):   # first use of an entry point: kept as a plain attribute from then on
        if _Lazy._cdll is None:
            _Lazy._cdll = _load()
        fn = getattr(_Lazy._cdll, name)
        setattr(self, name, fn)
        return fn


_lib = _Lazy()


def _check(status: int, what: str) -> None:
    if status != 0:
        raise AeroError(f"{what}: {_lib.aero_status_string(status).decode()} (status {status})")


def _ptr(t: Optional[torch.Tensor], dtype=None, name: str = "") -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise AeroError(f"{name}: expected a GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise AeroError(f"{name}: expected dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise AeroError(f"{name}: expected a contiguous tensor")
    return t.data_ptr()


class _Marshal:
    """The native module (csrc/marshal.cpp).  ``pointers(t, dtype, name, ...)``: `_ptr` of every triple in one call;
    ``group_advantage`` and the others: a whole call whose arguments are all plain, NotImplemented for any other."""

    def __getattr__(self, name):
        if name not in ("pointers", "group_advantage", "logprob_fwd", "loss_bwd", "fused", "topk", "distill", "verify", "embed_fwd",
                        "embed_bwd", "pair", "pair_bwd", "norm", "adamw"):
            raise AttributeError(name)
        try:
            from . import _marshal
        except ImportError as e:
            raise AeroError("the package's _marshal module is missing: build it with "
                            "`python -m paper_2602_14338_amd.build` (there is no fallback path)") from e
        if name == "pointers":
            _marshal.setup(AeroError, _ptr)
        else:
            entries = (_lib.aero_group_advantage, _lib.aero_logprob_fwd, _lib.aero_grpo_loss_bwd,
                       _lib.aero_grpo_loss_bwd_noalloc, _lib.aero_lmhead_logprob_fused, _lib.aero_topk_logprob,
                       _lib.aero_distill_loss_bwd, _lib.aero_verify_draft, _lib.aero_embedding_fwd, _lib.aero_embedding_bwd,
                       _lib.aero_preference_loss, _lib.aero_preference_loss_bwd, _lib.aero_grad_norm, _lib.aero_adamw_step)
            _marshal.bind(torch._C._cuda_getCurrentRawStream, AdvParams, PreferenceParams, AdamWParams, *(C.cast(f, C.c_void_p).value for f in entries))
        fn = getattr(_marshal, name)
        setattr(self, name, fn)
        return fn


_m = _Marshal()
_F32, _I32, _U8, _BF16 = torch.float32, torch.int32, torch.uint8, torch.bfloat16


def _stream(t: torch.Tensor) -> int:
    """Handle of torch's current stream on the tensor's device (a GPU tensor: its pointer was taken before)."""
    return torch._C._cuda_getCurrentRawStream(t.get_device())


_DTYPE_CODES = {torch.bfloat16: AERO_BF16, torch.float32: AERO_F32, torch.float16: AERO_F16,
                torch.float8_e4m3fn: AERO_F8E4M3}


def _dtype_code(t: torch.Tensor) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise AeroError(f"unsupported dtype {t.dtype}")
    return code


def aero_workspace_bytes(op: int, T: int = 0, V: int = 0, H: int = 0, R: int = 0, Q: int = 0) -> int:
    return int(_lib.aero_workspace_bytes(op, T, V, H, R, Q))


def aero_group_advantage(rewards, lengths, group_offsets, keep_priority, Q: int, R: int, params: AdvParams,
                         adv, weight, keep_mask, kept_index, kept_offsets, group_zero_var, group_category,
                         err_flag=None) -> None:
    st = _m.group_advantage(rewards, lengths, group_offsets, keep_priority, Q, R, params, adv, weight, keep_mask,
                            kept_index, kept_offsets, group_zero_var, group_category, err_flag)
    if st is not NotImplemented:
        return _check(st, "aero_group_advantage")
    pc = params.to_c()
    p = _m.pointers(rewards, _F32, "rewards", lengths, _I32, "lengths", group_offsets, _I32, "group_offsets",
                    keep_priority, None, "keep_priority", adv, _F32, "adv", weight, _F32, "weight",
                    keep_mask, _U8, "keep_mask", kept_index, _I32, "kept_index", kept_offsets, _I32, "kept_offsets",
                    group_zero_var, _U8, "group_zero_var", group_category, _U8, "group_category",
                    err_flag, _I32, "err_flag")
    st = _lib.aero_group_advantage(*p[:4], Q, R, C.byref(pc), *p[4:], _stream(group_offsets))
    _check(st, "aero_group_advantage")


def aero_logprob_fwd(logits, T: int, V: int, ld: int, targets, row_active, logprob, entropy, lse,
                     err_flag=None) -> None:
    st = _m.logprob_fwd(logits, T, V, ld, targets, row_active, logprob, entropy, lse, err_flag)
    if st is not NotImplemented:
        return _check(st, "aero_logprob_fwd")
    z, *p = _m.pointers(logits, None, "logits", targets, _I32, "targets", row_active, _U8, "row_active",
                        logprob, _F32, "logprob", entropy, _F32, "entropy", lse, _F32, "lse",
                        err_flag, _I32, "err_flag")
    st = _lib.aero_logprob_fwd(z, _dtype_code(logits), T, V, ld, *p, _stream(logits))
    _check(st, "aero_logprob_fwd")


def _loss_pointers(logits, targets, lse, entropy, old_logprob, token_rollout, adv, weight, ref_logprob, loss, clip_frac,
                   logprob_out, entropy_out, lse_out, dlogits, err_flag):
    if dlogits is not None and dlogits.dtype != logits.dtype:
        raise AeroError("dlogits must have the dtype of logits")
    return _m.pointers(
        logits, None, "logits", targets, _I32, "targets", lse, _F32, "lse", entropy, _F32, "entropy",
        old_logprob, _F32, "old_logprob", token_rollout, _I32, "token_rollout", adv, _F32, "adv",
        weight, _F32, "weight", ref_logprob, _F32, "ref_logprob", loss, _F32, "loss", clip_frac, _F32, "clip_frac",
        logprob_out, _F32, "logprob_out", entropy_out, _F32, "entropy_out", lse_out, _F32, "lse_out",
        dlogits, None, "dlogits", err_flag, _I32, "err_flag")


def aero_grpo_loss_bwd(logits, T: int, V: int, ld: int, targets, lse, old_logprob, token_rollout, adv, weight,
                       R: int, eps_lo: float, eps_hi: float, grad_scale: float, loss, clip_frac, logprob_out,
                       dlogits, workspace, err_flag=None, entropy_out=None, lse_out=None,
                       entropy_coef: float = 0.0, entropy=None, kl_coef: float = 0.0, ref_logprob=None) -> None:
    st = _m.loss_bwd(logits, T, V, ld, targets, lse, entropy, old_logprob, token_rollout, adv, weight, R, eps_lo, eps_hi,
                     grad_scale, entropy_coef, kl_coef, ref_logprob, loss, clip_frac, logprob_out, entropy_out, lse_out,
                     dlogits, err_flag, workspace)
    if st is not NotImplemented:
        return _check(st, "aero_grpo_loss_bwd")
    z, *p = _loss_pointers(logits, targets, lse, entropy, old_logprob, token_rollout, adv, weight, ref_logprob, loss,
                           clip_frac, logprob_out, entropy_out, lse_out, dlogits, err_flag)
    ws, = _m.pointers(workspace, None, "workspace")
    st = _lib.aero_grpo_loss_bwd(
        z, _dtype_code(logits), T, V, ld, *p[:7], R, eps_lo, eps_hi, grad_scale, entropy_coef, kl_coef, *p[7:], ws,
        workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream(logits))
    _check(st, "aero_grpo_loss_bwd")


def aero_grpo_loss_bwd_noalloc(logits, T: int, V: int, ld: int, targets, lse, old_logprob, token_rollout, adv, weight,
                               R: int, eps_lo: float, eps_hi: float, grad_scale: float, loss, clip_frac,
                               logprob_out, dlogits, err_flag=None, entropy_out=None, lse_out=None,
                               entropy_coef: float = 0.0, entropy=None, kl_coef: float = 0.0,
                               ref_logprob=None) -> None:
    """aero_grpo_loss_bwd without a workspace argument: the library's own fixed scratch is used."""
    st = _m.loss_bwd(logits, T, V, ld, targets, lse, entropy, old_logprob, token_rollout, adv, weight, R, eps_lo, eps_hi,
                     grad_scale, entropy_coef, kl_coef, ref_logprob, loss, clip_frac, logprob_out, entropy_out, lse_out,
                     dlogits, err_flag)
    if st is not NotImplemented:
        return _check(st, "aero_grpo_loss_bwd_noalloc")
    z, *p = _loss_pointers(logits, targets, lse, entropy, old_logprob, token_rollout, adv, weight, ref_logprob, loss,
                           clip_frac, logprob_out, entropy_out, lse_out, dlogits, err_flag)
    st = _lib.aero_grpo_loss_bwd_noalloc(z, _dtype_code(logits), T, V, ld, *p[:7], R, eps_lo, eps_hi, grad_scale,
                                         entropy_coef, kl_coef, *p[7:], _stream(logits))
    _check(st, "aero_grpo_loss_bwd_noalloc")


def aero_lmhead_logprob_fused(hidden, weight, T: int, H: int, V: int, targets, logprob, entropy, lse,
                              old_logprob=None, token_rollout=None, adv=None, weight_rollout=None, R: int = 0,
                              eps_lo: float = 0.2, eps_hi: float = 0.2, grad_scale: float = 1.0,
                              loss=None, clip_frac=None, dhidden=None, dweight=None, workspace=None,
                              err_flag=None, entropy_coef: float = 0.0, kl_coef: float = 0.0,
                              ref_logprob=None, dweight_accumulate: bool = False) -> None:
    st = _m.fused(hidden, weight, T, H, V, targets, logprob, entropy, lse, old_logprob, token_rollout, adv, weight_rollout,
                  R, eps_lo, eps_hi, grad_scale, entropy_coef, kl_coef, ref_logprob, loss, clip_frac, dhidden, dweight,
                  dweight_accumulate, err_flag, workspace)
    if st is not NotImplemented:
        return _check(st, "aero_lmhead_logprob_fused")
    p = _m.pointers(
        hidden, _BF16, "hidden", weight, _BF16, "weight", targets, _I32, "targets", logprob, _F32, "logprob",
        entropy, _F32, "entropy", lse, _F32, "lse", old_logprob, _F32, "old_logprob",
        token_rollout, _I32, "token_rollout", adv, _F32, "adv", weight_rollout, _F32, "weight_rollout",
        ref_logprob, _F32, "ref_logprob", loss, _F32, "loss", clip_frac, _F32, "clip_frac", dhidden, _BF16, "dhidden",
        dweight, None, "dweight", err_flag, _I32, "err_flag", workspace, None, "workspace")
    dweight_dtype = (_dtype_code(dweight) if dweight is not None else AERO_F32) | \
        (AERO_DW_ACCUMULATE if dweight_accumulate else 0)
    st = _lib.aero_lmhead_logprob_fused(
        *p[:2], T, H, V, *p[2:10], R, eps_lo, eps_hi, grad_scale, entropy_coef, kl_coef, *p[10:15], dweight_dtype,
        *p[15:], workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream(hidden))
    _check(st, "aero_lmhead_logprob_fused")


def _bytes(t: Optional[torch.Tensor]) -> int:
    return t.numel() * t.element_size() if t is not None else 0


def aero_topk_logprob(logits, T: int, V: int, ld: int, row_active, K: int, index, logprob, lse, workspace) -> None:
    st = _m.topk(logits, T, V, ld, row_active, K, index, logprob, lse, workspace)
    if st is not NotImplemented:
        return _check(st, "aero_topk_logprob")
    z, *p, ws = _m.pointers(logits, None, "logits", row_active, _U8, "row_active", index, _I32, "index", logprob, _F32, "logprob",
                            lse, _F32, "lse", workspace, None, "workspace")
    st = _lib.aero_topk_logprob(z, _dtype_code(logits), T, V, ld, p[0], K, *p[1:], ws, _bytes(workspace), _stream(logits))
    _check(st, "aero_topk_logprob")


def aero_distill_loss_bwd(logits, T: int, V: int, ld: int, teacher_index, teacher_logprob, K: int, token_weight, tail: int,
                          grad_scale: float, loss, row_loss, dlogits, workspace, err_flag=None) -> None:
    st = _m.distill(logits, T, V, ld, teacher_index, teacher_logprob, K, token_weight, tail, grad_scale, loss, row_loss, dlogits, err_flag,
                    workspace)
    if st is not NotImplemented:
        return _check(st, "aero_distill_loss_bwd")
    if dlogits is not None and dlogits.dtype != logits.dtype:
        raise AeroError("dlogits must have the dtype of logits")
    z, index, lp, w, *p = _m.pointers(
        logits, None, "logits", teacher_index, _I32, "teacher_index", teacher_logprob, _F32, "teacher_logprob",
        token_weight, _F32, "token_weight", loss, _F32, "loss", row_loss, _F32, "row_loss", dlogits, None, "dlogits",
        err_flag, _I32, "err_flag", workspace, None, "workspace")
    st = _lib.aero_distill_loss_bwd(z, _dtype_code(logits), T, V, ld, index, lp, K, w, tail, grad_scale, *p, _bytes(workspace),
                                    _stream(logits))
    _check(st, "aero_distill_loss_bwd")


def aero_verify_draft(target_logits, draft_logits, B: int, G: int, V: int, ld: int, draft_tokens, draft_count, uniform, noise,
                      accepted, tokens, logprob, workspace, err_flag=None) -> None:
    st = _m.verify(target_logits, draft_logits, B, G, V, ld, draft_tokens, draft_count, uniform, noise, accepted, tokens, logprob, err_flag,
                   workspace)
    if st is not NotImplemented:
        return _check(st, "aero_verify_draft")
    if draft_logits is not None and draft_logits.dtype != target_logits.dtype:
        raise AeroError("draft_logits must have the dtype of target_logits")
    zt, zd, *p, err, ws = _m.pointers(
        target_logits, None, "target_logits", draft_logits, None, "draft_logits", draft_tokens, _I32, "draft_tokens",
        draft_count, _I32, "draft_count", uniform, _F32, "uniform", noise, _F32, "noise", accepted, _I32, "accepted",
        tokens, _I32, "tokens", logprob, _F32, "logprob", err_flag, _I32, "err_flag", workspace, None, "workspace")
    st = _lib.aero_verify_draft(zt, zd, _dtype_code(target_logits), B, G, V, ld, *p, err, ws, _bytes(workspace),
                                _stream(target_logits))
    _check(st, "aero_verify_draft")


def aero_embedding_fwd(table, V: int, H: int, ids, T: int, scale: float, out, ld_out: int, err_flag=None) -> None:
    st = _m.embed_fwd(table, V, H, ids, T, scale, out, ld_out, err_flag)
    if st is not NotImplemented:
        return _check(st, "aero_embedding_fwd")
    if out.dtype != table.dtype:
        raise AeroError("out must have the dtype of table")
    e, i, o, err = _m.pointers(table, None, "table", ids, _I32, "ids", out, None, "out", err_flag, _I32, "err_flag")
    st = _lib.aero_embedding_fwd(e, _dtype_code(table), V, H, i, T, scale, o, ld_out, err, _stream(table))
    _check(st, "aero_embedding_fwd")


def aero_embedding_bwd(dout, T: int, H: int, ld_dout: int, ids, V: int, scale: float, dtable, workspace,
                       accumulate: bool = False, err_flag=None) -> None:
    st = _m.embed_bwd(dout, T, H, ld_dout, ids, V, scale, dtable, accumulate, err_flag, workspace)
    if st is not NotImplemented:
        return _check(st, "aero_embedding_bwd")
    d, i, g, err, ws = _m.pointers(dout, None, "dout", ids, _I32, "ids", dtable, None, "dtable", err_flag, _I32, "err_flag",
                                   workspace, None, "workspace")
    code = _dtype_code(dtable) | (AERO_DW_ACCUMULATE if accumulate else 0)
    st = _lib.aero_embedding_bwd(d, _dtype_code(dout), T, H, ld_dout, i, V, scale, g, code, err, ws, _bytes(workspace), _stream(dout))
    _check(st, "aero_embedding_bwd")


def aero_preference_loss(logprob, T: int, ref_logprob, token_rollout, R: int, pair_chosen, pair_rejected, pair_weight, P: int,
                         params: PreferenceParams, loss, pair_margin, rollout_ratio, drollout, workspace, err_flag=None) -> None:
    st = _m.pair(logprob, T, ref_logprob, token_rollout, R, pair_chosen, pair_rejected, pair_weight, P, params, loss, pair_margin,
                 rollout_ratio, drollout, err_flag, workspace)
    if st is not NotImplemented:
        return _check(st, "aero_preference_loss")
    lp, ref, owner, c, j, w, *p = _m.pointers(
        logprob, _F32, "logprob", ref_logprob, _F32, "ref_logprob", token_rollout, _I32, "token_rollout", pair_chosen, _I32, "pair_chosen",
        pair_rejected, _I32, "pair_rejected", pair_weight, _F32, "pair_weight", loss, _F32, "loss", pair_margin, _F32, "pair_margin",
        rollout_ratio, _F32, "rollout_ratio", drollout, _F32, "drollout", err_flag, _I32, "err_flag", workspace, None, "workspace")
    on = next((t for t in (loss, logprob, workspace) if t is not None), None)
    st = _lib.aero_preference_loss(lp, T, ref, owner, R, c, j, w, P, C.byref(params.to_c()), *p, _bytes(workspace),
                                   _stream(on) if on is not None else None)
    _check(st, "aero_preference_loss")


def aero_preference_loss_bwd(logits, T: int, V: int, ld: int, targets, ref_logprob, token_rollout, R: int, pair_chosen, pair_rejected,
                             pair_weight, P: int, params: PreferenceParams, grad_scale: float, loss, pair_margin, rollout_ratio,
                             logprob_out, dlogits, workspace, err_flag=None) -> None:
    st = _m.pair_bwd(logits, T, V, ld, targets, ref_logprob, token_rollout, R, pair_chosen, pair_rejected, pair_weight, P, params,
                     grad_scale, loss, pair_margin, rollout_ratio, logprob_out, dlogits, err_flag, workspace)
    if st is not NotImplemented:
        return _check(st, "aero_preference_loss_bwd")
    if dlogits is not None and dlogits.dtype != logits.dtype:
        raise AeroError("dlogits must have the dtype of logits")
    z, y, ref, owner, c, j, w, *p = _m.pointers(
        logits, None, "logits", targets, _I32, "targets", ref_logprob, _F32, "ref_logprob", token_rollout, _I32, "token_rollout",
        pair_chosen, _I32, "pair_chosen", pair_rejected, _I32, "pair_rejected", pair_weight, _F32, "pair_weight", loss, _F32, "loss",
        pair_margin, _F32, "pair_margin", rollout_ratio, _F32, "rollout_ratio", logprob_out, _F32, "logprob_out", dlogits, None, "dlogits",
        err_flag, _I32, "err_flag", workspace, None, "workspace")
    st = _lib.aero_preference_loss_bwd(z, _dtype_code(logits), T, V, ld, y, ref, owner, R, c, j, w, P, C.byref(params.to_c()), grad_scale, *p,
                                       _bytes(workspace), _stream(logits))
    _check(st, "aero_preference_loss_bwd")


class TensorTable:
    """The tensors that norm, step and moments work on, described once.  Entries: dicts of the tensors ``param``, ``grad``, ``master``,
    ``exp_avg``, ``exp_avg_sq``, ``exp_avg_scale``, ``exp_avg_sq_scale`` (``grad`` alone: it takes part in the norm) and the number
    ``decay``.  Keeps the tensors alive; calls on one table have to be ordered on one stream."""

    _NAMES = ("param", "grad", "master", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale")

    def __init__(self, entries):
        self.entries = [dict(e) for e in entries]
        if not self.entries:
            raise AeroError("a table needs a tensor")
        self.device = None
        self.n_moments = 0
        rows = (_TensorC * len(self.entries))()
        for k, e in enumerate(self.entries):
            self._fill(rows[k], e, f"entry {k}")
        self._check_apart()
        size = int(_lib.aero_tensor_table_bytes(rows, len(self.entries)))
        self._host = torch.empty(size + 16, dtype=torch.uint8)
        self.image = (self._host.data_ptr() + 15) & ~15
        _check(_lib.aero_tensor_table(rows, len(self.entries), self.image, size), "aero_tensor_table")
        at = self.image - self._host.data_ptr()
        with torch.cuda.device(self.device):
            self.table = torch.empty(size, dtype=torch.uint8, device=self.device)
            self.table.copy_(self._host[at:at + size])

    def _check_apart(self) -> None:
        """What a step writes overlaps nothing else (the same tensor twice, say)."""
        spans = sorted((e[name].data_ptr(), e[name].data_ptr() + _bytes(e[name]), name == "grad", f"entry {k}: {name}")
                       for k, e in enumerate(self.entries) for name in self._NAMES if e.get(name) is not None and e[name].numel())
        end = {False: (0, ""), True: (0, "")}   # of what is written, of gradients: the furthest so far
        for first, last, reads, what in spans:
            for kind in (False, True):
                if first < end[kind][0] and not (reads and kind):
                    raise AeroError(f"{what} overlaps {end[kind][1]}")
            if last > end[reads][0]:
                end[reads] = (last, what)

    def _fill(self, row: _TensorC, e: dict, where: str) -> None:
        unknown = set(e) - set(self._NAMES) - {"decay"}
        if unknown:
            raise AeroError(f"{where}: unknown {', '.join(sorted(unknown))}")
        if e.get("grad") is None:
            raise AeroError(f"{where}: grad is missing")
        n = e["grad"].numel()
        small = e.get("exp_avg_scale") is not None
        blocks = (n + AERO_MOMENT_BLOCK - 1) // AERO_MOMENT_BLOCK
        for name in self._NAMES:
            t = e.get(name)
            if t is None:
                continue
            dtype = {"master": _F32, "exp_avg": torch.int8 if small else _F32, "exp_avg_sq": _U8 if small else _F32,
                     "exp_avg_scale": _F32, "exp_avg_sq_scale": _F32}.get(name)
            address = _ptr(t, dtype, f"{where}: {name}")
            if t.numel() != (blocks if name.endswith("scale") else n):
                raise AeroError(f"{where}: {name} has {t.numel()} elements, grad {n}")
            if self.device is None:
                self.device = t.device
            if t.device != self.device:
                raise AeroError(f"{where}: {name} is on {t.device}, the table on {self.device}")
            setattr(row, name, address)
        row.n = n
        row.grad_dtype = _dtype_code(e["grad"])
        if e.get("param") is not None:
            row.param_dtype = _dtype_code(e["param"])
            self.n_moments += n
        row.decay = e.get("decay", 1.0)


def aero_grad_norm(table: TensorTable, grad_scale: float, max_norm: float, norm, factor, workspace) -> None:
    st = _m.norm(table.image, table.table, grad_scale, max_norm, norm, factor, workspace)
    if st is not NotImplemented:
        return _check(st, "aero_grad_norm")
    p = _m.pointers(table.table, None, "table", norm, _F32, "norm", factor, _F32, "factor", workspace, None, "workspace")
    st = _lib.aero_grad_norm(table.image, p[0], grad_scale, max_norm, *p[1:], _bytes(workspace), _stream(table.table))
    _check(st, "aero_grad_norm")


def aero_adamw_step(table: TensorTable, params: AdamWParams, step, factor=None, lr_factor=None) -> None:
    st = _m.adamw(table.image, table.table, params, step, factor, lr_factor)
    if st is not NotImplemented:
        return _check(st, "aero_adamw_step")
    p = _m.pointers(table.table, None, "table", step, _I32, "step", factor, _F32, "factor", lr_factor, _F32, "lr_factor")
    st = _lib.aero_adamw_step(table.image, p[0], C.byref(params.to_c()), *p[1:], _stream(table.table))
    _check(st, "aero_adamw_step")


def aero_adamw_moments(table: TensorTable, avg, avg_sq) -> None:
    if avg.dtype != avg_sq.dtype:
        raise AeroError("avg and avg_sq must have the same dtype")
    for name, t in (("avg", avg), ("avg_sq", avg_sq)):
        if t.numel() != table.n_moments:
            raise AeroError(f"{name} has {t.numel()} elements, the table's moments {table.n_moments}")
    p = _m.pointers(table.table, None, "table", avg, None, "avg", avg_sq, None, "avg_sq")
    st = _lib.aero_adamw_moments(table.image, p[0], _dtype_code(avg), *p[1:], _stream(table.table))
    _check(st, "aero_adamw_moments")
