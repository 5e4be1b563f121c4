"""ctypes binding of libunity.so: argument marshalling only.

Every function mirrors the C entry point of the same name in ``include/unity.h``; tensors are
torch CUDA tensors whose ``data_ptr()`` is passed through, small host tables are python
sequences.  No arithmetic of the path happens here, and there is no fallback: if the shared
library cannot be loaded the import of a symbol raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import torch

from . import build as _build

UNITY_OK = 0
ERR_NAMES = {0: "UNITY_OK", -1: "UNITY_ERR_INVALID_ARG", -2: "UNITY_ERR_SHAPE", -3: "UNITY_ERR_ALIGNMENT",
             -4: "UNITY_ERR_WORKSPACE", -5: "UNITY_ERR_CUDA", -6: "UNITY_ERR_UNSUPPORTED_ARCH",
             -7: "UNITY_ERR_BAD_INDEX", -8: "UNITY_ERR_TIMEOUT"}
UNITY_MAX_MODELS = 16
UNITY_MAX_ROLES = 64
UNITY_N_METRICS = 8

EXPORTS = ["unity_create", "unity_destroy", "unity_workspace_hint", "unity_workspace_bytes", "unity_workspace_min_bytes",
           "unity_workspace_bytes_stash",
           "unity_check_status", "unity_last_error", "unity_launch_count", "unity_set_profiling",
           "unity_get_profile", "unity_set_option", "unity_advantage_workspace_bytes", "unity_role_advantage", "unity_reward_assembly", "unity_gae", "unity_value_loss_fwd_bwd",
           "unity_ready_batch_plan", "unity_ready_batch_gather", "unity_align_rewards",
           "unity_role_advantage_noalloc",
           "unity_logprob_fwd", "unity_ppo_loss_fwd_bwd",
           "unity_token_loss_workspace_bytes", "unity_cross_entropy_fwd_bwd", "unity_distill_fwd_bwd",
           "unity_rms_norm_workspace_bytes", "unity_rms_norm_fwd", "unity_rms_norm_bwd",
           "unity_clip_grad_norm_workspace_bytes", "unity_clip_grad_norm", "unity_sample"]


class UnityError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERR_NAMES.get(code, code)}: {msg}")
        self.code = code


class unity_adv_params(C.Structure):
    _fields_ = [("eps", C.c_float), ("ddof", C.c_int)]


class unity_reward_rule(C.Structure):
    _fields_ = [("mode", C.c_int), ("shift", C.c_int)]


class unity_batch_params(C.Structure):
    _fields_ = [("seed", C.c_uint64), ("n_parts", C.c_int32), ("pad_to", C.c_int32)]


class unity_rows(C.Structure):
    _fields_ = [("n_tok", C.c_int64), ("H", C.c_int32), ("V", C.c_int32), ("K", C.c_int32),
                ("n_inv", C.c_int32), ("n_roles", C.c_int32),
                ("hidden", C.c_void_p), ("W", C.POINTER(C.c_void_p)), ("cu_seqlens", C.c_void_p),
                ("inv_role", C.c_void_p), ("role_model", C.POINTER(C.c_int32)), ("target", C.c_void_p),
                ("tok_mask", C.c_void_p), ("inv_temperature", C.c_float)]


class unity_ppo_params(C.Structure):
    _fields_ = [("clip_lo", C.c_float), ("clip_hi", C.c_float), ("kl_coef", C.c_float), ("kl_mode", C.c_int),
                ("ent_coef", C.c_float), ("norm", C.POINTER(C.c_float)), ("accumulate_dW", C.c_int),
                ("logp_in", C.c_void_p), ("entropy_in", C.c_void_p), ("lse_in", C.c_void_p)]


class unity_ce_params(C.Structure):
    _fields_ = [("label_smoothing", C.c_float), ("z_loss", C.c_float), ("norm", C.POINTER(C.c_float)),
                ("accumulate_dW", C.c_int), ("dW_type", C.c_int)]


class unity_distill_params(C.Structure):
    _fields_ = [("n_top", C.c_int32), ("teacher_mode", C.c_int), ("kd_coef", C.c_float), ("hard_coef", C.c_float),
                ("norm", C.POINTER(C.c_float)), ("accumulate_dW", C.c_int), ("dW_type", C.c_int)]


class unity_norm_rows(C.Structure):
    _fields_ = [("n_tok", C.c_int64), ("H", C.c_int32), ("K", C.c_int32), ("n_inv", C.c_int32), ("n_roles", C.c_int32),
                ("cu_seqlens", C.c_void_p), ("inv_role", C.c_void_p), ("role_model", C.POINTER(C.c_int32)),
                ("tok_mask", C.c_void_p), ("gamma", C.POINTER(C.c_void_p)), ("gamma_type", C.c_int), ("eps", C.c_float)]


class unity_tensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("model", C.c_int32), ("type", C.c_int16),
                ("out_type", C.c_int16)]


class unity_sampling_rule(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_k", C.c_int32), ("top_p", C.c_float), ("min_p", C.c_float)]


_LIB = None


def load_library(path: Optional[str] = None) -> C.CDLL:
    """Load (building first if the sources are newer) libunity.so.  Raises if that is impossible."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    if path is None:
        path = _build.LIB_PATH
        if _build.needs_build():
            _build.build()
    if not os.path.exists(path):
        raise RuntimeError(f"libunity.so not found at {path}: build it with python -m paper_2605_26646_b200.build")
    lib = C.CDLL(path)
    vp, i32, i64, f32p = C.c_void_p, C.c_int32, C.c_int64, C.POINTER(C.c_float)
    lib.unity_create.argtypes = [C.POINTER(vp), C.c_int, vp, vp, C.c_size_t]
    lib.unity_create.restype = C.c_int
    lib.unity_destroy.argtypes = [vp]
    lib.unity_destroy.restype = C.c_int
    for fn in (lib.unity_workspace_bytes, lib.unity_workspace_min_bytes, lib.unity_workspace_bytes_stash):
        fn.argtypes = [i64, i32, i32, i32, i32]
        fn.restype = C.c_size_t
    lib.unity_workspace_hint.argtypes = [i64, i32, i32, i32]
    lib.unity_workspace_hint.restype = C.c_size_t
    lib.unity_check_status.argtypes = [vp]
    lib.unity_check_status.restype = C.c_int
    lib.unity_last_error.argtypes = [vp]
    lib.unity_last_error.restype = C.c_char_p
    lib.unity_launch_count.argtypes = [vp]
    lib.unity_launch_count.restype = i64
    lib.unity_set_profiling.argtypes = [vp, C.c_int]
    lib.unity_set_profiling.restype = C.c_int
    lib.unity_set_option.argtypes = [vp, C.c_int, C.c_int]
    lib.unity_set_option.restype = C.c_int
    lib.unity_get_profile.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(i64)]
    lib.unity_get_profile.restype = C.c_int
    lib.unity_advantage_workspace_bytes.argtypes = [i32, i32, i32]
    lib.unity_advantage_workspace_bytes.restype = C.c_size_t
    lib.unity_role_advantage.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, f32p,
                                         C.POINTER(unity_adv_params), i64, vp, vp, vp, vp, vp, vp]
    lib.unity_role_advantage.restype = C.c_int
    lib.unity_role_advantage_noalloc.argtypes = [C.c_int, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, f32p,
                                                 C.POINTER(unity_adv_params), i64, vp, vp, vp, vp, vp, vp, vp,
                                                 C.c_char_p, C.c_size_t]
    lib.unity_role_advantage_noalloc.restype = C.c_int
    lib.unity_reward_assembly.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp,
                                          C.POINTER(unity_reward_rule), vp]
    lib.unity_reward_assembly.restype = C.c_int
    lib.unity_gae.argtypes = [vp, i32, i64, vp, vp, vp, vp, C.c_float, C.c_float, vp, vp]
    lib.unity_gae.restype = C.c_int
    lib.unity_value_loss_fwd_bwd.argtypes = [vp, i32, i32, i32, i64, vp, vp, C.POINTER(i32), vp, vp, vp, vp, C.c_float,
                                             f32p, vp, vp, vp, vp]
    lib.unity_value_loss_fwd_bwd.restype = C.c_int
    lib.unity_ready_batch_plan.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, C.POINTER(i32),
                                           C.POINTER(unity_batch_params), vp, vp, vp, vp, vp]
    lib.unity_ready_batch_plan.restype = C.c_int
    lib.unity_ready_batch_gather.argtypes = [vp, i32, i64, vp, vp, vp, vp, i64, vp, vp, vp, i32]
    lib.unity_ready_batch_gather.restype = C.c_int
    lib.unity_align_rewards.argtypes = [vp, i32, i64, vp, vp, vp, vp]
    lib.unity_align_rewards.restype = C.c_int
    lib.unity_logprob_fwd.argtypes = [vp, C.POINTER(unity_rows), vp, vp, vp]
    lib.unity_logprob_fwd.restype = C.c_int
    lib.unity_ppo_loss_fwd_bwd.argtypes = [vp, C.POINTER(unity_rows), C.POINTER(unity_ppo_params), vp, vp, vp,
                                           vp, vp, vp, vp, vp, vp, C.POINTER(vp)]
    lib.unity_ppo_loss_fwd_bwd.restype = C.c_int
    lib.unity_token_loss_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i32]
    lib.unity_token_loss_workspace_bytes.restype = C.c_size_t
    lib.unity_cross_entropy_fwd_bwd.argtypes = [vp, C.POINTER(unity_rows), C.POINTER(unity_ce_params), vp, vp, vp, vp, vp,
                                                C.POINTER(vp)]
    lib.unity_cross_entropy_fwd_bwd.restype = C.c_int
    lib.unity_distill_fwd_bwd.argtypes = [vp, C.POINTER(unity_rows), C.POINTER(unity_distill_params), vp, vp, vp, vp, vp,
                                          vp, vp, C.POINTER(vp)]
    lib.unity_distill_fwd_bwd.restype = C.c_int
    lib.unity_rms_norm_workspace_bytes.argtypes = [i64, i32, i32]
    lib.unity_rms_norm_workspace_bytes.restype = C.c_size_t
    lib.unity_rms_norm_fwd.argtypes = [vp, C.POINTER(unity_norm_rows), vp, vp, C.c_int, vp, vp]
    lib.unity_rms_norm_fwd.restype = C.c_int
    lib.unity_rms_norm_bwd.argtypes = [vp, C.POINTER(unity_norm_rows), vp, C.c_int, vp, vp, vp, C.POINTER(vp), C.c_int]
    lib.unity_rms_norm_bwd.restype = C.c_int
    lib.unity_clip_grad_norm_workspace_bytes.argtypes = [i32, i32]
    lib.unity_clip_grad_norm_workspace_bytes.restype = C.c_size_t
    lib.unity_clip_grad_norm.argtypes = [vp, i32, C.POINTER(unity_tensor), i32, f32p, vp, vp]
    lib.unity_clip_grad_norm.restype = C.c_int
    lib.unity_sample.argtypes = [vp, i32, i32, vp, C.c_int, i64, i32, vp, C.POINTER(unity_sampling_rule), vp, vp, vp, vp, vp,
                                 vp]
    lib.unity_sample.restype = C.c_int
    if path == _build.LIB_PATH:
        _LIB = lib
    return lib


def _ptr(t: Optional[torch.Tensor], dtype=None, name="tensor", host=False) -> Optional[int]:
    if t is None:
        return None
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if not host and not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return t.data_ptr()


def _raise(ctx, code: int):
    if code != UNITY_OK:
        raise UnityError(code, load_library().unity_last_error(ctx).decode())


# ------------------------------------------------------------------------------------------------
# functions with the names of the C entry points
# ------------------------------------------------------------------------------------------------
def unity_workspace_hint(n_tok: int, H: int, V: int, K: int) -> int:
    return int(load_library().unity_workspace_hint(n_tok, H, V, K))


def unity_workspace_bytes(n_tok: int, H: int, V: int, K: int, n_inv: int) -> int:
    return int(load_library().unity_workspace_bytes(n_tok, H, V, K, n_inv))


def unity_workspace_min_bytes(n_tok: int, H: int, V: int, K: int, n_inv: int) -> int:
    return int(load_library().unity_workspace_min_bytes(n_tok, H, V, K, n_inv))


def unity_advantage_workspace_bytes(n_inv: int, n_groups: int, n_roles: int) -> int:
    return int(load_library().unity_advantage_workspace_bytes(n_inv, n_groups, n_roles))


def unity_workspace_bytes_stash(n_tok: int, H: int, V: int, K: int, n_inv: int) -> int:
    return int(load_library().unity_workspace_bytes_stash(n_tok, H, V, K, n_inv))


OPT_LOGIT_STASH = 15
OPT_WAIT_KCYCLES = 20
OPT_HOST_COUNTS = 25
OPT_TEST_DROP_SLAB = 21
OPT_GRAD_ROUNDS = 26
OPT_GRAD_BLOCK = 27
OPT_GRAD_RUNS = 28


def unity_create(device: int, stream_ptr: int, workspace: torch.Tensor) -> C.c_void_p:
    ctx = C.c_void_p()
    code = load_library().unity_create(C.byref(ctx), device, stream_ptr, workspace.data_ptr(),
                                       workspace.numel() * workspace.element_size())
    if code != UNITY_OK:
        raise UnityError(code, "unity_create failed")
    return ctx


def unity_destroy(ctx) -> None:
    load_library().unity_destroy(ctx)


def unity_check_status(ctx) -> None:
    _raise(ctx, load_library().unity_check_status(ctx))


def unity_launch_count(ctx) -> int:
    return int(load_library().unity_launch_count(ctx))


PROF_CLASSES = ["fwd_gemm", "grad_gemm", "dh_gemm", "dw_gemm"]


def unity_set_profiling(ctx, enable: bool) -> None:
    _raise(ctx, load_library().unity_set_profiling(ctx, 1 if enable else 0))


OPT_CTAS = {"fwd_gemm": 0, "grad_gemm": 1, "dh_gemm": 2, "dw_gemm": 3}


def unity_set_option(ctx, option: int, value: int) -> None:
    _raise(ctx, load_library().unity_set_option(ctx, option, value))


def unity_get_profile(ctx) -> dict:
    n = len(PROF_CLASSES)
    ms = (C.c_double * n)()
    cnt = (C.c_int64 * n)()
    _raise(ctx, load_library().unity_get_profile(ctx, ms, cnt))
    return {name: {"ms": float(ms[i]), "launches": int(cnt[i])} for i, name in enumerate(PROF_CLASSES)}


def unity_role_advantage(ctx, n_traj: int, n_roles: int, n_groups: int, inv_role, inv_group, inv_traj,
                         r_node, r_turn, r_traj, lam: Optional[Sequence[float]], eps: float, ddof: int,
                         cu_seqlens, tok_mask, adv_inv, adv_tok, seg_mean=None, seg_std=None) -> None:
    n_inv = int(inv_role.numel())
    n_tok = int(adv_tok.numel()) if adv_tok is not None else 0
    lam_arr = None
    if lam is not None:
        flat = [float(x) for row in lam for x in (row if hasattr(row, "__iter__") else [row])]
        lam_arr = (C.c_float * len(flat))(*flat)
    p = unity_adv_params(eps, ddof)
    i32, f32 = torch.int32, torch.float32
    code = load_library().unity_role_advantage(
        ctx, n_inv, n_traj, n_roles, n_groups, _ptr(inv_role, i32, "inv_role"), _ptr(inv_group, i32, "inv_group"),
        _ptr(inv_traj, i32, "inv_traj"), _ptr(r_node, f32, "r_node"), _ptr(r_turn, f32, "r_turn"),
        _ptr(r_traj, f32, "r_traj"), lam_arr, C.byref(p), n_tok, _ptr(cu_seqlens, torch.int64, "cu_seqlens"),
        _ptr(tok_mask, torch.uint8, "tok_mask"), _ptr(adv_inv, f32, "adv_inv"), _ptr(adv_tok, f32, "adv_tok"),
        _ptr(seg_mean, f32, "seg_mean"), _ptr(seg_std, f32, "seg_std"))
    _raise(ctx, code)


RULE_NONE, RULE_ABSOLUTE, RULE_MARGINAL = 0, 1, 2


def unity_reward_assembly(ctx, inv_role, inv_traj, inv_turn, score, n_scores, inv_end, rules, r_turn) -> None:
    """score: f32 CUDA tensor [n_traj, max_turns]; rules: sequence of (mode, shift) per role."""
    n_traj, max_turns = int(score.shape[0]), int(score.shape[1])
    arr = (unity_reward_rule * len(rules))(*[unity_reward_rule(int(m), int(sh)) for m, sh in rules])
    i32 = torch.int32
    code = load_library().unity_reward_assembly(
        ctx, int(inv_role.numel()), n_traj, len(rules), max_turns, _ptr(inv_role, i32, "inv_role"),
        _ptr(inv_traj, i32, "inv_traj"), _ptr(inv_turn, i32, "inv_turn"), _ptr(score, torch.float32, "score"),
        _ptr(n_scores, i32, "n_scores"), _ptr(inv_end, torch.uint8, "inv_end"), arr,
        _ptr(r_turn, torch.float32, "r_turn"))
    _raise(ctx, code)


def unity_gae(ctx, cu_seqlens, rewards, values, tok_mask, gamma: float, lam: float, advantages, returns) -> None:
    f32 = torch.float32
    code = load_library().unity_gae(ctx, int(cu_seqlens.numel()) - 1, int(rewards.numel()),
                                    _ptr(cu_seqlens, torch.int64, "cu_seqlens"), _ptr(rewards, f32, "rewards"),
                                    _ptr(values, f32, "values"), _ptr(tok_mask, torch.uint8, "tok_mask"), gamma, lam,
                                    _ptr(advantages, f32, "advantages"), _ptr(returns, f32, "returns"))
    _raise(ctx, code)


def unity_value_loss_fwd_bwd(ctx, cu_seqlens, inv_role, role_model: Sequence[int], K: int, tok_mask, values,
                             old_values, returns, clip_v: float, norm: Optional[Sequence[float]], loss,
                             clip_frac=None, tok_loss=None, dvalues=None) -> None:
    f32 = torch.float32
    rm = (C.c_int32 * len(role_model))(*[int(x) for x in role_model])
    norm_arr = None if norm is None else (C.c_float * len(norm))(*[float(x) for x in norm])
    code = load_library().unity_value_loss_fwd_bwd(
        ctx, int(inv_role.numel()), len(role_model), K, int(values.numel()),
        _ptr(cu_seqlens, torch.int64, "cu_seqlens"), _ptr(inv_role, torch.int32, "inv_role"), rm,
        _ptr(tok_mask, torch.uint8, "tok_mask"), _ptr(values, f32, "values"), _ptr(old_values, f32, "old_values"),
        _ptr(returns, f32, "returns"), float(clip_v), norm_arr, _ptr(loss, f32, "loss"),
        _ptr(clip_frac, f32, "clip_frac"), _ptr(tok_loss, f32, "tok_loss"), _ptr(dvalues, f32, "dvalues"))
    _raise(ctx, code)


def unity_ready_batch_plan(ctx, cu_seqlens, inv_role, inv_traj, traj_done, role_model: Sequence[int], K: int,
                           seed: int, n_parts: int, pad_to: int, order, out_cu_seqlens, model_offsets, part_offsets,
                           totals) -> None:
    """order: int32 [n_inv]; out_cu_seqlens: int64 [n_inv+1]; model_offsets: int32 [K+1]; part_offsets: int32
    [K*n_parts+1]; totals: int64 [2] - all CUDA tensors written by the call."""
    i32, i64 = torch.int32, torch.int64
    rm = (C.c_int32 * len(role_model))(*[int(x) for x in role_model])
    p = unity_batch_params(int(seed) & 0xFFFFFFFFFFFFFFFF, int(n_parts), int(pad_to))
    code = load_library().unity_ready_batch_plan(
        ctx, int(inv_role.numel()), int(traj_done.numel()), len(role_model), K, _ptr(cu_seqlens, i64, "cu_seqlens"),
        _ptr(inv_role, i32, "inv_role"), _ptr(inv_traj, i32, "inv_traj"), _ptr(traj_done, torch.uint8, "traj_done"),
        rm, C.byref(p), _ptr(order, i32, "order"), _ptr(out_cu_seqlens, i64, "out_cu_seqlens"),
        _ptr(model_offsets, i32, "model_offsets"), _ptr(part_offsets, i32, "part_offsets"), _ptr(totals, i64, "totals"))
    _raise(ctx, code)


def unity_ready_batch_gather(ctx, order, src_cu_seqlens, out_cu_seqlens, totals, src, dst, pad_value=0) -> None:
    """src: CUDA tensor [n_tok_src, ...] in buffer order; dst: CUDA tensor [>= totals[1], ...] of the same dtype and
    trailing shape; pad rows are filled with pad_value."""
    if src.dtype != dst.dtype or tuple(src.shape[1:]) != tuple(dst.shape[1:]):
        raise TypeError("src and dst must agree in dtype and trailing shape")
    row_bytes = src.element_size()
    for d in src.shape[1:]:
        row_bytes *= int(d)
    pad = bytes(torch.tensor([pad_value], dtype=src.dtype).view(torch.uint8).tolist())
    code = load_library().unity_ready_batch_gather(
        ctx, int(order.numel()), int(src.shape[0]), _ptr(order, torch.int32, "order"),
        _ptr(src_cu_seqlens, torch.int64, "src_cu_seqlens"), _ptr(out_cu_seqlens, torch.int64, "out_cu_seqlens"),
        _ptr(totals, torch.int64, "totals"), row_bytes, _ptr(src, None, "src"), _ptr(dst, None, "dst"), pad, len(pad))
    _raise(ctx, code)


def unity_align_rewards(ctx, cu_seqlens, tok_mask, r_inv, tok_reward) -> None:
    code = load_library().unity_align_rewards(
        ctx, int(r_inv.numel()), int(tok_reward.numel()), _ptr(cu_seqlens, torch.int64, "cu_seqlens"),
        _ptr(tok_mask, torch.uint8, "tok_mask"), _ptr(r_inv, torch.float32, "r_inv"),
        _ptr(tok_reward, torch.float32, "tok_reward"))
    _raise(ctx, code)


UNITY_NOALLOC_MAX_INV = 65536
UNITY_NOALLOC_MAX_SEG = 65536


def unity_role_advantage_noalloc(device: int, stream_ptr: int, n_traj: int, n_roles: int, n_groups: int, inv_role,
                                 inv_group, inv_traj, r_node, r_turn, r_traj, lam: Optional[Sequence[float]],
                                 eps: float, ddof: int, cu_seqlens, tok_mask, adv_inv, adv_tok, seg_mean=None,
                                 seg_std=None, bad_index_out=None) -> None:
    """Context-free, allocation-free form of unity_role_advantage (scratch is a fixed array inside the library;
    at most UNITY_NOALLOC_MAX_INV invocations).  Same arguments otherwise; `bad_index_out` is an optional int32
    CUDA tensor of one element."""
    n_inv = int(inv_role.numel())
    n_tok = int(adv_tok.numel()) if adv_tok is not None else 0
    lam_arr = None
    if lam is not None:
        flat = [float(x) for row in lam for x in (row if hasattr(row, "__iter__") else [row])]
        lam_arr = (C.c_float * len(flat))(*flat)
    p = unity_adv_params(eps, ddof)
    i32, f32 = torch.int32, torch.float32
    msg = C.create_string_buffer(256)
    code = load_library().unity_role_advantage_noalloc(
        device, stream_ptr, n_inv, n_traj, n_roles, n_groups, _ptr(inv_role, i32, "inv_role"),
        _ptr(inv_group, i32, "inv_group"), _ptr(inv_traj, i32, "inv_traj"), _ptr(r_node, f32, "r_node"),
        _ptr(r_turn, f32, "r_turn"), _ptr(r_traj, f32, "r_traj"), lam_arr, C.byref(p), n_tok,
        _ptr(cu_seqlens, torch.int64, "cu_seqlens"), _ptr(tok_mask, torch.uint8, "tok_mask"),
        _ptr(adv_inv, f32, "adv_inv"), _ptr(adv_tok, f32, "adv_tok"), _ptr(seg_mean, f32, "seg_mean"),
        _ptr(seg_std, f32, "seg_std"), _ptr(bad_index_out, i32, "bad_index_out"), msg, 256)
    if code != UNITY_OK:
        raise UnityError(code, msg.value.decode())


def _make_rows(hidden, W, cu_seqlens, inv_role, role_model, target, tok_mask, inv_temperature, keep):
    K = len(W)
    n_tok, H = int(hidden.shape[0]), int(hidden.shape[1])
    V = int(W[0].shape[0])
    for k, w in enumerate(W):
        if tuple(w.shape) != (V, H):
            raise ValueError(f"W[{k}] has shape {tuple(w.shape)}, expected {(V, H)}")
    Wp = (C.c_void_p * K)(*[_ptr(w, torch.bfloat16, "W") for w in W])
    rm = (C.c_int32 * len(role_model))(*[int(x) for x in role_model])
    keep.extend([Wp, rm])
    rows = unity_rows(n_tok, H, V, K, int(inv_role.numel()), len(role_model),
                      _ptr(hidden, torch.bfloat16, "hidden"), Wp, _ptr(cu_seqlens, torch.int64, "cu_seqlens"),
                      _ptr(inv_role, torch.int32, "inv_role"), rm, _ptr(target, torch.int32, "target"),
                      _ptr(tok_mask, torch.uint8, "tok_mask"), float(inv_temperature))
    return rows


def unity_logprob_fwd(ctx, hidden, W, cu_seqlens, inv_role, role_model, target, tok_mask, inv_temperature,
                      logp, entropy=None, lse=None) -> None:
    keep = []
    rows = _make_rows(hidden, W, cu_seqlens, inv_role, role_model, target, tok_mask, inv_temperature, keep)
    f32 = torch.float32
    code = load_library().unity_logprob_fwd(ctx, C.byref(rows), _ptr(logp, f32, "logp"),
                                            _ptr(entropy, f32, "entropy"), _ptr(lse, f32, "lse"))
    _raise(ctx, code)


def unity_ppo_loss_fwd_bwd(ctx, hidden, W, cu_seqlens, inv_role, role_model, target, tok_mask, inv_temperature,
                           clip_lo, clip_hi, kl_coef, kl_mode, ent_coef, norm: Optional[Sequence[float]],
                           accumulate_dW: bool, old_logp, ref_logp, adv_tok, loss, metrics, logp, entropy,
                           tok_loss, dHidden, dW, logp_in=None, entropy_in=None, lse_in=None) -> None:
    keep = []
    rows = _make_rows(hidden, W, cu_seqlens, inv_role, role_model, target, tok_mask, inv_temperature, keep)
    norm_arr = None
    if norm is not None:
        norm_arr = (C.c_float * len(norm))(*[float(x) for x in norm])
    f32_ = torch.float32
    p = unity_ppo_params(clip_lo, clip_hi, kl_coef, kl_mode, ent_coef, norm_arr, 1 if accumulate_dW else 0,
                         _ptr(logp_in, f32_, "logp_in"), _ptr(entropy_in, f32_, "entropy_in"), _ptr(lse_in, f32_, "lse_in"))
    dWp = (C.c_void_p * len(dW))(*[_ptr(g, torch.float32, "dW") for g in dW])
    f32 = torch.float32
    code = load_library().unity_ppo_loss_fwd_bwd(
        ctx, C.byref(rows), C.byref(p), _ptr(old_logp, f32, "old_logp"), _ptr(ref_logp, f32, "ref_logp"),
        _ptr(adv_tok, f32, "adv_tok"), _ptr(loss, f32, "loss"), _ptr(metrics, f32, "metrics"),
        _ptr(logp, f32, "logp"), _ptr(entropy, f32, "entropy"), _ptr(tok_loss, f32, "tok_loss"),
        _ptr(dHidden, torch.bfloat16, "dHidden"), dWp)
    _raise(ctx, code)


# ------------------------------------------------------------------------------------------------
# token losses: cross entropy and distillation from a teacher's listed entries
# ------------------------------------------------------------------------------------------------
UNITY_F32, UNITY_BF16 = 0, 1
TEACHER_LOGITS, TEACHER_LOGPROBS = 0, 1
UNITY_MAX_TOP = 128


def unity_token_loss_workspace_bytes(n_tok: int, H: int, V: int, K: int, n_top: int = 0, backward: bool = True) -> int:
    return int(load_library().unity_token_loss_workspace_bytes(n_tok, H, V, K, n_top, 1 if backward else 0))


def _sized(t: Optional[torch.Tensor], shape, dtype, device, name) -> Optional[int]:
    """data_ptr of an optional tensor that must have exactly this shape, type and device."""
    if t is None:
        return None
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the call on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _token_loss_args(hidden, W, cu_seqlens, inv_role, role_model, target, tok_mask, inv_temperature, norm, tok_weight,
                     loss, tok_loss, lse, dHidden, dW, top=None):
    """What both losses take: (rows, norm array, pointers of the per-token arrays and outputs, dW array, dW type, pointers
    of the teacher's lists).  `top` = (top_ids, top_vals)."""
    if hidden.dim() != 2 or not W or W[0].dim() != 2 or inv_role.dim() != 1 or loss is None:
        raise ValueError("hidden must be [n_tok, H], W a non-empty sequence of [V, H], inv_role [n_inv] and loss a tensor")
    n_tok, H = hidden.shape
    K, V, n_inv, dev = len(W), W[0].shape[0], inv_role.shape[0], hidden.device
    f32, i32, b16 = torch.float32, torch.int32, torch.bfloat16
    per_tok = (n_tok,)
    h = _sized(hidden, (n_tok, H), b16, dev, "hidden")
    Wp = (C.c_void_p * K)(*[_sized(w, (V, H), b16, dev, "W") for w in W])
    rm = (C.c_int32 * len(role_model))(*[int(x) for x in role_model])
    rows = unity_rows(n_tok, H, V, K, n_inv, len(role_model), h, Wp,
                      _sized(cu_seqlens, (n_inv + 1,), torch.int64, dev, "cu_seqlens"),
                      _sized(inv_role, (n_inv,), i32, dev, "inv_role"), rm, _sized(target, per_tok, i32, dev, "target"),
                      _sized(tok_mask, per_tok, torch.uint8, dev, "tok_mask"), float(inv_temperature))
    norm_arr = None
    if norm is not None:
        if len(norm) != K:
            raise ValueError(f"norm: expected {K} values, got {len(norm)}")
        norm_arr = (C.c_float * K)(*[float(x) for x in norm])
    per = (_sized(tok_weight, per_tok, f32, dev, "tok_weight"), _sized(loss, (K,), f32, dev, "loss"),
           _sized(tok_loss, per_tok, f32, dev, "tok_loss"), _sized(lse, per_tok, f32, dev, "lse"),
           _sized(dHidden, (n_tok, H), b16, dev, "dHidden"))
    dWp, dw_type = None, UNITY_F32
    if dW is not None:
        if len(dW) != K:
            raise ValueError(f"dW: expected {K} tensors, got {len(dW)}")
        dtype = dW[0].dtype
        if dtype not in (f32, b16):
            raise TypeError(f"dW: expected float32 or bfloat16, got {dtype}")
        dw_type = UNITY_BF16 if dtype == b16 else UNITY_F32
        dWp = (C.c_void_p * K)(*[_sized(g, (V, H), dtype, dev, "dW") for g in dW])
    lists = ()
    if top is not None:
        if top[0].dim() != 2:
            raise ValueError("top_ids must be [n_tok, n_top]")
        shape = (n_tok, top[0].shape[1])
        lists = (_sized(top[0], shape, i32, dev, "top_ids"), _sized(top[1], shape, f32, dev, "top_vals"))
    if not hidden.is_cuda:
        raise ValueError("hidden must be a CUDA tensor")
    return rows, norm_arr, per, dWp, dw_type, lists


def unity_cross_entropy_fwd_bwd(ctx, hidden, W, cu_seqlens, inv_role, role_model, target, tok_mask, inv_temperature,
                                label_smoothing: float, z_loss: float, norm: Optional[Sequence[float]],
                                accumulate_dW: bool, tok_weight, loss, tok_loss=None, lse=None, dHidden=None,
                                dW=None) -> None:
    """dHidden / dW None: that gradient is not computed; dW: K tensors [V, H], all f32 or all bf16."""
    rows, norm_arr, per, dWp, dw_type, _ = _token_loss_args(hidden, W, cu_seqlens, inv_role, role_model, target, tok_mask,
                                                            inv_temperature, norm, tok_weight, loss, tok_loss, lse,
                                                            dHidden, dW)
    p = unity_ce_params(float(label_smoothing), float(z_loss), norm_arr, 1 if accumulate_dW else 0, dw_type)
    _raise(ctx, load_library().unity_cross_entropy_fwd_bwd(ctx, C.byref(rows), C.byref(p), *per, dWp))


def unity_distill_fwd_bwd(ctx, hidden, W, cu_seqlens, inv_role, role_model, target, tok_mask, inv_temperature, top_ids,
                          top_vals, teacher_mode: int, kd_coef: float, hard_coef: float,
                          norm: Optional[Sequence[float]], accumulate_dW: bool, tok_weight, loss, tok_loss=None,
                          lse=None, dHidden=None, dW=None) -> None:
    """top_ids int32 / top_vals f32: CUDA tensors [n_tok, n_top]; target may be None when hard_coef is 0."""
    rows, norm_arr, per, dWp, dw_type, lists = _token_loss_args(hidden, W, cu_seqlens, inv_role, role_model, target,
                                                                tok_mask, inv_temperature, norm, tok_weight, loss,
                                                                tok_loss, lse, dHidden, dW, (top_ids, top_vals))
    p = unity_distill_params(top_ids.shape[1], int(teacher_mode), float(kd_coef), float(hard_coef), norm_arr,
                             1 if accumulate_dW else 0, dw_type)
    _raise(ctx, load_library().unity_distill_fwd_bwd(ctx, C.byref(rows), C.byref(p), *lists, *per, dWp))


# ------------------------------------------------------------------------------------------------
# around the update: final norm, gradient clipping, sampling
# ------------------------------------------------------------------------------------------------
def unity_rms_norm_workspace_bytes(n_tok: int, H: int, K: int) -> int:
    return int(load_library().unity_rms_norm_workspace_bytes(n_tok, H, K))


def unity_clip_grad_norm_workspace_bytes(n_tensors: int, K: int) -> int:
    return int(load_library().unity_clip_grad_norm_workspace_bytes(n_tensors, K))


_TYPES = {torch.float32: UNITY_F32, torch.bfloat16: UNITY_BF16}
_PTRS = [C.c_void_p * k for k in range(UNITY_MAX_MODELS + 1)]      # (making an array type costs as much as filling it)
_INTS = [C.c_int32 * k for k in range(UNITY_MAX_ROLES + 1)]


def _fit(t: Optional[torch.Tensor], shape, dtype, device: int, name) -> Optional[int]:
    """_sized on a CUDA device, with the fewest calls where all is well: these calls take microseconds themselves."""
    if t is None:
        return None
    if t.shape == shape and t.dtype is dtype and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    return _sized(t, shape, dtype, torch.device("cuda", device), name)


def _type_of(t: torch.Tensor, name) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"{name}: expected float32 or bfloat16, got {t.dtype}")
    return kind


def _norm_rows(x, shape, gamma, cu_seqlens, inv_role, role_model, tok_mask, eps):
    if len(shape) != 2 or not gamma or inv_role.dim() != 1:
        raise ValueError("token rows must be [n_tok, H], gamma a non-empty sequence of [H] and inv_role [n_inv]")
    dev = x.get_device()
    if dev < 0:
        raise ValueError("token rows must be a CUDA tensor")
    K, R = len(gamma), len(role_model)
    n_tok, H = shape
    per_model, kind, n_inv = (H,), gamma[0].dtype, inv_role.shape[0]
    if K > UNITY_MAX_MODELS or R > UNITY_MAX_ROLES:
        raise ValueError(f"at most {UNITY_MAX_MODELS} models and {UNITY_MAX_ROLES} roles")
    return unity_norm_rows(n_tok, H, K, n_inv, R, _fit(cu_seqlens, (n_inv + 1,), torch.int64, dev, "cu_seqlens"),
                           _fit(inv_role, (n_inv,), torch.int32, dev, "inv_role"), _INTS[R](*role_model),
                           _fit(tok_mask, (n_tok,), torch.uint8, dev, "tok_mask"),
                           _PTRS[K](*[_fit(g, per_model, kind, dev, "gamma") for g in gamma]), _type_of(gamma[0], "gamma"), eps)


def unity_rms_norm_fwd(ctx, x, gamma, cu_seqlens, inv_role, role_model, tok_mask, eps: float, y, residual=None,
                       res_out=None) -> None:
    """x, y: bf16 [n_tok, H]; gamma: K tensors [H], all f32 or all bf16; residual, res_out: f32 or bf16 [n_tok, H]."""
    shape, b16, dev = x.shape, torch.bfloat16, x.get_device()
    rows = _norm_rows(x, shape, gamma, cu_seqlens, inv_role, role_model, tok_mask, eps)
    rtype, kind = (UNITY_BF16, b16) if residual is None else (_type_of(residual, "residual"), residual.dtype)
    if y is None:
        raise ValueError("y is None")
    code = load_library().unity_rms_norm_fwd(
        ctx, rows, _fit(x, shape, b16, dev, "x"), _fit(residual, shape, kind, dev, "residual"), rtype,
        _fit(y, shape, b16, dev, "y"), _fit(res_out, shape, kind, dev, "res_out"))
    if code:
        _raise(ctx, code)


def unity_rms_norm_bwd(ctx, res, gamma, cu_seqlens, inv_role, role_model, tok_mask, eps: float, dy, dx, dres=None,
                       dgamma=None, accumulate_dgamma: bool = False) -> None:
    """res, dres, dx: all f32 or all bf16 [n_tok, H]; dy: bf16; dgamma: K f32 tensors [H], or None for a frozen norm."""
    shape, kind, dev = res.shape, res.dtype, res.get_device()
    rows = _norm_rows(res, shape, gamma, cu_seqlens, inv_role, role_model, tok_mask, eps)
    if dy is None or dx is None:
        raise ValueError("dy / dx is None")
    dg = None
    if dgamma is not None:
        if len(dgamma) != len(gamma):
            raise ValueError(f"dgamma: expected {len(gamma)} tensors, got {len(dgamma)}")
        dg = _PTRS[len(dgamma)](*[_fit(g, shape[1:], torch.float32, dev, "dgamma") for g in dgamma])
    code = load_library().unity_rms_norm_bwd(
        ctx, rows, _fit(res, shape, kind, dev, "res"), _type_of(res, "res"), _fit(dy, shape, torch.bfloat16, dev, "dy"),
        _fit(dres, shape, kind, dev, "dres"), _fit(dx, shape, kind, dev, "dx"), dg, 1 if accumulate_dgamma else 0)
    if code:
        _raise(ctx, code)


class GradTensors:
    """The tensors of a clipping call, checked and laid out once: gradients usually stay where they are from step to step.

    grads: contiguous f32 or bf16 CUDA tensors of any shape; models: the model of each; outs: tensors that take the scaled
    gradients (of the same type or bf16, None for in place), or None for all in place.  Keeps the tensors and their memory alive; a
    tensor that is given other memory later (set_, .data) is not followed there."""

    def __init__(self, grads: Sequence[torch.Tensor], models: Sequence[int], outs: Optional[Sequence[Optional[torch.Tensor]]] = None):
        self.grads, self.outs = list(grads), [None] * len(grads) if outs is None else list(outs)
        models = [int(m) for m in models]
        if len(models) != len(self.grads) or len(self.outs) != len(self.grads):
            raise ValueError("grads, models and outs must have the same length")
        self.device = self.grads[0].device if self.grads else None
        self.array = (unity_tensor * len(models))()
        for e, g, o, m in zip(self.array, self.grads, self.outs, models):
            e.type = _type_of(g, "grads")
            e.data, e.n, e.model = _sized(g, g.shape, g.dtype, self.device, "grads"), g.numel(), m
            if o is not None:
                e.out_type = _type_of(o, "outs")
                e.out = _sized(o, g.shape, o.dtype, self.device, "outs")
            if not g.is_cuda:
                raise ValueError("grads must be CUDA tensors")
        self.memory = [t.untyped_storage() for t in (*self.grads, *self.outs) if t is not None]

    def __len__(self):
        return len(self.grads)


def unity_clip_grad_norm(ctx, tensors: GradTensors, max_norm: Optional[Sequence[float]], norm, coef=None) -> None:
    """norm, coef: f32 CUDA tensors [K]; max_norm: K bounds (inf: none), or None to compute the norms only."""
    K = norm.shape[0]
    if max_norm is not None and len(max_norm) != K:
        raise ValueError(f"max_norm: expected {K} values, got {len(max_norm)}")
    bounds = None if max_norm is None else (C.c_float * K)(*max_norm)
    dev = norm.get_device()
    if dev < 0 or (tensors.grads and tensors.grads[0].get_device() != dev):
        raise ValueError("norm must be a CUDA tensor on the gradients' device")
    code = load_library().unity_clip_grad_norm(ctx, len(tensors.grads), tensors.array, K, bounds,
                                               _fit(norm, (K,), torch.float32, dev, "norm"),
                                               _fit(coef, (K,), torch.float32, dev, "coef"))
    if code:
        _raise(ctx, code)


def unity_sample(ctx, logits, rules, u, token, row_role=None, row_mask=None, logp=None, logp_kept=None, n_kept=None) -> None:
    """logits: f32 or bf16 [n_rows, V], rows of any pitch; rules: (temperature, top_k, top_p, min_p) of each role."""
    shape = logits.shape
    if len(shape) != 2 or (shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [n_rows, V] with consecutive entries in a row")
    dev = logits.get_device()
    if dev < 0:
        raise ValueError("logits must be a CUDA tensor")
    if u is None or token is None:
        raise ValueError("u / token is None")
    n, V = shape
    f32, i32, per = torch.float32, torch.int32, (n,)
    arr = (unity_sampling_rule * len(rules))(*rules)
    code = load_library().unity_sample(
        ctx, n, V, logits.data_ptr(), _type_of(logits, "logits"), logits.stride(0) if n > 1 else V, len(rules),
        _fit(row_role, per, i32, dev, "row_role"), arr, _fit(row_mask, per, torch.uint8, dev, "row_mask"),
        _fit(u, per, f32, dev, "u"), _fit(token, per, i32, dev, "token"), _fit(logp, per, f32, dev, "logp"),
        _fit(logp_kept, per, f32, dev, "logp_kept"), _fit(n_kept, per, i32, dev, "n_kept"))
    if code:
        _raise(ctx, code)


# ------------------------------------------------------------------------------------------------
class Context:
    """Owns a workspace tensor and a unity_ctx bound to a torch stream."""

    def __init__(self, device: int = 0, workspace_bytes: int = 1 << 28, stream: Optional[torch.cuda.Stream] = None):
        self.device = int(device)
        with torch.cuda.device(self.device):
            self.stream = stream or torch.cuda.current_stream()
            self.workspace = torch.empty(int(workspace_bytes), dtype=torch.uint8, device=f"cuda:{self.device}")
        self.ctx = unity_create(self.device, self.stream.cuda_stream, self.workspace)

    def close(self):
        if self.ctx is not None:
            unity_destroy(self.ctx)
            self.ctx = None
            self.workspace = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def check_status(self):
        unity_check_status(self.ctx)

    @property
    def launch_count(self) -> int:
        return unity_launch_count(self.ctx)

    def set_profiling(self, enable: bool):
        unity_set_profiling(self.ctx, enable)

    def set_option(self, option: int, value: int):
        unity_set_option(self.ctx, option, value)

    def get_profile(self) -> dict:
        return unity_get_profile(self.ctx)

    def role_advantage(self, *a, **kw):
        return unity_role_advantage(self.ctx, *a, **kw)

    def reward_assembly(self, *a, **kw):
        return unity_reward_assembly(self.ctx, *a, **kw)

    def gae(self, *a, **kw):
        return unity_gae(self.ctx, *a, **kw)

    def value_loss_fwd_bwd(self, *a, **kw):
        return unity_value_loss_fwd_bwd(self.ctx, *a, **kw)

    def ready_batch_plan(self, *a, **kw):
        return unity_ready_batch_plan(self.ctx, *a, **kw)

    def ready_batch_gather(self, *a, **kw):
        return unity_ready_batch_gather(self.ctx, *a, **kw)

    def align_rewards(self, *a, **kw):
        return unity_align_rewards(self.ctx, *a, **kw)

    def logprob_fwd(self, *a, **kw):
        return unity_logprob_fwd(self.ctx, *a, **kw)

    def ppo_loss_fwd_bwd(self, *a, **kw):
        return unity_ppo_loss_fwd_bwd(self.ctx, *a, **kw)

    def _on_device(self, hidden, name="hidden"):
        if hidden.get_device() not in (self.device, -1):
            raise ValueError(f"{name} is on {hidden.device}, the context on cuda:{self.device}")

    def cross_entropy_fwd_bwd(self, hidden, *a, **kw):
        self._on_device(hidden)
        return unity_cross_entropy_fwd_bwd(self.ctx, hidden, *a, **kw)

    def distill_fwd_bwd(self, hidden, *a, **kw):
        self._on_device(hidden)
        return unity_distill_fwd_bwd(self.ctx, hidden, *a, **kw)

    def rms_norm_fwd(self, x, *a, **kw):
        self._on_device(x, "x")
        return unity_rms_norm_fwd(self.ctx, x, *a, **kw)

    def rms_norm_bwd(self, res, *a, **kw):
        self._on_device(res, "res")
        return unity_rms_norm_bwd(self.ctx, res, *a, **kw)

    def clip_grad_norm(self, tensors, max_norm, norm, *a, **kw):
        self._on_device(norm, "norm")
        return unity_clip_grad_norm(self.ctx, tensors, max_norm, norm, *a, **kw)

    def sample(self, logits, *a, **kw):
        self._on_device(logits, "logits")
        return unity_sample(self.ctx, logits, *a, **kw)
