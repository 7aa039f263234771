"""Binding of include/mrl.h: ctypes, and a CPython extension for the calls whose
host side would take longer than their kernels.  Argument marshalling only.

Every function takes torch tensors that already live on the GPU (the library
only accepts device pointers), checks dtype / contiguity / device on the host,
and forwards raw pointers plus the current torch stream.  There is no CPU or
PyTorch fallback: if the shared library is missing, loading raises.  The
extension only marshals faster: without it every call goes through ctypes.
"""
from __future__ import annotations

import ctypes
import importlib.util
import operator
import os
import warnings
from ctypes import POINTER, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_uint64, c_void_p
from dataclasses import dataclass

import torch

F32, BF16, E4M3 = 0, 1, 2
ADV_CENTER, ADV_GROUP_ZN, ADV_BATCH_ZN = 0, 1, 2
PROF_CLASSES = ("prep", "adv", "gemm_fwd", "row_epilogue", "operand_prep", "gemm_dh", "gemm_dw", "final")

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None


class MrlError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: mrl status {status} ({status_string(status)})")


def library_path() -> str:
    return os.path.join(_HERE, "libmrl.so")


class _LossConfig(ctypes.Structure):
    _fields_ = [("clip_eps_low", c_float), ("clip_eps_high", c_float), ("kl_beta", c_float),
                ("sgt_lambda", c_float), ("loss_agg", c_int32), ("accumulate_dw", c_int32),
                ("dh_dtype", c_int32), ("chunk_rows", c_int32), ("scored_rows_hint", c_int64),
                ("ratio_level", c_int32), ("debug_sync", c_int32)]


class _DistillConfig(ctypes.Structure):
    _fields_ = [("temperature", c_float), ("renormalize", c_int32), ("accumulate_dw", c_int32), ("dh_dtype", c_int32), ("dw_dtype", c_int32),
                ("chunk_rows", c_int32)]


class _ParamTensor(ctypes.Structure):
    _fields_ = [("param", c_void_p), ("copy", c_void_p), ("grad", c_void_p), ("m", c_void_p), ("v", c_void_p), ("m_scale", c_void_p),
                ("v_scale", c_void_p), ("n", c_int64), ("weight_decay", c_float), ("grad_dtype", c_int32)]


class _AdamWConfig(ctypes.Structure):
    _fields_ = [("lr", c_double), ("beta1", c_double), ("beta2", c_double), ("eps", c_double), ("step", c_int64), ("seed", c_uint64),
                ("state_dtype", c_int32), ("skip_nonfinite", c_int32), ("lr_dev", c_void_p), ("step_dev", c_void_p)]


@dataclass
class LossConfig:
    clip_eps_low: float = 0.2
    clip_eps_high: float = 0.2
    kl_beta: float = 0.04
    sgt_lambda: float = 0.1
    loss_agg: int = 0
    accumulate_dw: int = 0
    dh_dtype: int = BF16
    chunk_rows: int = 0
    scored_rows_hint: int = 0
    ratio_level: int = 0
    debug_sync: int = 0

    def to_c(self) -> _LossConfig:
        return _LossConfig(self.clip_eps_low, self.clip_eps_high, self.kl_beta, self.sgt_lambda,
                           self.loss_agg, self.accumulate_dw, self.dh_dtype, self.chunk_rows,
                           self.scored_rows_hint, self.ratio_level, self.debug_sync)


@dataclass
class DistillConfig:
    temperature: float = 1.0
    renormalize: int = 1
    accumulate_dw: int = 0
    dh_dtype: int = BF16
    dw_dtype: int = F32
    chunk_rows: int = 0

    def to_c(self) -> _DistillConfig:
        return _DistillConfig(self.temperature, int(self.renormalize), int(self.accumulate_dw), self.dh_dtype, self.dw_dtype, self.chunk_rows)


DISTILL_STATS_FIELDS = ("loss_total", "n_scored_rows", "n_empty_rows", "n_saturated_rows", "n_bad_ids")
DISTILL_STATS_BYTES = 8 + 4 * 8
STATS_FIELDS = ("loss_total", "loss_pg", "loss_kl", "loss_sgt", "mean_ratio", "max_ratio", "mean_k3",
                "n_scored_tokens", "n_clipped_tokens", "n_zero_grad_tokens", "n_bad_targets",
                "n_unprocessed_rows", "n_saturated_rows")
STATS_BYTES = 7 * 8 + 6 * 8


def lib() -> ctypes.CDLL:
    """Loads libmrl.so (once).  Raises if it has not been built."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} not found: build it with `python -m paper_2605_07244_amd.build` "
            "(there is no fallback implementation)")
    L = ctypes.CDLL(path)
    L.mrl_status_string.restype = c_char_p
    L.mrl_status_string.argtypes = [c_int]
    L.mrl_version.restype = c_int
    L.mrl_token_logprobs_workspace.restype = c_size_t
    L.mrl_token_logprobs_workspace.argtypes = [c_int64, c_int32, c_int32, c_int32]
    L.mrl_token_logprobs.restype = c_int
    L.mrl_token_logprobs.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_int32,
                                     c_int32, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    L.mrl_token_logprobs_static.restype = c_int
    L.mrl_token_logprobs_static.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_int32,
                                            c_int32, c_void_p, c_void_p, c_void_p]
    L.mrl_token_scores_workspace.restype = c_size_t
    L.mrl_token_scores_workspace.argtypes = [c_int64, c_int32, c_int32, c_int32]
    L.mrl_token_scores.restype = c_int
    L.mrl_token_scores.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_int32,
                                   c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    L.mrl_group_advantages.restype = c_int
    L.mrl_group_advantages.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int32,
                                       c_int32, c_float, c_int32, c_float, c_float, c_float,
                                       c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
    L.mrl_grpo_loss_workspace.restype = c_size_t
    L.mrl_grpo_loss_workspace.argtypes = [c_int64, c_int32, c_int32, c_int32, c_int32, POINTER(_LossConfig)]
    L.mrl_grpo_loss_fwd_bwd.restype = c_int
    L.mrl_grpo_loss_fwd_bwd.argtypes = [c_void_p] * 9 + [c_int64, c_int32, c_int32, c_int32, c_int32, c_int32,
                                                         POINTER(_LossConfig), c_void_p, c_void_p, c_void_p,
                                                         c_void_p, c_void_p, c_size_t, c_void_p]
    L.mrl_profile_enable.restype = c_int
    L.mrl_profile_enable.argtypes = [c_int]
    L.mrl_profile_collect.restype = c_int
    L.mrl_profile_collect.argtypes = [POINTER(c_double), POINTER(c_int64)]
    L.mrl_thl_word_align.restype = c_int
    L.mrl_thl_word_align.argtypes = [c_void_p] * 7 + [c_int64, c_int32, c_int32, c_int32, c_float, c_void_p,
                                                      c_void_p, c_void_p]
    L.mrl_rms_norm.restype = c_int
    L.mrl_rms_norm.argtypes = [c_void_p] * 4 + [c_int64, c_int32, c_float] + [c_int32] * 5 + [c_void_p] * 4
    L.mrl_rms_norm_backward_workspace.restype = c_size_t
    L.mrl_rms_norm_backward_workspace.argtypes = [c_int64, c_int32]
    L.mrl_rms_norm_backward.restype = c_int
    L.mrl_rms_norm_backward.argtypes = [c_void_p] * 5 + [c_int64, c_int32, c_float] + [c_int32] * 5 + [c_void_p] * 3 + [c_size_t, c_void_p]
    L.mrl_grad_norm_workspace.restype = c_size_t
    L.mrl_grad_norm_workspace.argtypes = [POINTER(_ParamTensor), c_int32]
    L.mrl_grad_norm.restype = c_int
    L.mrl_grad_norm.argtypes = [POINTER(_ParamTensor), c_int32, c_double, c_void_p, c_void_p, c_size_t, c_void_p]
    L.mrl_adamw.restype = c_int
    L.mrl_adamw.argtypes = [POINTER(_ParamTensor), c_int32, POINTER(_AdamWConfig), c_void_p, c_void_p]
    L.mrl_adamw_check.restype = c_int
    L.mrl_adamw_check.argtypes = [POINTER(_ParamTensor), c_int32, c_int32]
    L.mrl_top_logprobs_workspace.restype = c_size_t
    L.mrl_top_logprobs_workspace.argtypes = [c_int64, c_int32, c_int32]
    L.mrl_top_logprobs.restype = c_int
    L.mrl_top_logprobs.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_int32, c_int32, c_int32, c_float] + [c_void_p] * 6 + [c_size_t, c_void_p]
    L.mrl_embedding.restype = c_int
    L.mrl_embedding.argtypes = [c_void_p] * 3 + [c_int64, c_int32, c_int32, c_float, c_int32, c_int32, c_void_p, c_void_p]
    L.mrl_embedding_backward_workspace.restype = c_size_t
    L.mrl_embedding_backward_workspace.argtypes = [c_int64, c_int32, c_int32]
    L.mrl_embedding_backward.restype = c_int
    L.mrl_embedding_backward.argtypes = [c_void_p] * 3 + [c_int64, c_int32, c_int32, c_float] + [c_int32] * 3 + [c_void_p] * 2 + [c_size_t, c_void_p]
    L.mrl_distill_loss_workspace.restype = c_size_t
    L.mrl_distill_loss_workspace.argtypes = [c_int64] + [c_int32] * 4 + [POINTER(_DistillConfig)]
    L.mrl_distill_loss_fwd_bwd.restype = c_int
    L.mrl_distill_loss_fwd_bwd.argtypes = [c_void_p] * 6 + [c_int64] + [c_int32] * 4 + [POINTER(_DistillConfig)] + [c_void_p] * 5 + [c_size_t, c_void_p]
    L.mrl_diag_dw_tail_plan.restype = c_int
    L.mrl_diag_dw_tail_plan.argtypes = [c_int32, c_int32, POINTER(c_int32)]
    L.mrl_diag_gemm_cut.restype = c_int
    L.mrl_diag_gemm_cut.argtypes = [c_int32] * 7 + [POINTER(c_int32)]
    L.mrl_diag_dw_few_rows.restype = c_int
    L.mrl_diag_dw_few_rows.argtypes = []
    L.mrl_probe_mfma_rate.restype = c_int
    L.mrl_probe_mfma_rate.argtypes = [c_int32, c_double, c_void_p, c_size_t, POINTER(c_double)]
    _LIB = L
    return L


_HOST = None


class _NoHost:
    """Takes nothing as it is: every call goes through ctypes."""
    advantages = align = rms_norm = rms_norm_backward = grad_norm = adamw = top_logprobs = embedding = embedding_backward = distill = staticmethod(lambda *args: None)


def _load_host():
    """mrl_host.so, or None with a warning where it is not there, does not load, or was built against another torch (whose C++
    interface it uses: a tree built elsewhere still has its C library)."""
    path = os.path.join(_HERE, "mrl_host.so")
    try:
        spec = importlib.util.spec_from_file_location("mrl_host", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        if module.torch_version == str(torch.__version__):
            return module
        why = f"was built against torch {module.torch_version}, this is {torch.__version__}"
    except (ImportError, OSError) as e:        # (a file that is not there is an ImportError or FileNotFoundError)
        why = str(e)
    warnings.warn(f"{path}: {why}; all but the scoring and GRPO calls go through ctypes, which takes 2 - 6 us more a call "
                  "(`python -m paper_2605_07244_amd.build` builds it)", RuntimeWarning, stacklevel=4)
    return None


def _host():
    """The native part of the binding (once).  Its functions return None for what they do not take as it is; the ctypes
    path below, whose checks raise, is for that."""
    global _HOST
    if _HOST is None:
        lib()                                  # (first, so that a missing library is reported as such)
        _HOST = _load_host() or _NoHost
    return _HOST


def status_string(status: int) -> str:
    return lib().mrl_status_string(int(status)).decode()


def version() -> int:
    return lib().mrl_version()


def _ptr(t, dtype=None, name="tensor"):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU torch tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"hidden / lm_head_w must be bfloat16 or float32, got {t.dtype}")


# the current stream's handle without the Stream object torch.cuda.current_stream() builds, which is 2.8 of the
# 15 us of host time of a small call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)
_native = _raw_stream is not None and _get_device is not None


def _stream() -> int:
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _check(rc: int, where: str):
    if rc != 0:
        raise MrlError(rc, where)


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def token_logprobs_workspace(N: int, d: int, V: int, dtype: int) -> int:
    return int(lib().mrl_token_logprobs_workspace(N, d, V, dtype))


def token_logprobs(hidden, lm_head_w, target_ids, token_mask=None, workspace=None, want_lse=True):
    """mrl_token_logprobs: returns (logp[N] f32, lse[N] f32 or None)."""
    N, d = hidden.shape
    V = lm_head_w.shape[0]
    dt = _dtype_code(hidden)
    if lm_head_w.dtype != hidden.dtype or lm_head_w.shape[1] != d:
        raise ValueError("lm_head_w must be [V, d] with the dtype of hidden")
    out_logp = torch.empty(N, dtype=torch.float32, device=hidden.device)
    out_lse = torch.empty(N, dtype=torch.float32, device=hidden.device) if want_lse else None
    if N == 0:            # empty tensors have no device pointer; the library treats N = 0 as a no-op too
        return out_logp, out_lse
    if workspace is None:
        workspace = _workspace(token_logprobs_workspace(N, d, V, dt), hidden.device)
    rc = lib().mrl_token_logprobs(_ptr(hidden, name="hidden"), _ptr(lm_head_w, name="lm_head_w"),
                                  _ptr(target_ids, torch.int32, "target_ids"),
                                  _ptr(token_mask, torch.uint8, "token_mask"), N, d, V, dt,
                                  _ptr(out_logp), _ptr(out_lse), _ptr(workspace), workspace.numel(), _stream())
    _check(rc, "mrl_token_logprobs")
    return out_logp, out_lse


STATIC_SCRATCH_BYTES = 32 << 20


def token_logprobs_static(hidden, lm_head_w, target_ids, token_mask, out_logp, out_lse=None):
    """mrl_token_logprobs_static: the log-prob call on the library's built-in scratch buffer.  The
    caller passes the output tensors; nothing is allocated here or in the library."""
    N, d = hidden.shape
    V = lm_head_w.shape[0]
    rc = lib().mrl_token_logprobs_static(_ptr(hidden, name="hidden"), _ptr(lm_head_w, name="lm_head_w"),
                                         _ptr(target_ids, torch.int32, "target_ids"),
                                         _ptr(token_mask, torch.uint8, "token_mask"), N, d, V, _dtype_code(hidden),
                                         _ptr(out_logp, torch.float32, "out_logp"),
                                         _ptr(out_lse, torch.float32, "out_lse"), _stream())
    _check(rc, "mrl_token_logprobs_static")


def token_scores(hidden, lm_head_w, target_ids, token_mask=None, workspace=None, want_lse=True,
                 want_entropy=True):
    """Forward-only scoring pass: (logp, lse | None, entropy | None), each [N] float32."""
    N, d = hidden.shape
    V = lm_head_w.shape[0]
    dt = _dtype_code(hidden)
    dev = hidden.device
    need = lib().mrl_token_scores_workspace(N, d, V, dt) if want_entropy else \
        lib().mrl_token_logprobs_workspace(N, d, V, dt)
    if workspace is None:
        workspace = _workspace(need, dev)
    out_logp = torch.empty(N, dtype=torch.float32, device=dev)
    out_lse = torch.empty(N, dtype=torch.float32, device=dev) if want_lse else None
    out_ent = torch.empty(N, dtype=torch.float32, device=dev) if want_entropy else None
    _check(lib().mrl_token_scores(_ptr(hidden), _ptr(lm_head_w), _ptr(target_ids, torch.int32, "target_ids"),
                                  _ptr(token_mask, torch.uint8, "token_mask"), N, d, V, dt, _ptr(out_logp),
                                  _ptr(out_lse), _ptr(out_ent), _ptr(workspace), workspace.numel(), _stream()),
           "mrl_token_scores")
    return out_logp, out_lse, out_ent


def group_advantages(rewards, group_id, G, in_stats=None, scored=None, is_own=None, mode=ADV_GROUP_ZN,
                     eps_norm=1e-6, ddof=0, mix_alpha=1.0, neg_thresh=0.2, pos_thresh=0.8, baseline_shift=None):
    """mrl_group_advantages: returns (adv[B], mean[G], std[G], flags[G] uint8)."""
    if _native and type(rewards) is torch.Tensor and rewards.is_cuda:
        r = (_HOST or _host()).advantages(rewards, group_id, G, in_stats, scored, is_own, mode, eps_norm, ddof, mix_alpha, neg_thresh,
                                          pos_thresh, baseline_shift, _raw_stream(_get_device()))
        if r is not None:
            _check(r[0], "mrl_group_advantages")
            return r[1:]
    if baseline_shift is not None and baseline_shift.numel() != G:
        raise ValueError("baseline_shift must have G entries")
    B = rewards.numel()
    dev = rewards.device
    adv = torch.empty(B, dtype=torch.float32, device=dev)
    mean = torch.empty(G, dtype=torch.float32, device=dev)
    std = torch.empty(G, dtype=torch.float32, device=dev)
    flags = torch.empty(G, dtype=torch.uint8, device=dev)
    rc = lib().mrl_group_advantages(_ptr(rewards, torch.float32, "rewards"), _ptr(group_id, torch.int32, "group_id"),
                                    _ptr(in_stats, torch.uint8, "in_stats"), _ptr(scored, torch.uint8, "scored"),
                                    _ptr(is_own, torch.uint8, "is_own"),
                                    _ptr(baseline_shift, torch.float32, "baseline_shift"), B, G, mode, eps_norm, ddof, mix_alpha,
                                    neg_thresh, pos_thresh, _ptr(adv), _ptr(mean), _ptr(std), _ptr(flags), _stream())
    _check(rc, "mrl_group_advantages")
    return adv, mean, std, flags


def grpo_loss_workspace(B: int, T: int, d: int, V: int, dtype: int, cfg: LossConfig) -> int:
    c = cfg.to_c()
    return int(lib().mrl_grpo_loss_workspace(B, T, d, V, dtype, ctypes.byref(c)))


def grpo_loss_fwd_bwd(hidden, lm_head_w, target_ids, token_mask, behav_logp, ref_logp, seq_adv, group_id,
                      seq_kind, B, T, G, cfg: LossConfig, out_dH=None, out_dW=None, want_dH=True, want_dW=True,
                      workspace=None, out_logp=None, out_stats=None):
    """mrl_grpo_loss_fwd_bwd.  Returns dict(logp, dH, dW, stats); `read_stats`
    turns the device stats block into a Python dict (synchronises)."""
    N, d = hidden.shape
    if N != B * T:
        raise ValueError("hidden must be [B*T, d]")
    V = lm_head_w.shape[0]
    dt = _dtype_code(hidden)
    dev = hidden.device
    if out_logp is None:
        out_logp = torch.empty(N, dtype=torch.float32, device=dev)
    if out_dH is None and want_dH:
        out_dH = torch.empty((N, d), dtype=torch.bfloat16 if cfg.dh_dtype == BF16 else torch.float32, device=dev)
    if out_dW is None and want_dW:
        out_dW = torch.empty((V, d), dtype=torch.float32, device=dev)
    if out_stats is None:
        out_stats = torch.empty(STATS_BYTES, dtype=torch.uint8, device=dev)
    if workspace is None:
        workspace = _workspace(grpo_loss_workspace(B, T, d, V, dt, cfg), dev)
    c = cfg.to_c()
    rc = lib().mrl_grpo_loss_fwd_bwd(
        _ptr(hidden, name="hidden"), _ptr(lm_head_w, name="lm_head_w"), _ptr(target_ids, torch.int32, "target_ids"),
        _ptr(token_mask, torch.uint8, "token_mask"), _ptr(behav_logp, torch.float32, "behav_logp"),
        _ptr(ref_logp, torch.float32, "ref_logp"), _ptr(seq_adv, torch.float32, "seq_adv"),
        _ptr(group_id, torch.int32, "group_id"), _ptr(seq_kind, torch.uint8, "seq_kind"),
        B, T, G, d, V, dt, ctypes.byref(c), _ptr(out_logp), _ptr(out_dH), _ptr(out_dW, torch.float32, "out_dW"),
        _ptr(out_stats), _ptr(workspace), workspace.numel(), _stream())
    _check(rc, "mrl_grpo_loss_fwd_bwd")
    return dict(logp=out_logp, dH=out_dH, dW=out_dW, stats=out_stats)


def read_stats(stats: torch.Tensor) -> dict:
    """Copies the device stats block to the host (synchronises) and decodes it."""
    raw = stats.cpu().numpy().tobytes()
    import struct
    vals = struct.unpack("<7d6q", raw)
    return dict(zip(STATS_FIELDS, vals))


def distill_loss_workspace(N: int, d: int, V: int, k: int, dtype: int, cfg: DistillConfig) -> int:
    c = cfg.to_c()
    return int(lib().mrl_distill_loss_workspace(N, d, V, k, dtype, ctypes.byref(c)))


def distill_loss_fwd_bwd(hidden, lm_head_w, teacher_ids, teacher_logp, cfg: DistillConfig, token_mask=None, row_weight=None, out_dH=None, out_dW=None,
                         want_dH=True, want_dW=True, workspace=None, out_kl=None, out_stats=None):
    """mrl_distill_loss_fwd_bwd: dict(kl [N], dH, dW, stats) of hidden [N, d] and a teacher's alternatives, ids [N, k] int32 and log-probs [N, k] float32 (those of
    top_logprobs, at cfg.temperature); `read_distill_stats` turns the device stats block into a Python dict (synchronises)."""
    if (_native and out_dH is None and out_dW is None and workspace is None and out_kl is None and out_stats is None and not cfg.accumulate_dw
            and type(hidden) is torch.Tensor and hidden.is_cuda):
        dev = _get_device()
        r = (_HOST or _host()).distill(hidden, lm_head_w, teacher_ids, teacher_logp, token_mask, row_weight, cfg.temperature, cfg.renormalize, cfg.dh_dtype,
                                       cfg.dw_dtype, cfg.chunk_rows, want_dH, want_dW, dev, _raw_stream(dev))
        if r is not None:
            _check(r[0], "mrl_distill_loss_fwd_bwd")
            return dict(kl=r[1], dH=r[2], dW=r[3], stats=r[4])
    if hidden.dim() != 2 or lm_head_w.dim() != 2 or teacher_ids.dim() != 2:
        raise ValueError("hidden must be [N, d], lm_head_w [V, d] and teacher_ids [N, k]")
    N, d = hidden.shape
    V, k = lm_head_w.shape[0], teacher_ids.shape[1]
    dt = _dtype_code(hidden)
    if lm_head_w.dtype != hidden.dtype or lm_head_w.shape[1] != d:
        raise ValueError("lm_head_w must be [V, d] with the dtype of hidden")
    _shaped(teacher_ids, (N, k), "teacher_ids")
    _shaped(teacher_logp, (N, k), "teacher_logp")
    for t, name in ((token_mask, "token_mask"), (row_weight, "row_weight"), (out_kl, "out_kl")):
        if t is not None and t.numel() != N:
            raise ValueError(f"{name} must have N entries")
    types = {F32: torch.float32, BF16: torch.bfloat16}
    if cfg.dh_dtype not in types or cfg.dw_dtype not in types:
        raise TypeError("dh_dtype and dw_dtype must be F32 or BF16")
    _shaped(out_dH, (N, d), "out_dH")
    _shaped(out_dW, (V, d), "out_dW")
    if cfg.accumulate_dw and want_dW and out_dW is None:
        raise ValueError("accumulate_dw needs out_dW")
    args = [_ptr(hidden, name="hidden"), _ptr(lm_head_w, name="lm_head_w"), _ptr(teacher_ids, torch.int32, "teacher_ids"),
            _ptr(teacher_logp, torch.float32, "teacher_logp"), _ptr(token_mask, torch.uint8, "token_mask"), _ptr(row_weight, torch.float32, "row_weight")]
    _here(hidden, lm_head_w, teacher_ids, teacher_logp, token_mask, row_weight, out_dH, out_dW, workspace, out_kl, out_stats)
    dev = hidden.device
    if out_kl is None:
        out_kl = torch.empty(N, dtype=torch.float32, device=dev)
    if out_dH is None and want_dH:
        out_dH = torch.empty((N, d), dtype=types[cfg.dh_dtype], device=dev)
    if out_dW is None and want_dW:
        out_dW = torch.empty((V, d), dtype=types[cfg.dw_dtype], device=dev)
    if out_stats is None:
        out_stats = torch.empty(DISTILL_STATS_BYTES, dtype=torch.uint8, device=dev)
    elif out_stats.numel() < DISTILL_STATS_BYTES:
        raise ValueError(f"out_stats must have {DISTILL_STATS_BYTES} bytes")
    if workspace is None:
        workspace = _workspace(distill_loss_workspace(N, d, V, k, dt, cfg), dev)
    c = cfg.to_c()
    _check(lib().mrl_distill_loss_fwd_bwd(*args, N, d, V, k, dt, ctypes.byref(c), _ptr(out_kl, torch.float32, "out_kl"), _ptr(out_dH, types[cfg.dh_dtype], "out_dH"),
                                          _ptr(out_dW, types[cfg.dw_dtype], "out_dW"), _ptr(out_stats, torch.uint8, "out_stats"),
                                          _ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()), "mrl_distill_loss_fwd_bwd")
    return dict(kl=out_kl, dH=out_dH, dW=out_dW, stats=out_stats)


def read_distill_stats(stats: torch.Tensor) -> dict:
    """Copies the device stats block to the host (synchronises) and decodes it."""
    import struct
    return dict(zip(DISTILL_STATS_FIELDS, struct.unpack("<d4q", stats.cpu().numpy().tobytes()[:DISTILL_STATS_BYTES])))


def profile_enable(on: bool = True):
    _check(lib().mrl_profile_enable(1 if on else 0), "mrl_profile_enable")


def profile_collect() -> dict:
    """Returns {class: (milliseconds, launches)} since the last collect (synchronises)."""
    ms = (c_double * len(PROF_CLASSES))()
    n = (c_int64 * len(PROF_CLASSES))()
    _check(lib().mrl_profile_collect(ms, n), "mrl_profile_collect")
    return {name: (ms[i], n[i]) for i, name in enumerate(PROF_CLASSES)}


def dw_tail_plan(V: int, d: int) -> dict:
    """Launch plan of the dW GEMM's K-split tail for a [V, d] head (host code only)."""
    out = (c_int32 * 12)()
    _check(lib().mrl_diag_dw_tail_plan(int(V), int(d), out), "mrl_diag_dw_tail_plan")
    return dict(first_tile_row=out[0], tile_rows=out[1], split=out[2], items_before_xcd=list(out[3:12]))


GEMM_FWD, GEMM_DH, GEMM_DW = 2, 5, 6      # MRL_PROF_GEMM_*


def gemm_cut(launch: int, rows: int, V: int, d: int, chunk_rows: int = 0, expected: int = 0, tail_items: int = 0) -> dict:
    """The tiles of a large bf16 launch (mrl_diag_gemm_cut); chunk_rows 0: rows rounded up to 256, expected 0: chunk_rows."""
    chunk = int(chunk_rows) or -(-int(rows) // 256) * 256
    out = (c_int32 * 9)()
    _check(lib().mrl_diag_gemm_cut(int(launch), int(rows), int(expected) or chunk, chunk, int(V), int(d), int(tail_items), out), "mrl_diag_gemm_cut")
    return dict(zip(("wide", "narrow", "half", "tiles", "rest", "split", "blocks", "tail_items", "last_start"), out))


def dw_few_rows() -> int:
    """Rows of a bf16 pass up to which dW takes the launch for few rows, without a tail (host code only)."""
    return int(lib().mrl_diag_dw_few_rows())


def probe_mfma_rate(random_operands: bool, seconds: float = 0.5, device="cuda:0") -> float:
    """TFLOP/s the matrix cores sustain on the GEMM kernels' MFMA instruction, registers only."""
    scratch = torch.empty(512 * 1024, dtype=torch.uint8, device=device)
    out = c_double(0.0)
    torch.cuda.synchronize()
    _check(lib().mrl_probe_mfma_rate(1 if random_operands else 0, float(seconds), _ptr(scratch),
                                     scratch.numel(), ctypes.byref(out)), "mrl_probe_mfma_rate")
    return out.value


def thl_word_align(src_logp, src_mask, src_word_map, src_map_len, tgt_mask, tgt_word_map, tgt_map_len,
                   max_words: int, ignore_value: float = -100.0, want_bad_count: bool = True):
    """Word-level trace alignment (App. D, Alg. 2).  Returns (out [B, S_tgt] float32, bad-entry count tensor)."""
    if _native and type(src_logp) is torch.Tensor and src_logp.is_cuda:
        r = (_HOST or _host()).align(src_logp, src_mask, src_word_map, src_map_len, tgt_mask, tgt_word_map, tgt_map_len, max_words,
                                     ignore_value, want_bad_count, _raw_stream(_get_device()))
        if r is not None:
            _check(r[0], "mrl_thl_word_align")
            return r[1:]
    B, S_src = src_logp.shape
    S_tgt = tgt_mask.shape[1]
    dev = src_logp.device
    out = torch.empty((B, S_tgt), dtype=torch.float32, device=dev)
    bad = torch.empty(1, dtype=torch.int64, device=dev) if want_bad_count else None
    _check(lib().mrl_thl_word_align(
        _ptr(src_logp, torch.float32, "src_logp"), _ptr(src_mask, torch.uint8, "src_mask"),
        _ptr(src_word_map, torch.int32, "src_word_map"), _ptr(src_map_len, torch.int32, "src_map_len"),
        _ptr(tgt_mask, torch.uint8, "tgt_mask"), _ptr(tgt_word_map, torch.int32, "tgt_word_map"),
        _ptr(tgt_map_len, torch.int32, "tgt_map_len"), B, S_src, S_tgt, int(max_words), float(ignore_value),
        _ptr(out), _ptr(bad) if bad is not None else None, _stream()), "mrl_thl_word_align")
    return out, bad


def _here(*tensors):
    """The device that the tensors are on: the current one, on whose stream a call runs."""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.is_cuda and t.get_device() != dev:
            raise ValueError(f"tensors must be on the current device (cuda:{dev}), got one on {t.device}")


def _float_code(t, name):
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    return _dtype_code(t)


def _shaped(t, shape, name):
    if t is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _fits(n, bits, name):
    """ctypes cuts a number to the bits that the C interface has for it; one that needs more is refused here."""
    if not -(1 << bits - 1) <= n < 1 << bits - 1:
        raise ValueError(f"{name} does not fit in {bits} bits: {n}")
    return n


def rms_norm(x, weight, eps=1e-6, residual=None, token_mask=None, out_dtype=None, scale_block=0):
    """mrl_rms_norm: (y [N, d], h [N, d] or None, scale or None) of x [N, d].  h = x + residual is returned with a residual, in
    its type; out_dtype float8_e4m3fn (None: the type of x) makes y codes, to be multiplied by scale [N] or, with
    scale_block = 128, by scale [N, ceil(d / 128)]."""
    if _native and type(x) is torch.Tensor and x.is_cuda:
        dev = _get_device()
        r = (_HOST or _host()).rms_norm(x, weight, eps, residual, token_mask, x.dtype if out_dtype is None else out_dtype, scale_block, dev, _raw_stream(dev))
        if r is not None:
            _check(r[0], "mrl_rms_norm")
            return r[1:]
    out_dtype = x.dtype if out_dtype is None else out_dtype
    codes = {torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3}
    if out_dtype not in codes:
        raise TypeError(f"out_dtype must be float32, bfloat16 or float8_e4m3fn, got {out_dtype}")
    if x.dim() != 2:
        raise ValueError("x must be [N, d]")
    N, d = x.shape
    _fits(d, 32, "the number of columns")
    scale_block = _fits(operator.index(scale_block), 32, "scale_block")
    _shaped(weight, (d,), "weight")
    _shaped(residual, (N, d), "residual")
    if token_mask is not None and token_mask.numel() != N:
        raise ValueError("token_mask must have N entries")
    xt, wt = _float_code(x, "x"), _float_code(weight, "weight")
    rt = _float_code(residual, "residual") if residual is not None else F32
    args = [_ptr(x, name="x"), _ptr(residual, name="residual"), _ptr(weight, name="weight"), _ptr(token_mask, torch.uint8, "token_mask")]
    _here(x, residual, weight, token_mask)
    y = torch.empty((N, d), dtype=out_dtype, device=x.device)
    h = torch.empty((N, d), dtype=residual.dtype, device=x.device) if residual is not None else None
    scale = torch.empty((N, -(-d // scale_block)) if scale_block > 0 else (N,), dtype=torch.float32, device=x.device) if out_dtype == torch.float8_e4m3fn else None
    _check(lib().mrl_rms_norm(*args, N, d, float(eps), xt, rt, wt, codes[out_dtype], scale_block, _ptr(h), _ptr(y), _ptr(scale), _stream()),
           "mrl_rms_norm")
    return y, h, scale


def rms_norm_backward(dy, h, weight, eps=1e-6, d_residual=None, token_mask=None, dx_dtype=None, out_dweight=None, accumulate=False,
                      want_dweight=True, workspace=None):
    """mrl_rms_norm_backward: (dx [N, d] in dx_dtype (None: the type of h), dweight [d] float32 or None).  h is what rms_norm returned as h
    or, without a residual, its x; accumulate adds into out_dweight.  Rows with mask 0 are those whose y was not used: dx is d_residual there, or zero.  (Behind an
    rms_norm that had the mask too, h does not depend on x there: d_residual must be zero in those rows, as this call's dx is without one.)"""
    if dx_dtype is None:
        dx_dtype = h.dtype
    if _native and type(h) is torch.Tensor and h.is_cuda:
        dev = _get_device()
        r = (_HOST or _host()).rms_norm_backward(dy, h, weight, eps, d_residual, token_mask, dx_dtype, out_dweight, accumulate, want_dweight,
                                                 workspace, dev, _raw_stream(dev))
        if r is not None:
            _check(r[0], "mrl_rms_norm_backward")
            return r[1:]
    if dx_dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"dx_dtype must be float32 or bfloat16, got {dx_dtype}")
    if h.dim() != 2:
        raise ValueError("h must be [N, d]")
    N, d = h.shape
    _fits(d, 32, "the number of columns")
    _shaped(dy, (N, d), "dy")
    _shaped(weight, (d,), "weight")
    _shaped(d_residual, (N, d), "d_residual")
    _shaped(out_dweight, (d,), "out_dweight")
    if token_mask is not None and token_mask.numel() != N:
        raise ValueError("token_mask must have N entries")
    if d_residual is not None and d_residual.dtype != h.dtype:
        raise TypeError("d_residual must have the dtype of h")
    if accumulate and out_dweight is None:
        raise ValueError("accumulate needs out_dweight")
    types = [_float_code(dy, "dy"), _float_code(h, "h"), _float_code(weight, "weight"), F32 if dx_dtype == torch.float32 else BF16]
    args = [_ptr(dy, name="dy"), _ptr(h, name="h"), _ptr(weight, name="weight"), _ptr(d_residual, name="d_residual"),
            _ptr(token_mask, torch.uint8, "token_mask")]
    dw_ptr = _ptr(out_dweight, torch.float32, "out_dweight")
    _here(dy, h, weight, d_residual, token_mask, out_dweight, workspace)
    dx = torch.empty((N, d), dtype=dx_dtype, device=h.device)
    if out_dweight is None and want_dweight:
        out_dweight = torch.empty(d, dtype=torch.float32, device=h.device)
        dw_ptr = out_dweight.data_ptr()
    if workspace is None and out_dweight is not None:
        workspace = _workspace(lib().mrl_rms_norm_backward_workspace(N, d), h.device)
    _check(lib().mrl_rms_norm_backward(*args, N, d, float(eps), *types, int(bool(accumulate)), _ptr(dx), dw_ptr, _ptr(workspace, torch.uint8, "workspace"),
                                       workspace.numel() if workspace is not None else 0, _stream()), "mrl_rms_norm_backward")
    return dx, out_dweight


STATE_BLOCK = 256              # elements of a tensor that share the scales of 8-bit moments


def _tensors(given, name, optional=False):
    given = list(given)
    for t in given:
        if not (isinstance(t, torch.Tensor) or (optional and t is None)):
            raise TypeError(f"{name} must hold tensors{' or None' if optional else ''}, got {type(t).__name__}")
    return given


class GradPlan:
    """The gradients of a set of tensors, laid out for grad_norm: built once, good for as long as the tensors keep their memory.  (The plan holds on to that
    memory, so that one whose tensors were given other memory, by `t.data = ...` or a new entry in its lists, still writes to the old.)  Calls with one plan share its workspace: they belong on one stream,
    the one that was current when the plan was made, or must be ordered; a captured call needs the plan for as long as it is replayed."""

    def __init__(self, grads):
        self.grads = _tensors(grads, "grads")
        self._fill(len(self.grads))
        for row, g in zip(self.table, self.grads):
            row.n, row.grad, row.grad_dtype = g.numel(), _ptr(g, name="grad"), _float_code(g, "grad")
        _here(*self.grads)
        self._memory = [g.untyped_storage() for g in self.grads]
        self.device = self.grads[0].device if self.grads else torch.device("cuda", torch.cuda.current_device())
        self.workspace = _workspace(lib().mrl_grad_norm_workspace(self.table, self.count), self.device)

    def _fill(self, count):
        self.count, self.table = count, (_ParamTensor * count)()
        self.address = ctypes.addressof(self.table)


class AdamWPlan(GradPlan):
    """Parameters, gradients and moments of a set of tensors, laid out for adamw_step (and grad_norm); see adamw_plan.  m, v, m_scale and
    v_scale are its lists of moments, updated in place: what a checkpoint saves and a new plan is given."""

    def __init__(self, params, grads, copies, m, v, m_scale, v_scale, state_dtype, weight_decay):
        super().__init__(grads)
        if state_dtype not in (torch.float32, torch.float8_e4m3fn):
            raise TypeError(f"state_dtype must be float32 or float8_e4m3fn, got {state_dtype}")
        codes = state_dtype == torch.float8_e4m3fn
        self.state_dtype, self.params = E4M3 if codes else F32, _tensors(params, "params")
        sizes = [g.numel() for g in self.grads]

        def of(given, dtype, sizes, name, optional=False):
            if given is None:
                return [torch.zeros(n, dtype=dtype, device=self.device) for n in sizes]
            given = _tensors(given, name, optional)
            if len(given) != len(sizes) or any(t is not None and t.numel() != n for t, n in zip(given, sizes)):
                raise ValueError(f"{name} must hold a tensor for each of {len(sizes)}, of their sizes")
            return given

        if [p.numel() for p in self.params] != sizes:
            raise ValueError("params and grads must be as many, and of the same sizes")
        self.copies = None if copies is None else of(copies, torch.bfloat16, sizes, "copies", optional=True)
        self.m, self.v = of(m, state_dtype, sizes, "m"), of(v, state_dtype, sizes, "v")
        if codes and ((m is None) != (m_scale is None) or (v is None) != (v_scale is None)):
            raise ValueError("8-bit moments and their scales are given together")
        blocks = [-(-n // STATE_BLOCK) for n in sizes]
        self.m_scale, self.v_scale = (of(x, torch.float32, blocks, name) if codes else None for x, name in ((m_scale, "m_scale"), (v_scale, "v_scale")))
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * self.count
        if len(decay) != self.count:
            raise ValueError("weight_decay must be a number or one for each tensor")
        for i, row in enumerate(self.table):
            row.param, row.m, row.v = (_ptr(t[i], dt, name) for t, dt, name in
                                       ((self.params, torch.float32, "param"), (self.m, state_dtype, "m"), (self.v, state_dtype, "v")))
            row.copy = _ptr(self.copies[i], torch.bfloat16, "copy") if self.copies is not None else None
            if codes:
                row.m_scale, row.v_scale = (_ptr(t[i], torch.float32, name) for t, name in ((self.m_scale, "m_scale"), (self.v_scale, "v_scale")))
            row.weight_decay = decay[i]
        held = [*self.params, *(self.copies or []), *self.m, *self.v, *(self.m_scale or []), *(self.v_scale or [])]
        _here(*held)
        self._memory += [t.untyped_storage() for t in held if t is not None]
        _check(lib().mrl_adamw_check(self.table, self.count, self.state_dtype), "mrl_adamw_check")


def grad_plan(grads) -> GradPlan:
    """A plan of gradients (float32 or bfloat16) for grad_norm."""
    return GradPlan(grads)


def adamw_plan(params, grads, copies=None, m=None, v=None, m_scale=None, v_scale=None, state_dtype=None, weight_decay=0.01) -> AdamWPlan:
    """A plan for adamw_step: params float32 tensors, grads (float32 or bfloat16) the buffers that their gradients are written to, copies
    the bfloat16 tensors that new weights are copied to, None for tensors without one or for all.  Moments that are not given start at zero, in state_dtype: float32 (the default, or that
    of m) or float8_e4m3fn.  weight_decay: a number, or one for each tensor."""
    if state_dtype is None:
        m = None if m is None else _tensors(m, "m")
        state_dtype = m[0].dtype if m else torch.float32
    return AdamWPlan(params, grads, copies, m, v, m_scale, v_scale, state_dtype, weight_decay)


def grad_norm(plan: GradPlan, max_norm: float = float("inf"), out=None):
    """mrl_grad_norm: a float32 tensor [norm, clip coefficient] of the plan's gradients (not synchronised)."""
    if out is None:
        if _native:
            dev = _get_device()
            r = (_HOST or _host()).grad_norm(plan.address, plan.count, max_norm, plan.workspace, dev, _raw_stream(dev))
            if r is not None:
                _check(r[0], "mrl_grad_norm")
                return r[1]
        out = torch.empty(2, dtype=torch.float32, device=plan.device)
    elif out.numel() != 2:
        raise ValueError("out must have two entries")
    _here(out, plan.workspace)
    _check(lib().mrl_grad_norm(plan.table, plan.count, float(max_norm), _ptr(out, torch.float32, "out"), plan.workspace.data_ptr(),
                               plan.workspace.numel(), _stream()), "mrl_grad_norm")
    return out


def adamw_step(plan: AdamWPlan, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, norm_coef=None, seed=0, skip_nonfinite=False):
    """mrl_adamw: updates the plan's params, moments and copies in place.  step counts from 1.  lr and step are numbers or, for graphs that are
    replayed with other values, tensors of one float32 and one int64 on the GPU.  norm_coef: what grad_norm returned, whose coefficient the gradients
    are multiplied by; skip_nonfinite leaves everything as it is where that is not finite.  seed and step make the roundings of 8-bit moments: plans
    that are stepped side by side need a seed each, and a graph step as a tensor that it counts up, or every replay rounds alike."""
    if _native:
        dev = _get_device()
        r = (_HOST or _host()).adamw(plan.address, plan.count, plan.workspace, lr, step, beta1, beta2, eps, norm_coef, seed, skip_nonfinite,
                                     plan.state_dtype, dev, _raw_stream(dev))
        if r is not None:
            return _check(r[0], "mrl_adamw")
    c = _AdamWConfig(0.0, beta1, beta2, eps, 1, int(seed) & 0xFFFFFFFFFFFFFFFF, plan.state_dtype, int(bool(skip_nonfinite)), None, None)
    for name, x, dtype in (("lr", lr, torch.float32), ("step", step, torch.int64)):
        if isinstance(x, torch.Tensor):
            if x.numel() != 1:
                raise ValueError(f"{name} must have one entry")
            setattr(c, name + "_dev", _ptr(x, dtype, name))
            _here(x)
        else:
            setattr(c, name, float(x) if name == "lr" else _fits(int(x), 64, name))
    if norm_coef is not None and norm_coef.numel() != 2:
        raise ValueError("norm_coef must have two entries")
    coef = None if norm_coef is None else _ptr(norm_coef, torch.float32, "norm_coef") + 4
    _here(norm_coef, plan.workspace)
    _check(lib().mrl_adamw(plan.table, plan.count, ctypes.byref(c), coef, _stream()), "mrl_adamw")


def _mask(t, N):
    if t is not None and t.numel() != N:
        raise ValueError("token_mask must have N entries")
    return _ptr(t, torch.uint8, "token_mask")


def _rows(t, n, name):
    """A tensor of one int32 for each row."""
    if t is not None and t.numel() != n:
        raise ValueError(f"{name} must have {n} entries")
    return _ptr(t, torch.int32, name)


def top_logprobs(logits, k, target_ids=None, token_mask=None, temperature=1.0, want_lse=True, want_entropy=True, workspace=None):
    """mrl_top_logprobs of logits [N, V], float32 or bfloat16, whose rows may lie apart (a slice of wider rows): dict(ids [N, k] int32, top_logp [N, k],
    logp [N] of target_ids, lse [N], entropy [N]), with None for what is not asked for; ids and top_logp are None with k = 0."""
    if _native and workspace is None and type(logits) is torch.Tensor and logits.is_cuda:
        dev = _get_device()
        r = (_HOST or _host()).top_logprobs(logits, k, target_ids, token_mask, temperature, want_lse, want_entropy, dev, _raw_stream(dev))
        if r is not None:
            _check(r[0], "mrl_top_logprobs")
            return dict(ids=r[1], top_logp=r[2], logp=r[3], lse=r[4], entropy=r[5])
    if logits.dim() != 2:
        raise ValueError("logits must be [N, V]")
    N, V = logits.shape
    k = _fits(operator.index(k), 32, "k")
    _fits(V, 32, "the vocabulary")
    dt = _float_code(logits, "logits")
    if not logits.is_cuda:
        raise TypeError("logits must be a GPU torch tensor")
    if N > 0 and V > 0 and (logits.stride(1) != 1 and V > 1 or logits.stride(0) < V and N > 1):
        raise ValueError("logits must have rows of adjacent elements that do not overlap")
    args = [_rows(target_ids, N, "target_ids"), _mask(token_mask, N)]
    _here(logits, target_ids, token_mask, workspace)
    dev, out = logits.device, torch.float32
    r = dict(ids=torch.empty((N, k), dtype=torch.int32, device=dev) if k > 0 else None, top_logp=torch.empty((N, k), dtype=out, device=dev) if k > 0 else None,
             logp=torch.empty(N, dtype=out, device=dev) if target_ids is not None else None, lse=torch.empty(N, dtype=out, device=dev) if want_lse else None,
             entropy=torch.empty(N, dtype=out, device=dev) if want_entropy else None)
    need = lib().mrl_top_logprobs_workspace(N, V, k)
    if workspace is None and need > 256:
        workspace = _workspace(need, dev)
    _check(lib().mrl_top_logprobs(logits.data_ptr(), max(logits.stride(0), V) if N > 1 else V, *args, N, V, k, dt, float(temperature), _ptr(r["ids"]), _ptr(r["top_logp"]),
                                  _ptr(r["logp"]), _ptr(r["lse"]), _ptr(r["entropy"]), _ptr(workspace, torch.uint8, "workspace"),
                                  workspace.numel() if workspace is not None else 0, _stream()), "mrl_top_logprobs")
    return r


def embedding(table, ids, scale=1.0, token_mask=None, out_dtype=None, out=None):
    """mrl_embedding: scale * table[ids], [N, d] in out_dtype (None: the type of table), of ids [N] int32.  Ids outside the table, and tokens with mask 0, give zero rows."""
    if _native and out is None and type(table) is torch.Tensor and table.is_cuda:
        dev = _get_device()
        r = (_HOST or _host()).embedding(table, ids, scale, token_mask, table.dtype if out_dtype is None else out_dtype, dev, _raw_stream(dev))
        if r is not None:
            _check(r[0], "mrl_embedding")
            return r[1]
    if table.dim() != 2 or ids.dim() != 1:
        raise ValueError("table must be [V, d] and ids [N]")
    V, d = table.shape
    N = ids.numel()
    if out is None:
        out_dtype = table.dtype if out_dtype is None else out_dtype
        if out_dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"out_dtype must be float32 or bfloat16, got {out_dtype}")
    elif out_dtype is not None and out.dtype != out_dtype:
        raise TypeError(f"out must have dtype {out_dtype}, got {out.dtype}")
    _fits(V, 32, "the vocabulary")
    _fits(d, 32, "the number of columns")
    _shaped(out, (N, d), "out")
    args = [_ptr(table, name="table"), _rows(ids, N, "ids"), _mask(token_mask, N)]
    tt = _float_code(table, "table")
    _here(table, ids, token_mask, out)
    if out is None:
        out = torch.empty((N, d), dtype=out_dtype, device=table.device)
    _check(lib().mrl_embedding(*args, N, d, V, float(scale), tt, _float_code(out, "out"), _ptr(out, name="out"), _stream()), "mrl_embedding")
    return out


def embedding_backward(dy, ids, V, scale=1.0, token_mask=None, out_dtype=None, out=None, accumulate=False, workspace=None):
    """mrl_embedding_backward: the gradient [V, d] of the table of an embedding whose output's gradient is dy [N, d], in out_dtype (None: float32).  accumulate
    adds into out (float32), the gradient of a head that shares the table, say; without it every row of out is written."""
    if _native and out is None and workspace is None and not accumulate and type(dy) is torch.Tensor and dy.is_cuda:
        dev = _get_device()
        r = (_HOST or _host()).embedding_backward(dy, ids, V, scale, token_mask, torch.float32 if out_dtype is None else out_dtype, dev, _raw_stream(dev))
        if r is not None:
            _check(r[0], "mrl_embedding_backward")
            return r[1]
    if dy.dim() != 2 or ids.dim() != 1:
        raise ValueError("dy must be [N, d] and ids [N]")
    N, d = dy.shape
    V = _fits(operator.index(V), 32, "V")
    _fits(d, 32, "the number of columns")
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    if out is None:
        out_dtype = torch.float32 if out_dtype is None else out_dtype
        if out_dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"out_dtype must be float32 or bfloat16, got {out_dtype}")
    elif out_dtype is not None and out.dtype != out_dtype:
        raise TypeError(f"out must have dtype {out_dtype}, got {out.dtype}")
    _shaped(out, (V, d), "out")
    args = [_ptr(dy, name="dy"), _rows(ids, N, "ids"), _mask(token_mask, N)]
    yt = _float_code(dy, "dy")
    _here(dy, ids, token_mask, out, workspace)
    if out is None:
        out = torch.empty((max(V, 0), d), dtype=out_dtype, device=dy.device)
    if workspace is None:
        workspace = _workspace(lib().mrl_embedding_backward_workspace(N, d, V), dy.device)
    _check(lib().mrl_embedding_backward(*args, N, d, V, float(scale), yt, _float_code(out, "out"), int(bool(accumulate)), _ptr(out, name="out"),
                                        _ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()), "mrl_embedding_backward")
    return out
