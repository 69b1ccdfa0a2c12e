"""Thin ctypes binding of the C-ABI CUDA library (include/rlf.h).

Argument marshalling only: every function takes torch tensors (device memory and
streams are PyTorch's), checks dtypes / devices, and passes raw pointers to the
entry point of the same name.  Nothing is computed here and there is no fallback:
importing this module raises if the library has not been built.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "librlf.so")

RLF_BF16, RLF_F32 = 0, 1
FN_LOGP_LOSS, FN_FUSED_LMHEAD, FN_LOGP_ENTROPY, FN_FUSED_LOGP_ENTROPY, FN_NORM_BWD, FN_CROSS_ENTROPY, FN_FUSED_CROSS_ENTROPY = 3, 4, 5, 6, 7, 8, 9
FN_FUSED_CROSS_ENTROPY_FWD, FN_LINEAR_BWD, FN_BLOCK_NORM_BWD = 10, 11, 12
DEV_BAD_TARGET, DEV_BAD_SEQ, DEV_NONFINITE, DEV_TIMEOUT = 1, 2, 4, 8

EXPORTS = [
    "rlf_build_loss_mask", "rlf_count_live_responses", "rlf_group_advantage", "rlf_rule_reward", "rlf_kl_in_reward", "rlf_grpo_logp_loss_fwd_bwd",
    "rlf_grpo_logp_loss_fwd_bwd_static", "rlf_grpo_logp_loss_fwd_bwd_skip_masked", "rlf_grpo_logp_loss_fwd_bwd_obj", "rlf_logp_entropy_fwd", "rlf_fused_lmhead_grpo", "rlf_fused_lmhead_grpo_obj", "rlf_fused_lmhead_logp_entropy", "rlf_cross_entropy_fwd_bwd", "rlf_fused_lmhead_cross_entropy", "rlf_norm_fwd", "rlf_norm_bwd", "rlf_linear_fwd", "rlf_linear_bwd", "rlf_block_norm_fwd", "rlf_block_norm_bwd", "rlf_workspace_bytes", "rlf_grpo_step_host", "rlf_step_arena_bytes",
    "rlf_tune_logits_kernel", "rlf_tune_logits_grid", "rlf_tune_lmhead", "rlf_tune_lmhead_schedule", "rlf_tune_lmhead_backward", "rlf_tune_lmhead_pacing", "rlf_tune_linear", "rlf_launch_count", "rlf_status_string", "rlf_version",
]

if not os.path.exists(_LIB_PATH):
    raise ImportError(
        "CUDA library %s is missing: build it with `python -m paper_2509_06980_b200.build` "
        "(there is no CPU fallback)" % _LIB_PATH)

_lib = ctypes.CDLL(_LIB_PATH)

_vp, _i32, _i64, _f32, _sz, _int = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                    ctypes.c_size_t, ctypes.c_int)
_lib.rlf_build_loss_mask.argtypes = [_vp, _vp, _i32, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.rlf_count_live_responses.argtypes = [_vp, _vp, _i32, _i64, _vp, _vp, _vp]
_lib.rlf_group_advantage.argtypes = [_vp, _vp, _i32, _i32, _f32, _int, _vp, _vp, _vp]
_lib.rlf_grpo_logp_loss_fwd_bwd.argtypes = [_vp, _int, _i64, _i32, _i64, _vp, _vp, _vp, _i32, _vp, _vp, _vp,
                                            _f32, _f32, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp]
_lib.rlf_grpo_logp_loss_fwd_bwd_static.argtypes = [_vp, _int, _i64, _i32, _i64, _vp, _vp, _vp, _i32, _vp, _vp, _vp,
                                                   _f32, _f32, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.rlf_grpo_logp_loss_fwd_bwd_static.restype = _int
_lib.rlf_fused_lmhead_grpo.argtypes = [_vp, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _f32,
                                       _f32, _vp, _vp, _vp, _vp, _vp, _int, _vp, _sz, _vp, _vp]
_lib.rlf_workspace_bytes.argtypes = [_int, _i64, _i32, _i32, _int]
_lib.rlf_workspace_bytes.restype = _sz
_lib.rlf_grpo_step_host.argtypes = [_vp, _int, _i64, _i32, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _i32, _i32,
                                    _f32, _f32, _f32, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.rlf_step_arena_bytes.argtypes = [_i64, _i32, _i32, _int]
_lib.rlf_step_arena_bytes.restype = _sz
_lib.rlf_tune_logits_kernel.argtypes = [_int, _int, _int]
_lib.rlf_launch_count.restype = _i64
_lib.rlf_status_string.argtypes = [_int]
_lib.rlf_status_string.restype = ctypes.c_char_p
_lib.rlf_version.restype = _int
_lib.rlf_tune_logits_grid.argtypes = [_int, _int]
_lib.rlf_tune_lmhead.argtypes = [_int]
_lib.rlf_tune_lmhead_schedule.argtypes = [_int, _int, _int]
_lib.rlf_tune_lmhead_backward.argtypes = [_int, _int]
_lib.rlf_tune_lmhead_pacing.argtypes = [_int]
_lib.rlf_rule_reward.argtypes = [_vp, _vp, _i32, _i32, _vp, _vp]
_lib.rlf_kl_in_reward.argtypes = [_vp, _vp, _vp, _vp, _vp, _i32, _i64, _f32, _int, _vp, _vp, _vp, _vp]
_lib.rlf_grpo_logp_loss_fwd_bwd_obj.argtypes = [_vp, _int, _i64, _i32, _i64, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _f32,
                                                _f32, _f32, _int, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp]
_lib.rlf_grpo_logp_loss_fwd_bwd_skip_masked.argtypes = [_vp, _int, _i64, _i32, _i64, _vp, _vp, _vp, _i32, _vp, _vp, _vp,
                                                        _f32, _f32, _vp, _vp, _vp, _vp, _int, _vp, _sz, _vp, _vp]
_lib.rlf_logp_entropy_fwd.argtypes = [_vp, _int, _i64, _i32, _i64, _vp, _vp, _vp, _vp, _sz, _vp, _vp]
_lib.rlf_fused_lmhead_grpo_obj.argtypes = [_vp, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _f32, _f32,
                                           _f32, _int, _int, _vp, _vp, _vp, _vp, _vp, _int, _vp, _sz, _vp, _vp]
_lib.rlf_fused_lmhead_logp_entropy.argtypes = [_vp, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp, _vp]
_lib.rlf_cross_entropy_fwd_bwd.argtypes = [_vp, _int, _i64, _i32, _i64, _vp, _vp, _f32, _f32, _vp, _vp, _vp, _vp, _vp, _vp,
                                           _sz, _vp, _vp]
_lib.rlf_fused_lmhead_cross_entropy.argtypes = [_vp, _vp, _i64, _i32, _i32, _vp, _vp, _f32, _f32, _vp, _vp, _vp, _vp, _vp,
                                                _vp, _int, _int, _vp, _sz, _vp, _vp]
_lib.rlf_norm_fwd.argtypes = [_vp, _vp, _int, _i64, _i32, _i64, _vp, _vp, _int, _int, _f32, _vp, _vp, _vp, _vp, _vp]
_lib.rlf_norm_bwd.argtypes = [_vp, _i64, _vp, _i64, _int, _i64, _i32, _vp, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp,
                              _int, _vp, _sz, _vp]
_lib.rlf_linear_fwd.argtypes = [_vp, _i64, _i32, _i64, _vp, _i32, _vp, _int, _int, _int, _vp, _i64, _vp, _int, _vp, _vp, _vp]
_lib.rlf_linear_bwd.argtypes = [_vp, _int, _i64, _vp, _vp, _i64, _i32, _i64, _vp, _i32, _int, _int, _vp, _vp, _int, _vp, _int,
                                _vp, _sz, _vp, _vp]
_lib.rlf_block_norm_fwd.argtypes = [_vp, _i64, _vp, _int, _i64, _i32, _vp, _vp, _int, _vp, _vp, _int, _int, _vp, _int, _f32, _f32, _f32,
                                    _vp, _vp, _vp, _vp]
_lib.rlf_block_norm_bwd.argtypes = [_vp, _vp, _vp, _i64, _vp, _int, _i64, _i32, _vp, _vp, _int, _vp, _int, _int, _vp, _int, _f32, _f32, _vp,
                                    _vp, _vp, _vp, _vp, _vp, _vp, _vp, _int, _vp, _sz, _vp]
_lib.rlf_tune_linear.argtypes = [_int, _int, _int]
# every entry point that returns an rlf_status
for _n in ("rlf_build_loss_mask", "rlf_count_live_responses", "rlf_group_advantage", "rlf_rule_reward", "rlf_kl_in_reward",
           "rlf_grpo_logp_loss_fwd_bwd", "rlf_grpo_logp_loss_fwd_bwd_obj", "rlf_grpo_logp_loss_fwd_bwd_skip_masked",
           "rlf_logp_entropy_fwd", "rlf_fused_lmhead_grpo", "rlf_fused_lmhead_grpo_obj",
           "rlf_fused_lmhead_logp_entropy", "rlf_cross_entropy_fwd_bwd", "rlf_fused_lmhead_cross_entropy", "rlf_norm_fwd", "rlf_norm_bwd", "rlf_linear_fwd", "rlf_linear_bwd", "rlf_block_norm_fwd", "rlf_block_norm_bwd", "rlf_grpo_step_host", "rlf_tune_logits_kernel", "rlf_tune_logits_grid",
           "rlf_tune_lmhead", "rlf_tune_lmhead_schedule", "rlf_tune_lmhead_backward", "rlf_tune_lmhead_pacing", "rlf_tune_linear"):
    getattr(_lib, _n).restype = _int


class RlfError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__("%s: %s (%d)" % (where, _lib.rlf_status_string(code).decode(), code))


def _check(code, where):
    if code != 0:
        raise RlfError(code, where)


def _ptr(t, dtype=None, cuda=True):
    if t is None:
        return None
    if dtype is not None and t.dtype != dtype:
        raise TypeError("expected %s, got %s" % (dtype, t.dtype))
    if cuda and not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not cuda and t.is_cuda:
        raise ValueError("expected a host tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _dt(t, what="logits"):
    if t.dtype == torch.bfloat16:
        return RLF_BF16
    if t.dtype == torch.float32:
        return RLF_F32
    raise TypeError("%s must be bfloat16 or float32" % what)


def version():
    return int(_lib.rlf_version())


def launch_count():
    return int(_lib.rlf_launch_count())


def status_string(code):
    return _lib.rlf_status_string(int(code)).decode()


def workspace_bytes(which_fn, T, V, D=0, dt=RLF_BF16):
    return int(_lib.rlf_workspace_bytes(which_fn, T, V, D, dt))


def new_workspace(which_fn, T, V, D=0, dt=RLF_BF16, device="cuda"):
    n = max(workspace_bytes(which_fn, T, V, D, dt), 256)
    return torch.empty(n, dtype=torch.uint8, device=device)


def tune_logits_kernel(cluster_ctas=0, threads_per_cta=0, one_exp=-1):
    _check(_lib.rlf_tune_logits_kernel(cluster_ctas, threads_per_cta, one_exp), "rlf_tune_logits_kernel")


def tune_logits_grid(rows_per_cluster=0, units_per_cta=0):
    _check(_lib.rlf_tune_logits_grid(int(rows_per_cluster), int(units_per_cta)), "rlf_tune_logits_grid")


def tune_lmhead(pair_ctas=1):
    _check(_lib.rlf_tune_lmhead(int(pair_ctas)), "rlf_tune_lmhead")


def tune_lmhead_backward(row_reference=1, two_accumulators=1):
    _check(_lib.rlf_tune_lmhead_backward(int(row_reference), int(two_accumulators)), "rlf_tune_lmhead_backward")


def tune_lmhead_pacing(on=1):
    _check(_lib.rlf_tune_lmhead_pacing(int(on)), "rlf_tune_lmhead_pacing")


def tune_lmhead_schedule(m_block=0, max_workers=0, chunk_tiles=0):
    _check(_lib.rlf_tune_lmhead_schedule(int(m_block), int(max_workers), int(chunk_tiles)),
           "rlf_tune_lmhead_schedule")


def tune_linear(form=0, tile=0, split=0):
    _check(_lib.rlf_tune_linear(int(form), int(tile), int(split)), "rlf_tune_linear")


def rlf_build_loss_mask(ids, cu_seqlens, open_id, close_id, valid=None, mask_out=None, seq_id_out=None,
                        n_out=None, dev_status=None, want_seq_id=True):
    """-> (mask u8[T], seq_id i32[T] | None, n i64[1]) on the device."""
    T = ids.shape[0]
    B = cu_seqlens.shape[0] - 1
    dev = ids.device
    if mask_out is None:
        mask_out = torch.empty(T, dtype=torch.uint8, device=dev)
    if seq_id_out is None and want_seq_id:
        seq_id_out = torch.empty(T, dtype=torch.int32, device=dev)
    if n_out is None:
        n_out = torch.empty(1, dtype=torch.int64, device=dev)
    _check(_lib.rlf_build_loss_mask(_ptr(ids, torch.int32), _ptr(cu_seqlens, torch.int32), B, T, open_id,
                                    close_id, _ptr(valid, torch.uint8), _ptr(mask_out, torch.uint8),
                                    _ptr(seq_id_out, torch.int32), _ptr(n_out, torch.int64),
                                    _ptr(dev_status, torch.int32), _stream()), "rlf_build_loss_mask")
    return mask_out, seq_id_out, n_out


def rlf_count_live_responses(mask, cu_seqlens, count_out=None, dev_status=None):
    """-> int64[1] on the device: responses with at least one token of mask 1."""
    T = mask.shape[0]
    B = cu_seqlens.shape[0] - 1
    if count_out is None:
        count_out = torch.zeros(1, dtype=torch.int64, device=mask.device)
    _check(_lib.rlf_count_live_responses(_ptr(mask, torch.uint8), _ptr(cu_seqlens, torch.int32), B, T,
                                         _ptr(count_out, torch.int64), _ptr(dev_status, torch.int32), _stream()),
           "rlf_count_live_responses")
    return count_out


def rlf_group_advantage(rewards, group_size=None, group_id=None, num_groups=None, eps=1e-6,
                        unbiased_std=True, adv_out=None, dev_status=None):
    """-> adv fp32[B] on the device."""
    B = rewards.shape[0]
    if adv_out is None:
        adv_out = torch.zeros(B, dtype=torch.float32, device=rewards.device)
    g = int(num_groups) if group_id is not None else int(group_size)
    _check(_lib.rlf_group_advantage(_ptr(rewards, torch.float32), _ptr(group_id, torch.int32), B, g,
                                    float(eps), 1 if unbiased_std else 0, _ptr(adv_out, torch.float32),
                                    _ptr(dev_status, torch.int32), _stream()), "rlf_group_advantage")
    return adv_out


def rlf_rule_reward(scores, weights, reward_out=None):
    """Eq. 1: weighted sum of rule scores.  scores [B, n], weights [n] -> rewards fp32[B]."""
    B, n = scores.shape
    if reward_out is None:
        reward_out = torch.empty(B, dtype=torch.float32, device=scores.device)
    _check(_lib.rlf_rule_reward(_ptr(scores, torch.float32), _ptr(weights, torch.float32), B, n,
                                _ptr(reward_out, torch.float32), _stream()), "rlf_rule_reward")
    return reward_out


KL_K1, KL_K2, KL_K3 = 0, 1, 2


def rlf_kl_in_reward(rewards, old_logp, ref_logp, mask, cu_seqlens, beta, kl_kind=KL_K1, reward_out=None,
                     kl_seq_out=None, dev_status=None):
    """KL penalty folded into the outcome reward: R'_b = R_b - beta * sum_t mask_t k(old_t - ref_t).
    -> (rewards fp32[B], summed estimate per response fp32[B])."""
    B = cu_seqlens.shape[0] - 1
    T = mask.shape[0]
    dev = rewards.device
    if reward_out is None:
        reward_out = torch.empty(B, dtype=torch.float32, device=dev)
    if kl_seq_out is None:
        kl_seq_out = torch.empty(B, dtype=torch.float32, device=dev)
    _check(_lib.rlf_kl_in_reward(_ptr(rewards, torch.float32), _ptr(old_logp, torch.float32),
                                 _ptr(ref_logp, torch.float32), _ptr(mask, torch.uint8),
                                 _ptr(cu_seqlens, torch.int32), B, T, float(beta), int(kl_kind),
                                 _ptr(reward_out, torch.float32), _ptr(kl_seq_out, torch.float32),
                                 _ptr(dev_status, torch.int32), _stream()), "rlf_kl_in_reward")
    return reward_out, kl_seq_out


def rlf_grpo_logp_loss_fwd_bwd(logits, ids, seq_id, adv, old_logp, ref_logp, mask, eps_clip, beta_kl,
                               denom=None, grad_logits=None, want_grad=True, in_place=False,
                               logp_out=None, loss_out=None, workspace=None, dev_status=None):
    """logits: [T, V] (rows may be strided, last dim contiguous).
    -> (logp fp32[T], loss fp64[4], grad_logits | None), all on the device."""
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [T, V] with a contiguous last dimension")
    T, V = logits.shape
    stride = logits.stride(0) if T > 1 else max(V, logits.stride(0) if T == 1 else V)
    dev = logits.device
    if grad_logits is None and want_grad:
        grad_logits = logits if in_place else torch.empty_strided((T, V), (stride, 1), dtype=logits.dtype, device=dev)
    if grad_logits is not None and T > 1 and grad_logits.stride(0) != stride:
        raise ValueError("grad_logits must have the row stride of logits")
    if logp_out is None:
        logp_out = torch.empty(T, dtype=torch.float32, device=dev)
    if loss_out is None:
        loss_out = torch.empty(4, dtype=torch.float64, device=dev)
    dt = _dt(logits)
    if workspace is None:
        workspace = new_workspace(FN_LOGP_LOSS, T, V, 0, dt, dev)
    B = adv.shape[0]
    _check(_lib.rlf_grpo_logp_loss_fwd_bwd(
        logits.data_ptr() if T > 0 else None, dt, T, V, stride, _ptr(ids, torch.int32),
        _ptr(seq_id, torch.int32), _ptr(adv, torch.float32), B, _ptr(old_logp, torch.float32),
        _ptr(ref_logp, torch.float32), _ptr(mask, torch.uint8), float(eps_clip), float(beta_kl),
        _ptr(denom, torch.int64), _ptr(logp_out, torch.float32), _ptr(loss_out, torch.float64),
        None if grad_logits is None else grad_logits.data_ptr(), workspace.data_ptr(), workspace.numel(),
        _ptr(dev_status, torch.int32), _stream()), "rlf_grpo_logp_loss_fwd_bwd")
    return logp_out, loss_out, grad_logits


def rlf_grpo_logp_loss_fwd_bwd_obj(logits, ids, seq_id, adv, old_logp, ref_logp, mask, eps_clip_low, eps_clip_high,
                                   beta_kl, aggregation=0, denom=None, grad_logits=None, want_grad=True,
                                   in_place=False, logp_out=None, loss_out=None, workspace=None, dev_status=None):
    """Objective variants: asymmetric clip range; aggregation 0 = token mean, 1 = sequence mean."""
    T, V = logits.shape
    stride = logits.stride(0) if T > 1 else V
    dev = logits.device
    if grad_logits is None and want_grad:
        grad_logits = logits if in_place else torch.empty_strided((T, V), (stride, 1), dtype=logits.dtype, device=dev)
    if logp_out is None:
        logp_out = torch.empty(T, dtype=torch.float32, device=dev)
    if loss_out is None:
        loss_out = torch.empty(4, dtype=torch.float64, device=dev)
    dt = _dt(logits)
    if workspace is None:
        workspace = new_workspace(FN_LOGP_LOSS, T, V, 0, dt, dev)
    f = _lib.rlf_grpo_logp_loss_fwd_bwd_obj
    _check(f(logits.data_ptr() if T > 0 else None, dt, T, V, stride, _ptr(ids, torch.int32), _ptr(seq_id, torch.int32),
             _ptr(adv, torch.float32), adv.shape[0], _ptr(old_logp, torch.float32), _ptr(ref_logp, torch.float32),
             _ptr(mask, torch.uint8), float(eps_clip_low), float(eps_clip_high), float(beta_kl), int(aggregation),
             _ptr(denom, torch.int64), _ptr(logp_out, torch.float32), _ptr(loss_out, torch.float64),
             None if grad_logits is None else grad_logits.data_ptr(), workspace.data_ptr(), workspace.numel(),
             _ptr(dev_status, torch.int32), _stream()), "rlf_grpo_logp_loss_fwd_bwd_obj")
    return logp_out, loss_out, grad_logits


def rlf_grpo_logp_loss_fwd_bwd_skip_masked(logits, ids, seq_id, adv, old_logp, ref_logp, mask, eps_clip, beta_kl,
                                           denom=None, grad_logits=None, want_grad=True, in_place=False,
                                           zero_masked_grad=True, logp_out=None, loss_out=None, workspace=None,
                                           dev_status=None):
    """As rlf_grpo_logp_loss_fwd_bwd, but rows without loss weight are neither read nor computed."""
    T, V = logits.shape
    stride = logits.stride(0) if T > 1 else V
    dev = logits.device
    if grad_logits is None and want_grad:
        grad_logits = logits if in_place else torch.empty_strided((T, V), (stride, 1), dtype=logits.dtype, device=dev)
    if logp_out is None:
        logp_out = torch.empty(T, dtype=torch.float32, device=dev)
    if loss_out is None:
        loss_out = torch.empty(4, dtype=torch.float64, device=dev)
    dt = _dt(logits)
    if workspace is None:
        workspace = new_workspace(FN_LOGP_LOSS, T, V, 0, dt, dev)
    f = _lib.rlf_grpo_logp_loss_fwd_bwd_skip_masked
    _check(f(logits.data_ptr() if T > 0 else None, dt, T, V, stride, _ptr(ids, torch.int32), _ptr(seq_id, torch.int32),
             _ptr(adv, torch.float32), adv.shape[0], _ptr(old_logp, torch.float32), _ptr(ref_logp, torch.float32),
             _ptr(mask, torch.uint8), float(eps_clip), float(beta_kl), _ptr(denom, torch.int64),
             _ptr(logp_out, torch.float32), _ptr(loss_out, torch.float64),
             None if grad_logits is None else grad_logits.data_ptr(), 1 if zero_masked_grad else 0,
             workspace.data_ptr(), workspace.numel(), _ptr(dev_status, torch.int32), _stream()),
           "rlf_grpo_logp_loss_fwd_bwd_skip_masked")
    return logp_out, loss_out, grad_logits


def rlf_logp_entropy_fwd(logits, ids, want_entropy=True, logp_out=None, entropy_out=None, workspace=None,
                         dev_status=None):
    """Forward only: -> (logp fp32[T], entropy fp32[T] | None) of the rows of `logits` at targets `ids`."""
    T, V = logits.shape
    stride = logits.stride(0) if T > 1 else V
    dev = logits.device
    if logp_out is None:
        logp_out = torch.empty(T, dtype=torch.float32, device=dev)
    if entropy_out is None and want_entropy:
        entropy_out = torch.empty(T, dtype=torch.float32, device=dev)
    dt = _dt(logits)
    if workspace is None:
        workspace = new_workspace(FN_LOGP_ENTROPY, T, V, 0, dt, dev)
    _check(_lib.rlf_logp_entropy_fwd(logits.data_ptr() if T > 0 else None, dt, T, V, stride, _ptr(ids, torch.int32),
                                     _ptr(logp_out, torch.float32), _ptr(entropy_out, torch.float32),
                                     workspace.data_ptr(), workspace.numel(), _ptr(dev_status, torch.int32),
                                     _stream()), "rlf_logp_entropy_fwd")
    return logp_out, entropy_out


STATIC_MAX_TOKENS = 65536


def rlf_grpo_logp_loss_fwd_bwd_static(logits, ids, seq_id, adv, old_logp, ref_logp, mask, eps_clip, beta_kl,
                                      denom, logp_out, loss_out, grad_logits=None, dev_status=None):
    """The loss entry point for callers that cannot allocate: no workspace argument (the scratch is a
    fixed array inside the library, at most STATIC_MAX_TOKENS tokens) and, unlike the wrapper above,
    this wrapper creates no tensor either: every output buffer is passed in.  Calls on one device
    share the scratch, so do not let two of them overlap on the GPU."""
    T, V = logits.shape
    stride = logits.stride(0) if T > 1 else V
    _check(_lib.rlf_grpo_logp_loss_fwd_bwd_static(
        logits.data_ptr() if T > 0 else None, _dt(logits), T, V, stride, _ptr(ids, torch.int32),
        _ptr(seq_id, torch.int32), _ptr(adv, torch.float32), adv.shape[0], _ptr(old_logp, torch.float32),
        _ptr(ref_logp, torch.float32), _ptr(mask, torch.uint8), float(eps_clip), float(beta_kl),
        _ptr(denom, torch.int64), _ptr(logp_out, torch.float32), _ptr(loss_out, torch.float64),
        None if grad_logits is None else grad_logits.data_ptr(), _ptr(dev_status, torch.int32), _stream()),
        "rlf_grpo_logp_loss_fwd_bwd_static")
    return logp_out, loss_out, grad_logits


def rlf_fused_lmhead_grpo(hidden, W, ids, seq_id, adv, old_logp, ref_logp, mask, eps_clip, beta_kl,
                          denom=None, want_grad_hidden=True, want_grad_W=True, grad_hidden=None, grad_W=None,
                          accumulate_grad_W=False, logp_out=None, loss_out=None, workspace=None,
                          dev_status=None):
    """-> (logp fp32[T], loss fp64[4], grad_hidden bf16[T,D] | None, grad_W fp32[V,D] | None)."""
    T, D = hidden.shape
    V = W.shape[0]
    dev = hidden.device
    if grad_hidden is None and want_grad_hidden:
        grad_hidden = torch.empty((T, D), dtype=torch.bfloat16, device=dev)
    if grad_W is None and want_grad_W:
        grad_W = torch.zeros((V, D), dtype=torch.float32, device=dev)
    if logp_out is None:
        logp_out = torch.empty(T, dtype=torch.float32, device=dev)
    if loss_out is None:
        loss_out = torch.empty(4, dtype=torch.float64, device=dev)
    if workspace is None:
        workspace = new_workspace(FN_FUSED_LMHEAD, T, V, D, RLF_BF16, dev)
    _check(_lib.rlf_fused_lmhead_grpo(
        _ptr(hidden, torch.bfloat16), _ptr(W, torch.bfloat16), T, D, V, _ptr(ids, torch.int32),
        _ptr(seq_id, torch.int32), _ptr(adv, torch.float32), adv.shape[0], _ptr(old_logp, torch.float32),
        _ptr(ref_logp, torch.float32), _ptr(mask, torch.uint8), float(eps_clip), float(beta_kl),
        _ptr(denom, torch.int64), _ptr(logp_out, torch.float32), _ptr(loss_out, torch.float64),
        _ptr(grad_hidden, torch.bfloat16), _ptr(grad_W, torch.float32), 1 if accumulate_grad_W else 0,
        workspace.data_ptr(), workspace.numel(), _ptr(dev_status, torch.int32), _stream()),
        "rlf_fused_lmhead_grpo")
    return logp_out, loss_out, grad_hidden, grad_W


def rlf_fused_lmhead_grpo_obj(hidden, W, ids, seq_id, adv, old_logp, ref_logp, mask, eps_clip_low, eps_clip_high,
                              beta_kl, aggregation=0, skip_masked=False, denom=None, want_grad_hidden=True,
                              want_grad_W=True, grad_hidden=None, grad_W=None, accumulate_grad_W=False,
                              logp_out=None, loss_out=None, workspace=None, dev_status=None):
    """The fused LM-head call with an asymmetric clip range, token- or sequence-mean aggregation and
    the option of not multiplying masked rows at all (their log-prob is NaN).
    -> (logp fp32[T], loss fp64[4], grad_hidden bf16[T,D] | None, grad_W fp32[V,D] | None)."""
    T, D = hidden.shape
    V = W.shape[0]
    dev = hidden.device
    if grad_hidden is None and want_grad_hidden:
        grad_hidden = torch.empty((T, D), dtype=torch.bfloat16, device=dev)
    if grad_W is None and want_grad_W:
        grad_W = torch.zeros((V, D), dtype=torch.float32, device=dev)
    if logp_out is None:
        logp_out = torch.empty(T, dtype=torch.float32, device=dev)
    if loss_out is None:
        loss_out = torch.empty(4, dtype=torch.float64, device=dev)
    if workspace is None:
        workspace = new_workspace(FN_FUSED_LMHEAD, T, V, D, RLF_BF16, dev)
    _check(_lib.rlf_fused_lmhead_grpo_obj(
        _ptr(hidden, torch.bfloat16), _ptr(W, torch.bfloat16), T, D, V, _ptr(ids, torch.int32),
        _ptr(seq_id, torch.int32), _ptr(adv, torch.float32), adv.shape[0], _ptr(old_logp, torch.float32),
        _ptr(ref_logp, torch.float32), _ptr(mask, torch.uint8), float(eps_clip_low), float(eps_clip_high),
        float(beta_kl), int(aggregation), 1 if skip_masked else 0, _ptr(denom, torch.int64),
        _ptr(logp_out, torch.float32), _ptr(loss_out, torch.float64), _ptr(grad_hidden, torch.bfloat16),
        _ptr(grad_W, torch.float32), 1 if accumulate_grad_W else 0, workspace.data_ptr(), workspace.numel(),
        _ptr(dev_status, torch.int32), _stream()), "rlf_fused_lmhead_grpo_obj")
    return logp_out, loss_out, grad_hidden, grad_W


def rlf_fused_lmhead_logp_entropy(hidden, W, ids, want_entropy=True, logp_out=None, entropy_out=None,
                                  workspace=None, dev_status=None):
    """Forward only, from hidden states: -> (logp fp32[T], entropy fp32[T] | None); logits are never stored."""
    T, D = hidden.shape
    V = W.shape[0]
    dev = hidden.device
    if logp_out is None:
        logp_out = torch.empty(T, dtype=torch.float32, device=dev)
    if entropy_out is None and want_entropy:
        entropy_out = torch.empty(T, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = new_workspace(FN_FUSED_LOGP_ENTROPY, T, V, D, RLF_BF16, dev)
    _check(_lib.rlf_fused_lmhead_logp_entropy(
        _ptr(hidden, torch.bfloat16) if T > 0 else None, _ptr(W, torch.bfloat16), T, D, V, _ptr(ids, torch.int32),
        _ptr(logp_out, torch.float32), _ptr(entropy_out, torch.float32), workspace.data_ptr(), workspace.numel(),
        _ptr(dev_status, torch.int32), _stream()), "rlf_fused_lmhead_logp_entropy")
    return logp_out, entropy_out


NORM_RMS, NORM_LAYER, NORM_NONE = 0, 1, 2      # (NORM_NONE: the block norm's only)

# The calls below are short next to a decoding step or a small batch, so their host side is kept lean: outputs are made by
# the cheapest factory call and not checked again, workspace sizes are computed once per shape.
# (torch's own short cuts where this build of it has them; without CUDA it has neither, and the module is still to be imported)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_f32, _f64, _bf16, _i32t, _i64t, _u8 = (torch.float32, torch.float64, torch.bfloat16, torch.int32, torch.int64, torch.uint8)
_DTYPES = {torch.bfloat16: RLF_BF16, torch.float32: RLF_F32}


def _device_of(t):
    """Index of the current device.  The kernels run there, so a tensor of another device is refused."""
    here = t.get_device()
    if here < 0:
        raise ValueError("expected a CUDA tensor")
    if here != _get_device():
        raise ValueError("a tensor is on cuda:%d, the current device is cuda:%d" % (here, _get_device()))
    return here


def _at(t, here, what, dtype=None, shape=None):
    """Address of a dense tensor on the current device (None passes)."""
    if t is None:
        return None
    if t.get_device() != here:
        raise ValueError("%s must be on the current device, cuda:%d" % (what, here))
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (what, dtype, t.dtype))
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (what, tuple(shape), tuple(t.shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % what)
    return t.data_ptr()


def _rows(t, here, what):
    """Base address and row stride of a [T, D] tensor whose rows may be strided (last dimension dense)."""
    if t.get_device() != here:
        raise ValueError("%s must be on the current device, cuda:%d" % (what, here))
    if t.dim() != 2:
        raise ValueError("%s must be 2-dimensional" % what)
    T, D = t.shape
    rs, cs = t.stride()
    if cs != 1 and D > 1:
        raise ValueError("%s must have a contiguous last dimension" % what)
    return (t.data_ptr() if T > 0 else None), (rs if T > 1 else D)


def _dense_like(t):
    """An empty dense tensor of t's shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _empty_rows_like(t, stride):
    """An empty [T, V] tensor whose rows sit in their 16-byte vectors as t's rows do (what the fast kernels need)."""
    off = t.data_ptr() % 16 // t.element_size()
    if off == 0 and t.is_contiguous():
        return torch.empty_like(t)
    T, V = t.shape
    return t.new_empty((max(T, 1) - 1) * stride + V + off).as_strided((T, V), (stride, 1), off)


_bytes_of = {}


def _workspace(workspace, here, like, *key):
    """(tensor, address, bytes): the caller's workspace, or a new one of rlf_workspace_bytes(*key)."""
    if workspace is None:
        n = _bytes_of.get(key)
        if n is None:
            if len(_bytes_of) > 4096:
                _bytes_of.clear()
            n = _bytes_of[key] = max(int(_lib.rlf_workspace_bytes(*key)), 256)
        workspace = like.new_empty(n, dtype=_u8)
        return workspace, workspace.data_ptr(), n
    return workspace, _at(workspace, here, "workspace"), workspace.numel() * workspace.element_size()


def rlf_cross_entropy_fwd_bwd(logits, ids, mask=None, label_smoothing=0.0, z_coef=0.0, denom=None, grad_logits=None,
                              want_grad=True, in_place=False, logp_out=None, lse_out=None, want_lse=True, loss_out=None,
                              workspace=None, dev_status=None):
    """Softmax cross entropy of the rows of logits [T, V] (rows may be strided) at targets ids, masked mean.
    A grad_logits of the caller's is fast where its address differs from the logits' by a multiple of 16 bytes.
    -> (logp fp32[T], lse fp32[T] | None, loss fp64[4], grad_logits | None), all on the device."""
    here = _device_of(logits)
    zp, stride = _rows(logits, here, "logits")
    T, V = logits.shape
    n = (T,)
    gp = None
    if grad_logits is None:
        if want_grad:
            grad_logits = logits if in_place else _empty_rows_like(logits, stride)
            gp = grad_logits.data_ptr() if T > 0 else None
    else:
        if grad_logits.shape != logits.shape or grad_logits.dtype != logits.dtype:
            raise ValueError("grad_logits must have the shape and type of logits")
        gp, gs = _rows(grad_logits, here, "grad_logits")
        if T > 1 and gs != stride:
            raise ValueError("grad_logits must have the row stride of logits")
    if logp_out is None:
        logp_out = logits.new_empty(T, dtype=_f32)
    if lse_out is None and want_lse:
        lse_out = logits.new_empty(T, dtype=_f32)
    if loss_out is None:
        loss_out = logits.new_empty(4, dtype=_f64)
    workspace, wp, wn = _workspace(workspace, here, logits, FN_CROSS_ENTROPY, T, V, 0, _dt(logits))
    _check(_lib.rlf_cross_entropy_fwd_bwd(
        zp, _dt(logits), T, V, stride, _at(ids, here, "ids", _i32t, n), _at(mask, here, "mask", _u8, n), label_smoothing,
        z_coef, _at(denom, here, "denom", _i64t), _at(logp_out, here, "logp_out", _f32, n),
        _at(lse_out, here, "lse_out", _f32, n), _at(loss_out, here, "loss_out", _f64, (4,)), gp, wp, wn,
        _at(dev_status, here, "dev_status", _i32t), _raw_stream(here)), "rlf_cross_entropy_fwd_bwd")
    return logp_out, lse_out, loss_out, grad_logits


def rlf_fused_lmhead_cross_entropy(hidden, W, ids, mask=None, label_smoothing=0.0, z_coef=0.0, denom=None,
                                   want_grad_hidden=True, want_grad_W=True, grad_hidden=None, grad_W=None,
                                   grad_W_dtype=torch.float32, accumulate_grad_W=False, logp_out=None, lse_out=None,
                                   want_lse=True, loss_out=None, workspace=None, dev_status=None):
    """rlf_cross_entropy_fwd_bwd of the logits hidden W^T, which are never stored.
    -> (logp fp32[T], lse fp32[T] | None, loss fp64[4], grad_hidden bf16[T,D] | None, grad_W [V,D] | None);
    grad_W is fp32 or (grad_W_dtype=torch.bfloat16) bf16."""
    here = _device_of(hidden)
    T, D = hidden.shape
    V = W.shape[0]
    n = (T,)
    if accumulate_grad_W and grad_W is None:
        raise ValueError("accumulate_grad_W needs the buffer that is added to")
    if grad_hidden is None and want_grad_hidden:
        grad_hidden = hidden.new_empty((T, D), dtype=_bf16)
    if grad_W is None and want_grad_W:
        grad_W = hidden.new_empty((V, D), dtype=grad_W_dtype)
    if logp_out is None:
        logp_out = hidden.new_empty(T, dtype=_f32)
    if lse_out is None and want_lse:
        lse_out = hidden.new_empty(T, dtype=_f32)
    if loss_out is None:
        loss_out = hidden.new_empty(4, dtype=_f64)
    w_dt = RLF_F32 if grad_W is None else _dt(grad_W, "grad_W")
    fn = FN_FUSED_CROSS_ENTROPY_FWD if grad_hidden is None and grad_W is None else FN_FUSED_CROSS_ENTROPY
    workspace, wp, wn = _workspace(workspace, here, hidden, fn, T, V, D, w_dt)
    _check(_lib.rlf_fused_lmhead_cross_entropy(
        _at(hidden, here, "hidden", _bf16), _at(W, here, "W", _bf16, (V, D)), T, D, V, _at(ids, here, "ids", _i32t, n),
        _at(mask, here, "mask", _u8, n), label_smoothing, z_coef, _at(denom, here, "denom", _i64t),
        _at(logp_out, here, "logp_out", _f32, n), _at(lse_out, here, "lse_out", _f32, n),
        _at(loss_out, here, "loss_out", _f64, (4,)), _at(grad_hidden, here, "grad_hidden", _bf16, (T, D)),
        _at(grad_W, here, "grad_W", None, (V, D)), w_dt, 1 if accumulate_grad_W else 0, wp, wn,
        _at(dev_status, here, "dev_status", _i32t), _raw_stream(here)), "rlf_fused_lmhead_cross_entropy")
    return logp_out, lse_out, loss_out, grad_hidden, grad_W


def rlf_norm_fwd(x, weight, bias=None, residual=None, kind=NORM_RMS, eps=1e-6, y_out=None, sum_out=None,
                 mean_out=None, rstd_out=None):
    """Layer norm (NORM_LAYER) or its RMS form (NORM_RMS) of the rows of x (+ residual).
    x, residual: [T, D] (rows may be strided, the same stride); weight, bias: [D], bf16 or fp32.
    -> (y [T, D], x + residual [T, D] | None without residual, mean fp32[T] | None for the RMS form, rstd fp32[T])."""
    here = _device_of(x)
    xp, xs = _rows(x, here, "x")
    shape = T, D = x.shape
    dt, w_dt = x.dtype, weight.dtype
    if dt not in _DTYPES or w_dt not in _DTYPES:
        raise TypeError("x and weight must be bfloat16 or float32")
    rp = None
    if residual is not None:
        if residual.shape != shape or residual.dtype != dt:
            raise ValueError("residual must have the shape and type of x")
        rp, rs = _rows(residual, here, "residual")
        if T > 1 and rs != xs:
            raise ValueError("residual must have the row stride of x")
        if sum_out is None:
            sum_out = _dense_like(x)
            sp = sum_out.data_ptr()
        else:
            sp = _at(sum_out, here, "sum_out", dt, shape)
    else:
        sp = _at(sum_out, here, "sum_out", dt, shape)
    if y_out is None:
        y_out = _dense_like(x)
        yp = y_out.data_ptr()
    else:
        yp = _at(y_out, here, "y_out", dt, shape)
    if mean_out is None and kind == NORM_LAYER:
        mean_out = x.new_empty(T, dtype=_f32)
    if rstd_out is None:
        rstd_out = x.new_empty(T, dtype=_f32)
        qp = rstd_out.data_ptr()
    else:
        qp = _at(rstd_out, here, "rstd_out", _f32, (T,))
    _check(_lib.rlf_norm_fwd(
        xp, rp, _DTYPES[dt], T, D, xs, _at(weight, here, "weight", w_dt, (D,)), _at(bias, here, "bias", w_dt, (D,)),
        _DTYPES[w_dt], kind, eps, sp, yp, _at(mean_out, here, "mean_out", _f32, (T,)), qp, _raw_stream(here)), "rlf_norm_fwd")
    return y_out, sum_out, mean_out, rstd_out


def rlf_norm_bwd(grad_y, x, weight, mean, rstd, kind=NORM_RMS, grad_skip=None, want_grad_x=True, want_grad_weight=True,
                 want_grad_bias=False, grad_x=None, grad_weight=None, grad_bias=None, accumulate=False, workspace=None):
    """Backward of rlf_norm_fwd; x is what was normalised (the sum, with a residual); grad_skip is added to grad_x.
    -> (grad_x [T, D] | None, grad_weight fp32[D] | None, grad_bias fp32[D] | None)."""
    here = _device_of(x)
    xp, xs = _rows(x, here, "x")
    shape = T, D = x.shape
    dt, w_dt = x.dtype, weight.dtype
    if dt not in _DTYPES or w_dt not in _DTYPES:
        raise TypeError("x and weight must be bfloat16 or float32")
    if grad_y.shape != shape or grad_y.dtype != dt:
        raise ValueError("grad_y must have the shape and type of x")
    gp, gs = _rows(grad_y, here, "grad_y")
    if accumulate and ((grad_weight is None and want_grad_weight) or (grad_bias is None and want_grad_bias)):
        raise ValueError("accumulate needs the buffers that are added to")
    if grad_x is None:
        xo = None
        if want_grad_x:
            grad_x = _dense_like(x)
            xo = grad_x.data_ptr()
    else:
        xo = _at(grad_x, here, "grad_x", dt, shape)
    if grad_weight is None and want_grad_weight:
        grad_weight = x.new_empty(D, dtype=_f32)
    if grad_bias is None and want_grad_bias:
        grad_bias = x.new_empty(D, dtype=_f32)
    wp, wn = None, 0
    if workspace is not None or grad_weight is not None or grad_bias is not None:
        workspace, wp, wn = _workspace(workspace, here, x, FN_NORM_BWD, T, 0, D, RLF_F32)
    _check(_lib.rlf_norm_bwd(
        gp, gs, xp, xs, _DTYPES[dt], T, D, _at(weight, here, "weight", w_dt, (D,)), _DTYPES[w_dt], kind,
        _at(mean, here, "mean", _f32, (T,)), _at(rstd, here, "rstd", _f32, (T,)),
        _at(grad_skip, here, "grad_skip", dt, shape), xo, _at(grad_weight, here, "grad_weight", _f32, (D,)),
        _at(grad_bias, here, "grad_bias", _f32, (D,)), 1 if accumulate else 0, wp, wn, _raw_stream(here)), "rlf_norm_bwd")
    return grad_x, grad_weight, grad_bias


ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU, ACT_GELU_TANH = 0, 1, 2, 3, 4


def rlf_linear_fwd(x, W, bias=None, act=ACT_NONE, gated=False, residual=None, out_dtype=None, want_pre=False, y_out=None,
                   pre_out=None, dev_status=None):
    """Linear layer with its epilogue: act(x W^T + bias) + residual, or gated, with W's rows the N gate rows and then the
    N up rows: act(z_gate) z_up + residual.  x [T, D] bf16 (rows may be strided), W [N | 2 N, D] bf16, bias bf16 or fp32.
    The output's type is out_dtype, or the residual's, or bf16.
    -> (y [T, N], z bf16 [T, N | 2 N] | None: what rlf_linear_bwd takes as pre, with want_pre)."""
    here = _device_of(x)
    xp, xs = _rows(x, here, "x")
    T, D = x.shape
    if x.dtype != _bf16:
        raise TypeError("x must be bfloat16")
    if W.dim() != 2 or W.shape[1] != D or (gated and W.shape[0] % 2):
        raise ValueError("W must be [N, %d], gated [2 N, %d]" % (D, D))
    rows = W.shape[0]
    N = rows // 2 if gated else rows
    shape = (T, N)
    if y_out is None:
        y_out = x.new_empty(shape, dtype=out_dtype or (_bf16 if residual is None else residual.dtype))
        yp = y_out.data_ptr()
    else:
        yp = _at(y_out, here, "y_out", out_dtype, shape)
    dt = _dt(y_out, "the output")
    rp, rs = None, 0
    if residual is not None:
        if residual.shape != shape or residual.dtype != y_out.dtype:
            raise ValueError("residual must have the shape and type of the output")
        rp, rs = _rows(residual, here, "residual")
    zp = None
    if pre_out is not None:
        zp = _at(pre_out, here, "pre_out", _bf16, (T, rows))
    elif want_pre:
        pre_out = x.new_empty((T, rows))
        zp = pre_out.data_ptr()
    _check(_lib.rlf_linear_fwd(
        xp, T, D, xs, _at(W, here, "W", _bf16), N, _at(bias, here, "bias", None, (rows,)), 0 if bias is None else _dt(bias, "bias"),
        act, 1 if gated else 0, rp, rs, yp, dt, zp, _at(dev_status, here, "dev_status", _i32t), _raw_stream(here)), "rlf_linear_fwd")
    return y_out, pre_out


def rlf_linear_bwd(grad_y, x, W, pre=None, act=ACT_NONE, gated=False, want_grad_x=True, want_grad_W=True, want_grad_bias=False,
                   grad_x=None, grad_W=None, grad_W_dtype=torch.float32, grad_bias=None, accumulate=False, workspace=None,
                   dev_status=None):
    """Backward of rlf_linear_fwd; pre is the z it left (needed with an activation or a gate); the residual's gradient is
    grad_y.  accumulate adds to the buffers given as grad_W (fp32) and grad_bias.
    -> (grad_x bf16 [T, D] | None, grad_W [N | 2 N, D] | None, grad_bias fp32 [N | 2 N] | None)."""
    here = _device_of(x)
    xp, xs = _rows(x, here, "x")
    T, D = x.shape
    if x.dtype != _bf16:
        raise TypeError("x must be bfloat16")
    if W.dim() != 2 or W.shape[1] != D or (gated and W.shape[0] % 2):
        raise ValueError("W must be [N, %d], gated [2 N, %d]" % (D, D))
    rows = W.shape[0]
    N = rows // 2 if gated else rows
    if grad_y.shape != (T, N):
        raise ValueError("grad_y must have shape %s, got %s" % ((T, N), tuple(grad_y.shape)))
    gp, gs = _rows(grad_y, here, "grad_y")
    if pre is None and (gated or act != ACT_NONE):
        raise ValueError("an activation or a gate needs pre, the z of the forward call")
    if accumulate and ((grad_W is None and want_grad_W) or (grad_bias is None and want_grad_bias)):
        raise ValueError("accumulate needs the buffers that are added to")
    xo = wo = bo = None
    w_dt = RLF_F32
    if grad_x is not None:
        xo = _at(grad_x, here, "grad_x", _bf16, (T, D))
    elif want_grad_x:
        grad_x = x.new_empty((T, D))
        xo = grad_x.data_ptr()
    if grad_W is not None:
        wo, w_dt = _at(grad_W, here, "grad_W", None, (rows, D)), _dt(grad_W, "grad_W")
    elif want_grad_W:
        grad_W = x.new_empty((rows, D), dtype=grad_W_dtype)
        wo, w_dt = grad_W.data_ptr(), _dt(grad_W, "grad_W")
    if grad_bias is not None:
        bo = _at(grad_bias, here, "grad_bias", _f32, (rows,))
    elif want_grad_bias:
        grad_bias = x.new_empty(rows, dtype=_f32)
        bo = grad_bias.data_ptr()
    workspace, wp, wn = _workspace(workspace, here, x, FN_LINEAR_BWD, T, rows, D, RLF_BF16)
    _check(_lib.rlf_linear_bwd(
        gp, _dt(grad_y, "grad_y"), gs, _at(pre, here, "pre", _bf16, (T, rows)), xp, T, D, xs, _at(W, here, "W", _bf16), N, act,
        1 if gated else 0, xo, wo, w_dt, bo, 1 if accumulate else 0, wp, wn, _at(dev_status, here, "dev_status", _i32t),
        _raw_stream(here)), "rlf_linear_bwd")
    return grad_x, grad_W, grad_bias


GATE_NONE, GATE_COLUMN, GATE_ROW = 0, 1, 2


def _norm_vectors(T, D, here, post_kind, pre_kind, gate_form, gate, post_weight, post_bias, pre_weight, pre_bias):
    """Checks of the block norm's [D] vectors (one type among them) and its gate.
    -> (their type's code, the addresses of post_weight, post_bias, pre_weight, pre_bias and the gate)"""
    if (gate is None) != (gate_form == GATE_NONE):
        raise ValueError("gate and gate_form go together")
    if (post_kind == NORM_NONE) != (post_weight is None) or (post_weight is None and post_bias is not None):
        raise ValueError("post_weight (and post_bias) belong to the post norm, which needs post_weight")
    if (pre_kind == NORM_NONE) != (pre_weight is None) or (pre_weight is None and pre_bias is not None):
        raise ValueError("pre_weight (and pre_bias) belong to the pre norm, which needs pre_weight")
    first = post_weight if post_weight is not None else pre_weight
    w_dt = _f32 if first is None else first.dtype
    if w_dt not in _DTYPES:
        raise TypeError("weights, biases and a column gate must be bfloat16 or float32")
    row = (D,)
    if gate is None:
        gp = None
    elif gate_form == GATE_ROW:
        gp = _at(gate, here, "gate", _f32, (T,))
    else:
        gp = _at(gate, here, "gate", w_dt, row)
    return (_DTYPES[w_dt], _at(post_weight, here, "post_weight", w_dt, row), _at(post_bias, here, "post_bias", w_dt, row),
            _at(pre_weight, here, "pre_weight", w_dt, row), _at(pre_bias, here, "pre_bias", w_dt, row), gp)


def rlf_block_norm_fwd(x, residual, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None, post_kind=NORM_RMS,
                       pre_kind=NORM_RMS, gate=None, gate_form=GATE_NONE, alpha=1.0, beta=1.0, eps=1e-6, h_out=None, y_out=None,
                       stats_out=None):
    """The norm after a block, its gate, the residual and the norm before the next block:
    h = alpha residual + beta gate norm_post(x), y = norm_pre(h).  x [T, D] (rows may be strided), residual [T, D]; weights,
    biases and a column gate [D] of one type, bf16 or fp32; a row gate [T] fp32; NORM_NONE leaves a norm out.
    -> (h [T, D], y [T, D] | None without the pre norm, stats fp32 [4, T]: post mean and rstd, pre mean and rstd)."""
    here = _device_of(x)
    xp, xs = _rows(x, here, "x")
    shape = T, D = x.shape
    dt = x.dtype
    if dt not in _DTYPES:
        raise TypeError("x must be bfloat16 or float32")
    if residual is None:
        raise ValueError("residual is needed")
    w_dt, w1, b1, w2, b2, gp = _norm_vectors(T, D, here, post_kind, pre_kind, gate_form, gate, post_weight, post_bias, pre_weight, pre_bias)
    if h_out is None:
        h_out = _dense_like(x)
        hp = h_out.data_ptr()
    else:
        hp = _at(h_out, here, "h_out", dt, shape)
    yp = None
    if y_out is not None:
        yp = _at(y_out, here, "y_out", dt, shape)
    elif pre_kind != NORM_NONE:
        y_out = _dense_like(x)
        yp = y_out.data_ptr()
    if stats_out is None:
        stats_out = x.new_empty((4, T), dtype=_f32)
        sp = stats_out.data_ptr()
    else:
        sp = _at(stats_out, here, "stats_out", _f32, (4, T))
    _check(_lib.rlf_block_norm_fwd(
        xp, xs, _at(residual, here, "residual", dt, shape), _DTYPES[dt], T, D, w1, b1, post_kind, w2, b2, pre_kind, w_dt, gp, gate_form,
        alpha, beta, eps, hp, yp, sp, _raw_stream(here)), "rlf_block_norm_fwd")
    return h_out, y_out, stats_out


def rlf_block_norm_bwd(grad_y, grad_h, x, h, stats, post_weight=None, post_bias=None, pre_weight=None, post_kind=NORM_RMS,
                       pre_kind=NORM_RMS, gate=None, gate_form=GATE_NONE, alpha=1.0, beta=1.0, want_grad_x=True,
                       want_grad_residual=True, want_grad_weight=True, want_grad_bias=False, want_grad_gate=True, grad_x=None,
                       grad_residual=None, grad_gate=None, grad_post_weight=None, grad_post_bias=None, grad_pre_weight=None,
                       grad_pre_bias=None, accumulate=False, workspace=None):
    """Backward of rlf_block_norm_fwd; h and stats are what it left (h is not read without the pre norm, grad_y neither);
    grad_h is the gradient that reaches h by another path, or None.  accumulate adds to the [D] gradients' buffers.
    -> dict(grad_x, grad_residual [T, D], grad_gate, grad_post_weight, grad_post_bias, grad_pre_weight, grad_pre_bias fp32), None
    where not wanted or not there."""
    here = _device_of(x)
    xp, xs = _rows(x, here, "x")
    shape = T, D = x.shape
    dt = x.dtype
    if dt not in _DTYPES:
        raise TypeError("x must be bfloat16 or float32")
    w_dt, w1, b1, w2, _, gp = _norm_vectors(T, D, here, post_kind, pre_kind, gate_form, gate, post_weight, post_bias, pre_weight, None)
    pre, post = pre_kind != NORM_NONE, post_kind != NORM_NONE
    if pre and (grad_y is None or h is None):
        raise ValueError("the pre norm needs grad_y and h")
    if not pre and grad_h is None:
        raise ValueError("without the pre norm grad_h is needed")

    def rows(t, want, what):                     # a [T, D] output: (the tensor, its address)
        if t is not None:
            return t, _at(t, here, what, dt, shape)
        if not want:
            return None, None
        t = _dense_like(x)
        return t, t.data_ptr()

    def vector(t, want, what, n, summed=True):   # a gradient over tokens (or, not summed, one per token)
        if t is not None:
            return t, _at(t, here, what, _f32, (n,))
        if not want:
            return None, None
        if accumulate and summed:
            raise ValueError("accumulate needs the buffers that are added to")
        t = x.new_empty(n, dtype=_f32)
        return t, t.data_ptr()

    per_row = gate_form == GATE_ROW
    grad_x, gxp = rows(grad_x, want_grad_x, "grad_x")
    grad_residual, grp = rows(grad_residual, want_grad_residual, "grad_residual")
    grad_gate, ggp = vector(grad_gate, want_grad_gate and gate is not None, "grad_gate", T if per_row else D, not per_row)
    grad_post_weight, gw1 = vector(grad_post_weight, want_grad_weight and post, "grad_post_weight", D)
    grad_post_bias, gb1 = vector(grad_post_bias, want_grad_bias and post, "grad_post_bias", D)
    grad_pre_weight, gw2 = vector(grad_pre_weight, want_grad_weight and pre, "grad_pre_weight", D)
    grad_pre_bias, gb2 = vector(grad_pre_bias, want_grad_bias and pre, "grad_pre_bias", D)
    wp, wn = None, 0
    if workspace is not None or gw1 or gb1 or gw2 or gb2 or (ggp and not per_row):
        workspace, wp, wn = _workspace(workspace, here, x, FN_BLOCK_NORM_BWD, T, 0, D, RLF_F32)
    _check(_lib.rlf_block_norm_bwd(
        _at(grad_y, here, "grad_y", dt, shape) if pre else None, _at(grad_h, here, "grad_h", dt, shape), xp, xs,
        _at(h, here, "h", dt, shape) if pre else None, _DTYPES[dt], T, D, w1, b1, post_kind, w2, pre_kind, w_dt, gp, gate_form, alpha, beta,
        _at(stats, here, "stats", _f32, (4, T)), gxp, grp, ggp, gw1, gb1, gw2, gb2, 1 if accumulate else 0, wp, wn, _raw_stream(here)),
        "rlf_block_norm_bwd")
    return dict(grad_x=grad_x, grad_residual=grad_residual, grad_gate=grad_gate, grad_post_weight=grad_post_weight,
                grad_post_bias=grad_post_bias, grad_pre_weight=grad_pre_weight, grad_pre_bias=grad_pre_bias)


def step_arena_bytes(T, V, B, dt=RLF_BF16):
    return int(_lib.rlf_step_arena_bytes(T, V, B, dt))


def rlf_grpo_step_host(h_logits, h_ids, h_cu_seqlens, group_size, h_rewards, h_old_logp, h_ref_logp,
                       open_id, close_id, adv_eps, eps_clip, beta_kl, h_loss_out, d_arena, h_logp_out=None,
                       h_mask_out=None, h_dev_status=None):
    """One whole step from host tensors (pinned for full copy rate); waits for completion."""
    T, V = h_logits.shape
    B = h_rewards.shape[0]
    _check(_lib.rlf_grpo_step_host(
        _ptr(h_logits, cuda=False), _dt(h_logits), T, V, _ptr(h_ids, torch.int32, False),
        _ptr(h_cu_seqlens, torch.int32, False), B, int(group_size), _ptr(h_rewards, torch.float32, False),
        _ptr(h_old_logp, torch.float32, False), _ptr(h_ref_logp, torch.float32, False), open_id, close_id,
        float(adv_eps), float(eps_clip), float(beta_kl), _ptr(h_loss_out, torch.float64, False),
        _ptr(h_logp_out, torch.float32, False), _ptr(h_mask_out, torch.uint8, False),
        _ptr(h_dev_status, torch.int32, False), d_arena.data_ptr(), d_arena.numel(), _stream()),
        "rlf_grpo_step_host")
    return h_loss_out
