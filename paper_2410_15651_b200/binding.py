"""ctypes binding of librlhf_ppo.so: argument marshalling only.

Every function has the name and meaning of the C entry point it calls (include/rlhf_ppo.h);
torch supplies device memory and the current stream, nothing else.  There is no fallback: if
the library is missing or a call returns an error status, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "librlhf_ppo.so")

_i64 = ctypes.c_longlong
_int = ctypes.c_int
_f32 = ctypes.c_float
_vp = ctypes.c_void_p
_sz = ctypes.c_size_t


class ShapingStruct(ctypes.Structure):
    """rlhf_shaping_t"""
    _fields_ = [("prompt", _vp), ("prompt_stride_b", _i64), ("prompt_lengths", _vp), ("prompt_len", _int),
                ("tokens_len", _int), ("tokens", _vp), ("tokens_stride_b", _i64), ("start", _vp), ("repetition", _vp),
                ("frequency", _vp), ("presence", _vp), ("temperature", _vp), ("bias", _vp), ("bias_stride_b", _i64),
                ("mask", _vp), ("mask_stride_b", _i64), ("mask_stride_t", _i64)]


_shp = ctypes.POINTER(ShapingStruct)

# name -> (restype, argtypes); mirrors include/rlhf_ppo.h
SIGNATURES = {
    "rlhf_status_string": (ctypes.c_char_p, [_int]),
    "rlhf_last_cuda_error": (ctypes.c_char_p, []),
    "rlhf_pad_share": (_int, [_i64, _i64, _int, _int, _vp, _vp]),
    "rlhf_workspace_bytes": (_sz, [_int, _int]),
    "rlhf_workspace_init": (_int, [_vp, _sz, _vp]),
    "rlhf_poll_status": (_int, [_vp, _vp]),
    "rlhf_selftest_bounded_wait": (_int, [_vp, _sz, ctypes.c_ulonglong, _vp]),
    "rlhf_gather_logprobs": (_int, [_vp, _i64, _i64, _vp, _i64, _vp, _int, _int, _int, _vp, _vp, _sz, _vp]),
    "rlhf_gather_logprobs_ex": (_int, [_vp, _int, _i64, _i64, _vp, _i64, _vp, _int, _int, _int, _vp, _vp, _vp, _sz, _vp]),
    "rlhf_experience_ex": (_int, [_vp, _i64, _i64, _vp, _i64, _i64, _int, _vp, _i64, _vp, _vp, _vp, _vp,
                                  _int, _int, _int, _f32, _f32, _f32, _f32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "rlhf_ppo_loss_fwd_bwd_ex": (_int, [_vp, _int, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp,
                                        _int, _int, _int, _f32, _f32, _f32, _vp, _vp,
                                        _vp, _i64, _i64, _vp, _vp, _vp, _sz, _vp]),
    "rlhf_kl_reward": (_int, [_vp, _vp, _vp, _vp, _int, _int, _f32, _f32, _vp, _vp]),
    "rlhf_gae": (_int, [_vp, _vp, _vp, _int, _int, _f32, _f32, _vp, _vp, _vp]),
    "rlhf_whiten_advantages": (_int, [_vp, _vp, _int, _int, _f32, _vp, _vp, _sz, _vp]),
    "rlhf_ppo_stats": (_int, [_vp, _vp, _vp, _vp, _int, _int, _f32, _vp, _vp, _sz, _vp]),
    "rlhf_experience": (_int, [_vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _vp,
                               _int, _int, _int, _f32, _f32, _f32, _f32, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "rlhf_ppo_loss_fwd_bwd": (_int, [_vp, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp,
                                     _int, _int, _int, _f32, _f32, _f32, _vp, _vp,
                                     _vp, _i64, _i64, _vp, _vp, _vp, _sz, _vp]),
    "rlhf_ppo_loss_fwd_bwd_noalloc": (_int, [_vp, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp,
                                             _int, _int, _int, _f32, _f32, _f32, _vp, _vp,
                                             _vp, _i64, _i64, _vp, _vp, _vp, _vp]),
    "rlhf_topk_logprobs": (_int, [_vp, _int, _i64, _i64, _vp, _int, _int, _int, _int, _f32, _vp, _vp, _vp, _sz, _vp]),
    "rlhf_distill_loss_fwd_bwd": (_int, [_vp, _int, _i64, _i64, _vp, _vp, _i64, _i64, _int, _vp, _int, _int, _int, _int,
                                         _f32, _f32, _vp, _vp, _vp, _i64, _i64, _vp, _sz, _vp]),
    "rlhf_policy_kl_loss_fwd_bwd": (_int, [_vp, _int, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _i64, _i64,
                                           _int, _int, _int, _f32, _f32, _f32, _int, _f32, _vp, _vp,
                                           _vp, _i64, _i64, _vp, _vp, _sz, _vp]),
    "rlhf_preference_loss_fwd_bwd": (_int, [_vp, _int, _i64, _i64, _vp, _i64, _vp, _vp, _int, _int, _int,
                                            _int, _f32, _f32, _f32, _int, _f32, _vp, _vp,
                                            _vp, _i64, _i64, _vp, _vp, _sz, _vp]),
    "rlhf_shape_logits": (_int, [_vp, _int, _i64, _i64, _shp, _vp, _int, _int, _int, _vp, _int, _i64, _i64, _vp, _sz, _vp]),
    "rlhf_shape_logits_bwd": (_int, [_vp, _int, _i64, _i64, _vp, _i64, _i64, _shp, _vp, _int, _int, _int, _vp, _i64, _i64,
                                     _vp, _sz, _vp]),
    "rlhf_shaped_logprobs": (_int, [_vp, _int, _i64, _i64, _vp, _i64, _shp, _vp, _int, _int, _int, _vp, _vp, _vp,
                                    _vp, _sz, _vp]),
    "rlhf_shaped_logprobs_bwd": (_int, [_vp, _int, _i64, _i64, _vp, _i64, _shp, _vp, _int, _int, _int, _vp, _vp, _vp, _vp, _vp,
                                        _vp, _i64, _i64, _vp, _sz, _vp]),
    "rlhf_router_workspace_bytes": (_sz, [_int, _int, _int, _int]),
    "rlhf_router_loss_fwd_bwd": (_int, [_vp, _int, _i64, _i64, _i64, _vp, _i64, _i64, _i64, _vp, _int, _int, _int, _int, _int,
                                        _int, _int, _f32, _f32, _f32, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _sz, _vp]),
}

NOALLOC_MAX_TOKENS = 65536
MEAN_TOKENS, MEAN_SEQUENCES = 0, 1                    # rlhf_reduction_t
DISTILL_PLAIN, DISTILL_NORMALISED, DISTILL_TAIL = 0, 1, 2   # rlhf_distill_t
PREF_SIGMOID, PREF_HINGE, PREF_SQUARED = 0, 1, 2      # rlhf_preference_t
ROUTER_SOFTMAX, ROUTER_SIGMOID = 0, 1                 # rlhf_router_scoring_t
ROUTER_BATCH, ROUTER_SEQUENCE = 0, 1                  # rlhf_router_scope_t

_lib = None


class RlhfError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        name = lib().rlhf_status_string(status).decode()
        detail = lib().rlhf_last_cuda_error().decode() if status == 7 else ""
        super().__init__(f"{where}: {name}" + (f" ({detail})" if detail else ""))


def lib() -> ctypes.CDLL:
    """Load the CUDA library (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2410_15651_b200.build` "
                "(there is no CPU or PyTorch fallback)")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def pad_share(n_valid: int, n_padded: int, n_blocks: int, block: int) -> Tuple[int, int]:
    """(start, count) of the padded rows that `block` zero-fills in a loss launch (host-side helper)."""
    start, count = _i64(0), _i64(0)
    _check(lib().rlhf_pad_share(n_valid, n_padded, n_blocks, block, ctypes.byref(start), ctypes.byref(count)),
           "rlhf_pad_share")
    return int(start.value), int(count.value)


def _check(status: int, where: str) -> None:
    if status != 0:
        raise RlhfError(status, where)


def _stream(t: torch.Tensor) -> int:
    return torch.cuda.current_stream(t.device).cuda_stream


def _dev(t: torch.Tensor, dtype, what: str) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor (the library has no CPU path)")
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    return t


def _bt(t: torch.Tensor, B: int, T: int, what: str) -> torch.Tensor:
    _dev(t, torch.float32, what)
    if tuple(t.shape) != (B, T) or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous [{B},{T}] tensor")
    return t


DTYPES = {torch.bfloat16: 0, torch.float16: 1}        # rlhf_dtype_t


def _logits(t: torch.Tensor, what: str) -> Tuple[int, int, int, int, int]:
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor (the library has no CPU path)")
    if t.dtype not in DTYPES:
        raise TypeError(f"{what} must be bfloat16 or float16, got {t.dtype}")
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{what} must be [B,T,V] with a contiguous vocabulary axis")
    return t.shape[0], t.shape[1], t.shape[2], t.stride(0), t.stride(1)


def _ids(t: torch.Tensor, B: int, T: int) -> int:
    _dev(t, torch.int64, "ids")
    if tuple(t.shape) != (B, T) or (T > 1 and t.stride(1) != 1):
        raise ValueError("ids must be [B,T] with a contiguous time axis")
    return t.stride(0)


def _lengths(t: torch.Tensor, B: int) -> torch.Tensor:
    _dev(t, torch.int32, "lengths")
    if tuple(t.shape) != (B,) or not t.is_contiguous():
        raise ValueError("lengths must be a contiguous int32 [B] tensor")
    return t


def workspace_bytes(B: int, T: int) -> int:
    return int(lib().rlhf_workspace_bytes(B, T))


def workspace(B: int, T: int, device) -> torch.Tensor:
    """Allocate (through torch) and initialise a workspace for batches of up to B x T tokens."""
    ws = torch.empty(workspace_bytes(B, T), dtype=torch.uint8, device=device)
    _check(lib().rlhf_workspace_init(ws.data_ptr(), ws.numel(), _stream(ws)), "rlhf_workspace_init")
    return ws


def poll_status(ws: torch.Tensor) -> int:
    """Synchronise and return (then clear) the device-detected status flags."""
    return int(lib().rlhf_poll_status(ws.data_ptr(), _stream(ws)))


def selftest_bounded_wait(ws: torch.Tensor, limit_ns: int) -> None:
    """Launch the kernel whose only wait can never be satisfied; poll_status(ws) then reports the timeout flag."""
    _check(lib().rlhf_selftest_bounded_wait(ws.data_ptr(), ws.numel(), int(limit_ns), _stream(ws)),
           "rlhf_selftest_bounded_wait")


def status_string(status: int) -> str:
    return lib().rlhf_status_string(int(status)).decode()


def gather_logprobs(logits: torch.Tensor, ids: torch.Tensor, lengths: torch.Tensor,
                    ws: torch.Tensor, out: Optional[torch.Tensor] = None,
                    out_entropy: Optional[torch.Tensor] = None) -> torch.Tensor:
    """rlhf_gather_logprobs for bf16 logits without an entropy output, else rlhf_gather_logprobs_ex."""
    B, T, V, sb, st = _logits(logits, "logits")
    isb = _ids(ids, B, T)
    _lengths(lengths, B)
    if out is None:
        out = torch.empty((B, T), dtype=torch.float32, device=logits.device)
    _bt(out, B, T, "out")
    if logits.dtype == torch.bfloat16 and out_entropy is None:
        _check(lib().rlhf_gather_logprobs(logits.data_ptr(), sb, st, ids.data_ptr(), isb, lengths.data_ptr(),
                                          B, T, V, out.data_ptr(), ws.data_ptr(), ws.numel(), _stream(logits)),
               "rlhf_gather_logprobs")
        return out
    ent_ptr = _bt(out_entropy, B, T, "out_entropy").data_ptr() if out_entropy is not None else None
    _check(lib().rlhf_gather_logprobs_ex(logits.data_ptr(), DTYPES[logits.dtype], sb, st, ids.data_ptr(), isb,
                                         lengths.data_ptr(), B, T, V, out.data_ptr(), ent_ptr,
                                         ws.data_ptr(), ws.numel(), _stream(logits)), "rlhf_gather_logprobs_ex")
    return out


def kl_reward(lp_old: torch.Tensor, lp_ref: torch.Tensor, score: torch.Tensor, lengths: torch.Tensor,
              beta_kl: float, reward_clip: float, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    B, T = lp_old.shape
    _bt(lp_old, B, T, "lp_old")
    _bt(lp_ref, B, T, "lp_ref")
    _dev(score, torch.float32, "score")
    if tuple(score.shape) != (B,) or not score.is_contiguous():
        raise ValueError("score must be a contiguous [B] tensor")
    _lengths(lengths, B)
    if out is None:
        out = torch.empty_like(lp_old)
    _bt(out, B, T, "out")
    _check(lib().rlhf_kl_reward(lp_old.data_ptr(), lp_ref.data_ptr(), score.data_ptr(), lengths.data_ptr(),
                                B, T, beta_kl, reward_clip, out.data_ptr(), _stream(lp_old)),
           "rlhf_kl_reward")
    return out


def gae(rewards: torch.Tensor, values_old: torch.Tensor, lengths: torch.Tensor, gamma: float, lam: float,
        out_adv: Optional[torch.Tensor] = None, out_returns: Optional[torch.Tensor] = None):
    B, T = rewards.shape
    _bt(rewards, B, T, "rewards")
    _bt(values_old, B, T, "values_old")
    _lengths(lengths, B)
    if out_adv is None:
        out_adv = torch.empty_like(rewards)
    if out_returns is None:
        out_returns = torch.empty_like(rewards)
    _bt(out_adv, B, T, "out_adv")
    _bt(out_returns, B, T, "out_returns")
    _check(lib().rlhf_gae(rewards.data_ptr(), values_old.data_ptr(), lengths.data_ptr(), B, T, gamma, lam,
                          out_adv.data_ptr(), out_returns.data_ptr(), _stream(rewards)), "rlhf_gae")
    return out_adv, out_returns


def whiten_advantages(adv: torch.Tensor, lengths: torch.Tensor, eps: float, ws: torch.Tensor,
                      out: Optional[torch.Tensor] = None) -> torch.Tensor:
    B, T = adv.shape
    _bt(adv, B, T, "adv")
    _lengths(lengths, B)
    if out is None:
        out = torch.empty_like(adv)
    _bt(out, B, T, "out")
    _check(lib().rlhf_whiten_advantages(adv.data_ptr(), lengths.data_ptr(), B, T, eps, out.data_ptr(),
                                        ws.data_ptr(), ws.numel(), _stream(adv)), "rlhf_whiten_advantages")
    return out


def ppo_stats(lp_new: torch.Tensor, lp_old: torch.Tensor, adv: torch.Tensor, lengths: torch.Tensor,
              clip_eps: float, ws: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """[approx_kl, clip_frac] of the policy step, as a device tensor of two floats."""
    B, T = lp_new.shape
    for name, t in (("lp_new", lp_new), ("lp_old", lp_old), ("adv", adv)):
        _bt(t, B, T, name)
    _lengths(lengths, B)
    if out is None:
        out = torch.empty(2, dtype=torch.float32, device=lp_new.device)
    _dev(out, torch.float32, "out")
    _check(lib().rlhf_ppo_stats(lp_new.data_ptr(), lp_old.data_ptr(), adv.data_ptr(), lengths.data_ptr(), B, T,
                                clip_eps, out.data_ptr(), ws.data_ptr(), ws.numel(), _stream(lp_new)),
           "rlhf_ppo_stats")
    return out


class Experience:
    """Buffers written by experience(); reusable from call to call."""

    def __init__(self, B: int, T: int, device):
        f = lambda: torch.empty((B, T), dtype=torch.float32, device=device)
        self.lp_actor, self.lp_ref, self.rewards, self.adv, self.returns = f(), f(), f(), f(), f()


def experience(actor_logits: torch.Tensor, ref_logits: torch.Tensor, ids: torch.Tensor, lengths: torch.Tensor,
               score: torch.Tensor, values_old: torch.Tensor, beta_kl: float, reward_clip: float,
               gamma: float, lam: float, ws: torch.Tensor, out: Optional[Experience] = None,
               lp_old: Optional[torch.Tensor] = None, out_entropy: Optional[torch.Tensor] = None) -> Experience:
    """rlhf_experience for bf16 logits without an entropy output, else rlhf_experience_ex."""
    B, T, V, asb, ast = _logits(actor_logits, "actor_logits")
    rB, rT, rV, rsb, rst = _logits(ref_logits, "ref_logits")
    if (rB, rT, rV) != (B, T, V):
        raise ValueError("actor and reference logits must have the same shape")
    isb = _ids(ids, B, T)
    _lengths(lengths, B)
    _dev(score, torch.float32, "score")
    if tuple(score.shape) != (B,) or not score.is_contiguous():
        raise ValueError("score must be a contiguous [B] tensor")
    _bt(values_old, B, T, "values_old")
    if out is None:
        out = Experience(B, T, actor_logits.device)
    for name in ("lp_actor", "lp_ref", "rewards", "adv", "returns"):
        _bt(getattr(out, name), B, T, "out." + name)
    lp_old_ptr = _bt(lp_old, B, T, "lp_old").data_ptr() if lp_old is not None else None
    if actor_logits.dtype != ref_logits.dtype:
        raise TypeError("actor and reference logits must have the same element type")
    if actor_logits.dtype != torch.bfloat16 or out_entropy is not None:
        ent_ptr = _bt(out_entropy, B, T, "out_entropy").data_ptr() if out_entropy is not None else None
        _check(lib().rlhf_experience_ex(
            actor_logits.data_ptr(), asb, ast, ref_logits.data_ptr(), rsb, rst, DTYPES[actor_logits.dtype],
            ids.data_ptr(), isb, lengths.data_ptr(), score.data_ptr(), values_old.data_ptr(), lp_old_ptr, B, T, V,
            beta_kl, reward_clip, gamma, lam, out.lp_actor.data_ptr(), out.lp_ref.data_ptr(),
            out.rewards.data_ptr(), out.adv.data_ptr(), out.returns.data_ptr(), ent_ptr,
            ws.data_ptr(), ws.numel(), _stream(actor_logits)), "rlhf_experience_ex")
        return out
    _check(lib().rlhf_experience(
        actor_logits.data_ptr(), asb, ast, ref_logits.data_ptr(), rsb, rst, ids.data_ptr(), isb,
        lengths.data_ptr(), score.data_ptr(), values_old.data_ptr(), lp_old_ptr, B, T, V,
        beta_kl, reward_clip, gamma, lam, out.lp_actor.data_ptr(), out.lp_ref.data_ptr(),
        out.rewards.data_ptr(), out.adv.data_ptr(), out.returns.data_ptr(),
        ws.data_ptr(), ws.numel(), _stream(actor_logits)), "rlhf_experience")
    return out


class PPOOutputs:
    """Buffers written by ppo_loss_fwd_bwd; reusable from call to call."""

    def __init__(self, logits: torch.Tensor, in_place: bool = False, want_lp_new: bool = True):
        B, T = logits.shape[0], logits.shape[1]
        dev = logits.device
        self.loss = torch.empty(2, dtype=torch.float32, device=dev)       # [loss_pg, loss_vf]
        self.dlogits = logits if in_place else torch.empty(logits.shape, dtype=logits.dtype, device=dev)
        self.dvalues = torch.empty((B, T), dtype=torch.float32, device=dev)
        self.lp_new = torch.empty((B, T), dtype=torch.float32, device=dev) if want_lp_new else None


def ppo_loss_fwd_bwd(logits: torch.Tensor, ids: torch.Tensor, lengths: torch.Tensor,
                     lp_old: torch.Tensor, adv: torch.Tensor, values_new: torch.Tensor,
                     values_old: torch.Tensor, returns: torch.Tensor,
                     clip_eps: float, value_clip: float, grad_scale: float,
                     ws: torch.Tensor, out: Optional[PPOOutputs] = None) -> PPOOutputs:
    B, T, V, sb, st = _logits(logits, "logits")
    isb = _ids(ids, B, T)
    _lengths(lengths, B)
    for name, t in (("lp_old", lp_old), ("adv", adv), ("values_new", values_new),
                    ("values_old", values_old), ("returns", returns)):
        _bt(t, B, T, name)
    if out is None:
        out = PPOOutputs(logits)
    dB, dT, dV, dsb, dst = _logits(out.dlogits, "out.dlogits")
    if (dB, dT, dV) != (B, T, V):
        raise ValueError("out.dlogits must have the shape of logits")
    _bt(out.dvalues, B, T, "out.dvalues")
    lp_new_ptr = None
    if out.lp_new is not None:
        lp_new_ptr = _bt(out.lp_new, B, T, "out.lp_new").data_ptr()
    loss = _dev(out.loss, torch.float32, "out.loss")
    if out.dlogits.dtype != logits.dtype:
        raise TypeError("out.dlogits must have the element type of logits")
    if logits.dtype != torch.bfloat16:
        _check(lib().rlhf_ppo_loss_fwd_bwd_ex(
            logits.data_ptr(), DTYPES[logits.dtype], sb, st, ids.data_ptr(), isb, lengths.data_ptr(),
            lp_old.data_ptr(), adv.data_ptr(), values_new.data_ptr(), values_old.data_ptr(), returns.data_ptr(),
            B, T, V, clip_eps, value_clip, grad_scale,
            loss.data_ptr(), loss.data_ptr() + 4,
            out.dlogits.data_ptr(), dsb, dst, out.dvalues.data_ptr(), lp_new_ptr,
            ws.data_ptr(), ws.numel(), _stream(logits)), "rlhf_ppo_loss_fwd_bwd_ex")
        return out
    _check(lib().rlhf_ppo_loss_fwd_bwd(
        logits.data_ptr(), sb, st, ids.data_ptr(), isb, lengths.data_ptr(),
        lp_old.data_ptr(), adv.data_ptr(), values_new.data_ptr(), values_old.data_ptr(), returns.data_ptr(),
        B, T, V, clip_eps, value_clip, grad_scale,
        loss.data_ptr(), loss.data_ptr() + 4,
        out.dlogits.data_ptr(), dsb, dst, out.dvalues.data_ptr(), lp_new_ptr,
        ws.data_ptr(), ws.numel(), _stream(logits)), "rlhf_ppo_loss_fwd_bwd")
    return out


def ppo_loss_fwd_bwd_noalloc(logits: torch.Tensor, ids: torch.Tensor, lengths: torch.Tensor,
                             lp_old: torch.Tensor, adv: torch.Tensor, values_new: torch.Tensor,
                             values_old: torch.Tensor, returns: torch.Tensor,
                             clip_eps: float, value_clip: float, grad_scale: float,
                             out: PPOOutputs, device_status: Optional[torch.Tensor] = None) -> PPOOutputs:
    """rlhf_ppo_loss_fwd_bwd_noalloc: the same computation with no workspace argument, for callers
    that cannot allocate scratch memory (at most NOALLOC_MAX_TOKENS tokens; calls on one device must
    not overlap).  `out` must be given (this wrapper allocates nothing either); `device_status`,
    if given, is an int32 CUDA tensor of one element that receives the device-detected flags."""
    B, T, V, sb, st = _logits(logits, "logits")
    if logits.dtype != torch.bfloat16 or out.dlogits.dtype != torch.bfloat16:
        raise TypeError("rlhf_ppo_loss_fwd_bwd_noalloc takes bf16 logits")
    isb = _ids(ids, B, T)
    _lengths(lengths, B)
    for name, t in (("lp_old", lp_old), ("adv", adv), ("values_new", values_new),
                    ("values_old", values_old), ("returns", returns)):
        _bt(t, B, T, name)
    dB, dT, dV, dsb, dst = _logits(out.dlogits, "out.dlogits")
    if (dB, dT, dV) != (B, T, V):
        raise ValueError("out.dlogits must have the shape of logits")
    _bt(out.dvalues, B, T, "out.dvalues")
    lp_new_ptr = None
    if out.lp_new is not None:
        lp_new_ptr = _bt(out.lp_new, B, T, "out.lp_new").data_ptr()
    loss = _dev(out.loss, torch.float32, "out.loss")
    st_ptr = None
    if device_status is not None:
        st_ptr = _dev(device_status, torch.int32, "device_status").data_ptr()
    _check(lib().rlhf_ppo_loss_fwd_bwd_noalloc(
        logits.data_ptr(), sb, st, ids.data_ptr(), isb, lengths.data_ptr(),
        lp_old.data_ptr(), adv.data_ptr(), values_new.data_ptr(), values_old.data_ptr(), returns.data_ptr(),
        B, T, V, clip_eps, value_clip, grad_scale,
        loss.data_ptr(), loss.data_ptr() + 4,
        out.dlogits.data_ptr(), dsb, dst, out.dvalues.data_ptr(), lp_new_ptr,
        st_ptr, _stream(logits)), "rlhf_ppo_loss_fwd_bwd_noalloc")
    return out


# ---------------------------------------------------------------- objectives beside the PPO step
# On small batches a call costs the host more than the device, so these wrappers look at each argument in one
# expression and say what is wrong only where something is.
_F32 = torch.float32


def _rows(t: torch.Tensor) -> Tuple[int, int, int, int, int, int]:
    """(B, T, V, stride_b, stride_t, device index) of a logits tensor."""
    if t.dtype not in DTYPES or not t.is_cuda or t.dim() != 3:
        _logits(t, "logits")
    B, T, V = t.shape
    sb, st, sv = t.stride()
    if sv != 1 and V > 1:
        _logits(t, "logits")
    return B, T, V, sb, st, t.get_device()


def _arg(t: torch.Tensor, shape: Tuple[int, ...], dtype, dev: int, what: str) -> int:
    """Address of a contiguous tensor of this shape and type on the device of the logits."""
    if t.dtype is dtype and t.get_device() == dev and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    _dev(t, dtype, what)
    _same_device(t, dev, what)
    raise ValueError(f"{what} must be a contiguous {list(shape)} tensor")


def _opt(t: Optional[torch.Tensor], shape: Tuple[int, ...], dtype, dev: int, what: str) -> Optional[int]:
    return None if t is None else _arg(t, shape, dtype, dev, what)


def _same_device(t: torch.Tensor, dev: int, what: str) -> None:
    if t.get_device() != dev:
        raise ValueError(f"{what} is on {t.device}, the logits on cuda:{dev}")


def _ids_arg(t: torch.Tensor, B: int, T: int, dev: int) -> Tuple[int, int]:
    """(address, stride between sequences) of the generated tokens."""
    stride = _ids(t, B, T)
    _same_device(t, dev, "ids")
    return t.data_ptr(), stride


def _ws(ws: torch.Tensor, dev: int) -> Tuple[int, int]:
    if not ws.is_cuda or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous CUDA tensor (see workspace())")
    _same_device(ws, dev, "ws")
    return ws.data_ptr(), ws.nbytes


def _dlogits(t: torch.Tensor, logits: torch.Tensor, dev: int) -> Tuple[int, int, int]:
    """(address, stride_b, stride_t) of the gradient tensor, which has the shape and type of the logits."""
    if t.dtype is not logits.dtype:
        raise TypeError("out.dlogits must have the element type of logits")
    if t.shape != logits.shape:
        raise ValueError("out.dlogits must have the shape of logits")
    _same_device(t, dev, "out.dlogits")
    sb, st, sv = t.stride()
    if sv != 1 and t.shape[2] > 1:
        raise ValueError("out.dlogits must have a contiguous vocabulary axis")
    return t.data_ptr(), sb, st


def _like(logits: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(logits, memory_format=torch.contiguous_format)


def _raw_stream(dev: int) -> int:
    return torch.cuda.current_stream(dev).cuda_stream


# the same without the Stream object (0.1 us against 2.2 us)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)


def _call(name: str, dev: int, *args) -> None:
    """Calls the entry point with the device of its tensors current and that device's current stream."""
    if torch.cuda.current_device() == dev:
        status = getattr(_lib or lib(), name)(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            status = getattr(_lib or lib(), name)(*args, _raw_stream(dev))
    if status != 0:
        raise RlhfError(status, name)


TOPK_MAX = 256


class TopK:
    """Buffers written by topk_logprobs: int32 ids and fp32 log-probs, [B,T,K]; reusable from call to call."""

    def __init__(self, B: int, T: int, K: int, device):
        self.ids = torch.empty((B, T, K), dtype=torch.int32, device=device)
        self.logprobs = torch.empty((B, T, K), dtype=_F32, device=device)


def topk_logprobs(logits: torch.Tensor, lengths: torch.Tensor, k: int, temperature: float, ws: torch.Tensor,
                  out: Optional[TopK] = None) -> TopK:
    """rlhf_topk_logprobs: the k largest log-probs of every row and their entries (1 <= k <= TOPK_MAX)."""
    B, T, V, sb, st, dev = _rows(logits)
    if out is None:
        out = TopK(B, T, max(k, 0), logits.device)
    _call("rlhf_topk_logprobs", dev, logits.data_ptr(), DTYPES[logits.dtype], sb, st,
          _arg(lengths, (B,), torch.int32, dev, "lengths"), B, T, V, k, temperature,
          _arg(out.ids, (B, T, k), torch.int32, dev, "out.ids"),
          _arg(out.logprobs, (B, T, k), _F32, dev, "out.logprobs"), *_ws(ws, dev))
    return out


class DistillOutputs:
    """Buffers written by distill_loss_fwd_bwd; reusable from call to call."""

    def __init__(self, logits: torch.Tensor, in_place: bool = False, want_row_loss: bool = True):
        B, T, _ = logits.shape
        self.loss = logits.new_empty(1, dtype=_F32)
        self.dlogits = logits if in_place else _like(logits)
        self.row_loss = logits.new_empty((B, T), dtype=_F32) if want_row_loss else None


def distill_loss_fwd_bwd(logits: torch.Tensor, topk_ids: torch.Tensor, topk_logprobs: torch.Tensor, lengths: torch.Tensor,
                         mode: int, temperature: float, grad_scale: float, ws: torch.Tensor,
                         out: Optional[DistillOutputs] = None) -> DistillOutputs:
    """rlhf_distill_loss_fwd_bwd.  topk_ids (int32) and topk_logprobs (fp32) are [B,T,K] with equal strides and a contiguous
    last axis; `mode` is DISTILL_PLAIN, DISTILL_NORMALISED or DISTILL_TAIL."""
    B, T, V, sb, st, dev = _rows(logits)
    _dev(topk_ids, torch.int32, "topk_ids")
    _dev(topk_logprobs, _F32, "topk_logprobs")
    _same_device(topk_ids, dev, "topk_ids")
    _same_device(topk_logprobs, dev, "topk_logprobs")
    if topk_ids.dim() != 3 or topk_ids.shape[:2] != (B, T) or topk_ids.shape != topk_logprobs.shape:
        raise ValueError(f"topk_ids and topk_logprobs must be [{B},{T},K]")
    K = topk_ids.shape[2]
    ksb, kst, ks = topk_ids.stride()
    lsb, lst, ls = topk_logprobs.stride()                # (the stride of an axis with one position says nothing)
    if (B > 1 and ksb != lsb) or (T > 1 and kst != lst) or (K > 1 and (ks != 1 or ls != 1)):
        raise ValueError("topk_ids and topk_logprobs must have the same strides and a contiguous last axis")
    if out is None:
        out = DistillOutputs(logits)
    _call("rlhf_distill_loss_fwd_bwd", dev, logits.data_ptr(), DTYPES[logits.dtype], sb, st,
          topk_ids.data_ptr(), topk_logprobs.data_ptr(), ksb, kst, K, _arg(lengths, (B,), torch.int32, dev, "lengths"),
          B, T, V, mode, temperature, grad_scale, _arg(out.loss, (1,), _F32, dev, "out.loss"),
          _opt(out.row_loss, (B, T), _F32, dev, "out.row_loss"), *_dlogits(out.dlogits, logits, dev), *_ws(ws, dev))
    return out


class PolicyKlOutputs:
    """Buffers written by policy_kl_loss_fwd_bwd; reusable from call to call."""

    def __init__(self, logits: torch.Tensor, in_place: bool = False, want_lp_new: bool = True):
        B, T, _ = logits.shape
        self.loss = logits.new_empty(2, dtype=_F32)                                  # [loss_pg, loss_kl]
        self.dlogits = logits if in_place else _like(logits)
        self.lp_new = logits.new_empty((B, T), dtype=_F32) if want_lp_new else None


def policy_kl_loss_fwd_bwd(logits: torch.Tensor, ids: torch.Tensor, lengths: torch.Tensor, lp_old: torch.Tensor,
                           lp_ref: Optional[torch.Tensor], adv: torch.Tensor, clip_low: float, clip_high: float,
                           kl_coef: float, reduction: int, grad_scale: float, ws: torch.Tensor,
                           out: Optional[PolicyKlOutputs] = None) -> PolicyKlOutputs:
    """rlhf_policy_kl_loss_fwd_bwd.  `adv` is [B,T] (any strides) or [B], one advantage per sequence; `reduction` is
    MEAN_TOKENS or MEAN_SEQUENCES."""
    B, T, V, sb, st, dev = _rows(logits)
    _dev(adv, _F32, "adv")
    _same_device(adv, dev, "adv")
    if adv.shape == (B, T):
        asb, ast = adv.stride()
    elif adv.shape == (B,):
        asb, ast = adv.stride(0), 0
    else:
        raise ValueError(f"adv must be [{B},{T}] or [{B}]")
    if out is None:
        out = PolicyKlOutputs(logits)
    loss = _arg(out.loss, (2,), _F32, dev, "out.loss")
    _call("rlhf_policy_kl_loss_fwd_bwd", dev, logits.data_ptr(), DTYPES[logits.dtype], sb, st, *_ids_arg(ids, B, T, dev),
          _arg(lengths, (B,), torch.int32, dev, "lengths"), _arg(lp_old, (B, T), _F32, dev, "lp_old"),
          _opt(lp_ref, (B, T), _F32, dev, "lp_ref"), adv.data_ptr(), asb, ast, B, T, V, clip_low, clip_high, kl_coef,
          reduction, grad_scale, loss, loss + 4, *_dlogits(out.dlogits, logits, dev),
          _opt(out.lp_new, (B, T), _F32, dev, "out.lp_new"), *_ws(ws, dev))
    return out


class PreferenceOutputs:
    """Buffers written by preference_loss_fwd_bwd; reusable from call to call."""

    def __init__(self, logits: torch.Tensor, in_place: bool = False, want_lp_new: bool = True):
        B, T, _ = logits.shape
        self.loss = logits.new_empty(1, dtype=_F32)
        self.rewards = logits.new_empty(B, dtype=_F32)                               # beta * log ratio of every sequence
        self.dlogits = logits if in_place else _like(logits)
        self.lp_new = logits.new_empty((B, T), dtype=_F32) if want_lp_new else None


def preference_loss_fwd_bwd(logits: torch.Tensor, ids: torch.Tensor, lengths: torch.Tensor,
                            lp_ref: Optional[torch.Tensor], kind: int, beta: float, margin: float,
                            label_smoothing: float, length_mean: bool, grad_scale: float, ws: torch.Tensor,
                            out: Optional[PreferenceOutputs] = None) -> PreferenceOutputs:
    """rlhf_preference_loss_fwd_bwd: sequences 0..B/2-1 are the chosen, B/2..B-1 the rejected responses; `kind` is
    PREF_SIGMOID, PREF_HINGE or PREF_SQUARED."""
    B, T, V, sb, st, dev = _rows(logits)
    if out is None:
        out = PreferenceOutputs(logits)
    _call("rlhf_preference_loss_fwd_bwd", dev, logits.data_ptr(), DTYPES[logits.dtype], sb, st, *_ids_arg(ids, B, T, dev),
          _arg(lengths, (B,), torch.int32, dev, "lengths"), _opt(lp_ref, (B, T), _F32, dev, "lp_ref"), B, T, V, kind, beta,
          margin, label_smoothing, int(length_mean), grad_scale, _arg(out.loss, (1,), _F32, dev, "out.loss"),
          _arg(out.rewards, (B,), _F32, dev, "out.rewards"), *_dlogits(out.dlogits, logits, dev),
          _opt(out.lp_new, (B, T), _F32, dev, "out.lp_new"), *_ws(ws, dev))
    return out


# ---------------------------------------------------------------- shaped logits
class Shaping:
    """rlhf_shaping_t for B sequences over a vocabulary of V: the settings of a rollout and the history that its penalties
    look at.  The tensors are read by every call that is given this object (they may be changed in place between calls, as a
    decoding loop does with `tokens` and `start`), and are kept alive by it.

      tokens [B,S] int64      the answer's tokens; those before a row are its history
      start [B] int32         tokens before the first row (none: 0)
      prompt [B,P] int64      -1: padding;  prompt_lengths [B] int32 (none: P)
      repetition, frequency, presence, temperature [B] fp32
      bias [V] or [B,V] fp32
      mask [B,W] or [B,T,W] int32, W = ceil(V / 32) words of allowed entries (any strides; a first axis of 1 is shared)
    """

    def __init__(self, B: int, V: int, tokens: Optional[torch.Tensor] = None, start: Optional[torch.Tensor] = None,
                 prompt: Optional[torch.Tensor] = None, prompt_lengths: Optional[torch.Tensor] = None,
                 repetition: Optional[torch.Tensor] = None, frequency: Optional[torch.Tensor] = None,
                 presence: Optional[torch.Tensor] = None, temperature: Optional[torch.Tensor] = None,
                 bias: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None):
        given = {k: t for k, t in dict(tokens=tokens, start=start, prompt=prompt, prompt_lengths=prompt_lengths,
                                       repetition=repetition, frequency=frequency, presence=presence,
                                       temperature=temperature, bias=bias, mask=mask).items() if t is not None}
        for name, t in given.items():
            if not t.is_cuda:
                raise ValueError(f"{name} must be a CUDA tensor (the library has no CPU path)")
        self.B, self.V, self.tensors = B, V, given
        self.mask_rows = 0                               # rows that the mask has of a sequence; 0: any number
        self.dev = next((t.get_device() for t in given.values()), None)
        c = self.struct = ShapingStruct()
        for name in ("tokens", "prompt"):
            if name not in given:
                continue
            t = _dev(given[name], torch.int64, name)
            if t.dim() != 2 or t.shape[0] != B or (t.shape[1] > 1 and t.stride(1) != 1):
                raise ValueError(f"{name} must be [{B},n] with a contiguous last axis")
            setattr(c, name, t.data_ptr())
            setattr(c, name + "_stride_b", t.stride(0))
            setattr(c, name + "_len", t.shape[1])
        for name, dtype in (("start", torch.int32), ("prompt_lengths", torch.int32), ("repetition", _F32), ("frequency", _F32),
                            ("presence", _F32), ("temperature", _F32)):
            if name in given:
                setattr(c, name, _arg(given[name], (B,), dtype, self.dev, name))
        if bias is not None:
            _dev(bias, _F32, "bias")
            if bias.shape not in ((V,), (B, V)) or (V > 1 and bias.stride(-1) != 1):
                raise ValueError(f"bias must be [{V}] or [{B},{V}] with a contiguous vocabulary axis")
            c.bias, c.bias_stride_b = bias.data_ptr(), bias.stride(0) if bias.dim() == 2 else 0
        if mask is not None:
            _dev(mask, torch.int32, "mask")
            W = (V + 31) // 32
            if mask.dim() not in (2, 3) or mask.shape[0] not in (1, B) or mask.shape[-1] != W or (W > 1 and mask.stride(-1) != 1):
                raise ValueError(f"mask must be [{B},{W}] or [{B},T,{W}] with contiguous words")
            c.mask, c.mask_stride_b = mask.data_ptr(), mask.stride(0) if mask.shape[0] > 1 else 0
            if mask.dim() == 3 and mask.shape[1] != 1:
                self.mask_rows, c.mask_stride_t = mask.shape[1], mask.stride(1)
        for name, t in given.items():
            _same_device(t, self.dev, name)
        self._pointer = ctypes.pointer(c)

    def pointer(self, B: int, T: int, V: int, dev: int):
        """The struct for a call on [B,T,V] logits of this device."""
        if self.B != B or self.V != V or (self.mask_rows and self.mask_rows != T):
            raise ValueError(f"the shaping is for {self.B} sequences over {self.V} entries"
                             + (f" and {self.mask_rows} rows" if self.mask_rows else "") + f", the logits are [{B},{T},{V}]")
        if self.dev is not None and self.dev != dev:
            raise ValueError(f"the shaping is on cuda:{self.dev}, the logits on cuda:{dev}")
        return self._pointer


SHAPED_DTYPES = {torch.bfloat16: 0, torch.float16: 1, _F32: 2}


def _rows_out(t: torch.Tensor, logits: torch.Tensor, dev: int, what: str) -> Tuple[int, int, int]:
    """(address, stride_b, stride_t) of a tensor of the logits' shape."""
    if t.shape != logits.shape:
        raise ValueError(f"{what} must have the shape of logits")
    _same_device(t, dev, what)
    sb, st, sv = t.stride()
    if sv != 1 and t.shape[2] > 1:
        raise ValueError(f"{what} must have a contiguous vocabulary axis")
    return t.data_ptr(), sb, st


def shape_logits(logits: torch.Tensor, lengths: torch.Tensor, shaping: Shaping, ws: torch.Tensor,
                 out: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """rlhf_shape_logits: the shaped logits, in the logits' type or fp32 (`dtype`, or that of `out`); `out` may be the logits."""
    B, T, V, sb, st, dev = _rows(logits)
    if out is None:
        out = torch.empty((B, T, V), dtype=dtype or logits.dtype, device=logits.device)
    if out.dtype is not (dtype or out.dtype) or out.dtype not in (logits.dtype, _F32):
        raise TypeError("out must have the element type of logits, or float32")
    p, osb, ost = _rows_out(out, logits, dev, "out")
    _call("rlhf_shape_logits", dev, logits.data_ptr(), DTYPES[logits.dtype], sb, st, shaping.pointer(B, T, V, dev),
          _arg(lengths, (B,), torch.int32, dev, "lengths"), B, T, V, p, SHAPED_DTYPES[out.dtype], osb, ost, *_ws(ws, dev))
    return out


def shape_logits_bwd(dshaped: torch.Tensor, logits: torch.Tensor, lengths: torch.Tensor, shaping: Shaping, ws: torch.Tensor,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """rlhf_shape_logits_bwd: the gradient with respect to the logits, from the one with respect to the shaped logits (of the
    logits' type); `out` may be dshaped."""
    B, T, V, sb, st, dev = _rows(logits)
    if dshaped.dtype is not logits.dtype:
        raise TypeError("dshaped must have the element type of logits")
    if out is None:
        out = _like(logits)
    d, dsb, dst = _rows_out(dshaped, logits, dev, "dshaped")
    _call("rlhf_shape_logits_bwd", dev, d, DTYPES[logits.dtype], dsb, dst, logits.data_ptr(), sb, st,
          shaping.pointer(B, T, V, dev), _arg(lengths, (B,), torch.int32, dev, "lengths"), B, T, V,
          *_dlogits(out, logits, dev), *_ws(ws, dev))
    return out


class ShapedLogprobs:
    """What shaped_logprobs writes and shaped_logprobs_bwd reads: log-probs [B,T], the normaliser in two parts [B,T,2] and,
    if wanted, the entropy [B,T]; reusable from call to call."""

    def __init__(self, logits: torch.Tensor, want_entropy: bool = False, logprobs: Optional[torch.Tensor] = None,
                 lse: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None):
        B, T, _ = logits.shape
        new = lambda *n: logits.new_empty(n, dtype=_F32)  # noqa: E731
        self.logprobs = new(B, T) if logprobs is None else logprobs
        self.lse = new(B, T, 2) if lse is None else lse
        self.entropy = new(B, T) if entropy is None and want_entropy else entropy


def shaped_logprobs(logits: torch.Tensor, ids: torch.Tensor, lengths: torch.Tensor, shaping: Shaping, ws: torch.Tensor,
                    want_entropy: bool = False, out: Optional[ShapedLogprobs] = None) -> ShapedLogprobs:
    """rlhf_shaped_logprobs: log-probs (and entropy, if wanted or if `out` has a place for it) under the shaped logits."""
    B, T, V, sb, st, dev = _rows(logits)
    if out is None:
        out = ShapedLogprobs(logits, want_entropy)
    _call("rlhf_shaped_logprobs", dev, logits.data_ptr(), DTYPES[logits.dtype], sb, st, *_ids_arg(ids, B, T, dev),
          shaping.pointer(B, T, V, dev), _arg(lengths, (B,), torch.int32, dev, "lengths"), B, T, V,
          _arg(out.logprobs, (B, T), _F32, dev, "out.logprobs"), _arg(out.lse, (B, T, 2), _F32, dev, "out.lse"),
          _opt(out.entropy, (B, T), _F32, dev, "out.entropy"), *_ws(ws, dev))
    return out


def shaped_logprobs_bwd(logits: torch.Tensor, ids: torch.Tensor, lengths: torch.Tensor, shaping: Shaping,
                        forward: ShapedLogprobs, grad_logprobs: torch.Tensor, grad_entropy: Optional[torch.Tensor],
                        ws: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """rlhf_shaped_logprobs_bwd: the gradient with respect to the logits; `out` may be the logits."""
    B, T, V, sb, st, dev = _rows(logits)
    if out is None:
        out = _like(logits)
    _call("rlhf_shaped_logprobs_bwd", dev, logits.data_ptr(), DTYPES[logits.dtype], sb, st, *_ids_arg(ids, B, T, dev),
          shaping.pointer(B, T, V, dev), _arg(lengths, (B,), torch.int32, dev, "lengths"), B, T, V,
          _arg(forward.logprobs, (B, T), _F32, dev, "forward.logprobs"), _arg(forward.lse, (B, T, 2), _F32, dev, "forward.lse"),
          _opt(forward.entropy, (B, T), _F32, dev, "forward.entropy"),
          _arg(grad_logprobs, (B, T), _F32, dev, "grad_logprobs"), _opt(grad_entropy, (B, T), _F32, dev, "grad_entropy"),
          *_dlogits(out, logits, dev), *_ws(ws, dev))
    return out


# ---------------------------------------------------------------- the router of a policy with experts
def router_workspace_bytes(L: int, B: int, T: int, E: int) -> int:
    return int(lib().rlhf_router_workspace_bytes(L, B, T, E))


def router_workspace(L: int, B: int, T: int, E: int, device) -> torch.Tensor:
    """Allocate (through torch) and initialise a workspace for router_loss_fwd_bwd on [L,B,T,E] logits."""
    ws = torch.empty(router_workspace_bytes(L, B, T, E), dtype=torch.uint8, device=device)
    with torch.cuda.device(ws.device):
        _check(lib().rlhf_workspace_init(ws.data_ptr(), ws.numel(), _stream(ws)), "rlhf_workspace_init")
    return ws


def _router_logits(t: torch.Tensor) -> None:
    """Says what is wrong with router logits."""
    if not t.is_cuda:
        raise ValueError("logits must be a CUDA tensor (the library has no CPU path)")
    if t.dtype not in SHAPED_DTYPES:
        raise TypeError(f"logits must be bfloat16, float16 or float32, got {t.dtype}")
    raise ValueError("logits must be [L,B,T,E] with a contiguous expert axis")


class RouterOutputs:
    """Buffers written by router_loss_fwd_bwd; reusable from call to call."""

    def __init__(self, logits: torch.Tensor, k: int, scope: int, in_place: bool = False, want_ids: bool = True):
        L, B, T, E = logits.shape
        self.loss = logits.new_empty((L, 2), dtype=_F32)                             # [balance, z-loss] of every layer
        self.counts = logits.new_empty((L, B, E) if scope == ROUTER_SEQUENCE else (L, E), dtype=torch.int32)
        self.dlogits = logits if in_place else _like(logits)
        self.ids = logits.new_empty((L, B, T, max(k, 0)), dtype=torch.int32) if want_ids else None


def router_loss_fwd_bwd(logits: torch.Tensor, lengths: torch.Tensor, k: int, scoring: int, scope: int, balance_coef: float,
                        z_coef: float, grad_scale: float, ws: torch.Tensor, expert_ids: Optional[torch.Tensor] = None,
                        out: Optional[RouterOutputs] = None) -> RouterOutputs:
    """rlhf_router_loss_fwd_bwd on [L,B,T,E] router logits (bf16, fp16 or fp32).  The k experts of a token are `expert_ids`
    ([L,B,T,k] int32, -1: none) or, without them, its k largest logits, which `out.ids` then holds; `scoring` is ROUTER_SOFTMAX or
    ROUTER_SIGMOID, `scope` ROUTER_BATCH or ROUTER_SEQUENCE."""
    if logits.dtype not in SHAPED_DTYPES or not logits.is_cuda or logits.dim() != 4:
        _router_logits(logits)
    L, B, T, E = logits.shape
    sl, sb, st, se = logits.stride()
    if se != 1 and E > 1:
        _router_logits(logits)
    dev = logits.get_device()
    if out is None:
        out = RouterOutputs(logits, k, scope, want_ids=expert_ids is None)
    d = out.dlogits
    if d.dtype is not logits.dtype:
        raise TypeError("out.dlogits must have the element type of logits")
    dl, db, dt, de = d.stride()
    if d.shape != logits.shape or (E > 1 and de != 1):
        raise ValueError("out.dlogits must have the shape of logits and a contiguous expert axis")
    _same_device(d, dev, "out.dlogits")
    given, gl, gb, gt = None, 0, 0, 0
    if expert_ids is not None:
        _dev(expert_ids, torch.int32, "expert_ids")
        _same_device(expert_ids, dev, "expert_ids")
        if expert_ids.shape != (L, B, T, k) or (k > 1 and expert_ids.stride(3) != 1):
            raise ValueError(f"expert_ids must be [{L},{B},{T},{k}] with a contiguous last axis")
        given = expert_ids.data_ptr()
        gl, gb, gt, _ = expert_ids.stride()
    _call("rlhf_router_loss_fwd_bwd", dev, logits.data_ptr(), SHAPED_DTYPES[logits.dtype], sl, sb, st, given, gl, gb, gt,
          _arg(lengths, (B,), torch.int32, dev, "lengths"), L, B, T, E, k, scoring, scope, balance_coef, z_coef, grad_scale,
          _arg(out.loss, (L, 2), _F32, dev, "out.loss"),
          _arg(out.counts, (L, B, E) if scope == ROUTER_SEQUENCE else (L, E), torch.int32, dev, "out.counts"),
          _opt(out.ids, (L, B, T, k), torch.int32, dev, "out.ids"), d.data_ptr(), dl, db, dt, *_ws(ws, dev))
    return out
