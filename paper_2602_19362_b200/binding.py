"""ctypes binding of liboapl.so: same names as the C entry points, argument
marshalling only.  Tensors are torch CUDA tensors used as device memory; every
step of the path runs in the library's kernels.  There is no fallback: a missing
library raises at first use.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liboapl.so")

OAPL_OK = 0
STATUS = {0: "OK", -1: "INVALID_ARG", -2: "MISALIGNED", -3: "WORKSPACE_TOO_SMALL",
          -4: "UNSUPPORTED_SHAPE", -5: "BAD_TARGET", -6: "BAD_SEQ_ORDER", -7: "NONFINITE_INPUT",
          -8: "DEVICE_TIMEOUT", -9: "CUDA", -10: "BAD_STATE", -11: "SEQUENCE_TOO_LONG", -12: "OUT_OF_RANGE",
          -13: "BOUND_EXCEEDED"}
OAPL_FLAG_FUSED = 1

EXPORTS = ["oapl_workspace_bytes", "oapl_token_logprobs", "oapl_value_estimate", "oapl_loss_fwd",
           "oapl_loss_bwd", "oapl_get_last_status", "oapl_get_live_rows", "oapl_launch_count",
           "oapl_status_string", "oapl_debug_gemm", "oapl_profile_enable", "oapl_profile_read",
           "oapl_token_logprobs_static", "oapl_loss_fwd_bwd", "oapl_profile_read_clocks", "oapl_entropy", "oapl_group_advantage",
           "oapl_grpo_loss_fwd_bwd", "oapl_adamw_workspace_bytes", "oapl_adamw_step", "oapl_loss_fwd_bwd_ex",
           "oapl_get_range_count", "oapl_profile_applies", "oapl_range_slots", "oapl_batch_stats",
           "oapl_logits_logprobs", "oapl_logits_logprobs_bwd", "oapl_quantize", "oapl_scaled_matmul",
           "oapl_debug_scaled_matmul", "oapl_embedding", "oapl_embedding_workspace_bytes", "oapl_embedding_bwd",
           "oapl_residual_norm", "oapl_residual_norm_workspace_bytes", "oapl_residual_norm_bwd",
           "oapl_grad_norm_workspace_bytes", "oapl_grad_norm", "oapl_grad_clip", "oapl_grad_clip_ex",
           "oapl_logits_adjust", "oapl_logits_adjust_bwd"]


class OaplProblem(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("d", ctypes.c_int32), ("V", ctypes.c_int32),
                ("S", ctypes.c_int32), ("P", ctypes.c_int32),
                ("H", ctypes.c_void_p), ("W", ctypes.c_void_p), ("targets", ctypes.c_void_p),
                ("mask", ctypes.c_void_p), ("seq_id", ctypes.c_void_p), ("group_id", ctypes.c_void_p),
                ("reward", ctypes.c_void_p), ("logp_inf", ctypes.c_void_p),
                ("beta_v", ctypes.c_float), ("beta_loss", ctypes.c_float), ("loss_scale", ctypes.c_float)]


class OaplCallOptions(ctypes.Structure):
    _fields_ = [("live_rows_bound", ctypes.c_int64), ("max_seq_rows_bound", ctypes.c_int32),
                ("dW_ready_event", ctypes.c_void_p)]


class OaplLogits(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("N", ctypes.c_int64), ("ld", ctypes.c_int64), ("V", ctypes.c_int32),
                ("type", ctypes.c_int32), ("targets", ctypes.c_void_p), ("mask", ctypes.c_void_p),
                ("scale", ctypes.c_float)]


class OaplScaled(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld", ctypes.c_int64), ("scale_row_stride", ctypes.c_int64),
                ("scale_col_stride", ctypes.c_int64), ("type", ctypes.c_int32), ("block_rows", ctypes.c_int32)]


class OaplLookup(ctypes.Structure):
    _fields_ = [("ids", ctypes.c_void_p), ("mask", ctypes.c_void_p), ("N", ctypes.c_int64), ("V", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class OaplResidual(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("d", ctypes.c_int32), ("type", ctypes.c_int32), ("x", ctypes.c_void_p),
                ("ld_x", ctypes.c_int64), ("y", ctypes.c_void_p), ("ld_y", ctypes.c_int64), ("gate", ctypes.c_void_p),
                ("ld_gate", ctypes.c_int64), ("gate_kind", ctypes.c_int32), ("gate_type", ctypes.c_int32),
                ("w_post", ctypes.c_void_p), ("w_pre", ctypes.c_void_p), ("weight_type", ctypes.c_int32),
                ("weight_offset", ctypes.c_float), ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
                ("branch_scale", ctypes.c_float)]


class OaplTensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("type", ctypes.c_int32),
                ("out_type", ctypes.c_int32)]


class OaplAdjust(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_void_p), ("T", ctypes.c_int64), ("spans", ctypes.c_void_p),
                ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p),
                ("bias_start", ctypes.c_void_p), ("bias_id", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("biases", ctypes.c_int64), ("allowed", ctypes.c_void_p), ("ld_allowed", ctypes.c_int64),
                ("allowed_rows", ctypes.c_int64), ("allowed_row", ctypes.c_void_p)]


class OaplError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)} ({lib().oapl_status_string(status).decode()})")


_lib = None


def lib() -> ctypes.CDLL:
    """Load liboapl.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2602_19362_b200.build` "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        pp = ctypes.POINTER(OaplProblem)
        L.oapl_workspace_bytes.restype = sz
        L.oapl_workspace_bytes.argtypes = [pp, i32]
        L.oapl_token_logprobs.restype = i32
        L.oapl_token_logprobs.argtypes = [pp, vp, vp, vp, sz, i32, vp]
        L.oapl_value_estimate.restype = i32
        L.oapl_value_estimate.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, f32, vp, vp]
        L.oapl_loss_fwd.restype = i32
        L.oapl_loss_fwd.argtypes = [pp, vp, vp, vp, vp, vp, vp, sz, i32, vp]
        L.oapl_loss_bwd.restype = i32
        L.oapl_loss_bwd.argtypes = [pp, vp, vp, i32, vp, sz, i32, vp]
        L.oapl_get_last_status.restype = i32
        L.oapl_get_last_status.argtypes = [vp, vp]
        L.oapl_get_live_rows.restype = i64
        L.oapl_get_live_rows.argtypes = [vp, vp]
        L.oapl_launch_count.restype = ctypes.c_uint64
        L.oapl_launch_count.argtypes = []
        L.oapl_status_string.restype = ctypes.c_char_p
        L.oapl_status_string.argtypes = [i32]
        L.oapl_debug_gemm.restype = i32
        L.oapl_debug_gemm.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, ctypes.c_longlong, i32, vp, vp]
        L.oapl_loss_fwd_bwd_ex.restype = i32
        L.oapl_loss_fwd_bwd_ex.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, i32,
                                           ctypes.POINTER(OaplCallOptions), vp]
        L.oapl_get_range_count.restype = i32
        L.oapl_get_range_count.argtypes = [vp, vp]
        L.oapl_batch_stats.restype = i32
        L.oapl_batch_stats.argtypes = [pp, vp, vp, vp, sz, i32, vp]
        L.oapl_range_slots.restype = i32
        L.oapl_range_slots.argtypes = [i64, i64, ctypes.c_int32, ctypes.c_int32]
        L.oapl_profile_applies.restype = i32
        L.oapl_profile_applies.argtypes = [i32, i32]
        L.oapl_loss_fwd_bwd.restype = i32
        L.oapl_loss_fwd_bwd.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, i32, vp]
        L.oapl_token_logprobs_static.restype = i32
        L.oapl_token_logprobs_static.argtypes = [pp, vp, vp, vp, vp]
        L.oapl_group_advantage.restype = i32
        L.oapl_group_advantage.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, f32, vp, vp]
        L.oapl_grpo_loss_fwd_bwd.restype = i32
        L.oapl_grpo_loss_fwd_bwd.argtypes = [pp, vp, vp, f32, vp, vp, vp, vp, vp, vp, i32, vp, sz, i32, vp]
        L.oapl_adamw_workspace_bytes.restype = sz
        L.oapl_adamw_workspace_bytes.argtypes = []
        L.oapl_adamw_step.restype = i32
        L.oapl_adamw_step.argtypes = [vp, vp, vp, vp, vp, i64, i64, f32, f32, f32, f32, f32, f32, vp, vp, vp, sz, vp]
        L.oapl_entropy.restype = i32
        L.oapl_entropy.argtypes = [pp, vp, vp, vp, vp, sz, i32, vp]
        pl, ps = ctypes.POINTER(OaplLogits), ctypes.POINTER(OaplScaled)
        L.oapl_logits_logprobs.restype = i32
        L.oapl_logits_logprobs.argtypes = [pl, vp, vp, vp, ctypes.c_int32, vp, vp, vp, vp]
        L.oapl_logits_logprobs_bwd.restype = i32
        L.oapl_logits_logprobs_bwd.argtypes = [pl, vp, vp, vp, vp, ctypes.c_int32, vp, vp, vp, i64, vp]
        L.oapl_quantize.restype = i32
        L.oapl_quantize.argtypes = [vp, ctypes.c_int32, i64, i64, i64, ps, i32, vp]
        L.oapl_scaled_matmul.restype = i32
        L.oapl_scaled_matmul.argtypes = [ps, ps, vp, ctypes.c_int32, i64, i32, vp, vp]
        L.oapl_debug_scaled_matmul.restype = i32
        L.oapl_debug_scaled_matmul.argtypes = [ps, ps, vp, ctypes.c_int32, i64, i32, vp, ctypes.c_longlong, i32, vp]
        pk, pr, pt, pa = (ctypes.POINTER(t) for t in (OaplLookup, OaplResidual, OaplTensor, OaplAdjust))
        c32 = ctypes.c_int32
        L.oapl_embedding.restype = i32
        L.oapl_embedding.argtypes = [pk, vp, c32, i64, c32, vp, c32, i64, vp, vp]
        L.oapl_embedding_workspace_bytes.restype = sz
        L.oapl_embedding_workspace_bytes.argtypes = [i64, c32, c32]
        L.oapl_embedding_bwd.restype = i32
        L.oapl_embedding_bwd.argtypes = [pk, vp, c32, i64, c32, vp, i64, i32, vp, vp, sz, vp]
        L.oapl_residual_norm.restype = i32
        L.oapl_residual_norm.argtypes = [pr, vp, i64, vp, i64, vp, vp, vp]
        L.oapl_residual_norm_workspace_bytes.restype = sz
        L.oapl_residual_norm_workspace_bytes.argtypes = [i64, c32]
        L.oapl_residual_norm_bwd.restype = i32
        L.oapl_residual_norm_bwd.argtypes = [pr, vp, i64, vp, vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp,
                                             i32, vp, sz, vp]
        L.oapl_grad_norm_workspace_bytes.restype = sz
        L.oapl_grad_norm_workspace_bytes.argtypes = [c32]
        L.oapl_grad_norm.restype = i32
        L.oapl_grad_norm.argtypes = [pt, c32, f32, vp, vp, vp, vp, sz, vp]
        L.oapl_grad_clip.restype = i32
        L.oapl_grad_clip.argtypes = [pt, c32, f32, vp, f32, vp]
        L.oapl_grad_clip_ex.restype = i32
        L.oapl_grad_clip_ex.argtypes = [pt, c32, f32, vp, vp, f32, vp]
        L.oapl_logits_adjust.restype = i32
        L.oapl_logits_adjust.argtypes = [pl, pa, vp, i64, vp, vp]
        L.oapl_logits_adjust_bwd.restype = i32
        L.oapl_logits_adjust_bwd.argtypes = [pl, pa, vp, i64, vp, i64, vp, vp]
        L.oapl_profile_enable.restype = i32
        L.oapl_profile_enable.argtypes = [i32]
        L.oapl_profile_read.restype = i32
        L.oapl_profile_read.argtypes = [vp, vp, i32, vp]
        L.oapl_profile_read_clocks.restype = i32
        L.oapl_profile_read_clocks.argtypes = [vp, i32]
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check_dev(t, dtype, name):
    if t is None:
        return
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous CUDA tensor of {dtype}")


def make_problem(batch: dict, beta_v=None, beta_loss=None, loss_scale=None) -> OaplProblem:
    """Fill the C struct from a batch dict (see synth.make_batch).  The dict's
    tensors must stay alive while the struct is in use."""
    _check_dev(batch["H"], torch.bfloat16, "H")
    _check_dev(batch["W"], torch.bfloat16, "W")
    _check_dev(batch["targets"], torch.int32, "targets")
    _check_dev(batch["mask"], torch.uint8, "mask")
    _check_dev(batch["seq_id"], torch.int32, "seq_id")
    _check_dev(batch.get("group_id"), torch.int32, "group_id")
    _check_dev(batch.get("reward"), torch.float32, "reward")
    _check_dev(batch.get("logp_inf"), torch.float32, "logp_inf")
    p = OaplProblem()
    p.N, p.d, p.V, p.S, p.P = batch["N"], batch["d"], batch["V"], batch["S"], batch["P"]
    p.H, p.W = batch["H"].data_ptr(), batch["W"].data_ptr()
    p.targets, p.mask, p.seq_id = batch["targets"].data_ptr(), batch["mask"].data_ptr(), batch["seq_id"].data_ptr()
    for k in ("group_id", "reward", "logp_inf"):
        t = batch.get(k)
        setattr(p, k, None if t is None else t.data_ptr())
    p.beta_v = batch.get("beta_v", 1.0) if beta_v is None else beta_v
    p.beta_loss = batch.get("beta_loss", 1.0) if beta_loss is None else beta_loss
    p.loss_scale = batch.get("loss_scale", 1.0) if loss_scale is None else loss_scale
    return p


def oapl_workspace_bytes(problem: OaplProblem, flags: int = 0) -> int:
    return int(lib().oapl_workspace_bytes(ctypes.byref(problem), flags))


def alloc_workspace(problem: OaplProblem, flags: int = 0, device="cuda") -> torch.Tensor:
    n = oapl_workspace_bytes(problem, flags)
    if n == 0:
        raise OaplError(-1, "oapl_workspace_bytes")
    ws = torch.empty(n + 1024, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 1024
    return ws[off:off + n]


def oapl_token_logprobs(problem, token_logp, seq_logp, ws, flags=0):
    rc = lib().oapl_token_logprobs(ctypes.byref(problem), _ptr(token_logp), _ptr(seq_logp), _ptr(ws),
                                   ws.numel(), flags, _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_token_logprobs")


def oapl_value_estimate(reward, group_id, P, beta_v, vhat):
    rc = lib().oapl_value_estimate(_ptr(reward), _ptr(group_id), reward.numel(), P, beta_v, _ptr(vhat), _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_value_estimate")


def oapl_loss_fwd(problem, loss, seq_logp, vhat, delta, token_logp, ws, flags=0):
    rc = lib().oapl_loss_fwd(ctypes.byref(problem), _ptr(loss), _ptr(seq_logp), _ptr(vhat), _ptr(delta),
                             _ptr(token_logp), _ptr(ws), ws.numel(), flags, _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_loss_fwd")


def oapl_loss_bwd(problem, dH, dW, accumulate_dW, ws, flags=0):
    rc = lib().oapl_loss_bwd(ctypes.byref(problem), _ptr(dH), _ptr(dW), int(accumulate_dW), _ptr(ws),
                             ws.numel(), flags, _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_loss_bwd")


def oapl_group_advantage(reward, group_id, P, eps, advantage):
    rc = lib().oapl_group_advantage(_ptr(reward), _ptr(group_id), reward.numel(), P, eps, _ptr(advantage),
                                    _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_group_advantage")


def oapl_grpo_loss_fwd_bwd(problem, logp_old, advantage, clip_eps, loss, seq_logp, token_logp, clip_frac, dH, dW,
                           accumulate_dW, ws, flags=0):
    rc = lib().oapl_grpo_loss_fwd_bwd(ctypes.byref(problem), _ptr(logp_old), _ptr(advantage), clip_eps,
                                      _ptr(loss), _ptr(seq_logp), _ptr(token_logp), _ptr(clip_frac), _ptr(dH),
                                      _ptr(dW), int(accumulate_dW), _ptr(ws), ws.numel(), flags, _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_grpo_loss_fwd_bwd")


def oapl_adamw_step(W, master, dW, m, v, step, lr, beta1, beta2, eps, weight_decay, clip_norm,
                    other_sq_norm=None, grad_norm=None, ws=None):
    if ws is None:
        ws = torch.empty(int(lib().oapl_adamw_workspace_bytes()), dtype=torch.uint8, device=W.device)
    rc = lib().oapl_adamw_step(_ptr(W), _ptr(master), _ptr(dW), _ptr(m), _ptr(v), W.numel(), int(step), lr, beta1,
                               beta2, eps, weight_decay, clip_norm, _ptr(other_sq_norm), _ptr(grad_norm), _ptr(ws),
                               ws.numel(), _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_adamw_step")
    return ws


def oapl_entropy(problem, token_entropy, seq_entropy, mean_entropy, ws, flags=0):
    rc = lib().oapl_entropy(ctypes.byref(problem), _ptr(token_entropy), _ptr(seq_entropy), _ptr(mean_entropy),
                            _ptr(ws), ws.numel(), flags, _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_entropy")


STATS = ("live_tokens", "mean_abs_log_ratio", "max_abs_log_ratio", "mean_token_log_ratio", "mean_advantage",
         "frac_groups_all_equal", "mean_reward")


def oapl_batch_stats(problem, vhat, stats, ws, flags=0):
    rc = lib().oapl_batch_stats(ctypes.byref(problem), _ptr(vhat), _ptr(stats), _ptr(ws), ws.numel(), flags,
                                _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_batch_stats")


def oapl_get_last_status(ws) -> int:
    return int(lib().oapl_get_last_status(_ptr(ws), _stream()))


def oapl_get_live_rows(ws) -> int:
    return int(lib().oapl_get_live_rows(_ptr(ws), _stream()))


def oapl_launch_count() -> int:
    return int(lib().oapl_launch_count())


def oapl_debug_gemm(A, B, C, M, N, K, a_mn, b_mn, err, wide=False, wait_cycles=0, skip_step=0):
    if err is None or err.numel() < 2 or err.dtype != torch.int32:
        raise TypeError("err: int32 CUDA tensor of two elements (status word, lock-step counter)")
    rc = lib().oapl_debug_gemm(_ptr(A), _ptr(B), _ptr(C), M, N, K, int(a_mn), int(b_mn), int(wide),
                               int(wait_cycles), int(skip_step), _ptr(err), _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_debug_gemm")


KINDS = ("lse_fwd", "grad_chunk", "dH", "dW", "debug", "lse_e")


def oapl_profile_enable(on: bool):
    rc = lib().oapl_profile_enable(int(on))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_profile_enable")


def oapl_profile_read(with_dropped: bool = False):
    """{kind: (milliseconds, launches)} since the last read; with_dropped=True also returns the
    number of launches that were not recorded."""
    ms = (ctypes.c_float * len(KINDS))()
    cnt = (ctypes.c_int * len(KINDS))()
    dropped = ctypes.c_int(0)
    rc = lib().oapl_profile_read(ms, cnt, len(KINDS), ctypes.byref(dropped))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_profile_read")
    out = {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(KINDS)}
    return (out, int(dropped.value)) if with_dropped else out


def oapl_profile_read_clocks() -> dict:
    """{kind: SM MHz the kind's launches ran at} since the last read (0 = did not run)."""
    mhz = (ctypes.c_float * len(KINDS))()
    rc = lib().oapl_profile_read_clocks(mhz, len(KINDS))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_profile_read_clocks")
    return {k: float(mhz[i]) for i, k in enumerate(KINDS)}


def oapl_token_logprobs_static(problem, token_logp, seq_logp, device_status=None):
    """oapl_token_logprobs without a workspace: the scratch is a fixed array inside the
    library, for callers that must not allocate (N <= 2048, d <= 1024, S <= 2048)."""
    rc = lib().oapl_token_logprobs_static(ctypes.byref(problem), _ptr(token_logp), _ptr(seq_logp),
                                          _ptr(device_status), _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_token_logprobs_static")


def make_options(live_rows_bound: int = 0, max_seq_rows_bound: int = 0, dW_ready_event=None) -> OaplCallOptions:
    """Fill oapl_call_options.  dW_ready_event is a torch.cuda.Event that has been recorded at
    least once (torch creates the underlying CUDA event at the first record) or None."""
    o = OaplCallOptions()
    o.live_rows_bound = int(live_rows_bound)
    o.max_seq_rows_bound = int(max_seq_rows_bound)
    if dW_ready_event is None:
        o.dW_ready_event = None
    else:
        handle = int(dW_ready_event.cuda_event)
        if handle == 0:
            raise ValueError("dW_ready_event: record the torch.cuda.Event once before passing it")
        o.dW_ready_event = handle
    return o


def oapl_loss_fwd_bwd_ex(problem, loss, seq_logp, vhat, delta, token_logp, dH, dW, accumulate_dW, ws, options,
                         flags=0):
    rc = lib().oapl_loss_fwd_bwd_ex(ctypes.byref(problem), _ptr(loss), _ptr(seq_logp), _ptr(vhat), _ptr(delta),
                                    _ptr(token_logp), _ptr(dH), _ptr(dW), int(accumulate_dW), _ptr(ws),
                                    ws.numel(), flags, ctypes.byref(options) if options is not None else None,
                                    _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_loss_fwd_bwd_ex")


def oapl_get_range_count(ws) -> int:
    return int(lib().oapl_get_range_count(_ptr(ws), _stream()))


def oapl_loss_fwd_bwd(problem, loss, seq_logp, vhat, delta, token_logp, dH, dW, accumulate_dW, ws, flags=0):
    rc = lib().oapl_loss_fwd_bwd(ctypes.byref(problem), _ptr(loss), _ptr(seq_logp), _ptr(vhat), _ptr(delta),
                                 _ptr(token_logp), _ptr(dH), _ptr(dW), int(accumulate_dW), _ptr(ws),
                                 ws.numel(), flags, _stream())
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_loss_fwd_bwd")


# ---- logits in memory, and 8-bit matrices with a scale per block -----------------------------------

OAPL_QUANT_TRANSPOSE, OAPL_QUANT_POW2 = 1, 2
FLOAT_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
SCALED_TYPES = {torch.float8_e4m3fn: 3, torch.float8_e5m2: 4}
MAX_TOP = 32


def _rows(t, types, name):
    """Check a [rows, cols] CUDA tensor with contiguous rows: its type code, rows, cols and leading dimension."""
    code = types.get(t.dtype)
    if code is None or t.dim() != 2 or not t.is_cuda:
        raise TypeError(f"{name}: expected a 2-D CUDA tensor of one of {[str(x) for x in types]}")
    (rows, cols), (ld, step) = t.shape, t.stride()
    if step != 1 and cols > 1:
        raise TypeError(f"{name}: elements of a row must be contiguous")
    return code, rows, cols, (ld if rows > 1 else max(ld, cols))


def _vec(t, dtype, shape, device, name):
    """Address of a contiguous tensor of that type, shape and device; None for None."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
        raise TypeError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{device}")
    return t.data_ptr()


def _stream_of(device):
    """The current stream of `device`, which has to be the current device."""
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"the tensors are on cuda:{device}, the current device is cuda:{torch.cuda.current_device()}")
    return torch._C._cuda_getCurrentRawStream(device)


def make_logits(logits, targets=None, mask=None, scale: float = 1.0) -> OaplLogits:
    """Fill oapl_logits.  logits: [N, V] bf16, fp16 or fp32, rows any stride apart; targets: int32 [N];
    mask: uint8 [N].  The struct keeps the tensors alive."""
    code, N, V, ld = _rows(logits, FLOAT_TYPES, "logits")
    dev = logits.get_device()
    L = OaplLogits(logits.data_ptr(), N, ld, V, code, _vec(targets, torch.int32, (N,), dev, "targets"),
                   _vec(mask, torch.uint8, (N,), dev, "mask"), scale)
    L.tensors, L.device = (logits, targets, mask), dev
    return L


def oapl_logits_logprobs(L, token_logp=None, token_entropy=None, token_lse=None, top_logp=None, top_id=None,
                         device_status=None):
    """Log-probability of the targets, entropy, log-sum-exp [N] and the top K alternatives [N, K]; each
    output may be None.  device_status: int32 [1], zero before the call."""
    dev, N = L.device, L.N
    first = top_id if top_id is not None else top_logp
    K = 0 if first is None else first.shape[-1]
    f32 = torch.float32
    rc = lib().oapl_logits_logprobs(
        L, _vec(token_logp, f32, (N,), dev, "token_logp"), _vec(token_entropy, f32, (N,), dev, "token_entropy"),
        _vec(token_lse, f32, (N,), dev, "token_lse"), K, _vec(top_logp, f32, (N, K), dev, "top_logp"),
        _vec(top_id, torch.int32, (N, K), dev, "top_id"), _vec(device_status, torch.int32, (1,), dev, "device_status"),
        _stream_of(dev))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_logits_logprobs")


def oapl_logits_logprobs_bwd(L, token_lse, token_entropy, g_logp, g_entropy, g_top, top_id, dlogits):
    """Gradient of the logits from the gradients of token_logp, token_entropy (each [N] or None) and of the
    log-probabilities of the ids top_id ([N, K] or None).  dlogits may be the logits themselves."""
    dev, N = L.device, L.N
    K = 0 if g_top is None else g_top.shape[-1]
    f32 = torch.float32
    code, rows, cols, ld_d = _rows(dlogits, FLOAT_TYPES, "dlogits")
    if code != L.type or rows != N or cols != L.V or dlogits.get_device() != dev:
        raise TypeError("dlogits: expected the logits' type, shape and device")
    rc = lib().oapl_logits_logprobs_bwd(
        L, _vec(token_lse, f32, (N,), dev, "token_lse"), _vec(token_entropy, f32, (N,), dev, "token_entropy"),
        _vec(g_logp, f32, (N,), dev, "g_logp"), _vec(g_entropy, f32, (N,), dev, "g_entropy"), K,
        _vec(g_top, f32, (N, K), dev, "g_top"), _vec(top_id, torch.int32, (N, K), dev, "top_id") if K else None,
        dlogits.data_ptr(), ld_d, _stream_of(dev))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_logits_logprobs_bwd")


def make_scaled(data, scale, block_rows: int) -> OaplScaled:
    """Fill oapl_scaled.  data: [rows, cols] float8_e4m3fn or float8_e5m2, rows a multiple of 16 bytes apart;
    scale: fp32 [ceil(rows / block_rows), ceil(cols / 128)] of any strides; block_rows 1 or 128.  The struct
    keeps the tensors alive."""
    code, rows, cols, ld = _rows(data, SCALED_TYPES, "data")
    if rows == 1:
        ld = -(-ld // 16) * 16      # one row: no second one to find
    if block_rows != 1 and block_rows != 128:
        raise ValueError("block_rows: 1 or 128")
    dev = data.get_device()
    if (scale.dtype != torch.float32 or scale.shape != ((rows + block_rows - 1) // block_rows, (cols + 127) // 128)
            or scale.get_device() != dev):
        raise TypeError("scale: expected fp32 [ceil(rows / block_rows), ceil(cols / 128)] on the data's device")
    m = OaplScaled(data.data_ptr(), scale.data_ptr(), rows, cols, ld, *scale.stride(), code, block_rows)
    m.tensors, m.device = (data, scale), dev
    return m


def alloc_scaled(rows: int, cols: int, block_rows: int, dtype=torch.float8_e4m3fn, device="cuda") -> OaplScaled:
    """An oapl_scaled with uninitialised memory laid out for the product: padded rows, and the scales of a
    block of 128 columns next to one another.  Its tensors are `.tensors` = (data, scale)."""
    data = torch.empty(rows, -(-cols // 16) * 16, dtype=dtype, device=device)[:, :cols]
    scale = torch.empty(-(-cols // 128), -(-rows // block_rows), dtype=torch.float32, device=device).t()
    return make_scaled(data, scale, block_rows)


def oapl_quantize(x, out: OaplScaled, transpose: bool = False, pow2: bool = False):
    """Quantise x [rows, cols] (bf16, fp16, fp32) into `out`, turned when transpose is set."""
    code, rows, cols, ld = _rows(x, FLOAT_TYPES, "x")
    if x.get_device() != out.device:
        raise TypeError("out: expected x's device")
    rc = lib().oapl_quantize(x.data_ptr(), code, rows, cols, ld, out,
                             (OAPL_QUANT_TRANSPOSE if transpose else 0) | (OAPL_QUANT_POW2 if pow2 else 0),
                             _stream_of(out.device))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_quantize")


def _product_args(A, B, C, accumulate, device_status):
    code, rows, cols, ldc = _rows(C, FLOAT_TYPES, "C")
    if rows != A.rows or cols != B.rows:
        raise TypeError(f"C: expected shape {(A.rows, B.rows)}")
    dev = C.get_device()
    if A.device != dev or B.device != dev:
        raise TypeError("A, B: expected C's device")
    return A, B, C.data_ptr(), code, ldc, accumulate, _vec(device_status, torch.int32, (1,), dev, "device_status")


def oapl_scaled_matmul(A: OaplScaled, B: OaplScaled, C, accumulate: bool = False, device_status=None):
    """C [A.rows, B.rows] (bf16, fp16, fp32) = A . B^T, or C += A . B^T.  NaN where a pipeline wait ran out, and
    OAPL_ERR_DEVICE_TIMEOUT in device_status (int32 [1], zero before the call)."""
    rc = lib().oapl_scaled_matmul(*_product_args(A, B, C, accumulate, device_status), _stream_of(C.get_device()))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_scaled_matmul")


def oapl_debug_scaled_matmul(A: OaplScaled, B: OaplScaled, C, device_status, accumulate: bool = False, wait_cycles=0,
                             skip_step=0):
    rc = lib().oapl_debug_scaled_matmul(*_product_args(A, B, C, accumulate, device_status), int(wait_cycles),
                                        int(skip_step), _stream_of(C.get_device()))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_debug_scaled_matmul")


# ---- the embedding, the norms around a block, the gradient norm, adjustments of logits ---------------------

OAPL_GATE_NONE, OAPL_GATE_ROW, OAPL_GATE_COLUMN, OAPL_GATE_FULL = 0, 1, 2, 3


def _ws(ws, device):
    """Address and size of a workspace: a contiguous uint8 tensor of that device, or None."""
    if ws is None:
        return None, 0
    if ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.get_device() != device:
        raise TypeError(f"ws: expected a contiguous uint8 tensor on cuda:{device}")
    return ws.data_ptr(), ws.numel()


def make_lookup(ids, V: int, mask=None, scale: float = 1.0) -> OaplLookup:
    """Fill oapl_lookup.  ids: int32 [N]; mask: uint8 [N].  The struct keeps the tensors alive."""
    if not ids.is_cuda or ids.dim() != 1:
        raise TypeError("ids: expected a 1-D CUDA tensor")
    dev, N = ids.get_device(), ids.shape[0]
    k = OaplLookup(_vec(ids, torch.int32, (N,), dev, "ids"), _vec(mask, torch.uint8, (N,), dev, "mask"), N, V, scale)
    k.tensors, k.device = (ids, mask), dev
    return k


def oapl_embedding(k: OaplLookup, table, out, device_status=None):
    """out [N, d] = scale * table[ids]; table [V, d]; each bf16, fp16 or fp32, rows any stride apart."""
    dev = k.device
    ct, V, d, ld_t = _rows(table, FLOAT_TYPES, "table")
    co, N, do, ld_o = _rows(out, FLOAT_TYPES, "out")
    if V != k.V or N != k.N or d != do or table.get_device() != dev or out.get_device() != dev:
        raise TypeError(f"table, out: expected shapes {(k.V, d)} and {(k.N, d)} on cuda:{dev}")
    rc = lib().oapl_embedding(k, table.data_ptr(), ct, ld_t, d, out.data_ptr(), co, ld_o,
                              _vec(device_status, torch.int32, (1,), dev, "device_status"), _stream_of(dev))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_embedding")


def oapl_embedding_workspace_bytes(N: int, V: int, d: int) -> int:
    return int(lib().oapl_embedding_workspace_bytes(N, V, d))


def oapl_embedding_bwd(k: OaplLookup, dout, dtable, accumulate: bool, ws, device_status=None):
    """dtable [V, d] fp32 = (or +=) scale * the rows of dout [N, d] added up by token.  ws: uint8,
    oapl_embedding_workspace_bytes(N, V, d)."""
    dev = k.device
    ct, N, d, ld = _rows(dout, FLOAT_TYPES, "dout")
    c32, V, dt, ld_t = _rows(dtable, FLOAT_TYPES, "dtable")
    if V != k.V or N != k.N or d != dt or c32 != 2 or dout.get_device() != dev or dtable.get_device() != dev:
        raise TypeError(f"dout, dtable: expected shapes {(k.N, d)} and {(k.V, d)}, the latter fp32, on cuda:{dev}")
    at, size = _ws(ws, dev)
    rc = lib().oapl_embedding_bwd(k, dout.data_ptr(), ct, ld, d, dtable.data_ptr(), ld_t, int(accumulate),
                                  _vec(device_status, torch.int32, (1,), dev, "device_status"), at, size, _stream_of(dev))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_embedding_bwd")


def make_residual(x, y=None, gate=None, w_post=None, w_pre=None, eps: float = 1e-6, residual_scale: float = 1.0,
                  branch_scale: float = 1.0, weight_offset: float = 0.0) -> OaplResidual:
    """Fill oapl_residual.  x, y: [N, d] of one type; gate: [N, 1] a factor per row, [d] one per channel, [N, d] one per
    element (of x's type); w_post, w_pre: [d] of one type.  The struct keeps the tensors alive."""
    code, N, d, ld_x = _rows(x, FLOAT_TYPES, "x")
    dev, ld_y, at_y = x.get_device(), 0, None
    if y is not None:
        cy, ny, dy, ld_y = _rows(y, FLOAT_TYPES, "y")
        if cy != code or ny != N or dy != d or y.get_device() != dev:
            raise TypeError("y: expected x's type, shape and device")
        at_y = y.data_ptr()
    kind = gate_type = ld_gate = 0
    at_gate = None
    if gate is not None:
        gate_type = FLOAT_TYPES.get(gate.dtype)
        if gate_type is None or gate.get_device() != dev:
            raise TypeError("gate: expected bf16, fp16 or fp32 on x's device")
        if gate.dim() == 1 and gate.shape[0] == d and gate.is_contiguous():
            kind = OAPL_GATE_COLUMN
        elif gate.dim() == 2 and gate.shape == (N, d) and (d > 1 or gate_type == code):
            kind, ld_gate = OAPL_GATE_FULL, _rows(gate, {x.dtype: code}, "gate")[3]
        elif gate.dim() == 2 and gate.shape == (N, 1):
            kind, ld_gate = OAPL_GATE_ROW, (gate.stride(0) if N > 1 else 1)
        else:
            raise TypeError("gate: expected [N, 1], a contiguous [d], or [N, d]")
        at_gate = gate.data_ptr()
    weight = w_pre if w_pre is not None else w_post
    weight_type = 0
    if weight is not None:
        weight_type = FLOAT_TYPES.get(weight.dtype)
        if weight_type is None:
            raise TypeError("w_post, w_pre: expected bf16, fp16 or fp32")
    r = OaplResidual(N, d, code, x.data_ptr(), ld_x, at_y, ld_y, at_gate, ld_gate, kind, gate_type,
                     None if w_post is None else _vec(w_post, weight.dtype, (d,), dev, "w_post"),
                     None if w_pre is None else _vec(w_pre, weight.dtype, (d,), dev, "w_pre"), weight_type, weight_offset,
                     eps, residual_scale, branch_scale)
    r.tensors, r.device = (x, y, gate, w_post, w_pre), dev
    return r


def _like(r, t, name):
    """Address and leading dimension of a matrix of the residual's type, shape and device; None and 0 for None."""
    if t is None:
        return None, 0
    code, N, d, ld = _rows(t, FLOAT_TYPES, name)
    if code != r.type or N != r.N or d != r.d or t.get_device() != r.device:
        raise TypeError(f"{name}: expected x's type, shape and device")
    return t.data_ptr(), ld


def oapl_residual_norm(r: OaplResidual, x_out, h=None, rstd_post=None, rstd_pre=None):
    """x_out [N, d] = residual_scale x + branch_scale gate norm(y), h [N, d] = norm(x_out); rstd_post, rstd_pre: fp32
    [N], what the gradient reads.  x_out and h may be x, y or a full gate."""
    dev, N = r.device, r.N
    f32 = torch.float32
    rc = lib().oapl_residual_norm(r, *_like(r, x_out, "x_out"), *_like(r, h, "h"),
                                  _vec(rstd_post, f32, (N,), dev, "rstd_post"), _vec(rstd_pre, f32, (N,), dev, "rstd_pre"),
                                  _stream_of(dev))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_residual_norm")


def oapl_residual_norm_workspace_bytes(N: int, d: int) -> int:
    return int(lib().oapl_residual_norm_workspace_bytes(N, d))


def oapl_residual_norm_bwd(r: OaplResidual, x_out, rstd_post, rstd_pre, dh, dx_out, dx=None, dy=None, dgate=None,
                           dw_post=None, dw_pre=None, accumulate: bool = False, ws=None):
    """Gradients of x, y, the gate and the weights from dh and dx_out (None: 0).  dgate: fp32 [N, 1] or [d], or [N, d]
    like y.  ws: uint8, oapl_residual_norm_workspace_bytes(N, d), for dw_post, dw_pre and a channel gate's dgate."""
    dev, N, d = r.device, r.N, r.d
    f32 = torch.float32
    at_dg, ld_dg = None, 0
    if dgate is not None:
        if r.gate_kind == OAPL_GATE_FULL:
            at_dg, ld_dg = _like(r, dgate, "dgate")
        elif r.gate_kind == OAPL_GATE_ROW:
            if dgate.dtype != f32 or dgate.shape != (N, 1) or dgate.get_device() != dev:
                raise TypeError(f"dgate: expected fp32 {(N, 1)} on cuda:{dev}")
            at_dg, ld_dg = dgate.data_ptr(), dgate.stride(0) if N > 1 else 1
        else:
            at_dg = _vec(dgate, f32, (d,), dev, "dgate")
    rc = lib().oapl_residual_norm_bwd(
        r, *_like(r, x_out, "x_out"), _vec(rstd_post, f32, (N,), dev, "rstd_post"),
        _vec(rstd_pre, f32, (N,), dev, "rstd_pre"), *_like(r, dh, "dh"), *_like(r, dx_out, "dx_out"), *_like(r, dx, "dx"),
        *_like(r, dy, "dy"), at_dg, ld_dg, _vec(dw_post, f32, (d,), dev, "dw_post"), _vec(dw_pre, f32, (d,), dev, "dw_pre"),
        int(accumulate), *_ws(ws, dev), _stream_of(dev))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_residual_norm_bwd")


class TensorList:
    """A host array of oapl_tensor for the tensors of a model, which it keeps alive.  Made once for gradients that keep
    their memory (zero_grad(set_to_none=False)); checking and filling it takes 1.15 us a tensor, 690 for 600 of them, which
    a list made anew at every step adds to the two calls' 22."""

    def __init__(self, tensors, outs=None):
        if not tensors:
            raise ValueError("tensors: expected at least one")
        if outs is not None and len(outs) != len(tensors):
            raise ValueError("outs: expected one for each tensor")
        self.device = tensors[0].get_device()
        self.array = (OaplTensor * len(tensors))()
        for t, o, e in zip(tensors, tensors if outs is None else outs, self.array):
            for x in (t, o):
                if x.dtype not in FLOAT_TYPES or not x.is_cuda or not x.is_contiguous() or x.get_device() != self.device:
                    raise TypeError("tensors, outs: expected contiguous CUDA tensors of bf16, fp16 or fp32 on one device")
            if t.numel() != o.numel():
                raise TypeError("outs: expected as many elements as the tensor has")
            e.data, e.out, e.n = t.data_ptr(), o.data_ptr(), t.numel()
            e.type, e.out_type = FLOAT_TYPES[t.dtype], FLOAT_TYPES[o.dtype]
        self.count, self.tensors = len(tensors), (list(tensors), None if outs is None else list(outs))


def make_tensor_list(tensors, outs=None) -> TensorList:
    """The list that oapl_grad_norm and oapl_grad_clip take.  outs: where clipped elements go (None: in place)."""
    return TensorList(tensors, outs)


def oapl_grad_norm_workspace_bytes(count: int) -> int:
    return int(lib().oapl_grad_norm_workspace_bytes(count))


def oapl_grad_norm(tensors: TensorList, sq_norm, norm, ws, scale: float = 1.0, device_status=None):
    """sq_norm, norm: fp32 [1] or None: the squared norm of scale * all tensors, and the norm.  ws: uint8,
    oapl_grad_norm_workspace_bytes(count).  sq_norm serves oapl_adamw_step as other_sq_norm."""
    dev, f32 = tensors.device, torch.float32
    rc = lib().oapl_grad_norm(tensors.array, tensors.count, scale, _vec(sq_norm, f32, (1,), dev, "sq_norm"),
                              _vec(norm, f32, (1,), dev, "norm"),
                              _vec(device_status, torch.int32, (1,), dev, "device_status"), *_ws(ws, dev), _stream_of(dev))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_grad_norm")


def oapl_grad_clip(tensors: TensorList, sq_norm, clip_norm: float, scale: float = 1.0, norm=None):
    """Every tensor times scale * min(1, clip_norm / (sqrt(sq_norm) + 1e-6)), into the list's outs.  norm: fp32 [1] of
    oapl_grad_norm, read in the place of the root of sq_norm, which may then be None: a norm above 1.8e19 makes sq_norm
    infinite, and the tensors would leave with the factor scale."""
    dev, f32 = tensors.device, torch.float32
    if sq_norm is None and norm is None:
        raise TypeError("sq_norm, norm: expected the fp32 [1] of oapl_grad_norm")
    rc = lib().oapl_grad_clip_ex(tensors.array, tensors.count, scale, _vec(sq_norm, f32, (1,), dev, "sq_norm"),
                                 _vec(norm, f32, (1,), dev, "norm"), clip_norm, _stream_of(dev))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_grad_clip")


def make_adjust(L: OaplLogits, tokens=None, spans=None, repetition=None, frequency=None, presence=None, bias_start=None,
                bias_id=None, bias=None, allowed=None, allowed_row=None) -> OaplAdjust:
    """Fill oapl_adjust for the rows of L.  tokens: int32 [T]; spans: int64 [N, 3], begin of a row's prompt, of its answer,
    and the answer's end in tokens; repetition, frequency, presence: fp32 [N]; bias_start: int64 [N + 1] into bias_id
    (int32) and bias (fp32); allowed: int32 [rows, words], bit v % 32 of word v / 32 set where token v is allowed, row n
    of it for row n or row allowed_row[n] (int32 [N], negative: all tokens).  The struct keeps the tensors alive."""
    dev, N, f32, i32 = L.device, L.N, torch.float32, torch.int32
    T = 0 if tokens is None else tokens.numel()
    biases = 0 if bias_id is None else bias_id.numel()
    at_allowed, ld, rows = None, 0, 0
    if allowed is not None:
        _, rows, words, ld = _rows(allowed, {i32: 0}, "allowed")
        if words * 32 < L.V or allowed.get_device() != dev or (allowed_row is None and rows != N):
            raise TypeError(f"allowed: expected int32 [{N}, at least {-(-L.V // 32)}] on cuda:{dev}")
        at_allowed = allowed.data_ptr()
    a = OaplAdjust(_vec(tokens, i32, (T,), dev, "tokens"), T, _vec(spans, torch.int64, (N, 3), dev, "spans"),
                   _vec(repetition, f32, (N,), dev, "repetition"), _vec(frequency, f32, (N,), dev, "frequency"),
                   _vec(presence, f32, (N,), dev, "presence"), _vec(bias_start, torch.int64, (N + 1,), dev, "bias_start"),
                   _vec(bias_id, i32, (biases,), dev, "bias_id"), _vec(bias, f32, (biases,), dev, "bias"), biases, at_allowed,
                   ld, rows, _vec(allowed_row, i32, (N,), dev, "allowed_row"))
    a.tensors = (tokens, spans, repetition, frequency, presence, bias_start, bias_id, bias, allowed, allowed_row)
    return a


def _of_logits(L, t, name):
    code, N, V, ld = _rows(t, FLOAT_TYPES, name)
    if code != L.type or N != L.N or V != L.V or t.get_device() != L.device:
        raise TypeError(f"{name}: expected the logits' type, shape and device")
    return t.data_ptr(), ld


def oapl_logits_adjust(L: OaplLogits, a: OaplAdjust, out, device_status=None):
    """out = the logits with penalties, biases and the mask applied; it may be the logits themselves."""
    rc = lib().oapl_logits_adjust(L, a, *_of_logits(L, out, "out"),
                                  _vec(device_status, torch.int32, (1,), L.device, "device_status"), _stream_of(L.device))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_logits_adjust")


def oapl_logits_adjust_bwd(L: OaplLogits, a: OaplAdjust, d_out, dlogits, device_status=None):
    """Gradient of the logits that L holds (before the adjustment) from that of the adjusted ones; dlogits may be d_out."""
    rc = lib().oapl_logits_adjust_bwd(L, a, *_of_logits(L, d_out, "d_out"), *_of_logits(L, dlogits, "dlogits"),
                                      _vec(device_status, torch.int32, (1,), L.device, "device_status"),
                                      _stream_of(L.device))
    if rc != OAPL_OK:
        raise OaplError(rc, "oapl_logits_adjust_bwd")
