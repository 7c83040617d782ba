"""Python binding of libturnopd, the GB300 (sm_103a) turn-aware OPD loss.

Argument marshalling only: every function forwards torch tensors' device
pointers, sizes and the current CUDA stream to the C entry point of the same
name (``include/turnopd.h``), and raises ``TurnopdError`` on a non-OK status.
All compute runs in the library's CUDA kernels; there is no other path.  If
the library has not been built, importing works but the first call raises.

Build it with ``python -c "import __graft_entry__ as g; g.build()"`` (or
``python paper_2607_05804_gb300/build.py``).
"""
from __future__ import annotations

import ctypes
import os

__all__ = [
    "TurnopdError", "library_path", "load",
    "TURNOPD_FULL_VOCAB", "TURNOPD_SAMPLED_TOKEN", "TURNOPD_F32", "TURNOPD_BF16",
    "TURNOPD_SCOPE_TRAJ", "TURNOPD_SCOPE_BATCH", "TURNOPD_ZERO_MASKED_GRAD",
    "TURNOPD_FORCE_PORTABLE", "TURNOPD_MAX_TURNS",
    "turnopd_turn_counts", "turnopd_weights", "turnopd_weights_workspace_bytes",
    "turnopd_loss_fwd_bwd", "turnopd_loss_workspace_bytes", "turnopd_turn_stats",
    "turnopd_alpha_schedule", "turnopd_turn_floor", "turnopd_status_string", "turnopd_loss_fwd_bwd_static",
    "turnopd_selftest_wait_timeout",
    "TURNOPD_STATIC_MAX_TOKENS", "turnopd_fused_lmhead_fwd_bwd", "turnopd_fused_workspace_bytes",
    "turnopd_fused_workspace_min_bytes",
    "turnopd_topk_loss_fwd_bwd", "TURNOPD_TOPK_MAX", "TURNOPD_TOPK_MAX_VOCAB",
    "turnopd_depth_params", "turnopd_depth_state", "turnopd_depth_default_params",
    "turnopd_depth_init", "turnopd_depth_plan", "turnopd_depth_update", "turnopd_depth_efficiency",
    "turnopd_depth_coverage", "turnopd_turn_diagnostics",
    "turnopd_vocab_stats_bytes", "turnopd_vocab_shard_stats", "turnopd_vocab_stats_merge",
    "turnopd_vocab_shard_loss_grad",
    "TURNOPD_TOP_ALTERNATIVES_MAX", "TURNOPD_LAYER_NORM", "TURNOPD_RMS_NORM",
    "turnopd_token_logprobs", "turnopd_token_logprobs_bwd", "turnopd_token_logprobs_workspace_bytes",
    "turnopd_norm_fwd", "turnopd_norm_bwd", "turnopd_norm_bwd_workspace_bytes",
    "TURNOPD_E4M3", "TURNOPD_INT8", "TURNOPD_ACCUMULATE_GRAD",
    "turnopd_embedding_fwd", "turnopd_embedding_bwd", "turnopd_embedding_bwd_workspace_bytes",
    "turnopd_block_norm_fwd", "turnopd_block_norm_bwd", "turnopd_block_norm_bwd_workspace_bytes",
    "turnopd_act8_store", "turnopd_act8_load",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libturnopd.so")

TURNOPD_FULL_VOCAB, TURNOPD_SAMPLED_TOKEN = 0, 1
TURNOPD_F32, TURNOPD_BF16 = 0, 1
TURNOPD_E4M3, TURNOPD_INT8 = 2, 3
TURNOPD_SCOPE_TRAJ, TURNOPD_SCOPE_BATCH = 0, 1
TURNOPD_ZERO_MASKED_GRAD = 0x1
TURNOPD_ACCUMULATE_GRAD = 0x2
TURNOPD_FORCE_PORTABLE = 0x100
TURNOPD_MAX_TURNS = 4096
TURNOPD_STATIC_MAX_TOKENS = 65536
TURNOPD_TOPK_MAX = 1024
TURNOPD_TOPK_MAX_VOCAB = 737280
TURNOPD_TOP_ALTERNATIVES_MAX = 32
TURNOPD_LAYER_NORM, TURNOPD_RMS_NORM = 0, 1

STATUS_NAMES = {
    0: "TURNOPD_OK", 1: "TURNOPD_ERR_NULL", 2: "TURNOPD_ERR_SHAPE", 3: "TURNOPD_ERR_OFFSETS",
    4: "TURNOPD_ERR_TURN_RANGE", 5: "TURNOPD_ERR_TOKEN_RANGE", 6: "TURNOPD_ERR_UNSUPPORTED",
    7: "TURNOPD_ERR_CUDA", 8: "TURNOPD_ERR_TIMEOUT", 9: "TURNOPD_ERR_NONFINITE",
    10: "TURNOPD_ERR_WORKSPACE",
}


class TurnopdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = int(code)
        super().__init__(f"{where}: {STATUS_NAMES.get(self.code, self.code)} "
                         f"({turnopd_status_string(self.code)})")


def library_path() -> str:
    return _LIB_PATH


_lib = None


def load():
    """Load libturnopd.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"libturnopd.so not found at {_LIB_PATH}: the CUDA library has not "
                           "been built (run __graft_entry__.build())")
    lib = ctypes.CDLL(_LIB_PATH)
    P, i32, i64, u32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32
    f64, sz = ctypes.c_double, ctypes.c_size_t
    sig = {
        "turnopd_turn_counts": [P, P, P, i32, i64, i32, P, P, P, P],
        "turnopd_weights": [P, P, P, i32, i64, i32, f64, i32, i32, P, P, P, sz, P, P],
        "turnopd_loss_fwd_bwd": [P, P, i32, i64, i64, i64, P, P, P, P, i64, i32, P, i32, u32,
                                 P, P, P, sz, P, P],
        "turnopd_turn_stats": [P, P, P, P, i32, i64, i32, P, P, P, P, P, P, P],
        "turnopd_loss_fwd_bwd_static": [P, P, i32, i64, i64, i64, P, P, P, P, i64, i32, P, i32,
                                        u32, P, P, P, P],
        "turnopd_fused_lmhead_fwd_bwd": [P, P, i64, P, P, i64, i64, P, P, i64, i32, P, P, P, P, P,
                                         sz, P, P],
        "turnopd_topk_loss_fwd_bwd": [P, P, i32, i64, i64, i64, P, P, P, i64, i32, P, P, P, i32, u32,
                                      P, P, P, sz, P, P],
    }
    D, Pp = ctypes.c_double, ctypes.POINTER
    sig.update({
        "turnopd_depth_default_params": [P],
        "turnopd_depth_init": [P, P],
        "turnopd_depth_plan": [P, P, i64, P, P, P],
        "turnopd_depth_update": [P, P, i64, P, P, P, i32, P, P, i32, P, P],
        "turnopd_depth_efficiency": [P, P, P, i32, D, P, P, P, P],
        "turnopd_depth_coverage": [P, P, i32, D, i32, i32, i32, P],
        "turnopd_turn_diagnostics": [P, P, P, i32, i32, P, P, P],
        "turnopd_vocab_shard_stats": [P, P, i32, i64, i64, i64, P, P, i64, P, P, ctypes.c_size_t, P, P],
        "turnopd_vocab_stats_merge": [P, i32, P, i64, P, P],
        "turnopd_selftest_wait_timeout": [u32, P, P],
        "turnopd_vocab_shard_loss_grad": [P, P, i32, i64, i64, i64, P, P, P, i64, P, P, i32, u32, P, P, P,
                                          sz, P, P],
        "turnopd_token_logprobs": [P, i32, i64, i64, i64, P, P, P, i64, i32, P, P, P, P, P, P, sz, P, P],
        "turnopd_token_logprobs_bwd": [P, i32, i64, i64, i64, P, P, P, i64, P, P, P, P, P, P, i32, u32, P, sz,
                                       P, P],
        "turnopd_norm_fwd": [P, i32, i64, P, P, i32, P, i64, i64, i32, f64, P, i32, i64, P, P, P, P],
        "turnopd_norm_bwd": [P, i32, i64, P, i32, P, i64, i64, i32, P, P, P, i32, i64, P, i32, i64, P, P, P, sz,
                             P],
        "turnopd_embedding_fwd": [P, i32, i64, i64, P, P, i64, i64, f64, P, i32, i64, P, P],
        "turnopd_embedding_bwd": [P, i32, i64, P, P, i64, i64, f64, P, i32, i64, i64, u32, P, sz, P, P],
        "turnopd_block_norm_fwd": [P, i32, i64, P, i32, i64, P, P, P, i64, P, P, i32, P, i64, i64, i32, f64, f64, f64,
                                   P, i64, P, i64, P, P, P],
        "turnopd_block_norm_bwd": [P, i32, i64, P, P, i32, i64, P, P, P, P, i64, P, i32, P, i64, i64, i32, f64, f64, P,
                                   i32, i32, P, i64, P, i64, P, i64, P, i64, P, i64, P, P, P, P, P, sz, P],
        "turnopd_act8_store": [P, i32, i64, P, i64, i64, P, i32, i64, P, P, P],
        "turnopd_act8_load": [P, i32, i64, P, i64, i64, P, i32, i64, P],
    })
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    lib.turnopd_weights_workspace_bytes.argtypes = [i32, i32]
    lib.turnopd_weights_workspace_bytes.restype = sz
    lib.turnopd_loss_workspace_bytes.argtypes = [i64]
    lib.turnopd_loss_workspace_bytes.restype = sz
    lib.turnopd_fused_workspace_bytes.argtypes = [i64, i64, i64, i64]
    lib.turnopd_fused_workspace_bytes.restype = sz
    lib.turnopd_fused_workspace_min_bytes.argtypes = [i64, i64, i64, i64]
    lib.turnopd_fused_workspace_min_bytes.restype = sz
    lib.turnopd_alpha_schedule.argtypes = [i64, i64, f64, f64]
    lib.turnopd_alpha_schedule.restype = f64
    lib.turnopd_turn_floor.argtypes = [i64, i32, f64]
    lib.turnopd_turn_floor.restype = i32
    lib.turnopd_depth_default_params.restype = None
    lib.turnopd_token_logprobs_workspace_bytes.argtypes = [i64]
    lib.turnopd_token_logprobs_workspace_bytes.restype = sz
    lib.turnopd_norm_bwd_workspace_bytes.argtypes = [i64, i64]
    lib.turnopd_norm_bwd_workspace_bytes.restype = sz
    lib.turnopd_embedding_bwd_workspace_bytes.argtypes = [i64, i64, i64]
    lib.turnopd_embedding_bwd_workspace_bytes.restype = sz
    lib.turnopd_block_norm_bwd_workspace_bytes.argtypes = [i64, i64]
    lib.turnopd_block_norm_bwd_workspace_bytes.restype = sz
    lib.turnopd_vocab_stats_bytes.argtypes = [i64]
    lib.turnopd_vocab_stats_bytes.restype = sz
    lib.turnopd_status_string.argtypes = [ctypes.c_int]
    lib.turnopd_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


# ---------------------------------------------------------------- marshalling helpers

def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    import torch

    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _need(t, name, dtype=None, numel=None):
    import torch

    if t is None:
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} needs at least {numel} elements, has {t.numel()}")


def _dtype_code(t, name):
    import torch

    if t.dtype == torch.bfloat16:
        return TURNOPD_BF16
    if t.dtype == torch.float32:
        return TURNOPD_F32
    raise ValueError(f"{name} must be float32 or bfloat16")


def _check(code, where):
    if code != 0:
        raise TurnopdError(code, where)


# ---------------------------------------------------------------- entry points

def turnopd_status_string(code: int) -> str:
    return load().turnopd_status_string(int(code)).decode()


def turnopd_selftest_wait_timeout(poll_limit: int, dev_status, stream=None):
    """One CTA polls a barrier that nothing arrives on; after poll_limit polls it
    records TURNOPD_ERR_TIMEOUT in dev_status (device int32[1])."""
    import torch

    _need(dev_status, "dev_status", torch.int32, 1)
    _check(load().turnopd_selftest_wait_timeout(int(poll_limit), _ptr(dev_status), _stream(stream)),
           "turnopd_selftest_wait_timeout")


def turnopd_alpha_schedule(k: int, K: int, s: float = 0.0, e: float = 1.0) -> float:
    return float(load().turnopd_alpha_schedule(int(k), int(K), float(s), float(e)))


def turnopd_turn_floor(n_traj: int, min_floor: int = 8, min_frac: float = 0.15) -> int:
    """n_min = max(min_floor, ceil(min_frac * n_traj)) for turnopd_weights; defaults
    are the paper's internal-blend settings.  n_traj counts the step's trajectories
    over all ranks."""
    n = int(load().turnopd_turn_floor(int(n_traj), int(min_floor), float(min_frac)))
    if n < 0:
        raise ValueError("turnopd_turn_floor: n_traj and min_floor must be >= 0, min_frac in [0, 1]")
    return n


def turnopd_weights_workspace_bytes(num_traj: int, max_turns: int) -> int:
    return int(load().turnopd_weights_workspace_bytes(int(num_traj), int(max_turns)))


def turnopd_loss_workspace_bytes(num_tokens: int) -> int:
    return int(load().turnopd_loss_workspace_bytes(int(num_tokens)))


def turnopd_fused_workspace_bytes(num_tokens: int, vocab: int, d_s: int, d_t: int) -> int:
    return int(load().turnopd_fused_workspace_bytes(int(num_tokens), int(vocab), int(d_s), int(d_t)))


def turnopd_fused_workspace_min_bytes(num_tokens: int, vocab: int, d_s: int, d_t: int) -> int:
    """The least a call accepts: without room for a chunk's logits, which the backward pass then
    computes a second time."""
    return int(load().turnopd_fused_workspace_min_bytes(int(num_tokens), int(vocab), int(d_s), int(d_t)))


def turnopd_fused_lmhead_fwd_bwd(h_s, W_s, h_t, W_t, loss_mask, w, mode, dh_s_out, token_loss_out,
                                 loss_out, workspace, dev_status, stream=None, dW_s_out=None):
    """h_s [T, d_s], W_s [V, d_s], h_t [T, d_t], W_t [V, d_t] bf16; dh_s_out [T, d_s] fp32 or
    None; dW_s_out [V, d_s] fp32 or None."""
    import torch

    T, d_s = h_s.shape
    d_t = h_t.shape[1]
    V = W_s.shape[0]
    _need(h_s, "h_s", torch.bfloat16)
    _need(W_s, "W_s", torch.bfloat16)
    _need(h_t, "h_t", torch.bfloat16, T * d_t)
    _need(W_t, "W_t", torch.bfloat16, V * d_t)
    if W_s.shape[1] != d_s or W_t.shape[0] != V or h_t.shape[0] != T:
        raise ValueError("shape mismatch between hidden states and heads")
    _need(loss_mask, "loss_mask", torch.uint8, T)
    _need(w, "w", torch.float32, T)
    _need(dh_s_out, "dh_s_out", torch.float32, T * d_s)
    _need(dW_s_out, "dW_s_out", torch.float32, V * d_s)
    _need(token_loss_out, "token_loss_out", torch.float32, T)
    _need(loss_out, "loss_out", torch.float64, 1)
    _need(workspace, "workspace")
    _need(dev_status, "dev_status", torch.int32, 1)
    _check(load().turnopd_fused_lmhead_fwd_bwd(
        _ptr(h_s), _ptr(W_s), d_s, _ptr(h_t), _ptr(W_t), d_t, V, _ptr(loss_mask), _ptr(w), T,
        int(mode), _ptr(dh_s_out), _ptr(dW_s_out), _ptr(token_loss_out), _ptr(loss_out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(dev_status), _stream(stream)),
        "turnopd_fused_lmhead_fwd_bwd")


def turnopd_turn_counts(turn_id, loss_mask, traj_offsets, max_turns, traj_turn_cnt, counts,
                        dev_status, stream=None):
    import torch

    T, B = turn_id.numel(), traj_offsets.numel() - 1
    _need(turn_id, "turn_id", torch.int32)
    _need(loss_mask, "loss_mask", torch.uint8, T)
    _need(traj_offsets, "traj_offsets", torch.int64)
    _need(traj_turn_cnt, "traj_turn_cnt", torch.int32, B * max_turns)
    _need(counts, "counts", torch.int64, 2 * max_turns + 1)
    _need(dev_status, "dev_status", torch.int32, 1)
    _check(load().turnopd_turn_counts(_ptr(turn_id), _ptr(loss_mask), _ptr(traj_offsets), B, T,
                                      int(max_turns), _ptr(traj_turn_cnt), _ptr(counts),
                                      _ptr(dev_status), _stream(stream)), "turnopd_turn_counts")


def turnopd_weights(turn_id, loss_mask, traj_offsets, max_turns, alpha, scope, n_min,
                    global_counts, w_out, workspace, dev_status, stream=None):
    import torch

    T, B = turn_id.numel(), traj_offsets.numel() - 1
    _need(turn_id, "turn_id", torch.int32)
    _need(loss_mask, "loss_mask", torch.uint8, T)
    _need(traj_offsets, "traj_offsets", torch.int64)
    _need(global_counts, "global_counts", torch.int64, 2 * max_turns + 1)
    _need(w_out, "w_out", torch.float32, T)
    _need(workspace, "workspace")
    _need(dev_status, "dev_status", torch.int32, 1)
    _check(load().turnopd_weights(_ptr(turn_id), _ptr(loss_mask), _ptr(traj_offsets), B, T,
                                  int(max_turns), float(alpha), int(scope), int(n_min),
                                  _ptr(global_counts), _ptr(w_out), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(),
                                  _ptr(dev_status), _stream(stream)), "turnopd_weights")


def turnopd_loss_fwd_bwd(z_student, z_teacher, vocab, row_of_token, sampled_ids, loss_mask, w,
                         mode, grad_student, flags, token_loss_out, loss_out, workspace,
                         dev_status, stream=None):
    """z_student, z_teacher: [num_rows, ld] tensors (row stride ld, unit column stride);
    grad_student: None or a tensor of the same shape and strides."""
    import torch

    T = loss_mask.numel()
    for name, z in (("z_student", z_student), ("z_teacher", z_teacher)):
        if not z.is_cuda or z.dim() != 2 or z.stride(1) != 1:
            raise ValueError(f"{name} must be a 2-D CUDA tensor with unit column stride")
    if z_teacher.shape != z_student.shape or z_teacher.stride() != z_student.stride() \
            or z_teacher.dtype != z_student.dtype:
        raise ValueError("z_teacher must match z_student in shape, stride and dtype")
    ld = z_student.stride(0)
    if grad_student is not None and (grad_student.shape != z_student.shape
                                     or grad_student.stride(0) != ld or grad_student.stride(1) != 1
                                     or not grad_student.is_cuda):
        raise ValueError("grad_student must match z_student in shape and row stride")
    _need(row_of_token, "row_of_token", torch.int32, T)
    _need(sampled_ids, "sampled_ids", torch.int32, T)
    _need(loss_mask, "loss_mask", torch.uint8)
    _need(w, "w", torch.float32, T)
    _need(token_loss_out, "token_loss_out", torch.float32, T)
    _need(loss_out, "loss_out", torch.float64, 1)
    _need(workspace, "workspace")
    _need(dev_status, "dev_status", torch.int32, 1)
    gdt = _dtype_code(grad_student, "grad_student") if grad_student is not None else TURNOPD_F32
    _check(load().turnopd_loss_fwd_bwd(
        _ptr(z_student), _ptr(z_teacher), _dtype_code(z_student, "z_student"), ld, int(vocab),
        z_student.shape[0], _ptr(row_of_token), _ptr(sampled_ids), _ptr(loss_mask), _ptr(w), T,
        int(mode), _ptr(grad_student), gdt, int(flags), _ptr(token_loss_out), _ptr(loss_out),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(dev_status),
        _stream(stream)), "turnopd_loss_fwd_bwd")


def turnopd_topk_loss_fwd_bwd(z_student, z_teacher, vocab, row_of_token, loss_mask, w, k_top,
                              topk_ids_out, topk_grad_out, grad_student, flags, token_loss_out,
                              loss_out, workspace, dev_status, stream=None):
    """Teacher top-K reverse KL.  z_student, z_teacher: [num_rows, ld] tensors;
    topk_ids_out int32 / topk_grad_out float32 [T, k_top] or None; grad_student None or
    a tensor shaped like z_student."""
    import torch

    T = loss_mask.numel()
    for name, z in (("z_student", z_student), ("z_teacher", z_teacher)):
        if not z.is_cuda or z.dim() != 2 or z.stride(1) != 1:
            raise ValueError(f"{name} must be a 2-D CUDA tensor with unit column stride")
    if z_teacher.shape != z_student.shape or z_teacher.stride() != z_student.stride() \
            or z_teacher.dtype != z_student.dtype:
        raise ValueError("z_teacher must match z_student in shape, stride and dtype")
    ld = z_student.stride(0)
    if grad_student is not None and (grad_student.shape != z_student.shape
                                     or grad_student.stride(0) != ld or grad_student.stride(1) != 1
                                     or not grad_student.is_cuda):
        raise ValueError("grad_student must match z_student in shape and row stride")
    _need(row_of_token, "row_of_token", torch.int32, T)
    _need(loss_mask, "loss_mask", torch.uint8)
    _need(w, "w", torch.float32, T)
    _need(topk_ids_out, "topk_ids_out", torch.int32, T * int(k_top))
    _need(topk_grad_out, "topk_grad_out", torch.float32, T * int(k_top))
    _need(token_loss_out, "token_loss_out", torch.float32, T)
    _need(loss_out, "loss_out", torch.float64, 1)
    _need(workspace, "workspace")
    _need(dev_status, "dev_status", torch.int32, 1)
    gdt = _dtype_code(grad_student, "grad_student") if grad_student is not None else TURNOPD_F32
    _check(load().turnopd_topk_loss_fwd_bwd(
        _ptr(z_student), _ptr(z_teacher), _dtype_code(z_student, "z_student"), ld, int(vocab),
        z_student.shape[0], _ptr(row_of_token), _ptr(loss_mask), _ptr(w), T, int(k_top),
        _ptr(topk_ids_out), _ptr(topk_grad_out), _ptr(grad_student), gdt, int(flags),
        _ptr(token_loss_out), _ptr(loss_out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(dev_status), _stream(stream)),
        "turnopd_topk_loss_fwd_bwd")


# ---------------------------------------------------------------- vocabulary-parallel split

def _shard_logits(z_student, z_teacher):
    for name, z in (("z_student", z_student), ("z_teacher", z_teacher)):
        if not z.is_cuda or z.dim() != 2 or z.stride(1) != 1:
            raise ValueError(f"{name} must be a 2-D CUDA tensor with unit column stride")
    if z_teacher.shape != z_student.shape or z_teacher.stride() != z_student.stride() \
            or z_teacher.dtype != z_student.dtype:
        raise ValueError("z_teacher must match z_student in shape, stride and dtype")
    return z_student.stride(0), z_student.shape[1]


def turnopd_vocab_stats_bytes(num_tokens: int) -> int:
    return int(load().turnopd_vocab_stats_bytes(int(num_tokens)))


def turnopd_vocab_shard_stats(z_student, z_teacher, row_of_token, loss_mask, stats_out, workspace, dev_status,
                              stream=None):
    """z_student, z_teacher: this rank's [num_rows, shard_vocab] column shard (row stride ld);
    stats_out float32 [T, 6]; workspace of turnopd_loss_workspace_bytes(T) bytes."""
    import torch

    ld, Vr = _shard_logits(z_student, z_teacher)
    T = loss_mask.numel()
    _need(row_of_token, "row_of_token", torch.int32, T)
    _need(loss_mask, "loss_mask", torch.uint8)
    _need(stats_out, "stats_out", torch.float32, T * 6)
    _need(workspace, "workspace")
    _need(dev_status, "dev_status", torch.int32, 1)
    _check(load().turnopd_vocab_shard_stats(
        _ptr(z_student), _ptr(z_teacher), _dtype_code(z_student, "z_student"), ld, Vr, z_student.shape[0],
        _ptr(row_of_token), _ptr(loss_mask), T, _ptr(stats_out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(dev_status), _stream(stream)),
        "turnopd_vocab_shard_stats")


def turnopd_vocab_stats_merge(parts, loss_mask, merged_out, stream=None):
    """parts float32 [n_shards, T, 6] (shard order) -> merged_out [T, 6]."""
    import torch

    T = loss_mask.numel()
    _need(parts, "parts", torch.float32)
    _need(loss_mask, "loss_mask", torch.uint8)
    _need(merged_out, "merged_out", torch.float32, T * 6)
    _check(load().turnopd_vocab_stats_merge(_ptr(parts), parts.shape[0], _ptr(loss_mask), T, _ptr(merged_out),
                                            _stream(stream)), "turnopd_vocab_stats_merge")


def turnopd_vocab_shard_loss_grad(z_student, z_teacher, row_of_token, loss_mask, w, merged_stats, grad_shard,
                                  flags, token_loss_out, loss_out, workspace, dev_status, stream=None):
    import torch

    ld, Vr = _shard_logits(z_student, z_teacher)
    T = loss_mask.numel()
    if grad_shard is not None and (grad_shard.shape != z_student.shape or grad_shard.stride(0) != ld
                                   or grad_shard.stride(1) != 1 or not grad_shard.is_cuda):
        raise ValueError("grad_shard must match the logit shard in shape and row stride")
    _need(row_of_token, "row_of_token", torch.int32, T)
    _need(loss_mask, "loss_mask", torch.uint8)
    _need(w, "w", torch.float32, T)
    _need(merged_stats, "merged_stats", torch.float32, T * 6)
    _need(token_loss_out, "token_loss_out", torch.float32, T)
    _need(loss_out, "loss_out", torch.float64, 1)
    _need(workspace, "workspace")
    _need(dev_status, "dev_status", torch.int32, 1)
    gdt = _dtype_code(grad_shard, "grad_shard") if grad_shard is not None else TURNOPD_F32
    _check(load().turnopd_vocab_shard_loss_grad(
        _ptr(z_student), _ptr(z_teacher), _dtype_code(z_student, "z_student"), ld, Vr, z_student.shape[0],
        _ptr(row_of_token), _ptr(loss_mask), _ptr(w), T, _ptr(merged_stats), _ptr(grad_shard), gdt, int(flags),
        _ptr(token_loss_out), _ptr(loss_out), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _ptr(dev_status), _stream(stream)), "turnopd_vocab_shard_loss_grad")


# ---------------------------------------------------------------- log probabilities of given tokens
#
# These calls are made once per decoding step too, where a few microseconds of marshalling count.

def _arg(t, name, dtype=None, numel=0):
    """The device pointer of a contiguous CUDA tensor (None stays None); _need says what is wrong with others."""
    if t is None:
        return None
    if not t.is_cuda or (dtype is not None and t.dtype is not dtype) or t.numel() < numel or not t.is_contiguous():
        _need(t, name, dtype, numel)
    return t.data_ptr()


def _handle(stream, t):
    """The cudaStream_t of `stream`, or of the current stream of t's device (without the Stream object that
    torch.cuda.current_stream() makes)."""
    if stream is not None:
        return stream.cuda_stream
    import torch

    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _rows_2d(t, name, like=None):
    """The row stride of a 2-D CUDA tensor with unit column stride."""
    shape, (ld, step) = t.shape, t.stride() if t.dim() == 2 else (0, 0)
    if not t.is_cuda or ld == step == 0 or (step != 1 and shape[1] > 1):
        raise ValueError(f"{name} must be a 2-D CUDA tensor with unit column stride")
    if like is not None and (shape != like.shape or ld != like.stride(0)):
        raise ValueError(f"{name} must match the logits in shape and row stride")
    return ld if shape[0] > 1 else max(ld, shape[1])


def turnopd_token_logprobs_workspace_bytes(num_tokens: int) -> int:
    return int(load().turnopd_token_logprobs_workspace_bytes(int(num_tokens)))


def _num_tokens(logits, row_of_token, token_ids, loss_mask):
    for t in (loss_mask, token_ids, row_of_token):
        if t is not None:
            return t.numel()
    return logits.shape[0]


def _ws(workspace):
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def turnopd_token_logprobs(logits, vocab, row_of_token, token_ids, loss_mask, n_top, logprob_out, entropy_out,
                           stats_out, top_ids_out, top_logprob_out, workspace, dev_status, stream=None):
    """Log probability of token_ids[i] in its row, the row's entropy, (m, log S) and the n_top best ids.
    logits [num_rows, ld]; row_of_token, token_ids int32 [T] or None; loss_mask uint8 [T] or None (every
    token; workspace may be None then); the outputs float32 [T] / [T, 2] / int32 and float32 [T, n_top], or None."""
    import torch

    f32, i32 = torch.float32, torch.int32
    ld, rows = _rows_2d(logits, "logits"), logits.shape[0]
    T = _num_tokens(logits, row_of_token, token_ids, loss_mask)
    if vocab > logits.shape[1]:
        raise ValueError("vocab is larger than the rows of logits")
    code = load().turnopd_token_logprobs(
        logits.data_ptr(), _dtype_code(logits, "logits"), ld, int(vocab), rows, _arg(row_of_token, "row_of_token", i32, T),
        _arg(token_ids, "token_ids", i32, T), _arg(loss_mask, "loss_mask", torch.uint8, T), T, int(n_top),
        _arg(logprob_out, "logprob_out", f32, T), _arg(entropy_out, "entropy_out", f32, T),
        _arg(stats_out, "stats_out", f32, 2 * T), _arg(top_ids_out, "top_ids_out", i32, T * n_top),
        _arg(top_logprob_out, "top_logprob_out", f32, T * n_top), _arg(workspace, "workspace"), _ws(workspace),
        _arg(dev_status, "dev_status", i32, 1), _handle(stream, logits))
    if code:
        raise TurnopdError(code, "turnopd_token_logprobs")


def turnopd_token_logprobs_bwd(logits, vocab, row_of_token, token_ids, loss_mask, stats, logprob, entropy, d_logprob,
                               d_entropy, grad_out, flags, workspace, dev_status, stream=None):
    """Gradient with respect to the logits from d_logprob and / or d_entropy (float32 [T] or None);
    stats, logprob and entropy are the forward call's outputs; grad_out is shaped like the logits, or is
    the logits."""
    import torch

    f32, i32 = torch.float32, torch.int32
    ld, rows = _rows_2d(logits, "logits"), logits.shape[0]
    _rows_2d(grad_out, "grad_out", logits)
    T = _num_tokens(logits, row_of_token, token_ids, loss_mask)
    if vocab > logits.shape[1]:
        raise ValueError("vocab is larger than the rows of logits")
    code = load().turnopd_token_logprobs_bwd(
        logits.data_ptr(), _dtype_code(logits, "logits"), ld, int(vocab), rows, _arg(row_of_token, "row_of_token", i32, T),
        _arg(token_ids, "token_ids", i32, T), _arg(loss_mask, "loss_mask", torch.uint8, T), T,
        _arg(stats, "stats", f32, 2 * T), _arg(logprob, "logprob", f32, T), _arg(entropy, "entropy", f32, T),
        _arg(d_logprob, "d_logprob", f32, T), _arg(d_entropy, "d_entropy", f32, T), grad_out.data_ptr(),
        _dtype_code(grad_out, "grad_out"), int(flags), _arg(workspace, "workspace"), _ws(workspace),
        _arg(dev_status, "dev_status", i32, 1), _handle(stream, logits))
    if code:
        raise TurnopdError(code, "turnopd_token_logprobs_bwd")


# ---------------------------------------------------------------- the norm before the LM head

def turnopd_norm_fwd(x, gamma, beta, loss_mask, kind, eps, y_out, mean_out, rstd_out, dev_status, stream=None):
    """x [T, d] -> y_out [T, d] (rows any stride); gamma, beta [d] (beta or None); loss_mask uint8 [T] or None;
    mean_out, rstd_out float32 [T] or None; kind TURNOPD_LAYER_NORM or TURNOPD_RMS_NORM."""
    import torch

    f32 = torch.float32
    ldx, ldy = _rows_2d(x, "x"), _rows_2d(y_out, "y_out")
    T, d = x.shape
    if y_out.shape != x.shape:
        raise ValueError("y_out must match x in shape")
    if beta is not None and beta.dtype is not gamma.dtype:
        raise ValueError("gamma and beta must have one dtype")
    code = load().turnopd_norm_fwd(
        x.data_ptr(), _dtype_code(x, "x"), ldx, _arg(gamma, "gamma", None, d), _arg(beta, "beta", None, d),
        _dtype_code(gamma, "gamma"), _arg(loss_mask, "loss_mask", torch.uint8, T), T, d, int(kind), float(eps), y_out.data_ptr(),
        _dtype_code(y_out, "y_out"), ldy, _arg(mean_out, "mean_out", f32, T), _arg(rstd_out, "rstd_out", f32, T),
        _arg(dev_status, "dev_status", torch.int32, 1), _handle(stream, x))
    if code:
        raise TurnopdError(code, "turnopd_norm_fwd")


def turnopd_norm_bwd_workspace_bytes(num_tokens: int, d: int) -> int:
    return int(load().turnopd_norm_bwd_workspace_bytes(int(num_tokens), int(d)))


def turnopd_norm_bwd(x, gamma, loss_mask, kind, mean, rstd, dy, dx_out, dgamma_out, dbeta_out, workspace, stream=None):
    """dx_out [T, d] (or None), dgamma_out and dbeta_out float32 [d] (or None) from dy [T, d]; mean (None for the
    root-mean-square norm) and rstd are the forward call's."""
    import torch

    f32 = torch.float32
    ldx, lddy = _rows_2d(x, "x"), _rows_2d(dy, "dy")
    T, d = x.shape
    if dy.shape != x.shape or (dx_out is not None and dx_out.shape != x.shape):
        raise ValueError("dy and dx_out must match x in shape")
    lddx = _rows_2d(dx_out, "dx_out") if dx_out is not None else d
    code = load().turnopd_norm_bwd(
        x.data_ptr(), _dtype_code(x, "x"), ldx, _arg(gamma, "gamma", None, d), _dtype_code(gamma, "gamma"),
        _arg(loss_mask, "loss_mask", torch.uint8, T), T, d, int(kind), _arg(mean, "mean", f32, T), _arg(rstd, "rstd", f32, T),
        dy.data_ptr(), _dtype_code(dy, "dy"), lddy, None if dx_out is None else dx_out.data_ptr(),
        TURNOPD_F32 if dx_out is None else _dtype_code(dx_out, "dx_out"), lddx, _arg(dgamma_out, "dgamma_out", f32, d),
        _arg(dbeta_out, "dbeta_out", f32, d), _arg(workspace, "workspace"), _ws(workspace), _handle(stream, x))
    if code:
        raise TurnopdError(code, "turnopd_norm_bwd")


# ---------------------------------------------------------------- from the token ids to the norm before the LM head

def _rows_like(t, name, shape, dtype=None):
    """Pointer and row stride of a 2-D CUDA tensor of a given shape and type (None stays None)."""
    if t is None:
        return None, shape[1]
    # the common case first: these calls are made between any two blocks of a decoding step
    if t.shape == shape and t.is_cuda and t.is_contiguous() and (dtype is None or t.dtype is dtype):
        return t.data_ptr(), shape[1]
    ld = _rows_2d(t, name)
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, has {tuple(t.shape)}")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    return t.data_ptr(), ld


def turnopd_embedding_fwd(w, token_ids, mask, scale, out, dev_status, stream=None):
    """out[i] = scale w[token_ids[i]]: w [vocab, d], token_ids int32 [T], mask uint8 [T] or None (every token),
    out [T, d]; rows of masked tokens are zero."""
    import torch

    if w.dim() != 2:
        raise ValueError("w must be a 2-D CUDA tensor with unit column stride")
    T, (V, d) = token_ids.numel(), w.shape
    pw, ldw = _rows_like(w, "w", w.shape)
    po, ldo = _rows_like(out, "out", (T, d))
    code = load().turnopd_embedding_fwd(
        pw, _dtype_code(w, "w"), ldw, V, _arg(token_ids, "token_ids", torch.int32, T),
        _arg(mask, "mask", torch.uint8, T), T, d, float(scale), po, _dtype_code(out, "out"), ldo,
        _arg(dev_status, "dev_status", torch.int32, 1), _handle(stream, w))
    if code:
        raise TurnopdError(code, "turnopd_embedding_fwd")


def turnopd_embedding_bwd_workspace_bytes(num_tokens: int, d: int, vocab: int) -> int:
    return int(load().turnopd_embedding_bwd_workspace_bytes(int(num_tokens), int(d), int(vocab)))


def turnopd_embedding_bwd(dout, token_ids, mask, scale, dw, flags, workspace, dev_status, stream=None):
    """dw [vocab, d] from dout [T, d]: the whole table, zeros included, or with TURNOPD_ACCUMULATE_GRAD added to the rows of
    the ids that occur."""
    import torch

    T, (V, d) = token_ids.numel(), dw.shape
    ldw = _rows_2d(dw, "dw")
    pg, ldg = _rows_like(dout, "dout", (T, d))
    code = load().turnopd_embedding_bwd(
        pg, _dtype_code(dout, "dout"), ldg, _arg(token_ids, "token_ids", torch.int32, T), _arg(mask, "mask", torch.uint8, T),
        T, d, float(scale), dw.data_ptr(), _dtype_code(dw, "dw"), ldw, V, int(flags), _arg(workspace, "workspace"),
        _ws(workspace), _arg(dev_status, "dev_status", torch.int32, 1), _handle(stream, dw))
    if code:
        raise TurnopdError(code, "turnopd_embedding_bwd")


def _gate_arg(gate, T, d, dtype, param_dtype, name="gate"):
    """Pointer and stride of a gate: [d] (stride 0) or [T, d]."""
    if gate is None:
        return None, 0
    if gate.dim() == 1:
        return _arg(gate, name, param_dtype, d), 0
    return _rows_like(gate, name, (T, d), dtype)


def _param_dtype(*params):
    """The dtype of the parameters that are given, which have to share one."""
    import torch

    t = None
    for p in params:
        if p is not None:
            if t is not None and p.dtype is not t:
                raise ValueError("the norms' parameters and a gate per channel must have one dtype")
            t = p.dtype
    if t is None:
        return torch.float32
    if t is not torch.float32 and t is not torch.bfloat16:
        raise ValueError("the norms' parameters and a gate per channel must be float32 or bfloat16")
    return t


def _code_of(dtype):
    import torch

    return TURNOPD_BF16 if dtype is torch.bfloat16 else TURNOPD_F32


def turnopd_block_norm_fwd(resid, y, gamma_post, beta_post, gate, gamma_pre, beta_pre, mask, kind, eps, resid_scale,
                           branch_scale, resid_out, h_out, stats_out, dev_status, stream=None):
    """resid_out = resid_scale resid + branch_scale gate N_post(y) and h_out = N_pre(resid_out), all [T, d].  resid_out
    has resid's type and may be resid, h_out has y's.  Vectors [d] or None: without gamma_post y is taken as it is, without
    gamma_pre there is no h_out.  gate [d], [T, d] (of y's type) or None; mask uint8 [T] or None; stats_out float32 [T, 4]
    or None."""
    import torch

    if resid.dim() != 2:
        raise ValueError("resid must be a 2-D CUDA tensor with unit column stride")
    T, d = shape = resid.shape
    pr, ldr = _rows_like(resid, "resid", shape)
    py, ldy = _rows_like(y, "y", shape)
    pt = _param_dtype(gamma_post, beta_post, gamma_pre, beta_pre, gate if gate is not None and gate.dim() == 1 else None)
    pg, ldg = _gate_arg(gate, T, d, y.dtype, pt)
    po, ldro = _rows_like(resid_out, "resid_out", shape, resid.dtype)
    ph, ldh = _rows_like(h_out, "h_out", shape, y.dtype)
    code = load().turnopd_block_norm_fwd(
        pr, _dtype_code(resid, "resid"), ldr, py, _dtype_code(y, "y"), ldy,
        _arg(gamma_post, "gamma_post", pt, d), _arg(beta_post, "beta_post", pt, d), pg, ldg,
        _arg(gamma_pre, "gamma_pre", pt, d), _arg(beta_pre, "beta_pre", pt, d), _code_of(pt),
        _arg(mask, "mask", torch.uint8, T), T, d, int(kind), float(eps), float(resid_scale), float(branch_scale), po, ldro,
        ph, ldh, _arg(stats_out, "stats_out", torch.float32, 4 * T), _arg(dev_status, "dev_status", torch.int32, 1),
        _handle(stream, resid))
    if code:
        raise TurnopdError(code, "turnopd_block_norm_fwd")


def turnopd_block_norm_bwd_workspace_bytes(num_tokens: int, d: int) -> int:
    return int(load().turnopd_block_norm_bwd_workspace_bytes(int(num_tokens), int(d)))


def _kept(x, name, shape):
    """Pointer, type code, row stride and exponents of an activation: a tensor, (codes, exponents), or None."""
    import torch

    if x is None:
        return None, TURNOPD_F32, shape[1], None
    if isinstance(x, (tuple, list)):
        codes, exps = x
        p, ld = _rows_like(codes, name, shape)
        return p, _act8_code(codes, name), ld, _arg(exps, f"{name}'s exponents", torch.uint8, shape[0] * ((shape[1] + 31) // 32))
    p, ld = _rows_like(x, name, shape)
    return p, _dtype_code(x, name), ld, None


def turnopd_block_norm_bwd(resid, y, gamma_post, beta_post, gate, gamma_pre, mask, kind, resid_scale, branch_scale, stats, dh,
                           d_resid_out, d_resid, dy, dgate, dgamma_post, dbeta_post, dgamma_pre, dbeta_pre, workspace,
                           stream=None):
    """Gradients from dh and d_resid_out (either None where the forward call makes no h, or nothing comes back through the
    residual stream).  resid (what the forward call wrote) and y are tensors [T, d] or the (codes, exponents) of
    turnopd_act8_store, and None where nothing needs them.  d_resid [T, d] of d_resid_out's type (it may be d_resid_out), dy
    and a gate's gradient for every element [T, d] of dh's; dgate [d] and the norms' gradients float32 [d]; each output
    may be None."""
    import torch

    f32 = torch.float32
    first = dh if dh is not None else d_resid_out
    if first is None or first.dim() != 2:
        raise ValueError("dh or d_resid_out must be a 2-D CUDA tensor")
    T, d = shape = first.shape
    channel = gate is not None and gate.dim() == 1
    gy = next((t.dtype for t in (dh, dy, dgate if not channel else None, None if channel else gate) if t is not None), f32)
    gr = next((t.dtype for t in (d_resid_out, d_resid) if t is not None), f32)
    pt = _param_dtype(gamma_post, beta_post, gamma_pre, gate if channel else None)
    pr, rcode, ldr, rexps = _kept(resid, "resid", shape)
    py, ycode, ldy, yexps = _kept(y, "y", shape)
    pg, ldg = _gate_arg(gate, T, d, gy, pt)
    ph, lddh = _rows_like(dh, "dh", shape, gy)
    pro, lddro = _rows_like(d_resid_out, "d_resid_out", shape, gr)
    pdr, lddr = _rows_like(d_resid, "d_resid", shape, gr)
    pdy, lddy = _rows_like(dy, "dy", shape, gy)
    pdg, lddg = (_arg(dgate, "dgate", f32, d), 0) if channel else _rows_like(dgate, "dgate", shape, gy)
    if not (gy in (f32, torch.bfloat16) and gr in (f32, torch.bfloat16)):
        raise ValueError("gradients must be float32 or bfloat16")
    code = load().turnopd_block_norm_bwd(
        pr, rcode, ldr, rexps, py, ycode, ldy, yexps, _arg(gamma_post, "gamma_post", pt, d),
        _arg(beta_post, "beta_post", pt, d), pg, ldg, _arg(gamma_pre, "gamma_pre", pt, d), _code_of(pt),
        _arg(mask, "mask", torch.uint8, T), T, d, int(kind), float(resid_scale), float(branch_scale),
        _arg(stats, "stats", f32, 4 * T), _code_of(gr), _code_of(gy), ph, lddh, pro, lddro, pdr, lddr, pdy, lddy, pdg, lddg,
        _arg(dgamma_post, "dgamma_post", f32, d), _arg(dbeta_post, "dbeta_post", f32, d),
        _arg(dgamma_pre, "dgamma_pre", f32, d), _arg(dbeta_pre, "dbeta_pre", f32, d), _arg(workspace, "workspace"),
        _ws(workspace), _handle(stream, first))
    if code:
        raise TurnopdError(code, "turnopd_block_norm_bwd")


def _act8_code(codes, name):
    import torch

    if codes.dtype is torch.float8_e4m3fn:
        return TURNOPD_E4M3
    if codes.dtype is torch.int8:
        return TURNOPD_INT8
    raise ValueError(f"{name}: codes must be float8_e4m3fn or int8")


def turnopd_act8_store(x, mask, codes, exps, dev_status, stream=None):
    """x [T, d] -> codes [T, d] (float8_e4m3fn or int8) and exps uint8 [T, ceil(d / 32)]: x is about codes 2^(exps - 127)."""
    import torch

    ldx, (T, d) = _rows_2d(x, "x"), x.shape
    pc, ldc = _rows_like(codes, "codes", x.shape)
    code = load().turnopd_act8_store(
        x.data_ptr(), _dtype_code(x, "x"), ldx, _arg(mask, "mask", torch.uint8, T), T, d, pc, _act8_code(codes, "codes"), ldc,
        _arg(exps, "exps", torch.uint8, T * ((d + 31) // 32)), _arg(dev_status, "dev_status", torch.int32, 1),
        _handle(stream, x))
    if code:
        raise TurnopdError(code, "turnopd_act8_store")


def turnopd_act8_load(codes, exps, out, stream=None):
    """What codes and exps stand for, into out [T, d] (float32 or bfloat16)."""
    import torch

    ldc, (T, d) = _rows_2d(codes, "codes"), codes.shape
    po, ldo = _rows_like(out, "out", codes.shape)
    code = load().turnopd_act8_load(codes.data_ptr(), _act8_code(codes, "codes"), ldc,
                                    _arg(exps, "exps", torch.uint8, T * ((d + 31) // 32)), T, d, po, _dtype_code(out, "out"),
                                    ldo, _handle(stream, out))
    if code:
        raise TurnopdError(code, "turnopd_act8_load")


# ---------------------------------------------------------------- rollout-depth controller (host)

class turnopd_depth_params(ctypes.Structure):
    _fields_ = [("h_min", ctypes.c_int32), ("h_max", ctypes.c_int32), ("ema_alpha", ctypes.c_double),
                ("coverage_p", ctypes.c_double), ("min_cov_traj", ctypes.c_int32),
                ("use_success", ctypes.c_int32), ("warmup_steps", ctypes.c_int32),
                ("probe_interval", ctypes.c_int32), ("eps", ctypes.c_double)]


class turnopd_depth_state(ctypes.Structure):
    _fields_ = [("h_bar", ctypes.c_double), ("h_eff_bar", ctypes.c_double), ("h_eff", ctypes.c_int32),
                ("h_cov", ctypes.c_int32), ("h_ctrl", ctypes.c_int32)]


def _host(a, dtype):
    import numpy as np

    if hasattr(a, "detach"):  # torch tensor (any device): copied to host memory
        a = a.detach().cpu().numpy()
    return np.ascontiguousarray(a, dtype=dtype)


def _hp(a):
    return None if a is None else ctypes.c_void_p(a.ctypes.data)


def turnopd_depth_default_params() -> turnopd_depth_params:
    p = turnopd_depth_params()
    load().turnopd_depth_default_params(ctypes.byref(p))
    return p


def turnopd_depth_init(params: turnopd_depth_params) -> turnopd_depth_state:
    st = turnopd_depth_state()
    _check(load().turnopd_depth_init(ctypes.byref(params), ctypes.byref(st)), "turnopd_depth_init")
    return st


def turnopd_depth_plan(params, state, k: int):
    """-> (h_hat, is_probe, h_roll) for step k (1-based)."""
    h, pr, roll = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check(load().turnopd_depth_plan(ctypes.byref(params), ctypes.byref(state), int(k), ctypes.byref(h),
                                     ctypes.byref(pr), ctypes.byref(roll)), "turnopd_depth_plan")
    return h.value, bool(pr.value), roll.value


def turnopd_depth_update(params, state, k: int, turn_sum, turn_cnt, turn_surv, traj_len, traj_success,
                         want_mq=False):
    """Host arrays (numpy or torch, copied to host).  Updates `state` in place; returns
    (m, q) when want_mq."""
    import numpy as np

    ts, tc, sv = _host(turn_sum, np.float64), _host(turn_cnt, np.int64), _host(turn_surv, np.int32)
    tl, su = _host(traj_len, np.int32), _host(traj_success, np.uint8)
    T = ts.size
    m = np.zeros(max(T, 1)) if want_mq else None
    q = np.zeros(max(T, 1)) if want_mq else None
    _check(load().turnopd_depth_update(ctypes.byref(params), ctypes.byref(state), int(k), _hp(ts), _hp(tc),
                                       _hp(sv), T, _hp(tl), _hp(su), tl.size, _hp(m), _hp(q)),
           "turnopd_depth_update")
    return (m[:T], q[:T]) if want_mq else None


def turnopd_depth_efficiency(turn_sum, turn_cnt, turn_surv, eps=1e-8):
    """-> (m, q, h_eff_bar, h_eff)."""
    import numpy as np

    ts, tc, sv = _host(turn_sum, np.float64), _host(turn_cnt, np.int64), _host(turn_surv, np.int32)
    T = ts.size
    m, q = np.zeros(max(T, 1)), np.zeros(max(T, 1))
    hb, he = ctypes.c_double(), ctypes.c_int32()
    _check(load().turnopd_depth_efficiency(_hp(ts), _hp(tc), _hp(sv), T, float(eps), _hp(m), _hp(q),
                                           ctypes.byref(hb), ctypes.byref(he)), "turnopd_depth_efficiency")
    return m[:T], q[:T], hb.value, he.value


def turnopd_depth_coverage(traj_len, traj_success, p=0.8, min_cov_traj=8, use_success=True, previous=0):
    import numpy as np

    tl, su = _host(traj_len, np.int32), _host(traj_success, np.uint8)
    h = ctypes.c_int32()
    _check(load().turnopd_depth_coverage(_hp(tl), _hp(su), tl.size, float(p), int(min_cov_traj),
                                         int(bool(use_success)), int(previous), ctypes.byref(h)),
           "turnopd_depth_coverage")
    return h.value


def turnopd_turn_diagnostics(turn_sum, turn_cnt, turn_surv, n_min=1):
    """-> (b [T], s [T], deep [4] = prefix, deep/shallow KL ratio, deep support, deep loss budget)."""
    import numpy as np

    ts, tc, sv = _host(turn_sum, np.float64), _host(turn_cnt, np.int64), _host(turn_surv, np.int32)
    T = ts.size
    b, sh, deep = np.zeros(max(T, 1)), np.zeros(max(T, 1)), np.zeros(4)
    _check(load().turnopd_turn_diagnostics(_hp(ts), _hp(tc), _hp(sv), T, int(n_min), _hp(b), _hp(sh),
                                           _hp(deep)), "turnopd_turn_diagnostics")
    return b[:T], sh[:T], deep


def turnopd_turn_stats(token_loss, turn_id, loss_mask, traj_offsets, max_turns, traj_turn_sum,
                       traj_turn_cnt, turn_sum, turn_cnt, turn_surv, dev_status, stream=None):
    import torch

    T, B = turn_id.numel(), traj_offsets.numel() - 1
    _need(token_loss, "token_loss", torch.float32, T)
    _need(turn_id, "turn_id", torch.int32)
    _need(loss_mask, "loss_mask", torch.uint8, T)
    _need(traj_offsets, "traj_offsets", torch.int64)
    _need(traj_turn_sum, "traj_turn_sum", torch.float64, B * max_turns)
    _need(traj_turn_cnt, "traj_turn_cnt", torch.int32, B * max_turns)
    _need(turn_sum, "turn_sum", torch.float64, max_turns)
    _need(turn_cnt, "turn_cnt", torch.int64, max_turns)
    _need(turn_surv, "turn_surv", torch.int32, max_turns)
    _need(dev_status, "dev_status", torch.int32, 1)
    _check(load().turnopd_turn_stats(_ptr(token_loss), _ptr(turn_id), _ptr(loss_mask),
                                     _ptr(traj_offsets), B, T, int(max_turns), _ptr(traj_turn_sum),
                                     _ptr(traj_turn_cnt), _ptr(turn_sum), _ptr(turn_cnt),
                                     _ptr(turn_surv), _ptr(dev_status), _stream(stream)),
           "turnopd_turn_stats")


def turnopd_loss_fwd_bwd_static(z_student, z_teacher, vocab, row_of_token, sampled_ids, loss_mask,
                                w, mode, grad_student, flags, token_loss_out, loss_out, dev_status,
                                stream=None):
    """turnopd_loss_fwd_bwd without a workspace argument, for callers that cannot
    allocate device memory: the library's own static device scratch is used instead
    (at most TURNOPD_STATIC_MAX_TOKENS tokens; calls must not overlap on the GPU)."""
    import torch

    T = loss_mask.numel()
    for name, z in (("z_student", z_student), ("z_teacher", z_teacher)):
        if not z.is_cuda or z.dim() != 2 or z.stride(1) != 1:
            raise ValueError(f"{name} must be a 2-D CUDA tensor with unit column stride")
    if z_teacher.shape != z_student.shape or z_teacher.stride() != z_student.stride() \
            or z_teacher.dtype != z_student.dtype:
        raise ValueError("z_teacher must match z_student in shape, stride and dtype")
    ld = z_student.stride(0)
    if grad_student is not None and (grad_student.shape != z_student.shape
                                     or grad_student.stride(0) != ld or grad_student.stride(1) != 1
                                     or not grad_student.is_cuda):
        raise ValueError("grad_student must match z_student in shape and row stride")
    _need(row_of_token, "row_of_token", torch.int32, T)
    _need(sampled_ids, "sampled_ids", torch.int32, T)
    _need(loss_mask, "loss_mask", torch.uint8)
    _need(w, "w", torch.float32, T)
    _need(token_loss_out, "token_loss_out", torch.float32, T)
    _need(loss_out, "loss_out", torch.float64, 1)
    _need(dev_status, "dev_status", torch.int32, 1)
    gdt = _dtype_code(grad_student, "grad_student") if grad_student is not None else TURNOPD_F32
    _check(load().turnopd_loss_fwd_bwd_static(
        _ptr(z_student), _ptr(z_teacher), _dtype_code(z_student, "z_student"), ld, int(vocab),
        z_student.shape[0], _ptr(row_of_token), _ptr(sampled_ids), _ptr(loss_mask), _ptr(w), T,
        int(mode), _ptr(grad_student), gdt, int(flags), _ptr(token_loss_out), _ptr(loss_out),
        _ptr(dev_status), _stream(stream)), "turnopd_loss_fwd_bwd_static")
