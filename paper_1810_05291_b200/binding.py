"""Python names for the C ABI of libsignsgd.so -- argument marshalling only.

Each function below has the name and the argument order of its C entry point (see
``include/signsgd.h`` and ``include/signsgd_train.h``) and does nothing but check tensor types, take ``data_ptr()`` and the
current CUDA stream, call into the library and raise on a non-zero status. All arithmetic
of Algorithm 1 happens in the CUDA kernels. There is no CPU fallback: if the library has
not been built (``python -m paper_1810_05291_b200.build``), the first call raises.

Tensors: gradients ``float32`` or ``bfloat16``; momenta and parameters ``float32``; packed
signs and votes ``int32`` (bit pattern of the uint32 words), ``ceil(d/32)`` of them.
"""

from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsignsgd.so")

SS_F32 = 0
SS_BF16 = 1
SS_MAX_WORKERS = 64
SS_STATIC_STAGING_BYTES = 64 << 20
SS_FLAGS_MAX_TIMEOUT_NS = 2_000_000_000

SS_ACT8_GROUP = 32
SS_ACT_GELU, SS_ACT_SILU = 0, 1
SS_PREF_SIGMOID, SS_PREF_HINGE, SS_PREF_SQUARED = 0, 1, 2

SS_OK = 0
SS_ERR_INVALID_ARG = -1
SS_ERR_MISALIGNED = -2
SS_ERR_UNSUPPORTED = -3
SS_ERR_CUDA = -4

EXPORTS = ("ss_packed_words", "ss_status_string", "ss_last_cuda_error", "ss_sign_pack",
           "ss_majority_vote", "ss_signum_update", "ss_apply_vote", "ss_fused_step",
           "ss_segments_upload", "ss_fused_step_segments", "ss_apply_vote_segments",
           "ss_vote_apply", "ss_vote_apply_segments", "ss_signum_update_push", "ss_vote_tally", "ss_fused_step_host", "ss_fused_step_host_static", "ss_set_launch_option",
           "ss_ternary_words", "ss_absmax", "ss_ternary_pack", "ss_ternary_unpack",
           "ss_flags_signal", "ss_flags_wait", "ss_flags_signal_wait", "ss_vote_apply_guarded",
           "ss_vote_apply_guarded_segments",
           "ss_act8_bytes", "ss_act8_pack", "ss_act8_unpack", "ss_act8_forward", "ss_act8_backward",
           "ss_weight_grad8", "ss_weight_grad8_workspace", "ss_loss_workspace", "ss_policy_loss",
           "ss_preference_loss")


class ss_segment(ctypes.Structure):
    """One tensor of a fused flat vector: first coordinate, learning rate, weight decay."""
    _fields_ = [("begin", ctypes.c_int64), ("lr", ctypes.c_float), ("weight_decay", ctypes.c_float)]


SEGMENT_BYTES = ctypes.sizeof(ss_segment)  # 16

_lib = None


class SignSGDError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().ss_status_string(status).decode()
        if status == SS_ERR_CUDA:
            msg += " [cudaError %d]" % lib().ss_last_cuda_error()
        super().__init__("%s: %s" % (where, msg))


def lib() -> ctypes.CDLL:
    """Load libsignsgd.so (once). Raises if it has not been built: there is no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "libsignsgd.so is missing (%s). Build it with `python -m paper_1810_05291_b200.build`; "
            "this package has no CPU or PyTorch fallback." % LIB_PATH)
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, u64, f32 = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint64,
                              ctypes.c_float)
    L.ss_packed_words.argtypes = [i64]
    L.ss_packed_words.restype = i64
    L.ss_status_string.argtypes = [i32]
    L.ss_status_string.restype = ctypes.c_char_p
    L.ss_last_cuda_error.argtypes = []
    L.ss_last_cuda_error.restype = i32
    L.ss_sign_pack.argtypes = [vp, i32, i64, vp, vp]
    L.ss_majority_vote.argtypes = [vp, i32, i64, u64, vp, vp]
    L.ss_signum_update.argtypes = [vp, i32, vp, f32, i64, vp, vp]
    L.ss_apply_vote.argtypes = [vp, vp, i64, f32, f32, vp]
    L.ss_fused_step.argtypes = [vp, i32, vp, i32, i64, f32, u64, vp, f32, f32, vp, vp]
    L.ss_fused_step_host.argtypes = [vp, i32, vp, vp, i32, i64, f32, u64, vp, f32, f32, vp, vp, vp]
    L.ss_fused_step_host_static.argtypes = [vp, i32, vp, i32, i64, f32, u64, vp, f32, f32, vp, vp, vp]
    L.ss_set_launch_option.argtypes = [ctypes.c_char_p, i32]
    L.ss_segments_upload.argtypes = [vp, i32, i64, vp, vp]
    L.ss_fused_step_segments.argtypes = [vp, i32, vp, i32, i64, f32, u64, vp, vp, i32, vp, vp]
    L.ss_apply_vote_segments.argtypes = [vp, vp, i64, vp, i32, vp]
    L.ss_signum_update_push.argtypes = [vp, i32, vp, f32, i64, vp, i32, vp]
    L.ss_vote_tally.argtypes = [vp, i32, i64, u64, vp, vp]
    L.ss_vote_apply.argtypes = [vp, i32, i64, u64, vp, f32, f32, vp, vp]
    L.ss_vote_apply_segments.argtypes = [vp, i32, i64, u64, vp, vp, i32, vp, vp]
    L.ss_ternary_words.argtypes = [i64]
    L.ss_ternary_words.restype = i64
    L.ss_absmax.argtypes = [vp, i32, i64, vp, vp]
    L.ss_ternary_pack.argtypes = [vp, i32, i64, vp, u64, vp, vp]
    L.ss_ternary_unpack.argtypes = [vp, i64, vp, vp, vp]
    L.ss_flags_signal.argtypes = [vp, i32, i32, ctypes.c_uint32, vp]
    L.ss_flags_wait.argtypes = [vp, i32, ctypes.c_uint32, u64, vp, vp]
    L.ss_vote_apply_guarded.argtypes = [vp, i32, i64, u64, vp, f32, f32, vp, vp, vp]
    L.ss_vote_apply_guarded_segments.argtypes = [vp, i32, i64, u64, vp, vp, i32, vp, vp, vp]
    L.ss_flags_signal_wait.argtypes = [vp, i32, i32, vp, i32, ctypes.c_uint32, u64, vp, vp]
    L.ss_act8_bytes.argtypes = [i64, i64]
    L.ss_act8_pack.argtypes = [vp, i64, i32, i64, i64, vp, vp]
    L.ss_act8_unpack.argtypes = [vp, i64, i64, vp, i64, i32, vp]
    L.ss_act8_forward.argtypes = [vp, i64, vp, i64, i32, i32, i64, i64, vp, i64, vp, vp, vp, vp]
    L.ss_act8_backward.argtypes = [vp, i64, vp, vp, i32, i32, i64, i64, vp, i64, vp, i64, vp]
    L.ss_weight_grad8_workspace.argtypes = [vp, i64, i32, i64, i64, i64]
    L.ss_weight_grad8.argtypes = [vp, i64, i32, vp, i64, i64, i64, vp, i64, i32, vp, i64, vp]
    L.ss_loss_workspace.argtypes = [i64, i64]
    L.ss_policy_loss.argtypes = [vp, i64, i32, i64, i64, vp, vp, vp, vp, vp, f32, f32, f32, f32, vp, vp, vp, vp, i64,
                                 vp, i64, vp]
    L.ss_preference_loss.argtypes = [vp, i64, i32, i64, i64, vp, vp, vp, i64, vp, f32, i32, f32, f32, f32, vp, vp, vp,
                                     vp, vp, vp, i64, vp, i64, vp]
    for name in ("ss_act8_bytes", "ss_weight_grad8_workspace", "ss_loss_workspace"):
        getattr(L, name).restype = i64
    for name in ("ss_act8_pack", "ss_act8_unpack", "ss_act8_forward", "ss_act8_backward", "ss_weight_grad8",
                 "ss_policy_loss", "ss_preference_loss"):
        getattr(L, name).restype = i32
    for name in ("ss_flags_signal", "ss_flags_wait", "ss_flags_signal_wait", "ss_vote_apply_guarded",
                 "ss_vote_apply_guarded_segments"):
        getattr(L, name).restype = i32
    for name in ("ss_absmax", "ss_ternary_pack", "ss_ternary_unpack"):
        getattr(L, name).restype = i32
    for name in ("ss_sign_pack", "ss_majority_vote", "ss_signum_update", "ss_apply_vote",
                 "ss_fused_step", "ss_fused_step_host", "ss_fused_step_host_static",
                 "ss_set_launch_option", "ss_segments_upload", "ss_fused_step_segments",
                 "ss_apply_vote_segments", "ss_vote_apply", "ss_vote_apply_segments",
                 "ss_signum_update_push", "ss_vote_tally"):
        getattr(L, name).restype = i32
    _lib = L
    return L


# ---- marshalling helpers ------------------------------------------------------------------

def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return SS_F32
    if t.dtype == torch.bfloat16:
        return SS_BF16
    raise TypeError("gradient dtype must be float32 or bfloat16, got %s" % t.dtype)


def _dev(t: torch.Tensor, dtype, name: str, n: Optional[int] = None) -> int:
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.dim() != 1 or not t.is_contiguous():
        raise ValueError("%s must be a contiguous 1-D tensor" % name)
    if n is not None and t.numel() != n:
        raise ValueError("%s must have %d elements, has %d" % (name, n, t.numel()))
    return t.data_ptr()


def _words(t: torch.Tensor, d: int, name: str) -> int:
    return _dev(t, torch.int32, name, ss_packed_words(d))


def _ptr_array(ptrs: Sequence[int]):
    return (ctypes.c_void_p * len(ptrs))(*ptrs)


def _stream(stream):
    if stream is None:  # the handle alone: a Stream object costs as much as a launch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _check(status: int, where: str) -> None:
    if status != SS_OK:
        raise SignSGDError(status, where)


# ---- the entry points -----------------------------------------------------------------------

def ss_packed_words(d: int) -> int:
    return int(lib().ss_packed_words(int(d)))


def ss_status_string(status: int) -> str:
    return lib().ss_status_string(int(status)).decode()


def ss_set_launch_option(key: str, value: int) -> None:
    _check(lib().ss_set_launch_option(key.encode(), int(value)), "ss_set_launch_option")


def ss_sign_pack(grad: torch.Tensor, out_words: torch.Tensor, stream=None) -> None:
    d = grad.numel()
    _check(lib().ss_sign_pack(_dev(grad, None, "grad"), _dtype_code(grad), d,
                              _words(out_words, d, "out_words"), _stream(stream)), "ss_sign_pack")


def ss_majority_vote(packed: Sequence[torch.Tensor], d: int, flip_mask: int,
                     vote_words: torch.Tensor, stream=None) -> None:
    ptrs = [_words(p, d, "packed[%d]" % m) for m, p in enumerate(packed)]
    _check(lib().ss_majority_vote(_ptr_array(ptrs), len(ptrs), int(d), int(flip_mask),
                                  _words(vote_words, d, "vote_words"), _stream(stream)),
           "ss_majority_vote")


def ss_signum_update(grad: torch.Tensor, momentum: torch.Tensor, beta: float,
                     out_words: torch.Tensor, stream=None) -> None:
    d = grad.numel()
    _check(lib().ss_signum_update(_dev(grad, None, "grad"), _dtype_code(grad),
                                  _dev(momentum, torch.float32, "momentum", d), float(beta), d,
                                  _words(out_words, d, "out_words"), _stream(stream)),
           "ss_signum_update")


def ss_signum_update_push(grad: torch.Tensor, momentum: torch.Tensor, beta: float,
                          dests: Sequence[torch.Tensor], stream=None) -> None:
    """``dests`` may be tensors on this GPU or raw integer addresses of peer buffers."""
    d = grad.numel()
    ptrs = [p if isinstance(p, int) else _words(p, d, "dests[%d]" % i) for i, p in enumerate(dests)]
    _check(lib().ss_signum_update_push(_dev(grad, None, "grad"), _dtype_code(grad),
                                       _dev(momentum, torch.float32, "momentum", d), float(beta), d,
                                       _ptr_array(ptrs), len(ptrs), _stream(stream)),
           "ss_signum_update_push")


def ss_vote_tally(packed: Sequence[torch.Tensor], d: int, flip_mask: int, tally_out: torch.Tensor,
                  stream=None) -> None:
    ptrs = [_words(p, d, "packed[%d]" % m) for m, p in enumerate(packed)]
    _check(lib().ss_vote_tally(_ptr_array(ptrs), len(ptrs), int(d), int(flip_mask),
                               _dev(tally_out, torch.int8, "tally_out", int(d)), _stream(stream)),
           "ss_vote_tally")


def ss_apply_vote(param: torch.Tensor, vote_words: torch.Tensor, lr: float,
                  weight_decay: float = 0.0, stream=None) -> None:
    d = param.numel()
    _check(lib().ss_apply_vote(_dev(param, torch.float32, "param"), _words(vote_words, d, "vote_words"),
                               d, float(lr), float(weight_decay), _stream(stream)), "ss_apply_vote")


def ss_vote_apply(packed: Sequence[torch.Tensor], param: torch.Tensor, lr: float,
                  weight_decay: float = 0.0, flip_mask: int = 0,
                  vote_words_out: Optional[torch.Tensor] = None, stream=None) -> None:
    d = param.numel()
    ptrs = [_words(p, d, "packed[%d]" % m) for m, p in enumerate(packed)]
    w_ptr = None if vote_words_out is None else _words(vote_words_out, d, "vote_words_out")
    _check(lib().ss_vote_apply(_ptr_array(ptrs), len(ptrs), d, int(flip_mask),
                               _dev(param, torch.float32, "param"), float(lr), float(weight_decay),
                               w_ptr, _stream(stream)), "ss_vote_apply")


def _step_args(grads, momenta, param, vote_words_out):
    """Marshalling shared by the fused-step entry points: (dtype code, gradient pointer array,
    momentum pointer array or None, vote pointer or None, M, d)."""
    M = len(grads)
    d = param.numel()
    codes = {_dtype_code(g) for g in grads}
    if len(codes) != 1:
        raise TypeError("all gradients must share one dtype")
    g_ptrs = [_dev(g, None, "grads[%d]" % m, d) for m, g in enumerate(grads)]
    v_arr = None
    if momenta is not None:
        if len(momenta) != M:
            raise ValueError("need one momentum buffer per worker")
        v_arr = _ptr_array([_dev(v, torch.float32, "momenta[%d]" % m, d) for m, v in enumerate(momenta)])
    w_ptr = None if vote_words_out is None else _words(vote_words_out, d, "vote_words_out")
    return codes.pop(), _ptr_array(g_ptrs), v_arr, w_ptr, M, d


def ss_fused_step(grads: Sequence[torch.Tensor], momenta: Optional[Sequence[torch.Tensor]],
                  param: torch.Tensor, beta: float, lr: float, weight_decay: float = 0.0,
                  flip_mask: int = 0, vote_words_out: Optional[torch.Tensor] = None,
                  stream=None) -> None:
    code, g_arr, v_arr, w_ptr, M, d = _step_args(grads, momenta, param, vote_words_out)
    _check(lib().ss_fused_step(g_arr, code, v_arr, M, d, float(beta),
                               int(flip_mask), _dev(param, torch.float32, "param"), float(lr),
                               float(weight_decay), w_ptr, _stream(stream)), "ss_fused_step")


def segment_table(n_segments: int, device) -> torch.Tensor:
    """Device storage for a table of n_segments ss_segment entries (16 bytes each)."""
    return torch.zeros(2 * int(n_segments), dtype=torch.int64, device=device)


def _segments(t: torch.Tensor, n_segments: int) -> int:
    if not t.is_cuda or t.dtype != torch.int64 or not t.is_contiguous() or t.numel() < 2 * n_segments:
        raise ValueError("segments_dev must come from segment_table(n_segments, device)")
    return t.data_ptr()


def ss_segments_upload(begins: Sequence[int], lrs: Sequence[float], weight_decays: Sequence[float],
                       d: int, segments_dev: torch.Tensor, stream=None) -> None:
    n = len(begins)
    if len(lrs) != n or len(weight_decays) != n:
        raise ValueError("begins, lrs and weight_decays must have one entry per tensor")
    host = (ss_segment * max(n, 1))()
    for k in range(n):
        host[k].begin, host[k].lr, host[k].weight_decay = int(begins[k]), float(lrs[k]), float(weight_decays[k])
    _check(lib().ss_segments_upload(ctypes.cast(host, ctypes.c_void_p), n, int(d),
                                    _segments(segments_dev, n), _stream(stream)), "ss_segments_upload")


def ss_fused_step_segments(grads: Sequence[torch.Tensor], momenta: Optional[Sequence[torch.Tensor]],
                           param: torch.Tensor, beta: float, segments_dev: torch.Tensor,
                           n_segments: int, flip_mask: int = 0,
                           vote_words_out: Optional[torch.Tensor] = None, stream=None) -> None:
    code, g_arr, v_arr, w_ptr, M, d = _step_args(grads, momenta, param, vote_words_out)
    _check(lib().ss_fused_step_segments(g_arr, code, v_arr, M, d, float(beta),
                                        int(flip_mask), _dev(param, torch.float32, "param"),
                                        _segments(segments_dev, n_segments), int(n_segments), w_ptr,
                                        _stream(stream)), "ss_fused_step_segments")


def ss_vote_apply_segments(packed: Sequence[torch.Tensor], param: torch.Tensor,
                           segments_dev: torch.Tensor, n_segments: int, flip_mask: int = 0,
                           vote_words_out: Optional[torch.Tensor] = None, stream=None) -> None:
    d = param.numel()
    ptrs = [_words(p, d, "packed[%d]" % m) for m, p in enumerate(packed)]
    w_ptr = None if vote_words_out is None else _words(vote_words_out, d, "vote_words_out")
    _check(lib().ss_vote_apply_segments(_ptr_array(ptrs), len(ptrs), d, int(flip_mask),
                                        _dev(param, torch.float32, "param"),
                                        _segments(segments_dev, n_segments), int(n_segments), w_ptr,
                                        _stream(stream)), "ss_vote_apply_segments")


def ss_apply_vote_segments(param: torch.Tensor, vote_words: torch.Tensor, segments_dev: torch.Tensor,
                           n_segments: int, stream=None) -> None:
    d = param.numel()
    _check(lib().ss_apply_vote_segments(_dev(param, torch.float32, "param"),
                                        _words(vote_words, d, "vote_words"), d,
                                        _segments(segments_dev, n_segments), int(n_segments),
                                        _stream(stream)), "ss_apply_vote_segments")


def _host_step_args(host_grads, momenta, param, host_vote_out):
    """Marshalling shared by the two host-gradient entry points: (dtype code, host pointer array,
    momentum pointer array or None, host vote pointer or None, M, d)."""
    M = len(host_grads)
    d = param.numel()
    codes = {_dtype_code(g) for g in host_grads}
    if len(codes) != 1:
        raise TypeError("all gradients must share one dtype")
    h_ptrs = []
    for m, g in enumerate(host_grads):
        if g.is_cuda or g.dim() != 1 or not g.is_contiguous() or g.numel() != d:
            raise ValueError("host_grads[%d] must be a contiguous 1-D host tensor of d elements" % m)
        h_ptrs.append(g.data_ptr())
    v_arr = None
    if momenta is not None:
        if len(momenta) != M:
            raise ValueError("need one momentum buffer per worker")
        v_arr = _ptr_array([_dev(v, torch.float32, "momenta[%d]" % m, d) for m, v in enumerate(momenta)])
    hv = None
    if host_vote_out is not None:
        if (host_vote_out.is_cuda or host_vote_out.dtype != torch.int32
                or host_vote_out.numel() != ss_packed_words(d) or not host_vote_out.is_contiguous()):
            raise ValueError("host_vote_out must be a contiguous host int32 tensor of ceil(d/32) words")
        hv = host_vote_out.data_ptr()
    return codes.pop(), _ptr_array(h_ptrs), v_arr, hv, M, d


def ss_fused_step_host(host_grads: Sequence[torch.Tensor], staging: Sequence[torch.Tensor],
                       momenta: Optional[Sequence[torch.Tensor]], param: torch.Tensor, beta: float,
                       lr: float, weight_decay: float, flip_mask: int,
                       vote_words_dev: torch.Tensor, host_vote_out: Optional[torch.Tensor],
                       stream=None) -> None:
    code, h_arr, v_arr, hv, M, d = _host_step_args(host_grads, momenta, param, host_vote_out)
    if len(staging) != M:
        raise ValueError("need one staging buffer per worker")
    s_ptrs = [_dev(s, host_grads[0].dtype, "staging[%d]" % m, d) for m, s in enumerate(staging)]
    _check(lib().ss_fused_step_host(h_arr, code, _ptr_array(s_ptrs), v_arr, M, d,
                                    float(beta), int(flip_mask), _dev(param, torch.float32, "param"),
                                    float(lr), float(weight_decay),
                                    _words(vote_words_dev, d, "vote_words_dev"), hv, _stream(stream)),
           "ss_fused_step_host")


def ss_fused_step_host_static(host_grads: Sequence[torch.Tensor],
                              momenta: Optional[Sequence[torch.Tensor]], param: torch.Tensor,
                              beta: float, lr: float, weight_decay: float, flip_mask: int,
                              vote_words_dev: torch.Tensor, host_vote_out: Optional[torch.Tensor],
                              stream=None) -> None:
    """ss_fused_step_host for callers that may not allocate device memory: the gradients are
    staged in a fixed array inside the library (at most SS_STATIC_STAGING_BYTES for all M workers
    together), so no staging tensors are passed. The first call on a device looks up that array's
    address (and, with lazy module loading, is what reserves the array); make it during start-up.
    Calls that overlap on the GPU race on the array."""
    code, h_arr, v_arr, hv, M, d = _host_step_args(host_grads, momenta, param, host_vote_out)
    _check(lib().ss_fused_step_host_static(h_arr, code, v_arr, M, d, float(beta),
                                           int(flip_mask), _dev(param, torch.float32, "param"),
                                           float(lr), float(weight_decay),
                                           _words(vote_words_dev, d, "vote_words_dev"), hv,
                                           _stream(stream)), "ss_fused_step_host_static")


# ---- the comparison codec of Appendix B (1-bit max-norm QSGD) -------------------------------

def ss_ternary_words(d: int) -> int:
    return int(lib().ss_ternary_words(int(d)))


def ss_absmax(grad: torch.Tensor, absmax_dev: torch.Tensor, stream=None) -> None:
    _check(lib().ss_absmax(_dev(grad, None, "grad"), _dtype_code(grad), grad.numel(),
                           _dev(absmax_dev, torch.float32, "absmax_dev", 1), _stream(stream)), "ss_absmax")


def ss_ternary_pack(grad: torch.Tensor, absmax_dev: torch.Tensor, seed: int, out_codes: torch.Tensor,
                    stream=None) -> None:
    d = grad.numel()
    _check(lib().ss_ternary_pack(_dev(grad, None, "grad"), _dtype_code(grad), d,
                                 _dev(absmax_dev, torch.float32, "absmax_dev", 1), int(seed),
                                 _dev(out_codes, torch.int32, "out_codes", ss_ternary_words(d)),
                                 _stream(stream)), "ss_ternary_pack")


def ss_ternary_unpack(codes: torch.Tensor, scale_dev: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    d = out.numel()
    _check(lib().ss_ternary_unpack(_dev(codes, torch.int32, "codes", ss_ternary_words(d)), d,
                                   _dev(scale_dev, torch.float32, "scale_dev", 1),
                                   _dev(out, torch.float32, "out"), _stream(stream)), "ss_ternary_unpack")


# ---- flag-ordered exchange (one worker per GPU) -------------------------------------------------

def flag_array(device) -> torch.Tensor:
    """Storage for one worker's flag array: SS_MAX_WORKERS words, zeroed (epoch 0 = nothing arrived)."""
    return torch.zeros(SS_MAX_WORKERS, dtype=torch.int32, device=device)


def ss_flags_signal(flags: Sequence, index: int, epoch: int, stream=None) -> None:
    """``flags`` may be tensors on this GPU or raw integer addresses of peers' flag arrays."""
    ptrs = [p if isinstance(p, int) else _dev(p, torch.int32, "flags[%d]" % i) for i, p in enumerate(flags)]
    _check(lib().ss_flags_signal(_ptr_array(ptrs), len(ptrs), int(index), int(epoch) & 0xFFFFFFFF,
                                 _stream(stream)), "ss_flags_signal")


def ss_flags_wait(flags_local: torch.Tensor, M: int, epoch: int, timeout_ns: int, status_dev: torch.Tensor,
                  stream=None) -> None:
    _check(lib().ss_flags_wait(_dev(flags_local, torch.int32, "flags_local"), int(M), int(epoch) & 0xFFFFFFFF,
                               int(timeout_ns), _dev(status_dev, torch.int32, "status_dev", 1),
                               _stream(stream)), "ss_flags_wait")


def ss_flags_signal_wait(flags: Sequence, index: int, flags_local: torch.Tensor, M: int, epoch: int,
                         timeout_ns: int, status_dev: torch.Tensor, stream=None) -> None:
    ptrs = [p if isinstance(p, int) else _dev(p, torch.int32, "flags[%d]" % i) for i, p in enumerate(flags)]
    _check(lib().ss_flags_signal_wait(_ptr_array(ptrs), len(ptrs), int(index),
                                      _dev(flags_local, torch.int32, "flags_local"), int(M),
                                      int(epoch) & 0xFFFFFFFF, int(timeout_ns),
                                      _dev(status_dev, torch.int32, "status_dev", 1), _stream(stream)),
           "ss_flags_signal_wait")


def ss_vote_apply_guarded(packed: Sequence[torch.Tensor], param: torch.Tensor, lr: float,
                          weight_decay: float, flip_mask: int, vote_words_out: Optional[torch.Tensor],
                          skip_if_nonzero_dev: torch.Tensor, stream=None) -> None:
    d = param.numel()
    ptrs = [_words(p, d, "packed[%d]" % m) for m, p in enumerate(packed)]
    w_ptr = None if vote_words_out is None else _words(vote_words_out, d, "vote_words_out")
    _check(lib().ss_vote_apply_guarded(_ptr_array(ptrs), len(ptrs), d, int(flip_mask),
                                       _dev(param, torch.float32, "param"), float(lr), float(weight_decay),
                                       w_ptr, _dev(skip_if_nonzero_dev, torch.int32, "skip_if_nonzero_dev", 1),
                                       _stream(stream)), "ss_vote_apply_guarded")


def ss_vote_apply_guarded_segments(packed: Sequence[torch.Tensor], param: torch.Tensor,
                                   segments_dev: torch.Tensor, n_segments: int, flip_mask: int,
                                   vote_words_out: Optional[torch.Tensor], skip_if_nonzero_dev: torch.Tensor,
                                   stream=None) -> None:
    d = param.numel()
    ptrs = [_words(p, d, "packed[%d]" % m) for m, p in enumerate(packed)]
    w_ptr = None if vote_words_out is None else _words(vote_words_out, d, "vote_words_out")
    _check(lib().ss_vote_apply_guarded_segments(_ptr_array(ptrs), len(ptrs), d, int(flip_mask),
                                                _dev(param, torch.float32, "param"),
                                                _segments(segments_dev, n_segments), int(n_segments), w_ptr,
                                                _dev(skip_if_nonzero_dev, torch.int32, "skip_if_nonzero_dev", 1),
                                                _stream(stream)), "ss_vote_apply_guarded_segments")


# ---- training operators (include/signsgd_train.h) -----------------------------------------------

def _mat(t: torch.Tensor, dtype, name: str, shape=None):
    """(address, row stride) of a 2-D CUDA tensor with unit column stride (one without elements has none)."""
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError("%s must have shape %s, has %s" % (name, "[rows, cols]" if shape is None else list(shape), list(t.shape)))
    stride, unit = t.stride()
    if unit != 1 and t.shape[1] > 1 and t.shape[0] > 0:
        raise ValueError("%s must have unit column stride" % name)
    return t.data_ptr(), stride


def _vec(t: torch.Tensor, dtype, name: str, n: int) -> int:
    if t.dtype is dtype and t.is_cuda and t.dim() == 1 and t.numel() == n and t.is_contiguous():
        return t.data_ptr()
    raise (ValueError if t.dtype is dtype else TypeError)("%s must be a contiguous CUDA tensor of %d %s" % (name, n, dtype))


def _opt_vec(t: Optional[torch.Tensor], dtype, name: str, n: int) -> Optional[int]:
    return None if t is None else _vec(t, dtype, name, n)


def _scratch(workspace: Optional[torch.Tensor], need: int, like: torch.Tensor, stream):
    """(address, bytes) of the caller's workspace, or of one of the size asked for from PyTorch's
    allocator, and the tensor to keep until the call returns (its memory is safe after that: it
    belongs to the call's stream, and is given out again in the order of that stream)."""
    if workspace is None:
        if need <= 0:
            return None, 0, None
        if stream is None:
            workspace = like.new_empty(need, dtype=torch.uint8)
        else:
            own = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), like.device)
            with torch.cuda.stream(own):
                workspace = like.new_empty(need, dtype=torch.uint8)
    elif not workspace.is_cuda or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA uint8 tensor")
    return workspace.data_ptr(), workspace.numel(), workspace


def ss_act8_bytes(rows: int, cols: int) -> int:
    return int(lib().ss_act8_bytes(int(rows), int(cols)))


def act8_checkpoint(rows: int, cols: int, device) -> torch.Tensor:
    """Storage for the 8-bit checkpoint of a [rows, cols] matrix."""
    return torch.empty(ss_act8_bytes(rows, cols), dtype=torch.uint8, device=device)


def _ckpt(t: torch.Tensor, rows: int, cols: int, name: str) -> int:
    return _vec(t, torch.uint8, name, rows * (SS_ACT8_GROUP + 1) * -(-cols // SS_ACT8_GROUP))


def _written(tensors) -> None:
    """Tells autograd that a kernel wrote to these, so that a checkpoint which a backward pass has yet to read is not
    written again without a word."""
    try:
        torch._C._increment_version(tensors)
    except RuntimeError:  # inference tensors, which no backward pass reads, have no version
        torch._C._increment_version([t for t in tensors if not t.is_inference()])


def ss_act8_pack(x: torch.Tensor, ckpt: torch.Tensor, stream=None) -> None:
    code, (ptr, stride) = _dtype_code(x), _mat(x, x.dtype, "x")
    rows, cols = x.shape
    _check(lib().ss_act8_pack(ptr, stride, code, rows, cols, _ckpt(ckpt, rows, cols, "ckpt"), _stream(stream)),
           "ss_act8_pack")
    _written((ckpt,))


def ss_act8_unpack(ckpt: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    code, (ptr, stride) = _dtype_code(out), _mat(out, out.dtype, "out")
    rows, cols = out.shape
    _check(lib().ss_act8_unpack(_ckpt(ckpt, rows, cols, "ckpt"), rows, cols, ptr, stride, code, _stream(stream)),
           "ss_act8_unpack")


def ss_act8_forward(x: torch.Tensor, up: Optional[torch.Tensor], act: int, y: torch.Tensor,
                    ckpt_x: Optional[torch.Tensor] = None, ckpt_up: Optional[torch.Tensor] = None, ckpt_y: Optional[torch.Tensor] = None,
                    stream=None) -> None:
    code, dt, shape = _dtype_code(x), x.dtype, x.shape
    x_ptr, x_stride = _mat(x, dt, "x")
    rows, cols = shape
    u_ptr, u_stride = (None, 0) if up is None else _mat(up, dt, "up", shape)
    y_ptr, y_stride = _mat(y, dt, "y", shape)
    _check(lib().ss_act8_forward(x_ptr, x_stride, u_ptr, u_stride, code, act, rows, cols, y_ptr, y_stride,
                                 None if ckpt_x is None else _ckpt(ckpt_x, rows, cols, "ckpt_x"),
                                 None if ckpt_up is None else _ckpt(ckpt_up, rows, cols, "ckpt_up"),
                                 None if ckpt_y is None else _ckpt(ckpt_y, rows, cols, "ckpt_y"), _stream(stream)),
           "ss_act8_forward")
    _written([c for c in (ckpt_x, ckpt_up, ckpt_y) if c is not None])


def ss_act8_backward(dy: torch.Tensor, ckpt_x: torch.Tensor, ckpt_up: Optional[torch.Tensor], act: int,
                     dx: torch.Tensor, dup: Optional[torch.Tensor] = None, stream=None) -> None:
    code, dt, shape = _dtype_code(dy), dy.dtype, dy.shape
    dy_ptr, dy_stride = _mat(dy, dt, "dy")
    rows, cols = shape
    dx_ptr, dx_stride = _mat(dx, dt, "dx", shape)
    du_ptr, du_stride = (None, 0) if dup is None else _mat(dup, dt, "dup", shape)
    _check(lib().ss_act8_backward(dy_ptr, dy_stride, _ckpt(ckpt_x, rows, cols, "ckpt_x"),
                                  None if ckpt_up is None else _ckpt(ckpt_up, rows, cols, "ckpt_up"), code, act, rows,
                                  cols, dx_ptr, dx_stride, du_ptr, du_stride, _stream(stream)), "ss_act8_backward")


def ss_weight_grad8_workspace(dy: torch.Tensor, n_in: int) -> int:
    ptr, stride = _mat(dy, dy.dtype, "dy")
    return int(lib().ss_weight_grad8_workspace(ptr, stride, _dtype_code(dy), dy.shape[0], dy.shape[1], int(n_in)))


def ss_weight_grad8(dy: torch.Tensor, ckpt_x: torch.Tensor, dw: torch.Tensor, accumulate: bool = False,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    code, (dy_ptr, dy_stride) = _dtype_code(dy), _mat(dy, dy.dtype, "dy")
    rows, n_out = dy.shape
    dw_ptr, dw_stride = _mat(dw, torch.float32, "dw")
    if dw.shape[0] != n_out:
        raise ValueError("dw must have one row for each of dy's %d columns" % n_out)
    n_in = dw.shape[1]
    L = lib()
    need = 0 if workspace is not None else L.ss_weight_grad8_workspace(dy_ptr, dy_stride, code, rows, n_out, n_in)
    w_ptr, w_bytes, workspace = _scratch(workspace, need, dy, stream)
    _check(L.ss_weight_grad8(dy_ptr, dy_stride, code, _ckpt(ckpt_x, rows, n_in, "ckpt_x"), rows, n_out, n_in, dw_ptr,
                             dw_stride, int(bool(accumulate)), w_ptr, w_bytes, _stream(stream)), "ss_weight_grad8")


@functools.lru_cache(maxsize=256)
def ss_loss_workspace(rows: int, n_pairs: int = 0) -> int:
    return int(lib().ss_loss_workspace(int(rows), int(n_pairs)))


def ss_policy_loss(logits: torch.Tensor, targets: torch.Tensor, old_logp: torch.Tensor,
                   ref_logp: Optional[torch.Tensor], advantages: torch.Tensor, weights: torch.Tensor,
                   totals: torch.Tensor, logp: torch.Tensor, dlogits: Optional[torch.Tensor] = None,
                   inv_temperature: float = 1.0, clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                   grad_scale: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                   stream=None) -> None:
    f32, code = torch.float32, _dtype_code(logits)
    z_ptr, z_stride = _mat(logits, logits.dtype, "logits")
    rows, vocab = logits.shape
    d_ptr, d_stride = (None, 0) if dlogits is None else _mat(dlogits, logits.dtype, "dlogits", logits.shape)
    L = lib()
    w_ptr, w_bytes, workspace = _scratch(workspace, ss_loss_workspace(rows, 0), logits, stream)
    _check(L.ss_policy_loss(z_ptr, z_stride, code, rows, vocab, _vec(targets, torch.int64, "targets", rows),
                            _vec(old_logp, f32, "old_logp", rows), _opt_vec(ref_logp, f32, "ref_logp", rows),
                            _vec(advantages, f32, "advantages", rows), _vec(weights, f32, "weights", rows),
                            inv_temperature, clip_low, clip_high, kl_coef, _opt_vec(grad_scale, f32, "grad_scale", 1),
                            _vec(totals, f32, "totals", 3), _vec(logp, f32, "logp", rows), d_ptr, d_stride,
                            w_ptr, w_bytes, _stream(stream)), "ss_policy_loss")


def ss_preference_loss(logits: torch.Tensor, targets: torch.Tensor, weights: torch.Tensor, seq_begin: torch.Tensor,
                       ref_seq_logp: torch.Tensor, loss: torch.Tensor, margins: torch.Tensor, seq_logp: torch.Tensor,
                       logp: torch.Tensor, dlogits: Optional[torch.Tensor] = None, inv_temperature: float = 1.0,
                       kind: int = SS_PREF_SIGMOID, beta: float = 0.1, label_smoothing: float = 0.0,
                       scale: float = 1.0, grad_scale: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    f32, i64, code = torch.float32, torch.int64, _dtype_code(logits)
    z_ptr, z_stride = _mat(logits, logits.dtype, "logits")
    rows, vocab = logits.shape
    pairs = margins.shape[0]
    d_ptr, d_stride = (None, 0) if dlogits is None else _mat(dlogits, logits.dtype, "dlogits", logits.shape)
    L = lib()
    w_ptr, w_bytes, workspace = _scratch(workspace, ss_loss_workspace(rows, pairs), logits, stream)
    _check(L.ss_preference_loss(z_ptr, z_stride, code, rows, vocab, _vec(targets, i64, "targets", rows),
                                _vec(weights, f32, "weights", rows), _vec(seq_begin, i64, "seq_begin", 2 * pairs + 1),
                                pairs, _vec(ref_seq_logp, f32, "ref_seq_logp", 2 * pairs), inv_temperature, kind, beta,
                                label_smoothing, scale, _opt_vec(grad_scale, f32, "grad_scale", 1),
                                _vec(loss, f32, "loss", 1), _vec(margins, f32, "margins", pairs),
                                _vec(seq_logp, f32, "seq_logp", 2 * pairs), _vec(logp, f32, "logp", rows), d_ptr,
                                d_stride, w_ptr, w_bytes, _stream(stream)), "ss_preference_loss")
