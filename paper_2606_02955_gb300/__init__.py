"""Python binding of libfdllm.so: Frechet profile commit-set selection on GB300 (sm_103a).

The functions carry the names of the C interface (include/fdllm.h) and only marshal
arguments: every step of the selection runs in the library's CUDA kernels.  PyTorch
supplies device memory and the current stream.  The first call loads the compiled library
and raises when it has not been built (``paper_2606_02955_gb300.build``); there is no
fallback implementation.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

from .build import LIB_PATH

__all__ = [
    "BF16", "FP32", "FP16", "PROFILE", "FACTOR", "THRESHOLD", "ROW_NONFINITE", "ROW_DEVICE_ERROR",
    "FdllmError", "fdllm_select", "fdllm_select_ws", "fdllm_workspace_bytes",
    "fdllm_confidence", "fdllm_select_from_conf", "fdllm_device_status",
    "fdllm_workspace_status", "fdllm_static_status", "fdllm_release_workspace",
    "fdllm_status_string",
    "fdllm_version", "library_path", "fdllm_select_static", "fdllm_select_robust",
    "fdllm_profile_terms", "fdllm_check_bounded_wait", "fdllm_decode_loop", "FORWARD_FN",
    "fdllm_lmhead_select", "fdllm_lmhead_confidence", "fdllm_lmhead_logits",
    "fdllm_gather_masked_rows", "fdllm_decode_loop_lmhead", "fdllm_vocab_reduce",
    "fdllm_select_host",
    "KvCache", "fdllm_qk_norm_rope", "fdllm_cache_append", "fdllm_cache_read",
    "fdllm_cache_attention", "fdllm_cache_attention_workspace_bytes",
    "fdllm_cache_key_weights", "fdllm_cache_evict", "fdllm_cache_status",
    "fdllm_cache_check_wait",
]

BF16, FP32, FP16 = 0, 1, 2
PROFILE, FACTOR, THRESHOLD = 0, 1, 2
ROW_NONFINITE, ROW_DEVICE_ERROR = -1, -2
OK, ERR_ARG, ERR_ALIGN, ERR_NONFINITE, ERR_CUDA, ERR_WORKSPACE, ERR_DEVICE = range(7)
MODES = {"profile": PROFILE, "factor": FACTOR, "threshold": THRESHOLD}

_lib = None

# fdllm_forward_fn: (user, loop_state, block_mask, logits, stream) -> int
FORWARD_FN = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                              ctypes.c_void_p, ctypes.c_void_p)


def _load():
    """Load libfdllm.so once; a missing library is an error, never a fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libfdllm.so is not built (%s); run paper_2606_02955_gb300.build.build_library() "
            "or __graft_entry__.build()" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    p, i, d, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_double, ctypes.c_size_t
    lib.fdllm_select.argtypes = [p, i, i, i, i, p, d, i, p, p, p, p]
    lib.fdllm_select.restype = i
    lib.fdllm_select_ws.argtypes = [p, i, i, i, i, p, d, i, p, p, p, p, sz, p]
    lib.fdllm_select_ws.restype = i
    lib.fdllm_select_robust.argtypes = [p, i, i, i, i, p, d, d, p, p, p, p, p]
    lib.fdllm_select_robust.restype = i
    lib.fdllm_select_static.argtypes = [p, i, i, i, i, p, d, i, p, p, p, p]
    lib.fdllm_select_static.restype = i
    lib.fdllm_workspace_bytes.argtypes = [i, i, i, i]
    lib.fdllm_workspace_bytes.restype = sz
    lib.fdllm_lmhead_select.argtypes = [p, p, i, i, i, i, p, d, i, p, p, p, p]
    lib.fdllm_lmhead_select.restype = i
    lib.fdllm_lmhead_confidence.argtypes = [p, p, i, i, i, i, p, p, p, p]
    lib.fdllm_lmhead_confidence.restype = i
    lib.fdllm_lmhead_logits.argtypes = [p, p, i, i, i, i, p, p, p]
    lib.fdllm_lmhead_logits.restype = i
    lib.fdllm_gather_masked_rows.argtypes = [p, p, i, i, i, i, p, p]
    lib.fdllm_gather_masked_rows.restype = i
    lib.fdllm_confidence.argtypes = [p, i, i, i, i, p, p, p, p]
    lib.fdllm_confidence.restype = i
    lib.fdllm_vocab_reduce.argtypes = [p, i, i, i, i, p, p]
    lib.fdllm_vocab_reduce.restype = i
    lib.fdllm_select_from_conf.argtypes = [p, p, i, i, p, d, i, p, p, p, p]
    lib.fdllm_select_from_conf.restype = i
    lib.fdllm_profile_terms.argtypes = [p, p, i, i, d, p, p, p, p, p, p]
    lib.fdllm_profile_terms.restype = i
    lib.fdllm_decode_loop.argtypes = [i, i, i, i, i, d, i, FORWARD_FN, p, p, p, p, i,
                                      ctypes.POINTER(ctypes.c_int), p]
    lib.fdllm_decode_loop.restype = i
    lib.fdllm_decode_loop_lmhead.argtypes = [i, i, i, i, i, p, d, i, FORWARD_FN, p, p, p, p, i,
                                             ctypes.POINTER(ctypes.c_int), p]
    lib.fdllm_decode_loop_lmhead.restype = i
    lib.fdllm_qk_norm_rope.argtypes = [p, p, p, p, i, i, i, i, i, p, p, d, p, i, p, p, i, i, p,
                                       p, p]
    lib.fdllm_qk_norm_rope.restype = i
    lib.fdllm_cache_append.argtypes = [p, p, i, i, p, p, p, p, p, p, i, i, p]
    lib.fdllm_cache_append.restype = i
    lib.fdllm_cache_read.argtypes = [p, p, i, i, p, p, p, p, i, i, p]
    lib.fdllm_cache_read.restype = i
    lib.fdllm_cache_attention.argtypes = [p, p, i, i, i, i, p, p, i, p, p, p, p, p, i, p, i, d, p,
                                          p, p, sz, p]
    lib.fdllm_cache_attention.restype = i
    lib.fdllm_cache_attention_workspace_bytes.argtypes = [i, i, i, i, i]
    lib.fdllm_cache_attention_workspace_bytes.restype = sz
    lib.fdllm_cache_key_weights.argtypes = [p, p, i, i, i, i, p, p, i, p, p, d, p, p, i, p]
    lib.fdllm_cache_key_weights.restype = i
    lib.fdllm_cache_evict.argtypes = [p, p, i, i, p, p, i, i, i, i, p, i, p, p, p, p]
    lib.fdllm_cache_evict.restype = i
    lib.fdllm_cache_status.argtypes = [p]
    lib.fdllm_cache_status.restype = i
    lib.fdllm_cache_check_wait.argtypes = [i, p]
    lib.fdllm_cache_check_wait.restype = i
    lib.fdllm_check_bounded_wait.argtypes = [d, p]
    lib.fdllm_check_bounded_wait.restype = i
    lib.fdllm_device_status.argtypes = [p]
    lib.fdllm_device_status.restype = i
    lib.fdllm_workspace_status.argtypes = [p, p]
    lib.fdllm_workspace_status.restype = i
    lib.fdllm_static_status.argtypes = [p]
    lib.fdllm_static_status.restype = i
    lib.fdllm_select_host.argtypes = [p, i, i, i, i, p, d, i, p, p, p, p]
    lib.fdllm_select_host.restype = i
    lib.fdllm_release_workspace.argtypes = []
    lib.fdllm_release_workspace.restype = None
    lib.fdllm_status_string.argtypes = [i]
    lib.fdllm_status_string.restype = ctypes.c_char_p
    lib.fdllm_version.argtypes = []
    lib.fdllm_version.restype = i
    _lib = lib
    return lib


class FdllmError(RuntimeError):
    def __init__(self, status: int, call: str):
        super().__init__("%s failed: status %d (%s)" % (call, status, fdllm_status_string(status)))
        self.status = status


def library_path() -> str:
    return LIB_PATH



def _on_device(fn):
    """Runs an entry point on the device of its CUDA tensor arguments (the library works on
    the current device: its workspace and launches), and rejects calls whose CUDA tensors
    live on different devices."""
    @functools.wraps(fn)
    def call(*args, **kwargs):
        cuda = [a for a in (*args, *kwargs.values()) if isinstance(a, torch.Tensor) and a.is_cuda]
        if not cuda:
            return fn(*args, **kwargs)
        dev = cuda[0].device
        for t in cuda[1:]:
            if t.device != dev:
                raise ValueError("the CUDA tensors of one call must share a device (%s, %s)"
                                 % (dev, t.device))
        with torch.cuda.device(dev):
            return fn(*args, **kwargs)
    return call


def fdllm_status_string(status: int) -> str:
    return _load().fdllm_status_string(int(status)).decode()


def fdllm_version() -> int:
    return _load().fdllm_version()


def _check(status: int, call: str):
    if status != 0:
        raise FdllmError(status, call)


def _mode(mode) -> int:
    return MODES[mode] if isinstance(mode, str) else int(mode)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return FP32
    if t.dtype == torch.float16:
        return FP16
    raise TypeError("logits must be bfloat16, float16 or float32, got %s" % t.dtype)


def _stream(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _dev(t: torch.Tensor, name: str, dtype=None, shape=None):
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    return t.data_ptr()


def _outputs(B, L, device, out_tokens, out_commit, out_n):
    if out_tokens is None:
        out_tokens = torch.full((B, L), -1, dtype=torch.int32, device=device)
    if out_commit is None:
        out_commit = torch.empty((B, L), dtype=torch.uint8, device=device)
    if out_n is None:
        out_n = torch.empty((B,), dtype=torch.int32, device=device)
    return out_tokens, out_commit, out_n


@_on_device
def fdllm_select(logits: torch.Tensor, mask: torch.Tensor, param: float, mode=PROFILE,
                 out_tokens=None, out_commit=None, out_n=None, stream=None):
    """One selection step (fdllm_select).  ``logits`` [B, L, V] bf16/fp16/fp32, ``mask`` [B, L]
    uint8 (updated in place).  Returns (out_tokens, out_commit, out_n).

    Device tensors run asynchronously on ``stream`` (default: current stream).  With host
    tensors the call copies the inputs to the current CUDA device (pinned memory makes the
    copies asynchronous), runs the step, copies the outputs and the updated mask back and
    synchronises: the end-to-end form of the call."""
    if not logits.is_cuda:
        return _select_from_host(logits, mask, param, mode, out_tokens, out_commit, out_n)
    B, L, V = logits.shape
    lp = _dev(logits, "logits")
    mp = _dev(mask, "mask", torch.uint8, (B, L))
    out_tokens, out_commit, out_n = _outputs(B, L, logits.device, out_tokens, out_commit, out_n)
    st = _load().fdllm_select(lp, _dtype_code(logits), B, L, V, mp, float(param), _mode(mode),
                           _dev(out_tokens, "out_tokens", torch.int32, (B, L)),
                           _dev(out_commit, "out_commit", torch.uint8, (B, L)),
                           _dev(out_n, "out_n", torch.int32, (B,)), _stream(stream))
    _check(st, "fdllm_select")
    return out_tokens, out_commit, out_n


def _select_from_host(logits, mask, param, mode, out_tokens, out_commit, out_n):
    """fdllm_select_host: the whole step on host tensors in one library call (the GPU reads
    only the masked rows of page-locked logits; results and mask copied back)."""
    B, L, V = logits.shape
    if not logits.is_contiguous():
        raise FdllmError(1, "fdllm_select_host: contiguous logits required")
    pin = logits.is_pinned()

    def host(t, name, dtype, shape, fill=None):
        if t is None:
            t = torch.empty(shape, dtype=dtype, pin_memory=pin)
            if fill is not None:
                t.fill_(fill)
        if t.is_cuda or t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
            raise FdllmError(1, "%s: contiguous host %s %s required" % (name, dtype, shape))
        return t

    mask = host(mask, "mask", torch.uint8, (B, L))
    out_tokens = host(out_tokens, "out_tokens", torch.int32, (B, L), -1)
    out_commit = host(out_commit, "out_commit", torch.uint8, (B, L))
    out_n = host(out_n, "out_n", torch.int32, (B,))
    st = _load().fdllm_select_host(logits.data_ptr(), _dtype_code(logits), B, L, V,
                                   mask.data_ptr(), float(param), _mode(mode),
                                   out_tokens.data_ptr(), out_commit.data_ptr(),
                                   out_n.data_ptr(), _stream(None))
    _check(st, "fdllm_select_host")
    return out_tokens, out_commit, out_n


@_on_device
def fdllm_select_robust(logits: torch.Tensor, mask: torch.Tensor, param: float, eta: float = 0.0,
                        eta_per_position=None, out_tokens=None, out_commit=None, out_n=None,
                        stream=None):
    """Calibration-robust profile selection (App. C): confidences lowered to
    max(0, c - eta) (``eta_per_position``: [B, L] fp32 CUDA tensor, else the uniform eta)
    before the profile rule.  Returns (out_tokens, out_commit, out_n)."""
    B, L, V = logits.shape
    out_tokens, out_commit, out_n = _outputs(B, L, logits.device, out_tokens, out_commit, out_n)
    ep = None if eta_per_position is None else _dev(eta_per_position, "eta_per_position",
                                                     torch.float32, (B, L))
    st = _load().fdllm_select_robust(_dev(logits, "logits"), _dtype_code(logits), B, L, V,
                                     _dev(mask, "mask", torch.uint8, (B, L)), float(param),
                                     float(eta), ep,
                                     _dev(out_tokens, "out_tokens", torch.int32, (B, L)),
                                     _dev(out_commit, "out_commit", torch.uint8, (B, L)),
                                     _dev(out_n, "out_n", torch.int32, (B,)), _stream(stream))
    _check(st, "fdllm_select_robust")
    return out_tokens, out_commit, out_n


@_on_device
def fdllm_select_static(logits: torch.Tensor, mask: torch.Tensor, param: float, mode=PROFILE,
                        out_tokens=None, out_commit=None, out_n=None, stream=None):
    """fdllm_select using the library's fixed device scratch array instead of an allocated
    workspace (for callers that cannot allocate while stepping).  Pass preallocated outputs
    to keep the call free of allocations on the Python side too."""
    B, L, V = logits.shape
    out_tokens, out_commit, out_n = _outputs(B, L, logits.device, out_tokens, out_commit, out_n)
    st = _load().fdllm_select_static(_dev(logits, "logits"), _dtype_code(logits), B, L, V,
                                     _dev(mask, "mask", torch.uint8, (B, L)), float(param),
                                     _mode(mode),
                                     _dev(out_tokens, "out_tokens", torch.int32, (B, L)),
                                     _dev(out_commit, "out_commit", torch.uint8, (B, L)),
                                     _dev(out_n, "out_n", torch.int32, (B,)), _stream(stream))
    _check(st, "fdllm_select_static")
    return out_tokens, out_commit, out_n


def fdllm_workspace_bytes(B: int, L: int, V: int, dtype=BF16) -> int:
    return int(_load().fdllm_workspace_bytes(B, L, V, dtype))


@_on_device
def fdllm_select_ws(logits: torch.Tensor, mask: torch.Tensor, param: float, mode,
                    workspace: torch.Tensor, out_tokens=None, out_commit=None, out_n=None,
                    stream=None):
    """fdllm_select with a caller workspace (a zero-filled uint8 CUDA tensor of at least
    fdllm_workspace_bytes bytes, 256-byte aligned as torch allocations are)."""
    B, L, V = logits.shape
    out_tokens, out_commit, out_n = _outputs(B, L, logits.device, out_tokens, out_commit, out_n)
    st = _load().fdllm_select_ws(_dev(logits, "logits"), _dtype_code(logits), B, L, V,
                              _dev(mask, "mask", torch.uint8, (B, L)), float(param), _mode(mode),
                              _dev(out_tokens, "out_tokens", torch.int32, (B, L)),
                              _dev(out_commit, "out_commit", torch.uint8, (B, L)),
                              _dev(out_n, "out_n", torch.int32, (B,)),
                              _dev(workspace, "workspace", torch.uint8),
                              workspace.numel(), _stream(stream))
    _check(st, "fdllm_select_ws")
    return out_tokens, out_commit, out_n


@_on_device
def fdllm_confidence(logits: torch.Tensor, mask: torch.Tensor, out_conf=None, out_argmax=None,
                     stream=None):
    """Step a1 alone: (conf fp32 [B, L], argmax int32 [B, L]) written at masked positions
    (unwritten positions of freshly allocated outputs hold NaN / -1)."""
    B, L, V = logits.shape
    if out_conf is None:
        out_conf = torch.full((B, L), float("nan"), dtype=torch.float32, device=logits.device)
    if out_argmax is None:
        out_argmax = torch.full((B, L), -1, dtype=torch.int32, device=logits.device)
    st = _load().fdllm_confidence(_dev(logits, "logits"), _dtype_code(logits), B, L, V,
                               _dev(mask, "mask", torch.uint8, (B, L)),
                               _dev(out_conf, "out_conf", torch.float32, (B, L)),
                               _dev(out_argmax, "out_argmax", torch.int32, (B, L)),
                               _stream(stream))
    _check(st, "fdllm_confidence")
    return out_conf, out_argmax


@_on_device
def fdllm_vocab_reduce(logits: torch.Tensor, mask: torch.Tensor, stream=None):
    """Step a1's vocabulary reduction alone (unit partials in the library workspace, not
    folded into confidences), for timing the reduction kernel by itself."""
    B, L, V = logits.shape
    st = _load().fdllm_vocab_reduce(_dev(logits, "logits"), _dtype_code(logits), B, L, V,
                                    _dev(mask, "mask", torch.uint8, (B, L)), _stream(stream))
    _check(st, "fdllm_vocab_reduce")


def _lmhead_shapes(hidden: torch.Tensor, w_vocab: torch.Tensor):
    B, L, H = hidden.shape
    V, H2 = w_vocab.shape
    if H2 != H:
        raise ValueError("w_vocab must be [V, %d], got %s" % (H, tuple(w_vocab.shape)))
    hp = _dev(hidden, "hidden", torch.bfloat16)
    wp = _dev(w_vocab, "w_vocab", torch.bfloat16)
    return B, L, H, V, hp, wp


@_on_device
def fdllm_lmhead_select(hidden: torch.Tensor, w_vocab: torch.Tensor, mask: torch.Tensor,
                        param: float, mode=PROFILE, out_tokens=None, out_commit=None, out_n=None,
                        stream=None):
    """One selection step with the logits computed and reduced inside the LM-head GEMM
    (fdllm_lmhead_select): ``hidden`` [B, L, H] bf16, ``w_vocab`` [V, H] bf16, ``mask``
    [B, L] uint8 (updated in place).  Returns (out_tokens, out_commit, out_n)."""
    B, L, H, V, hp, wp = _lmhead_shapes(hidden, w_vocab)
    out_tokens, out_commit, out_n = _outputs(B, L, hidden.device, out_tokens, out_commit, out_n)
    st = _load().fdllm_lmhead_select(hp, wp, B, L, H, V, _dev(mask, "mask", torch.uint8, (B, L)),
                                     float(param), _mode(mode),
                                     _dev(out_tokens, "out_tokens", torch.int32, (B, L)),
                                     _dev(out_commit, "out_commit", torch.uint8, (B, L)),
                                     _dev(out_n, "out_n", torch.int32, (B,)), _stream(stream))
    _check(st, "fdllm_lmhead_select")
    return out_tokens, out_commit, out_n


@_on_device
def fdllm_lmhead_confidence(hidden: torch.Tensor, w_vocab: torch.Tensor, mask: torch.Tensor,
                            out_conf=None, out_argmax=None, stream=None):
    """Step a1 on the LM head: (conf fp32 [B, L], argmax int32 [B, L]) at masked positions."""
    B, L, H, V, hp, wp = _lmhead_shapes(hidden, w_vocab)
    if out_conf is None:
        out_conf = torch.full((B, L), float("nan"), dtype=torch.float32, device=hidden.device)
    if out_argmax is None:
        out_argmax = torch.full((B, L), -1, dtype=torch.int32, device=hidden.device)
    st = _load().fdllm_lmhead_confidence(hp, wp, B, L, H, V,
                                         _dev(mask, "mask", torch.uint8, (B, L)),
                                         _dev(out_conf, "out_conf", torch.float32, (B, L)),
                                         _dev(out_argmax, "out_argmax", torch.int32, (B, L)),
                                         _stream(stream))
    _check(st, "fdllm_lmhead_confidence")
    return out_conf, out_argmax


@_on_device
def fdllm_lmhead_logits(hidden: torch.Tensor, w_vocab: torch.Tensor, mask: torch.Tensor,
                        out_logits=None, stream=None):
    """The LM-head GEMM's fp32 logits [B, L, V] at masked rows (other rows untouched; a
    freshly allocated output holds NaN there)."""
    B, L, H, V, hp, wp = _lmhead_shapes(hidden, w_vocab)
    if out_logits is None:
        out_logits = torch.full((B, L, V), float("nan"), dtype=torch.float32,
                                device=hidden.device)
    st = _load().fdllm_lmhead_logits(hp, wp, B, L, H, V, _dev(mask, "mask", torch.uint8, (B, L)),
                                     _dev(out_logits, "out_logits", torch.float32, (B, L, V)),
                                     _stream(stream))
    _check(st, "fdllm_lmhead_logits")
    return out_logits


@_on_device
def fdllm_select_from_conf(conf: torch.Tensor, argmax: torch.Tensor, mask: torch.Tensor,
                           param: float, mode=PROFILE, out_tokens=None, out_commit=None,
                           out_n=None, stream=None):
    """Steps a2-a5 alone on given confidences; returns (out_tokens, out_commit, out_n)."""
    B, L = conf.shape
    out_tokens, out_commit, out_n = _outputs(B, L, conf.device, out_tokens, out_commit, out_n)
    st = _load().fdllm_select_from_conf(_dev(conf, "conf", torch.float32, (B, L)),
                                     _dev(argmax, "argmax", torch.int32, (B, L)), B, L,
                                     _dev(mask, "mask", torch.uint8, (B, L)), float(param),
                                     _mode(mode),
                                     _dev(out_tokens, "out_tokens", torch.int32, (B, L)),
                                     _dev(out_commit, "out_commit", torch.uint8, (B, L)),
                                     _dev(out_n, "out_n", torch.int32, (B,)), _stream(stream))
    _check(st, "fdllm_select_from_conf")
    return out_tokens, out_commit, out_n


@_on_device
def fdllm_profile_terms(conf: torch.Tensor, mask: torch.Tensor, delta: float = 0.0,
                        stream=None):
    """Heterogeneity-bonus diagnostics by rank of each row's sorted masked profile:
    dict(G, F, B, f_eff) fp64 [B, L] (f_eff = 1 - delta + B, the effective factor of the
    profile rule with margin ``delta``) and order int32 [B, L] (NaN / -1 beyond the masked
    count)."""
    B, L = conf.shape
    dev = conf.device
    G, F, Bn, Fe = (torch.empty((B, L), dtype=torch.float64, device=dev) for _ in range(4))
    order = torch.empty((B, L), dtype=torch.int32, device=dev)
    st = _load().fdllm_profile_terms(_dev(conf, "conf", torch.float32, (B, L)),
                                     _dev(mask, "mask", torch.uint8, (B, L)), B, L,
                                     float(delta), G.data_ptr(), F.data_ptr(), Bn.data_ptr(),
                                     Fe.data_ptr(), order.data_ptr(), _stream(stream))
    _check(st, "fdllm_profile_terms")
    return dict(G=G, F=F, B=Bn, f_eff=Fe, order=order)


@_on_device
def fdllm_decode_loop(forward, logits: torch.Tensor, gen_len: int, param: float, mode=PROFILE,
                      max_steps: int | None = None, stream=None):
    """Algorithm 1's outer loop on the GPU (fdllm_decode_loop).  ``logits`` is the
    [B, block_len, V] buffer the forward pass fills; ``forward(loop_state_ptr,
    block_mask_ptr, logits_ptr, stream_ptr)`` receives raw device pointers and the capture
    stream and must only enqueue stream-ordered GPU work.  Returns (seq_tokens [B, gen_len]
    int32, nfe_per_block int32, total steps); synchronous."""
    B, Lb, V = logits.shape
    nblocks = gen_len // Lb
    dev = logits.device
    seq = torch.empty((B, gen_len), dtype=torch.int32, device=dev)
    nfe = torch.empty((nblocks,), dtype=torch.int32, device=dev)
    steps = ctypes.c_int(0)

    def trampoline(user, state, mask, out, strm):
        try:
            r = forward(state, mask, out, strm)
            return 0 if r is None else int(r)
        except Exception:  # the library reports it as FDLLM_ERR_ARG; keep the cause visible
            import traceback
            import warnings
            warnings.warn("forward pass raised during loop capture:\n" + traceback.format_exc())
            return 1

    cb = FORWARD_FN(trampoline)
    st = _load().fdllm_decode_loop(B, gen_len, Lb, V, _dtype_code(logits), float(param),
                                   _mode(mode), cb, None, _dev(logits, "logits"),
                                   seq.data_ptr(), nfe.data_ptr(),
                                   int(max_steps if max_steps is not None else gen_len + 1),
                                   ctypes.byref(steps), _stream(stream))
    _check(st, "fdllm_decode_loop")
    return seq, nfe, steps.value


@_on_device
def fdllm_gather_masked_rows(src: torch.Tensor, mask: torch.Tensor, dst=None, stream=None):
    """Copy the masked positions' rows of ``src`` [B, L, V] (a CUDA tensor or a pinned host
    tensor, read by the GPU directly) into ``dst`` (a CUDA tensor of the same shape and
    dtype; allocated when None).  Returns dst; its unmasked rows are not written."""
    if not src.is_cuda and not src.is_pinned():
        raise ValueError("src must be a CUDA tensor or a pinned host tensor")
    if not src.is_contiguous():
        raise ValueError("src must be contiguous")
    B, L, V = src.shape
    if dst is None:
        dst = torch.empty(src.shape, dtype=src.dtype, device=mask.device)
    _check(_load().fdllm_gather_masked_rows(src.data_ptr(),
                                            _dev(dst, "dst", src.dtype, (B, L, V)),
                                            _dtype_code(src), B, L, V,
                                            _dev(mask, "mask", torch.uint8, (B, L)),
                                            _stream(stream)), "fdllm_gather_masked_rows")
    return dst


@_on_device
def fdllm_decode_loop_lmhead(forward, hidden: torch.Tensor, w_vocab: torch.Tensor, gen_len: int,
                             param: float, mode=PROFILE, max_steps: int | None = None,
                             stream=None):
    """fdllm_decode_loop with the LM head in the loop: ``hidden`` is the [B, block_len, H]
    bf16 buffer the forward pass fills, ``w_vocab`` the [V, H] bf16 head.  Returns
    (seq_tokens [B, gen_len] int32, nfe_per_block int32, total steps); synchronous."""
    B, Lb, H = hidden.shape
    V, H2 = w_vocab.shape
    if H2 != H:
        raise ValueError("w_vocab must be [V, %d]" % H)
    nblocks = gen_len // Lb
    dev = hidden.device
    seq = torch.empty((B, gen_len), dtype=torch.int32, device=dev)
    nfe = torch.empty((nblocks,), dtype=torch.int32, device=dev)
    steps = ctypes.c_int(0)

    def trampoline(user, state, mask, out, strm):
        try:
            r = forward(state, mask, out, strm)
            return 0 if r is None else int(r)
        except Exception:  # the library reports it as FDLLM_ERR_ARG; keep the cause visible
            import traceback
            import warnings
            warnings.warn("forward pass raised during loop capture:\n" + traceback.format_exc())
            return 1

    cb = FORWARD_FN(trampoline)
    st = _load().fdllm_decode_loop_lmhead(
        B, gen_len, Lb, H, V, _dev(w_vocab, "w_vocab", torch.bfloat16), float(param),
        _mode(mode), cb, None, _dev(hidden, "hidden", torch.bfloat16), seq.data_ptr(),
        nfe.data_ptr(), int(max_steps if max_steps is not None else gen_len + 1),
        ctypes.byref(steps), _stream(stream))
    _check(st, "fdllm_decode_loop_lmhead")
    return seq, nfe, steps.value


class _CacheStruct(ctypes.Structure):
    _fields_ = [("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_affine", ctypes.c_void_p), ("v_affine", ctypes.c_void_p),
                ("pages", ctypes.c_int), ("heads", ctypes.c_int), ("page_size", ctypes.c_int),
                ("head_dim", ctypes.c_int)]


_Two, _Three, _Four = ctypes.c_int64 * 2, ctypes.c_int64 * 3, ctypes.c_int * 4
_current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
_I32, _F32, _U8, _BF16, _F16 = (torch.int32, torch.float32, torch.uint8, torch.bfloat16,
                                torch.float16)
_CODES = {_BF16: BF16, _F32: FP32, _F16: FP16}


# A decode step makes these calls once a layer and step, on short blocks in a few microseconds of
# GPU time: the checks below look at each tensor once, and look up why only when one fails.

def _ptr(t, name, dtype, shape, dev):
    """Pointer of a contiguous tensor of this dtype, shape and device (None: a null pointer)."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.device == dev and t.is_contiguous():
        return t.data_ptr()
    _dev(t, name, dtype, shape)
    raise ValueError("the CUDA tensors of one call must share a device (%s, %s)" % (dev, t.device))


def _rows(t, name, dtype, shape, dev, kind):
    """(pointer, leading strides) of a tensor whose last axis is contiguous."""
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if t.device != dev or not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor on %s" % (name, dev))
    st = t.stride()
    if st[-1] != 1:
        raise ValueError("the channels of %s must be contiguous" % name)
    if 1 in shape:  # the stride of an axis of one is never taken
        st = [x if n > 1 else 0 for x, n in zip(st, shape)]
    return t.data_ptr(), kind(*st[:-1])


def _made(shape, dtype, dev, stream):
    """A tensor for the call's result.  Where the call runs on another stream than the current
    one, the allocator is told, and that stream waits for what may still use the memory."""
    t = torch.empty(shape, dtype=dtype, device=dev)
    if stream is not None and _stream(stream) != _raw_stream(dev.index):
        other = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream))
        other.wait_stream(torch.cuda.current_stream())
        t.record_stream(other)
    return t


def _called_on(which):
    """Runs a call on the device of its argument number `which`."""
    def wrap(fn):
        @functools.wraps(fn)
        def call(*args, **kwargs):
            t = args[which] if len(args) > which else kwargs[names[which]]
            if not isinstance(t, torch.Tensor) or not t.is_cuda:
                raise ValueError("%s must be a CUDA tensor" % names[which])
            if t.device.index == _current_device():
                return fn(*args, **kwargs)
            with torch.cuda.device(t.device):
                return fn(*args, **kwargs)
        names = fn.__code__.co_varnames[:fn.__code__.co_argcount]
        return call
    return wrap


class KvCache:
    """The 4-bit prefix cache of one layer (fdllm_cache): four CUDA tensors and their sizes.

    ``k_codes`` uint8 [pages, heads, page_size, D/2], ``v_codes`` uint8 [pages, heads, D,
    page_size/2], ``k_affine`` and ``v_affine`` bfloat16 [pages, heads, page_size, 2] (scale,
    offset).  ``KvCache.empty`` allocates them."""

    __slots__ = ("k_codes", "v_codes", "k_affine", "v_affine", "pages", "heads", "page_size",
                 "head_dim", "device", "_struct", "_ref")

    def __init__(self, k_codes, v_codes, k_affine, v_affine):
        if k_codes.dim() != 4 or not k_codes.is_cuda:
            raise ValueError("k_codes must be a CUDA tensor [pages, heads, page_size, D/2]")
        pages, heads, page, half = shape = k_codes.shape
        dev = k_codes.device
        affine = (pages, heads, page, 2)
        self._struct = _CacheStruct(
            _ptr(k_codes, "k_codes", _U8, shape, dev),
            _ptr(v_codes, "v_codes", _U8, (pages, heads, 2 * half, page // 2), dev),
            _ptr(k_affine, "k_affine", _BF16, affine, dev),
            _ptr(v_affine, "v_affine", _BF16, affine, dev), pages, heads, page, 2 * half)
        self._ref = ctypes.addressof(self._struct)
        self.device = dev
        self.k_codes, self.v_codes = k_codes, v_codes
        self.k_affine, self.v_affine = k_affine, v_affine
        self.pages, self.heads, self.page_size, self.head_dim = pages, heads, page, 2 * half

    @classmethod
    def empty(cls, pages: int, heads: int, page_size: int, head_dim: int, device="cuda"):
        affine = (pages, heads, page_size, 2)
        return cls(torch.empty((pages, heads, page_size, head_dim // 2), dtype=_U8, device=device),
                   torch.empty((pages, heads, head_dim, page_size // 2), dtype=_U8, device=device),
                   torch.empty(affine, dtype=_BF16, device=device),
                   torch.empty(affine, dtype=_BF16, device=device))


def _table(table, cache, dev, name="block_table", rows=None):
    if table.dim() != 2 or (rows is not None and table.shape[0] != rows):
        raise ValueError("%s must be [%s, max_pages], got %s"
                         % (name, "B" if rows is None else rows, tuple(table.shape)))
    if cache.device != dev:
        raise ValueError("the cache must be on %s" % dev)
    B, pages = shape = table.shape
    return _ptr(table, name, _I32, shape, dev), B, pages


@_called_on(0)
def fdllm_qk_norm_rope(q: torch.Tensor, k: torch.Tensor | None, positions: torch.Tensor,
                       inv_freq: torch.Tensor, q_weight=None, k_weight=None, eps: float = 1e-6,
                       sections=None, interleaved: bool = False, out_q=None, out_k=None,
                       stream=None):
    """Per-head RMS norm and rotary positions of queries and keys in one pass.

    ``q`` [T, Hq, D] and ``k`` [T, Hk, D] (or None), bf16/fp16/fp32, channels contiguous (rows
    of a packed projection are taken where they lie); ``positions`` int32 [T] or [axes, T];
    ``inv_freq`` a CPU float64 tensor of the pairs' frequencies in radians per position;
    ``sections`` the pairs of each axis; a weight of None skips that tensor's norm.
    ``out_q`` / ``out_k`` may be q / k themselves where those are contiguous.  Returns
    (out_q, out_k)."""
    dev, dt = q.device, q.dtype
    if q.dim() != 3:
        raise ValueError("q must be [T, Hq, D]")
    T, Hq, D = shape = q.shape
    qp, qs = _rows(q, "q", dt, shape, dev, _Two)
    Hk, kp, ks = 0, None, None
    if k is not None:
        Hk = k.shape[1] if k.dim() == 3 else -1
        kp, ks = _rows(k, "k", dt, (T, Hk, D), dev, _Two)
    axes = 1 if positions.dim() == 1 else positions.shape[0]
    pp = _ptr(positions, "positions", _I32, (T,) if positions.dim() == 1 else (axes, T), dev)
    if inv_freq.is_cuda or inv_freq.dtype is not torch.float64 or not inv_freq.is_contiguous():
        raise ValueError("inv_freq must be a contiguous CPU float64 tensor")
    if sections is not None and (len(sections) != axes or axes > 4):
        raise ValueError("sections must name the pairs of each of %d axes (at most 4)" % axes)
    if out_q is None:
        out_q = _made(shape, dt, dev, stream)
    if k is not None and out_k is None:
        out_k = _made((T, Hk, D), dt, dev, stream)
    st = _load().fdllm_qk_norm_rope(
        qp, qs, kp, ks, _dtype_code(q), T, Hq, Hk, D, _ptr(q_weight, "q_weight", dt, (D,), dev),
        _ptr(k_weight, "k_weight", dt, (D,), dev), eps, pp, axes,
        None if sections is None else _Four(*sections), inv_freq.data_ptr(), inv_freq.numel(),
        1 if interleaved else 0, _ptr(out_q, "out_q", dt, shape, dev),
        None if k is None else _ptr(out_k, "out_k", dt, (T, Hk, D), dev),
        _raw_stream(dev.index) if stream is None else _stream(stream))
    if st:
        _check(st, "fdllm_qk_norm_rope")
    return out_q, out_k


@_called_on(3)
def fdllm_cache_append(cache: KvCache, block_table: torch.Tensor, start, k: torch.Tensor,
                       v: torch.Tensor, count=None, stream=None):
    """Write k, v [B, n, heads, D] (bf16/fp16/fp32, channels contiguous) into slots
    start[b] .. start[b] + count[b] - 1 (int32 [B] each; None: 0 and n).  A sequence whose start
    is negative is not written."""
    dev, dt = k.device, k.dtype
    tp, B, mp = _table(block_table, cache, dev)
    n = k.shape[1] if k.dim() == 4 else -1
    shape = (B, n, cache.heads, cache.head_dim)
    kp, ks = _rows(k, "k", dt, shape, dev, _Three)
    vp, vs = _rows(v, "v", dt, shape, dev, _Three)
    st = _load().fdllm_cache_append(
        cache._ref, tp, B, mp, _ptr(start, "start", _I32, (B,), dev),
        _ptr(count, "count", _I32, (B,), dev), kp, ks, vp, vs, _dtype_code(k), n,
        _raw_stream(dev.index) if stream is None else _stream(stream))
    if st:
        _check(st, "fdllm_cache_append")


@_called_on(1)
def fdllm_cache_read(cache: KvCache, block_table: torch.Tensor, start, n: int,
                     dtype=torch.bfloat16, count=None, out_k=None, out_v=None, stream=None):
    """Slots start[b] .. start[b] + n - 1 as dense rows (out_k, out_v) [B, n, heads, D] of
    ``dtype``; rows from count[b] on are zero."""
    dev = block_table.device
    tp, B, mp = _table(block_table, cache, dev)
    shape = (B, n, cache.heads, cache.head_dim)
    if out_k is None:
        out_k = _made(shape, dtype, dev, stream)
    if out_v is None:
        out_v = _made(shape, dtype, dev, stream)
    st = _load().fdllm_cache_read(
        cache._ref, tp, B, mp, _ptr(start, "start", _I32, (B,), dev),
        _ptr(count, "count", _I32, (B,), dev), _ptr(out_k, "out_k", dtype, shape, dev),
        _ptr(out_v, "out_v", dtype, shape, dev), _dtype_code(out_k), n,
        _raw_stream(dev.index) if stream is None else _stream(stream))
    if st:
        _check(st, "fdllm_cache_read")
    return out_k, out_v


def fdllm_cache_attention_workspace_bytes(B: int, Lq: int, Hq: int, heads: int,
                                          head_dim: int) -> int:
    return int(_load().fdllm_cache_attention_workspace_bytes(B, Lq, Hq, heads, head_dim))


def _queries(q, cache, dev):
    if q.dim() != 4:
        raise ValueError("q must be [B, Lq, Hq, D]")
    if q.dtype is not _BF16 and q.dtype is not _F16:
        raise TypeError("q must be bfloat16 or float16, got %s" % q.dtype)
    B, Lq, Hq, D = shape = q.shape
    if D != cache.head_dim:
        raise ValueError("q must be [B, Lq, Hq, %d], got %s" % (cache.head_dim, tuple(shape)))
    qp, qs = _rows(q, "q", q.dtype, shape, dev, _Three)
    return qp, qs, B, Lq, Hq


@_called_on(0)
def fdllm_cache_attention(q: torch.Tensor, cache: KvCache, block_table: torch.Tensor,
                          cache_lens: torch.Tensor, k_new=None, v_new=None, new_lens=None,
                          causal: bool = False, scale: float | None = None, out=None,
                          return_lse: bool = False, out_lse=None, workspace=None, stream=None):
    """Attention of ``q`` [B, Lq, Hq, D] (bf16/fp16) over the first cache_lens[b] slots of the
    cache and the block's own ``k_new``, ``v_new`` [B, Ln, heads, D].  ``scale`` None: D^-0.5.
    ``workspace`` a uint8 CUDA tensor of fdllm_cache_attention_workspace_bytes bytes (None: one
    of the call's own from torch's allocator; pass one where another library captures the call).
    Returns out, or (out, lse fp32 [B, Lq, Hq]) with ``return_lse``."""
    dev, dt = q.device, q.dtype
    qp, qs, B, Lq, Hq = _queries(q, cache, dev)
    heads, D = cache.heads, cache.head_dim
    tp, _, mp = _table(block_table, cache, dev, rows=B)
    Ln, kp, ks, vp, vs = 0, None, None, None, None
    if (k_new is None) != (v_new is None):
        raise ValueError("k_new and v_new go together")
    if k_new is not None:
        Ln = k_new.shape[1] if k_new.dim() == 4 else -1
        own = (B, Ln, heads, D)
        kp, ks = _rows(k_new, "k_new", dt, own, dev, _Three)
        vp, vs = _rows(v_new, "v_new", dt, own, dev, _Three)
    if out is None:
        out = _made(q.shape, dt, dev, stream)
    if out_lse is None and return_lse:
        out_lse = _made((B, Lq, Hq), _F32, dev, stream)
    lib = _load()
    if workspace is None:
        # Of this call alone: it is two launches, between which another thread may enqueue a call
        # of its own on the stream.  (The allocator hands the memory out again in stream order.)
        need = lib.fdllm_cache_attention_workspace_bytes(B, Lq, Hq, heads, D)
        workspace = _made((need if need > 256 else 256,), _U8, dev, stream)
    st = lib.fdllm_cache_attention(
        qp, qs, _CODES[dt], B, Lq, Hq, cache._ref, tp, mp,
        _ptr(cache_lens, "cache_lens", _I32, (B,), dev), kp, ks, vp, vs, Ln,
        _ptr(new_lens, "new_lens", _I32, (B,), dev), 1 if causal else 0,
        D ** -0.5 if scale is None else scale, _ptr(out, "out", dt, q.shape, dev),
        _ptr(out_lse, "out_lse", _F32, (B, Lq, Hq), dev),
        _ptr(workspace, "workspace", _U8, workspace.shape, dev), workspace.numel(),
        _raw_stream(dev.index) if stream is None else _stream(stream))
    if st:
        _check(st, "fdllm_cache_attention")
    return (out, out_lse) if return_lse else out


@_called_on(0)
def fdllm_cache_key_weights(q: torch.Tensor, lse: torch.Tensor, cache: KvCache,
                            block_table: torch.Tensor, cache_lens: torch.Tensor, weights=None,
                            scale: float | None = None, max_len: int | None = None, out=None,
                            stream=None):
    """The attention each cached key receives from ``q`` given attention's ``lse`` [B, Lq, Hq],
    added to ``weights`` fp32 [B, heads, max_len] (None: from zero, ``max_len`` slots or the
    table's).  ``out`` may be ``weights``.  Returns the sums (0 behind cache_lens)."""
    dev = q.device
    qp, qs, B, Lq, Hq = _queries(q, cache, dev)
    tp, _, mp = _table(block_table, cache, dev, rows=B)
    if weights is not None:
        max_len = weights.shape[-1]
    elif max_len is None:
        max_len = mp * cache.page_size
    shape = (B, cache.heads, max_len)
    if out is None:
        out = _made(shape, _F32, dev, stream)
    st = _load().fdllm_cache_key_weights(
        qp, qs, _CODES[q.dtype], B, Lq, Hq, cache._ref, tp, mp,
        _ptr(cache_lens, "cache_lens", _I32, (B,), dev), _ptr(lse, "lse", _F32, (B, Lq, Hq), dev),
        cache.head_dim ** -0.5 if scale is None else scale,
        _ptr(weights, "weights", _F32, shape, dev), _ptr(out, "out", _F32, shape, dev), max_len,
        _raw_stream(dev.index) if stream is None else _stream(stream))
    if st:
        _check(st, "fdllm_cache_key_weights")
    return out


@_called_on(3)
def fdllm_cache_evict(cache: KvCache, block_table: torch.Tensor, cache_lens: torch.Tensor,
                      weights: torch.Tensor, budget: int, dst_table: torch.Tensor,
                      keep_first: int = 0, keep_last: int = 0, out_lens=None, out_weights=None,
                      out_index=None, stream=None):
    """Copy the ``budget`` heaviest keys of each sequence and head (the first ``keep_first`` and
    the last ``keep_last`` slots always) into the pages of ``dst_table`` [B, dst_max_pages],
    in slot order.  Returns (lens int32 [B], weights fp32 [B, heads, budget], the slots they
    came from int32 [B, heads, budget])."""
    dev = weights.device
    tp, B, mp = _table(block_table, cache, dev)
    dp, _, dmp = _table(dst_table, cache, dev, "dst_table", B)
    max_len = weights.shape[-1]
    shape = (B, cache.heads, budget)
    if out_lens is None:
        out_lens = _made((B,), _I32, dev, stream)
    if out_weights is None:
        out_weights = _made(shape, _F32, dev, stream)
    if out_index is None:
        out_index = _made(shape, _I32, dev, stream)
    st = _load().fdllm_cache_evict(
        cache._ref, tp, B, mp, _ptr(cache_lens, "cache_lens", _I32, (B,), dev),
        _ptr(weights, "weights", _F32, (B, cache.heads, max_len), dev), max_len, budget,
        keep_first, keep_last, dp, dmp, _ptr(out_lens, "out_lens", _I32, (B,), dev),
        _ptr(out_weights, "out_weights", _F32, shape, dev),
        _ptr(out_index, "out_index", _I32, shape, dev),
        _raw_stream(dev.index) if stream is None else _stream(stream))
    if st:
        _check(st, "fdllm_cache_evict")
    return out_lens, out_weights, out_index


def fdllm_cache_status(stream=None) -> int:
    """Synchronises and returns (clearing it) the sticky device status of the cache's attention
    and key-weight kernels on the current device."""
    return _load().fdllm_cache_status(_stream(stream))


def fdllm_cache_check_wait(tries: int = 0, stream=None) -> int:
    """Enqueues a warp of the cache kernels' kind that waits on a barrier nobody completes and
    gives up after ``tries`` tries (0: the kernels' own limit); fdllm_cache_status then reports
    FDLLM_ERR_DEVICE (6) once.  Returns the status code of the launch."""
    return _load().fdllm_cache_check_wait(tries, _stream(stream))


def fdllm_check_bounded_wait(seconds: float = 0.01, stream=None) -> int:
    """Makes one kernel wait on a barrier nobody completes; returns the status code
    (FDLLM_ERR_DEVICE = 6 when the bounded wait ran out and was reported)."""
    return _load().fdllm_check_bounded_wait(float(seconds), _stream(stream))


def fdllm_device_status(stream=None) -> int:
    """Synchronises and returns (clearing it) the library workspace's sticky device status."""
    return _load().fdllm_device_status(_stream(stream))


@_on_device
def fdllm_workspace_status(workspace: torch.Tensor, stream=None) -> int:
    return _load().fdllm_workspace_status(_dev(workspace, "workspace", torch.uint8), _stream(stream))


def fdllm_static_status(stream=None) -> int:
    """Synchronises and returns (clearing it) the sticky device status of
    fdllm_select_static's fixed array on the current device."""
    return _load().fdllm_static_status(_stream(stream))


def fdllm_release_workspace() -> None:
    _load().fdllm_release_workspace()
