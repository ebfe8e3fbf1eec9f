"""Python binding of libtim.so: batch-invariant fused LM-head token log-probs
and training-inference mismatch statistics on MI355X (gfx950).

Argument marshalling only: every step of the computation runs in the HIP
kernels behind the C ABI (include/tim.h). Tensors must live on the GPU; the
calls are enqueued on torch's current stream. There is no fallback: when the
library is missing or no GPU is present the calls raise.
"""

from __future__ import annotations

import ctypes
import dataclasses
import enum
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtim.so")

VOCAB_TILE = 256
MAX_VOCAB = 2048 * VOCAB_TILE


class Status(enum.IntEnum):
    OK = 0
    ERR_NULL = 1
    ERR_SHAPE = 2
    ERR_VALUE = 3
    ERR_WORKSPACE = 4
    ERR_HIP = 5


class Mode(enum.IntEnum):
    ROLLOUT = 0
    TRAINING = 1


class Order(enum.IntEnum):
    INVARIANT = 0
    SPLITK4 = 1


class Estimator(enum.IntEnum):
    K1 = 1
    K3 = 3


class TimError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{msg} (status {status})")
        self.status = Status(status)


class _LogitRules(ctypes.Structure):
    """tim_logit_rules"""
    _fields_ = [("history", ctypes.c_void_p), ("history_len", ctypes.c_int64), ("hist_begin", ctypes.c_void_p),
                ("hist_split", ctypes.c_void_p), ("hist_end", ctypes.c_void_p), ("repetition", ctypes.c_void_p),
                ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p), ("bias_ids", ctypes.c_void_p),
                ("bias_values", ctypes.c_void_p), ("bias_len", ctypes.c_int64), ("bias_begin", ctypes.c_void_p),
                ("bias_end", ctypes.c_void_p), ("mask", ctypes.c_void_p), ("n_masks", ctypes.c_int64),
                ("mask_ld", ctypes.c_int64), ("mask_rows", ctypes.c_void_p)]


class _Adapters(ctypes.Structure):
    """tim_adapters"""
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("n", ctypes.c_int32), ("r", ctypes.c_int32), ("d", ctypes.c_int32), ("N", ctypes.c_int32)]


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libtim.so and declare its C signatures. Raises if it is not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built; run `python -m paper_2605_14220_amd.build`")
    lib = ctypes.CDLL(path)
    c = ctypes
    lib.tim_logprobs_rows_per_launch.restype = c.c_int64
    lib.tim_logprobs_rows_per_launch.argtypes = [c.c_int64, c.c_int32, c.c_int32, c.c_int64]
    lib.tim_logprobs_workspace_size.restype = c.c_size_t
    lib.tim_logprobs_workspace_size.argtypes = [c.c_int64, c.c_int32, c.c_int32, c.c_int32, c.c_int64]
    lib.tim_logprobs.restype = c.c_int
    lib.tim_logprobs.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_int64, c.c_int32, c.c_int32,
                                 c.c_float, c.c_int32, c.c_int64, c.c_int32, c.c_void_p, c.c_void_p,
                                 c.c_void_p, c.c_void_p, c.c_size_t, c.c_void_p]
    lib.tim_logprobs_noalloc.restype = c.c_int
    lib.tim_logprobs_noalloc.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_int64, c.c_int32, c.c_int32,
                                         c.c_float, c.c_int32, c.c_int64, c.c_int32, c.c_void_p, c.c_void_p,
                                         c.c_void_p, c.c_void_p]
    lib.tim_logprobs_partials.restype = c.c_int
    lib.tim_logprobs_partials.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_int64, c.c_int32,
                                          c.c_int32, c.c_float, c.c_int32, c.c_int32, c.c_void_p,
                                          c.c_size_t, c.c_void_p]
    lib.tim_logprobs_merge.restype = c.c_int
    lib.tim_logprobs_merge.argtypes = [c.c_void_p, c.c_void_p, c.c_int64, c.c_int32, c.c_int32,
                                       c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p]
    lib.tim_mismatch.restype = c.c_int
    lib.tim_mismatch.argtypes = [c.c_void_p, c.c_void_p, c.c_int64, c.c_float, c.c_void_p, c.c_void_p,
                                 c.c_void_p, c.c_void_p]
    lib.tim_mismatch_seq.restype = c.c_int
    lib.tim_mismatch_seq.argtypes = [c.c_void_p, c.c_void_p, c.c_int64, c.c_void_p, c.c_int64, c.c_int32,
                                     c.c_float, c.c_double, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p]
    lib.tim_logprobs_backward_workspace_size.restype = c.c_size_t
    lib.tim_logprobs_backward_workspace_size.argtypes = [c.c_int64, c.c_int32, c.c_int32, c.c_int64]
    lib.tim_logprobs_backward.restype = c.c_int
    lib.tim_logprobs_backward.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_int64, c.c_int32, c.c_int32,
                                          c.c_float, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_int64,
                                          c.c_void_p, c.c_void_p, c.c_int32, c.c_void_p, c.c_size_t, c.c_void_p]
    lib.tim_logit_grads.restype = c.c_int
    lib.tim_logit_grads.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_int64, c.c_int32, c.c_int32,
                                    c.c_float, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
                                    c.c_void_p, c.c_size_t, c.c_void_p]
    lib.tim_rmsnorm.restype = c.c_int
    lib.tim_rmsnorm.argtypes = [c.c_void_p, c.c_void_p, c.c_int64, c.c_int32, c.c_float, c.c_void_p, c.c_void_p,
                                c.c_void_p]
    lib.tim_rmsnorm_backward_workspace_size.restype = c.c_size_t
    lib.tim_rmsnorm_backward_workspace_size.argtypes = [c.c_int64, c.c_int32]
    lib.tim_rmsnorm_backward.restype = c.c_int
    lib.tim_rmsnorm_backward.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_int64, c.c_int32,
                                         c.c_void_p, c.c_void_p, c.c_int32, c.c_void_p, c.c_size_t, c.c_void_p]
    lib.tim_ppo_loss.restype = c.c_int
    lib.tim_ppo_loss.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_int64, c.c_void_p, c.c_int64,
                                 c.c_float, c.c_float, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
                                 c.c_void_p, c.c_void_p]
    lib.tim_logits.restype = c.c_int
    lib.tim_logits.argtypes = [c.c_void_p, c.c_void_p, c.c_int64, c.c_int32, c.c_int32, c.c_float,
                               c.c_int32, c.c_void_p, c.c_void_p]
    lib.tim_mxfp4_quantize.restype = c.c_int
    lib.tim_mxfp4_quantize.argtypes = [c.c_void_p, c.c_int32, c.c_int64, c.c_int32, c.c_int64, c.c_void_p, c.c_void_p,
                                       c.c_void_p]
    lib.tim_mxfp4_dequantize.restype = c.c_int
    lib.tim_mxfp4_dequantize.argtypes = [c.c_void_p, c.c_void_p, c.c_int64, c.c_int32, c.c_void_p, c.c_int32,
                                         c.c_void_p]
    lib.tim_mxfp4_logits.restype = c.c_int
    lib.tim_mxfp4_logits.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_int64, c.c_int32, c.c_int32,
                                     c.c_float, c.c_void_p, c.c_int32, c.c_int64, c.c_void_p]
    lib.tim_embedding.restype = c.c_int
    lib.tim_embedding.argtypes = [c.c_void_p, c.c_int32, c.c_int32, c.c_int32, c.c_int64, c.c_void_p, c.c_int64, c.c_float,
                                  c.c_void_p, c.c_int32, c.c_int64, c.c_void_p]
    lib.tim_embedding_backward_workspace_size.restype = c.c_size_t
    lib.tim_embedding_backward_workspace_size.argtypes = [c.c_int64, c.c_int32, c.c_int32]
    lib.tim_embedding_backward.restype = c.c_int
    lib.tim_embedding_backward.argtypes = [c.c_void_p, c.c_int32, c.c_int64, c.c_int32, c.c_int64, c.c_void_p, c.c_int32,
                                           c.c_float, c.c_void_p, c.c_int64, c.c_int32, c.c_void_p, c.c_size_t,
                                           c.c_void_p]
    adapters = c.POINTER(_Adapters)
    for f in (lib.tim_adapters_add_workspace_size, lib.tim_adapters_backward_workspace_size):
        f.restype = c.c_size_t
        f.argtypes = [c.c_int64, c.c_int32, c.c_int32, c.c_int32, c.c_int32]
    lib.tim_adapters_add.restype = c.c_int
    lib.tim_adapters_add.argtypes = [adapters, c.c_void_p, c.c_int64, c.c_void_p, c.c_int64, c.c_void_p, c.c_int64,
                                     c.c_void_p, c.c_int32, c.c_int64, c.c_void_p, c.c_size_t, c.c_void_p]
    lib.tim_adapters_backward.restype = c.c_int
    lib.tim_adapters_backward.argtypes = [adapters, c.c_void_p, c.c_int64, c.c_void_p, c.c_int64, c.c_void_p, c.c_int32,
                                          c.c_int64, c.c_void_p, c.c_int32, c.c_int64, c.c_int32, c.c_void_p, c.c_void_p,
                                          c.c_int32, c.c_void_p, c.c_size_t, c.c_void_p]
    rules = c.POINTER(_LogitRules)
    lib.tim_logits_adjust.restype = c.c_int
    lib.tim_logits_adjust.argtypes = [c.c_void_p, c.c_int32, c.c_int64, c.c_int32, c.c_int64, rules, c.c_float,
                                      c.c_void_p, c.c_int64, c.c_void_p]
    lib.tim_logits_logprobs_workspace_size.restype = c.c_size_t
    lib.tim_logits_logprobs_workspace_size.argtypes = [c.c_int64, c.c_int32]
    lib.tim_logits_logprobs.restype = c.c_int
    lib.tim_logits_logprobs.argtypes = [c.c_void_p, c.c_int32, c.c_int64, c.c_int32, c.c_int64, c.c_void_p, rules,
                                        c.c_float, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_size_t,
                                        c.c_void_p]
    lib.tim_logits_logprobs_backward.restype = c.c_int
    lib.tim_logits_logprobs_backward.argtypes = [c.c_void_p, c.c_int32, c.c_int64, c.c_int32, c.c_int64, c.c_void_p,
                                                 rules, c.c_float, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
                                                 c.c_void_p, c.c_int32, c.c_int64, c.c_void_p]
    lib.tim_status_string.restype = c.c_char_p
    lib.tim_status_string.argtypes = [c.c_int]
    _lib = lib
    return lib


def _check(status: int):
    if status != 0:
        msg = load_library().tim_status_string(status).decode()
        raise TimError(status, msg)


def _ptr(t):
    return None if t is None else t.data_ptr()


# The current stream's handle alone: building the Stream object of torch.cuda.current_stream takes 2 us of every call.
# The name is private to torch, so a version without it takes the public call.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream if _raw_stream is None else _raw_stream(device.index)


def _require_gpu(*tensors):
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError("tim: tensors must be on the GPU")
        if t is not None and not t.is_contiguous():
            raise ValueError("tim: tensors must be contiguous")


def rows_per_launch(T: int, d: int, mode: Mode = Mode.TRAINING, micro_batch: int = 0) -> int:
    """Rows tim_logprobs hands to one launch (0 for invalid arguments); see include/tim.h."""
    return int(load_library().tim_logprobs_rows_per_launch(int(T), int(d), int(mode), int(micro_batch)))


def workspace_size(T: int, d: int, V: int, mode: Mode = Mode.TRAINING, micro_batch: int = 0) -> int:
    """Bytes of workspace tim_logprobs needs (0 for T == 0 or invalid shapes)."""
    return int(load_library().tim_logprobs_workspace_size(int(T), int(d), int(V), int(mode), int(micro_batch)))


def logprobs(hidden: torch.Tensor, w_vocab: torch.Tensor, tokens: torch.Tensor, temperature: float = 1.0,
             mode: Mode = Mode.TRAINING, micro_batch: int = 0, order: Order = Order.INVARIANT,
             entropy: bool = True, lse: bool = False, workspace: torch.Tensor | None = None,
             out: tuple | None = None):
    """Token log-probabilities (and entropies, log-normalisers) of T rows.

    hidden bf16 [T, d], w_vocab bf16 [V, d], tokens int32 [T], all on one GPU.
    Returns (logp, entropy or None, lse or None), fp32 [T] each."""
    lib = load_library()
    if hidden.dtype != torch.bfloat16 or w_vocab.dtype != torch.bfloat16:
        raise TypeError("tim.logprobs: hidden and w_vocab must be bfloat16")
    if tokens.dtype != torch.int32:
        raise TypeError("tim.logprobs: tokens must be int32")
    if hidden.dim() != 2 or w_vocab.dim() != 2 or hidden.shape[1] != w_vocab.shape[1]:
        raise ValueError("tim.logprobs: hidden [T, d] and w_vocab [V, d] must share d")
    T, d = hidden.shape
    V = w_vocab.shape[0]
    if tokens.shape != (T,):
        raise ValueError("tim.logprobs: tokens must be [T]")
    _require_gpu(hidden, w_vocab, tokens, workspace)
    dev = hidden.device
    if out is None:
        lp = torch.empty(T, dtype=torch.float32, device=dev)
        ent = torch.empty(T, dtype=torch.float32, device=dev) if entropy else None
        ls = torch.empty(T, dtype=torch.float32, device=dev) if lse else None
    else:
        lp, ent, ls = out
        _require_gpu(lp, ent, ls)
    if T == 0:
        return lp, ent, ls
    need = workspace_size(T, d, V, mode, micro_batch)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib.tim_logprobs(_ptr(hidden), _ptr(w_vocab), _ptr(tokens), T, d, V, float(temperature),
                            int(mode), int(micro_batch), int(order), _ptr(lp), _ptr(ent), _ptr(ls),
                            _ptr(workspace), ws_bytes, _stream(dev)))
    return lp, ent, ls


NOALLOC_SCRATCH_BYTES = 64 << 20  # TIM_NOALLOC_SCRATCH_BYTES


def logprobs_noalloc(hidden: torch.Tensor, w_vocab: torch.Tensor, tokens: torch.Tensor, temperature: float = 1.0,
                     mode: Mode = Mode.TRAINING, micro_batch: int = 0, order: Order = Order.INVARIANT,
                     out: tuple | None = None):
    """tim_logprobs_noalloc: logprobs() with the partials in the library's per-GPU device array instead of a
    workspace (the call allocates no device memory; pass `out` = (logp, entropy or None, lse or None) to keep
    the binding from allocating the outputs). Needs workspace_size(T, d, V, mode, micro_batch) <=
    NOALLOC_SCRATCH_BYTES."""
    lib = load_library()
    if hidden.dtype != torch.bfloat16 or w_vocab.dtype != torch.bfloat16:
        raise TypeError("tim.logprobs_noalloc: hidden and w_vocab must be bfloat16")
    if tokens.dtype != torch.int32:
        raise TypeError("tim.logprobs_noalloc: tokens must be int32")
    if hidden.dim() != 2 or w_vocab.dim() != 2 or hidden.shape[1] != w_vocab.shape[1]:
        raise ValueError("tim.logprobs_noalloc: hidden [T, d] and w_vocab [V, d] must share d")
    T, d = hidden.shape
    V = w_vocab.shape[0]
    if tokens.shape != (T,):
        raise ValueError("tim.logprobs_noalloc: tokens must be [T]")
    _require_gpu(hidden, w_vocab, tokens)
    dev = hidden.device
    if out is None:
        out = (torch.empty(T, dtype=torch.float32, device=dev), torch.empty(T, dtype=torch.float32, device=dev),
               None)
    lp, ent, ls = out
    _require_gpu(lp, ent, ls)
    _check(lib.tim_logprobs_noalloc(_ptr(hidden), _ptr(w_vocab), _ptr(tokens), T, d, V, float(temperature),
                                    int(mode), int(micro_batch), int(order), _ptr(lp), _ptr(ent), _ptr(ls),
                                    _stream(dev)))
    return lp, ent, ls


def logprobs_partials(hidden: torch.Tensor, w_vocab: torch.Tensor, tokens: torch.Tensor,
                      workspace: torch.Tensor, temperature: float = 1.0, mode: Mode = Mode.TRAINING,
                      order: Order = Order.INVARIANT):
    """First stage of logprobs over all rows in one launch: per-(row, vocab tile)
    partials written into `workspace`, which holds all T rows': workspace_size(T, d, V, Mode.ROLLOUT)
    bytes are enough in both modes (see include/tim.h)."""
    lib = load_library()
    _require_gpu(hidden, w_vocab, tokens, workspace)
    T, d = hidden.shape
    V = w_vocab.shape[0]
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib.tim_logprobs_partials(_ptr(hidden), _ptr(w_vocab), _ptr(tokens), T, d, V, float(temperature),
                                     int(mode), int(order), _ptr(workspace), ws_bytes, _stream(hidden.device)))


def logprobs_merge(workspace: torch.Tensor, tokens: torch.Tensor, V: int, order: Order = Order.INVARIANT,
                   out: tuple | None = None):
    """Second stage: partials in `workspace` -> (logp, entropy, lse) for len(tokens) rows."""
    lib = load_library()
    _require_gpu(workspace, tokens)
    T = tokens.numel()
    if out is None:
        out = tuple(torch.empty(T, dtype=torch.float32, device=tokens.device) for _ in range(3))
    _require_gpu(*out)
    _check(lib.tim_logprobs_merge(_ptr(workspace), _ptr(tokens), T, int(V), int(order), _ptr(out[0]),
                                  _ptr(out[1]), _ptr(out[2]), _stream(tokens.device)))
    return out


def mismatch(logp_a: torch.Tensor, logp_b: torch.Tensor, C: float = 2.0, out: tuple | None = None):
    """(log_ratio, k3, is_weight) fp32 [T]: delta = a - b, k3 = expm1(delta) - delta,
    w = min(exp(delta), C). a is the trainer's log-prob, b the rollout engine's."""
    lib = load_library()
    if logp_a.dtype != torch.float32 or logp_b.dtype != torch.float32 or logp_a.shape != logp_b.shape:
        raise TypeError("tim.mismatch: logp_a and logp_b must be fp32 of one shape")
    _require_gpu(logp_a, logp_b)
    T = logp_a.numel()
    if out is None:
        out = tuple(torch.empty_like(logp_a) for _ in range(3))
    _require_gpu(*out)
    _check(lib.tim_mismatch(_ptr(logp_a), _ptr(logp_b), T, float(C), _ptr(out[0]), _ptr(out[1]),
                            _ptr(out[2]), _stream(logp_a.device)))
    return out


def mismatch_seq(logp_a: torch.Tensor, logp_b: torch.Tensor, cu_seqlens: torch.Tensor, C: float = 2.0,
                 tau_seq: float = 1e-3, estimator: Estimator = Estimator.K3, out: tuple | None = None):
    """Per-response mismatch score, keep mask and per-token weights of a packed stream.

    logp_a (trainer) and logp_b (rollout) fp32 [T]; cu_seqlens int64 [n + 1] offsets of the
    n responses. Returns (score fp64 [n], keep uint8 [n], weight fp32 [T]) with
    score = sum_t K(delta_t) (K1 = -delta, K3 = expm1(delta) - delta), keep = score <= tau_seq,
    weight = keep * min(exp(delta), C). See include/tim.h."""
    lib = load_library()
    if logp_a.dtype != torch.float32 or logp_b.dtype != torch.float32 or logp_a.shape != logp_b.shape:
        raise TypeError("tim.mismatch_seq: logp_a and logp_b must be fp32 of one shape")
    if cu_seqlens.dtype != torch.int64 or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
        raise TypeError("tim.mismatch_seq: cu_seqlens must be a non-empty int64 vector")
    _require_gpu(logp_a, logp_b, cu_seqlens)
    T = logp_a.numel()
    n = cu_seqlens.numel() - 1
    dev = logp_a.device
    if out is None:
        out = (torch.empty(n, dtype=torch.float64, device=dev), torch.empty(n, dtype=torch.uint8, device=dev),
               torch.zeros(T, dtype=torch.float32, device=dev))
    _require_gpu(*out)
    _check(lib.tim_mismatch_seq(_ptr(logp_a), _ptr(logp_b), T, _ptr(cu_seqlens), n, int(estimator), float(C),
                                float(tau_seq), _ptr(out[0]), _ptr(out[1]), _ptr(out[2]), _stream(dev)))
    return out


def logits(hidden: torch.Tensor, w_vocab: torch.Tensor, temperature: float = 1.0,
           order: Order = Order.INVARIANT) -> torch.Tensor:
    """fp32 [T, V] logits exactly as tim_logprobs forms them (test/debug aid)."""
    lib = load_library()
    _require_gpu(hidden, w_vocab)
    T, d = hidden.shape
    V = w_vocab.shape[0]
    z = torch.empty((T, V), dtype=torch.float32, device=hidden.device)
    _check(lib.tim_logits(_ptr(hidden), _ptr(w_vocab), T, d, V, float(temperature), int(order), _ptr(z),
                          _stream(hidden.device)))
    return z


def backward_workspace_size(T: int, d: int, V: int, micro_batch: int = 0) -> int:
    """Bytes of workspace tim_logprobs_backward needs (0 for T == 0 or invalid arguments)."""
    return int(load_library().tim_logprobs_backward_workspace_size(int(T), int(d), int(V), int(micro_batch)))


def _grad_inputs(name, hidden, w_vocab, tokens, lse, grad_logp, entropy, grad_entropy):
    if hidden.dtype != torch.bfloat16 or w_vocab.dtype != torch.bfloat16:
        raise TypeError(f"tim.{name}: hidden and w_vocab must be bfloat16")
    if tokens.dtype != torch.int32:
        raise TypeError(f"tim.{name}: tokens must be int32")
    if hidden.dim() != 2 or w_vocab.dim() != 2 or hidden.shape[1] != w_vocab.shape[1]:
        raise ValueError(f"tim.{name}: hidden [T, d] and w_vocab [V, d] must share d")
    T = hidden.shape[0]
    for t in (tokens, lse, grad_logp, entropy, grad_entropy):
        if t is not None and t.shape != (T,):
            raise ValueError(f"tim.{name}: per-row arrays must be [T]")
    for t in (lse, grad_logp, entropy, grad_entropy):
        if t is not None and t.dtype != torch.float32:
            raise TypeError(f"tim.{name}: lse, entropy and the upstream gradients must be fp32")
    _require_gpu(hidden, w_vocab, tokens, lse, grad_logp, entropy, grad_entropy)


def logprobs_backward(hidden: torch.Tensor, w_vocab: torch.Tensor, tokens: torch.Tensor, lse: torch.Tensor,
                      grad_logp: torch.Tensor, temperature: float = 1.0, entropy: torch.Tensor | None = None,
                      grad_entropy: torch.Tensor | None = None, micro_batch: int = 0, want_hidden: bool = True,
                      want_w: bool = True, grad_w: torch.Tensor | None = None, accumulate: bool = False,
                      workspace: torch.Tensor | None = None):
    """Gradients of sum_t grad_logp[t] logp[t] + grad_entropy[t] entropy[t] with respect
    to hidden [T, d] and w_vocab [V, d], as fp32 (grad_hidden or None, grad_w or None).

    lse (and entropy, when grad_entropy is given) are tim.logprobs' outputs for the same
    inputs. grad_w, if given, is the fp32 [V, d] output buffer; with accumulate=True the
    gradient is added to its contents. See include/tim.h."""
    lib = load_library()
    _grad_inputs("logprobs_backward", hidden, w_vocab, tokens, lse, grad_logp, entropy, grad_entropy)
    T, d = hidden.shape
    V = w_vocab.shape[0]
    dev = hidden.device
    gh = torch.empty((T, d), dtype=torch.float32, device=dev) if want_hidden else None
    if want_w and grad_w is None:
        if accumulate:
            raise ValueError("tim.logprobs_backward: accumulate needs the grad_w buffer")
        grad_w = torch.empty((V, d), dtype=torch.float32, device=dev)
    gw = grad_w if want_w else None
    if gw is not None and (gw.dtype != torch.float32 or gw.shape != (V, d)):
        raise ValueError("tim.logprobs_backward: grad_w must be fp32 [V, d]")
    _require_gpu(gh, gw, workspace)
    need = backward_workspace_size(T, d, V, micro_batch)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib.tim_logprobs_backward(_ptr(hidden), _ptr(w_vocab), _ptr(tokens), T, d, V, float(temperature),
                                     _ptr(lse), _ptr(entropy), _ptr(grad_logp), _ptr(grad_entropy),
                                     int(micro_batch), _ptr(gh), _ptr(gw), 1 if accumulate else 0,
                                     _ptr(workspace), ws_bytes, _stream(dev)))
    return gh, gw


def logit_grads(hidden: torch.Tensor, w_vocab: torch.Tensor, tokens: torch.Tensor, lse: torch.Tensor,
                grad_logp: torch.Tensor, temperature: float = 1.0, entropy: torch.Tensor | None = None,
                grad_entropy: torch.Tensor | None = None) -> torch.Tensor:
    """bf16 [T, ceil(V / 256) * 256] gradients with respect to the LM-head contraction,
    exactly as the backward's first pass forms them (test/debug aid)."""
    lib = load_library()
    _grad_inputs("logit_grads", hidden, w_vocab, tokens, lse, grad_logp, entropy, grad_entropy)
    T, d = hidden.shape
    V = w_vocab.shape[0]
    dev = hidden.device
    v_pad = (V + VOCAB_TILE - 1) // VOCAB_TILE * VOCAB_TILE
    out = torch.empty((T, v_pad), dtype=torch.bfloat16, device=dev)
    ws = torch.empty(max(T * 16, 16), dtype=torch.uint8, device=dev)
    _check(lib.tim_logit_grads(_ptr(hidden), _ptr(w_vocab), _ptr(tokens), T, d, V, float(temperature), _ptr(lse),
                               _ptr(entropy), _ptr(grad_logp), _ptr(grad_entropy), _ptr(out), _ptr(ws),
                               ws.numel(), _stream(dev)))
    return out


def rmsnorm(x: torch.Tensor, gamma: torch.Tensor | None = None, eps: float = 1e-6, out: torch.Tensor | None = None):
    """Final RMS norm: (h bf16 [T, d], rstd fp32 [T]) of x bf16 [T, d] (see include/tim.h)."""
    lib = load_library()
    if x.dtype != torch.bfloat16 or x.dim() != 2 or (gamma is not None and gamma.dtype != torch.bfloat16):
        raise TypeError("tim.rmsnorm: x must be bf16 [T, d] and gamma bf16 [d]")
    T, d = x.shape
    if gamma is not None and gamma.shape != (d,):
        raise ValueError("tim.rmsnorm: gamma must be [d]")
    _require_gpu(x, gamma, out)
    h = torch.empty_like(x) if out is None else out
    rstd = torch.empty(T, dtype=torch.float32, device=x.device)
    _check(lib.tim_rmsnorm(_ptr(x), _ptr(gamma), T, d, float(eps), _ptr(h), _ptr(rstd), _stream(x.device)))
    return h, rstd


def rmsnorm_backward(x: torch.Tensor, gamma: torch.Tensor | None, rstd: torch.Tensor, grad_h: torch.Tensor,
                     want_x: bool = True, want_gamma: bool = True, grad_gamma: torch.Tensor | None = None,
                     accumulate: bool = False):
    """(grad_x fp32 [T, d] or None, grad_gamma fp32 [d] or None) of the final RMS norm."""
    lib = load_library()
    T, d = x.shape
    if grad_h.dtype != torch.float32 or grad_h.shape != (T, d) or rstd.shape != (T,):
        raise ValueError("tim.rmsnorm_backward: grad_h fp32 [T, d] and rstd [T]")
    _require_gpu(x, gamma, rstd, grad_h, grad_gamma)
    dev = x.device
    gx = torch.empty((T, d), dtype=torch.float32, device=dev) if want_x else None
    if want_gamma and grad_gamma is None:
        if accumulate:
            raise ValueError("tim.rmsnorm_backward: accumulate needs the grad_gamma buffer")
        grad_gamma = torch.empty(d, dtype=torch.float32, device=dev)
    gg = grad_gamma if want_gamma else None
    ws = torch.empty(max(int(lib.tim_rmsnorm_backward_workspace_size(T, d)), 16), dtype=torch.uint8, device=dev)
    _check(lib.tim_rmsnorm_backward(_ptr(x), _ptr(gamma), _ptr(rstd), _ptr(grad_h), T, d, _ptr(gx), _ptr(gg),
                                    1 if accumulate else 0, _ptr(ws), ws.numel(), _stream(dev)))
    return gx, gg


def logprobs_from_residual(x: torch.Tensor, gamma: torch.Tensor | None, w_vocab: torch.Tensor, tokens: torch.Tensor,
                           eps: float = 1e-6, temperature: float = 1.0, **kw):
    """The final norm followed by the LM-head log-probs: (logp, entropy, lse, h, rstd).
    Two C-ABI calls on the same stream; keyword arguments go to logprobs()."""
    h, rstd = rmsnorm(x, gamma, eps)
    lp, ent, lse = logprobs(h, w_vocab, tokens, temperature, **kw)
    return lp, ent, lse, h, rstd


def ppo_loss(logp: torch.Tensor, logp_old: torch.Tensor, advantages: torch.Tensor, cu_seqlens: torch.Tensor,
             eps_low: float = 0.2, eps_high: float = 0.2, weight: torch.Tensor | None = None,
             out: dict | None = None) -> dict:
    """Clipped PPO/GRPO loss of a packed stream (see include/tim.h): dict with seq_loss fp64 [n],
    batch_loss fp64 [1], token_loss / grad / contribution fp32 [T] and clipped uint8 [T]
    (freshly allocated outputs are zero outside every response; `out` reuses a previous dict)."""
    lib = load_library()
    for t in (logp, logp_old, advantages, weight):
        if t is not None and (t.dtype != torch.float32 or t.shape != logp.shape):
            raise TypeError("tim.ppo_loss: per-token inputs must be fp32 of one shape")
    if cu_seqlens.dtype != torch.int64 or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
        raise TypeError("tim.ppo_loss: cu_seqlens must be a non-empty int64 vector")
    _require_gpu(logp, logp_old, advantages, weight, cu_seqlens)
    T = logp.numel()
    n = cu_seqlens.numel() - 1
    dev = logp.device
    if out is not None:
        _require_gpu(*out.values())
    if not out:
        # every response's sum and the batch loss are written (with no response nothing is); only the tokens outside
        # the responses need clearing
        sums = torch.empty if n > 0 else torch.zeros
        tl, gr, ct = (torch.empty(T, dtype=torch.float32, device=dev) for _ in range(3))
        torch._foreach_zero_([tl, gr, ct])  # one launch
        out = {"seq_loss": sums(n, dtype=torch.float64, device=dev),
               "batch_loss": sums(1, dtype=torch.float64, device=dev),
               "token_loss": tl, "grad": gr, "contribution": ct,
               "clipped": torch.zeros(T, dtype=torch.uint8, device=dev)}
    _check(lib.tim_ppo_loss(_ptr(logp), _ptr(logp_old), _ptr(advantages), _ptr(weight), T, _ptr(cu_seqlens), n,
                            float(eps_low), float(eps_high), _ptr(out["seq_loss"]), _ptr(out["batch_loss"]),
                            _ptr(out["token_loss"]), _ptr(out["grad"]), _ptr(out["contribution"]),
                            _ptr(out["clipped"]), _stream(dev)))
    return out


# ------------------------------------------------------------------ the distribution a rollout engine samples from
# (include/tim_policy.h)

MXFP4_BLOCK = 32  # TIM_MXFP4_BLOCK
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}  # TIM_F32, TIM_BF16, TIM_F16


def _on_one_gpu(name, device, *tensors):
    """The operators below take tensors of one GPU, whatever the current one is."""
    for t in tensors:
        if t is not None and (not t.is_cuda or t.device != device):
            raise ValueError(f"tim.{name}: tensors must be on one GPU")


def _launch(device, call, *args):
    """call(*args, stream) on the device's current stream, with the device current while it launches."""
    if torch.cuda.current_device() == device.index:
        _check(call(*args, _stream(device)))
    else:
        with torch.cuda.device(device):
            _check(call(*args, _stream(device)))


def _dense_rows(name, what, t) -> int:
    """Elements from row to row of a matrix of dense rows that do not share elements; refuses any other."""
    if t.dim() != 2:
        raise ValueError(f"tim.{name}: {what} must be a matrix")
    (n, m), (row, col) = t.shape, t.stride()
    if n and m and ((m > 1 and col != 1) or (n > 1 and row < m)):
        raise ValueError(f"tim.{name}: {what} must have dense rows that do not overlap")
    return row if n > 1 and m else max(m, 1)  # a lone row's stride means nothing


class Mxfp4(NamedTuple):
    """Rows in 4-bit microscaled floating point: codes uint8 [rows, d / 2] (element 2j in the low half of byte j)
    and scales uint8 [rows, d / 32]; element k stands for E2M1(code) * 2^(scale of block k // 32 - 127)."""
    codes: torch.Tensor
    scales: torch.Tensor


def _mxfp4_shape(name, q) -> tuple[int, int]:
    if q.codes.dtype != torch.uint8 or q.scales.dtype != torch.uint8:
        raise TypeError(f"tim.{name}: codes and scales must be uint8")
    if q.codes.dim() != 2 or q.scales.dim() != 2:
        raise ValueError(f"tim.{name}: codes [rows, d / 2] and scales [rows, d / 32]")
    rows, d = q.codes.shape[0], 2 * q.codes.shape[1]
    if d % MXFP4_BLOCK or tuple(q.scales.shape) != (rows, d // MXFP4_BLOCK):
        raise ValueError(f"tim.{name}: codes [rows, d / 2] and scales [rows, d / 32]")
    _require_gpu(q.codes, q.scales)
    return rows, d


def mxfp4_quantize(x: torch.Tensor, out: Mxfp4 | None = None) -> Mxfp4:
    """4-bit microscaled rows of x (fp32, bf16 or fp16 [rows, d], dense rows, d a multiple of 32): each block of 32
    gets the scale 2^(floor(log2 max|x|) - 2) and its elements the nearest E2M1 values (see include/tim_policy.h)."""
    lib = load_library()
    if x.dtype not in _DTYPES:
        raise TypeError("tim.mxfp4_quantize: x must be fp32, bf16 or fp16")
    ld = _dense_rows("mxfp4_quantize", "x", x)
    rows, d = x.shape
    if d < MXFP4_BLOCK or d % MXFP4_BLOCK:
        raise ValueError("tim.mxfp4_quantize: d must be a multiple of 32")
    if out is None:
        out = Mxfp4(torch.empty((rows, d // 2), dtype=torch.uint8, device=x.device),
                    torch.empty((rows, d // MXFP4_BLOCK), dtype=torch.uint8, device=x.device))
    elif _mxfp4_shape("mxfp4_quantize", out) != (rows, d):
        raise ValueError("tim.mxfp4_quantize: out must hold [rows, d]")
    _on_one_gpu("mxfp4_quantize", x.device, x, *out)
    _launch(x.device, lib.tim_mxfp4_quantize, _ptr(x), _DTYPES[x.dtype], rows, d, ld, _ptr(out.codes),
            _ptr(out.scales))
    return out


def mxfp4_dequantize(q: Mxfp4, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values the codes stand for, exactly, as bf16 or fp32 [rows, d]."""
    lib = load_library()
    rows, d = _mxfp4_shape("mxfp4_dequantize", q)
    if out is not None:
        dtype = out.dtype
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("tim.mxfp4_dequantize: values are bf16 or fp32")
    if d == 0:
        raise ValueError("tim.mxfp4_dequantize: d must be a multiple of 32")
    if out is None:
        out = torch.empty((rows, d), dtype=dtype, device=q.codes.device)
    elif out.shape != (rows, d):
        raise ValueError("tim.mxfp4_dequantize: out must be [rows, d]")
    _require_gpu(out)
    _on_one_gpu("mxfp4_dequantize", q.codes.device, *q, out)
    _launch(q.codes.device, lib.tim_mxfp4_dequantize, _ptr(q.codes), _ptr(q.scales), rows, d, _ptr(out),
            _DTYPES[dtype])
    return out


def mxfp4_logits(hidden: Mxfp4, w_vocab: Mxfp4, temperature: float = 1.0, dtype: torch.dtype = torch.float32,
                 out: torch.Tensor | None = None) -> torch.Tensor:
    """[T, V] logits of 4-bit hidden rows [T, d] against a 4-bit head [V, d] (d a multiple of 128), accumulated in
    fp32 and rounded once to dtype (fp32, bf16 or fp16). out, if given, may have padded rows."""
    lib = load_library()
    T, d = _mxfp4_shape("mxfp4_logits", hidden)
    V, dw = _mxfp4_shape("mxfp4_logits", w_vocab)
    if d != dw:
        raise ValueError("tim.mxfp4_logits: hidden [T, d] and w_vocab [V, d] must share d")
    dev = hidden.codes.device
    if out is None:
        out = torch.empty((T, V), dtype=dtype, device=dev)
    elif out.shape != (T, V):
        raise ValueError("tim.mxfp4_logits: out must be [T, V]")
    if out.dtype not in _DTYPES:
        raise TypeError("tim.mxfp4_logits: logits are fp32, bf16 or fp16")
    ld = _dense_rows("mxfp4_logits", "out", out)
    _on_one_gpu("mxfp4_logits", dev, *hidden, *w_vocab, out)
    _launch(dev, lib.tim_mxfp4_logits, _ptr(hidden.codes), _ptr(hidden.scales), _ptr(w_vocab.codes),
            _ptr(w_vocab.scales), T, d, V, float(temperature), _ptr(out), _DTYPES[out.dtype], ld)
    return out


def _matrix_layout(t: torch.Tensor) -> tuple:
    """Where a tensor lies and how."""
    return t.data_ptr(), t.dtype, t.shape, t.stride()


@dataclasses.dataclass
class LogitRules:
    """What changes the logits of T rows before sampling (tim_logit_rules in include/tim_policy.h); leave out what
    does not apply. All tensors on the logits' GPU.

    history int32 [N] tokens; row i's are history[hist_begin[i]:hist_end[i]], generated from hist_split[i] on
    (int64 [T] each; no hist_split: all generated). repetition divides positive and multiplies other logits of
    tokens in the history, frequency is subtracted per occurrence in the generated part, presence once (fp32 [T]).
    bias_ids int32 [M] and bias_values fp32 [M]; row i adds the entries bias_begin[i]:bias_end[i] (int64 [T]; of an
    id listed twice the last). mask int32 [n, >= ceil(V / 32)], bit v % 32 of word v // 32 set where v is allowed;
    row i takes mask mask_rows[i] (int32 [T], outside [0, n): none) or, without mask_rows, mask i. The bias comes after
    the penalties; for an engine that adds it before them, logits_adjust with a rule set of the bias alone goes first."""
    history: torch.Tensor | None = None
    hist_begin: torch.Tensor | None = None
    hist_split: torch.Tensor | None = None
    hist_end: torch.Tensor | None = None
    repetition: torch.Tensor | None = None
    frequency: torch.Tensor | None = None
    presence: torch.Tensor | None = None
    bias_ids: torch.Tensor | None = None
    bias_values: torch.Tensor | None = None
    bias_begin: torch.Tensor | None = None
    bias_end: torch.Tensor | None = None
    mask: torch.Tensor | None = None
    mask_rows: torch.Tensor | None = None

    def __setattr__(self, field, value):
        object.__setattr__(self, field, value)
        object.__setattr__(self, "_built", None)

    def __getstate__(self):
        return {f.name: getattr(self, f.name) for f in dataclasses.fields(self)}

    def __setstate__(self, state):
        for field, value in state.items():
            setattr(self, field, value)

    def _struct(self, name, T, V, device) -> _LogitRules:
        """The C struct for T rows of V logits on the device. It is checked and filled once and kept until a field is
        set or a tensor's storage, size, strides or type are others; what the tensors hold may change in between."""
        if self._built is not None:
            s, held, rows, words, on, mask = self._built
            if rows == T and words * 32 >= V and on == device and (mask is None or _matrix_layout(self.mask) == mask):
                for t, ptr, n, dtype in held:
                    if t.data_ptr() != ptr or t.nbytes != n or t.dtype is not dtype or not t.is_contiguous():
                        break
                else:
                    return s
        s, held, words = _LogitRules(), [], MAX_VOCAB

        def take(field, dtype, n=None):
            t = getattr(self, field)
            if t is None:
                return
            if t.dtype != dtype:
                raise TypeError(f"tim.{name}: {field} must be {dtype}")
            if t.dim() != 1 or (n is not None and t.shape[0] != n):
                raise ValueError(f"tim.{name}: {field} must be a vector" + ("" if n is None else " of one value a row"))
            if t.device != device:
                raise ValueError(f"tim.{name}: tensors must be on one GPU")
            if not t.is_contiguous():
                raise ValueError(f"tim.{name}: {field} must be contiguous")
            setattr(s, field, t.data_ptr())
            held.append((t, t.data_ptr(), t.nbytes, dtype))

        if self.history is not None:
            if self.hist_begin is None or self.hist_end is None:
                raise ValueError(f"tim.{name}: history needs hist_begin and hist_end")
            take("history", torch.int32)
            s.history_len = self.history.shape[0]
            for f in ("hist_begin", "hist_split", "hist_end"):
                take(f, torch.int64, T)
        for f in ("repetition", "frequency", "presence"):
            take(f, torch.float32, T)
        if self.bias_ids is not None:
            if self.bias_values is None or self.bias_begin is None or self.bias_end is None:
                raise ValueError(f"tim.{name}: bias_ids needs bias_values, bias_begin and bias_end")
            take("bias_ids", torch.int32)
            s.bias_len = self.bias_ids.shape[0]
            take("bias_values", torch.float32, s.bias_len)
            take("bias_begin", torch.int64, T)
            take("bias_end", torch.int64, T)
        if self.mask is not None:
            if self.mask.dtype != torch.int32:
                raise TypeError(f"tim.{name}: mask must be torch.int32")
            ld = _dense_rows(name, "mask", self.mask)
            if self.mask.device != device:
                raise ValueError(f"tim.{name}: tensors must be on one GPU")
            words = self.mask.shape[1]
            if words * 32 < V:
                raise ValueError(f"tim.{name}: mask must have ceil(V / 32) words a row")
            if self.mask_rows is None and self.mask.shape[0] != T:
                raise ValueError(f"tim.{name}: without mask_rows there is one mask a row")
            s.mask, s.n_masks, s.mask_ld = self.mask.data_ptr(), self.mask.shape[0], ld
            take("mask_rows", torch.int32, T)
        mask = None if self.mask is None else _matrix_layout(self.mask)
        object.__setattr__(self, "_built", (s, held, T, words, device, mask))
        return s


def _changed(name, logits, rules):
    """(T, V, row stride, C rules or None) of the operators on changed logits."""
    if logits.dtype not in _DTYPES:
        raise TypeError(f"tim.{name}: logits must be fp32, bf16 or fp16")
    ld = _dense_rows(name, "logits", logits)
    if not logits.is_cuda:
        raise ValueError("tim: tensors must be on the GPU")
    T, V = logits.shape
    return T, V, ld, None if rules is None else ctypes.byref(rules._struct(name, T, V, logits.device))


def _row_vector(name, what, t, T, dtype):
    if t is None:
        return
    if t.dtype != dtype:
        raise TypeError(f"tim.{name}: {what} must be {dtype}")
    if t.shape != (T,):
        raise ValueError(f"tim.{name}: {what} must be [T]")
    _require_gpu(t)


def logits_adjust(logits: torch.Tensor, rules: LogitRules | None = None, temperature: float = 1.0,
                  out: torch.Tensor | None = None) -> torch.Tensor:
    """The logits [T, V] (fp32, bf16 or fp16, dense rows) as a sampler reads them: penalties, bias, temperature and
    mask applied, each entry rounded once to the logits' type. out may be logits itself (in place), but no other
    overlap of the two is allowed."""
    lib = load_library()
    T, V, ld, r = _changed("logits_adjust", logits, rules)
    if out is None:
        out = logits.new_empty(T, V)  # half a microsecond less than torch.empty with a type and a device
        out_ld = max(V, 1)
    else:
        if out.shape != (T, V) or out.dtype != logits.dtype:
            raise ValueError("tim.logits_adjust: out must be like logits")
        out_ld = _dense_rows("logits_adjust", "out", out)
        _on_one_gpu("logits_adjust", logits.device, out)
    _launch(logits.device, lib.tim_logits_adjust, _ptr(logits), _DTYPES[logits.dtype], T, V, ld, r, float(temperature),
            _ptr(out), out_ld)
    return out


def logits_logprobs_workspace_size(T: int, V: int) -> int:
    """Bytes of workspace tim_logits_logprobs needs (0 for T == 0 or invalid shapes)."""
    return int(load_library().tim_logits_logprobs_workspace_size(int(T), int(V)))


def logits_logprobs(logits: torch.Tensor, tokens: torch.Tensor, rules: LogitRules | None = None,
                    temperature: float = 1.0, entropy: bool = True, lse: bool = False,
                    workspace: torch.Tensor | None = None, out: tuple | None = None):
    """Log-probabilities (and entropies, log-normalisers) of tokens int32 [T] under the changed logits of
    logits_adjust, from the logits themselves. Returns (logp, entropy or None, lse or None), fp32 [T] each."""
    lib = load_library()
    T, V, ld, r = _changed("logits_logprobs", logits, rules)
    dev = logits.device
    _row_vector("logits_logprobs", "tokens", tokens, T, torch.int32)
    if out is None:
        rows = iter(torch.empty((1 + bool(entropy) + bool(lse), T), dtype=torch.float32, device=dev).unbind(0))
        lp = next(rows)
        ent = next(rows) if entropy else None
        ls = next(rows) if lse else None
        _on_one_gpu("logits_logprobs", dev, tokens)
    else:
        lp, ent, ls = out
        for what, t in (("logp", lp), ("entropy", ent), ("lse", ls)):
            _row_vector("logits_logprobs", what, t, T, torch.float32)
        _on_one_gpu("logits_logprobs", dev, tokens, lp, ent, ls)
    if T == 0:
        return lp, ent, ls
    if workspace is None:
        workspace = torch.empty(logits_logprobs_workspace_size(T, V), dtype=torch.uint8, device=dev)
    else:
        _require_gpu(workspace)
        _on_one_gpu("logits_logprobs", dev, workspace)
    _launch(dev, lib.tim_logits_logprobs, _ptr(logits), _DTYPES[logits.dtype], T, V, ld, _ptr(tokens), r,
            float(temperature), _ptr(lp), _ptr(ent), _ptr(ls), _ptr(workspace),
            workspace.numel() * workspace.element_size())
    return lp, ent, ls


def logits_logprobs_backward(logits: torch.Tensor, tokens: torch.Tensor, lse: torch.Tensor, grad_logp: torch.Tensor,
                             rules: LogitRules | None = None, temperature: float = 1.0,
                             entropy: torch.Tensor | None = None, grad_entropy: torch.Tensor | None = None,
                             dtype: torch.dtype | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient [T, V] of sum_t grad_logp[t] logp[t] + grad_entropy[t] entropy[t] with respect to the logits, through
    the changes. lse (and entropy, when grad_entropy is given) are logits_logprobs' outputs for the same inputs; rows of
    |lse| >= 1024, where it is too coarse, take their normaliser from the logits and longer.
    dtype (the logits' by default) is the gradient's type; out may be logits itself where the types agree,
    but no other overlap is allowed."""
    lib = load_library()
    T, V, ld, r = _changed("logits_logprobs_backward", logits, rules)
    dev = logits.device
    _row_vector("logits_logprobs_backward", "tokens", tokens, T, torch.int32)
    for what, t in (("lse", lse), ("grad_logp", grad_logp), ("entropy", entropy), ("grad_entropy", grad_entropy)):
        _row_vector("logits_logprobs_backward", what, t, T, torch.float32)
    if out is None:
        out = torch.empty((T, V), dtype=logits.dtype if dtype is None else dtype, device=dev)
    elif dtype is not None and out.dtype != dtype:
        raise ValueError("tim.logits_logprobs_backward: out must have the dtype asked for")
    if out.dtype not in _DTYPES:
        raise TypeError("tim.logits_logprobs_backward: the gradient is fp32, bf16 or fp16")
    if out.shape != (T, V):
        raise ValueError("tim.logits_logprobs_backward: out must be [T, V]")
    out_ld = _dense_rows("logits_logprobs_backward", "out", out)
    _on_one_gpu("logits_logprobs_backward", dev, tokens, lse, grad_logp, entropy, grad_entropy, out)
    _launch(dev, lib.tim_logits_logprobs_backward, _ptr(logits), _DTYPES[logits.dtype], T, V, ld, _ptr(tokens), r,
            float(temperature), _ptr(lse), _ptr(entropy), _ptr(grad_logp), _ptr(grad_entropy), _ptr(out),
            _DTYPES[out.dtype], out_ld)
    return out


# ------------------------------------------------------------------ what stands beside the head
# (include/tim_vocab.h)


def _scratch(name, workspace, device, size, *args) -> torch.Tensor:
    """The caller's workspace, or a new one of size(*args) bytes."""
    if workspace is None:
        return torch.empty(size(*args), dtype=torch.uint8, device=device)
    _require_gpu(workspace)
    _on_one_gpu(name, device, workspace)
    return workspace


def _int32(name, *sizes):
    """Sizes that the C interface takes as 32-bit integers."""
    if any(not 0 <= n < 1 << 31 for n in sizes):
        raise ValueError(f"tim.{name}: a size is out of range")


def embedding(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, dtype: torch.dtype | None = None,
              out: torch.Tensor | None = None) -> torch.Tensor:
    """scale * table[tokens]: rows [T, d] of table [V, d] (fp32, bf16 or fp16, dense rows) for tokens int32 [T], each
    element formed in fp32 and rounded once to dtype (the table's by default); zeros for a token outside [0, V)
    (padding). out, if given, may have padded rows, and shares no memory with the inputs."""
    lib = load_library()
    if table.dtype not in _DTYPES:
        raise TypeError("tim.embedding: the table must be fp32, bf16 or fp16")
    ld = _dense_rows("embedding", "table", table)
    V, d = table.shape
    _int32("embedding", V, d)
    if tokens.dim() != 1:
        raise ValueError("tim.embedding: tokens must be [T]")
    T = tokens.shape[0]
    _row_vector("embedding", "tokens", tokens, T, torch.int32)
    if out is None:
        out = torch.empty((T, d), dtype=table.dtype if dtype is None else dtype, device=table.device)
    elif dtype is not None and out.dtype != dtype:
        raise ValueError("tim.embedding: out must have the dtype asked for")
    if out.dtype not in _DTYPES:
        raise TypeError("tim.embedding: rows are fp32, bf16 or fp16")
    if out.shape != (T, d):
        raise ValueError("tim.embedding: out must be [T, d]")
    out_ld = _dense_rows("embedding", "out", out)
    _on_one_gpu("embedding", table.device, table, tokens, out)
    _launch(table.device, lib.tim_embedding, _ptr(table), _DTYPES[table.dtype], V, d, ld, _ptr(tokens), T, float(scale),
            _ptr(out), _DTYPES[out.dtype], out_ld)
    return out


def embedding_backward_workspace_size(T: int, V: int, d: int) -> int:
    """Bytes of workspace tim_embedding_backward needs (0 for T == 0 or invalid shapes)."""
    return int(load_library().tim_embedding_backward_workspace_size(int(T), int(V), int(d)))


def embedding_backward(grad: torch.Tensor, tokens: torch.Tensor, V: int, scale: float = 1.0,
                       grad_table: torch.Tensor | None = None, accumulate: bool = False,
                       workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient fp32 [V, d] of the embedding's table from that of its rows, grad [T, d] (fp32, bf16 or fp16, dense
    rows). With accumulate the sums are added to grad_table (the grad_w of logprobs_backward for a tied head) in the rows
    of the tokens that occur; otherwise every row is written. grad_table shares no memory with the inputs.
    Deterministic."""
    lib = load_library()
    if grad.dtype not in _DTYPES:
        raise TypeError("tim.embedding_backward: grad must be fp32, bf16 or fp16")
    ld = _dense_rows("embedding_backward", "grad", grad)
    T, d = grad.shape
    V = int(V)
    _int32("embedding_backward", V, d)
    _row_vector("embedding_backward", "tokens", tokens, T, torch.int32)
    dev = grad.device
    if grad_table is None:
        if accumulate:
            raise ValueError("tim.embedding_backward: accumulate needs the grad_table buffer")
        grad_table = torch.empty((V, d), dtype=torch.float32, device=dev)
    if grad_table.dtype != torch.float32:
        raise TypeError("tim.embedding_backward: grad_table must be fp32")
    if grad_table.shape != (V, d):
        raise ValueError("tim.embedding_backward: grad_table must be [V, d]")
    table_ld = _dense_rows("embedding_backward", "grad_table", grad_table)
    ws = _scratch("embedding_backward", workspace, dev, lib.tim_embedding_backward_workspace_size, T, V, d)
    _on_one_gpu("embedding_backward", dev, grad, tokens, grad_table)
    _launch(dev, lib.tim_embedding_backward, _ptr(grad), _DTYPES[grad.dtype], T, d, ld, _ptr(tokens), V, float(scale),
            _ptr(grad_table), table_ld, 1 if accumulate else 0, _ptr(ws), ws.numel() * ws.element_size())
    return grad_table


@dataclasses.dataclass
class Adapters:
    """Low-rank adapters of a projection from d to N elements: adapter k adds scales[k] (x a[k]^T) b[k]^T. a [n, r, d] and
    b [n, N, r] of one type (bf16 or fp16), contiguous; scales fp32 [n], None for ones. What the tensors hold may change
    between calls, as training changes it."""
    a: torch.Tensor
    b: torch.Tensor
    scales: torch.Tensor | None = None

    def __setattr__(self, field, value):
        object.__setattr__(self, field, value)
        object.__setattr__(self, "_built", None)

    def __getstate__(self):
        return {f.name: getattr(self, f.name) for f in dataclasses.fields(self)}

    def __setstate__(self, state):
        for field, value in state.items():
            setattr(self, field, value)

    def _struct(self, name) -> _Adapters:
        """The C struct. It is checked and filled once and kept until a field is set or a tensor's storage, size, strides or
        type are others."""
        a, b, scales = self.a, self.b, self.scales
        layout = (_matrix_layout(a), _matrix_layout(b), None if scales is None else _matrix_layout(scales))
        if self._built is not None and self._built[1] == layout:
            return self._built[0]
        if a.dtype not in (torch.bfloat16, torch.float16) or b.dtype != a.dtype:
            raise TypeError(f"tim.{name}: a, b and x must be bf16, or all fp16")
        if a.dim() != 3 or b.dim() != 3 or a.shape[0] != b.shape[0] or a.shape[1] != b.shape[2]:
            raise ValueError(f"tim.{name}: a [n, r, d] and b [n, N, r]")
        n, r, d = a.shape
        _int32(name, n, r, d, b.shape[1])
        if scales is not None:
            if scales.dtype != torch.float32:
                raise TypeError(f"tim.{name}: scales must be fp32")
            if scales.shape != (n,):
                raise ValueError(f"tim.{name}: scales must be [n]")
        _require_gpu(a, b, scales)
        _on_one_gpu(name, a.device, b, scales)
        s = _Adapters(_ptr(a), _ptr(b), _ptr(scales), _DTYPES[a.dtype], n, r, d, b.shape[1])
        object.__setattr__(self, "_built", (s, layout))
        return s


def _adapters(name, adapters, x, rows) -> tuple[_Adapters, int, int]:
    """(C struct, T, row stride of x) of the adapters and the rows they apply to."""
    ad = adapters._struct(name)
    if x.dtype != adapters.a.dtype:
        raise TypeError(f"tim.{name}: a, b and x must be bf16, or all fp16")
    x_ld = _dense_rows(name, "x", x)
    T, d = x.shape
    if d != ad.d:
        raise ValueError(f"tim.{name}: x must be [T, d]")
    _row_vector(name, "rows", rows, T, torch.int32)
    _on_one_gpu(name, x.device, x, rows, adapters.a)
    return ad, T, x_ld


def adapters_add_workspace_size(T: int, d: int, N: int, n: int, r: int) -> int:
    """Bytes of workspace tim_adapters_add needs (0 for T == 0 or invalid shapes)."""
    return int(load_library().tim_adapters_add_workspace_size(int(T), int(d), int(N), int(n), int(r)))


def adapters_add(base: torch.Tensor | None, x: torch.Tensor, rows: torch.Tensor, adapters: Adapters,
                 dtype: torch.dtype | None = None, out: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None) -> torch.Tensor:
    """base [T, N] (a shared projection's output, the head's logits among them; None: zeros) plus the adapter of each row
    of x [T, d]: row t's is adapters rows[t] (int32 [T]), none where that is outside [0, n). fp32 sums, rounded once to
    base's type (to dtype without a base, x's by default). out may be base itself (in place), and x may be too, but no other
    overlap is allowed."""
    lib = load_library()
    ad, T, x_ld = _adapters("adapters_add", adapters, x, rows)
    dev, N = x.device, ad.N
    base_ld = N
    if base is not None:
        if base.shape != (T, N):
            raise ValueError("tim.adapters_add: base must be [T, N]")
        base_ld = _dense_rows("adapters_add", "base", base)
        _on_one_gpu("adapters_add", dev, base)
        if dtype is not None and dtype != base.dtype:
            raise ValueError("tim.adapters_add: the output has base's type")
        dtype = base.dtype
    if out is None:
        out = x.new_empty(T, N) if base is None else base.new_empty(T, N)
        out_ld = max(N, 1)
        if base is None and dtype is not None and dtype != x.dtype:
            out = torch.empty((T, N), dtype=dtype, device=dev)
    else:
        if out.shape != (T, N) or (dtype is not None and out.dtype != dtype):
            raise ValueError("tim.adapters_add: out must be [T, N] of the output's type")
        out_ld = _dense_rows("adapters_add", "out", out)
        _on_one_gpu("adapters_add", dev, out)
    if out.dtype not in _DTYPES:
        raise TypeError("tim.adapters_add: the output is fp32, bf16 or fp16")
    ws = _scratch("adapters_add", workspace, dev, lib.tim_adapters_add_workspace_size, T, ad.d, ad.N, ad.n, ad.r)
    _launch(dev, lib.tim_adapters_add, ctypes.byref(ad), _ptr(x), x_ld, _ptr(rows), T, _ptr(base), base_ld, _ptr(out),
            _DTYPES[out.dtype], out_ld, _ptr(ws), ws.numel() * ws.element_size())
    return out


def adapters_backward_workspace_size(T: int, d: int, N: int, n: int, r: int) -> int:
    """Bytes of workspace tim_adapters_backward needs (0 for T == 0 or invalid shapes)."""
    return int(load_library().tim_adapters_backward_workspace_size(int(T), int(d), int(N), int(n), int(r)))


def adapters_backward(grad: torch.Tensor, x: torch.Tensor, rows: torch.Tensor, adapters: Adapters, want_x: bool = True,
                      want_a: bool = True, want_b: bool = True, dtype: torch.dtype | None = None,
                      grad_x: torch.Tensor | None = None, accumulate_x: bool = False,
                      grad_a: torch.Tensor | None = None, grad_b: torch.Tensor | None = None, accumulate: bool = False,
                      workspace: torch.Tensor | None = None):
    """(grad_x [T, d] or None, grad_a fp32 [n, r, d] or None, grad_b fp32 [n, N, r] or None) through adapters_add, from
    the gradient [T, N] of its output (fp32, bf16 or fp16, dense rows). grad_x is of dtype (x's by default); with
    accumulate_x it is added to the grad_x given, with accumulate grad_a and grad_b to theirs. Rows without an adapter and
    adapters without rows get zeros, or nothing added. The gradients share no memory with each other or with the inputs,
    but grad_x may take grad's place (not x's)."""
    lib = load_library()
    name = "adapters_backward"
    ad, T, x_ld = _adapters(name, adapters, x, rows)
    dev = x.device
    if grad.dtype not in _DTYPES:
        raise TypeError(f"tim.{name}: grad must be fp32, bf16 or fp16")
    if grad.shape != (T, ad.N):
        raise ValueError(f"tim.{name}: grad must be [T, N]")
    grad_ld = _dense_rows(name, "grad", grad)
    _on_one_gpu(name, dev, grad)
    gx_ld, gx_type = ad.d, 0
    if want_x:
        if grad_x is None:
            if accumulate_x:
                raise ValueError(f"tim.{name}: accumulate_x needs the grad_x buffer")
            grad_x = torch.empty((T, ad.d), dtype=x.dtype if dtype is None else dtype, device=dev)
        elif dtype is not None and grad_x.dtype != dtype:
            raise ValueError(f"tim.{name}: grad_x must have the dtype asked for")
        if grad_x.dtype not in _DTYPES:
            raise TypeError(f"tim.{name}: grad_x is fp32, bf16 or fp16")
        if grad_x.shape != (T, ad.d):
            raise ValueError(f"tim.{name}: grad_x must be [T, d]")
        gx_ld, gx_type = _dense_rows(name, "grad_x", grad_x), _DTYPES[grad_x.dtype]
        _on_one_gpu(name, dev, grad_x)
    weights = []
    for want, what, t, shape in ((want_a, "grad_a", grad_a, (ad.n, ad.r, ad.d)),
                                 (want_b, "grad_b", grad_b, (ad.n, ad.N, ad.r))):
        if want and t is None:
            if accumulate:
                raise ValueError(f"tim.{name}: accumulate needs the {what} buffer")
            t = torch.empty(shape, dtype=torch.float32, device=dev)
        if want:
            if t.dtype != torch.float32:
                raise TypeError(f"tim.{name}: {what} must be fp32")
            if t.shape != shape:
                raise ValueError(f"tim.{name}: {what} must be {list(shape)}")
            _require_gpu(t)
            _on_one_gpu(name, dev, t)
        weights.append(t if want else None)
    ws = _scratch(name, workspace, dev, lib.tim_adapters_backward_workspace_size, T, ad.d, ad.N, ad.n, ad.r)
    grad_x = grad_x if want_x else None
    _launch(dev, lib.tim_adapters_backward, ctypes.byref(ad), _ptr(x), x_ld, _ptr(rows), T, _ptr(grad),
            _DTYPES[grad.dtype], grad_ld, _ptr(grad_x), gx_type, gx_ld, 1 if accumulate_x else 0, _ptr(weights[0]),
            _ptr(weights[1]), 1 if accumulate else 0, _ptr(ws), ws.numel() * ws.element_size())
    return grad_x, weights[0], weights[1]
