"""What stands before a language model's quantized linears and behind its last one. Python binding of
the w8a8_rms_norm_* and w8a8_token_logprobs entry points (include/w8a8.h has the rules); imported by
the package, whose conventions hold here too.

  rms_norm_quantize(x, weight)    -> (codes, scales, h): for gemm, or for mx4_gemm
  token_logprobs(logits, tokens)  -> (logp, entropy, top_logp, top_ids)
"""
from __future__ import annotations

import functools

import torch

from . import _check, _check_out, _launch, _ptr, _same_device, _size, _workspace
from .mx import _mx4_shapes

_bytes = functools.lru_cache(maxsize=4096)(_size)

__all__ = ["rms_norm_quantize", "token_logprobs", "NORM_FORMATS", "MAX_TOP"]

NORM_FORMATS = ("int8", "mx4")
MAX_TOP = 64


def rms_norm_quantize(x, weight=None, *, residual=None, eps: float = 1e-6, fmt: str = "int8",
                      sum_out=None):
    """Root-mean-square norm of h = x + residual (rounded to bf16; h is x itself without a residual),
    quantized for the linear behind it: x, residual bf16 [M, K], weight fp32 [K] or None (ones; a
    smoothed linear's 1/s is folded in here). Returns (codes, scales, h):
      fmt "int8"  codes int8 [M, K], scales fp32 [M], as quantize_act gives them, for gemm
      fmt "mx4"   codes uint8 [M, 16 ceil(K/32)], scales uint8 [ceil(K/256), M, 8], as mx4_quantize
                  gives them, for mx4_gemm
    sum_out: where h goes (with a residual; x or residual themselves are allowed)."""
    if fmt not in NORM_FORMATS:
        raise ValueError(f"fmt must be one of {list(NORM_FORMATS)}, got {fmt!r}")
    _check(x, torch.bfloat16, 2, "x")
    M, K = x.shape
    device = x.device
    if weight is not None:
        _check(weight, torch.float32, 1, "weight")
        if weight.shape[0] != K:
            raise ValueError(f"weight must have {K} entries, got {weight.shape[0]}")
    h = x
    if residual is not None:
        _check(residual, torch.bfloat16, 2, "residual")
        if residual.shape != x.shape:
            raise ValueError("shape mismatch")
        if sum_out is not None:
            _check_out(sum_out, torch.bfloat16, (M, K), device, "sum_out")
        h = torch.empty_like(x) if sum_out is None else sum_out
    elif sum_out is not None:
        raise ValueError("sum_out needs a residual")
    _same_device(x, weight, residual)
    if fmt == "int8":
        name = "w8a8_rms_norm_quantize"
        codes = torch.empty_like(x, dtype=torch.int8)
        scales = torch.empty(M, dtype=torch.float32, device=device)
    else:
        name = "w8a8_rms_norm_mx4_quantize"
        cs, ss = _mx4_shapes(M, K)
        codes = torch.empty(cs, dtype=torch.uint8, device=device)
        scales = torch.empty(ss, dtype=torch.uint8, device=device)
    _launch(device, name, _ptr(x), _ptr(residual), None if residual is None else h.data_ptr(),
            _ptr(weight), eps, M, K, codes.data_ptr(), scales.data_ptr())
    return codes, scales, h


def token_logprobs(logits, tokens, *, top: int = 0, temperature: float = 1.0, workspace=None):
    """Log probabilities under softmax(logits / temperature), in fp32. logits: bf16 or fp32 [T, V],
    rows any stride apart; tokens int64 [T], negative (or past V) for padding. Returns
    (logp [T], entropy [T], top_logp [T, top], top_ids int64 [T, top]): of the given tokens (0 for
    padding), of the distribution, and of its `top` (up to 64) likeliest tokens, the lower index
    first where logits are equal. A row without a finite logit, or with a NaN or plus infinity,
    gives NaN."""
    if not isinstance(logits, torch.Tensor) or logits.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("logits must be a bf16 or fp32 torch.Tensor")
    if logits.dim() != 2 or logits.device.type != "cuda" or (
            logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError(f"logits must be [T, V] with contiguous rows on a HIP device, got "
                         f"{tuple(logits.shape)} on {logits.device}")
    T, V = logits.shape
    device = logits.device
    _check(tokens, torch.int64, 1, "tokens")
    if tokens.shape[0] != T:
        raise ValueError(f"tokens must have {T} entries, got {tokens.shape[0]}")
    _same_device(logits, tokens)
    top = int(top)
    if not 0 <= top <= min(MAX_TOP, V):
        raise ValueError(f"top must be 0 to {min(MAX_TOP, V)}, got {top}")
    logp = torch.empty_like(tokens, dtype=torch.float32)
    entropy = torch.empty_like(logp)
    top_logp, ids = logp.new_empty((T, top)), tokens.new_empty((T, top))
    ws = _workspace(_bytes("w8a8_token_logprobs_workspace_bytes", T, V, top), device, workspace)
    _launch(device, "w8a8_token_logprobs", logits.data_ptr(), int(logits.dtype == torch.float32),
            logits.stride(0), T, V, _ptr(tokens), top, temperature, logp.data_ptr(),
            entropy.data_ptr(), top_logp.data_ptr(), ids.data_ptr(), _ptr(ws),
            0 if ws is None else ws.nbytes)
    return logp, entropy, top_logp, ids
