"""torch.library registration of the W8A8 linear, and a drop-in module.

The fused op replaces the bf16 linear at a diffusion transformer's linear layers with
the surrounding runtime unchanged (Section 3, "Integration"). Registered as custom ops
with fake (meta) implementations, the calls stay inside one graph under torch.compile
instead of breaking it at an opaque Python call:

  torch.ops.w8a8.linear(x, wq, w_scale, bias, act, col_mul) -> y bf16 [..., N]
  torch.ops.w8a8.quantize_act(x, act, col_mul)             -> (xq int8, x_scale fp32)
  torch.ops.w8a8.gemm(xq, x_scale, wq, w_scale, bias)      -> y bf16 [M, N]

and, for the microscaled operators,

  torch.ops.w8a8.mx4_linear(x, wq, w_scale, bias, act, col_mul) -> y bf16 [..., N]
  torch.ops.w8a8.mx4_quantize(x, act, col_mul)                  -> (codes, scales) uint8
  torch.ops.w8a8.kv_write(cache, k, v, slots, fmt)              (writes to cache)
  torch.ops.w8a8.kv_read(cache, slots, head_dim, fmt)           -> (k, v) bf16
  torch.ops.w8a8.kv_attention(q, cache, block_table, kv_lens, q_starts, fmt, scale, causal,
                              max_q, max_kv)                    -> bf16 like q
  torch.ops.w8a8.kv_append(cache, k, v, slots, positions, inv_freq, q, fmt, sections, interleaved)
                                                 -> bf16 like q (writes to cache; empty without q)
  torch.ops.w8a8.kv_tree_attention(q, cache, block_table, kv_lens, tree, q_starts, fmt, scale,
                                   max_q, max_kv)               -> bf16 like q
  torch.ops.w8a8.rms_norm_quantize(x, weight, residual, eps, fmt) -> (codes, scales, h)
  torch.ops.w8a8.token_logprobs(logits, tokens, top, temperature)
                                                 -> (logp, entropy, top_logp, top_ids)

The ops are inference-only (no autograd formula): the integer codes have no useful
gradient. The real implementations are the HIP library's entry points; the fake ones
only compute output shapes and dtypes.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import (ACTS, gemm, kv_append, kv_attention, kv_read, kv_tree_attention, kv_write, linear,
               mx4_linear, mx4_quantize, quantize_act, quantize_weight, rms_norm_quantize,
               token_logprobs)

_ACT_NAMES = {v: k for k, v in ACTS.items()}


@torch.library.custom_op("w8a8::linear", mutates_args=())
def linear_op(x: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor,
              bias: Optional[torch.Tensor], act: int,
              col_mul: Optional[torch.Tensor]) -> torch.Tensor:
    return linear(x, wq, w_scale, bias, act=_ACT_NAMES[act], col_mul=col_mul)


@linear_op.register_fake
def _linear_fake(x, wq, w_scale, bias, act, col_mul):
    torch._check(x.shape[-1] == wq.shape[1], lambda: "K mismatch")
    return x.new_empty((*x.shape[:-1], wq.shape[0]), dtype=torch.bfloat16)


@torch.library.custom_op("w8a8::quantize_act", mutates_args=())
def quantize_act_op(x: torch.Tensor, act: int,
                    col_mul: Optional[torch.Tensor]) -> tuple[torch.Tensor, torch.Tensor]:
    return quantize_act(x, act=_ACT_NAMES[act], col_mul=col_mul)


@quantize_act_op.register_fake
def _quantize_act_fake(x, act, col_mul):
    return (x.new_empty(x.shape, dtype=torch.int8),
            x.new_empty((x.shape[0],), dtype=torch.float32))


@torch.library.custom_op("w8a8::gemm", mutates_args=())
def gemm_op(xq: torch.Tensor, x_scale: torch.Tensor, wq: torch.Tensor,
            w_scale: torch.Tensor, bias: Optional[torch.Tensor]) -> torch.Tensor:
    return gemm(xq, x_scale, wq, w_scale, bias)


@gemm_op.register_fake
def _gemm_fake(xq, x_scale, wq, w_scale, bias):
    torch._check(xq.shape[1] == wq.shape[1], lambda: "K mismatch")
    return xq.new_empty((xq.shape[0], wq.shape[0]), dtype=torch.bfloat16)


class W8A8Linear(torch.nn.Module):
    """Inference replacement for a bf16 nn.Linear: per-channel int8 weights (quantized
    once, here), per-token int8 activations and the fused int8 GEMM + dequantization
    epilogue on every call. With `smooth` (SmoothQuant factors s [K]) the weights are
    quantized as W * s and the activations multiplied by 1/s inside the quantizer; with
    act="gelu" the module consumes the pre-activation of a GELU MLP."""

    def __init__(self, wq: torch.Tensor, w_scale: torch.Tensor,
                 bias: Optional[torch.Tensor] = None, *, act: str = "none",
                 smooth_inv: Optional[torch.Tensor] = None):
        super().__init__()
        self.register_buffer("wq", wq)
        self.register_buffer("w_scale", w_scale)
        self.register_buffer("bias", bias)
        self.register_buffer("smooth_inv", smooth_inv)
        self.act = ACTS[act]
        self.in_features = wq.shape[1]
        self.out_features = wq.shape[0]

    @classmethod
    def from_linear(cls, lin: torch.nn.Linear, *, act: str = "none",
                    smooth: Optional[torch.Tensor] = None,
                    smooth_inv: Optional[torch.Tensor] = None) -> "W8A8Linear":
        if (smooth is None) != (smooth_inv is None):
            raise ValueError("pass both smooth and smooth_inv, or neither")
        w = lin.weight.detach().to(torch.bfloat16).contiguous()
        wq, sw = quantize_weight(w, col_mul=smooth)
        b = None if lin.bias is None else lin.bias.detach().to(torch.bfloat16).contiguous()
        return cls(wq, sw, b, act=act, smooth_inv=smooth_inv)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return torch.ops.w8a8.linear.default(x, self.wq, self.w_scale, self.bias, self.act,
                                             self.smooth_inv)

    def extra_repr(self) -> str:
        return (f"in_features={self.in_features}, out_features={self.out_features}, "
                f"act={_ACT_NAMES[self.act]}, smoothed={self.smooth_inv is not None}")


# ---------------------------------------------------------------- microscaled operators

@torch.library.custom_op("w8a8::mx4_linear", mutates_args=())
def mx4_linear_op(x: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor,
                  bias: Optional[torch.Tensor], act: int,
                  col_mul: Optional[torch.Tensor]) -> torch.Tensor:
    return mx4_linear(x, wq, w_scale, bias, act=_ACT_NAMES[act], col_mul=col_mul)


@mx4_linear_op.register_fake
def _mx4_linear_fake(x, wq, w_scale, bias, act, col_mul):
    torch._check((x.shape[-1] + 31) // 32 * 16 == wq.shape[1], lambda: "K mismatch")
    return x.new_empty((*x.shape[:-1], wq.shape[0]), dtype=torch.bfloat16)


@torch.library.custom_op("w8a8::mx4_quantize", mutates_args=())
def mx4_quantize_op(x: torch.Tensor, act: int,
                    col_mul: Optional[torch.Tensor]) -> tuple[torch.Tensor, torch.Tensor]:
    return mx4_quantize(x, act=_ACT_NAMES[act], col_mul=col_mul)


@mx4_quantize_op.register_fake
def _mx4_quantize_fake(x, act, col_mul):
    R, K = x.shape
    return (x.new_empty((R, (K + 31) // 32 * 16), dtype=torch.uint8),
            x.new_empty(((K + 255) // 256, R, 8), dtype=torch.uint8))


@torch.library.custom_op("w8a8::kv_write", mutates_args=("cache",))
def kv_write_op(cache: torch.Tensor, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
                fmt: str) -> None:
    kv_write(cache, k, v, slots, fmt=fmt)


@kv_write_op.register_fake
def _kv_write_fake(cache, k, v, slots, fmt):
    torch._check(k.shape == v.shape, lambda: "shape mismatch")


@torch.library.custom_op("w8a8::kv_read", mutates_args=())
def kv_read_op(cache: torch.Tensor, slots: torch.Tensor, head_dim: int,
               fmt: str) -> tuple[torch.Tensor, torch.Tensor]:
    return kv_read(cache, slots, head_dim, fmt=fmt)


@kv_read_op.register_fake
def _kv_read_fake(cache, slots, head_dim, fmt):
    shape = (slots.shape[0], cache.shape[2], head_dim)
    return (cache.new_empty(shape, dtype=torch.bfloat16),
            cache.new_empty(shape, dtype=torch.bfloat16))


@torch.library.custom_op("w8a8::kv_attention", mutates_args=())
def kv_attention_op(q: torch.Tensor, cache: torch.Tensor, block_table: torch.Tensor,
                    kv_lens: torch.Tensor, q_starts: Optional[torch.Tensor], fmt: str,
                    scale: Optional[float], causal: bool, max_q: Optional[int],
                    max_kv: Optional[int]) -> torch.Tensor:
    return kv_attention(q, cache, block_table, kv_lens, fmt=fmt, q_starts=q_starts, scale=scale,
                        causal=causal, max_q=max_q, max_kv=max_kv)


@kv_attention_op.register_fake
def _kv_attention_fake(q, cache, block_table, kv_lens, q_starts, fmt, scale, causal, max_q, max_kv):
    return q.new_empty(q.shape)


@torch.library.custom_op("w8a8::kv_append", mutates_args=("cache",))
def kv_append_op(cache: torch.Tensor, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
                 positions: torch.Tensor, inv_freq: torch.Tensor, q: Optional[torch.Tensor], fmt: str,
                 sections: Optional[list[int]], interleaved: bool) -> torch.Tensor:
    y = kv_append(cache, k, v, slots, positions, inv_freq, q=q, fmt=fmt, sections=sections,
                  interleaved=interleaved)
    return k.new_empty((k.shape[0], 0, k.shape[2])) if y is None else y


@kv_append_op.register_fake
def _kv_append_fake(cache, k, v, slots, positions, inv_freq, q, fmt, sections, interleaved):
    torch._check(k.shape == v.shape, lambda: "shape mismatch")
    return k.new_empty((k.shape[0], 0, k.shape[2])) if q is None else q.new_empty(q.shape)


@torch.library.custom_op("w8a8::kv_tree_attention", mutates_args=())
def kv_tree_attention_op(q: torch.Tensor, cache: torch.Tensor, block_table: torch.Tensor,
                         kv_lens: torch.Tensor, tree: torch.Tensor, q_starts: Optional[torch.Tensor],
                         fmt: str, scale: Optional[float], max_q: Optional[int],
                         max_kv: Optional[int]) -> torch.Tensor:
    return kv_tree_attention(q, cache, block_table, kv_lens, tree, fmt=fmt, q_starts=q_starts,
                             scale=scale, max_q=max_q, max_kv=max_kv)


@kv_tree_attention_op.register_fake
def _kv_tree_attention_fake(q, cache, block_table, kv_lens, tree, q_starts, fmt, scale, max_q, max_kv):
    return q.new_empty(q.shape)


@torch.library.custom_op("w8a8::rms_norm_quantize", mutates_args=())
def rms_norm_quantize_op(x: torch.Tensor, weight: Optional[torch.Tensor],
                         residual: Optional[torch.Tensor], eps: float,
                         fmt: str) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    codes, scales, h = rms_norm_quantize(x, weight, residual=residual, eps=eps, fmt=fmt)
    return codes, scales, x.clone() if residual is None else h     # an op's output is no input of it


@rms_norm_quantize_op.register_fake
def _rms_norm_quantize_fake(x, weight, residual, eps, fmt):
    M, K = x.shape
    if fmt == "int8":
        codes, scales = x.new_empty((M, K), dtype=torch.int8), x.new_empty((M,), dtype=torch.float32)
    else:
        codes = x.new_empty((M, (K + 31) // 32 * 16), dtype=torch.uint8)
        scales = x.new_empty(((K + 255) // 256, M, 8), dtype=torch.uint8)
    return codes, scales, x.new_empty((M, K))


@torch.library.custom_op("w8a8::token_logprobs", mutates_args=())
def token_logprobs_op(logits: torch.Tensor, tokens: torch.Tensor, top: int, temperature: float) -> tuple[
        torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    return token_logprobs(logits, tokens, top=top, temperature=temperature)


@token_logprobs_op.register_fake
def _token_logprobs_fake(logits, tokens, top, temperature):
    T, f = logits.shape[0], torch.float32
    return (logits.new_empty((T,), dtype=f), logits.new_empty((T,), dtype=f),
            logits.new_empty((T, top), dtype=f), logits.new_empty((T, top), dtype=torch.int64))


class MX4Linear(torch.nn.Module):
    """Inference replacement for a bf16 nn.Linear in 4 bits: weights quantized once, here, in
    microscaled blocks along the input channels, activations the same way on every call. smooth
    and act as in W8A8Linear."""

    def __init__(self, wq: torch.Tensor, w_scale: torch.Tensor, in_features: int,
                 bias: Optional[torch.Tensor] = None, *, act: str = "none",
                 smooth_inv: Optional[torch.Tensor] = None):
        super().__init__()
        if (in_features + 31) // 32 * 16 != wq.shape[1]:
            raise ValueError(f"in_features={in_features} does not fit codes {tuple(wq.shape)}")
        self.register_buffer("wq", wq)
        self.register_buffer("w_scale", w_scale)
        self.register_buffer("bias", bias)
        self.register_buffer("smooth_inv", smooth_inv)
        self.act = ACTS[act]
        self.in_features = in_features
        self.out_features = wq.shape[0]

    @classmethod
    def from_linear(cls, lin: torch.nn.Linear, *, act: str = "none",
                    smooth: Optional[torch.Tensor] = None,
                    smooth_inv: Optional[torch.Tensor] = None) -> "MX4Linear":
        if (smooth is None) != (smooth_inv is None):
            raise ValueError("pass both smooth and smooth_inv, or neither")
        w = lin.weight.detach().to(torch.bfloat16).contiguous()
        wq, sw = mx4_quantize(w, col_mul=smooth)
        b = None if lin.bias is None else lin.bias.detach().to(torch.bfloat16).contiguous()
        return cls(wq, sw, lin.in_features, b, act=act, smooth_inv=smooth_inv)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return torch.ops.w8a8.mx4_linear.default(x, self.wq, self.w_scale, self.bias, self.act,
                                                 self.smooth_inv)

    def extra_repr(self) -> str:
        return (f"in_features={self.in_features}, out_features={self.out_features}, "
                f"act={_ACT_NAMES[self.act]}, smoothed={self.smooth_inv is not None}")
