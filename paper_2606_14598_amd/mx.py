"""Microscaled (MX) operators: 4-bit linears, a quantized key/value cache and the attention
over it. Python binding of the w8a8_mx4_* and w8a8_kv_* entry points (include/w8a8.h has the
formats and rules); imported by the package, whose conventions hold here too.

  mx4_quantize(x)                          -> (codes uint8 [R, 16 ceil(K/32)],
                                               scales uint8 [ceil(K/256), R, 8])
  mx4_dequantize(codes, scales, K)         -> bf16 [R, K]
  mx4_gemm(xq, x_scale, wq, w_scale, b)    -> y bf16 [M, N]
  mx4_linear(x, wq, w_scale, b)            -> y bf16 [..., N]   (x [..., K])
  kv_cache(pages, heads, head_dim)         -> cache uint8 [pages, 2, heads, head bytes]
  kv_write(cache, k, v, slots)                quantizes k, v [T, heads, head_dim] into slots
  kv_read(cache, slots, head_dim)          -> k, v bf16 [T, heads, head_dim]
  kv_attention(q, cache, block_table, kv_lens) -> bf16 [T, q heads, head_dim]
"""
from __future__ import annotations

import functools

import torch

from . import (_act, _check, _check_out, _col_mul, _launch, _ptr, _same_device, _size, _workspace)

# Sizes of workspaces and caches, pure functions of a call's sizes, by the sizes asked last: a
# call's host time is what a small one costs.
_bytes = functools.lru_cache(maxsize=4096)(_size)

__all__ = ["mx4_quantize", "mx4_dequantize", "mx4_gemm", "mx4_linear", "kv_cache", "kv_write",
           "kv_read", "kv_attention", "KV_FORMATS", "MX4_MAX_K"]

MX4_MAX_K = 1 << 22
KV_FORMATS = {"fp8": 0, "fp4": 1}


def _mx4_shapes(R: int, K: int):
    return (R, 16 * (-(-K // 32))), (-(-K // 256), R, 8)


def _check_mx4(codes, scales, name: str):
    """(rows, blocks of 32 channels) of a 4-bit matrix."""
    _check(codes, torch.uint8, 2, name)
    _check(scales, torch.uint8, 3, f"{name}'s scales")
    R, n = codes.shape
    if n % 16 != 0 or tuple(scales.shape) != (-(-n // 128), R, 8):
        raise ValueError(f"{name}: codes {tuple(codes.shape)} and scales {tuple(scales.shape)} are "
                         "no 4-bit matrix")
    _same_device(codes, scales)
    return R, n // 16


def mx4_quantize(x: torch.Tensor, *, act: str = "none", col_mul=None):
    """4-bit microscaled matrix of T(x) * col_mul: x bf16 [R, K], activations or weights
    (T = identity or GELU; col_mul fp32 [K] or None)."""
    a = _act(act)
    _check(x, torch.bfloat16, 2, "x")
    R, K = x.shape
    cm = _col_mul(col_mul, K, x.device)
    qs, ss = _mx4_shapes(R, K)
    q = torch.empty(qs, dtype=torch.uint8, device=x.device)
    s = torch.empty(ss, dtype=torch.uint8, device=x.device)
    _launch(x.device, "w8a8_mx4_quantize", _ptr(x), R, K, a, _ptr(cm), _ptr(q), _ptr(s))
    return q, s


def mx4_dequantize(codes, scales, K: int | None = None, *, out=None):
    """The bf16 [R, K] values of a 4-bit matrix (K: all channels of its blocks by default)."""
    R, nb = _check_mx4(codes, scales, "codes")
    K = 32 * nb if K is None else int(K)
    if K < 0 or -(-K // 32) != nb:
        raise ValueError(f"K={K} does not fit {nb} blocks of 32")
    if out is not None:
        _check_out(out, torch.bfloat16, (R, K), codes.device)
    y = out if out is not None else torch.empty((R, K), dtype=torch.bfloat16, device=codes.device)
    _launch(codes.device, "w8a8_mx4_dequantize", _ptr(codes), _ptr(scales), R, K, _ptr(y))
    return y


def _bias(bias, N: int):
    if bias is not None:
        _check(bias, torch.bfloat16, 1, "bias")
        if bias.shape[0] != N:
            raise ValueError("shape mismatch")


def mx4_gemm(xq, x_scale, wq, w_scale, bias=None, *, out=None, workspace=None):
    """bf16(xv @ wv^T + b) of two 4-bit matrices xv [M, K], wv [N, K], accumulated in fp32."""
    M, nb = _check_mx4(xq, x_scale, "xq")
    N, nw = _check_mx4(wq, w_scale, "wq")
    _bias(bias, N)
    _same_device(xq, wq, bias)
    if nb != nw:
        raise ValueError("shape mismatch")
    if out is not None:
        _check_out(out, torch.bfloat16, (M, N), xq.device)
    y = out if out is not None else torch.empty((M, N), dtype=torch.bfloat16, device=xq.device)
    ws = _workspace(_bytes("w8a8_mx4_gemm_workspace_bytes", M, N, 32 * nb), xq.device, workspace)
    _launch(xq.device, "w8a8_mx4_gemm", _ptr(xq), _ptr(x_scale), _ptr(wq), _ptr(w_scale),
            _ptr(bias), _ptr(y), M, N, 32 * nb, _ptr(ws), 0 if ws is None else ws.nbytes)
    return y


def mx4_linear(x, wq, w_scale, bias=None, *, act: str = "none", col_mul=None, out=None,
               workspace=None):
    """The whole 4-bit linear: x bf16 [..., K] -> y bf16 [..., N], T(x) * col_mul quantized on
    the way, w quantized by mx4_quantize."""
    a = _act(act)
    if not isinstance(x, torch.Tensor) or x.dtype != torch.bfloat16:
        raise TypeError("x must be a bf16 torch.Tensor")
    lead = x.shape[:-1]
    K = x.shape[-1]
    x2 = x if x.dim() == 2 else x.reshape(lead.numel(), K)
    _check(x2, torch.bfloat16, 2, "x")
    N, nb = _check_mx4(wq, w_scale, "wq")
    _bias(bias, N)
    _same_device(x2, wq, bias)
    M = x2.shape[0]
    if -(-K // 32) != nb:
        raise ValueError("shape mismatch")
    cm = _col_mul(col_mul, K, x.device)
    if out is not None:
        _check_out(out, torch.bfloat16, (M, N), x.device)
    y = out if out is not None else torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    ws = _workspace(_bytes("w8a8_mx4_linear_workspace_bytes", M, N, K), x.device, workspace)
    _launch(x.device, "w8a8_mx4_linear", _ptr(x2), a, _ptr(cm), _ptr(wq), _ptr(w_scale),
            _ptr(bias), _ptr(y), M, N, K, _ptr(ws), 0 if ws is None else ws.nbytes)
    return y if x.dim() == 2 else y.reshape(*lead, N)


# ---------------------------------------------------------------- cache

def _format(fmt: str) -> int:
    if fmt not in KV_FORMATS:
        raise ValueError(f"fmt must be one of {sorted(KV_FORMATS)}, got {fmt!r}")
    return KV_FORMATS[fmt]


def kv_cache(pages: int, heads: int, head_dim: int, page_size: int = 64, *, fmt: str = "fp8",
             device="cuda") -> torch.Tensor:
    """An empty (zeroed) cache of `pages` pages of page_size tokens: uint8 [pages, 2, heads,
    bytes of a head's page], the layout of include/w8a8.h."""
    n = _size("w8a8_kv_page_bytes", page_size, heads, head_dim, _format(fmt))
    if n < 0 or pages < 0:
        raise ValueError(f"no cache of {pages} pages of {page_size} tokens, {heads} heads of "
                         f"{head_dim}: page_size is a multiple of 16 up to 4096, head_dim 64, 128, "
                         "192 or 256")
    return torch.zeros((pages, 2, heads, n // (2 * heads)), dtype=torch.uint8, device=device)


@functools.lru_cache(maxsize=1024)
def _cache_shape(shape, head_dim: int, fmt: str):
    """(pages, page size, heads, head_dim, format): the C ABI's description of a cache."""
    f = _format(fmt)
    pages, two, heads, n = shape
    token = (head_dim if f == 0 else head_dim // 2) + head_dim // 32
    page = n // token if token else 0
    if two != 2 or heads < 1 or page * token != n or _size("w8a8_kv_page_bytes", page, heads,
                                                           head_dim, f) != 2 * heads * n:
        raise ValueError(f"cache {tuple(shape)} is no {fmt} cache of heads of {head_dim}")
    return pages, page, heads, head_dim, f


def _check_cache(cache, head_dim: int, fmt: str):
    _check(cache, torch.uint8, 4, "cache")
    return _cache_shape(cache.shape, head_dim, fmt)


def _check_slots(slots, T, device):
    _check(slots, torch.int64, 1, "slots")
    if T is not None and slots.shape[0] != T:
        raise ValueError(f"slots must have {T} entries, got {slots.shape[0]}")
    if slots.device != device:
        raise ValueError(f"slots is on {slots.device}, expected {device}")


def _check_heads(t, name: str, device):
    """A bf16 [T, heads, head_dim] tensor whose last dimension is contiguous."""
    if not isinstance(t, torch.Tensor) or t.dtype != torch.bfloat16:
        raise TypeError(f"{name} must be a bf16 torch.Tensor")
    if t.dim() != 3:
        raise ValueError(f"{name} must be 3-D, got shape {tuple(t.shape)}")
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")


def kv_write(cache, k, v, slots, *, fmt: str = "fp8") -> None:
    """Quantizes keys and values k, v bf16 [T, heads, head_dim] (any strides of token and head)
    into the slots int64 [T] of the cache: slot = page * page_size + offset, negative for
    padding."""
    device = cache.device
    _check_heads(k, "k", device)
    _check_heads(v, "v", device)
    shape = _check_cache(cache, k.shape[2], fmt)
    if k.shape != v.shape or k.shape[1] != shape[2]:
        raise ValueError("shape mismatch")
    T = k.shape[0]
    _check_slots(slots, T, device)
    _launch(device, "w8a8_kv_write", _ptr(cache), *shape, _ptr(k), k.stride(0), k.stride(1),
            _ptr(v), v.stride(0), v.stride(1), _ptr(slots), T)


def kv_read(cache, slots, head_dim: int, *, fmt: str = "fp8"):
    """What the slots int64 [T] of a cache hold: k, v bf16 [T, heads, head_dim], zeros for
    negative slots."""
    shape = _check_cache(cache, head_dim, fmt)
    _check_slots(slots, None, cache.device)
    T = slots.shape[0]
    k = torch.empty((T, shape[2], head_dim), dtype=torch.bfloat16, device=cache.device)
    v = torch.empty_like(k)
    _launch(cache.device, "w8a8_kv_read", _ptr(cache), *shape, _ptr(slots), T, _ptr(k), _ptr(v))
    return k, v


def kv_attention(q, cache, block_table, kv_lens, *, fmt: str = "fp8", q_starts=None,
                 scale: float | None = None, causal: bool = True, max_q: int | None = None,
                 max_kv: int | None = None, out=None, workspace=None):
    """Attention of q bf16 [T, q heads, head_dim] over a cache.

    block_table int32 [B, pages]: the pages of each sequence; kv_lens int32 [B]: its cached
    tokens, those of its queries included. q_starts int32 [B + 1]: the first query of each
    sequence and T (None: T / B each, e.g. one in a decoding step). Query i of a sequence's lq
    sees the tokens j <= kv_len - lq + i (causal) or all kv_len; a query that sees none gives
    zeros. Query head h reads head h // (q heads / heads) of the cache. scale: of the scores,
    1 / sqrt(head_dim) by default. max_q, max_kv: bounds on a sequence's queries and tokens for
    laying out the launch, known to the caller on the host (by default T, or T / B without
    q_starts, and the table's width); the results do not depend on them beyond the rounding of
    the weights, and that not in sequences of up to 64 rows (queries x query heads that share
    a head of the cache), which always keep two bf16 terms. Tight bounds are faster: 64 prompts of
    1000 tokens take 0.8 ms with max_q and 1.0 without; one sequence of 2000 tokens, one query,
    16 us with max_kv and 24 by a table of 131072 tokens (8 heads of 128, 4 queries a head)."""
    device = cache.device
    _check_heads(q, "q", device)
    T, q_heads, dim = q.shape
    pages, page, heads, _, f = _check_cache(cache, dim, fmt)
    _check(kv_lens, torch.int32, 1, "kv_lens")
    B = kv_lens.shape[0]
    if not isinstance(block_table, torch.Tensor) or block_table.dtype != torch.int32:
        raise TypeError("block_table must be an int32 torch.Tensor")
    if block_table.dim() != 2 or block_table.shape[0] != B or (
            block_table.shape[1] > 1 and block_table.stride(1) != 1):
        raise ValueError(f"block_table must be [{B}, pages] with contiguous rows")
    if q_starts is not None:
        _check(q_starts, torch.int32, 1, "q_starts")
        if q_starts.shape[0] != B + 1:
            raise ValueError(f"q_starts must have {B + 1} entries, got {q_starts.shape[0]}")
    elif T != 0 and (B == 0 or T % B != 0):
        raise ValueError(f"{T} queries do not divide among {B} sequences")
    _same_device(cache, kv_lens, block_table, q_starts)
    if q_heads == 0 or q_heads % heads != 0:
        raise ValueError(f"{q_heads} query heads do not divide among {heads}")
    if max_q is None:
        max_q = T if q_starts is not None else T // max(B, 1)
    max_q = min(int(max_q), T)
    width = block_table.shape[1]
    max_kv = width * page if max_kv is None else min(int(max_kv), width * page)
    if out is not None:
        _check_out(out, torch.bfloat16, (T, q_heads, dim), device)
    y = out if out is not None else torch.empty((T, q_heads, dim), dtype=torch.bfloat16,
                                                device=device)
    if T == 0:
        return y
    group = q_heads // heads
    nws = _bytes("w8a8_kv_attention_workspace_bytes", page, heads, dim, f, group, T, B,
                max_q, max_kv)
    ws = _workspace(nws, device, workspace)
    _launch(device, "w8a8_kv_attention", _ptr(q), q.stride(0), q.stride(1), _ptr(cache), pages,
            page, heads, dim, f, _ptr(block_table), block_table.stride(0), width, _ptr(kv_lens),
            _ptr(q_starts), T, B, group, dim ** -0.5 if scale is None else float(scale),
            int(bool(causal)), max_q, max_kv, _ptr(y), _ptr(ws),
            0 if ws is None else ws.nbytes)
    return y
