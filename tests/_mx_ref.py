"""Plain 64-bit forms of the microscaled operators, from their definitions, on the CPU."""
import numpy as np
import torch

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
E4M3 = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10)
                                            for e in range(1, 16) for m in range(8)][:119]
GRIDS = {"fp4": (np.array(E2M1), 2), "fp8": (np.array(E4M3), 8)}


def f64(t):
    return t.detach().cpu().double().numpy()


def quantize_blocks(v, fmt):
    """(codes, scale bytes) of v [..., n] float64, n a multiple of 32: one code a value, the
    sign above the magnitude's bits."""
    grid, top = GRIDS[fmt]
    b = v.reshape(*v.shape[:-1], -1, 32)
    fin = np.isfinite(b).all(-1)
    a = np.abs(np.where(fin[..., None], b, 0.0))
    amax = a.max(-1)
    e = np.frexp(amax)[1] - 1 - top          # frexp: amax = m 2^(e + 1 + top), 0.5 <= m < 1
    s = np.where(amax > 0, np.maximum(e, -127), -127)
    x = np.ldexp(a, -s[..., None])
    mid = (grid[1:] + grid[:-1]) / 2
    lo, hi = np.searchsorted(mid, x, "left"), np.searchsorted(mid, x, "right")
    code = np.where(lo % 2 == 0, lo, hi)     # they differ on a tie: the even one
    sign = np.signbit(b) & fin[..., None]
    code = code + sign * len(grid if fmt == "fp4" else np.zeros(128))
    return code.reshape(v.shape).astype(np.uint8), np.where(fin, s + 127, 255).astype(np.uint8)


def block_values(codes, scales, fmt):
    """float64 values of one code per value and the blocks' scale bytes."""
    grid, _ = GRIDS[fmt]
    n = 8 if fmt == "fp4" else 128
    full = np.full(n, np.nan)
    full[:len(grid)] = grid
    v = full[codes % n] * np.where(codes >= n, -1.0, 1.0)
    s = scales.astype(np.int64) - 127
    v = np.ldexp(v.reshape(*scales.shape, 32), s[..., None])
    return np.where(scales[..., None] == 255, np.nan, v).reshape(codes.shape)


def pack4(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def unpack4(b):
    return np.stack((b & 15, b >> 4), -1).reshape(*b.shape[:-1], -1)


def pack_matrix(v):
    """(codes, scales) of a float64 matrix [R, K] in the library's layout."""
    R, K = v.shape
    nb = -(-K // 32)
    full = np.zeros((R, nb * 32))
    full[:, :K] = v
    codes, s = quantize_blocks(full, "fp4")
    out = np.zeros((-(-nb // 8), R, 8), np.uint8)
    for b in range(nb):
        out[b // 8, :, b % 8] = s[:, b]
    return pack4(codes), out


def matrix_values(codes, scales, K):
    nb = codes.shape[1] // 16
    s = np.stack([scales[b // 8, :, b % 8] for b in range(nb)], 1) if nb else \
        np.zeros((codes.shape[0], 0), np.uint8)
    return block_values(unpack4(codes), s, "fp4")[:, :K]


def code_bytes(dim, fmt):
    return dim if fmt == "fp8" else dim // 2


def cache_slot(cache, slot, page, dim, fmt):
    """(code bytes, scale bytes) views [2, heads, ...] of a slot in a numpy cache."""
    n = code_bytes(dim, fmt)
    p, o = divmod(slot, page)
    base = page * n
    return (cache[p, :, :, o * n:(o + 1) * n],
            cache[p, :, :, base + o * (dim // 32):base + (o + 1) * (dim // 32)])


def slot_values(cache, slot, page, dim, fmt):
    c, s = cache_slot(cache, slot, page, dim, fmt)
    return block_values(unpack4(c) if fmt == "fp4" else c, s, fmt)


def attention(q, k, v, scale, causal):
    """(out, weighted mean of |v|) [lq, dim] of one head: q [lq, dim], k, v [kv, dim]."""
    lq, kv = q.shape[0], k.shape[0]
    out, mag = np.zeros((lq, v.shape[1])), np.zeros((lq, v.shape[1]))
    for i in range(lq):
        n = min(kv, kv - lq + i + 1) if causal else kv
        if n <= 0:
            continue
        z = (k[:n] @ q[i]) * scale
        p = np.exp(z - z.max())
        p /= p.sum()
        out[i], mag[i] = p @ v[:n], p @ np.abs(v[:n])
    return out, mag
