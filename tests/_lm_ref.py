"""Plain 64-bit forms of the norm, rotary positions, tree attention and log probabilities, from
their definitions, on the CPU. What the operators round to 32 bits on the way is rounded here too."""
import numpy as np


def f32_inverse_rms(h, eps):
    """float32(1 / sqrt(mean h^2 + eps)) of rows h float64, and whether it hangs on the last bits
    of a 64-bit sum: the kernel's sum of K squares is 2^-52 K off at most, its square root, division
    and mean 2^-51 together."""
    K = h.shape[1]
    exact = 1.0 / np.sqrt((h.astype(np.longdouble) ** 2).sum(1) / K + np.longdouble(eps))
    r = exact.astype(np.float32)
    slack = np.longdouble((K + 8) * 2.0 ** -52)
    near = ((exact * (1 - slack)).astype(np.float32) != r) | ((exact * (1 + slack)).astype(np.float32) != r)
    return r, near


def norm_values(h, r, weight):
    v = h.astype(np.float32) * r[:, None]
    return v if weight is None else v * weight.astype(np.float32)


def int8_rows(v):
    """The int8 rule on float32 rows: (codes, scales)."""
    a = np.abs(v).max(1) if v.shape[1] else np.zeros(v.shape[0], np.float32)
    with np.errstate(divide="ignore", over="ignore"):
        inv = np.float32(127.0) / a
    zero = ~(a > 0) | ~np.isfinite(inv)
    inv, s = np.where(zero, np.float32(0), inv), np.where(zero, np.float32(0), a / np.float32(127.0))
    return np.clip(np.rint(v * inv[:, None]), -127, 127).astype(np.int8), s.astype(np.float32)


def cos_sin(positions, inv_freq, sections):
    """float32 cosines and sines [T, pairs], and the tokens where one of them hangs on the last bits
    of a 64-bit value: the kernel's are 2^-45 of the value off at most by the polynomials, and 2^-50 by
    the rounding of the reduced angle (of at most 2 quarter turns, 2^-52, times pi / 2) and of this
    reference; not at all at no angle."""
    p = positions.reshape(positions.shape[0], -1).astype(np.float64)
    axis = np.zeros(len(inv_freq), int) if sections is None else np.repeat(np.arange(len(sections)), sections)
    angle = p[:, axis] * inv_freq.astype(np.float64)
    out, near = [], np.zeros(p.shape[0], bool)
    for f in (np.cos(angle), np.sin(angle)):
        r = f.astype(np.float32)
        d = np.where(angle == 0, 0.0, 2.0 ** -45 * np.abs(f) + 2.0 ** -50)
        near |= (((f - d).astype(np.float32) != r) | ((f + d).astype(np.float32) != r)).any(1) \
            if f.size else near
        out.append(r)
    return (*out, near)


def rotate(x, cos, sin, interleaved):
    """float32 x [T, heads, dim] turned, every operation rounded."""
    n = cos.shape[1]
    y = x.astype(np.float32).copy()
    a, b = ((slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n)))
    c, s = cos[:, None], sin[:, None]
    u, v = y[..., a].copy(), y[..., b].copy()
    y[..., a] = u * c - v * s
    y[..., b] = v * c + u * s
    return y


def tree_bits(parents, words):
    """int64 [n, words] masks of a tree: node i sees itself and its ancestors (-1: none)."""
    seen = []
    for i, p in enumerate(parents):
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
    return bit_words(seen, words)


def bit_words(masks, words):
    out = np.zeros((len(masks), words), np.uint64)
    for i, m in enumerate(masks):
        for w in range(words):
            out[i, w] = (m >> 64 * w) & (1 << 64) - 1
    return out.view(np.int64)


def tree_visible(bits, lq, kv):
    """[lq, kv]: which cached tokens the nodes see; bits [lq, words]."""
    see = np.zeros((lq, kv), bool)
    for j in range(kv):
        n = j - (kv - lq)
        if n < 0:
            see[:, j] = True
        elif n < 64 * bits.shape[1]:
            see[:, j] = bits[:, n // 64].astype(np.uint64) >> np.uint64(n % 64) & np.uint64(1) != 0
    return see


def masked_attention(q, k, v, scale, see):
    """(out, weighted mean of |v|) of one head; zeros for rows that see nothing."""
    out, mag = np.zeros((q.shape[0], v.shape[1])), np.zeros((q.shape[0], v.shape[1]))
    for i in range(q.shape[0]):
        n = see[i]
        if not n.any():
            continue
        z = (k[n] @ q[i]) * scale
        p = np.exp(z - z.max())
        p /= p.sum()
        out[i], mag[i] = p @ v[n], p @ np.abs(v[n])
    return out, mag


def logprobs(x, tokens, top, temperature):
    """(logp, entropy, top_logp, top_ids) of float64 logits [T, V]."""
    T, V = x.shape
    y = x / temperature
    with np.errstate(invalid="ignore", over="ignore"):
        y = y - y.max(1, keepdims=True)
        e = np.exp(y)
        lse = np.log(e.sum(1, keepdims=True))
        p = e / e.sum(1, keepdims=True)
        lp = y - lse
        entropy = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), np.where(np.isnan(p), np.nan, 0.0)).sum(1)
    order = np.argsort(-x, axis=1, kind="stable")[:, :top]
    live = (tokens >= 0) & (tokens < V)
    mine = np.where(live, lp[np.arange(T), np.where(live, tokens, 0)], 0.0)
    return mine, entropy, np.take_along_axis(lp, order, 1), order
