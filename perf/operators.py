"""Measured cases of the microscaled operators: 4-bit quantization, the 4-bit linear, the
quantized key/value cache and the attention that reads it.

A microscaled (MX) block is 32 neighbouring values that share one power-of-two scale, kept as
a byte s (the scale is 2^(s - 127); 255 marks a block with an infinity or a NaN). Its elements
are 4-bit floats (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) or, in a cache, also
8-bit ones (e4m3, up to 448). The scale is 2^(floor(log2(largest magnitude)) - m) with m = 2
for e2m1 and m = 8 for e4m3; elements are rounded to nearest even and saturate.

Layouts (all uint8):
  matrix [R, K]   codes [R, 16 * ceil(K / 32)]: two elements a byte, the earlier one in the low
                  half; scales [ceil(K / 256), R, 8]: the 8 blocks of 256 channels side by side.
                  Channels past K are zero codes, blocks past K zero scales.
  cache           [pages, 2, heads, page bytes], keys then values: for each head of a page the
                  codes of its tokens (head_dim elements each), then their scales
                  (head_dim / 32 bytes each).

A case's "kind":
  quant   mx4_quantize of an activation matrix and mx4_dequantize of what it gives
  linear  mx4_linear of an activation matrix on weights already quantized
  cache   kv_write of new keys and values into a cache, and kv_read of the slots written
  attn    kv_attention of new queries over the pages of their sequences
"""
import math
import random

import torch

own = False

DEV = "cuda"
GRID4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------- cases

def _quant(M, K, act, smooth):
    return dict(kind="quant", M=M, K=K, act=act, smooth=smooth)


def _linear(M, K, N, act="none", smooth=False, bias=True):
    return dict(kind="linear", M=M, K=K, N=N, act=act, smooth=smooth, bias=bias)


def _cache(T, heads, dim, page, fmt, packed):
    return dict(kind="cache", T=T, heads=heads, dim=dim, page=page, fmt=fmt, packed=packed)


def _attn(seqs, q_max, kv_max, heads, group, dim, page, fmt, ragged):
    return dict(kind="attn", seqs=seqs, q_max=q_max, kv_max=kv_max, heads=heads, group=group,
                dim=dim, page=page, fmt=fmt, ragged=ragged)


def listed():
    return [
        # The smallest matrix: a short sequence in front of a small projection.
        dict(name="quant_tiny", **_quant(64, 256, "none", False)),
        # The MLP's down-projection input at 1024px: GELU and SmoothQuant in the quantizer.
        dict(name="quant_mlp", **_quant(4608, 16384, "gelu", True)),
        # One token (a decoding step, a timestep vector) through an MLP up-projection.
        dict(name="linear_one", **_linear(1, 4096, 16384)),
        # Text conditioning, or a batch of decoding sequences, through a square projection.
        dict(name="linear_text", **_linear(77, 4096, 4096)),
        # Odd sizes: ragged tokens, channels that fill no block, no bias.
        dict(name="linear_ragged", **_linear(2001, 1000, 3001, "gelu", False, False)),
        # The MLP up-projection at 1024px, the largest product.
        dict(name="linear_mlp", **_linear(4608, 4096, 16384, "none", True)),
        # A decoding step's keys and values: one token of each of 64 sequences, cut out of
        # the output of a fused qkv projection.
        dict(name="cache_step", **_cache(64, 8, 128, 64, "fp8", True)),
        # Prompts of 20000 tokens in one pass, in 4 bits.
        dict(name="cache_prompt", **_cache(20000, 8, 128, 64, "fp4", False)),
        # One short sequence, one token: latency.
        dict(name="attn_short", **_attn(1, 1, 301, 8, 4, 128, 16, "fp8", False)),
        # A serving batch: 48 sequences of very different lengths, one token each.
        dict(name="attn_batch", **_attn(48, 1, 16384, 8, 4, 128, 64, "fp8", True)),
        # A long document in 4 bits: one sequence of 200000 tokens, one token.
        dict(name="attn_long", **_attn(1, 1, 200001, 8, 8, 128, 128, "fp4", False)),
        # Prompt chunks on a cache that holds their beginnings, at the 18 heads of 256 of the
        # 4608-wide model.
        dict(name="attn_chunk", **_attn(4, 1000, 6000, 18, 1, 256, 64, "fp8", True)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quant", "linear", "linear", "cache", "attn", "attn"])
    while True:
        if kind == "quant":
            M, K = _log(rng, 1, 8192), _log(rng, 64, 24576)
            if M * K <= 4608 * 16384:
                return _quant(M, K, rng.choice(["none", "gelu"]), rng.random() < 0.5)
        elif kind == "linear":
            M, K, N = _log(rng, 1, 8192), _log(rng, 64, 24576), _log(rng, 64, 20480)
            if rng.random() < 0.75:   # as model widths are
                K, N = max(64, K // 64 * 64), max(64, N // 64 * 64)
            if 2.0 * M * K * N <= 6e11:
                return _linear(M, K, N, rng.choice(["none", "none", "gelu"]), rng.random() < 0.5,
                               rng.random() < 0.75)
        elif kind == "cache":
            T, heads = _log(rng, 1, 24000), rng.choice([1, 2, 5, 8, 18])
            dim, page = rng.choice([64, 128, 128, 192, 256]), rng.choice([16, 48, 64, 128])
            if T * heads * dim <= 20000 * 8 * 128:
                return _cache(T, heads, dim, page, rng.choice(["fp8", "fp4"]),
                              rng.random() < 0.5)
        else:
            seqs = _log(rng, 1, 64)
            q_max = 1 if rng.random() < 0.6 else _log(rng, 2, 1000)
            kv_max = q_max + _log(rng, 1, 100000)
            heads, group = rng.choice([1, 2, 5, 8, 18]), rng.choice([1, 3, 4, 8, 16])
            dim, page = rng.choice([64, 128, 128, 192, 256]), rng.choice([16, 48, 64, 128])
            c = _attn(seqs, q_max, kv_max, heads, group, dim, page, rng.choice(["fp8", "fp4"]),
                      rng.random() < 0.7)
            if (seqs * kv_max * heads * dim <= 8e8 and work(c)["flops"] <= 3e11
                    and seqs * q_max * heads * group * kv_max <= 6e8):
                return c


def _lens(case):
    """(queries, keys) of each sequence: whole or, where ragged, spread over the range, with
    one sequence that has nothing yet and one of a single token."""
    n, q, kv = case["seqs"], case["q_max"], case["kv_max"]
    if not case["ragged"]:
        return [q] * n, [kv] * n
    rng = random.Random(n * 1000003 + q * 1009 + kv)
    qs = [q if i == 0 else rng.randint(1, q) for i in range(n)]
    kvs = [kv if i == 0 else max(qs[i], _log(rng, max(1, kv // 64), kv)) for i in range(n)]
    if n >= 3:
        qs[1], kvs[1] = 1, 1
    if n >= 4:
        qs[2], kvs[2] = 1, 0
    return qs, kvs


def _element_bytes(fmt, dim):
    return dim if fmt == "fp8" else dim // 2


def work(case):
    if case["kind"] == "quant":
        M, K = case["M"], case["K"]
        packed = M * (16 * -(-K // 32)) + M * 8 * -(-K // 256)
        return {"bytes": 4 * M * K + 2 * packed + (4 * K if case["smooth"] else 0),
                "flops": 6 * M * K}
    if case["kind"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": 2 * M * K + N * K * 17 // 32 + 2 * M * N + 2 * N * case["bias"]
                + (4 * K if case["smooth"] else 0), "flops": 2 * M * N * K}
    token = 2 * case["heads"] * (_element_bytes(case["fmt"], case["dim"]) + case["dim"] // 32)
    if case["kind"] == "cache":
        values = 2 * case["T"] * case["heads"] * case["dim"]
        return {"bytes": 4 * values + 2 * case["T"] * token + 8 * case["T"], "flops": 6 * values}
    qs, kvs = _lens(case)
    heads = case["heads"] * case["group"]
    pairs = sum(q * max(0, kv - q) + q * (q + 1) // 2 if kv else 0 for q, kv in zip(qs, kvs))
    return {"bytes": sum(kvs) * token + 4 * sum(qs) * heads * case["dim"],
            "flops": 4 * pairs * heads * case["dim"]}


# ---------------------------------------------------------------- the formats, in 32 bits

def _gelu(x):
    return 0.5 * x * torch.erfc(-x * math.sqrt(0.5))


def _power(e):
    """2^e for whole e from -127 to 127, exactly: the exponent field itself (2^-127 is subnormal)."""
    return torch.where(e > -127, e + 127 << 23, 1 << 22).int().view(torch.float32)


def _scaled(x, most):
    """Blocks of 32 of x [..., 32 n] by their shared scale, and the scale bytes [..., n]."""
    b = x.unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1)
    e = torch.frexp(amax).exponent - 1 - most
    e = torch.where(amax > 0, e, -127).clamp(min=-127)
    ok = torch.isfinite(b).all(-1)
    v = torch.where(ok[..., None], b * _power(-e)[..., None], 0.0)
    return v, torch.where(ok, e + 127, 255).to(torch.uint8)


def _encode4(x):
    """(codes [..., n / 2], scale bytes [..., n / 32]) of x [..., n], n a multiple of 32."""
    v, scales = _scaled(x, 2)
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    c = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    c = (c + 8 * (v < 0)).flatten(-2).to(torch.uint8)
    return c[..., 0::2] | c[..., 1::2] << 4, scales


def _encode8(x):
    v, scales = _scaled(x, 8)
    c = v.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    return c.flatten(-2), scales


def _values(codes, scales, fmt):
    """What codes [..., n bytes] and scale bytes [..., blocks] stand for, in 32 bits."""
    if fmt == "fp4":
        grid = torch.tensor(GRID4 + tuple(-g for g in GRID4), device=codes.device)
        v = torch.stack((grid[(codes & 15).int()], grid[(codes >> 4).int()]), -1).flatten(-2)
    else:
        v = codes.view(torch.float8_e4m3fn).float()
    scale = torch.where(scales == 255, torch.nan, _power(scales.int() - 127))
    return (v.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def _encode(x, fmt):
    return _encode4(x) if fmt == "fp4" else _encode8(x)


def _pack_matrix(x):
    """codes and scales of a matrix [R, K] in their layout."""
    R, K = x.shape
    codes, scales = _encode4(torch.nn.functional.pad(x, (0, -K % 32)))
    scales = torch.nn.functional.pad(scales, (0, -scales.shape[1] % 8))
    return codes, scales.unflatten(-1, (-1, 8)).transpose(0, 1).contiguous()


def _unpack_matrix(codes, scales, K):
    scales = scales.transpose(0, 1).flatten(1)[:, :codes.shape[1] // 16]
    return _values(codes, scales, "fp4")[:, :K]


def _cache_views(cache, page, dim, fmt):
    """The codes [pages, 2, heads, page, bytes] and scales [pages, 2, heads, page, dim / 32]
    inside a cache."""
    n = _element_bytes(fmt, dim)
    return (cache[..., :page * n].unflatten(-1, (page, n)),
            cache[..., page * n:].unflatten(-1, (page, dim // 32)))


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _activations(g, M, K):
    """N(0, 1) with two outlier channels, as a transformer's activations have them."""
    x = torch.randn(M, K, generator=g, device=DEV)
    x[:, 17 % K] *= 20.0
    x[:, (3 * K // 4 + 5) % K] *= 20.0
    return x.to(torch.bfloat16)


def _kv(g, T, heads, dim):
    """Keys and values [T, 2, heads, dim]: N(0, 1), channels of the keys of different size."""
    x = torch.randn(T, 2, heads, dim, generator=g, device=DEV)
    x[:, 0] *= torch.exp(0.7 * torch.randn(heads, dim, generator=g, device=DEV))
    return x.to(torch.bfloat16)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["kind"] in ("quant", "linear"):
        M, K = case["M"], case["K"]
        s["x"] = _activations(g, M, K)
        s["col_mul"] = None
        if case["smooth"]:
            s["col_mul"] = torch.exp(0.5 * torch.randn(K, generator=g, device=DEV))
    if case["kind"] == "linear":
        N = case["N"]
        w = 0.02 * torch.randn(N, K, generator=g, device=DEV)
        w *= 0.5 + 1.5 * torch.rand(N, 1, generator=g, device=DEV)
        s["wq"], s["w_scale"] = _pack_matrix(w)
        s["b"] = None
        if case["bias"]:
            s["b"] = (0.01 * torch.randn(N, generator=g, device=DEV)).to(torch.bfloat16)
    if case["kind"] in ("cache", "attn"):
        heads, dim, page, fmt = case["heads"], case["dim"], case["page"], case["fmt"]
        n_page = page * (_element_bytes(fmt, dim) + dim // 32)
    if case["kind"] == "cache":
        T = case["T"]
        kv = _kv(g, T, heads, dim)
        if case["packed"]:   # keys and values lie behind the queries of a fused projection
            qkv = torch.randn(T, 6 * heads, dim, generator=g, device=DEV).to(torch.bfloat16)
            qkv[:, 4 * heads:] = kv.flatten(1, 2)
            s["k"], s["v"] = qkv[:, 4 * heads:5 * heads], qkv[:, 5 * heads:]
        else:
            s["k"], s["v"] = kv[:, 0].contiguous(), kv[:, 1].contiguous()
        # A token has a place of its own in pages taken at random, as an allocator hands them
        # out after a while; steps scatter over all pages, prompts fill theirs. The last few
        # tokens of a call are padding.
        pages = -(-T // page) + 8
        s["cache"] = torch.zeros(pages, 2, heads, n_page, dtype=torch.uint8, device=DEV)
        order = torch.randperm(pages, generator=g, device=DEV)
        if T <= 256:
            slots = torch.randperm(pages * page, generator=g, device=DEV)[:T]
        else:
            t = torch.arange(T, device=DEV)
            slots = order[t // page] * page + t % page
        if T >= 16:
            slots[-3:] = -1
        s["slots"] = slots.to(torch.int64)
    if case["kind"] == "attn":
        qs, kvs = _lens(case)
        per = -(-max(kvs) // page)
        need = [-(-n // page) for n in kvs]
        pages = sum(need) + 8
        s["cache"] = torch.zeros(pages, 2, heads, n_page, dtype=torch.uint8, device=DEV)
        codes, scales = _cache_views(s["cache"], page, dim, fmt)
        for lo in range(0, pages, 256):
            hi = min(pages, lo + 256)
            kv = _kv(g, (hi - lo) * page, heads, dim).unflatten(0, (hi - lo, page)).float()
            codes[lo:hi], scales[lo:hi] = _encode(kv.permute(0, 2, 3, 1, 4), fmt)
        order = torch.randperm(pages, generator=g, device=DEV).int()
        table = torch.zeros(len(kvs), per, dtype=torch.int32)
        flat = order.cpu()
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = flat[at:at + n]
            at += n
        starts = [0]
        for n in qs:
            starts.append(starts[-1] + n)
        s["table"] = table.to(DEV)
        s["kv_lens"] = torch.tensor(kvs, dtype=torch.int32, device=DEV)
        s["q_starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
        s["q"] = torch.randn(starts[-1], heads * case["group"], dim, generator=g,
                             device=DEV).to(torch.bfloat16)
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2606_14598_amd as w8a8
    if s["kind"] == "quant":
        q, scales = w8a8.mx4_quantize(s["x"], act=s["act"], col_mul=s["col_mul"])
        return w8a8.mx4_dequantize(q, scales, s["K"])
    if s["kind"] == "linear":
        return w8a8.mx4_linear(s["x"], s["wq"], s["w_scale"], s["b"], act=s["act"],
                               col_mul=s["col_mul"])
    if s["kind"] == "cache":
        w8a8.kv_write(s["cache"], s["k"], s["v"], s["slots"], fmt=s["fmt"])
        return w8a8.kv_read(s["cache"], s["slots"], s["dim"], fmt=s["fmt"])
    return w8a8.kv_attention(s["q"], s["cache"], s["table"], s["kv_lens"], fmt=s["fmt"],
                             q_starts=s["q_starts"], max_q=s["q_max"], max_kv=s["kv_max"])


def _transformed(s):
    x = s["x"].float()
    if s["act"] == "gelu":
        x = _gelu(x)
    return x if s["col_mul"] is None else x * s["col_mul"]


def _run_plain(s):
    if s["kind"] == "quant":
        return _unpack_matrix(*_pack_matrix(_transformed(s)), s["K"]).to(torch.bfloat16)
    if s["kind"] == "linear":
        K = s["K"]
        x = _unpack_matrix(*_pack_matrix(_transformed(s)), K)
        y = x @ _unpack_matrix(s["wq"], s["w_scale"], K).t()
        return (y if s["b"] is None else y + s["b"].float()).to(torch.bfloat16)
    if s["kind"] == "cache":
        codes, scales = _cache_views(s["cache"], s["page"], s["dim"], s["fmt"])
        live = s["slots"] >= 0
        page, at = s["slots"] // s["page"], s["slots"] % s["page"]
        c, e = _encode(torch.stack((s["k"], s["v"]), 1).float(), s["fmt"])
        codes[page[live], :, :, at[live]] = c[live]
        scales[page[live], :, :, at[live]] = e[live]
        kv = _values(codes[page, :, :, at], scales[page, :, :, at], s["fmt"])
        kv = torch.where(live[:, None, None, None], kv, 0.0).to(torch.bfloat16)
        return kv[:, 0], kv[:, 1]
    return _attend_plain(s)


def _attend_plain(s):
    """Attention of every sequence at once, padded to the longest."""
    heads, group, dim, page = s["heads"], s["group"], s["dim"], s["page"]
    q_len = s["q_starts"][1:] - s["q_starts"][:-1]
    codes, scales = _cache_views(s["cache"], page, dim, s["fmt"])
    kv = _values(codes[s["table"]], scales[s["table"]], s["fmt"])   # [B, P, 2, H, page, D]
    kv = kv.permute(2, 0, 3, 1, 4, 5).flatten(3, 4)                 # [2, B, H, P * page, D]
    j = torch.arange(kv.shape[3], device=DEV)
    held = (j < s["kv_lens"][:, None])[:, None, :, None]
    k, v = torch.where(held, kv[0], 0.0), torch.where(held, kv[1], 0.0)
    i = torch.arange(s["q_max"], device=DEV)
    rows = (s["q_starts"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[rows].unflatten(2, (heads, group))           # [B, L, H, G, D]
    q = q.permute(0, 2, 3, 1, 4)
    last = (s["kv_lens"] - q_len)[:, None] + i
    seen = (j <= last[:, :, None]) & (j < s["kv_lens"][:, None, None])
    seen = seen[:, None, None]                                      # [B, 1, 1, L, keys]
    p = (q.flatten(2, 3) @ k.transpose(2, 3)).unflatten(2, (group, -1)) * dim ** -0.5
    p = torch.where(seen, p, -torch.inf)
    top = p.amax(-1, keepdim=True)
    p = torch.exp(p - torch.where(top == -torch.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    y = (p.flatten(2, 3) @ v).unflatten(2, (group, -1))
    y = torch.where(total > 0, y / total, 0.0)                      # [B, H, G, L, D]
    y = y.permute(0, 3, 1, 2, 4).flatten(2, 3)
    return y[i < q_len[:, None]].to(torch.bfloat16)


# ---------------------------------------------------------------- the definition, in 64 bits

def _double_power(e):
    """2^e as a double, from its bits: a library's pow may be a rounding off."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(x, fmt):
    """What a row of blocks stands for once quantized, element by element from the formats'
    grids: the nearest representable magnitude, the one with the even code where two are."""
    if fmt == "fp4":
        grid, most = list(GRID4), 2
    else:
        grid = [m * 2.0 ** -9 for m in range(8)]
        grid += [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:119]
        most = 8
    grid = torch.tensor(grid, dtype=torch.float64, device=x.device)
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    big = b.abs().max(-1, keepdim=True).values
    # floor(log2) exactly: the exponent field of the double itself
    e = (big.view(torch.int64) >> 52) - 1023
    scale = _double_power((e - most).clamp(min=-127, max=128))
    a = b.abs() / scale
    mid = (grid[1:] + grid[:-1]) / 2
    below = torch.searchsorted(mid, a.contiguous(), right=False)   # a tie goes down ...
    above = torch.searchsorted(mid, a.contiguous(), right=True)    # ... or up
    code = torch.where(below % 2 == 0, below, above)
    v = grid[code] * scale * torch.sign(b)
    v = torch.where(torch.isfinite(big), v, torch.nan)
    return v.reshape(x.shape)


def _exact_matrix(x):
    K = x.shape[1]
    full = torch.zeros(x.shape[0], (K + 31) // 32 * 32, dtype=torch.float64, device=x.device)
    full[:, :K] = x
    return _exact_values(full, "fp4")[:, :K]


def _exact_decode(codes, scales, fmt):
    if fmt == "fp4":
        both = torch.empty(*codes.shape, 2, dtype=torch.float64, device=codes.device)
        for at, c in ((0, codes % 16), (1, codes // 16)):
            m, e = (c % 2).double(), (c // 2) % 4
            mag = torch.where(e == 0, m / 2, (1 + m / 2) * _double_power(e.long() - 1))
            both[..., at] = torch.where(c >= 8, -mag, mag)
        v = both.reshape(*codes.shape[:-1], -1)
    else:
        c = codes.long()
        m, e = (c % 8).double(), (c // 8) % 16
        v = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * _double_power(e - 7))
        v = torch.where(c >= 128, -v, v)
    scale = _double_power(scales.long() - 127)
    return v * scale.repeat_interleave(32, -1)


def _exact_input(s):
    x = s["x"].double()
    if s["act"] == "gelu":
        x = x * torch.special.ndtr(x)
    if s["col_mul"] is not None:
        x = x * s["col_mul"].double()
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quant":
        return _exact_matrix(_exact_input(s))
    if case["kind"] == "linear":
        K, N = case["K"], case["N"]
        x = _exact_matrix(_exact_input(s))
        nb = s["wq"].shape[1] // 16
        sc = torch.cat([s["w_scale"][p] for p in range(s["w_scale"].shape[0])], 1)[:, :nb]
        w = _exact_decode(s["wq"], sc, "fp4")[:, :K]
        y = torch.mm(x, w.t())
        return y + s["b"].double() if s["b"] is not None else y
    if case["kind"] == "cache":
        gone = (s["slots"] < 0)[:, None, None]
        k, v = (_exact_values(t.double().contiguous(), s["fmt"]) for t in (s["k"], s["v"]))
        return k.masked_fill(gone, 0.0), v.masked_fill(gone, 0.0)
    qs, kvs = _lens(case)
    heads, group, dim, page, fmt = (case[n] for n in ("heads", "group", "dim", "page", "fmt"))
    nb = _element_bytes(fmt, dim)
    out = torch.zeros(sum(qs), heads * group, dim, dtype=torch.float64, device=DEV)
    at = 0
    for n, (lq, lk) in enumerate(zip(qs, kvs)):
        used = s["table"][n, :-(-lk // page)].long()
        for h in range(heads if lk else 0):
            raw = s["cache"][used][:, :, h]                        # [pages, 2, page bytes]
            c = raw[:, :, :page * nb].reshape(-1, 2, page, nb)
            e = raw[:, :, page * nb:].reshape(-1, 2, page, dim // 32)
            kv = _exact_decode(c, e, fmt).transpose(0, 1).reshape(2, -1, dim)[:, :lk]
            for r in range(group):
                q = s["q"][at:at + lq, h * group + r].double()
                z = q @ kv[0].t() / math.sqrt(dim)
                hidden = torch.ones(lq, lk, dtype=torch.bool, device=DEV).triu(lk - lq + 1)
                z = z.masked_fill(hidden, -math.inf)
                out[at:at + lq, h * group + r] = torch.softmax(z, -1) @ kv[1]
        at += lq
    return out
