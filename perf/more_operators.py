"""Measured cases of a decoding step's operators: the norm in front of a quantized linear, keys
appended to a cache with their rotary positions, attention of drafted token trees over it, and
the log probabilities that accept or refuse the drafts.

Formats are those of the framework:
  int8   a row's codes q = clamp(rne(v 127 / a), -127, 127) with a = max |v|, scale a / 127
  mx     blocks of 32 values with one power-of-two scale byte s (2^(s - 127); 255: a block of NaN),
         2^(floor(log2(largest magnitude)) - m), elements rounded to nearest even and saturated: 4-bit
         floats (e2m1, m = 2: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) or 8-bit ones (e4m3,
         m = 8, up to 448)
  4-bit matrix [R, K]   codes [R, 16 ceil(K / 32)], two a byte, the earlier in the low half; scales
                        [ceil(K / 256), R, 8]
  cache                 uint8 [pages, 2, heads, page bytes], keys then values: for each head of a page
                        the codes of its tokens, then their scales

A case's "kind":
  norm    rms_norm_quantize of hidden states (and the residual's addition); what its codes stand for
  append  kv_append of new tokens into a cache, and kv_read of the slots written
  tree    kv_tree_attention of drafted trees over the pages of their sequences
  logp    token_logprobs of rows of logits
"""
import math
import random

import torch

own = False

DEV = "cuda"
GRID4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


# ---------------------------------------------------------------- cases

def _norm(M, K, fmt, residual):
    return dict(kind="norm", M=M, K=K, fmt=fmt, residual=residual)


def _append(T, heads, group, dim, rotary, page, fmt, axes, interleaved, far):
    return dict(kind="append", T=T, heads=heads, group=group, dim=dim, rotary=rotary, page=page,
                fmt=fmt, axes=axes, interleaved=interleaved, far=far)


def _tree(seqs, nodes, kv_max, heads, group, dim, page, fmt, ragged):
    return dict(kind="tree", seqs=seqs, nodes=nodes, kv_max=kv_max, heads=heads, group=group,
                dim=dim, page=page, fmt=fmt, ragged=ragged)


def _logp(T, V, dtype, top, temperature, masked):
    return dict(kind="logp", T=T, V=V, dtype=dtype, top=top, temperature=temperature,
                masked=masked)


def listed():
    return [
        # One token in front of a decoding step's projection: latency.
        dict(name="norm_one", **_norm(1, 4096, "int8", True)),
        # All tokens of a 1024px-like sequence in front of the int8 linears.
        dict(name="norm_block", **_norm(4608, 4096, "int8", True)),
        # Odd sizes in front of a 4-bit linear: channels that fill no block, the stack's first norm.
        dict(name="norm_ragged", **_norm(2001, 1000, "mx4", False)),
        # A decoding step's tokens, one of each of 64 sequences, cut out of a fused qkv projection,
        # far into long documents.
        dict(name="append_step", **_append(64, 8, 4, 128, 128, 64, "fp8", 1, False, 200000)),
        # Prompts of 20000 tokens in one pass, in 4 bits.
        dict(name="append_prompt", **_append(20000, 8, 4, 128, 128, 64, "fp4", 1, False, 20000)),
        # Frames of a video: time, height and width; a part of each head rotated, in neighbouring
        # pairs, at the 18 heads of 256 of the 4608-wide model.
        dict(name="append_video", **_append(4600, 18, 1, 256, 192, 48, "fp8", 3, True, 64)),
        # One sequence with a small tree of drafts: latency.
        dict(name="tree_one", **_tree(1, 13, 2001, 8, 4, 128, 16, "fp8", False)),
        # A serving batch, trees and lengths of its sequences very different.
        dict(name="tree_batch", **_tree(32, 60, 8192, 8, 4, 128, 64, "fp8", True)),
        # A wide tree over a long document in 4 bits; its nodes fill no word of the mask.
        dict(name="tree_wide", **_tree(1, 201, 40001, 8, 4, 128, 128, "fp4", False)),
        # One row of logits with its alternatives, as an interactive step returns them: latency.
        dict(name="logp_step", **_logp(1, 131072, "bf16", 20, 1.0, False)),
        # Drafted tokens of a batch, sharpened, a part of the vocabulary ruled out; an odd size.
        dict(name="logp_draft", **_logp(231, 100003, "fp32", 8, 0.7, True)),
        # Prompts scored.
        dict(name="logp_prompt", **_logp(4096, 131072, "bf16", 5, 1.0, False)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "append", "tree", "tree", "logp"])
    while True:
        if kind == "norm":
            M, K = _log(rng, 1, 8192), _log(rng, 64, 24576)
            if rng.random() < 0.6:   # as model widths are
                K = max(64, K // 64 * 64)
            if M * K <= 4608 * 4096:
                return _norm(M, K, rng.choice(["int8", "int8", "mx4"]), rng.random() < 0.7)
        elif kind == "append":
            T, heads, group = _log(rng, 1, 24000), rng.choice([1, 2, 5, 8, 18]), rng.choice([1, 3, 4, 8])
            dim, page = rng.choice([64, 128, 128, 192, 256]), rng.choice([16, 48, 64, 128])
            rotary = dim if rng.random() < 0.6 else 2 * rng.randint(3, dim // 2)
            if T * heads * (group + 2) * dim <= 20000 * 48 * 128:
                axes = rng.choice([1, 1, 2, 3])
                return _append(T, heads, group, dim, rotary, page, rng.choice(["fp8", "fp4"]), axes,
                               rng.random() < 0.4, _log(rng, 64, 1000000) if axes == 1 else 64)
        elif kind == "tree":
            seqs, nodes = _log(rng, 1, 64), _log(rng, 2, 300)
            kv_max = nodes + _log(rng, 1, 60000)
            heads, group = rng.choice([1, 2, 5, 8, 18]), rng.choice([1, 3, 4, 8])
            dim, page = rng.choice([64, 128, 128, 192, 256]), rng.choice([16, 48, 64, 128])
            c = _tree(seqs, nodes, kv_max, heads, group, dim, page, rng.choice(["fp8", "fp4"]),
                      rng.random() < 0.7)
            if (seqs * kv_max * heads * dim <= 3e8 and work(c)["flops"] <= 1.3e11
                    and seqs * nodes * heads * group * kv_max <= 4e8):
                return c
        else:
            T, V = _log(rng, 1, 8192), _log(rng, 1000, 250000)
            dtype = rng.choice(["bf16", "bf16", "fp32"])
            if T * V * (1 if dtype == "bf16" else 2) <= 4096 * 131072:
                return _logp(T, V, dtype, rng.choice([0, 1, 5, 20, rng.randint(2, 64)]),
                             rng.choice([1.0, 1.0, 0.6, 1.3]), rng.random() < 0.3)


def _lens(case):
    """(nodes, tokens) of each sequence: whole or, where ragged, spread over the range, with one
    that has nothing cached before its tree and one of a single node."""
    n, q, kv = case["seqs"], case["nodes"], case["kv_max"]
    if not case["ragged"]:
        return [q] * n, [kv] * n
    rng = random.Random(n * 1000003 + q * 1009 + kv)
    qs = [q if i == 0 else rng.randint(1, q) for i in range(n)]
    kvs = [kv if i == 0 else qs[i] + _log(rng, max(1, kv // 64), kv) for i in range(n)]
    kvs = [min(k, kv) for k in kvs]
    if n >= 3:
        kvs[1] = qs[1]
        qs[2] = 1
    return qs, kvs


def _sections(case):
    """Pairs of each axis: a half, a third ... of them, the last axis the rest."""
    pairs, axes = case["rotary"] // 2, case["axes"]
    cut = [pairs * i // axes for i in range(axes + 1)]
    return tuple(b - a for a, b in zip(cut, cut[1:]))


def _element_bytes(fmt, dim):
    return dim if fmt == "fp8" else dim // 2


def work(case):
    if case["kind"] == "norm":
        M, K = case["M"], case["K"]
        out = M * K + 4 * M if case["fmt"] == "int8" else M * (16 * -(-K // 32) + 8 * -(-K // 256))
        # codes are read again and what they stand for written
        return {"bytes": 2 * M * K * (3 if case["residual"] else 1) + 4 * K + 2 * out + 2 * M * K,
                "flops": 10 * M * K}
    if case["kind"] == "logp":
        T, V = case["T"], case["V"]
        return {"bytes": T * V * (2 if case["dtype"] == "bf16" else 4) + T * (16 + 12 * case["top"]),
                "flops": 6 * T * V}
    token = 2 * case["heads"] * (_element_bytes(case["fmt"], case["dim"]) + case["dim"] // 32)
    if case["kind"] == "append":
        T, kv, q = case["T"], 2 * case["heads"] * case["dim"], case["heads"] * case["group"] * case["dim"]
        return {"bytes": T * (4 * kv + 4 * q + 2 * token + 8 + 8 * case["axes"]),
                "flops": 6 * T * (kv + q)}
    qs, kvs = _lens(case)
    heads = case["heads"] * case["group"]
    pairs = sum(q * (kv - q) + q for q, kv in zip(qs, kvs))
    return {"bytes": sum(kvs) * token + 4 * sum(qs) * heads * case["dim"]
            + 8 * sum(qs) * -(-case["nodes"] // 64), "flops": 4 * pairs * heads * case["dim"]}


# ---------------------------------------------------------------- the formats, in 32 bits

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


def _encode(x, fmt):
    return _encode4(x) if fmt == "fp4" else _encode8(x)


def _values(codes, scales, fmt):
    """What codes [..., n bytes] and scale bytes [..., blocks] stand for, in 32 bits."""
    if fmt == "fp4":
        grid = torch.tensor(GRID4 + tuple(-g for g in GRID4), device=codes.device)
        v = torch.stack((grid[(codes & 15).int()], grid[(codes >> 4).int()]), -1).flatten(-2)
    else:
        v = codes.view(torch.float8_e4m3fn).float()
    scale = torch.where(scales == 255, torch.nan, _power(scales.int() - 127))
    return (v.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


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


def _kv(g, T, heads, dim):
    """Keys and values [T, 2, heads, dim]: N(0, 1), channels of the keys of different size."""
    x = torch.randn(T, 2, heads, dim, generator=g, device=DEV)
    x[:, 0] *= torch.exp(0.7 * torch.randn(heads, dim, generator=g, device=DEV))
    return x.to(torch.bfloat16)


def _prepare_norm(case, g, s):
    M, K = case["M"], case["K"]
    x = torch.randn(M, K, generator=g, device=DEV)
    s["x"] = x.to(torch.bfloat16)
    s["residual"] = None
    if case["residual"]:   # a residual stream has grown, and has two outlier channels
        r = 3.0 * torch.randn(M, K, generator=g, device=DEV)
        r[:, 17 % K] *= 20.0
        r[:, (3 * K // 4 + 5) % K] *= 20.0
        s["residual"] = r.to(torch.bfloat16)
    s["weight"] = torch.exp(0.3 * torch.randn(K, generator=g, device=DEV))


def _prepare_append(case, g, s):
    T, heads, group, dim, page = (case[n] for n in ("T", "heads", "group", "dim", "page"))
    q_heads = heads * group
    qkv = torch.randn(T, q_heads + 2 * heads, dim, generator=g, device=DEV).to(torch.bfloat16)
    qkv[:, q_heads:] = _kv(g, T, heads, dim).flatten(1, 2)
    s["q"], s["k"], s["v"] = qkv.split((q_heads, heads, heads), 1)
    t = torch.arange(T, device=DEV)
    if case["axes"] == 1:   # ends of documents in a step, whole documents in a prompt
        start = torch.randint(0, max(1, case["far"] - T if T > 256 else case["far"]), (T,),
                              generator=g, device=DEV)
        s["positions"] = start if T <= 256 else start[0] + t
    else:                   # time (of three axes), height, width
        side = max(1, math.isqrt(min(T, 1024)))
        grid = (t // (side * side), t // side % side, t % side)
        s["positions"] = torch.stack(grid[3 - case["axes"]:], 1)
    pairs = case["rotary"] // 2
    s["sections"] = _sections(case) if case["axes"] > 1 else None
    # each axis has frequencies of its own, from fast to slow
    span = torch.cat([torch.arange(n, dtype=torch.float64) / max(1, n) for n in _sections(case)])
    s["inv_freq"] = (10000.0 ** -span).float().to(DEV)
    assert s["inv_freq"].shape[0] == pairs
    # A token has a place of its own in pages taken at random, as an allocator hands them out
    # after a while; steps scatter over all pages, prompts fill theirs. The last few tokens of a
    # call are padding.
    pages = -(-T // page) + 8
    n_page = page * (_element_bytes(case["fmt"], dim) + dim // 32)
    s["cache"] = torch.zeros(pages, 2, heads, n_page, dtype=torch.uint8, device=DEV)
    order = torch.randperm(pages, generator=g, device=DEV)
    if T <= 256:
        slots = torch.randperm(pages * page, generator=g, device=DEV)[:T]
    else:
        slots = order[t // page] * page + t % page
    if T >= 16:
        slots[-3:] = -1
    s["slots"] = slots.to(torch.int64)


def _prepare_tree(case, g, s, seed):
    heads, dim, page, fmt = (case[n] for n in ("heads", "dim", "page", "fmt"))
    n_page = page * (_element_bytes(fmt, dim) + dim // 32)
    qs, kvs = _lens(case)
    need = [-(-n // page) for n in kvs]
    pages = sum(need) + 8
    s["cache"] = torch.zeros(pages, 2, heads, n_page, dtype=torch.uint8, device=DEV)
    codes, scales = _cache_views(s["cache"], page, dim, fmt)
    for lo in range(0, pages, 256):
        hi = min(pages, lo + 256)
        kv = _kv(g, (hi - lo) * page, heads, dim).unflatten(0, (hi - lo, page)).float()
        codes[lo:hi], scales[lo:hi] = _encode(kv.permute(0, 2, 3, 1, 4), fmt)
    order = torch.randperm(pages, generator=g, device=DEV).int().cpu()
    table = torch.zeros(len(kvs), -(-max(kvs) // page), dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    # Trees: a node hangs on one of those before it, or on the last token of the sequence, and
    # sees its ancestors and itself.
    rng = random.Random(seed)
    words = -(-case["nodes"] // 64)
    bits, starts = [], [0]
    for lq in qs:
        seen = []
        for i in range(lq):
            parent = rng.randrange(-1, i)
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
        bits += [[(m >> 64 * w) & (1 << 64) - 1 for w in range(words)] for m in seen]
        starts.append(starts[-1] + lq)
    bits = [[b - (1 << 64) if b >> 63 else b for b in row] for row in bits]
    s["tree"] = torch.tensor(bits, dtype=torch.int64).to(DEV)
    s["table"] = table.to(DEV)
    s["kv_lens"] = torch.tensor(kvs, dtype=torch.int32, device=DEV)
    s["q_starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["q"] = torch.randn(starts[-1], heads * case["group"], dim, generator=g,
                         device=DEV).to(torch.bfloat16)


def _prepare_logp(case, g, s):
    T, V = case["T"], case["V"]
    wide = -(-V // 64) * 64     # the vocabulary is padded in the projection's output
    x = torch.empty(T, wide, dtype=torch.bfloat16 if case["dtype"] == "bf16" else torch.float32,
                    device=DEV)
    for lo in range(0, T, 512):
        hi = min(T, lo + 512)
        y = 2.5 * torch.randn(hi - lo, wide, generator=g, device=DEV)
        # a few favourites of each row
        best = torch.randint(0, V, (hi - lo, 4), generator=g, device=DEV)
        y.scatter_(1, best, 8.0 + 6.0 * torch.rand(hi - lo, 4, generator=g, device=DEV))
        if case["masked"]:
            y.masked_fill_(torch.rand(hi - lo, wide, generator=g, device=DEV) < 0.5, -torch.inf)
        x[lo:hi] = y
    s["logits"] = x[:, :V]
    tokens = torch.randint(0, V, (T,), generator=g, device=DEV)
    likely = torch.rand(T, generator=g, device=DEV) < 0.7
    s["tokens"] = torch.where(likely, s["logits"].float().argmax(1) if T <= 1024 else tokens, tokens)
    if T >= 16:
        s["tokens"][-3:] = -1


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["kind"] == "norm":
        _prepare_norm(case, g, s)
    elif case["kind"] == "append":
        _prepare_append(case, g, s)
    elif case["kind"] == "tree":
        _prepare_tree(case, g, s, seed)
    else:
        _prepare_logp(case, g, s)
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2606_14598_amd as w8a8
    if s["kind"] == "norm":
        q, scale, h = w8a8.rms_norm_quantize(s["x"], s["weight"], residual=s["residual"], eps=EPS,
                                             fmt=s["fmt"])
        if s["fmt"] == "mx4":
            v = w8a8.mx4_dequantize(q, scale, s["K"])
        else:
            v = torch.empty_like(s["x"])
            torch.mul(q, scale[:, None], out=v)
        return (v, h) if s["residual"] is not None else v
    if s["kind"] == "append":
        q = w8a8.kv_append(s["cache"], s["k"], s["v"], s["slots"], s["positions"], s["inv_freq"],
                           q=s["q"], fmt=s["fmt"], sections=s["sections"],
                           interleaved=s["interleaved"])
        return q, *w8a8.kv_read(s["cache"], s["slots"], s["dim"], fmt=s["fmt"])
    if s["kind"] == "tree":
        return w8a8.kv_tree_attention(s["q"], s["cache"], s["table"], s["kv_lens"], s["tree"],
                                      fmt=s["fmt"], q_starts=s["q_starts"], max_q=s["nodes"],
                                      max_kv=s["kv_max"])
    return w8a8.token_logprobs(s["logits"], s["tokens"], top=s["top"], temperature=s["temperature"])


def _run_plain(s):
    return {"norm": _norm_plain, "append": _append_plain, "tree": _tree_plain,
            "logp": _logp_plain}[s["kind"]](s)


def _norm_plain(s):
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(torch.bfloat16)
    x = h.float()
    # The mean in 64 bits: codes hang on the last bit of a value next to a border.
    r = (1.0 / torch.sqrt(x.double().square().mean(-1, keepdim=True) + EPS)).float()
    v = x * r * s["weight"]
    if s["fmt"] == "mx4":
        K = v.shape[1]
        v = _values(*_encode4(torch.nn.functional.pad(v, (0, -K % 32))), "fp4")[:, :K]
    else:
        a = v.abs().amax(-1, keepdim=True)
        inv = 127.0 / a
        ok = (a > 0) & torch.isfinite(inv)
        q = torch.round(v * torch.where(ok, inv, 0.0)).clamp(-127.0, 127.0)
        v = q * torch.where(ok, a / 127.0, 0.0)
    v = v.to(torch.bfloat16)
    return (v, h) if s["residual"] is not None else v


def _rotated(x, cos, sin, interleaved):
    """x [T, heads, dim] with its first pairs turned, in 32 bits."""
    x, n = x.float(), cos.shape[-1]
    if interleaved:
        a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
    else:
        a, b = x[..., :n], x[..., n:2 * n]
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((c, d), -1).flatten(-2) if interleaved else torch.cat((c, d), -1)
    return torch.cat((turned, x[..., 2 * n:]), -1)


def _append_plain(s):
    p = s["positions"]
    if s["sections"] is not None:
        axis = torch.cat([torch.full((n,), i) for i, n in enumerate(s["sections"])]).to(DEV)
        p = p[:, axis]
    else:
        p = p[:, None]
    angle = (p.double() * s["inv_freq"].double())[:, None]     # far positions: 64 bits
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q = _rotated(s["q"], cos, sin, s["interleaved"]).to(torch.bfloat16)
    k = _rotated(s["k"], cos, sin, s["interleaved"])
    codes, scales = _cache_views(s["cache"], s["page"], s["dim"], s["fmt"])
    live = s["slots"] >= 0
    page, at = s["slots"] // s["page"], s["slots"] % s["page"]
    c, e = _encode(torch.stack((k, s["v"].float()), 1), s["fmt"])
    codes[page[live], :, :, at[live]] = c[live]
    scales[page[live], :, :, at[live]] = e[live]
    kv = _values(codes[page, :, :, at], scales[page, :, :, at], s["fmt"])
    kv = torch.where(live[:, None, None, None], kv, 0.0).to(torch.bfloat16)
    return q, kv[:, 0], kv[:, 1]


def _tree_plain(s):
    """Attention of every sequence at once, padded to the longest."""
    heads, group, dim, page = s["heads"], s["group"], s["dim"], s["page"]
    q_len = s["q_starts"][1:] - s["q_starts"][:-1]
    codes, scales = _cache_views(s["cache"], page, dim, s["fmt"])
    kv = _values(codes[s["table"]], scales[s["table"]], s["fmt"])   # [B, P, 2, H, page, D]
    kv = kv.permute(2, 0, 3, 1, 4, 5).flatten(3, 4)                 # [2, B, H, P * page, D]
    j = torch.arange(kv.shape[3], device=DEV)
    held = (j < s["kv_lens"][:, None])[:, None, :, None]
    k, v = torch.where(held, kv[0], 0.0), torch.where(held, kv[1], 0.0)
    i = torch.arange(s["nodes"], device=DEV)
    rows = (s["q_starts"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[rows].unflatten(2, (heads, group))           # [B, L, H, G, D]
    q = q.permute(0, 2, 3, 1, 4)
    node = j - (s["kv_lens"] - q_len)[:, None]                      # [B, keys]
    at = node.clamp(0, 64 * s["tree"].shape[1] - 1)[:, None].expand(-1, len(i), -1)
    bit = torch.gather(s["tree"][rows], 2, at // 64) >> at % 64 & 1
    seen = (node < 0)[:, None] | ((node < q_len[:, None])[:, None] & (bit == 1))
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


def _logp_plain(s):
    x, tokens, k = s["logits"].float(), s["tokens"], s["top"]
    V = x.shape[1]
    # Rank by value, the lower index first where values are equal: one whole number for both.
    bits = x.view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    best = (bits * V + (V - 1 - torch.arange(V, device=DEV))).topk(k, 1).indices
    x = x * (1.0 / s["temperature"])
    d = x - x.amax(1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    lse = torch.log(total)
    entropy = (lse - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total)[:, 0]
    live = (tokens >= 0) & (tokens < V)
    own_p = (d.gather(1, tokens.clamp(0, V - 1)[:, None]) - lse)[:, 0]
    return torch.where(live, own_p, 0.0), entropy, d.gather(1, best) - lse, best


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


def _exact_norm(case, s):
    h = s["x"].double()
    if s["residual"] is not None:   # the sum is kept in bf16: the norm is of what is kept
        h = (h + s["residual"].double()).to(torch.bfloat16).double()
    v = h * torch.rsqrt((h * h).sum(1) / case["K"] + EPS)[:, None] * s["weight"].double()
    if case["fmt"] == "mx4":
        K = case["K"]
        full = torch.zeros(v.shape[0], (K + 31) // 32 * 32, dtype=torch.float64, device=DEV)
        full[:, :K] = v
        v = _exact_values(full, "fp4")[:, :K]
    else:
        step = v.abs().max(1, keepdim=True).values / 127.0
        v = torch.where(step > 0, torch.round(v / step) * step, 0.0)
    return (v, h) if s["residual"] is not None else v


def _exact_append(case, s):
    T, pairs = case["T"], case["rotary"] // 2
    angle = torch.empty(T, pairs, dtype=torch.float64, device=DEV)
    at = 0
    for axis, n in enumerate(_sections(case)):
        p = s["positions"].reshape(T, -1)[:, axis].double()
        angle[:, at:at + n] = torch.outer(p, s["inv_freq"][at:at + n].double())
        at += n
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def rotate(x):
        y = x.double().clone()
        first, second = ((slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if case["interleaved"]
                         else (slice(0, pairs), slice(pairs, 2 * pairs)))
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        return y

    gone = (s["slots"] < 0)[:, None, None]
    k, v = (_exact_values(t, case["fmt"]).masked_fill(gone, 0.0)
            for t in (rotate(s["k"]), s["v"].double().contiguous()))
    return rotate(s["q"]), k, v


def _exact_tree(case, s):
    qs, kvs = _lens(case)
    heads, group, dim, page, fmt = (case[n] for n in ("heads", "group", "dim", "page", "fmt"))
    nb = _element_bytes(fmt, dim)
    out = torch.zeros(sum(qs), heads * group, dim, dtype=torch.float64, device=DEV)
    at = 0
    shift = torch.arange(64, device=DEV)
    for n, (lq, lk) in enumerate(zip(qs, kvs)):
        used = s["table"][n, :-(-lk // page)].long()
        hidden = torch.zeros(lq, lk, dtype=torch.bool, device=DEV)
        bits = (s["tree"][at:at + lq, :, None] >> shift & 1).reshape(lq, -1)
        hidden[:, lk - lq:] = bits[:, :lq] == 0
        for h in range(heads):
            raw = s["cache"][used][:, :, h]                        # [pages, 2, page bytes]
            c = raw[:, :, :page * nb].reshape(-1, 2, page, nb)
            e = raw[:, :, page * nb:].reshape(-1, 2, page, dim // 32)
            kv = _exact_decode(c, e, fmt).transpose(0, 1).reshape(2, -1, dim)[:, :lk]
            for r in range(group):
                q = s["q"][at:at + lq, h * group + r].double()
                z = (q @ kv[0].t() / math.sqrt(dim)).masked_fill(hidden, -math.inf)
                out[at:at + lq, h * group + r] = torch.softmax(z, -1) @ kv[1]
        at += lq
    return out


def _exact_logp(case, s):
    T, k = case["T"], case["top"]
    logp = torch.zeros(T, dtype=torch.float64, device=DEV)
    entropy = torch.zeros_like(logp)
    top = torch.zeros(T, k, dtype=torch.float64, device=DEV)
    ids = torch.zeros(T, k, dtype=torch.int64, device=DEV)
    for lo in range(0, T, 256):
        x = s["logits"][lo:lo + 256].double()
        p = torch.log_softmax(x / case["temperature"], 1)
        entropy[lo:lo + 256] = torch.special.entr(torch.exp(p)).sum(1)
        t = s["tokens"][lo:lo + 256]
        mine = p[torch.arange(len(t), device=DEV), t.clamp(min=0)]
        logp[lo:lo + 256] = torch.where(t < 0, 0.0, mine)
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
        ids[lo:lo + 256] = order
        top[lo:lo + 256] = p.gather(1, order)
    return logp, entropy, top, ids


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "append": _exact_append, "tree": _exact_tree,
            "logp": _exact_logp}[case["kind"]](case, s)
