"""The quantized key/value cache and the attention over it against plain 64-bit forms."""
import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from _mx_ref import (attention, block_values, cache_slot, code_bytes, f64, pack4, quantize_blocks,
                     slot_values)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _kv(T, heads, dim, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, 2, heads, dim, generator=g)
    x *= torch.exp(torch.randn(heads, dim, generator=g))
    return x.to(torch.bfloat16)


# ---------------------------------------------------------------- write and read

@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("heads,page,T", [(1, 16, 1), (3, 48, 37), (8, 64, 130)])
def test_write_and_read(fmt, dim, heads, page, T):
    pages = -(-T // page) + 2
    kv = _kv(T, heads, dim, T + dim)
    g = torch.Generator().manual_seed(T)
    slots = torch.randperm(pages * page, generator=g)[:T]
    if T > 8:
        slots[3], slots[5], slots[7] = -1, -1000, pages * page   # padding, padding, past the cache
    cache = w8a8.kv_cache(pages, heads, dim, page, fmt=fmt)
    cache.fill_(0x5A)
    # keys and values cut out of a fused projection
    qkv = torch.zeros(T, 4 * heads, dim, dtype=torch.bfloat16)
    qkv[:, heads:2 * heads], qkv[:, 3 * heads:] = kv[:, 0], kv[:, 1]
    qkv = qkv.cuda()
    w8a8.kv_write(cache, qkv[:, heads:2 * heads], qkv[:, 3 * heads:], slots.cuda(), fmt=fmt)
    want = np.full(tuple(cache.shape), 0x5A, np.uint8)
    codes, scales = quantize_blocks(f64(kv), fmt)
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < pages * page:
            c, e = cache_slot(want, s, page, dim, fmt)
            c[:] = pack4(codes[t]) if fmt == "fp4" else codes[t]
            e[:] = scales[t]
    assert np.array_equal(cache.cpu().numpy(), want)
    k, v = w8a8.kv_read(cache, slots.cuda(), dim, fmt=fmt)
    values = block_values(codes, scales, fmt)
    values[(slots.numpy() < 0) | (slots.numpy() >= pages * page)] = 0.0
    assert np.array_equal(f64(k), values[:, 0]) and np.array_equal(f64(v), values[:, 1])


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_every_bf16_value_written(fmt):
    bits = torch.arange(0x7F80, dtype=torch.int32)
    vals = torch.cat((bits, bits | 0x8000)).to(torch.int16).view(torch.bfloat16)
    for factor in (0, 2, 300):
        x = torch.zeros(vals.numel() // 8, 8, 64, dtype=torch.bfloat16)
        x[:, :, 3] = vals.view(-1, 8)
        x[:, :, 17] = (vals.float().abs() * factor).clamp(max=3e38).to(torch.bfloat16).view(-1, 8)
        T = x.shape[0]
        cache = w8a8.kv_cache(-(-T // 64), 8, 64, fmt=fmt)
        slots = torch.arange(T).cuda()
        w8a8.kv_write(cache, x.cuda(), -x.cuda(), slots, fmt=fmt)
        k, v = w8a8.kv_read(cache, slots, 64, fmt=fmt)
        want = block_values(*quantize_blocks(f64(x), fmt), fmt)
        want = torch.from_numpy(want).to(torch.bfloat16)     # the smallest e4m3 values round
        assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), -want)


def test_non_finite_blocks_and_unaligned_rows():
    for fmt in ("fp8", "fp4"):
        flat = _kv(4, 2, 128, 3).flatten().cuda()
        x = torch.empty(flat.numel() + 8, dtype=torch.bfloat16, device="cuda")
        for off in (0, 1, 3):
            x[off:off + flat.numel()] = flat
            k = x[off:off + 4 * 2 * 2 * 128].view(4, 2, 2, 128)[:, 0]
            v = x[off:off + 4 * 2 * 2 * 128].view(4, 2, 2, 128)[:, 1]
            k[1, 0, 40], v[2, 1, 127] = float("nan"), float("-inf")
            cache = w8a8.kv_cache(1, 2, 128, 16, fmt=fmt)
            slots = torch.tensor([5, 0, 15, 7]).cuda()
            w8a8.kv_write(cache, k, v, slots, fmt=fmt)
            gk, gv = w8a8.kv_read(cache, slots, 128, fmt=fmt)
            for got, src in ((gk, k), (gv, v)):
                want = block_values(*quantize_blocks(f64(src), fmt), fmt)
                assert np.array_equal(f64(got), want, equal_nan=True)
            assert np.isnan(f64(gk)).sum() == 32 and np.isnan(f64(gv)).sum() == 32


# ---------------------------------------------------------------- attention

class Case:
    """A cache filled through kv_write, its page table in random order, queries."""

    def __init__(self, fmt, dim, heads, group, page, qs, kvs, seed=0, spare=3, base=0):
        self.fmt, self.dim, self.heads, self.group, self.page = fmt, dim, heads, group, page
        self.qs, self.kvs = qs, kvs
        g = torch.Generator().manual_seed(seed)
        need = [-(-n // page) for n in kvs]
        pages = sum(need) + spare
        order = (torch.randperm(pages, generator=g) + base).tolist()
        self.cache = torch.empty(w8a8.kv_cache(0, heads, dim, page, fmt=fmt).shape[1:].numel() *
                                 (pages + base), dtype=torch.uint8, device="cuda")
        self.cache = self.cache.view(pages + base, 2, heads, -1)
        self.cache[base:] = 0xFF        # every scale and e4m3 code a NaN
        width = max(need + [1]) + 1
        self.table = torch.full((len(kvs), width), 0x7FFFFFFF, dtype=torch.int32)
        self.k, self.v, slots, at = [], [], [], 0
        for b, n in enumerate(kvs):
            p = order[at:at + need[b]]
            at += need[b]
            self.table[b, :need[b]] = torch.tensor(p, dtype=torch.int32)
            slots += [p[j // page] * page + j % page for j in range(n)]
        kv = _kv(sum(kvs), heads, dim, seed + 1)
        self.q = torch.randn(sum(qs), heads * group, dim, generator=g).to(torch.bfloat16)
        self.write(kv, slots)
        self.kv_lens = torch.tensor(kvs, dtype=torch.int32).cuda()
        self.q_starts = torch.tensor([0] + list(np.cumsum(qs)), dtype=torch.int32).cuda()

    def write(self, kv, slots):
        slots = torch.tensor(slots, dtype=torch.int64).cuda()
        d = kv.cuda()
        w8a8.kv_write(self.cache, d[:, 0], d[:, 1], slots, fmt=self.fmt)
        self.values = block_values(*quantize_blocks(f64(kv), self.fmt), self.fmt)

    def run(self, q=None, **kw):
        kw.setdefault("q_starts", self.q_starts)
        return w8a8.kv_attention(self.q.cuda() if q is None else q, self.cache, self.table.cuda(),
                                 self.kv_lens, fmt=self.fmt, **kw)

    def check(self, y, scale=None, causal=True):
        """Within the rounding of the weights and of the output to bf16 (2^-8 of the weighted
        mean of |v| each): 2^-7 of that mean."""
        scale = self.dim ** -0.5 if scale is None else scale
        y, q = f64(y), f64(self.q)
        assert np.isfinite(y).all()
        at_q = at_k = 0
        for lq, lk in zip(self.qs, self.kvs):
            for h in range(self.heads * self.group):
                kv = self.values[at_k:at_k + lk, :, h // self.group]
                want, mag = attention(q[at_q:at_q + lq, h], kv[:, 0], kv[:, 1], scale, causal)
                err = np.abs(y[at_q:at_q + lq, h] - want)
                assert (err <= mag * 2.0 ** -7 + 1e-30).all(), (lq, lk, h, err.max(), mag.max())
            at_q, at_k = at_q + lq, at_k + lk


ATTN = [
    # dim, heads, group, page, queries, keys
    (128, 2, 4, 16, [1], [1]),
    (128, 2, 4, 16, [1, 1, 1, 1], [1, 0, 17, 300]),
    (64, 1, 1, 16, [1, 1], [33, 64]),
    (192, 3, 3, 48, [1, 1, 1], [47, 48, 200]),
    (256, 2, 1, 64, [1, 1], [129, 1]),
    (128, 1, 16, 64, [1, 1], [1000, 31]),
    (128, 2, 20, 32, [1, 1], [70, 257]),          # more rows a head than a fragment has
    (128, 1, 8, 128, [1], [5000]),
    (128, 2, 4, 16, [5, 1, 3], [5, 40, 77]),       # a few queries each
    (64, 2, 3, 16, [33, 2], [33, 90]),
    (256, 1, 1, 64, [100, 17], [100, 300]),
    (128, 2, 4, 64, [70, 1, 130], [200, 1, 131]),
    (192, 1, 5, 16, [40], [41]),
    (128, 1, 1, 16, [300], [1100]),
    (128, 1, 2, 16, [9, 4], [3, 0]),               # more queries than keys: rows that see none
]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention(fmt, case):
    dim, heads, group, page, qs, kvs = ATTN[case]
    say(f"attention {fmt} {ATTN[case]}")
    c = Case(fmt, dim, heads, group, page, qs, kvs, seed=case)
    c.check(c.run())
    c.check(c.run(causal=False), causal=False)
    # what the launch is laid out for does not matter to the results beyond their rounding
    for mq, mk in ((1, 1), (max(qs), max(kvs)), (1000, 1 << 20)):
        c.check(c.run(max_q=mq, max_kv=mk))
    c.check(c.run(scale=0.3), scale=0.3)


# Sequences of very different lengths: shares that the kernels take from the sum of all lengths,
# of a few sequences, of more than a wavefront sums at once, and of more than it sums at all.
UNEQUAL = [
    (128, 1, 4, 16, [1, 3, 1, 2], [9000, 700, 0, 5000]),
    (64, 2, 1, 16, [1] * 70, [20000, 30000, 0, 1] + [1500] * 66),
    (64, 1, 2, 16, [1] * 600, [9000] + [i % 40 for i in range(599)]),
    (128, 1, 2, 64, [70, 1, 130], [2000, 1500, 900]),
    (256, 2, 1, 64, [128, 40, 0, 129], [6000, 40, 0, 700]),
    (64, 18, 2, 16, [17] * 9, [1300, 17, 20, 400, 17, 33, 100, 19, 600]),
]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("case", range(len(UNEQUAL)))
def test_unequal_lengths(fmt, case):
    dim, heads, group, page, qs, kvs = UNEQUAL[case]
    say(f"attention, unequal lengths {fmt} {UNEQUAL[case][:4]}")
    c = Case(fmt, dim, heads, group, page, qs, kvs, seed=case)
    first = c.run()
    c.check(first)
    assert torch.equal(first, c.run())
    c.check(c.run(max_q=max(qs), max_kv=max(kvs)))
    c.check(c.run(causal=False), causal=False)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_decoding_without_starts_and_strided_queries(fmt):
    c = Case(fmt, 128, 2, 4, 16, [1, 1, 1], [20, 0, 333], seed=5)
    wide = torch.zeros(3, 20, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, 7:15] = c.q.cuda()
    y = c.run(q=wide[:, 7:15], q_starts=None)
    c.check(y)
    assert torch.equal(y, c.run(q_starts=None)) and (y[1] == 0).all()
    c2 = Case(fmt, 64, 1, 2, 16, [4, 4], [50, 9], seed=6)
    c2.check(c2.run(q_starts=None))


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("qs,kvs,nan_at", [([6], [50], 47), ([1], [50], 20), ([200], [400], 300)])
def test_nan_tokens_reach_only_the_queries_that_see_them(fmt, qs, kvs, nan_at):
    for part in (0, 1):
        c = Case(fmt, 128, 1, 2, 16, qs, kvs, seed=7)
        kv = _kv(kvs[0], 1, 128, 8)
        kv[nan_at, part, 0, 70] = float("nan")
        page_of = c.table[0].tolist()
        c.write(kv, [page_of[j // 16] * 16 + j % 16 for j in range(kvs[0])])
        y = f64(c.run())
        lq = qs[0]
        sees = np.array([kvs[0] - lq + i >= nan_at for i in range(lq)])
        bad = np.zeros(y.shape, bool)
        bad[sees, :, :] = True
        if part == 1:                      # a value's block, not the others of its token
            bad[:, :, :64], bad[:, :, 96:] = False, False
        assert np.array_equal(np.isnan(y), bad)
        ok = ~sees
        if ok.any():
            kvv = c.values[:, :, 0]
            for h in range(2):
                n0 = kvs[0] - lq
                first = int(ok.sum())
                want, mag = attention(f64(c.q)[:first, h], kvv[:n0 + first, 0], kvv[:n0 + first, 1],
                                      128 ** -0.5, True)
                assert (np.abs(y[:first, h] - want) <= mag * 2.0 ** -7).all()


def test_scales():
    """Negative, zero and large scales, in both kernels."""
    for qs, kvs in (([1, 2], [300, 40]), ([60], [130])):
        c = Case("fp8", 128, 1, 2, 16, qs, kvs, seed=13)
        for scale in (-0.2, 0.0, 1e-6, 3.0):
            c.check(c.run(scale=scale), scale=scale)


def test_extreme_scores():
    """Rows whose scores differ by hundreds: one key takes all the weight, sums stay finite."""
    c = Case("fp8", 128, 1, 1, 16, [1, 1], [100, 37], seed=9)
    c.q = (c.q.float() * 300).to(torch.bfloat16)
    c.check(c.run(), None)
    c.q = torch.zeros_like(c.q)
    c.check(c.run(), None)


def test_offsets_beyond_32_bits():
    """Pages that lie more than 4 GiB into the cache."""
    page_bytes = w8a8.kv_cache(0, 2, 128, 128, fmt="fp8").shape[1:].numel()
    base = (1 << 32) // page_bytes + 5
    c = Case("fp8", 128, 2, 4, 128, [1, 3], [400, 129], seed=10, base=base)
    c.check(c.run())
    slots = torch.tensor([int(c.table[0, j // 128]) * 128 + j % 128 for j in range(400)])
    k, v = w8a8.kv_read(c.cache, slots.cuda(), 128)
    assert np.array_equal(f64(k), c.values[:400, 0]) and np.array_equal(f64(v), c.values[:400, 1])


@pytest.mark.parametrize("qs,kvs", [([1] * 3, [2000, 100, 1]), ([64, 100], [300, 100])])
def test_out_workspace_stream_and_repeats(qs, kvs):
    c = Case("fp8", 128, 2, 4, 64, qs, kvs, seed=11)
    want = c.run()
    T = sum(qs)
    guard = torch.full((T + 2, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    n = w8a8.load_library().w8a8_kv_attention_workspace_bytes(
        64, 2, 128, 0, 4, T, len(qs), T, c.table.shape[1] * 64)
    work = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    q = c.q.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(4):
            y = c.run(q=q, out=guard[1:-1], workspace=work[:n])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    assert (guard[0] == 7).all() and (guard[-1] == 7).all() and (work[n:] == 0xA5).all()
    if n > 0:
        with pytest.raises(ValueError):
            c.run(workspace=work[:n - 1])


def test_graph_of_a_decoding_step():
    """kv_write and kv_attention captured once, replayed with other inputs and lengths."""
    c = Case("fp4", 128, 2, 4, 16, [1, 1], [100, 40], seed=12, spare=6)
    table = c.table.cuda()
    q, k, v = c.q.cuda(), torch.empty(2, 2, 128, dtype=torch.bfloat16, device="cuda"), None
    v = torch.empty_like(k)
    lens = c.kv_lens.clone()
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    out = torch.empty_like(q)
    n = w8a8.load_library().w8a8_kv_attention_workspace_bytes(16, 2, 128, 1, 4, 2, 2, 1,
                                                              c.table.shape[1] * 16)
    work = torch.empty(n, dtype=torch.uint8, device="cuda")

    def step(o, w):
        w8a8.kv_write(c.cache, k, v, slots, fmt="fp4")
        return w8a8.kv_attention(q, c.cache, table, lens, fmt="fp4", out=o, workspace=w)

    def inputs(i):
        pos = [c.kvs[0] - 1 - i, c.kvs[1] - 1 - i]
        slots.copy_(torch.tensor([int(c.table[b, p // 16]) * 16 + p % 16 for b, p in enumerate(pos)]))
        lens.copy_(torch.tensor([p + 1 for p in pos], dtype=torch.int32))
        g = torch.Generator().manual_seed(i)
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g).to(torch.bfloat16))

    inputs(0)
    step(out, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, work)
    for i in range(1, 4):
        inputs(i)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step(None, None)) and code_bytes(128, "fp4") == 64
