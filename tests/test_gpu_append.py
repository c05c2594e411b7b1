"""Tokens appended to the cache with rotary positions, bit by bit against the definition."""
import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from _lm_ref import cos_sin, rotate
from _mx_ref import cache_slot, f64, pack4, quantize_blocks

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def freqs(pairs, base=10000.0):
    return (base ** -(torch.arange(pairs, dtype=torch.float64) / max(1, pairs))).float()


def bf16_of(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)


class Call:
    def __init__(self, fmt, dim, heads, q_heads, page, T, pairs, sections=None, interleaved=False,
                 far=100000, seed=0):
        self.fmt, self.dim, self.heads, self.q_heads, self.page = fmt, dim, heads, q_heads, page
        self.sections, self.interleaved = sections, interleaved
        g = torch.Generator().manual_seed(seed)
        self.pages = -(-T // page) + 2
        qkv = torch.randn(T, q_heads + 2 * heads, dim, generator=g)
        qkv *= torch.exp(torch.randn(q_heads + 2 * heads, dim, generator=g))
        self.qkv = qkv.to(torch.bfloat16)
        axes = 1 if sections is None else len(sections)
        self.positions = torch.randint(-far, far, (T, axes) if axes > 1 else (T,), generator=g)
        self.inv_freq = freqs(pairs)
        self.slots = torch.randperm(self.pages * page, generator=g)[:T]
        if T > 8:
            self.slots[3], self.slots[5], self.slots[7] = -1, -1000, self.pages * page

    def run(self, qkv=None, **kw):
        d = (self.qkv if qkv is None else qkv).cuda()
        q, k, v = d.split((self.q_heads, self.heads, self.heads), 1)
        self.cache = w8a8.kv_cache(self.pages, self.heads, self.dim, self.page, fmt=self.fmt)
        self.cache.fill_(0x5A)
        return w8a8.kv_append(self.cache, k, v, self.slots.cuda(), self.positions.cuda(),
                              self.inv_freq.cuda(), q=q if self.q_heads else None, fmt=self.fmt,
                              sections=self.sections, interleaved=self.interleaved, **kw)

    def check(self, q_out):
        cos, sin, near = cos_sin(self.positions.numpy(), self.inv_freq.numpy(), self.sections)
        assert near.sum() <= 1 + len(near) // 100
        x = self.qkv.float().numpy()
        turned = rotate(x, cos, sin, self.interleaved)
        if self.q_heads:
            want = bf16_of(turned[:, :self.q_heads])
            ok = torch.from_numpy(~near)
            assert torch.equal(q_out.cpu()[ok], want[ok])
        kv = turned.copy()
        kv[:, self.q_heads + self.heads:] = x[:, self.q_heads + self.heads:]
        kv = kv[:, self.q_heads:].reshape(len(x), 2, self.heads, self.dim).astype(np.float64)
        codes, scales = quantize_blocks(kv, self.fmt)
        got = self.cache.cpu().numpy()
        want = np.full(got.shape, 0x5A, np.uint8)
        for t, s in enumerate(self.slots.tolist()):
            if 0 <= s < self.pages * self.page:
                c, e = cache_slot(want, s, self.page, self.dim, self.fmt)
                c[:] = pack4(codes[t]) if self.fmt == "fp4" else codes[t]
                e[:] = scales[t]
                if near[t]:
                    for a, b in zip(cache_slot(got, s, self.page, self.dim, self.fmt), (c, e)):
                        a[:] = b
        assert np.array_equal(got, want)


CALLS = [
    # dim, heads, q heads, page, tokens, pairs, sections, interleaved
    (64, 1, 1, 16, 1, 32, None, False),
    (128, 8, 32, 64, 70, 64, None, False),
    (128, 8, 32, 64, 37, 64, None, True),
    (128, 2, 0, 16, 20, 64, None, False),              # keys and values alone
    (256, 5, 40, 48, 33, 96, (16, 40, 40), True),      # a part of each head, three axes
    (256, 18, 18, 64, 20, 128, (64, 64), False),
    (192, 3, 9, 16, 40, 96, None, False),
    (192, 1, 7, 16, 9, 33, (11, 0, 22), False),        # odd pairs, an axis of none
    (64, 2, 6, 32, 50, 5, None, False),
    (128, 3, 6, 16, 12, 63, (1, 20, 20, 22), True),
    (128, 2, 4, 16, 11, 0, None, False),               # no pairs: kv_write
    (256, 1, 3, 128, 130, 17, None, True),
]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("case", range(len(CALLS)))
def test_append(fmt, case):
    dim, heads, q_heads, page, T, pairs, sections, interleaved = CALLS[case]
    say(f"append {fmt} {CALLS[case]}")
    c = Call(fmt, dim, heads, q_heads, page, T, pairs, sections, interleaved, seed=case)
    c.check(c.run())


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_positions_of_zero_are_a_write(fmt):
    for pairs in (64, 0):
        c = Call(fmt, 128, 3, 6, 16, 30, pairs, seed=1)
        c.positions.zero_()
        q = c.run()
        assert torch.equal(q.cpu(), c.qkv[:, :6])
        d = c.qkv.cuda()
        other = torch.full_like(c.cache, 0x5A)
        w8a8.kv_write(other, d[:, 6:9], d[:, 9:], c.slots.cuda(), fmt=fmt)
        assert torch.equal(other, c.cache)


def test_every_float32_rounding():
    """Rotations by 45 degrees give float32 keys of all kinds: e4m3 and e2m1 roundings, ties and
    saturation from 32 bits, blocks of very small and very large keys."""
    for fmt in ("fp8", "fp4"):
        c = Call(fmt, 64, 4, 0, 16, 4000, 32, seed=2)
        scale = torch.logspace(-39, 37, 4000).to(torch.float32)
        c.qkv = (c.qkv.float().clamp(-9, 9) * scale[:, None, None]).to(torch.bfloat16)
        c.inv_freq[:] = 1.0
        c.positions = torch.arange(4000)
        c.check(c.run())


def test_far_positions():
    """Angles of up to 2^31 radians."""
    c = Call("fp8", 128, 1, 4, 16, 300, 64, far=2 ** 31 - 1, seed=3)
    c.check(c.run())


def test_non_finite_keys():
    c = Call("fp8", 128, 2, 2, 16, 8, 64, seed=4)
    c.qkv[2, 2, 40] = float("inf")       # a key: turned with its partner, 64 channels on
    c.qkv[4, 5, 100] = float("nan")      # a value
    c.run()
    k, v = w8a8.kv_read(c.cache, c.slots.cuda(), 128)
    bad = np.zeros((8, 2, 128), bool)
    bad[2, 0, 32:64] = bad[2, 0, 96:128] = True
    assert np.array_equal(np.isnan(f64(k)), bad)
    bad[:] = False
    bad[4, 1, 96:128] = True
    assert np.array_equal(np.isnan(f64(v)), bad)


@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_and_alignment(interleaved):
    """Operands anywhere in larger tensors, at any element."""
    c = Call("fp4", 128, 2, 4, 16, 10, 60 if interleaved else 40, interleaved=interleaved, seed=5)
    want = c.run()
    c.check(want)
    for off in (1, 3):
        flat = torch.zeros(10 * 12 * 128 + 8, dtype=torch.bfloat16, device="cuda")
        wide = flat[off:off + 10 * 12 * 128].view(10, 12, 128)
        wide[:, 2:10] = c.qkv.cuda()
        out = torch.zeros(10 * 4 * 128 + 8, dtype=torch.bfloat16, device="cuda")
        o = out[off:off + 10 * 4 * 128].view(10, 4, 128)
        cache = torch.full_like(c.cache, 0x5A)
        y = w8a8.kv_append(cache, wide[:, 6:8], wide[:, 8:10], c.slots.cuda(), c.positions.cuda(),
                           c.inv_freq.cuda(), q=wide[:, 2:6], fmt="fp4", interleaved=interleaved, out=o)
        assert y.data_ptr() == o.data_ptr() and torch.equal(y, want) and torch.equal(cache, c.cache)
        assert (out[:off] == 0).all() and (out[off + 10 * 4 * 128:] == 0).all()


def test_offsets_beyond_32_bits():
    """More than 2^31 elements of queries, pages more than 4 GiB into the cache."""
    T, q_heads, n = 530000, 32, 50
    page_bytes = w8a8.kv_cache(0, 1, 128, 128).shape[1:].numel()
    pages = (1 << 32) // page_bytes + 40
    q = torch.zeros(T, q_heads, 128, dtype=torch.bfloat16, device="cuda")
    q[-n:] = torch.randn(n, q_heads, 128, device="cuda").to(torch.bfloat16)
    k = torch.randn(T, 1, 128, device="cuda").to(torch.bfloat16)
    slots = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    slots[-n:] = pages * 128 - 1 - torch.arange(n, device="cuda")
    pos = torch.arange(T, device="cuda")
    cache = w8a8.kv_cache(pages, 1, 128, 128)
    f = freqs(64).cuda()
    y = w8a8.kv_append(cache, k, k, slots, pos, f, q=q)
    small = w8a8.kv_cache(1, 1, 128, 128)
    y2 = w8a8.kv_append(small, k[-n:], k[-n:], 127 - torch.arange(n, device="cuda"), pos[-n:], f, q=q[-n:])
    assert torch.equal(y[-n:], y2) and torch.equal(cache[-1], small[0]) and not cache[:-1].any()
    del q, y, cache
    torch.cuda.empty_cache()


def test_no_pages_and_no_tokens():
    c = Call("fp8", 64, 2, 4, 16, 5, 32, seed=6)
    want = c.run()
    d = c.qkv.cuda()
    none = w8a8.kv_cache(0, 2, 64, 16)
    args = (c.slots.cuda(), c.positions.cuda(), c.inv_freq.cuda())
    y = w8a8.kv_append(none, d[:, 4:6], d[:, 6:], *args, q=d[:, :4])
    assert torch.equal(y, want)
    y = w8a8.kv_append(c.cache, d[:0, 4:6], d[:0, 6:], args[0][:0], args[1][:0], args[2], q=d[:0, :4])
    assert y.shape == (0, 4, 64)


def test_binding_refusals():
    c = Call("fp8", 128, 2, 4, 16, 6, 64, seed=7)
    c.run()
    d = c.qkv.cuda()
    k, v = d[:, 4:6], d[:, 6:]
    ok = dict(slots=c.slots.cuda(), positions=c.positions.cuda(), inv_freq=c.inv_freq.cuda(), q=d[:, :4])

    def call(k=k, v=v, **kw):
        a = {**ok, **kw}
        return w8a8.kv_append(c.cache, k, v, a.pop("slots"), a.pop("positions"), a.pop("inv_freq"), **a)
    p2 = torch.zeros(6, 2, dtype=torch.int64, device="cuda")
    for bad in (dict(k=k[:, :1]), dict(v=v[:5]), dict(slots=ok["slots"][:5]), dict(positions=ok["positions"][:5]),
                dict(positions=p2), dict(positions=p2, sections=(32, 31)), dict(sections=(32, 32)),
                dict(positions=p2, sections=(-1, 65)), dict(inv_freq=torch.ones(65, device="cuda")),
                dict(q=d[:5, :4]), dict(q=None, out=d[:, :4]), dict(out=torch.empty_like(v)),
                dict(positions=ok["positions"].cpu()), dict(fmt="fp4"),
                dict(positions=torch.zeros(6, 5, dtype=torch.int64, device="cuda"), sections=(64, 0, 0, 0, 0))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(positions=ok["positions"].int()), dict(inv_freq=ok["inv_freq"].double()),
                dict(positions=[0] * 6), dict(q=d[:, :4].float())):
        with pytest.raises(TypeError):
            call(**bad)


@pytest.mark.parametrize("dim", [64, 192, 256])
def test_every_number_of_pairs(dim):
    """Halves that end anywhere in a unit of 8 channels."""
    for pairs in range(dim // 2 + 1):
        c = Call("fp8" if pairs % 2 else "fp4", dim, 1, 2, 16, 3, pairs, seed=pairs)
        c.check(c.run())
