"""The quantized cache and the attention over it at the ends of their ranges."""
import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from _mx_ref import attention, f64
from test_gpu_kv import Case, _kv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


# ---------------------------------------------------------------- launches beyond a grid

def test_many_sequences_without_bounds():
    """6000 sequences of one token each without max_q: 64 query heads' rows of 6000 tokens for every
    one of them would be more threads than a launch can have."""
    B, heads, group, dim = 6000, 8, 8, 64
    cache = w8a8.kv_cache(2, heads, dim, 16)
    kv = _kv(2, heads, dim, 25).cuda()
    w8a8.kv_write(cache, kv[:, 0], kv[:, 1], torch.tensor([0, 16]).cuda())
    _, v = w8a8.kv_read(cache, torch.tensor([0, 16]).cuda(), dim)
    table = (torch.arange(B, dtype=torch.int32) % 2)[:, None].cuda()
    q = torch.randn(B, heads * group, dim, generator=torch.Generator().manual_seed(26))
    q = q.to(torch.bfloat16).cuda()
    starts = torch.arange(B + 1, dtype=torch.int32).cuda()
    lens = torch.ones(B, dtype=torch.int32).cuda()
    want = v[torch.arange(B).cuda() % 2].repeat_interleave(group, 1)   # the only key's value
    say("6000 sequences, max_q left out")
    assert torch.equal(w8a8.kv_attention(q, cache, table, lens, q_starts=starts), want)
    assert torch.equal(w8a8.kv_attention(q, cache, table, lens, q_starts=starts, max_q=1), want)


def test_bounds_beyond_an_int():
    """Bounds that stand for none, past what the C ABI's ints hold; a negative one is refused."""
    c = Case("fp8", 64, 1, 2, 16, [3, 70], [40, 700], seed=28)
    want = c.run()
    for none in ((1 << 31) - 1, 1 << 31, (1 << 32) + 1, 1 << 62):
        assert torch.equal(c.run(max_q=none, max_kv=none), want)
    for bad in (dict(max_q=-1), dict(max_kv=-1)):
        with pytest.raises(w8a8.W8A8Error):
            c.run(**bad)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_more_tokens_than_a_grid_holds(fmt):
    """2^26 + 5 tokens in one call, padding but for the first two and the last three."""
    T, dim = (1 << 26) + 5, 64
    live = torch.tensor([0, 1, (1 << 25) + 7, T - 3, T - 2, T - 1]).cuda()
    slots = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    slots[live] = torch.tensor([3, 17, 9, 31, 0, 22]).cuda()
    kv = _kv(1, 1, dim, 27).cuda()
    cache = w8a8.kv_cache(2, 1, dim, 16, fmt=fmt)
    say(f"{T} tokens {fmt}")
    w8a8.kv_write(cache, kv[:, 0].expand(T, 1, dim), kv[:, 1].expand(T, 1, dim), slots, fmt=fmt)
    one = w8a8.kv_cache(1, 1, dim, 16, fmt=fmt)
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    w8a8.kv_write(one, kv[:, 0], kv[:, 1], zero, fmt=fmt)
    k, v = w8a8.kv_read(cache, slots, dim, fmt=fmt)
    for got, want in zip((k, v), w8a8.kv_read(one, zero, dim, fmt=fmt)):
        assert torch.equal(got[live], want.expand(6, 1, dim))
        for at in (2, 1 << 25, (1 << 26) - 3, T - 10):
            assert (got[at:at + 5] == 0).all()


# ---------------------------------------------------------------- scores without a finite one

def _slots(c):
    return [int(c.table[b, j // c.page]) * c.page + j % c.page
            for b, n in enumerate(c.kvs) for j in range(n)]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("qs,kvs", [([3], [40]), ([1], [3000]), ([200], [150]), ([150], [5000])])
def test_infinite_queries_give_nan(fmt, qs, kvs):
    """An infinity in a query makes all its scores infinite. exp(score - max) is then NaN whatever
    the sign; a query that sees no key still gives zeros."""
    c = Case(fmt, 64, 1, 2, 16, qs, kvs, seed=21)
    kv = _kv(sum(kvs), 1, 64, 22)
    kv[:, 0, 0, 5] = 2.0 ** 6
    c.write(kv, _slots(c))
    lq, lk = qs[0], kvs[0]
    c.q[::2, 0, 5], c.q[1::2, 0, 5] = -float("inf"), float("inf")
    c.q[::2, 1, 5] = float("inf")
    y = f64(c.run())
    sees = np.array([lk - lq + i >= 0 for i in range(lq)])
    assert (y[~sees] == 0).all()
    assert np.isnan(y[sees, 0]).all() and np.isnan(y[sees & (np.arange(lq) % 2 == 0), 1]).all()
    odd = sees & (np.arange(lq) % 2 == 1)
    assert np.isfinite(y[odd, 1]).all()


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("qs,kvs", [([2], [60]), ([1], [4000]), ([100], [4000])])
def test_scores_that_overflow_take_no_weight(fmt, qs, kvs):
    """Finite queries and keys whose products pass float32's least number: those keys' weights are
    zero, in a part of the keys that holds nothing else too."""
    c = Case(fmt, 64, 1, 1, 16, qs, kvs, seed=23)
    kv = _kv(sum(kvs), 1, 64, 24)
    n = kvs[0] // 2
    kv[:, 0, 0, :32] = 0.0
    kv[:n, 0, 0, 5] = 8.0
    c.write(kv, _slots(c))
    c.q[:, 0, 5] = -3e38
    y, at = f64(c.run()), kvs[0] - qs[0]
    q = f64(c.q)[:, 0]
    q[:, 5] = 0.0
    for i in range(qs[0]):
        v = c.values[n:at + i + 1, :, 0]
        want, mag = attention(q[i:i + 1], v[:, 0], v[:, 1], 64 ** -0.5, False)
        assert (np.abs(y[i, 0] - want[0]) <= mag[0] * 2.0 ** -7 + 1e-30).all()


# ---------------------------------------------------------------- rounding of the weights

class Cancelling(Case):
    """Values of +1 and -1 in pairs of tokens whose keys differ by one sign, so that outputs nearly
    cancel: what is left shows how the weights were rounded, not how the output was."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        kv = _kv(sum(self.kvs), self.heads, self.dim, 77)
        g = torch.Generator().manual_seed(78)
        kv[:, 0] = torch.randn(kv[:, 0].shape, generator=g).to(torch.bfloat16)
        sign = torch.where(torch.rand(kv[:, 1].shape, generator=g) < 0.5, -1.0, 1.0)
        kv[:, 1] = sign.to(torch.bfloat16)
        for at in range(0, kv.shape[0] - 1, 2):
            kv[at + 1, 0], kv[at + 1, 1] = kv[at, 0], -kv[at, 1]
            kv[at + 1, 0, :, 0] *= -1.0
        self.write(kv, _slots(self))

    def check_two_terms(self, y, only=None):
        """Each weight within 2^-16 of itself (two bf16 terms), the exponential and its argument
        within 2^-20, a score within dim 2^-23 of sum |q k|, sums of n weights within n 2^-23; all
        of it twice, for the sum of weights that divides; the output's own rounding 2^-8. Values
        are +1 and -1. One bf16 term would leave 2^-9 / sqrt(3 n) of noise, several times that."""
        scale = 1.0 / self.dim
        y, q = f64(y), f64(self.q)
        at_q = at_k = 0
        for b, (lq, lk) in enumerate(zip(self.qs, self.kvs)):
            for h in range(self.heads * self.group):
                if only is not None and b not in only:
                    continue
                kv = self.values[at_k:at_k + lk, :, h // self.group]
                rows = q[at_q:at_q + lq, h]
                want, _ = attention(rows, kv[:, 0], kv[:, 1], scale, True)
                score = (np.abs(rows) @ np.abs(kv[:, 0]).T).max(1) * scale
                tol = 2 * (2.0 ** -16 + 2.0 ** -20 + (self.dim * score[:, None] + lk) * 2.0 ** -23)
                err = np.abs(y[at_q:at_q + lq, h] - want)
                assert (err <= tol + np.abs(want) * 2.0 ** -8).all(), (b, lq, lk, h, (err / tol).max())
            at_q, at_k = at_q + lq, at_k + lk


TWO_TERMS = [
    # dim, heads, group, page, queries, keys: up to 64 rows of a sequence and head
    (128, 2, 4, 16, [10], [60]),
    (128, 2, 4, 16, [10], [1400]),                  # divided keys
    (64, 16, 4, 16, [10] * 8, [50] * 8),            # enough heads and sequences for 128-row tiles
    (256, 16, 2, 16, [28] * 8, [44] * 8),
    (128, 16, 4, 16, [12] * 8, [700, 30] * 4),
    (192, 8, 1, 16, [64] * 2, [80, 700]),
    (128, 2, 4, 16, [1] * 48, [40] * 48),           # one token each, of a batch
    (64, 4, 1, 16, [33, 64, 1], [50, 64, 3]),
    (128, 2, 4, 16, [1, 200, 12, 13, 3], [700, 300, 41, 70, 5000]),     # prompts among them
    (64, 16, 4, 16, [12, 1] * 6 + [60], [700, 5000] * 6 + [100]),
]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("case", range(len(TWO_TERMS)))
def test_weights_of_few_rows_in_two_terms(fmt, case):
    """Whatever the batch, the bounds that the launch is laid out for, and the kernel."""
    dim, heads, group, page, qs, kvs = TWO_TERMS[case]
    say(f"two terms {fmt} {TWO_TERMS[case]}")
    c = Cancelling(fmt, dim, heads, group, page, qs, kvs, seed=case)
    few = [b for b, n in enumerate(qs) if n * group <= 64]
    for hints in ({}, dict(max_q=max(qs), max_kv=max(kvs)), dict(max_q=1000), dict(max_q=1)):
        y = c.run(scale=1.0 / dim, **hints)
        c.check_two_terms(y, only=few)
        c.check(y, scale=1.0 / dim)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_weights_of_few_rows_beside_a_prompt(fmt):
    """Decoding sequences in one call with a prompt, which may round its weights to one term."""
    c = Cancelling(fmt, 128, 2, 4, 16, [1, 200, 16, 1], [50, 300, 41, 640], seed=3)
    y = c.run(scale=1.0 / 128)
    c.check_two_terms(y, only=(0, 2, 3))
    c.check(y, scale=1.0 / 128)


# ---------------------------------------------------------------- alignment

@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("dim,qs,kvs", [(128, [1, 3], [40, 300]), (64, [1], [9000]),
                                        (256, [2], [5000]), (128, [100, 2], [300, 7]),
                                        (192, [120], [6000])])
def test_queries_and_outputs_at_any_element(fmt, dim, qs, kvs):
    """Both kernels, keys whole and divided: q and out at odd elements give the same bits, and
    nothing around out is written."""
    c = Case(fmt, dim, 2, 2, 16, qs, kvs, seed=31)
    T, n = sum(qs), sum(qs) * 4 * dim
    say(f"any element {fmt} {dim} {qs} {kvs}")
    want = c.run()
    for off in (1, 2, 3):
        flat = torch.zeros(n + 8, dtype=torch.bfloat16, device="cuda")
        q = flat[off:off + n].view(T, 4, dim)
        q.copy_(c.q)
        guard = torch.full((n + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
        c.run(q=q, out=guard[off:off + n].view(T, 4, dim))
        assert torch.equal(guard[off:off + n].view(T, 4, dim), want)
        assert (guard[:off] == 7).all() and (guard[off + n:] == 7).all()


# ---------------------------------------------------------------- divided keys

def _expect(c, lens, y, queries=1):
    """Outputs of sequences cut to `lens` tokens against the 64-bit form, within 2^-7 of the weighted
    mean of |v| (the rounding of weights and output)."""
    y, q = f64(y), f64(c.q)
    starts = np.cumsum([0] + list(c.kvs))
    for b, n in enumerate(lens):
        kv = c.values[starts[b]:starts[b] + n]
        rows = slice(b * queries, (b + 1) * queries)
        for h in range(c.heads * c.group):
            want, mag = attention(q[rows, h], kv[:, 0, h // c.group], kv[:, 1, h // c.group],
                                  c.dim ** -0.5, True)
            assert (np.abs(y[rows, h] - want) <= mag * 2.0 ** -7 + 1e-30).all(), (lens, b, h)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("queries", [1, 40])
def test_graph_of_a_step_with_divided_keys(fmt, queries):
    """One captured call whose keys are divided among workgroups, replayed with lengths that grow
    past shares' ends, shrink and vanish; every replay as the eager call, over a workspace of NaN."""
    lens0 = [3000, 700, 150]
    c = Case(fmt, 128, 2, 4, 64, [queries] * 3, lens0, seed=41)
    table, lens, q = c.table.cuda(), c.kv_lens.clone(), c.q.cuda()
    bound = c.table.shape[1] * 64
    n = w8a8.load_library().w8a8_kv_attention_workspace_bytes(
        64, 2, 128, w8a8.KV_FORMATS[fmt], 4, 3 * queries, 3, queries, bound)
    assert n > 0
    work = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)

    def step(o=None, w=None):
        return w8a8.kv_attention(q, c.cache, table, lens, fmt=fmt, out=o, workspace=w)

    step(out, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, work)
    for now in (lens0, [130, 0, 1], [256, 257, 150], [2999, 700, 127], [1025, 513, 0], [0, 0, 0],
                [3000, 1, 129]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        work.fill_(0xFF)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step())
        _expect(c, now, got, queries)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("qs,kvs,nan_at", [([1], [5000], 4990), ([1], [5000], 100),
                                           ([150], [6000], 5900), ([150], [6000], 640)])
def test_nan_tokens_where_keys_are_divided(fmt, qs, kvs, nan_at):
    lib = w8a8.load_library()
    for part in (0, 1):
        c = Case(fmt, 128, 1, 2, 16, qs, kvs, seed=43)
        assert lib.w8a8_kv_attention_workspace_bytes(16, 1, 128, w8a8.KV_FORMATS[fmt], 2, qs[0], 1,
                                                     qs[0], kvs[0]) > 0
        kv = _kv(kvs[0], 1, 128, 44)
        kv[nan_at, part, 0, 70] = float("nan")
        c.write(kv, _slots(c))
        y = f64(c.run(max_q=qs[0], max_kv=kvs[0]))
        sees = np.array([kvs[0] - qs[0] + i >= nan_at for i in range(qs[0])])
        bad = np.zeros(y.shape, bool)
        bad[sees] = True
        if part == 1:                      # a value's block, not the others of its token
            bad[:, :, :64], bad[:, :, 96:] = False, False
        assert np.array_equal(np.isnan(y), bad)
