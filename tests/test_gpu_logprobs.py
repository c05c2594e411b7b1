"""Log probabilities, entropy and alternatives of rows of logits against a plain 64-bit form."""
import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from _lm_ref import logprobs
from _mx_ref import f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def check(out, x, tokens, top, temperature=1.0):
    """Ids equal; values within float32 arithmetic. With y = (x - m) / temperature in powers of two
    (a difference, a factor rounded twice, a product: 2^-24 of |y| each), 2^y and the logarithm are
    2^-22 off at most, a lane adds V / 256 + 8 values one after the other and 16 more joins follow:
      log p   2^-24 (4 |y| + n + 16) with n the additions
      H       log s - t / s, whose terms are y p: 2^-24 (4 max|y| + n + 16) (1 + log s + |t / s|),
    with max|y| over the values that have any weight (|y| < 150; smaller ones are zeros)."""
    lp, ent, tl, ti = out
    want = logprobs(x.astype(np.float64), tokens, top, temperature)
    assert np.array_equal(ti.cpu().numpy(), want[3])
    u, n = 2.0 ** -24, x.shape[1] / 256 + 24
    for got, ref in ((lp, want[0]), (tl, want[2])):
        got = f64(got)
        with np.errstate(over="ignore"):       # a value past float32's largest is an infinity in it
            ref = np.where(np.isfinite(ref.astype(np.float32)), ref, ref.astype(np.float32))
        with np.errstate(invalid="ignore"):
            ok = np.abs(got - ref) <= u * (4 * np.abs(ref) / np.log(2) + n + 16 + 4 * np.log2(x.shape[1]))
        assert (ok | (got == ref) | (np.isnan(got) & np.isnan(ref))).all(), np.abs(got - ref).max()
    got = f64(ent)
    with np.errstate(invalid="ignore"):
        tol = u * (4 * 150 + n + 16) * (1 + 2 * np.log(x.shape[1]))
        ok = np.abs(got - want[1]) <= tol
    assert (ok | (np.isnan(got) & np.isnan(want[1]))).all(), np.abs(got - want[1]).max()


def _logits(T, V, dtype, seed, masked=False):
    g = torch.Generator().manual_seed(seed)
    x = 2.5 * torch.randn(T, V, generator=g)
    x[torch.arange(T), torch.randint(0, V, (T,), generator=g)] += 9.0
    if masked:
        x[torch.rand(T, V, generator=g) < 0.6] = -torch.inf
        x[:, V // 2] = 1.0
    tokens = torch.randint(0, V, (T,), generator=g)
    if T > 3:
        tokens[1], tokens[2] = -1, V
    return x.to(dtype), tokens


SIZES = [(1, 1, 1), (1, 2, 2), (3, 7, 5), (5, 64, 64), (4, 65, 64), (2, 511, 20), (3, 512, 1), (9, 1000, 7),
         (2, 2048, 0), (2, 4096, 3), (1, 4097, 64), (4, 8192, 20), (3, 8200, 33), (1, 50001, 20),
         (2, 131072, 64), (70, 20001, 5), (600, 3001, 2), (1030, 9001, 5)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,top", SIZES)
def test_rows(dtype, T, V, top):
    say(f"logprobs {dtype} {T} x {V}, {top}")
    for masked, temperature in ((False, 1.0), (True, 0.7)):
        if masked and V < 512:
            continue
        x, t = _logits(T, V, dtype, T + V, masked)
        out = w8a8.token_logprobs(x.cuda(), t.cuda(), top=top, temperature=temperature)
        check(out, f64(x), t.numpy(), top, temperature)
        again = w8a8.token_logprobs(x.cuda(), t.cuda(), top=top, temperature=temperature)
        assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("V", [300, 5000, 70000])
def test_equal_logits(V):
    """Ties go to the lower index: rows of one value, of two, of zeros of both signs."""
    x = torch.zeros(5, V)
    x[1] = -3.0
    x[2, ::3] = 2.0
    x[3, 1::2] = -0.0
    x[4, V - 40:] = 1.0
    t = torch.tensor([0, 1, 2, 3, V - 1])
    for dtype in (BF, F32):
        check(w8a8.token_logprobs(x.to(dtype).cuda(), t.cuda(), top=64), f64(x), t.numpy(), 64)


@pytest.mark.parametrize("V", [700, 9000, 200000])
def test_order_of_the_values(V):
    """Rising, falling and alternating rows: every value, or none, passes those before it."""
    up = torch.arange(V, dtype=torch.float32) * (40.0 / V)
    x = torch.stack((up, up.flip(0), torch.where(torch.arange(V) % 2 == 0, up, -up),
                     up.roll(V // 3))).contiguous()
    t = torch.tensor([V - 1, 0, V // 2, 5])
    for dtype in (F32, BF):
        check(w8a8.token_logprobs(x.to(dtype).cuda(), t.cuda(), top=64), f64(x.to(dtype)), t.numpy(), 64)


def test_extreme_values():
    """Masks of minus infinity and of the types' lowest values, alone and beside others; the largest
    finite ones; rows of one live token; huge differences."""
    V = 6000
    low = torch.finfo(BF).min
    x = torch.zeros(9, V)
    x[0] = low
    x[1], x[1, 4000] = low, 3.0
    x[2], x[2, 77] = -torch.inf, -5.0
    x[3] = 3.38e38
    x[4, ::2] = 3.38e38
    x[5, 100] = 1e30
    x[6] = torch.linspace(-200, 200, V)
    x[7], x[7, 3000:] = low, -torch.inf
    x[8, 0], x[8, 1:] = 0.0, -90.0
    x = x.to(BF)
    t = torch.tensor([1, 4000, 77, 5, 1, 100, V - 1, 2999, 0])
    for dtype in (BF, F32):
        for temperature in (1.0, 0.5, 3.0):
            check(w8a8.token_logprobs(x.to(dtype).cuda(), t.cuda(), top=64, temperature=temperature),
                  f64(x), t.numpy(), 64, temperature)


@pytest.mark.parametrize("T,V", [(4, 40), (4, 30000), (1100, 3000)])
def test_rows_without_numbers(T, V):
    """NaN, plus infinity and rows of minus infinity: NaN, ids inside the row, other rows untouched."""
    x, t = _logits(T, V, BF, 3)
    x[0, V // 2], x[1, V - 1], x[2] = float("nan"), float("inf"), -torch.inf
    t[:3] = torch.tensor([0, V - 1, -1])
    lp, ent, tl, ti = w8a8.token_logprobs(x.cuda(), t.cuda(), top=7)
    assert lp[:2].isnan().all() and ent[:3].isnan().all() and tl[:3].isnan().all() and lp[2] == 0
    assert ((ti >= 0) & (ti < V)).all()
    check([o[3:] for o in (lp, ent, tl, ti)], f64(x[3:]), t[3:].numpy(), 7)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,top", [(2560, 1, 1), (2561, 700, 5), (2563, 5000, 64), (2600, 8192, 0),
                                     (2562, 515, 20)])
def test_many_short_rows(dtype, T, V, top):
    """Enough short rows for one wavefront each, the last workgroup's not all there; some of them masked,
    without numbers, or with a token outside."""
    x, t = _logits(T, V, dtype, T + V)
    if V > 1:
        x[5::7][torch.rand(len(x[5::7]), V, generator=torch.Generator().manual_seed(1)) < 0.6] = -torch.inf
        x[5::7, V // 2] = 1.0
    x[0], x[3, V // 3] = -torch.inf, float("nan")
    out = w8a8.token_logprobs(x.cuda(), t.cuda(), top=top, temperature=0.8)
    lp, ent, tl, ti = (o.cpu() for o in out)
    for r in (0, 3):
        assert lp[r].isnan() and ent[r].isnan() and tl[r].isnan().all() and ((ti[r] >= 0) & (ti[r] < V)).all()
    ok = torch.ones(T, dtype=torch.bool)
    ok[[0, 3]] = False
    check([o[ok] for o in (lp, ent, tl, ti)], f64(x[ok]), t[ok].numpy(), top, 0.8)


@pytest.mark.parametrize("dtype,signalling", [(BF, 0x7F81), (BF, -0x7F), (F32, 0x7F800001)])
@pytest.mark.parametrize("T,V", [(4, 600), (3, 5000), (3, 40000), (2700, 600)])
def test_signalling_nans(dtype, signalling, T, V):
    """Alone, in front of, behind and between the largest values, and everywhere."""
    x, t = _logits(T, V, dtype, 12)
    t[:3] = torch.tensor([1, 2, 3])
    bits = x.view(torch.int16 if dtype == BF else torch.int32)
    bits[0, 37], bits[1, ::2], bits[2] = signalling, signalling, signalling
    out = w8a8.token_logprobs(x.cuda(), t.cuda(), top=9)
    lp, ent, tl, ti = (o.cpu() for o in out)
    assert lp[:3].isnan().all() and ent[:3].isnan().all() and tl[:3].isnan().all()
    assert ((ti >= 0) & (ti < V)).all() and all(len(set(r.tolist())) == 9 for r in ti[:3])
    if T > 3:
        check([o[3:] for o in (lp, ent, tl, ti)], f64(x[3:]), t[3:].numpy(), 9)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides_alignment_and_buffers(dtype):
    """Rows inside padded ones, from any element on; a caller's workspace; another stream."""
    x, t = _logits(5, 20001, dtype, 8)
    want = w8a8.token_logprobs(x.cuda(), t.cuda(), top=9)
    check(want, f64(x), t.numpy(), 9)
    n = w8a8.load_library().w8a8_token_logprobs_workspace_bytes(5, 20001, 9)
    assert n > 0
    work = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    for off in (0, 1, 3):
        wide = torch.full((5, 20032), 50.0, dtype=dtype, device="cuda")
        wide[:, off:off + 20001] = x.cuda()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = w8a8.token_logprobs(wide[:, off:off + 20001], t.cuda(), top=9, workspace=work[:n])
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (work[n:] == 0xA5).all()
    with pytest.raises(ValueError):
        w8a8.token_logprobs(x.cuda(), t.cuda(), top=9, workspace=work[:n - 1])
    same = x[:1].cuda().expand(5, -1)          # one row for all
    got = w8a8.token_logprobs(same, t.cuda(), top=9)
    check(got, f64(x[:1].expand(5, -1)), t.numpy(), 9)


def test_offsets_beyond_32_bits():
    T, V, n = 17000, 131072, 1100
    x = torch.zeros(T, V, dtype=BF, device="cuda")
    x[-n:] = torch.randn(n, V, device="cuda").to(BF)
    t = torch.randint(0, V, (T,), device="cuda")
    whole = w8a8.token_logprobs(x, t, top=3)
    part = w8a8.token_logprobs(x[-n:], t[-n:], top=3)
    assert all(torch.equal(a[-n:], b) for a, b in zip(whole, part))
    del x
    torch.cuda.empty_cache()


def test_empty_calls_and_refusals():
    x, t = _logits(4, 100, BF, 1)
    x, t = x.cuda(), t.cuda()
    out = w8a8.token_logprobs(x[:0], t[:0], top=5)
    assert [tuple(o.shape) for o in out] == [(0,), (0,), (0, 5), (0, 5)]
    for bad in (dict(top=65), dict(top=-1), dict(tokens=t[:3]), dict(tokens=t.cpu()), dict(logits=x.t()),
                dict(logits=x[:, :50], top=51), dict(logits=x[0])):
        with pytest.raises(ValueError):
            w8a8.token_logprobs(bad.pop("logits", x), bad.pop("tokens", t), **bad)
    for bad in (dict(logits=x.half()), dict(tokens=t.int())):
        with pytest.raises(TypeError):
            w8a8.token_logprobs(bad.pop("logits", x), bad.pop("tokens", t), **bad)
    for temperature in (0.0, -1.0, float("nan")):
        with pytest.raises(w8a8.W8A8Error):
            w8a8.token_logprobs(x, t, temperature=temperature)


@pytest.mark.parametrize("T,V", [(3, 40000), (1100, 2000)])
def test_graph_replays(T, V):
    x = torch.empty(T, V, dtype=BF, device="cuda")
    t = torch.empty(T, dtype=torch.int64, device="cuda")

    def inputs(i):
        a, b = _logits(T, V, BF, i)
        x.copy_(a), t.copy_(b)
    inputs(0)
    w8a8.token_logprobs(x, t, top=5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = w8a8.token_logprobs(x, t, top=5)
    for i in range(1, 4):
        inputs(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        assert all(torch.equal(a, b) for a, b in zip(got, w8a8.token_logprobs(x, t, top=5)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,top", [(2560, 12001, 5), (2561, 16384, 20), (2560, 16385, 5), (2559, 16384, 3)])
def test_longest_short_rows(dtype, T, V, top):
    """Rows too long to stay whole where they are few, up to the longest that a wavefront takes, and just
    past that rule in length and number."""
    test_many_short_rows(dtype, T, V, top)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V", [(1100, 16384), (2600, 16384), (2, 70000)])
def test_entropy_behind_a_late_peak(dtype, T, V):
    """Whole logits in powers of two (the temperature is log2 e): 0 first, then one of 19 in each few, then
    -1. Relative to about the largest of them every weight is a power of two and the sums of a lane have at
    most 24 bits, so they are exact; relative to what a lane saw first, the rest is lost beside 19 2^19. With
    log2 s below 16: its ulp 2^-20; up to 20 joins of s and of t (below s), 2^-23 each, 2^-19 together; the
    quotient's and the difference's roundings, 2^-21: in all 2^-18, times ln 2. (A token's logits are
    exact, and an exponent of up to 20 is off by 2^-25 of it where the temperature is no float32.)"""
    temperature = float(np.float32(1.44269504088896341))
    x = torch.full((T, V), -1.0)
    x[:, :4096] = 0.0
    x[:, 4096:6144:8] = 19.0
    t = torch.arange(T) % V
    out = w8a8.token_logprobs(x.to(dtype).cuda(), t.cuda(), top=3, temperature=temperature)
    check(out, f64(x), t.numpy(), 3, temperature)
    want = logprobs(f64(x[:1]), t[:1].numpy(), 3, temperature)[1][0]
    assert np.abs(f64(out[1]) - want).max() <= 2.0 ** -18 * np.log(2), (f64(out[1])[0], want)
