"""The norm that quantizes for the next linear, code by code against its definition."""
import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from _lm_ref import f32_inverse_rms, int8_rows, norm_values
from _mx_ref import f64, pack_matrix

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _inputs(M, K, seed, residual, weight):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g)
    if K > 20:
        x[:, 17] *= 40.0
    r = (3.0 * torch.randn(M, K, generator=g)).to(torch.bfloat16) if residual else None
    w = torch.exp(0.3 * torch.randn(K, generator=g)) if weight else None
    return x.to(torch.bfloat16), r, w


def _dev(t):
    return None if t is None else t.cuda()


def check(out, x, r, w, fmt, eps=EPS):
    """Codes, scales and sum equal to the definition's, but for rows whose 64-bit root lies on a
    border (f32_inverse_rms says which: none of the inputs here, so all are compared)."""
    codes, scales, h = out
    hv = x if r is None else (x.float() + r.float()).to(torch.bfloat16)
    assert torch.equal(h.cpu(), hv)
    rms, near = f32_inverse_rms(f64(hv), eps)
    v = norm_values(f64(hv), rms, None if w is None else w.numpy())
    ok = ~near
    assert ok.mean() > 0.99
    if fmt == "int8":
        q, s = int8_rows(v)
        assert np.array_equal(scales.cpu().numpy()[ok], s[ok])
    else:
        q, s = pack_matrix(v.astype(np.float64))
        assert np.array_equal(scales.cpu().numpy()[:, ok], s[:, ok])
    assert np.array_equal(codes.cpu().numpy()[ok], q[ok])


# K around what a wavefront, a workgroup and a row in registers hold; odd ones; rows that are looped
SIZES = [(1, 1), (3, 7), (5, 8), (2, 31), (33, 64), (5, 200), (3, 255), (4, 256), (5, 257), (7, 512),
         (9, 520), (3, 1000), (5, 1024), (6, 1027), (5, 2048), (3, 2056), (2, 4096), (3, 4097),
         (2, 7696), (3, 8200), (2, 16384), (2, 16500), (1, 24577), (2, 32768), (2, 32776), (1, 50001)]


@pytest.mark.parametrize("fmt", ["int8", "mx4"])
@pytest.mark.parametrize("M,K", SIZES)
def test_codes(fmt, M, K):
    say(f"norm {fmt} {M} x {K}")
    for residual, weight in ((True, True), (False, True), (True, False)):
        x, r, w = _inputs(M, K, M * 1000 + K, residual, weight)
        check(w8a8.rms_norm_quantize(_dev(x), _dev(w), residual=_dev(r), eps=EPS, fmt=fmt), x, r, w, fmt)


@pytest.mark.parametrize("fmt", ["int8", "mx4"])
def test_many_rows(fmt):
    """More rows than the grid takes at once."""
    for M, K in ((9001, 64), (5000, 264)):
        x, r, w = _inputs(M, K, M, True, True)
        check(w8a8.rms_norm_quantize(_dev(x), _dev(w), residual=_dev(r), eps=EPS, fmt=fmt), x, r, w, fmt)


@pytest.mark.parametrize("fmt", ["int8", "mx4"])
def test_extreme_rows(fmt):
    """Rows of zeros, of the smallest and of the largest values; a large eps."""
    x, _, w = _inputs(6, 512, 1, False, True)
    x[1] = 0.0
    x[2] = (x[2].float() * 1e-38).to(torch.bfloat16)
    x[3] = (x[3].float().clamp(-3, 3) * 1e38).to(torch.bfloat16)
    x[4, 1:] = 0.0
    x[5] = -x[5].abs()
    for eps in (1e-6, 1e-30, 2.0):
        check(w8a8.rms_norm_quantize(x.cuda(), w.cuda(), eps=eps, fmt=fmt), x, None, w, fmt, eps)


def test_fits_the_quantizers():
    """Rows whose norm is 1 and weights of 1 leave the values: the codes of quantize_act and
    mx4_quantize."""
    x = torch.where(torch.rand(40, 1024, generator=torch.Generator().manual_seed(0)) < 0.5, 1.0, -1.0)
    x = x.to(torch.bfloat16).cuda()
    for fmt, f in (("int8", w8a8.quantize_act), ("mx4", w8a8.mx4_quantize)):
        q, s, h = w8a8.rms_norm_quantize(x, eps=1e-30, fmt=fmt)
        want = f(x)
        assert h is x and torch.equal(q, want[0]) and torch.equal(s, want[1])


def test_non_finite_blocks():
    """In 4 bits: a NaN in h takes its row, an infinity its block (r is zero), a weight its block."""
    x, r, w = _inputs(4, 512, 2, True, True)
    x[1, 40], x[2, 70] = float("nan"), float("inf")
    w[200] = float("nan")
    q, s, h = w8a8.rms_norm_quantize(x.cuda(), w.cuda(), residual=r.cuda(), fmt="mx4")
    y = f64(w8a8.mx4_dequantize(q, s, 512))
    bad = np.zeros((4, 512), bool)
    bad[1] = True
    bad[2, 64:96] = True
    bad[:, 192:224] = True
    assert np.array_equal(np.isnan(y), bad)
    assert (y[2][~bad[2]] == 0).all()


@pytest.mark.parametrize("fmt", ["int8", "mx4"])
@pytest.mark.parametrize("K", [512, 4096, 33000])
def test_unaligned_operands(fmt, K):
    x, r, w = _inputs(3, K, K, True, True)
    wide = torch.zeros(3, 3 * K + 16, dtype=torch.bfloat16, device="cuda")
    ww = torch.zeros(K + 8, device="cuda")
    for off in (1, 4):
        flat = wide.view(-1)
        xd, rd, sd = (flat[off + i * 3 * K:off + (i + 1) * 3 * K].view(3, K) for i in range(3))
        xd.copy_(x), rd.copy_(r), ww[off:off + K].copy_(w)
        out = w8a8.rms_norm_quantize(xd, ww[off:off + K], residual=rd, fmt=fmt, sum_out=sd)
        check(out, x, r, w, fmt)
        assert out[2].data_ptr() == sd.data_ptr()


@pytest.mark.parametrize("K", [200, 1000, 4096, 40000])
def test_sum_in_place(K):
    for which in (0, 1):
        x, r, w = _inputs(5, K, K + which, True, True)
        xd, rd = x.cuda(), r.cuda()
        out = w8a8.rms_norm_quantize(xd, w.cuda(), residual=rd, sum_out=(xd, rd)[which])
        check(out, x, r, w, "int8")
        assert torch.equal((rd, xd)[which].cpu(), (r, x)[which])


def test_empty_sizes():
    for fmt in ("int8", "mx4"):
        q, s, h = w8a8.rms_norm_quantize(torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"), fmt=fmt)
        assert q.shape[0] == 0
        x = torch.zeros(3, 0, dtype=torch.bfloat16, device="cuda")
        q, s, h = w8a8.rms_norm_quantize(x, residual=x, fmt=fmt)
        assert q.shape == (3, 0) and (s == 0).all()


def test_offsets_beyond_32_bits():
    M, K = 530000, 4096
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    part = torch.randn(100, K, device="cuda").to(torch.bfloat16)
    x[-100:] = part
    w = torch.rand(K, device="cuda") + 0.5
    for fmt in ("int8", "mx4"):
        q, s, _ = w8a8.rms_norm_quantize(x, w, fmt=fmt)
        q2, s2, _ = w8a8.rms_norm_quantize(part, w, fmt=fmt)
        assert torch.equal(q[-100:], q2)
        assert torch.equal(s[-100:], s2) if fmt == "int8" else torch.equal(s[:, -100:], s2)
    del x, q
    torch.cuda.empty_cache()


def test_stream_graph_and_linear():
    """Captured with the product behind it, replayed on other inputs, against the eager calls."""
    K, N = 1000, 512
    g = torch.Generator().manual_seed(3)
    wq, sw = w8a8.quantize_weight(torch.randn(N, K, generator=g).to(torch.bfloat16).cuda())
    w = (torch.rand(K, generator=g) + 0.5).cuda()
    x = torch.empty(5, K, dtype=torch.bfloat16, device="cuda")
    r = torch.empty_like(x)

    def step():
        q, s, h = w8a8.rms_norm_quantize(x, w, residual=r)
        return w8a8.gemm(q, s, wq, sw), h

    def inputs(i):
        for t in (x, r):
            t.copy_(torch.randn(5, K, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16))

    inputs(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, step()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(1, 4):
        inputs(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_binding_refusals():
    x = torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, device="cuda")
    for bad in (dict(weight=w[:63]), dict(residual=x[:2]), dict(sum_out=x), dict(fmt="e4m3"),
                dict(residual=x, sum_out=x[:2]), dict(weight=w.cpu())):
        with pytest.raises(ValueError):
            w8a8.rms_norm_quantize(x, bad.pop("weight", w), **bad)
    for bad in (dict(weight=w.to(torch.bfloat16)), dict(residual=x.float())):
        with pytest.raises(TypeError):
            w8a8.rms_norm_quantize(x, bad.pop("weight", w), **bad)
    with pytest.raises(ValueError):
        w8a8.rms_norm_quantize(x.t(), None)
    with pytest.raises(w8a8.W8A8Error):
        w8a8.rms_norm_quantize(x, w, eps=0.0)
