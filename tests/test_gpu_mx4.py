"""The microscaled 4-bit quantizer, product and linear against plain 64-bit forms."""
import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from _mx_ref import E2M1, f64, matrix_values, pack_matrix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _x(R, K, seed=0, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, K, generator=g) * torch.exp(spread * torch.randn(R, K, generator=g))
    return x.to(torch.bfloat16)


def _check_codes(x, q, s):
    cq, cs = pack_matrix(f64(x))
    assert np.array_equal(s.cpu().numpy(), cs)
    assert np.array_equal(q.cpu().numpy(), cq)


@pytest.mark.parametrize("R", [1, 3, 16, 33])
@pytest.mark.parametrize("K", [1, 7, 31, 32, 33, 255, 256, 257, 511, 513, 1000, 4096])
def test_codes_and_values(R, K):
    x = _x(R, K, R * 7 + K, 2.0)
    q, s = w8a8.mx4_quantize(x.cuda())
    _check_codes(x, q, s)
    y = w8a8.mx4_dequantize(q, s, K)
    assert np.array_equal(f64(y), matrix_values(q.cpu().numpy(), s.cpu().numpy(), K))


def test_every_bf16_value():
    """All finite bf16 values: each as the largest of its block, and below a larger one."""
    bits = torch.arange(0x7F80, dtype=torch.int32)
    v = torch.cat((bits, bits | 0x8000)).to(torch.int16).view(torch.bfloat16)
    for factor in (0, 2, 64):
        x = torch.zeros(v.numel(), 32, dtype=torch.bfloat16)
        x[:, 3] = v
        big = (v.float().abs() * factor).clamp(max=3e38).to(torch.bfloat16)
        x[:, 11] = big
        q, s = w8a8.mx4_quantize(x.cuda())
        _check_codes(x, q, s)


def test_non_finite_blocks():
    x = _x(5, 200, 3)
    x[0, 5], x[1, 40], x[2, 199], x[4, 64] = float("inf"), float("nan"), -float("inf"), -float("nan")
    q, s = w8a8.mx4_quantize(x.cuda())
    _check_codes(x, q, s)
    y = f64(w8a8.mx4_dequantize(q, s, 200))
    bad = np.zeros((5, 200), bool)
    bad[0, :32], bad[1, 32:64], bad[2, 192:], bad[4, 64:96] = True, True, True, True
    assert np.array_equal(np.isnan(y), bad)
    # such blocks reach the rows and channels they belong to, and no others
    w = _x(9, 200, 4)
    w[7, 100] = float("nan")
    wq, ws = w8a8.mx4_quantize(w.cuda())
    y = f64(w8a8.mx4_gemm(q, s, wq, ws))
    want = np.zeros((5, 9), bool)
    want[[0, 1, 2, 4], :], want[:, 7] = True, True
    assert np.array_equal(np.isnan(y), want) and not np.isinf(y).any()


def test_unaligned_rows():
    base = _x(1, 40 * 77 + 3, 5).flatten().cuda()
    for off in (1, 2, 3):
        x = base[off:off + 40 * 77].view(40, 77)
        q, s = w8a8.mx4_quantize(x)
        _check_codes(x, q, s)


def _gelu64(x):
    import scipy.special
    return x * scipy.special.ndtr(x)


@pytest.mark.parametrize("act,smooth", [("gelu", False), ("none", True), ("gelu", True)])
@pytest.mark.parametrize("R,K", [(1, 300), (37, 1000), (300, 512), (64, 4096)])
def test_transformed_values(act, smooth, R, K):
    """Each element within half a step of the grid from the 64-bit value of its transform, with
    the float32 evaluation's relative error of 1e-5 on top (GELU's far tail; 3e-7 elsewhere) and
    the scale of that value's block or, where it lies that near a power of two, its
    neighbour."""
    x = _x(R, K, K + R)
    cm = torch.rand(K, generator=torch.Generator().manual_seed(1)) * 4 + 0.1 if smooth else None
    q, s = w8a8.mx4_quantize(x.cuda(), act=act, col_mul=None if cm is None else cm.cuda())
    got = matrix_values(q.cpu().numpy(), s.cpu().numpy(), K)
    v = _gelu64(f64(x)) if act == "gelu" else f64(x)
    if smooth:
        v = v * cm.double().numpy()
    full = np.zeros((R, -(-K // 32) * 32))
    full[:, :K] = v
    amax = np.abs(full.reshape(R, -1, 32)).max(-1)
    lo, hi = (np.floor(np.log2(np.maximum(amax * f, 2.0 ** -125))) - 2 for f in (1 - 1e-5, 1 + 1e-5))
    sb = s.cpu().numpy().transpose(1, 0, 2).reshape(R, -1)[:, :amax.shape[1]].astype(int) - 127
    ok = (sb >= np.maximum(lo, -127)) & (sb <= np.maximum(hi, -127))
    assert ok[amax > 2.0 ** -125].all()
    step = np.repeat(2.0 ** sb, 32, 1)[:, :K]
    a = np.abs(v) / step
    half = np.where(a < 2, 0.25, np.where(a < 4, 0.5, 1.0)) * step
    over = np.maximum(a - 7, 0) * step       # saturated: 6 stands for up to 8 scales
    assert (np.abs(got - v) <= half * (1 + 1e-4) + over + 1e-5 * np.abs(v)).all()


def _bound(x, w, b):
    """64-bit product and how far a float32 accumulation rounded to bf16 may be from it: a
    relative 2^-8 for the rounding, and 2^-23 per term of sum |x w|."""
    y, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    if b is not None:
        y, mag = y + b, mag + np.abs(b)
    return y, np.abs(y) * 2.0 ** -8 + mag * (x.shape[1] + 8) * 2.0 ** -23 + 1e-37


SHAPES = [(1, 1, 1), (1, 16, 32), (2, 33, 100), (3, 128, 256), (16, 257, 520), (17, 64, 96),
          (31, 100, 2048), (33, 130, 1000), (64, 64, 64), (65, 300, 4096), (77, 512, 544),
          (128, 128, 288), (129, 255, 257), (200, 1001, 800), (256, 256, 256), (257, 640, 1024),
          (300, 513, 2080), (520, 768, 1536), (1, 4096, 8192), (5, 2000, 5000), (40, 96, 16384),
          (700, 1100, 40), (1, 5, 20000), (2100, 4200, 520), (5000, 1999, 96)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product_and_linear(M, N, K):
    x, w = _x(M, K, 1, 0.5), _x(N, K, 2, 0.5)
    b = _x(1, N, 3)[0]
    wq, ws = w8a8.mx4_quantize(w.cuda())
    xq, xs = w8a8.mx4_quantize(x.cuda())
    xv = matrix_values(*(t.cpu().numpy() for t in (xq, xs)), K)
    wv = matrix_values(*(t.cpu().numpy() for t in (wq, ws)), K)
    say(f"mx4 {M} x {N} x {K}")
    for bias in (b, None):
        want, tol = _bound(xv, wv, None if bias is None else f64(bias))
        bd = None if bias is None else bias.cuda()
        for y in (w8a8.mx4_gemm(xq, xs, wq, ws, bd), w8a8.mx4_linear(x.cuda(), wq, ws, bd)):
            err = np.abs(f64(y) - want)
            assert (err <= tol).all(), (err / tol).max()


# Either side of the streaming kernel's limits: 16 and 32 tokens, 4096 and 8192 channels, and
# of the sizes up to which the linear is one launch.
@pytest.mark.parametrize("M,N,K", [(1, 8193, 520), (2, 9000, 4096), (3, 8200, 4096), (16, 8192, 33),
                                   (12, 5001, 1100), (16, 4097, 1024), (17, 4096, 4096), (32, 4000, 600),
                                   (25, 4097, 300), (20, 600, 4128), (33, 4096, 512), (16, 8208, 300)])
def test_few_tokens(M, N, K):
    test_product_and_linear(M, N, K)


@pytest.mark.parametrize("M", [3, 40, 300])
def test_linear_with_transforms_is_quantizer_and_product(M):
    N, K = 200, 1000
    x, w = _x(M, K, 5).cuda(), _x(N, K, 6, 0.3).cuda()
    cm = (torch.rand(K) + 0.5).cuda()
    wq, ws = w8a8.mx4_quantize(w, col_mul=1 / cm)
    for act in ("none", "gelu"):
        for c in (None, cm):
            xq, xs = w8a8.mx4_quantize(x, act=act, col_mul=c)
            xv = matrix_values(*(t.cpu().numpy() for t in (xq, xs)), K)
            wv = matrix_values(*(t.cpu().numpy() for t in (wq, ws)), K)
            want, tol = _bound(xv, wv, None)
            y = w8a8.mx4_linear(x, wq, ws, act=act, col_mul=c)
            assert (np.abs(f64(y) - want) <= tol).all()


def test_empty_sizes():
    e = torch.empty(0, 96, dtype=torch.bfloat16, device="cuda")
    q, s = w8a8.mx4_quantize(e)
    assert q.shape == (0, 48) and s.shape == (1, 0, 8)
    wq, ws = w8a8.mx4_quantize(_x(5, 96).cuda())
    assert w8a8.mx4_linear(e, wq, ws).shape == (0, 5)
    b = _x(1, 5)[0].cuda()
    z = torch.empty(3, 0, dtype=torch.bfloat16, device="cuda")
    zq, zs = w8a8.mx4_quantize(torch.empty(5, 0, dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(w8a8.mx4_linear(z, zq, zs, b), b.expand(3, 5))


@pytest.mark.parametrize("M,N,K", [(3, 100, 512), (70, 300, 4096), (300, 260, 2048)])
def test_out_workspace_stream_and_repeats(M, N, K):
    """Caller's buffers with what lies around them, another stream, the same bits each time."""
    x, w = _x(M, K, 8).cuda(), _x(N, K, 9).cuda()
    wq, ws = w8a8.mx4_quantize(w)
    want = w8a8.mx4_linear(x, wq, ws)
    guard = torch.full((M + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
    n = w8a8.load_library().w8a8_mx4_linear_workspace_bytes(M, N, K)
    work = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(4):
            y = w8a8.mx4_linear(x, wq, ws, out=guard[1:-1], workspace=work[:n])
    torch.cuda.current_stream().wait_stream(side)
    assert y.data_ptr() == guard[1].data_ptr() and torch.equal(y, want)
    assert (guard[0] == 7).all() and (guard[-1] == 7).all() and (work[n:] == 0xA5).all()
    if n > 0:
        with pytest.raises(ValueError):
            w8a8.mx4_linear(x, wq, ws, workspace=work[:n - 1])


def test_graph_replays():
    M, N, K = 64, 512, 4096
    x, w = _x(M, K, 10).cuda(), _x(N, K, 11).cuda()
    wq, ws = w8a8.mx4_quantize(w)
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    work = torch.empty(w8a8.load_library().w8a8_mx4_linear_workspace_bytes(M, N, K),
                       dtype=torch.uint8, device="cuda")
    w8a8.mx4_linear(x, wq, ws, out=out, workspace=work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w8a8.mx4_linear(x, wq, ws, out=out, workspace=work)
    for i in range(3):
        x.copy_(_x(M, K, 20 + i))
        want = w8a8.mx4_linear(x, wq, ws)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_grid_order():
    """The elements' codes run through the grid in order, low half first."""
    x = torch.zeros(1, 32, dtype=torch.bfloat16)
    x[0, :8] = torch.tensor(E2M1)
    x[0, 8:16] = -torch.tensor(E2M1)
    q, s = w8a8.mx4_quantize(x.cuda())
    assert q[0, :8].tolist() == [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE]
    assert s.flatten().tolist() == [127, 0, 0, 0, 0, 0, 0, 0]
