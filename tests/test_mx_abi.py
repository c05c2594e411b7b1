"""The microscaled entry points without a GPU: what they refuse, before any launch."""
import ctypes

import pytest
import torch

import paper_2606_14598_amd as w8a8

P = ctypes.c_void_p
F, ODD = P(256), P(264)      # never dereferenced: validation fails first
OK, NULL, SHAPE, KOVER, WORK, ARG = 0, 1, 2, 3, 5, 6


@pytest.fixture(scope="module")
def lib():
    return w8a8.load_library()


def test_quantizer_refusals(lib):
    q, d = lib.w8a8_mx4_quantize, lib.w8a8_mx4_dequantize
    assert q(F, 4, 64, 2, None, F, F, None) == ARG
    assert q(F, -1, 64, 0, None, F, F, None) == SHAPE and d(F, F, 4, -1, F, None) == SHAPE
    assert q(F, 4, (1 << 22) + 1, 0, None, F, F, None) == KOVER
    assert q(F, 1 << 62, 1 << 20, 0, None, F, F, None) == SHAPE
    for a in ((None, F, F), (F, None, F), (F, F, None)):
        assert q(a[0], 4, 64, 0, None, a[1], a[2], None) == NULL
        assert d(a[0], a[1], 4, 64, a[2], None) == NULL
    assert q(F, 4, 64, 0, None, ODD, F, None) == ARG and q(F, 4, 64, 0, None, F, ODD, None) == ARG
    assert q(None, 0, 64, 0, None, None, None, None) == OK
    assert d(None, None, 4, 0, None, None) == OK


def test_product_refusals(lib):
    g, l = lib.w8a8_mx4_gemm, lib.w8a8_mx4_linear
    assert g(F, F, F, F, None, F, 4, 4, -1, F, 0, None) == SHAPE
    assert g(F, F, F, F, None, F, 4, 4, (1 << 22) + 1, F, 0, None) == KOVER
    for i in (0, 1, 2, 3, 5):
        a = [F, F, F, F, None, F]
        a[i] = None
        assert g(*a, 4, 4, 64, F, 1 << 30, None) == NULL
    for i in range(4):
        a = [F, F, F, F, None, F]
        a[i] = ODD
        assert g(*a, 4, 4, 64, F, 1 << 30, None) == ARG
    assert g(None, None, None, None, None, None, 0, 4, 64, None, 0, None) == OK
    assert l(F, 7, None, F, F, None, F, 4, 4, 64, F, 1 << 30, None) == ARG
    assert l(F, 0, None, ODD, F, None, F, 4, 4, 64, F, 1 << 30, None) == ARG
    assert l(F, 0, None, F, F, None, None, 4, 4, 64, F, 1 << 30, None) == NULL
    M, N, K = 300, 500, 4096
    need = lib.w8a8_mx4_linear_workspace_bytes(M, N, K)
    assert need >= M * K // 2 + M * K // 32
    for ws, n in ((None, need), (F, need - 1), (P(128), need)):
        assert l(F, 0, None, F, F, None, F, M, N, K, ws, n, None) == WORK
    assert lib.w8a8_mx4_gemm_workspace_bytes(-1, 4, 64) == 0
    assert lib.w8a8_mx4_linear_workspace_bytes(4, 4, 1 << 30) == 0


BAD_CACHES = [(8, 8, 2, 128, 0), (4, 20, 2, 128, 0), (4, 8192, 2, 128, 0), (4, 16, 0, 128, 0),
              (4, 16, 2000, 128, 0), (4, 16, 2, 96, 0), (4, 16, 2, 320, 0), (4, 16, 2, 128, 2),
              (-1, 16, 2, 128, 0)]


def test_cache_refusals(lib):
    w, r = lib.w8a8_kv_write, lib.w8a8_kv_read
    assert lib.w8a8_kv_page_bytes(64, 8, 128, 0) == 2 * 8 * 64 * (128 + 4)
    assert lib.w8a8_kv_page_bytes(16, 1, 64, 1) == 2 * 16 * (32 + 2)
    for c in BAD_CACHES:
        assert w(F, *c, F, 256, 128, F, 256, 128, F, 3, None) == ARG
        assert r(F, *c, F, 3, F, F, None) == ARG
        if c[0] >= 0:
            assert lib.w8a8_kv_page_bytes(*c[1:]) == -1
    c = (4, 16, 2, 128, 0)
    assert w(F, *c, F, 256, 128, F, 256, 128, F, -1, None) == SHAPE
    assert w(F, *c, None, 256, 128, F, 256, 128, F, 3, None) == NULL
    assert w(F, *c, F, 256, 128, F, 256, 128, None, 3, None) == NULL
    assert w(None, *c, F, 256, 128, F, 256, 128, F, 3, None) == NULL
    assert w(ODD, *c, F, 256, 128, F, 256, 128, F, 3, None) == ARG
    assert w(F, *c, F, -256, 128, F, 256, 128, F, 3, None) == ARG
    assert r(F, *c, F, 3, None, F, None) == NULL and r(ODD, *c, F, 3, F, F, None) == ARG
    assert w(None, *c, None, 0, 0, None, 0, 0, None, 0, None) == OK


def test_attention_refusals(lib):
    def call(q=F, q_token=1024, q_head=128, cache=F, shape=(4, 16, 2, 128, 0), table=F, stride=4,
             width=4, lens=F, starts=F, T=6, seqs=3, group=4, scale=0.1, causal=1, max_q=4,
             max_kv=64, out=F, ws=F, n=1 << 40):
        return lib.w8a8_kv_attention(q, q_token, q_head, cache, *shape, table, stride, width, lens,
                                     starts, T, seqs, group, scale, causal, max_q, max_kv, out, ws,
                                     n, None)
    for c in BAD_CACHES:
        assert call(shape=c) == ARG
    for bad in (dict(group=0), dict(causal=2), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(cache=ODD)):
        assert call(**bad) == ARG
    for bad in (dict(T=-1), dict(seqs=-1), dict(width=-1), dict(stride=-1), dict(q_token=-1),
                dict(q_head=-1), dict(max_q=-1), dict(max_kv=-1), dict(seqs=0),
                dict(starts=None, seqs=4), dict(width=1 << 30)):
        assert call(**bad) == SHAPE
    for bad in (dict(q=None), dict(out=None), dict(lens=None), dict(cache=None), dict(table=None)):
        assert call(**bad) == NULL
    assert call(T=0) == OK
    assert lib.w8a8_kv_attention_workspace_bytes(16, 2, 96, 0, 4, 6, 3, 4, 64) == 0


def test_attention_workspace_for_a_bound_of_no_queries(lib):
    """max_q = 0 is a bound like any other: the size that is asked for is the size that the call
    needs."""
    def size(max_q):
        return lib.w8a8_kv_attention_workspace_bytes(64, 8, 128, 0, 4, 48, 48, max_q, 16384)
    need = size(0)
    assert need == size(1) > 0 and size(-1) == 0
    st = lib.w8a8_kv_attention(F, 4096, 128, F, 4, 64, 8, 128, 0, F, 256, 256, F, F, 48, 48, 4, 0.1,
                               1, 0, 16384, F, F, need - 1, None)
    assert st == WORK


def test_binding_refusals():
    bf, u8 = torch.bfloat16, torch.uint8
    x = torch.zeros(4, 64, dtype=bf)
    codes, scales = torch.zeros(4, 32, dtype=u8), torch.zeros(1, 4, 8, dtype=u8)
    with pytest.raises(ValueError, match="HIP device"):
        w8a8.mx4_quantize(x)
    with pytest.raises(TypeError):
        w8a8.mx4_quantize(x.float())
    with pytest.raises(ValueError, match="act"):
        w8a8.mx4_quantize(x, act="relu")
    with pytest.raises(ValueError, match="HIP device"):
        w8a8.mx4_dequantize(codes, scales, 64)
    with pytest.raises(TypeError):
        w8a8.mx4_linear(x.float(), codes, scales)
    with pytest.raises(ValueError):
        w8a8.kv_cache(4, 2, 96, 16, device="cpu")
    with pytest.raises(ValueError):
        w8a8.kv_cache(4, 2, 128, 20, device="cpu")
    with pytest.raises(ValueError, match="fmt"):
        w8a8.kv_cache(4, 2, 128, fmt="int8", device="cpu")
    cache = w8a8.kv_cache(4, 2, 128, 16, device="cpu")
    assert cache.shape == (4, 2, 2, 16 * 132) and cache.dtype == u8
    k = torch.zeros(3, 2, 128, dtype=bf)
    with pytest.raises(ValueError, match="HIP device"):
        w8a8.kv_write(cache, k, k, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(TypeError):
        w8a8.kv_attention(k.float(), cache, torch.zeros(1, 4, dtype=torch.int32),
                          torch.zeros(1, dtype=torch.int32))


@pytest.mark.gpu
def test_binding_refusals_on_device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bf, i32 = torch.bfloat16, torch.int32
    x = torch.zeros(4, 64, dtype=bf, device="cuda")
    q, s = w8a8.mx4_quantize(x)
    q9, s9 = w8a8.mx4_quantize(torch.zeros(9, 96, dtype=bf, device="cuda"))
    with pytest.raises(ValueError, match="contiguous"):
        w8a8.mx4_quantize(x.t())
    with pytest.raises(ValueError, match="no 4-bit matrix"):
        w8a8.mx4_dequantize(q, s9)
    with pytest.raises(ValueError):
        w8a8.mx4_dequantize(q, s, 65)
    for bad in (lambda: w8a8.mx4_gemm(q, s, q9, s9), lambda: w8a8.mx4_linear(x, q9, s9),
                lambda: w8a8.mx4_gemm(q, s, q, s, torch.zeros(5, dtype=bf, device="cuda"))):
        with pytest.raises(ValueError, match="shape mismatch"):
            bad()
    cache = w8a8.kv_cache(4, 2, 128, 16)
    k = torch.zeros(3, 2, 128, dtype=bf, device="cuda")
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError, match="cache"):
        w8a8.kv_write(cache, *2 * [torch.zeros(3, 2, 192, dtype=bf, device="cuda")], slots)
    with pytest.raises(ValueError, match="cache"):
        w8a8.kv_write(cache, k, k, slots, fmt="fp4")
    with pytest.raises(ValueError, match="shape mismatch"):
        w8a8.kv_write(cache, k[:, :1], k[:, :1], slots)
    with pytest.raises(ValueError, match="slots"):
        w8a8.kv_write(cache, k, k, slots[:2])
    with pytest.raises(TypeError):
        w8a8.kv_write(cache, k, k, slots.int())
    with pytest.raises(ValueError, match="last dimension"):
        w8a8.kv_write(cache, k.transpose(1, 2).contiguous().transpose(1, 2), k, slots)
    table, lens = torch.zeros(3, 4, dtype=i32, device="cuda"), torch.zeros(3, dtype=i32, device="cuda")
    qq = torch.zeros(3, 8, 128, dtype=bf, device="cuda")
    assert (w8a8.kv_attention(qq, cache, table, lens) == 0).all()
    for bad in (dict(q=qq[:2]), dict(q=qq[:, :7]), dict(block_table=table[:2]),
                dict(block_table=table.t()), dict(q_starts=lens), dict(out=qq[:2].clone())):
        with pytest.raises((ValueError, TypeError)):
            w8a8.kv_attention(**{**dict(q=qq, cache=cache, block_table=table, kv_lens=lens), **bad})
    with pytest.raises(TypeError):
        w8a8.kv_attention(qq, cache, table.long(), lens)
