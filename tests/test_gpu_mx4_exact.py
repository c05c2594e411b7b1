"""The 4-bit product where float32 sums are exact: every channel counts, to the last block."""
import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from _mx_ref import matrix_values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _codes(R, K, seed):
    """Random elements in blocks of scales 1/2, 1 and 2, each with a 4 or 6 in it, as the quantizer
    would have made them; (codes, scales) on the CPU."""
    rng = np.random.default_rng(seed)
    nb = -(-K // 32)
    c = rng.integers(0, 16, (R, nb * 32), dtype=np.uint8)
    c[:, ::32] = rng.choice([6, 7, 14, 15], (R, nb)).astype(np.uint8)
    c[:, K:] = 0
    s = np.zeros((-(-K // 256), R, 8), np.uint8)
    for b in range(nb):
        s[b // 8, :, b % 8] = rng.integers(126, 129, R)
    return c[:, 0::2] | c[:, 1::2] << 4, s


# Products of elements and scales are multiples of 2^-4, up to 144; sums of K of them, in any
# order, stay whole multiples below 2^20 here, so float32 holds them all exactly and the output is
# the exact sum rounded to bf16 once.
@pytest.mark.parametrize("M,N,K", [(1, 5, 20000), (1, 70, 8225), (2, 9000, 4128), (16, 40, 1000),
                                   (16, 100, 8224), (17, 300, 4065), (32, 4096, 4096), (40, 96, 16416),
                                   (65, 300, 8480), (129, 257, 2080), (300, 130, 20001),
                                   (700, 1030, 4128), (2100, 600, 545), (520, 2000, 1001)])
def test_every_channel_counts(M, N, K):
    say(f"mx4 exact {M} x {N} x {K}")
    x, w = _codes(M, K, M + K), _codes(N, K, N + 7 * K)
    xv, wv = matrix_values(*x, K), matrix_values(*w, K)
    total = xv @ wv.T
    assert np.abs(xv).sum(1).max() * np.abs(wv).max() < 2.0 ** 20
    want = torch.from_numpy(total).float().to(torch.bfloat16)      # exact in float32
    assert np.array_equal(total, total.astype(np.float32))
    d = [torch.from_numpy(t).cuda() for t in (*x, *w)]
    assert torch.equal(w8a8.mx4_gemm(*d).cpu(), want)
    xb = torch.from_numpy(xv).to(torch.bfloat16).cuda()            # quantizes to the same codes
    assert torch.equal(w8a8.mx4_linear(xb, d[2], d[3]).cpu(), want)
