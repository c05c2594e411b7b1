"""The quantized cache and the attention over it at the ends of their ranges."""
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from test_gpu_kv import _kv

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
