"""Tree attention whose keys are divided among workgroups: the parts' place in the workspace."""
import random

import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from test_gpu_tree import Tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _size(c, T, seqs, max_q, max_kv):
    return w8a8.load_library().w8a8_kv_tree_attention_workspace_bytes(
        c.page, c.heads, c.dim, w8a8.KV_FORMATS[c.fmt], c.group, T, seqs, max_q, max_kv)


def test_most_parts_and_a_workspace_in_turn():
    """As many parts as there can be (682 row tiles of 682.7 / 682 shares each: two parts), few divided
    sequences among many that are whole, and the reverse: in one workspace of the largest of their
    sizes, one after the other, so that each finds the parts and notes of the one before."""
    g = random.Random(1)
    calls = [([3] * 341, [600] * 341),
             ([g.randint(1, 9) for _ in range(300)], [4000 if i % 50 == 7 else g.randint(9, 120) for i in range(300)]),
             ([g.randint(1, 20) for _ in range(60)], [90 if i % 9 == 3 else g.randint(600, 2500) for i in range(60)]),
             ([33, 1, 2], [9, 5000, 130])]
    cases = [Tree("fp8", 64, 2, 8, 16, nodes, kvs, seed=i) for i, (nodes, kvs) in enumerate(calls)]
    sizes = [_size(c, sum(c.qs), len(c.qs), max(c.qs), max(c.kvs)) for c in cases]
    assert all(n > 0 for n in sizes)
    n = max(sizes)
    work = torch.full((n + 4096,), 0x7F, dtype=torch.uint8, device="cuda")
    for i in (0, 1, 2, 3, 1, 0, 3, 2):
        say(f"call {i}: {len(cases[i].qs)} sequences")
        c = cases[i]
        c.check(c.run(max_q=max(c.qs), max_kv=max(c.kvs), workspace=work[:n]))
        assert (work[n:] == 0x7F).all()
