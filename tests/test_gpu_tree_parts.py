"""Tree attention whose keys are divided among workgroups: the parts' place in the workspace, and
keys that stay whole over several chunks of page places (4096 tokens), at every number of channels."""
import random

import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from _lm_ref import tree_visible
from _mx_ref import f64
from test_gpu_kv import _kv
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


LONG = [
    # heads, group, nodes, tokens: a row tile of 128 rows beside one of up to 64, and in the second some
    # sequences without either
    (1, 1, [180], [9001]),
    (1, 2, [40, 3, 70], [9100, 4097, 8200]),
]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("case", range(len(LONG)))
def test_long_keys_at_every_width(fmt, dim, case):
    """Keys divided into more parts than one group of lanes joins, and whole, which is three chunks."""
    heads, group, nodes, kvs = LONG[case]
    say(f"long {fmt} {dim} {LONG[case]}")
    c = Tree(fmt, dim, heads, group, 48, nodes, kvs, seed=dim + case)
    for max_kv in (max(kvs), 512):
        assert (_size(c, sum(nodes), len(nodes), max(nodes), max_kv) > 0) == (max_kv > 512)
        y = c.run(max_q=max(nodes), max_kv=max_kv)
        c.check(y)
        assert torch.equal(y, c.run(max_q=max(nodes), max_kv=max_kv))


@pytest.mark.parametrize("dim", [128, 192, 256])
@pytest.mark.parametrize("at", [20, 5000, 8500, 8900, -130])
def test_nan_in_long_keys(dim, at):
    """A NaN key and value in the first, second and third chunk, which every row sees, and in a node (the tree
    begins at 8861): in those who see it, the value's block alone."""
    nodes, kv = 140, 9001
    j = at % kv
    for part in (0, 1):
        c = Tree("fp8", dim, 1, 1, 16, [nodes], [kv], seed=dim)
        new = _kv(kv, 1, dim, 8)
        new[j, part, 0, 40] = float("nan")
        pages = c.table[0].tolist()
        c.write(new, [pages[i // 16] * 16 + i % 16 for i in range(kv)])
        see = tree_visible(c.bits, nodes, kv)
        bad = np.zeros((nodes, 1, dim), bool)
        bad[see[:, j]] = True
        if part == 1:
            bad[:, :, :32], bad[:, :, 64:] = False, False
        assert see[:, j].any() and see[:, j].all() == (j < kv - nodes)
        for max_kv in (kv, 512):
            assert np.array_equal(np.isnan(f64(c.run(max_kv=max_kv))), bad)


@pytest.mark.parametrize("dim,T", [(128, 9), (128, 500), (128, 9000), (256, 5000)])
def test_few_rows_in_a_call_laid_out_for_many(dim, T):
    """Three sequences of up to 4 nodes in T rows: those behind them are left as they were, whichever
    kernel runs."""
    c = Tree("fp8", dim, 2, 4, 16, [4, 1, 4], [5000, 1700, 3], seed=5)
    width = c.table.shape[1] * 16
    assert 0 < _size(c, T, 3, 4, width) <= 1 << 27
    q = torch.full((T, 8, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    q[:9] = c.q.cuda()
    c.tree = torch.cat((c.tree, torch.full((T - 9, 1), -1, device="cuda")))
    out = torch.full_like(q, 7.0)
    for bounds in ({"max_q": 4}, {"max_q": 4, "max_kv": 512}, {"max_q": 1}, {}):
        out[:9] = 7.0
        c.run(q=q, out=out, **bounds)
        c.check(out[:9])
        assert (out[9:] == 7).all()
