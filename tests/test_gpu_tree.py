"""Attention of drafted trees over the cache against a plain 64-bit form."""
import random

import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _helpers import say
from _lm_ref import bit_words, masked_attention, tree_bits, tree_visible
from _mx_ref import f64
from test_gpu_kv import Case, _kv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


class Tree(Case):
    """A cache and queries, and a tree a sequence: parents at random among the nodes before."""

    def __init__(self, *args, words=None, bits=None, **kw):
        super().__init__(*args, **kw)
        rng = random.Random(kw.get("seed", 0) + 1)
        words = words or -(-max(self.qs) // 64)
        if bits is None:
            bits = np.concatenate([tree_bits([rng.randrange(-1, i) for i in range(n)], words)
                                   for n in self.qs])
        self.bits = bits
        self.tree = torch.from_numpy(bits).cuda()

    def run(self, q=None, **kw):
        kw.setdefault("q_starts", self.q_starts)
        return w8a8.kv_tree_attention(self.q.cuda() if q is None else q, self.cache, self.table.cuda(),
                                      self.kv_lens, self.tree, fmt=self.fmt, **kw)

    def check(self, y, scale=None):
        """With e a weight's rounding (2^-16 of it in two bf16 terms, up to 64 rows; 2^-8 in one) the
        sum of p v is e A off at most, A the weighted mean of |v|, and the sum of p, which is of the
        rounded ones where there is one term, e: (e A + e |o|) <= 2 e A. The output's own rounding is
        2^-8 |o| <= 2^-8 A, and float32 sums of up to 2^14 weights stay below 2^-10 A."""
        scale = self.dim ** -0.5 if scale is None else scale
        y, q = f64(y), f64(self.q)
        assert np.isfinite(y).all()
        at_q = at_k = 0
        for lq, lk in zip(self.qs, self.kvs):
            see = tree_visible(self.bits[at_q:at_q + lq], lq, lk)
            terms = 2.0 ** -8 + 2.0 ** -10 + 2 * (2.0 ** -16 if lq * self.group <= 64 else 2.0 ** -8)
            for h in range(self.heads * self.group):
                kv = self.values[at_k:at_k + lk, :, h // self.group]
                want, mag = masked_attention(q[at_q:at_q + lq, h], kv[:, 0], kv[:, 1], scale, see)
                err = np.abs(y[at_q:at_q + lq, h] - want)
                assert (err <= mag * terms + 1e-30).all(), (lq, lk, h, err.max(), mag.max())
            at_q, at_k = at_q + lq, at_k + lk


TREES = [
    # dim, heads, group, page, nodes, tokens
    (128, 2, 4, 16, [1], [1]),
    (128, 2, 4, 16, [1, 5, 3, 2], [1, 5, 20, 300]),       # no tokens in front of two trees
    (64, 1, 1, 16, [33, 7], [64, 40]),
    (192, 3, 3, 48, [12, 1, 20], [60, 48, 220]),
    (256, 2, 1, 64, [26, 64], [129, 64]),
    (128, 1, 16, 64, [60, 13], [1000, 31]),
    (128, 2, 1, 128, [13], [5000]),                       # few rows, several parts
    (64, 2, 3, 16, [65, 2], [190, 90]),                   # more nodes than a word has bits
    (256, 1, 1, 64, [100, 17], [301, 300]),
    (128, 2, 4, 64, [70, 1, 130], [200, 1, 131]),
    (192, 1, 5, 16, [40], [41]),
    (128, 1, 4, 16, [300], [1100]),
    (128, 1, 2, 16, [200], [9000]),                       # many rows, several parts
    (128, 1, 2, 16, [9, 4, 70], [3, 0, 40]),              # nodes that are not cached
    (64, 1, 1, 16, [129] * 3 + [1] * 3, [2000, 129, 700, 1, 3000, 64]),
]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("case", range(len(TREES)))
def test_trees(fmt, case):
    dim, heads, group, page, nodes, kvs = TREES[case]
    say(f"tree {fmt} {TREES[case]}")
    c = Tree(fmt, dim, heads, group, page, nodes, kvs, seed=case)
    y = c.run()
    c.check(y)
    assert torch.equal(y, c.run())
    for mq, mk in ((1, 1), (max(nodes), max(kvs)), (1000, 1 << 20)):
        c.check(c.run(max_q=mq, max_kv=mk))
    c.check(c.run(scale=-0.3), scale=-0.3)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("dim,heads,group,nodes,kvs", [(128, 2, 4, [5, 1, 9], [5, 40, 300]),
                                                       (64, 1, 3, [100, 70], [2000, 70])])
def test_a_chain_is_the_causal_rule(fmt, dim, heads, group, nodes, kvs):
    """Every node on the one before: what kv_attention gives with the causal rule; masks of all
    nodes: without it."""
    for causal, bits in ((True, np.concatenate([tree_bits(range(-1, n - 1), -(-max(nodes) // 64)) for n in nodes])),
                         (False, np.full((sum(nodes), -(-max(nodes) // 64)), -1))):
        c = Tree(fmt, dim, heads, group, 16, nodes, kvs, seed=1, bits=bits)
        y = c.run()
        c.check(y)
        Case.check(c, Case.run(c, causal=causal), causal=causal)
        assert torch.allclose(y.float(), Case.run(c, causal=causal).float(), rtol=2 ** -5, atol=2 ** -5)


@pytest.mark.parametrize("seqs,most,uniform", [(2, 45, False), (63, 40, False), (64, 33, True), (65, 40, False),
                                               (700, 40, False), (4097, 20, False), (4100, 17, True)])
def test_whole_keys_of_many_sequences(seqs, most, uniform):
    """Row tiles found by the sequences' starts: numbers of sequences around powers of 64, some of them
    without queries, some of two tiles, with and without starts."""
    g = random.Random(seqs)
    nodes = [most if uniform else g.choice((0, 1, g.randint(0, most), most)) for _ in range(seqs)]
    nodes[0] = max(nodes[0], 1)
    kvs = [n + g.choice((0, 1, g.randint(0, 60))) for n in nodes]
    c = Tree("fp8", 64, 1, 4, 16, nodes, kvs, seed=seqs)
    starts = dict(q_starts=None) if uniform else {}
    c.check(c.run(**starts, max_q=most, max_kv=112))


def test_longer_keys_of_many_row_tiles():
    """More row tiles than rounds of the card take: keys past one part's length stay whole, up to a bound
    on the tokens, behind which they are divided."""
    g = random.Random(2)
    nodes = [g.randint(0, 9) for _ in range(290)]
    c = Tree("fp4", 64, 8, 4, 16, nodes, [g.choice((0, 5, 30, 700, 1500)) for _ in nodes], seed=3)
    need = [w8a8.load_library().w8a8_kv_tree_attention_workspace_bytes(16, 8, 64, 1, 4, sum(nodes), 290, 9, n)
            for n in (1504, 5000)]
    assert need[0] == 0 and need[1] > 0
    for max_kv in (1504, 5000):
        c.check(c.run(max_q=9, max_kv=max_kv))


def test_rows_behind_the_last_sequence():
    """q_starts that end before T: the rest of the output is left as it was, whatever the queries
    there hold; also where the keys are divided."""
    for nodes, kvs in (([9, 30], [40, 300]), ([20, 70], [3000, 5000]), ([4, 1], [4000, 9000])):
        c = Tree("fp8", 128, 2, 4, 16, nodes, kvs, seed=6)
        want = c.run()
        n = sum(nodes)
        q = torch.full((n + 50, 8, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
        q[:n] = c.q.cuda()
        c.tree = torch.cat((c.tree, torch.full((50, c.tree.shape[1]), -1, device="cuda")))
        out = torch.full_like(q, 7.0)
        c.run(q=q, out=out, max_q=max(nodes))
        c.check(out[:n])
        assert (out[n:] == 7).all() and torch.allclose(out[:n].float(), want.float(), rtol=2 ** -6, atol=2 ** -6)


@pytest.mark.parametrize("seqs", [70, 600])
def test_many_sequences(seqs):
    """More sequences than a wavefront sums at once, and than it sums at all; some without nodes."""
    rng = random.Random(seqs)
    nodes = [rng.choice([0, 1, 3, 9, 40]) for _ in range(seqs)]
    kvs = [n + rng.choice([0, 1, 50, 300]) for n in nodes]
    kvs[1] += 9000
    c = Tree("fp8", 64, 2, 3, 16, nodes, kvs, seed=8, words=1)
    y = c.run()
    c.check(y)
    assert torch.equal(y, c.run())


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("nodes,kvs", [([20], [20]), ([90, 40], [90, 41]), ([30], [12])])
def test_masks_of_any_kind(fmt, nodes, kvs):
    """Bits at random, also of later nodes; rows without any: zeros where nothing lies in front of
    the tree; bits and words past the tree are ignored."""
    rng = random.Random(5)
    words = -(-max(nodes) // 64) + 1
    masks = [rng.getrandbits(64 * words) & rng.getrandbits(64 * words) for _ in range(sum(nodes))]
    masks[0] = 0
    masks[7] = 1 << nodes[0] | 1 << 64 * words - 1
    c = Tree(fmt, 128, 1, 3, 16, nodes, kvs, seed=2, bits=bit_words(masks, words))
    y = c.run()
    c.check(y)
    if kvs[0] <= nodes[0]:
        assert (y[0] == 0).all() and (y[7] == 0).all()
    past = c.bits.copy()
    at = 0
    for n in nodes:
        for i in range(at, at + n):
            for b in range(n, 64 * words):
                past[i, b // 64] ^= np.int64(np.uint64(1 << b % 64).view(np.int64))
        at += n
    c.tree = torch.from_numpy(past).cuda()
    assert torch.equal(y, c.run())


def test_fewer_words_than_nodes():
    """Nodes past the words are seen by none."""
    c = Tree("fp8", 128, 1, 2, 16, [100], [150], seed=3)
    c.bits = np.ascontiguousarray(c.bits[:, :1])
    c.tree = torch.from_numpy(c.bits).cuda()
    c.check(c.run())


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("nodes,kv,node", [(6, 50, 2), (40, 40, 17), (200, 400, 130)])
def test_nan_nodes_reach_only_who_sees_them(fmt, nodes, kv, node):
    for part in (0, 1):
        c = Tree(fmt, 128, 1, 2, 16, [nodes], [kv], seed=7)
        new = _kv(kv, 1, 128, 8)
        j = kv - nodes + node
        new[j, part, 0, 70] = float("nan")
        pages = c.table[0].tolist()
        c.write(new, [pages[i // 16] * 16 + i % 16 for i in range(kv)])
        y = f64(c.run())
        see = tree_visible(c.bits, nodes, kv)
        bad = np.zeros(y.shape, bool)
        bad[see[:, j]] = True
        if part == 1:
            bad[:, :, :64], bad[:, :, 96:] = False, False
        assert np.array_equal(np.isnan(y), bad) and see[:, j].any() and not see[:, j].all()
        for h in range(2):
            want, mag = masked_attention(f64(c.q)[:, h], c.values[:, 0, 0], c.values[:, 1, 0], 128 ** -0.5, see)
            ok = ~see[:, j]
            assert (np.abs(y[ok, h] - want[ok]) <= mag[ok] * 3.5 * 2.0 ** -8).all()


@pytest.mark.parametrize("seqs,heads,nodes,kv", [(70, 1, 20, 3000), (60, 1, 18, 2500), (9, 3, 33, 4100)])
def test_more_pieces_than_run_at_once(seqs, heads, nodes, kv):
    """Alike sequences whose row tiles make more pieces than the target: all of them have a workgroup."""
    c = Tree("fp8", 64, heads, 1, 16, [nodes] * seqs, [kv] * seqs, seed=seqs)
    c.check(c.run())


def test_without_starts_strided_queries_and_a_buffer():
    c = Tree("fp8", 128, 2, 4, 16, [7, 7, 7], [20, 7, 333], seed=4)
    want = c.run()
    wide = torch.zeros(21, 20, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, 7:15] = c.q.cuda()
    guard = torch.full((23, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = c.run(q=wide[:, 7:15], q_starts=None, out=guard[1:-1])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    c.check(y)
    assert torch.equal(y, want) and (guard[0] == 7).all() and (guard[-1] == 7).all()


def test_offsets_beyond_32_bits():
    page_bytes = w8a8.kv_cache(0, 2, 128, 128, fmt="fp8").shape[1:].numel()
    c = Tree("fp8", 128, 2, 4, 128, [70, 3], [400, 129], seed=10, base=(1 << 32) // page_bytes + 5)
    c.check(c.run())


def test_graph_replays_with_other_trees():
    c = Tree("fp8", 128, 2, 4, 16, [20, 20], [700, 40], seed=12)
    q, table, out = c.q.cuda(), c.table.cuda(), None
    width = c.table.shape[1] * 16
    n = w8a8.load_library().w8a8_kv_tree_attention_workspace_bytes(16, 2, 128, 0, 4, 40, 2, 20, width)
    work = torch.empty(n, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)

    def step(o=None, w=None):
        return w8a8.kv_tree_attention(q, c.cache, table, c.kv_lens, c.tree, q_starts=c.q_starts, max_q=20,
                                      max_kv=width, out=o, workspace=w)
    step(out, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, work)
    for i in range(3):
        rng = random.Random(i)
        c.bits = np.concatenate([tree_bits([rng.randrange(-1, j) for j in range(20)], 1) for _ in range(2)])
        c.tree.copy_(torch.from_numpy(c.bits))
        c.kvs = [700 - 16 * i, 40 - i]
        c.kv_lens.copy_(torch.tensor(c.kvs, dtype=torch.int32))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step())
        values = c.values
        c.values = np.concatenate([values[:c.kvs[0]], values[700:700 + c.kvs[1]]])
        c.check(got)
        c.values = values


def test_binding_refusals():
    c = Tree("fp8", 128, 2, 4, 16, [5], [50], seed=13)
    good = c.tree
    for t in (good[:4], good[:, 0], good.cpu(), good.expand(5, 1)[:, :0], good.repeat(1, 65), good.t()):
        c.tree = t
        with pytest.raises(ValueError):
            c.run()
    c.tree = good.int()
    with pytest.raises(TypeError):
        c.run()
