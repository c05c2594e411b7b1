"""The operators of a decoding step together, as a program uses them: norm, int8 linear, keys appended
with their positions, attention of drafted trees, norm, linear, log probabilities; the drafts kept."""
import importlib.util
import os
import random

import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
import paper_2606_14598_amd.torch_ops as ops  # noqa: F401  (registers the ops)
from _lm_ref import cos_sin, f32_inverse_rms, int8_rows, masked_attention, norm_values, rotate, tree_bits, tree_visible
from _mx_ref import block_values, f64, quantize_blocks
from test_gpu_logprobs import check as check_logprobs

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


HIDDEN, HEADS, KV, DIM, PAGE, VOCAB = 512, 8, 2, 64, 16, 5000


class Step:
    """A layer and the vocabulary's projection behind it, over sequences that have `before` tokens
    cached and trees of drafts."""

    def __init__(self, fmt, before, nodes, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.fmt, self.before, self.nodes = fmt, before, nodes

        def weights(n, k):
            w = (torch.randn(n, k, generator=g) * k ** -0.5).to(torch.bfloat16)
            return w8a8.quantize_weight(w.cuda())
        self.qkv, self.out = weights((HEADS + 2 * KV) * DIM, HIDDEN), weights(HIDDEN, HEADS * DIM)
        self.head = weights(VOCAB, HIDDEN)
        self.norms = [(1 + 0.2 * torch.randn(HIDDEN, generator=g)).cuda() for _ in range(2)]
        self.inv_freq = (10000.0 ** -(torch.arange(DIM // 2, dtype=torch.float64) / (DIM // 2))).float().cuda()
        need = [-(-(b + n) // PAGE) for b, n in zip(before, nodes)]
        pages = torch.randperm(sum(need) + 2, generator=g)
        self.cache = w8a8.kv_cache(sum(need) + 2, KV, DIM, PAGE, fmt=fmt)
        self.table = torch.zeros(len(before), max(need), dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = pages[at:at + n]
            at += n
        rng = random.Random(seed)
        self.parents = [[rng.randrange(-1, i) for i in range(n)] for n in nodes]
        depth = []
        for p in self.parents:
            d = []
            for i in p:
                d.append(d[i] + 1 if i >= 0 else 0)
            depth.append(d)
        T = sum(nodes)
        # what is cached already
        slots = [self.slot(b, j) for b, n in enumerate(before) for j in range(n)]
        kv = torch.randn(len(slots), 2, KV, DIM, generator=g).to(torch.bfloat16).cuda()
        w8a8.kv_write(self.cache, kv[:, 0], kv[:, 1], torch.tensor(slots, dtype=torch.int64).cuda(), fmt=fmt)
        # the step's inputs, in tensors of its own; three rows of padding behind the last sequence
        pad = 3
        self.x = torch.zeros(T + pad, HIDDEN, dtype=torch.bfloat16, device="cuda")
        self.residual = torch.zeros_like(self.x)
        self.slots = torch.tensor([self.slot(b, before[b] + i) for b, n in enumerate(nodes) for i in range(n)]
                                  + [-1] * pad).cuda()
        self.positions = torch.tensor([before[b] + i for b, d in enumerate(depth) for i in d] + [0] * pad).cuda()
        self.lens = torch.tensor([b + n for b, n in zip(before, nodes)], dtype=torch.int32).cuda()
        self.starts = torch.tensor([0] + list(np.cumsum(nodes)), dtype=torch.int32).cuda()
        self.bits = np.concatenate([tree_bits(p, 1) for p in self.parents] + [np.zeros((pad, 1), np.int64)])
        self.tree = torch.from_numpy(self.bits).cuda()
        self.tokens = torch.randint(0, VOCAB, (T + pad,), generator=g).cuda()
        self.tokens[T:] = -1
        self.attended = torch.zeros(T + pad, HEADS, DIM, dtype=torch.bfloat16, device="cuda")

    def slot(self, b, j):
        return int(self.table[b, j // PAGE]) * PAGE + j % PAGE

    def inputs(self, seed):
        g = torch.Generator().manual_seed(seed)
        for t in (self.x, self.residual):
            t.copy_(torch.randn(t.shape, generator=g).to(torch.bfloat16))

    def run(self, cache=None):
        cache = self.cache if cache is None else cache
        q1, s1, h = w8a8.rms_norm_quantize(self.x, self.norms[0], residual=self.residual)
        y = w8a8.gemm(q1, s1, *self.qkv).view(-1, HEADS + 2 * KV, DIM)
        q, k, v = y.split((HEADS, KV, KV), 1)
        q = w8a8.kv_append(cache, k, v, self.slots, self.positions, self.inv_freq, q=q, fmt=self.fmt)
        o = w8a8.kv_tree_attention(q, cache, self.table_dev, self.lens, self.tree, fmt=self.fmt,
                                   q_starts=self.starts, max_kv=int(self.table.shape[1] * PAGE),
                                   out=self.attended)
        q2, s2 = w8a8.quantize_act(o.flatten(1))
        z = w8a8.gemm(q2, s2, *self.out)
        q3, s3, h2 = w8a8.rms_norm_quantize(z, self.norms[1], residual=h)
        logits = w8a8.gemm(q3, s3, *self.head)
        return (q1, s1, h, y, q, o, z, h2, logits, *w8a8.token_logprobs(logits, self.tokens, top=4))

    @property
    def table_dev(self):
        if not hasattr(self, "_table"):
            self._table = self.table.cuda()
        return self._table

    def check(self, r):
        q1, s1, h, y, q, o, z, h2, logits, *lp = r
        hv = (self.x.float() + self.residual.float()).to(torch.bfloat16)
        assert torch.equal(h, hv) and torch.equal(h2, (z.float() + h.float()).to(torch.bfloat16))
        rms, near = f32_inverse_rms(f64(hv), 1e-6)
        codes, scales = int8_rows(norm_values(f64(hv), rms, self.norms[0].cpu().numpy()))
        assert not near.any()
        assert np.array_equal(q1.cpu().numpy(), codes) and np.array_equal(s1.cpu().numpy(), scales)
        cos, sin, near = cos_sin(self.positions.cpu().numpy(), self.inv_freq.cpu().numpy(), None)
        assert not near.any()
        turned = rotate(y.float().cpu().numpy(), cos, sin, False)
        assert torch.equal(q.cpu(), torch.from_numpy(turned[:, :HEADS]).to(torch.bfloat16))
        T = sum(self.nodes)
        kv = np.concatenate([turned[:, HEADS:HEADS + KV], y.float().cpu().numpy()[:, HEADS + KV:]], 1)[:T]
        want = block_values(*quantize_blocks(kv.reshape(T, 2, KV, DIM).astype(np.float64), self.fmt), self.fmt)
        k, v = w8a8.kv_read(self.cache, self.slots[:T], DIM, fmt=self.fmt)
        assert np.array_equal(f64(k), want[:, 0]) and np.array_equal(f64(v), want[:, 1])
        at = 0
        for b, (n0, n) in enumerate(zip(self.before, self.nodes)):
            slots = torch.tensor([self.slot(b, j) for j in range(n0 + n)]).cuda()
            ks, vs = (f64(t) for t in w8a8.kv_read(self.cache, slots, DIM, fmt=self.fmt))
            see = tree_visible(self.bits[at:at + n], n, n0 + n)
            for hd in range(HEADS):
                w, mag = masked_attention(f64(q[at:at + n, hd]), ks[:, hd * KV // HEADS], vs[:, hd * KV // HEADS],
                                          DIM ** -0.5, see)
                # two roundings to bf16 where a sequence has over 64 rows, and the weights' own sum
                assert (np.abs(f64(o[at:at + n, hd]) - w) <= mag * 3.25 * 2.0 ** -8).all()
            at += n
        assert (o[T:] == 0).all()              # rows behind the last sequence are left as they were
        check_logprobs(lp, f64(logits), self.tokens.cpu().numpy(), 4)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_a_step_and_its_graph(fmt):
    s = Step(fmt, [0, 40, 700, 5], [6, 1, 30, 12])
    s.inputs(0)
    s.check(s.run())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = s.run()
    for i in range(1, 4):
        s.inputs(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        s.check(got)
        assert all(torch.equal(a, b) for a, b in zip(got, s.run()))


def test_ops_are_the_calls():
    """The same step through torch.ops, eager and compiled."""
    s = Step("fp8", [0, 40], [6, 20])
    s.inputs(7)
    o = torch.ops.w8a8
    table, width = s.table.cuda(), int(s.table.shape[1] * PAGE)

    def step(cache, x, residual):
        q1, s1, h = o.rms_norm_quantize(x, s.norms[0], residual, 1e-6, "int8")
        y = o.gemm(q1, s1, *s.qkv, None).view(-1, HEADS + 2 * KV, DIM)
        q, k, v = y.split((HEADS, KV, KV), 1)
        q = o.kv_append(cache, k, v, s.slots, s.positions, s.inv_freq, q, s.fmt, None, False)
        a = o.kv_tree_attention(q, cache, table, s.lens, s.tree, s.starts, s.fmt, None, None, width)
        # what the op leaves in rows behind the last sequence is nothing
        a = torch.where((s.tokens >= 0)[:, None, None], a, 0.0)
        q3, s3, h2 = o.rms_norm_quantize(a.flatten(1), s.norms[1], h, 1e-6, "int8")
        return h2, *o.token_logprobs(o.gemm(q3, s3, *s.head, None), s.tokens, 4, 1.0)
    caches = [s.cache.clone() for _ in range(2)]
    want = step(caches[0], s.x, s.residual)
    got = torch.compile(step, fullgraph=True, backend="aot_eager")(caches[1], s.x, s.residual)
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and torch.equal(*caches)
    s.run()
    assert torch.equal(caches[0], s.cache)


def test_opcheck_and_fake_shapes():
    s = Step("fp8", [0, 40], [6, 20])
    s.inputs(1)
    r = s.run()
    tests = ("test_schema", "test_faketensor")
    o = torch.ops.w8a8
    for fmt in ("int8", "mx4"):
        for residual in (None, s.residual):
            torch.library.opcheck(o.rms_norm_quantize.default, (s.x, s.norms[0], residual, 1e-6, fmt), test_utils=tests)
    torch.library.opcheck(o.token_logprobs.default, (r[8], s.tokens, 4, 1.0), test_utils=tests)
    q, k, v = r[3].split((HEADS, KV, KV), 1)
    for qq in (q, None):
        torch.library.opcheck(o.kv_append.default, (s.cache, k, v, s.slots, s.positions, s.inv_freq, qq, "fp8", None,
                                                    False), test_utils=tests)
    torch.library.opcheck(o.kv_tree_attention.default, (r[4], s.cache, s.table.cuda(), s.lens, s.tree, s.starts, "fp8",
                                                        None, None, 64), test_utils=tests)


def _example():
    spec = importlib.util.spec_from_file_location("mx_decoder", os.path.join(ROOT, "examples", "mx_decoder.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_example_verifies_drafts(fmt):
    """The example's decoder with rotary positions: prompts, captured steps equal to eager ones, trees
    verified; the kept path's tokens have, bit for bit, the keys and values that appending them alone
    gives."""
    ex = _example()
    torch.manual_seed(2)
    hidden, heads, kv_heads, dim, ffn = 256, 4, 2, 64, 512
    model = ex.Decoder(1, hidden, heads, kv_heads, dim, ffn, 1e4)
    lens, steps, n = [37, 5, 1], 3, 9
    prompts = [torch.randn(m, hidden, device="cuda").to(torch.bfloat16) for m in lens]

    def paged():
        return ex.PagedCache(1, 20, kv_heads, dim, 16, fmt, 5, len(lens))
    cache = paged()
    y, out = ex.generate(model, cache, prompts, steps)
    other = paged()
    y2, out2 = ex.generate(model, other, prompts, steps, use_graph=False)
    assert torch.equal(y, y2) and torch.equal(out, out2) and torch.equal(cache.layers[0], other.layers[0])
    head = w8a8.quantize_weight((torch.randn(1000, hidden, device="cuda") / 16).to(torch.bfloat16))
    norm = torch.ones(hidden, device="cuda")
    parents = [[-1, 0, 0, 1, 2, 4, 3, 6, -1]] * 3
    x = torch.randn(3 * n, hidden, device="cuda").to(torch.bfloat16)
    tokens = torch.randint(0, 1000, (3 * n,), device="cuda")
    calls = []
    hook = model.layers[0].qkv.register_forward_hook(lambda m, a, r: calls.append(r.clone()))
    logp, entropy, _, ids = ex.verify(model, head, norm, cache, x, parents, tokens)
    hook.remove()
    assert logp.shape == (3 * n,) and (logp <= 0).all() and (entropy >= 0).all() and ids.shape == (3 * n, 4)
    assert cache.lens_host == [m + steps + n for m in lens]
    path = [0, 2, 4, 5]
    qkv = calls[0].view(3, n, -1, dim)
    for b in range(3):
        cache.keep(b, n, path)
        # the same tokens appended to the other cache, one behind the other
        first = other.lens_host[b]
        slots = torch.tensor(other.extend(b, len(path))).cuda()
        k, v = (t.contiguous() for t in qkv[b, path, heads:].split((kv_heads, kv_heads), 1))
        positions = torch.arange(first, first + len(path)).cuda()
        w8a8.kv_append(other.layers[0], k, v, slots, positions, model.layers[0].inv_freq, fmt=fmt)
        assert cache.lens_host[b] == other.lens_host[b]
        for c in (cache, other):
            c.read = w8a8.kv_read(c.layers[0], torch.tensor(
                [int(c.table_host[b, p // 16]) * 16 + p % 16 for p in range(c.lens_host[b])]).cuda(), dim, fmt=fmt)
        assert all(torch.equal(a, d) for a, d in zip(cache.read, other.read))
