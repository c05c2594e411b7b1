"""A transformer decoder served in microscaled formats: 4-bit linears, keys and values kept in
a paged 4- or 8-bit cache, attention straight over it.

    python examples/mx_decoder.py [--layers 4] [--steps 64] [--fmt fp8] [--drafts 24]

Prompts of different lengths go through the stack in one pass (their keys and values written to
the cache as they are computed), then every sequence decodes one token at a time; a decoding
step is captured once in a HIP graph and replayed. With --drafts each sequence then gets a tree of
drafted tokens, which one pass verifies: their keys turned by their positions as they are cached,
attention by the tree's mask, log probabilities of the drafts; the best path's tokens stay in the
cache. Weights are random: the program shows how the operators are used together and how long they
take.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2606_14598_amd as w8a8  # noqa: E402
from paper_2606_14598_amd.torch_ops import MX4Linear  # noqa: E402


class PagedCache:
    """Caches of all layers over one set of pages, and which of them each sequence has."""

    def __init__(self, layers, pages, heads, head_dim, page_size, fmt, max_pages, sequences):
        self.fmt, self.page_size, self.max_tokens = fmt, page_size, max_pages * page_size
        self.head_dim = head_dim
        self.layers = [w8a8.kv_cache(pages, heads, head_dim, page_size, fmt=fmt)
                       for _ in range(layers)]
        self.free = list(range(pages))
        self.table_host = torch.zeros(sequences, max_pages, dtype=torch.int32)
        self.lens_host = [0] * sequences
        self.pages_of = [0] * sequences
        self.table = self.table_host.cuda()
        self.lens = torch.zeros(sequences, dtype=torch.int32, device="cuda")

    def extend(self, seq: int, n: int) -> list[int]:
        """Slots of the next n tokens of a sequence, with pages for them."""
        slots = []
        for pos in range(self.lens_host[seq], self.lens_host[seq] + n):
            page, at = divmod(pos, self.page_size)
            if at == 0 and page >= self.pages_of[seq]:      # dropped tokens leave theirs
                self.table_host[seq, page] = self.free.pop()
                self.pages_of[seq] = page + 1
            slots.append(int(self.table_host[seq, page]) * self.page_size + at)
        self.lens_host[seq] += n
        return slots

    def drop(self, seq: int, n: int) -> None:
        """The last n tokens of a sequence are no more; its pages stay."""
        self.lens_host[seq] -= n

    def keep(self, seq: int, nodes: int, path: list[int]) -> None:
        """Of a sequence's last `nodes` tokens only those of a path stay, one behind the other. What is
        read from the cache is written back bit for bit, and a node on a path has the position that it
        has in the sequence, so nothing is computed again."""
        first = self.lens_host[seq] - nodes
        at = [first + i for i in path] + [first + i for i in range(len(path))]
        slots = torch.tensor([int(self.table_host[seq, p // self.page_size]) * self.page_size
                              + p % self.page_size for p in at]).cuda()
        for cache in self.layers:
            k, v = w8a8.kv_read(cache, slots[:len(path)], self.head_dim, fmt=self.fmt)
            w8a8.kv_write(cache, k, v, slots[len(path):], fmt=self.fmt)
        self.drop(seq, nodes - len(path))

    def publish(self) -> None:
        """The host's table and lengths to the device, into the tensors that kernels read."""
        self.table.copy_(self.table_host)
        self.lens.copy_(torch.tensor(self.lens_host, dtype=torch.int32))


class DecoderLayer(torch.nn.Module):
    def __init__(self, hidden, heads, kv_heads, head_dim, ffn, inv_freq=None):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.register_buffer("inv_freq", inv_freq)

        def linear(k, n, act="none"):
            lin = torch.nn.Linear(k, n, bias=False, device="cuda", dtype=torch.bfloat16)
            return MX4Linear.from_linear(lin, act=act)

        self.qkv = linear(hidden, (heads + 2 * kv_heads) * head_dim)
        self.out = linear(heads * head_dim, hidden)
        self.up = linear(hidden, ffn)
        self.down = linear(ffn, hidden, act="gelu")     # GELU in front of its quantizer

    def forward(self, x, cache, paged, slots, q_starts, max_q, max_kv, positions=None, tree=None):
        """x [T, hidden]: the queries of all sequences one after the other. positions int64 [T] with
        rotary positions; tree: the mask of drafted trees, whose nodes the queries are."""
        norm = torch.nn.functional.rms_norm
        qkv = self.qkv(norm(x, x.shape[-1:])).view(x.shape[0], -1, self.head_dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 1)
        if self.inv_freq is None:
            torch.ops.w8a8.kv_write(cache, k, v, slots, paged.fmt)
        else:
            q = torch.ops.w8a8.kv_append(cache, k, v, slots, positions, self.inv_freq, q, paged.fmt,
                                         None, False)
        if tree is None:
            y = torch.ops.w8a8.kv_attention(q, cache, paged.table, paged.lens, q_starts, paged.fmt,
                                            None, True, max_q, max_kv)
        else:
            y = torch.ops.w8a8.kv_tree_attention(q, cache, paged.table, paged.lens, tree, q_starts,
                                                 paged.fmt, None, max_q, max_kv)
        x = x + self.out(y.flatten(1))
        return x + self.down(self.up(norm(x, x.shape[-1:])))


class Decoder(torch.nn.Module):
    def __init__(self, layers, hidden, heads, kv_heads, head_dim, ffn, theta=None):
        super().__init__()
        inv_freq = None
        if theta is not None:       # rotary positions of that base
            pairs = torch.arange(head_dim // 2, dtype=torch.float64) / (head_dim // 2)
            inv_freq = (theta ** -pairs).float().cuda()
        self.rotary = theta is not None
        self.layers = torch.nn.ModuleList(
            DecoderLayer(hidden, heads, kv_heads, head_dim, ffn, inv_freq) for _ in range(layers))

    def forward(self, x, paged, slots, q_starts, max_q, max_kv, positions=None, tree=None):
        for layer, cache in zip(self.layers, paged.layers):
            x = layer(x, cache, paged, slots, q_starts, max_q, max_kv, positions, tree)
        return x


@torch.no_grad()
def generate(model, paged, prompts, steps, use_graph=True):
    """prompts: [tokens, hidden] of each sequence. Returns the stack's outputs for the prompts
    [T, hidden] and for `steps` decoding steps [steps, sequences, hidden], each step fed with
    the one before; without use_graph every step runs eagerly."""
    lens = [p.shape[0] for p in prompts]
    starts = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    slots = torch.tensor([s for i, n in enumerate(lens) for s in paged.extend(i, n)]).cuda()
    paged.publish()
    positions = torch.cat([torch.arange(n) for n in lens]).cuda() if model.rotary else None
    y = model(torch.cat(prompts), paged, slots, starts, max(lens), max(lens), positions)
    x = y[(starts[1:] - 1).long()]

    # One decoding step reads its inputs from fixed tensors; only their contents change.
    n = len(prompts)
    slots = torch.empty(n, dtype=torch.int64, device="cuda")
    state = x.clone()

    def step():
        # a token's position is that of the last one cached
        return model(state, paged, slots, None, 1, paged.max_tokens,
                     paged.lens.long() - 1 if model.rotary else None)

    def prepare():
        slots.copy_(torch.tensor([paged.extend(i, 1)[0] for i in range(n)]))
        paged.publish()

    out = torch.empty(steps, *x.shape, dtype=x.dtype, device="cuda")
    graph = None
    for i in range(steps):
        prepare()
        if not use_graph:
            out[i] = step()
            state.copy_(out[i])
        elif graph is None:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                result = step()                 # the first step runs eagerly: it warms up
                first = result.clone()
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                result = step()
            state.copy_(first)
            out[i] = first
        else:
            graph.replay()
            out[i] = result
            state.copy_(result)
    return y, out


def tree_mask(parents):
    """int64 [nodes, words]: a node (its parent's number, -1 for none) sees its ancestors and itself."""
    seen = []
    for i, p in enumerate(parents):
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
    words = [[m >> 64 * w & (1 << 64) - 1 for w in range(-(-len(parents) // 64))] for m in seen]
    return torch.tensor([[w - (1 << 64) if w >> 63 else w for w in row] for row in words])


@torch.no_grad()
def verify(model, head, norm, paged, x, parents, tokens, top=4):
    """One pass over drafted trees of alike size, one a sequence: x [sequences * nodes, hidden], the
    nodes' inputs; parents: of the nodes of each sequence; tokens int64 [sequences * nodes]: the token
    to be scored at each node. head: W8A8 weights (wq, w_scale) of the vocabulary's projection, norm:
    the weight of the norm in front of it. Returns token_logprobs' results; the nodes are the last
    tokens of their sequences then (PagedCache.keep)."""
    n = len(parents[0])
    depth = []
    for p in parents:
        d = []
        for i in p:
            d.append(d[i] + 1 if i >= 0 else 0)
        depth.append(d)
    before = list(paged.lens_host)
    slots = torch.tensor([s for b in range(len(parents)) for s in paged.extend(b, n)]).cuda()
    paged.publish()
    positions = torch.tensor([before[b] + i for b, d in enumerate(depth) for i in d]).cuda()
    tree = torch.cat([tree_mask(p) for p in parents]).cuda()
    y = model(x, paged, slots, None, n, max(paged.lens_host), positions, tree)
    q, scale, _ = w8a8.rms_norm_quantize(y, norm)
    return w8a8.token_logprobs(w8a8.gemm(q, scale, *head), tokens, top=top)


def best_path(parents, logp):
    """The nodes from a root to the one whose path has the largest sum of log probabilities a node."""
    sums, length = [], []
    for i, p in enumerate(parents):
        sums.append((sums[p] if p >= 0 else 0.0) + logp[i])
        length.append((length[p] if p >= 0 else 0) + 1)
    at = max(range(len(parents)), key=lambda i: sums[i] / length[i])
    path = []
    while at >= 0:
        path.append(at)
        at = parents[at]
    return path[::-1]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--sequences", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=2000, help="tokens of the longest prompt")
    ap.add_argument("--drafts", type=int, default=0, help="drafted tokens of each sequence to verify")
    ap.add_argument("--fmt", choices=sorted(w8a8.KV_FORMATS), default="fp8")
    a = ap.parse_args()
    hidden, heads, kv_heads, head_dim, ffn, page = 4096, 32, 8, 128, 16384, 64
    torch.manual_seed(0)
    model = Decoder(a.layers, hidden, heads, kv_heads, head_dim, ffn, 1e4 if a.drafts else None)
    lens = [max(1, a.prompt * (i + 1) // a.sequences) for i in range(a.sequences)]
    more = a.steps + a.drafts
    per = -(-(a.prompt + more) // page)
    paged = PagedCache(a.layers, sum(-(-(n + more) // page) for n in lens), kv_heads, head_dim,
                       page, a.fmt, per, a.sequences)
    prompts = [torch.randn(n, hidden, device="cuda").to(torch.bfloat16) for n in lens]
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    _, out = generate(model, paged, prompts, a.steps)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t0) * 1e3
    print(f"{a.layers} layers, {sum(lens)} prompt tokens of {a.sequences} sequences and {a.steps} "
          f"steps in {ms:.1f} ms; finite: {bool(out.isfinite().all())}")
    if a.drafts:
        vocabulary, n = 32000, a.drafts
        head = w8a8.quantize_weight(
            (0.02 * torch.randn(vocabulary, hidden, device="cuda")).to(torch.bfloat16))
        norm = torch.ones(hidden, device="cuda")
        parents = [[(i - 1) // 2 if i else -1 for i in range(n)]] * a.sequences
        x = torch.randn(a.sequences * n, hidden, device="cuda").to(torch.bfloat16)
        tokens = torch.randint(0, vocabulary, (a.sequences * n,), device="cuda")
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        logp, entropy, _, _ = verify(model, head, norm, paged, x, parents, tokens)
        scores = logp.view(a.sequences, n).tolist()
        ms = (time.perf_counter() - t0) * 1e3
        kept = 0
        for b, p in enumerate(parents):
            path = best_path(p, scores[b])
            paged.keep(b, n, path)
            kept += len(path)
        paged.publish()
        print(f"{a.sequences} trees of {n} drafts in {ms:.1f} ms; {kept} tokens kept, mean entropy "
              f"{float(entropy.mean()):.2f}")


if __name__ == "__main__":
    main()
