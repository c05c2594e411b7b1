"""A transformer decoder served in microscaled formats: 4-bit linears, keys and values kept in
a paged 4- or 8-bit cache, attention straight over it.

    python examples/mx_decoder.py [--layers 4] [--steps 64] [--fmt fp8]

Prompts of different lengths go through the stack in one pass (their keys and values written to
the cache as they are computed), then every sequence decodes one token at a time; a decoding
step is captured once in a HIP graph and replayed. Weights are random: the program shows how
the operators are used together and how long they take.
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
        self.layers = [w8a8.kv_cache(pages, heads, head_dim, page_size, fmt=fmt)
                       for _ in range(layers)]
        self.free = list(range(pages))
        self.table_host = torch.zeros(sequences, max_pages, dtype=torch.int32)
        self.lens_host = [0] * sequences
        self.table = self.table_host.cuda()
        self.lens = torch.zeros(sequences, dtype=torch.int32, device="cuda")

    def extend(self, seq: int, n: int) -> list[int]:
        """Slots of the next n tokens of a sequence, with pages for them."""
        slots = []
        for pos in range(self.lens_host[seq], self.lens_host[seq] + n):
            page, at = divmod(pos, self.page_size)
            if at == 0:
                self.table_host[seq, page] = self.free.pop()
            slots.append(int(self.table_host[seq, page]) * self.page_size + at)
        self.lens_host[seq] += n
        return slots

    def publish(self) -> None:
        """The host's table and lengths to the device, into the tensors that kernels read."""
        self.table.copy_(self.table_host)
        self.lens.copy_(torch.tensor(self.lens_host, dtype=torch.int32))


class DecoderLayer(torch.nn.Module):
    def __init__(self, hidden, heads, kv_heads, head_dim, ffn):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim

        def linear(k, n, act="none"):
            lin = torch.nn.Linear(k, n, bias=False, device="cuda", dtype=torch.bfloat16)
            return MX4Linear.from_linear(lin, act=act)

        self.qkv = linear(hidden, (heads + 2 * kv_heads) * head_dim)
        self.out = linear(heads * head_dim, hidden)
        self.up = linear(hidden, ffn)
        self.down = linear(ffn, hidden, act="gelu")     # GELU in front of its quantizer

    def forward(self, x, cache, paged, slots, q_starts, max_q, max_kv):
        """x [T, hidden]: the queries of all sequences one after the other."""
        norm = torch.nn.functional.rms_norm
        qkv = self.qkv(norm(x, x.shape[-1:])).view(x.shape[0], -1, self.head_dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 1)
        torch.ops.w8a8.kv_write(cache, k, v, slots, paged.fmt)
        y = torch.ops.w8a8.kv_attention(q, cache, paged.table, paged.lens, q_starts, paged.fmt,
                                        None, True, max_q, max_kv)
        x = x + self.out(y.flatten(1))
        return x + self.down(self.up(norm(x, x.shape[-1:])))


class Decoder(torch.nn.Module):
    def __init__(self, layers, hidden, heads, kv_heads, head_dim, ffn):
        super().__init__()
        self.layers = torch.nn.ModuleList(
            DecoderLayer(hidden, heads, kv_heads, head_dim, ffn) for _ in range(layers))

    def forward(self, x, paged, slots, q_starts, max_q, max_kv):
        for layer, cache in zip(self.layers, paged.layers):
            x = layer(x, cache, paged, slots, q_starts, max_q, max_kv)
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
    y = model(torch.cat(prompts), paged, slots, starts, max(lens), max(lens))
    x = y[(starts[1:] - 1).long()]

    # One decoding step reads its inputs from fixed tensors; only their contents change.
    n = len(prompts)
    slots = torch.empty(n, dtype=torch.int64, device="cuda")
    state = x.clone()

    def step():
        return model(state, paged, slots, None, 1, paged.max_tokens)

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


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--sequences", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=2000, help="tokens of the longest prompt")
    ap.add_argument("--fmt", choices=sorted(w8a8.KV_FORMATS), default="fp8")
    a = ap.parse_args()
    hidden, heads, kv_heads, head_dim, ffn, page = 4096, 32, 8, 128, 16384, 64
    torch.manual_seed(0)
    model = Decoder(a.layers, hidden, heads, kv_heads, head_dim, ffn)
    lens = [max(1, a.prompt * (i + 1) // a.sequences) for i in range(a.sequences)]
    per = -(-(a.prompt + a.steps) // page)
    paged = PagedCache(a.layers, sum(-(-(n + a.steps) // page) for n in lens), kv_heads, head_dim,
                       page, a.fmt, per, a.sequences)
    prompts = [torch.randn(n, hidden, device="cuda").to(torch.bfloat16) for n in lens]
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    _, out = generate(model, paged, prompts, a.steps)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t0) * 1e3
    print(f"{a.layers} layers, {sum(lens)} prompt tokens of {a.sequences} sequences and {a.steps} "
          f"steps in {ms:.1f} ms; finite: {bool(out.isfinite().all())}")


if __name__ == "__main__":
    main()
