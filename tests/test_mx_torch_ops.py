"""The microscaled operators as torch.library ops and modules, and the example that serves a
decoder with them."""
import importlib.util
import os

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2606_14598_amd as w8a8
import paper_2606_14598_amd.torch_ops as ops
from _mx_ref import attention, block_values, f64, matrix_values, quantize_blocks

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_fake_shapes_and_dtypes():
    bf, u8 = torch.bfloat16, torch.uint8
    with FakeTensorMode():
        def e(*shape, dtype=bf):
            return torch.empty(*shape, dtype=dtype, device="cuda")
        y = torch.ops.w8a8.mx4_linear(e(2, 7, 1000), e(300, 512, dtype=u8), e(4, 300, 8, dtype=u8),
                                      None, 1, None)
        assert y.shape == (2, 7, 300) and y.dtype == bf
        q, s = torch.ops.w8a8.mx4_quantize(e(14, 1000), 0, None)
        assert q.shape == (14, 512) and s.shape == (4, 14, 8) and q.dtype == s.dtype == u8
        cache, slots = e(4, 2, 2, 16 * 132, dtype=u8), e(3, dtype=torch.int64)
        k = e(3, 2, 128)
        assert torch.ops.w8a8.kv_write(cache, k, k, slots, "fp8") is None
        a, b = torch.ops.w8a8.kv_read(cache, slots, 128, "fp8")
        assert a.shape == b.shape == (3, 2, 128) and a.dtype == bf
        y = torch.ops.w8a8.kv_attention(e(3, 8, 128), cache, e(3, 4, dtype=torch.int32),
                                        e(3, dtype=torch.int32), None, "fp8", None, True, None, None)
        assert y.shape == (3, 8, 128) and y.dtype == bf


def test_module_checks_its_sizes():
    wq, sw = torch.zeros(5, 32, dtype=torch.uint8), torch.zeros(1, 5, 8, dtype=torch.uint8)
    m = ops.MX4Linear(wq, sw, 40)
    assert m.in_features == 40 and m.out_features == 5
    for k in (32, 65):
        with pytest.raises(ValueError):
            ops.MX4Linear(wq, sw, k)


@pytest.mark.gpu
def test_module_and_compile_without_graph_breaks():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.manual_seed(0)
    a = torch.nn.Linear(1000, 512, device="cuda", dtype=torch.bfloat16)
    b = torch.nn.Linear(512, 300, device="cuda", dtype=torch.bfloat16)
    m1, m2 = ops.MX4Linear.from_linear(a), ops.MX4Linear.from_linear(b, act="gelu")

    def block(x):
        return m2(m1(x)) + 1.0

    x = torch.randn(3, 50, 1000, device="cuda").to(torch.bfloat16)
    eager = block(x)
    h = w8a8.mx4_linear(x, m1.wq, m1.w_scale, m1.bias)
    assert torch.equal(eager, w8a8.mx4_linear(h, m2.wq, m2.w_scale, m2.bias, act="gelu") + 1.0)
    assert torch._dynamo.explain(block)(x).graph_break_count == 0
    assert torch.equal(torch.compile(block, fullgraph=True, backend="aot_eager")(x), eager)
    # smoothing moves factors between operands
    s = torch.rand(1000, device="cuda") + 0.5
    m3 = ops.MX4Linear.from_linear(a, smooth=s, smooth_inv=1 / s)
    assert torch.equal(m3.wq, w8a8.mx4_quantize(a.weight.detach(), col_mul=s)[0])
    with pytest.raises(ValueError):
        ops.MX4Linear.from_linear(a, smooth=s)


@pytest.mark.gpu
def test_opcheck():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    x = torch.randn(33, 256, device="cuda").to(torch.bfloat16)
    wq, sw = w8a8.mx4_quantize(torch.randn(64, 256, device="cuda").to(torch.bfloat16))
    tests = ("test_schema", "test_faketensor")
    o = torch.ops.w8a8
    torch.library.opcheck(o.mx4_linear.default, (x, wq, sw, None, 1, None), test_utils=tests)
    torch.library.opcheck(o.mx4_quantize.default, (x, 0, None), test_utils=tests)
    cache = w8a8.kv_cache(4, 2, 128, 16)
    k = torch.randn(3, 2, 128, device="cuda").to(torch.bfloat16)
    slots = torch.tensor([0, 1, 2], device="cuda")
    torch.library.opcheck(o.kv_write.default, (cache, k, k, slots, "fp8"), test_utils=tests)
    torch.library.opcheck(o.kv_read.default, (cache, slots, 128, "fp8"), test_utils=tests)
    table = torch.zeros(1, 4, dtype=torch.int32, device="cuda")
    lens = torch.tensor([3], dtype=torch.int32, device="cuda")
    q = torch.randn(2, 4, 128, device="cuda").to(torch.bfloat16)
    torch.library.opcheck(o.kv_attention.default,
                          (q, cache, table, lens, None, "fp8", None, True, 2, 3), test_utils=tests)


def _example():
    spec = importlib.util.spec_from_file_location("mx_decoder",
                                                  os.path.join(ROOT, "examples", "mx_decoder.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _check_linear(m, x, y, act):
    """A call of an MX4Linear against its definition in float64: the codes of the kernel's own
    quantizer (its tests pin it down), the product within float32 accumulation and the rounding
    to bf16."""
    x, y = x.reshape(-1, x.shape[-1]), y.reshape(-1, y.shape[-1])
    xq, xs = w8a8.mx4_quantize(x.contiguous(), act=act)
    xv = matrix_values(xq.cpu().numpy(), xs.cpu().numpy(), m.in_features)
    wv = matrix_values(m.wq.cpu().numpy(), m.w_scale.cpu().numpy(), m.in_features)
    want, mag = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    tol = np.abs(want) * 2.0 ** -8 + mag * (m.in_features + 8) * 2.0 ** -23 + 1e-37
    assert (np.abs(f64(y) - want) <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_example_is_made_of_the_operators(fmt):
    """Prompts and decoding steps of one layer: every linear on the inputs it had, every
    attention on the queries, keys and values that the projection gave, against 64-bit forms;
    the steps replayed from a graph bit for bit as the eager ones."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ex = _example()
    torch.manual_seed(1)
    hidden, heads, kv_heads, dim, ffn = 256, 4, 2, 64, 512
    model = ex.Decoder(1, hidden, heads, kv_heads, dim, ffn)
    layer = model.layers[0]
    lens, steps = [37, 5, 1], 4
    prompts = [torch.randn(n, hidden, device="cuda").to(torch.bfloat16) for n in lens]

    def paged():
        return ex.PagedCache(1, 20, kv_heads, dim, 16, fmt, 4, len(lens))

    cache = paged()
    y, out = ex.generate(model, cache, prompts, steps)
    assert cache.lens_host == [n + steps for n in lens]
    calls = {name: [] for name in ("qkv", "out", "up", "down")}
    hooks = [getattr(layer, name).register_forward_hook(
        lambda m, x, r, name=name: calls[name].append((x[0].clone(), r.clone())))
        for name in calls]
    y2, out2 = ex.generate(model, paged(), prompts, steps, use_graph=False)
    for h in hooks:
        h.remove()
    assert torch.equal(y, y2) and torch.equal(out, out2)
    for name in calls:
        assert len(calls[name]) == 1 + steps
        for x, r in calls[name]:
            _check_linear(getattr(layer, name), x, r, "gelu" if name == "down" else "none")
    seen = [np.zeros((0, heads + 2 * kv_heads, dim)) for _ in lens]
    for i in range(1 + steps):
        qkv, got = f64(calls["qkv"][i][1]), f64(calls["out"][i][0])
        qkv, got = qkv.reshape(-1, heads + 2 * kv_heads, dim), got.reshape(-1, heads, dim)
        at = 0
        for b, n in enumerate(lens):
            n = n if i == 0 else 1
            seen[b] = np.concatenate([seen[b], qkv[at:at + n]])
            kv = block_values(*quantize_blocks(seen[b][:, heads:], fmt), fmt)
            for h in range(heads):
                g = h * kv_heads // heads
                want, mag = attention(qkv[at:at + n, h], kv[:, g], kv[:, kv_heads + g], dim ** -0.5,
                                      True)
                assert (np.abs(got[at:at + n, h] - want) <= mag * 2.0 ** -7 + 1e-30).all()
            at += n


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_cache_ops_under_compile(fmt):
    """A step that writes to the cache and attends over it, compiled whole: the cache is mutated
    where it is read afterwards, bit for bit as in the eager step."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    o = torch.ops.w8a8
    table = torch.tensor([[2, 0], [1, 3]], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(5)

    def step(cache, qkv, slots, lens):
        q, k, v = qkv.split((4, 2, 2), 1)
        o.kv_write(cache, k, v, slots, fmt)
        y = o.kv_attention(q, cache, table, lens, None, fmt, None, True, 1, 32)
        rk, rv = o.kv_read(cache, slots, 64, fmt)
        return y + 1.0, rk - rv

    caches = [w8a8.kv_cache(4, 2, 64, 16, fmt=fmt) for _ in range(2)]
    compiled = torch.compile(step, fullgraph=True, backend="aot_eager")
    for pos in range(18):
        qkv = torch.randn(2, 8, 64, generator=g).to(torch.bfloat16).cuda()
        slots = torch.tensor([[2, 0], [1, 3]], device="cuda")[:, pos // 16] * 16 + pos % 16
        lens = torch.full((2,), pos + 1, dtype=torch.int32, device="cuda")
        want = step(caches[0], qkv, slots, lens)
        got = compiled(caches[1], qkv, slots, lens)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(*caches)
    assert caches[0].any()
