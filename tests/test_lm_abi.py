"""The entry points of the norm, the appending cache write, tree attention and log probabilities
without a GPU: what they refuse, before any launch, and what their references compute."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2606_14598_amd as w8a8
from _lm_ref import (cos_sin, f32_inverse_rms, int8_rows, logprobs, rotate, tree_bits, tree_visible)

P = ctypes.c_void_p
F, ODD = P(256), P(264)      # never dereferenced: validation fails first
OK, NULL, SHAPE, KOVER, WORK, ARG = 0, 1, 2, 3, 5, 6
CACHE = (4, 16, 2, 128, 0)
BAD_CACHES = [(8, 8, 2, 128, 0), (4, 20, 2, 128, 0), (4, 16, 0, 128, 0), (4, 16, 2, 96, 0),
              (4, 16, 2, 128, 2), (-1, 16, 2, 128, 0)]


@pytest.fixture(scope="module")
def lib():
    return w8a8.load_library()


def test_norm_refusals(lib):
    a, b = lib.w8a8_rms_norm_quantize, lib.w8a8_rms_norm_mx4_quantize
    for f in (a, b):
        assert f(F, None, None, None, 1e-6, -1, 64, F, F, None) == SHAPE
        assert f(F, None, None, None, 1e-6, 4, -1, F, F, None) == SHAPE
        assert f(F, None, None, None, 1e-6, 1 << 62, 1 << 20 if f is b else 1 << 17, F, F, None) == SHAPE
        for eps in (0.0, -1e-6, float("nan"), float("inf")):
            assert f(F, None, None, None, eps, 4, 64, F, F, None) == ARG
        for x, codes, scales in ((None, F, F), (F, None, F), (F, F, None)):
            assert f(x, None, None, None, 1e-6, 4, 64, codes, scales, None) == NULL
        assert f(F, F, None, None, 1e-6, 4, 64, F, F, None) == NULL      # a residual, no sum
        assert f(None, None, None, None, 1e-6, 0, 64, None, None, None) == OK
    assert a(F, None, None, None, 1e-6, 4, w8a8.MAX_K + 1, F, F, None) == KOVER
    assert b(F, None, None, None, 1e-6, 4, w8a8.MX4_MAX_K + 1, F, F, None) == KOVER
    assert b(F, None, None, None, 1e-6, 4, 64, ODD, F, None) == ARG
    assert b(F, None, None, None, 1e-6, 4, 64, F, ODD, None) == ARG
    assert b(None, None, None, None, 1e-6, 4, 0, None, None, None) == OK
    assert a(None, None, None, None, 1e-6, 4, 0, None, None, None) == NULL   # scales are written


def test_norm_refuses_what_its_formula_has_no_result_for(lib):
    """An eps whose inverse root is past float32 (rows of zeros would be NaN), a sum that overwrites other
    elements than its own."""
    for f in (lib.w8a8_rms_norm_quantize, lib.w8a8_rms_norm_mx4_quantize):
        for eps in (1e-100, 2.0 ** -127):
            assert f(F, None, None, None, eps, 4, 64, F, F, None) == ARG
        for x, r, s in ((1024, 8192, 1026), (1024, 8192, 1022), (8192, 1024, 1024 + 2 * 4 * 64 - 2),
                        (8192, 8192 + 4096, 8192 + 4096 - 2 * 4 * 64 + 2)):
            assert f(P(x), P(r), P(s), None, 1e-6, 4, 64, P(1 << 20), P(1 << 20), None) == ARG


def test_append_refuses_queries_over_its_inputs(lib):
    """Queries written where queries, keys or values are read: whole, the first or last element, and the
    gaps between heads."""
    T, q_heads, heads, dim = 3, 8, 2, 128

    def call(q, k, v, out, q_token=q_heads * dim, q_head=dim):
        return lib.w8a8_kv_append(F, *CACHE, P(q), q_token, q_head, q_heads, P(k), heads * dim, dim, P(v),
                                  heads * dim, dim, F, F, 1, None, F, 64, 0, T, P(out), None)
    size, far = 2 * T * q_heads * dim, (1 << 24, 1 << 25, 1 << 26)
    for q_token, q_head in ((q_heads * dim, dim), (2 * q_heads * dim, dim), (dim, T * dim)):
        last = 2 * ((T - 1) * q_token + (q_heads - 1) * q_head + dim - 1)
        for out in (far[0], far[0] + last, far[0] - size + 2, far[0] + 2 * dim):
            assert call(*far, out, q_token, q_head) == ARG
    for at in far[1:]:
        assert call(*far, at) == ARG and call(*far, at + 2 * (T * heads * dim - 1)) == ARG


def test_append_refusals(lib):
    def call(cache=F, shape=CACHE, q=F, q_token=1024, q_head=128, q_heads=8, k=F, k_token=256,
             k_head=128, v=F, v_token=256, v_head=128, slots=F, positions=F, axes=1, sections=None,
             inv_freq=F, pairs=64, interleaved=0, T=3, out=F):
        sec = None if sections is None else (ctypes.c_int32 * len(sections))(*sections)
        return lib.w8a8_kv_append(cache, *shape, q, q_token, q_head, q_heads, k, k_token, k_head, v,
                                  v_token, v_head, slots, positions, axes, sec, inv_freq, pairs,
                                  interleaved, T, out, None)
    for c in BAD_CACHES:
        assert call(shape=c) == ARG
    for bad in (dict(pairs=-1), dict(pairs=65), dict(interleaved=2), dict(axes=0), dict(axes=5),
                dict(q_heads=-1), dict(axes=2, sections=(32, 31)), dict(axes=2, sections=(-1, 65)),
                dict(axes=2, sections=(64, 1)), dict(axes=3, sections=(2 ** 31 - 1, 2, 63)),
                dict(cache=ODD), dict(q_token=-1), dict(q_head=-1), dict(k_token=-1),
                dict(k_head=-1), dict(v_token=-1), dict(v_head=-1)):
        assert call(**bad) == ARG, bad
    for bad in (dict(k=None), dict(v=None), dict(slots=None), dict(q=None), dict(out=None),
                dict(positions=None), dict(inv_freq=None), dict(cache=None), dict(axes=2)):
        assert call(**bad) == NULL, bad
    assert call(T=-1) == SHAPE and call(T=1 << 60) == SHAPE
    assert call(T=0, k=None, v=None, slots=None, q=None, out=None) == OK


def test_tree_refusals(lib):
    def call(q=F, cache=F, shape=CACHE, table=F, width=4, lens=F, starts=F, T=6, seqs=3, group=4,
             scale=0.1, tree=F, words=1, max_q=4, max_kv=64, out=F, ws=F, n=1 << 40):
        return lib.w8a8_kv_tree_attention(q, 1024, 128, cache, *shape, table, 4, width, lens, starts,
                                          T, seqs, group, scale, tree, words, max_q, max_kv, out, ws,
                                          n, None)
    for c in BAD_CACHES:
        assert call(shape=c) == ARG
    for bad in (dict(words=0), dict(words=65), dict(group=0), dict(scale=float("nan")), dict(cache=ODD)):
        assert call(**bad) == ARG, bad
    for bad in (dict(tree=None), dict(q=None), dict(out=None), dict(lens=None), dict(table=None)):
        assert call(**bad) == NULL, bad
    for bad in (dict(T=-1), dict(seqs=0), dict(max_q=-1), dict(max_kv=-1), dict(starts=None, seqs=4), dict(width=1 << 30)):
        assert call(**bad) == SHAPE, bad
    assert call(T=0, tree=None) == OK
    # long enough for several parts
    big = dict(T=64, seqs=1, max_q=64, max_kv=100000, width=7000)
    size = lib.w8a8_kv_tree_attention_workspace_bytes
    need = size(16, 2, 128, 0, 4, 64, 1, 64, 100000)
    assert size(16, 2, 128, 0, 4, 64, 1, 64, 512) == 0 and size(16, 2, 96, 0, 4, 64, 1, 64, 100000) == 0
    assert size(16, 2, 128, 0, 4, 64, 64, 0, 100000) == size(16, 2, 128, 0, 4, 64, 64, 1, 100000) > 0
    assert need > 0
    assert call(**big, n=need - 1) == WORK and call(**big, ws=None) == WORK and call(**big, ws=P(128)) == WORK


def test_logprobs_refusals(lib):
    def call(x=F, f32=0, stride=5000, T=3, V=5000, tokens=F, top=5, temperature=1.0, logp=F, ent=F,
             tl=F, ti=F, ws=F, n=1 << 40):
        return lib.w8a8_token_logprobs(x, f32, stride, T, V, tokens, top, temperature, logp, ent, tl,
                                       ti, ws, n, None)
    for bad in (dict(f32=2), dict(top=-1), dict(top=65), dict(temperature=0.0),
                dict(temperature=-1.0), dict(temperature=float("nan")),
                dict(temperature=float("inf")), dict(temperature=1e-45), dict(temperature=3e38)):
        assert call(**bad) == ARG, bad
    for bad in (dict(T=-1), dict(V=0), dict(V=1 << 31), dict(stride=-1), dict(V=4, top=5),
                dict(T=1 << 60, V=1 << 20)):
        assert call(**bad) == SHAPE, bad
    for name in ("x", "tokens", "logp", "ent", "tl", "ti"):
        assert call(**{name: None}) == NULL
    assert call(T=0, x=None) == OK
    need = lib.w8a8_token_logprobs_workspace_bytes(1, 131072, 20)
    assert need > 0 and lib.w8a8_token_logprobs_workspace_bytes(5000, 131072, 20) == 0
    big = dict(T=1, V=131072, stride=131072, top=20)
    assert call(**big, n=need - 1) == WORK and call(**big, ws=None) == WORK and call(**big, ws=P(128)) == WORK
    assert lib.w8a8_token_logprobs_workspace_bytes(1, 0, 0) == 0


def test_binding_refuses_what_is_not_on_a_device():
    x, w = torch.zeros(3, 64, dtype=torch.bfloat16), torch.ones(64)
    with pytest.raises(ValueError):
        w8a8.rms_norm_quantize(x, w)
    with pytest.raises(ValueError):
        w8a8.rms_norm_quantize(x, w, fmt="fp8")
    with pytest.raises(TypeError):
        w8a8.rms_norm_quantize(x.float(), w)
    t = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(TypeError):
        w8a8.token_logprobs(x.half(), t)
    with pytest.raises(ValueError):
        w8a8.token_logprobs(x, t)
    cache = w8a8.kv_cache(2, 2, 64, 16, device="cpu")
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        w8a8.kv_append(cache, k, k, t, t, torch.ones(32))
    with pytest.raises(TypeError):
        w8a8.kv_tree_attention(k, cache, t, t, None)


# ---------------------------------------------------------------- the references, by hand

def test_references_on_worked_cases():
    r, near = f32_inverse_rms(np.array([[3.0, 4.0], [0.0, 0.0]]), 1e-6)
    assert r[0] == np.float32(1 / np.sqrt(12.5 + 1e-6)) and r[1] == np.float32(1000.0) and not near.any()
    q, s = int8_rows(np.array([[1.0, -2.0, 0.0], [0, 0, 0]], np.float32))
    assert q.tolist() == [[64, -127, 0], [0, 0, 0]] and s[0] == np.float32(2) / np.float32(127) and s[1] == 0
    c, sn, _ = cos_sin(np.array([[0, 1], [2, 3]]), np.array([1.0, 0.5], np.float32), (1, 1))
    assert c[0, 0] == 1 and c[1, 0] == np.float32(np.cos(2.0)) and sn[1, 1] == np.float32(np.sin(1.5))
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    quarter = (np.array([[0.0, 0.0]], np.float32), np.array([[1.0, 1.0]], np.float32))
    assert rotate(x, *quarter, False).tolist() == [[[-3, -4, 1, 2, 5]]]
    assert rotate(x, *quarter, True).tolist() == [[[-2, 1, -4, 3, 5]]]
    bits = tree_bits([-1, 0, 0, 1], 1)
    assert bits[:, 0].tolist() == [1, 3, 5, 11]
    see = tree_visible(bits, 4, 6)
    assert see[2].tolist() == [True, True, True, False, True, False]
    assert tree_visible(bits, 4, 3)[3].tolist() == [True, False, True]    # node 0 is not cached
    lp, h, tl, ti = logprobs(np.array([[0.0, np.log(3.0), -np.inf]]), np.array([0]), 2, 1.0)
    assert np.isclose(lp[0], np.log(0.25)) and ti.tolist() == [[1, 0]] and np.isclose(tl[0, 0], np.log(0.75))
    assert np.isclose(h[0], -(0.25 * np.log(0.25) + 0.75 * np.log(0.75)))


def test_tree_workspace_does_not_grow_with_the_call(lib):
    """Partial results of 8 / 3 of the workgroups that run at once (512 of two a CU, 256 above 128
    channels), 128 rows of dim + 4 float32 each, and notes of 32 bytes: whatever the queries and sequences.
    (Up to 32 rows a sequence another kernel may run, which may need none.)"""
    size = lib.w8a8_kv_tree_attention_workspace_bytes
    for dim, at_once in ((64, 512), (128, 512), (192, 256), (256, 256)):
        most = (8 * at_once / 3 + 1) * 128 * (dim + 4) * 4 + (4 * at_once / 3 + 2) * 32
        for seqs in (1, 3, 64, 512):
            for nodes in (13, 60, 300, 4000):
                for max_kv in (4097, 32768, 1 << 24):
                    for heads, group in ((8, 4), (1, 64), (128, 1)):
                        n = size(64, heads, dim, 0, group, seqs * nodes, seqs, nodes, max_kv)
                        assert n <= most and (n > 0 or nodes * group <= 32), (dim, seqs, nodes, max_kv, heads, group, n)


def test_tree_workspace_of_few_rows_does_not_grow_with_padding(lib):
    """Calls laid out for more queries than their sequences have (q_starts may end before T), and a max_q
    below what there is: up to 2^27 bytes."""
    size = lib.w8a8_kv_tree_attention_workspace_bytes
    for dim in (64, 128, 192, 256):
        for heads, group in ((8, 4), (1, 1), (18, 1), (128, 1)):
            for T in (16, 1024, 8192, 100000):
                for seqs, max_q in ((1, 4), (2, 1), (4, 4), (64, 2), (600, 1)):
                    for max_kv in (513, 8192, 131072, 1 << 24):
                        assert size(64, heads, dim, 0, group, T, seqs, max_q, max_kv) <= 1 << 27
