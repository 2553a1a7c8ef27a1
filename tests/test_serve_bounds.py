"""What the 8-bit serving operators may be off by, from the roundings that they
make and no more, against 64 bits.

Attention: softmax weights enter the product with the values in fp16 (11
significant bits: 2^-11 of each), below 2^-14 at its fixed step (half of 2^-24,
against a largest weight of at least 2^7); the sum they are divided by is that
of the unrounded weights.  Scores of a few dozen and their exponentials in fp32
add less than 2^-14.  The output is rounded to bf16: 2^-8 of itself.

Experts: the activation stays in fp32 until its rounding to int8, so that only
values next to a boundary take another step: a value is off by up to 2^-21 of
itself, 2^-14 of a step, on either side of a boundary, which at most 2^-13 of
the values are near.  Of n values one, or that share, may be off by a step
against 10 steps rms; the output is rounded to bf16.
"""
import importlib.util
import os

import numpy as np
import pytest

from tests import serve_ref as R
from tests.test_gpu_serve import BF, Pages, bf16, dev, expert_weights, gen, host, i32, say

gpu = pytest.mark.gpu


def attention_bound(ref, mag, keys, top):
    """`top`: largest value that the cache can hold."""
    t = (2.0 ** -11 + 2.0 ** -14) * mag + keys * 2.0 ** -32 * top
    return t + BF * (np.abs(ref) + t)


def expert_bound(n):
    """Relative to the norm of the rows of n activation values."""
    return BF + np.sqrt(2.0 ** -13 + 1.0 / n) / 10


def to_bf16(x):
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + (u >> 16 & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def test_the_attention_bound_tells_fp16_weights_from_bf16():
    g = gen(51)
    bad = {np.float16: 0, "bf16": 0}
    for _ in range(200):
        n = int(g.integers(2, 6))
        v8 = g.integers(-127, 128, (n, 64)).astype(np.float64)
        c = g.uniform(0.5, 1.5, n) / 64
        s = 0.5 * g.standard_normal(n)
        p = np.exp(s - s.max()) / np.exp(s - s.max()).sum()
        ref, mag = p @ (v8 * c[:, None]), p @ np.abs(v8 * c[:, None])
        w = 128.0 * c * np.exp(s) / (c * np.exp(s)).max()
        for kind in bad:
            r = to_bf16(w).astype(np.float64) if kind == "bf16" else w.astype(kind).astype(np.float64)
            out = to_bf16(r @ v8 / (w / c).sum()).astype(np.float64)
            bad[kind] += (np.abs(out - ref) > attention_bound(ref, mag, n, 127 * 1.5 / 64)).sum()
    assert bad[np.float16] == 0 and bad["bf16"] > 100


@gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,kv_heads,bt", [(64, 2, 16), (128, 1, 64)])
@pytest.mark.parametrize("n", [1, 4, 40])
def test_attention_is_off_by_its_own_roundings(n, D, kv_heads, bt, causal):
    """Few keys of like weight, whose values cancel: what the weights' rounding leaves shows."""
    import paper_2608_00916_amd as moe
    say("attention bound", n, D, kv_heads, bt, causal)
    kv = [2, 3, 5, 17, 64, 200, 3000]
    new = [min(n, L) for L in kv]
    pg = Pages(gen(D + n), kv, bt, kv_heads, D)
    start = np.concatenate([[0], np.cumsum(new)])
    q = bf16(2.0 * gen(n).standard_normal((sum(new), 8, D)))
    scale = 0.25 / D ** 0.5
    op = moe.KVAttention(pg.cache, sum(new), 8, len(kv), n, max(kv), causal, scale)
    got = host(op.forward(q, pg.cache, dev(pg.table), i32(start), i32(kv)))
    for b, L in enumerate(kv):
        rows = slice(start[b], start[b + 1])
        ref, mag = R.attention(host(q)[rows], *pg.rows(b, L), L - new[b], L, causal, scale)
        assert (np.abs(got[rows] - ref) <= attention_bound(ref, mag, L, 127 * 1.5 / 64)).all(), (b, L)


@gpu
@pytest.mark.parametrize("rows,counts,H,F", [
    (1, [1], 128, 128),
    (300, [128, 129, 0, 43], 128, 384),
    (700, [257, 0, 131, 300], 384, 640),
    (520, [1] * 8 + [512], 512, 256),
    (4500, [1401, 0, 2899, 200], 1024, 640),
    (6144, [64] * 96, 256, 256),
    (12000, [5001, 0, 6743, 200], 1024, 640),
])
def test_experts_are_off_by_their_own_roundings(rows, counts, H, F):
    """Every row tile, part-filled ones among them."""
    import paper_2608_00916_amd as moe
    say("experts bound", rows, counts, H, F)
    g = gen(52)
    w8, w = expert_weights(g, len(counts), H, F)
    x = bf16(g.standard_normal((rows, H)))
    got, xs, r0 = host(moe.MoEExpertsI8(rows, H, len(counts), F).forward(x, i32(counts), w8)), host(x), 0
    for e, n in enumerate(counts):
        if n:
            ref = R.expert(xs[r0:r0 + n], w[0][e], w[1][e], w[2][e])
            assert np.linalg.norm(got[r0:r0 + n] - ref) <= expert_bound(n * F) * np.linalg.norm(ref), e
        r0 += n


@gpu
@pytest.mark.parametrize("T,H,E,F,k,masked", [(1, 128, 8, 128, 2, False), (70, 256, 16, 128, 4, True),
                                              (600, 512, 32, 384, 8, False), (3000, 512, 32, 384, 8, False)])
def test_infer_against_64_bits(T, H, E, F, k, masked):
    """The block's forward from x alone: logits, selection, gates, experts and combine in 64 bits."""
    import paper_2608_00916_amd as moe
    say("infer bound", T, H, E, F, k, masked)
    g = gen(53)
    w8, w = expert_weights(g, E, H, F)
    x, w_r = bf16(g.standard_normal((T, H))), bf16(0.05 * g.standard_normal((H, E)))
    mask = (g.random(T) > 0.3).astype(np.uint8) if masked else np.ones(T, np.uint8)
    got = host(moe.MoEInferI8(T, H, E, F, k, mask=masked).forward(x, w_r, w8, dev(mask) if masked else None))
    xs = host(x)
    z = xs @ host(w_r)
    order = np.argsort(-z, axis=1, kind="stable")
    top = np.take_along_axis(z, order, 1)
    clear = top[:, k - 1] - top[:, min(k, E - 1)] > 1e-4 if k < E else np.ones(T, bool)  # fp32 logits may swap the others
    gate = np.exp(top[:, :k] - top[:, :1])
    gate /= gate.sum(1, keepdims=True)
    ref, mag = np.zeros((T, H)), np.zeros(T)
    for e in range(E):
        t, j = np.nonzero(order[:, :k] == e)
        if len(t):
            o = R.expert(xs[t], w[0][e], w[1][e], w[2][e])
            ref[t] += gate[t, j, None] * o
            mag[t] += gate[t, j] * np.linalg.norm(o, axis=1)
    assert not got[mask == 0].any() and clear.mean() > 0.9
    at = (mask != 0) & clear
    err = np.linalg.norm(got - ref, axis=1)
    assert (err <= expert_bound(F) * mag + BF * np.linalg.norm(ref, axis=1))[at].all()
    # of many tokens together the steps that are off average out
    if T >= 600:
        assert np.linalg.norm(err[at]) <= np.linalg.norm((expert_bound(T * F) * mag + BF * np.linalg.norm(ref, axis=1))[at])


def example():
    spec = importlib.util.spec_from_file_location("serve_int8", os.path.join(
        os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_int8.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    return ex


@gpu
@pytest.mark.parametrize("part", ["attention", "experts"])
def test_the_example_part_by_part(part):
    """What attention and the experts add to x, each without the other and larger than x, so that the
    roundings of their sum to bf16 stay under 2^-7 of what is added.  A rounding of normal values to
    8 bits is off by 5 / 127 / sqrt(12) = 1.1 percent rms for a largest one of 5 sigma; attention takes
    six (x, weights, keys, values and their second rounding, rows, weights), the experts x twice over,
    three weights and an activation of 8 sigma: 2.8 and 3.7 percent."""
    import torch
    import paper_2608_00916_amd as moe
    say("example", part)
    ex = example()
    B, H, steps = 4, 256, 2
    m = ex.Layer(H, heads=32, kv_heads=4, D=128, E=16, F=768, k=8)
    m.qkv *= 4  # scores that matter
    m.out *= 100 if part == "attention" else 0
    m.down *= 0 if part == "attention" else 400
    m.qkv8, m.out8 = moe.moe_i8_quant_weight(m.qkv), moe.moe_i8_quant_weight(m.out)
    m.experts8 = moe.i8_weights(*(t for w in (m.gate, m.up, m.down) for t in moe.moe_i8_quant_weight(w)))
    g = gen(54)
    lens = [40, 1, 33, 64]
    prompts = [bf16(g.standard_normal((n, H))) for n in lens]
    server = ex.Server(m, B, 64 + steps)
    server.step(torch.cat(prompts), i32(lens), 64)
    one = i32([1] * B)
    for _ in range(steps):
        x = bf16(g.standard_normal((B, H)))
        h = server.step(x, one, 1)
        prompts = [torch.cat([p, x[b:b + 1]]) for b, p in enumerate(prompts)]
    for b in range(B):
        add = ex.reference(m, prompts[b]).double() - x[b].double()
        assert add.norm() > x[b].double().norm()
        assert (h[b].double() - x[b].double() - add).norm() <= 0.05 * add.norm(), b
