"""Refusals of the 8-bit serving entry points, without a GPU: every argument
error comes back before any device work, with its code and a message."""
import ctypes

import pytest

from paper_2608_00916_amd import _lib
from tests import serve_ref as R

FAKE = 1 << 24  # aligned, never dereferenced: every call below fails its checks first
ARG, SHAPE, ALIGN, WS = _lib.MOE_ERR_ARG, _lib.MOE_ERR_SHAPE, _lib.MOE_ERR_ALIGN, _lib.MOE_ERR_WORKSPACE
ref = ctypes.byref


def err():
    return _lib.lib().moe_last_error().decode()


def call(name, want, *args):
    assert getattr(_lib.lib(), name)(*args) == want, (name, args, err())
    assert err()


def test_quant_refusals():
    rows = "moe_i8_quant_rows"
    call(rows, ARG, 0, 128, FAKE, 128, FAKE, FAKE, None)
    call(rows, ARG, 1, 0, FAKE, 128, FAKE, FAKE, None)
    call(rows, ARG, 1, 131072 + 16, FAKE, 1 << 20, FAKE, FAKE, None)
    call(rows, SHAPE, 1, 24, FAKE, 24, FAKE, FAKE, None)
    call(rows, ARG, 1, 128, FAKE, 120, FAKE, FAKE, None)
    call(rows, SHAPE, 1, 128, FAKE, 132, FAKE, FAKE, None)
    call(rows, ARG, 1, 128, None, 128, FAKE, FAKE, None)
    call(rows, ALIGN, 1, 128, FAKE + 8, 128, FAKE, FAKE, None)
    w = "moe_i8_quant_weight"
    call(w, ARG, 0, 128, 8, FAKE, FAKE, FAKE, None)
    call(w, ARG, 65536, 128, 8, FAKE, FAKE, FAKE, None)
    call(w, ARG, 1, 128, 0, FAKE, FAKE, FAKE, None)
    call(w, SHAPE, 1, 8, 8, FAKE, FAKE, FAKE, None)
    call(w, ARG, 1, 128, 8, FAKE, None, FAKE, None)


@pytest.mark.parametrize("d,code", [((0, 8, 128, 0), ARG), ((8, 0, 128, 0), ARG), ((8, 8, 0, 0), ARG),
                                    ((8, 8, 20, 0), SHAPE), ((8, 8, 131088, 0), ARG), ((8, 8, 128, 1), ARG),
                                    ((2 ** 31 - 1, 2 ** 31 - 1, 128, 0), ARG)])
def test_product_dims(d, code):
    d = _lib.MoeI8Dims(*d)
    call("moe_i8_matmul", code, ref(d), FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, None)
    call("moe_i8_linear", code, ref(d), FAKE, 1 << 20, FAKE, FAKE, FAKE, 1 << 40, FAKE, 1 << 40, None)
    assert _lib.lib().moe_i8_linear_workspace_bytes(ref(d)) == 0


def test_product_refusals():
    d = _lib.MoeI8Dims(8, 40, 128, 0)
    call("moe_i8_matmul", ARG, None, FAKE, FAKE, FAKE, FAKE, FAKE, 40, None)
    call("moe_i8_matmul", ARG, ref(d), FAKE, FAKE, FAKE, FAKE, FAKE, 39, None)
    call("moe_i8_matmul", ARG, ref(d), FAKE, None, FAKE, FAKE, FAKE, 40, None)
    call("moe_i8_matmul", ALIGN, ref(d), FAKE, FAKE, FAKE + 4, FAKE, FAKE, 40, None)
    need = _lib.lib().moe_i8_linear_workspace_bytes(ref(d))
    assert need >= 8 * 128 + 8 * 4
    call("moe_i8_linear", WS, ref(d), FAKE, 128, FAKE, FAKE, FAKE, 40, FAKE, need - 1, None)
    call("moe_i8_linear", ARG, ref(d), FAKE, 120, FAKE, FAKE, FAKE, 40, FAKE, need, None)
    call("moe_i8_linear", SHAPE, ref(d), FAKE, 129, FAKE, FAKE, FAKE, 40, FAKE, need, None)


def test_expert_refusals():
    L = _lib.lib()
    w = _lib.MoeI8Experts(*[FAKE] * 6)
    d = _lib.MoeExpertsDims(100, 128, 4, 128, 0)
    need = L.moe_experts_i8_workspace_bytes(ref(d))
    assert need >= 100 * (128 + 3 * 128)
    name = "moe_experts_i8"
    call(name, WS, ref(d), FAKE, FAKE, ref(w), FAKE, FAKE, need - 1, None)
    call(name, ARG, ref(d), FAKE, None, ref(w), FAKE, FAKE, need, None)
    call(name, ARG, ref(d), FAKE, FAKE, None, FAKE, FAKE, need, None)
    call(name, ARG, ref(d), FAKE, FAKE, ref(_lib.MoeI8Experts(*[FAKE] * 5)), FAKE, FAKE, need, None)
    call(name, ARG, ref(_lib.MoeExpertsDims(100, 128, 4, 128, _lib.MOE_F_RECOMPUTE)), FAKE, FAKE, ref(w), FAKE, FAKE, need, None)
    call(name, SHAPE, ref(_lib.MoeExpertsDims(100, 128, 4, 100, 0)), FAKE, FAKE, ref(w), FAKE, FAKE, need, None)
    call(name, ARG, ref(_lib.MoeExpertsDims(100, 128, 4, 262144, 0)), FAKE, FAKE, ref(w), FAKE, FAKE, 1 << 50, None)
    t = _lib.MoeDims(10, 128, 8, 128, 2, 0, 0.0, 0.0)
    need = L.moe_infer_i8_workspace_bytes(ref(t))
    call("moe_infer_i8", WS, ref(t), FAKE, FAKE, ref(w), None, FAKE, FAKE, need - 1, None)
    call("moe_infer_i8", ALIGN, ref(t), FAKE, FAKE + 2, ref(w), None, FAKE, FAKE, need, None)
    t.flags = _lib.MOE_F_MASK
    call("moe_infer_i8", ARG, ref(t), FAKE, FAKE, ref(w), None, FAKE, FAKE, need, None)
    t.E = 12
    call("moe_infer_i8", SHAPE, ref(t), FAKE, FAKE, ref(w), FAKE, FAKE, FAKE, need, None)
    assert L.moe_infer_i8_workspace_bytes(ref(t)) == 0


def cache(n=10, bt=16, heads=2, D=64, k=FAKE):
    return _lib.MoeKvCache(n, bt, heads, D, k, FAKE, FAKE, FAKE)


def batch(B=2, T=5, W=4, table=FAKE):
    return _lib.MoeKvBatch(B, T, W, FAKE, FAKE, table)


def attn(heads=4, max_q=3, max_kv=64, scale=1.0, flags=0):
    return _lib.MoeKvAttn(heads, max_q, max_kv, scale, flags)


@pytest.mark.parametrize("c,code", [(cache(n=0), ARG), (cache(heads=0), ARG), (cache(bt=24), SHAPE), (cache(bt=256), SHAPE),
                                    (cache(D=96), SHAPE), (cache(n=2 ** 28), ARG), (cache(k=None), ARG),
                                    (cache(k=FAKE + 8), ALIGN)])
def test_bad_cache(c, code):
    call("moe_kv_append", code, ref(c), ref(batch()), FAKE, FAKE, 4096, None)
    call("moe_kv_read", code, ref(c), 1, 1, FAKE, FAKE, 5, FAKE, FAKE, None)
    call("moe_kv_attention", code, ref(c), ref(batch()), ref(attn()), FAKE, 4096, FAKE, 4096, FAKE, 1 << 40, None)
    assert _lib.lib().moe_kv_attention_workspace_bytes(ref(c), ref(batch()), ref(attn())) == 0


@pytest.mark.parametrize("b", [batch(B=0), batch(T=-1), batch(W=0), batch(W=2 ** 28), batch(table=None)])
def test_bad_batch(b):
    call("moe_kv_append", ARG, ref(cache()), ref(b), FAKE, FAKE, 4096, None)
    call("moe_kv_attention", ARG, ref(cache()), ref(b), ref(attn()), FAKE, 4096, FAKE, 4096, FAKE, 1 << 40, None)


@pytest.mark.parametrize("a,code", [(attn(heads=3), SHAPE), (attn(heads=0), SHAPE), (attn(max_q=0), ARG),
                                    (attn(max_kv=0), ARG), (attn(scale=float("nan")), ARG), (attn(flags=1), ARG)])
def test_bad_attention(a, code):
    call("moe_kv_attention", code, ref(cache()), ref(batch()), ref(a), FAKE, 4096, FAKE, 4096, FAKE, 1 << 40, None)


def test_cache_call_refusals():
    c, b, a = cache(), batch(), attn()
    call("moe_kv_append", ARG, None, ref(b), FAKE, FAKE, 128, None)
    call("moe_kv_append", ARG, ref(c), ref(b), FAKE, None, 128, None)
    call("moe_kv_append", ARG, ref(c), ref(b), FAKE, FAKE, 120, None)
    call("moe_kv_append", SHAPE, ref(c), ref(b), FAKE, FAKE, 132, None)
    call("moe_kv_append", ALIGN, ref(c), ref(b), FAKE + 2, FAKE, 128, None)
    call("moe_kv_read", ARG, ref(c), 0, 1, FAKE, FAKE, 5, FAKE, FAKE, None)
    call("moe_kv_read", ARG, ref(c), 1, 1, FAKE, FAKE, 5, FAKE, None, None)
    L = _lib.lib()
    need = L.moe_kv_attention_workspace_bytes(ref(c), ref(b), ref(a))
    assert need > 0
    call("moe_kv_attention", WS, ref(c), ref(b), ref(a), FAKE, 256, FAKE, 256, FAKE, need - 1, None)
    call("moe_kv_attention", ARG, ref(c), ref(b), ref(a), FAKE, 248, FAKE, 256, FAKE, need, None)
    call("moe_kv_attention", SHAPE, ref(c), ref(b), ref(a), FAKE, 256, FAKE, 260, FAKE, need, None)
    call("moe_kv_attention", ARG, ref(c), ref(b), ref(a), None, 256, FAKE, 256, FAKE, need, None)
    # no new tokens: nothing to do, nothing else looked at
    assert L.moe_kv_append(ref(c), ref(batch(T=0)), None, None, 0, None) == 0
    assert L.moe_kv_attention(ref(c), ref(batch(T=0)), ref(a), None, 0, None, 0, None, 0, None) == 0
    assert L.moe_kv_read(ref(c), 1, 1, FAKE, FAKE, 0, None, None, None) == 0


def test_plan_refusals():
    P = _lib.MoeKvPlanDims
    ok = [FAKE] * 11
    for d, code in ((P(0, 4, 4, 10, 16, 4), ARG), (P(1, -1, 4, 10, 16, 4), ARG), (P(1, 4, 0, 10, 16, 4), ARG),
                    (P(1, 4, 4, 0, 16, 4), ARG), (P(1, 4, 4, 10, 20, 4), SHAPE), (P(1, 4, 4, 10, 16, -1), ARG),
                    (P(1, 4, 2 ** 28, 10, 16, 4), ARG), (P(1, 4, 4, 2 ** 28, 16, 4), ARG)):
        call("moe_kv_plan", code, ref(d), *ok, None)
    for i in range(11):
        args = list(ok)
        args[i] = None
        call("moe_kv_plan", ARG, ref(P(1, 4, 4, 10, 16, 4)), *args, None)
        args[i] = FAKE + 4
        call("moe_kv_plan", ALIGN, ref(P(1, 4, 4, 10, 16, 4)), *args, None)


def test_reference_pins():
    """The plain forms on values worked by hand."""
    import numpy as np
    q, s = R.quant_rows(np.array([[2.0, -1.0, 0.25, 0.0]]))
    assert q.tolist() == [[127, -64, 16, 0]] and s[0, 0] == 2 / 127  # 63.5 and 15.875
    blk = np.zeros((4, 2))
    blk, s = R.append_block(blk, 9.0, np.array([[1.27, -0.635]], np.float32), 0)
    assert blk[0].tolist() == [127, -64] and abs(s - 0.01) < 1e-8
    blk, s = R.append_block(blk, s, np.array([[2.54, 0.0]], np.float32), 1)
    assert blk[0].tolist() == [64, -32] and blk[1].tolist() == [127, 0] and abs(s - 0.02) < 1e-8
    one = np.ones((2, 1, 2))
    out, mag = R.attention(one, np.array([[[0.0, 0.0]], [[np.log(3.0), 0.0]]]), np.array([[[4.0, 0.0]], [[-8.0, 1.0]]]), 0, 2,
                           True, 1.0)
    assert np.allclose(out[0, 0], [4, 0]) and np.allclose(out[1, 0], [-5, 0.75]) and np.allclose(mag[1, 0], [7, 0.75])
    table = [[3, -1, -1], [-1, -1, -1]]
    got = R.plan([5, 0], [12, 1], table, [0, 1, 2], 3, 14, 8, 16)
    assert got[0] == [0, 12, 13] and got[1] == [17, 1] and table == [[3, 2, -1], [1, -1, -1]]
    assert got[3][:12] == [53 + i for i in range(11)] + [32] and got[3][12:] == [16, -1] and got[5] == [1, 0]
