"""Argument checks of the 8-bit serving operators that need no GPU."""
import ctypes

import pytest
import torch

import paper_2608_00916_amd as moe
from paper_2608_00916_amd import _lib
from tests.test_serve_abi import FAKE, call

ref = ctypes.byref


def test_plan_refuses_lengths_that_overlap_in_part():
    d = _lib.MoeKvPlanDims(100, 4, 4, 10, 16, 4)
    old, new, table, ids, n_free, start, kv, pos, slots, seq, state = (FAKE + i * (1 << 16) for i in range(11))
    for at in (old, new):
        for shift in (-384, -16, 16, 384):
            call("moe_kv_plan", _lib.MOE_ERR_ARG, ref(d), old, new, table, ids, n_free, start, at + shift, pos, slots, seq,
                 state, None)
            assert "overlaps" in _lib.lib().moe_last_error().decode()


def test_plan_without_a_stack_needs_no_ids():
    """The stack is looked at only where it has entries: what is refused here is `state`."""
    for cap, name in ((0, "state"), (1, "free_ids")):
        d = _lib.MoeKvPlanDims(1, 4, 4, 10, 16, cap)
        args = [FAKE] * 11
        args[3] = None
        if cap == 0:
            args[10] = None
        call("moe_kv_plan", _lib.MOE_ERR_ARG, ref(d), *args, None)
        assert _lib.lib().moe_last_error().decode().startswith(name)


def test_tensors_that_are_too_small():
    """The functions refuse a tensor of fewer elements than the call reads or writes, before anything else of it."""
    def t(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype)

    def refused(name, f, *args):
        with pytest.raises(ValueError, match=f"^{name} has"):
            f(*args)

    f32, i32, i8 = torch.float32, torch.int32, torch.int8
    d = moe.i8_dims(4, 32, 16)
    x, b, s, out, ws = t(4, 16), t(32, 16, dtype=i8), t(32, dtype=f32), t(4, 32), t(4096, dtype=torch.uint8)
    refused("b", moe.moe_i8_linear, d, x, b[:31], s, out, ws)
    refused("b_scale", moe.moe_i8_linear, d, x, b, s[:31], out, ws)

    d = moe.experts_dims(8, 128, 2, 128)
    w = _lib.MoeI8Experts(*[FAKE] * 6)
    xp, counts = t(8, 128), t(2, dtype=i32)
    refused("xp", moe.moe_experts_i8, d, xp[:7], counts, w, xp, ws)
    refused("counts", moe.moe_experts_i8, d, xp, counts[:1], w, xp, ws)
    refused("o", moe.moe_experts_i8, d, xp, counts, w, xp[:7], ws)
    w.shape = (2, 128, 256)
    with pytest.raises(ValueError, match="weights of"):
        moe.moe_experts_i8(d, xp, counts, w, xp, ws)

    d = _lib.MoeDims(8, 128, 8, 128, 2, 0, 0.0, 0.0)
    w = _lib.MoeI8Experts(*[FAKE] * 6)
    w_r, mask = t(128, 8), t(8, dtype=torch.uint8)
    refused("x", moe.moe_infer_i8, d, xp[:7], w_r, w, None, xp, ws)
    refused("w_r", moe.moe_infer_i8, d, xp, w_r[:127], w, None, xp, ws)
    refused("y", moe.moe_infer_i8, d, xp, w_r, w, None, xp[:7], ws)
    refused("token_mask", moe.moe_infer_i8, d, xp, w_r, w, mask[:7], xp, ws)

    d = _lib.MoeKvPlanDims(3, 5, 2, 10, 16, 4)
    sizes = dict(old_len=3, new_len=3, block_table=6, free_ids=4, n_free=1, row_start=4, kv_len=3, positions=5, slots=5,
                 seq=5, state=2)
    for name in sizes:
        refused(name, moe.moe_kv_plan, d, *(t(n - (k == name), dtype=i32) for k, n in sizes.items()))
