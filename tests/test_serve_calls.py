"""Argument checks of the 8-bit serving operators that need no GPU."""
import ctypes

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
