"""Refusals of a decoding step's entry points, without a GPU, and the 64-bit
forms that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_00916_amd as moe
from paper_2608_00916_amd import _lib
from tests import step_ref as R
from tests.test_serve_abi import ALIGN, ARG, FAKE, SHAPE, WS, call

ref = ctypes.byref
BIG = 1 << 40
P = [FAKE + i * BIG for i in range(12)]  # far apart


def norm(T=4, H=128, flags=0, eps=1e-6):
    return _lib.MoeNormDims(T, H, flags, eps)


@pytest.mark.parametrize("d,code", [(norm(T=0), ARG), (norm(H=0), ARG), (norm(H=32776), ARG), (norm(H=12), SHAPE),
                                    (norm(flags=1), ARG), (norm(eps=0.0), ARG), (norm(eps=-1.0), ARG),
                                    (norm(eps=float("nan")), ARG), (norm(eps=float("inf")), ARG), (norm(eps=1e-40), ARG)])
def test_norm_dims(d, code):
    call("moe_norm_fwd", code, ref(d), P[0], 32768, None, 0, P[1], None, P[2], None, None, None)
    call("moe_norm_bwd", code, ref(d), P[0], 32768, P[1], P[2], 32768, None, 0, P[3], P[4], P[5], BIG, None)
    assert _lib.lib().moe_norm_bwd_workspace_bytes(ref(d)) == 0


def test_norm_refusals():
    d, f = norm(), "moe_norm_fwd"
    x, r, w, h, y, q, s = P[:7]
    call(f, ARG, None, x, 128, r, 128, w, h, y, q, s, None)
    call(f, ARG, ref(d), None, 128, r, 128, w, h, y, q, s, None)
    call(f, ALIGN, ref(d), x, 128, r + 8, 128, w, h, y, q, s, None)
    call(f, ARG, ref(d), x, 120, r, 128, w, h, y, q, s, None)
    call(f, SHAPE, ref(d), x, 132, r, 128, w, h, y, q, s, None)
    call(f, ARG, ref(d), x, 128, r, 64, w, h, y, q, s, None)
    call(f, ARG, ref(d), x, 128, None, 0, w, h, y, q, s, None)  # h without a residual
    call(f, ARG, ref(d), x, 128, r, 128, w, h, None, None, None, None)
    call(f, ARG, ref(d), x, 128, r, 128, w, h, y, q, None, None)
    call(f, ARG, ref(d), x, 128, r, 128, w, h, y, None, s, None)
    call(f, SHAPE, ref(norm(H=136)), x, 136, r, 136, w, h, y, q, s, None)
    # in place only as a whole
    for out in ((x + 16, y), (x + 256, y), (h, x + 256), (h, h), (h, w), (w, y), (h, r + 1008)):
        call(f, ARG, ref(d), x, 128, r, 128, w, *out, q, s, None)
        assert "overlaps" in _lib.lib().moe_last_error().decode()
    call(f, ARG, ref(d), x, 256, r, 128, w, x, y, q, s, None)  # x has gaps
    call(f, ARG, ref(d), x, 128, r, 128, w, h, y, x, s, None)
    call(f, ARG, ref(d), x, 128, r, 128, w, h, y, q, q, None)


def test_norm_backward_refusals():
    d, f = norm(), "moe_norm_bwd"
    h, w, dy, dh, dx, dw, ws = P[:7]
    need = _lib.lib().moe_norm_bwd_workspace_bytes(ref(d))
    assert need >= 128 * 4
    call(f, WS, ref(d), h, 128, w, dy, 128, dh, 128, dx, dw, ws, need - 1, None)
    call(f, ARG, ref(d), h, 128, w, dy, 128, dh, 120, dx, dw, ws, need, None)
    call(f, SHAPE, ref(d), h, 130, w, dy, 128, dh, 128, dx, dw, ws, need, None)
    call(f, ARG, ref(d), h, 128, w, dy, 128, dh, 128, dx, None, ws, need, None)
    call(f, ALIGN, ref(d), h, 128, w, dy, 128, dh, 128, dx + 2, dw, ws, need, None)
    for bad in (h, w, dy + 256, dh + 16):
        call(f, ARG, ref(d), h, 128, w, dy, 128, dh, 128, bad, dw, ws, need, None)
        assert "overlaps" in _lib.lib().moe_last_error().decode()
    call(f, ARG, ref(d), h, 128, w, dy, 128, dh, 256, dh, dw, ws, need, None)  # dh has gaps
    call(f, ARG, ref(d), h, 128, w, dy, 128, dh, 128, dx, dx, ws, need, None)


def test_decode_refusals():
    L = _lib.lib()
    w = _lib.MoeI8Experts(*[FAKE] * 6)
    d = _lib.MoeDims(10, 128, 8, 128, 2, 0, 0.0, 0.0)
    for name, args in (("moe_decode", (FAKE,) * 3), ("moe_decode_i8", (ref(w),))):
        need = getattr(L, name + "_workspace_bytes")(ref(d))
        assert need >= 20 * 128 * 4
        call(name, WS, ref(d), FAKE, FAKE, *args, None, FAKE, FAKE, need - 1, None)
        call(name, ARG, ref(d), None, FAKE, *args, None, FAKE, FAKE, need, None)
        call(name, ALIGN, ref(d), FAKE, FAKE, *args, None, FAKE + 2, FAKE, need, None)
        for bad, code in ((dict(T=65), ARG), (dict(T=0), ARG), (dict(flags=_lib.MOE_F_MASK), ARG), (dict(H=64), SHAPE),
                          (dict(E=12), SHAPE), (dict(top_k=9), ARG), (dict(F=100), SHAPE), (dict(F=1 << 25), ARG)):
            e = _lib.MoeDims(10, 128, 8, 128, 2, 0, 0.0, 0.0)
            for n, v in bad.items():
                setattr(e, n, v)
            call(name, code, ref(e), FAKE, FAKE, *args, None, FAKE, FAKE, 1 << 60, None)
            if "flags" not in bad:
                assert getattr(L, name + "_workspace_bytes")(ref(e)) == 0
    call("moe_decode_i8", ARG, ref(d), FAKE, FAKE, None, None, FAKE, FAKE, BIG, None)
    call("moe_decode_i8", ARG, ref(d), FAKE, FAKE, ref(_lib.MoeI8Experts(*[FAKE] * 5)), None, FAKE, FAKE, BIG, None)
    call("moe_decode", ARG, ref(d), FAKE, FAKE, FAKE, None, FAKE, None, FAKE, FAKE, BIG, None)
    e = _lib.MoeDims(10, 128, 8, 131200, 2, 0, 0.0, 0.0)
    call("moe_decode_i8", ARG, ref(e), FAKE, FAKE, ref(w), None, FAKE, FAKE, 1 << 60, None)


def test_sample_refusals():
    L = _lib.lib()
    for bad in ((0, 8, 0), (65536, 8, 0), (4, 0, 0), (4, 2 ** 20 + 1, 0), (4, 8, 1)):
        d = _lib.MoeSampleDims(*bad)
        call("moe_sample", ARG, ref(d), FAKE, BIG, None, None, None, None, FAKE, FAKE, None, FAKE, BIG, None)
        assert L.moe_sample_workspace_bytes(ref(d)) == 0
    d = _lib.MoeSampleDims(4, 1000, _lib.MOE_F_LOGITS_FP32)
    need = L.moe_sample_workspace_bytes(ref(d))
    ok = [ref(d), FAKE, 1000, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, need, None]
    for at, v, code in ((0, None, ARG), (1, None, ARG), (1, FAKE + 2, ALIGN), (2, 999, ARG), (3, FAKE + 2, ALIGN),
                        (4, FAKE + 1, ALIGN), (7, None, ARG), (8, None, ARG), (9, FAKE + 2, ALIGN), (10, None, ARG),
                        (10, FAKE + 8, ALIGN), (11, need - 1, WS), (2, 1 << 33, ARG)):
        args = list(ok)
        args[at] = v
        call("moe_sample", code, *args)


def test_tensors_that_do_not_fit():
    def t(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype)

    f32 = torch.float32
    d = moe.norm_dims(4, 16)
    with pytest.raises(ValueError, match="^x has shape"):
        moe.moe_norm_fwd(d, t(3, 16), None, t(16), y=t(4, 16))
    with pytest.raises(ValueError, match="^scale has shape"):
        moe.moe_norm_fwd(d, t(4, 16), None, t(16), q=t(4, 16, dtype=torch.int8), scale=t(3, dtype=f32))
    with pytest.raises(ValueError, match="^dw has shape"):
        moe.moe_norm_bwd(d, t(4, 16), t(16), t(4, 16), None, t(4, 16), t(8), t(64))
    with pytest.raises(ValueError, match="must be on the GPU"):
        moe.moe_norm_fwd(d, t(4, 16), None, t(16), y=t(4, 16))
    d = _lib.MoeDims(4, 128, 8, 128, 2, 0, 0.0, 0.0)
    w = t(8, 128, 128)
    for name, args in dict(x=(t(3, 128), t(128, 8), w, w, w, None, t(4, 128)),
                           w_down=(t(4, 128), t(128, 8), w, w, w[:7], None, t(4, 128)),
                           y=(t(4, 128), t(128, 8), w, w, w, None, t(3, 128))).items():
        with pytest.raises(ValueError, match=f"^{name} has"):
            moe.moe_decode(d, *args, t(64, dtype=torch.uint8))
    d = moe.sample_dims(4, 10)
    with pytest.raises(ValueError, match="^logits has shape"):
        moe.moe_sample(d, t(4, 9, dtype=f32), None, None, None, None, t(4, dtype=f32), t(4, dtype=torch.int32), None, t(64))
    with pytest.raises(ValueError, match='^out must be'):
        moe.RMSNorm(4, t(16), out="fp8")
    with pytest.raises(moe.MoeError):
        moe.RMSNorm(4, t(24), out="i8")
    with pytest.raises(moe.MoeError):
        moe.MoEDecode(65, 128, 8, 128, 2, device="cpu")
    with pytest.raises(moe.MoeError):
        moe.Sampler(1, 2 ** 20 + 1, device="cpu")


def test_masks_and_devices_that_do_not_fit(monkeypatch):
    from paper_2608_00916_amd import step
    d = _lib.MoeDims(4, 128, 8, 128, 2, 0, 0.0, 0.0)
    for mask in (torch.ones(4, dtype=torch.uint8), torch.ones(4, dtype=torch.bool)):
        with pytest.raises(ValueError, match="no mask"):
            step._mask(mask, d)
    d.flags = _lib.MOE_F_MASK
    with pytest.raises(ValueError, match="must be uint8 or bool"):
        step._mask(torch.ones(4), d)
    with pytest.raises(ValueError, match="token_mask has"):
        step._mask(torch.ones(3, dtype=torch.bool), d)

    class There:
        def get_device(self):
            return 1

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="on device 1, the current one is 0"):
        step._on(There(), None)

    class Here:
        def get_device(self):
            return 0

    with pytest.raises(ValueError, match="on device 1, the current one is 0"):  # not the first alone
        step._on(Here(), 0, None, There())
    assert step._on(Here(), 17, None, Here()) == 17


def test_norm_workspace_of_the_most_rows():
    """As many shares of dw as for fewer rows: their number must not overflow near 2^31 rows."""
    for H in (8, 2048, 32768):
        few, most = (moe.moe_norm_bwd_workspace_bytes(moe.norm_dims(T, H)) for T in (10 ** 6, 2 ** 31 - 1))
        assert 0 < most == few, H


def test_norm_backward_form_against_differences():
    """The 64-bit gradient is that of the 64-bit norm, by central differences of sum(dy v) + sum(dh h)."""
    g = np.random.default_rng(0)
    h, w, dy, dh = g.standard_normal((3, 8)), g.standard_normal(8), g.standard_normal((3, 8)), g.standard_normal((3, 8))

    def loss(h, w):
        return (R.norm(h, w, 1e-3)[0] * dy).sum() + (h * dh).sum()

    dx, dw, _, _ = R.norm_bwd(h, w, dy, dh, 1e-3)
    for at in np.ndindex(h.shape):
        e = np.zeros_like(h)
        e[at] = 1e-6
        assert abs((loss(h + e, w) - loss(h - e, w)) / 2e-6 - dx[at]) < 1e-7
    for c in range(8):
        e = np.zeros(8)
        e[c] = 1e-6
        assert abs((loss(h, w + e) - loss(h, w - e)) / 2e-6 - dw[c]) < 1e-7


def test_sample_form():
    """The 64-bit choice on a row whose answers are known by hand: weights 1, 2, 4, 1 (in 8ths), ties to the lower index."""
    row = np.log(np.array([1.0, 2.0, 4.0, 1.0]))
    assert [R.sample(row, u)[0] for u in (0.0, 0.124, 0.126, 0.374, 0.376, 0.874, 0.876, 1.0)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [R.sample(row, u, top_k=2)[0] for u in (0.0, 0.332, 0.334)] == [1, 1, 2]
    assert [R.sample(row, u, top_k=3)[0] for u in (0.0, 0.99)] == [0, 2]
    assert [R.sample(row, 0.99, top_p=p)[0] for p in (0.0, 0.49, 0.51, 0.76, 0.9)] == [2, 2, 2, 2, 3]
    assert [R.sample(row, 0.0, top_p=p)[0] for p in (0.49, 0.51, 0.76, 0.9)] == [2, 1, 0, 0]
    assert R.sample(row, 0.0, min_p=0.3)[0] == 1 and R.sample(row, 0.0, min_p=2.0)[0] == 2
    assert R.sample(row, 0.9, temperature=0.0) == (2, 0.0)
    assert np.isclose(R.sample(row, 0.5)[1], np.log(0.5))
    assert R.sample(np.array([-np.inf, np.nan]), 0.5)[0] == -1
