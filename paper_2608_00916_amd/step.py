"""A decoding step's operators around the products and the attention: the sum
with the residual and its norm (forward and backward), the expert layer for a
few tokens, and the next token from the logits (the decoding part of the C ABI
in include/moe.h).

As in the rest of the package the functions turn tensors into pointers and the
classes own the caller-side buffers; the work runs in the library's kernels.
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib
from ._lib import (MOE_DECODE_MAX_T, MOE_F_DW_FP32, MOE_F_LOGITS_FP32, MOE_F_MASK, MOE_NORM_MAX_H, MOE_SAMPLE_MAX_V,
                   MoeDims, MoeError, MoeI8Experts, MoeNormDims, MoeSampleDims, check, lib)
from .serve import _check_weights, _Held, _least, _p, _rows, _s, _shape, _take_ws, _ws

__all__ = [
    "norm_dims", "moe_norm_fwd", "moe_norm_bwd_workspace_bytes", "moe_norm_bwd", "moe_decode_workspace_bytes",
    "moe_decode", "moe_decode_i8_workspace_bytes", "moe_decode_i8", "sample_dims", "moe_sample_workspace_bytes",
    "moe_sample", "RMSNorm", "MoEDecode", "MoEDecodeI8", "Sampler", "MOE_F_LOGITS_FP32", "MOE_NORM_MAX_H",
    "MOE_DECODE_MAX_T", "MOE_SAMPLE_MAX_V",
]

_ref = ctypes.byref
_bf, _f32, _i32 = torch.bfloat16, torch.float32, torch.int32


def _bf_rows(name, t, shape):
    """Pointer and row pitch of bf16 rows of a shape; the common case first, in few calls."""
    if t.dtype is _bf and t.shape == shape and t.is_cuda and t.is_contiguous():
        return t.data_ptr(), shape[1]
    _shape(name, t, shape)
    return _rows(t)


def _on(t, stream, *others):
    """The stream's handle; tensors of another device than the current one are refused."""
    at = torch.cuda.current_device()
    for t in (t, *others):
        if t is not None and t.get_device() != at:
            raise ValueError(f"tensors on device {t.get_device()}, the current one is {at}")
    return _s(stream)


def _need(nb):
    if nb == 0:
        raise MoeError(_lib.MOE_ERR_ARG, lib().moe_last_error().decode())
    return nb


# ------------------------------------------------------------------ norms
def norm_dims(T, H, eps=1e-6, dw_fp32=False) -> MoeNormDims:
    return MoeNormDims(T, H, MOE_F_DW_FP32 if dw_fp32 else 0, eps)


def moe_norm_fwd(d, x, residual, w, h=None, y=None, q=None, scale=None, stream=None):
    """h = x + residual (bf16; without a residual h is None), y and the int8 rows
    q, scale of its norm; x and residual [T, H] bf16 (rows may be strided)."""
    shape = (d.T, d.H)
    _shape("x", x, shape)
    _shape("w", w, shape[1:])
    for name, t in (("residual", residual), ("h", h), ("y", y), ("q", q)):
        if t is not None:
            _shape(name, t, shape)
    if scale is not None:
        _shape("scale", scale, shape[:1])
    pr, ldr = (None, 0) if residual is None else _rows(residual)
    check(lib().moe_norm_fwd(_ref(d), *_rows(x), pr, ldr, _p(w, _bf), _p(h, _bf), _p(y, _bf), _p(q, torch.int8),
                             _p(scale, _f32), _on(x, stream, residual, w, h, y, q, scale)))


def moe_norm_bwd_workspace_bytes(d: MoeNormDims) -> int:
    return lib().moe_norm_bwd_workspace_bytes(_ref(d))


def moe_norm_bwd(d, h, w, dy, dh, dx, dw, ws, stream=None):
    """dx (of x and the residual alike) and dw from the rows h that were normed;
    dh, or None, is the gradient that reaches h past the norm."""
    shape = (d.T, d.H)
    for name, t in (("h", h), ("dy", dy), ("dh", dh), ("dx", dx)):
        if t is not None:
            _shape(name, t, shape)
    _shape("w", w, shape[1:])
    _shape("dw", dw, shape[1:])
    pu, ldu = (None, 0) if dh is None else _rows(dh)
    check(lib().moe_norm_bwd(_ref(d), *_rows(h), _p(w, _bf), *_rows(dy), pu, ldu, _p(dx, _bf),
                             _p(dw, _f32 if d.flags & MOE_F_DW_FP32 else _bf), _p(ws), ws.numel() * ws.element_size(),
                             _on(h, stream, w, dy, dh, dx, dw, ws)))


class RMSNorm(_Held):
    """Root-mean-square norm with weight [H] of up to T rows: the caller-side
    outputs.  `out` says what the forward writes: "bf16" rows, "i8" rows, or
    "both"; `backward` makes the gradients' buffers too."""

    def __init__(self, T, weight, eps=1e-6, out="bf16", dw_fp32=False, backward=False):
        if out not in ("bf16", "i8", "both"):
            raise ValueError(f'out must be "bf16", "i8" or "both", not {out!r}')
        H, dev = weight.numel(), weight.device
        self.d = norm_dims(T, H, eps, dw_fp32)
        nb = _need(moe_norm_bwd_workspace_bytes(self.d))
        if out != "bf16" and H % 16:
            raise MoeError(_lib.MOE_ERR_SHAPE, f"H={H} must be a multiple of 16 for int8 rows")
        self.weight = weight

        def rows(dtype):
            return torch.empty((T, H), dtype=dtype, device=dev)

        self.h = rows(_bf)
        self.y = rows(_bf) if out != "i8" else None
        self.q = rows(torch.int8) if out != "bf16" else None
        self.scale = torch.empty(T, dtype=_f32, device=dev) if out != "bf16" else None
        self.dx = self.dw = self.ws = None
        if backward:
            self.dx = rows(_bf)
            self.dw = torch.empty(H, dtype=_f32 if dw_fp32 else _bf, device=dev)
            self.ws = _ws(nb, dev)
        self._nb = nb
        self._take()

    def _take(self):
        d = self.d
        _shape("weight", self.weight, (d.H,))
        for name in ("h", "y", "q", "dx"):
            if getattr(self, name) is not None:
                _shape(name, getattr(self, name), (d.T, d.H))
        if self.scale is not None:
            _shape("scale", self.scale, (d.T,))
        w = _p(self.weight, _bf)
        self._full = (torch.Size((d.T, d.H)), _ref(d))
        self._b = w, _p(self.h, _bf), _p(self.y, _bf), _p(self.q, torch.int8), _p(self.scale, _f32)
        if self.dx is not None:
            _shape("dw", self.dw, (d.H,))
            self._g = (_p(self.dx, _bf), _p(self.dw, _f32 if d.flags & MOE_F_DW_FP32 else _bf),
                       *_take_ws(self.ws, self._nb))

    def _dims(self, x):
        """The shape and dims of x's rows."""
        if x.shape == self._full[0]:
            return self._full
        d, t = self.d, x.shape[0]
        if not 1 <= t <= d.T:
            raise ValueError(f"{t} rows, made for 1 to {d.T}")
        return (t, d.H), _ref(MoeNormDims(t, d.H, d.flags, d.eps))

    def forward(self, x, residual=None, stream=None):
        """(h, y, q, scale) of x [t, H], t <= T (rows may be strided): the sum with
        the residual (None without one), its norm, and the norm's int8 rows;
        those that the norm was not made for are None."""
        shape, d = self._dims(x)
        w, h, y, q, scale = self._b
        if residual is None:
            check(lib().moe_norm_fwd(d, *_bf_rows("x", x, shape), None, 0, w, None, y, q, scale,
                                     _on(x, stream, self.weight)))
            outs = None, self.y, self.q, self.scale
        else:
            check(lib().moe_norm_fwd(d, *_bf_rows("x", x, shape), *_bf_rows("residual", residual, shape), w, h, y, q,
                                     scale, _on(x, stream, residual, self.weight)))
            outs = self.h, self.y, self.q, self.scale
        return outs if shape is self._full[0] else tuple(None if o is None else o[:shape[0]] for o in outs)

    def backward(self, h, dy, dh=None, stream=None):
        """(dx, dw): the gradients of x (and the residual) and of the weight, from
        the normed rows h, the gradient dy of the norm and, or None, the gradient
        dh that reaches h past it."""
        if self.dx is None:
            raise ValueError("made without backward=True")
        shape, d = self._dims(h)
        u = (None, 0) if dh is None else _bf_rows("dh", dh, shape)
        check(lib().moe_norm_bwd(d, *_bf_rows("h", h, shape), self._b[0], *_bf_rows("dy", dy, shape), *u, *self._g,
                                 _on(h, stream, dy, dh, self.weight)))
        return (self.dx if shape is self._full[0] else self.dx[:shape[0]]), self.dw


# ------------------------------------------------------------------ the expert layer for a few tokens
def moe_decode_workspace_bytes(d: MoeDims) -> int:
    return lib().moe_decode_workspace_bytes(_ref(d))


def moe_decode_i8_workspace_bytes(d: MoeDims) -> int:
    return lib().moe_decode_i8_workspace_bytes(_ref(d))


def _mask(token_mask, d):
    if token_mask is None:
        return None
    if not d.flags & MOE_F_MASK:
        raise ValueError("token_mask given, but the dims have no mask")
    if token_mask.dtype not in (torch.uint8, torch.bool):
        raise ValueError(f"token_mask must be uint8 or bool, not {token_mask.dtype}")
    _least(token_mask=(token_mask, d.T))
    return _p(token_mask)


def moe_decode(d, x, w_r, w_gate, w_up, w_down, token_mask, y, ws, stream=None):
    """moe_infer for at most MOE_DECODE_MAX_T tokens."""
    n = d.E * d.H * d.F
    _least(x=(x, d.T * d.H), w_r=(w_r, d.H * d.E), w_gate=(w_gate, n), w_up=(w_up, n), w_down=(w_down, n),
           y=(y, d.T * d.H))
    check(lib().moe_decode(_ref(d), *(_p(t, _bf) for t in (x, w_r, w_gate, w_up, w_down)), _mask(token_mask, d),
                           _p(y, _bf), _p(ws), ws.numel() * ws.element_size(),
                           _on(x, stream, w_r, w_gate, w_up, w_down, token_mask, y, ws)))


def moe_decode_i8(d, x, w_r, w: MoeI8Experts, token_mask, y, ws, stream=None):
    """moe_infer_i8 for at most MOE_DECODE_MAX_T tokens."""
    _check_weights(w, d.E, d.H, d.F)
    _least(x=(x, d.T * d.H), w_r=(w_r, d.H * d.E), y=(y, d.T * d.H))
    check(lib().moe_decode_i8(_ref(d), _p(x, _bf), _p(w_r, _bf), _ref(w), _mask(token_mask, d), _p(y, _bf), _p(ws),
                              ws.numel() * ws.element_size(),
                              _on(x, stream, w_r, token_mask, y, ws, *_tensors(w))))


def _tensors(w):
    """Those of an int8 experts' descriptor; one made by hand holds pointers alone."""
    return getattr(w, "tensors", ())


class MoEDecode(_Held):
    """Caller-side buffers of the expert layer for up to T <= MOE_DECODE_MAX_T tokens."""

    _bytes = staticmethod(moe_decode_workspace_bytes)

    def __init__(self, T, H, E, F, top_k, mask=False, device="cuda"):
        self.d = MoeDims(T, H, E, F, top_k, MOE_F_MASK if mask else 0, 0.0, 0.0)
        self._nb = _need(self._bytes(self.d))
        self.ws = _ws(self._nb, device)
        self.y = torch.empty((T, H), dtype=_bf, device=device)
        self._take()

    def _take(self):
        _shape("y", self.y, (self.d.T, self.d.H))
        self._b = _p(self.y, _bf), *_take_ws(self.ws, self._nb)

    def _args(self, x, w_r):
        """Dims of x's tokens and the leading pointers."""
        d, t = self.d, x.shape[0]
        if t != d.T:
            if not 1 <= t <= d.T:
                raise ValueError(f"{t} tokens, made for 1 to {d.T}")
            d = MoeDims(t, d.H, d.E, d.F, d.top_k, d.flags, 0.0, 0.0)
        _shape("x", x, (t, d.H))
        _shape("w_r", w_r, (d.H, d.E))
        return d, (_p(x, _bf), _p(w_r, _bf))

    def _out(self, t):
        return self.y if t == self.d.T else self.y[:t]

    def forward(self, x, w_r, w_gate, w_up, w_down, token_mask=None, stream=None):
        """The layer's output for x [t, H], t <= T."""
        d, p = self._args(x, w_r)
        _shape("w_gate", w_gate, (d.E, d.H, d.F))
        _shape("w_up", w_up, (d.E, d.H, d.F))
        _shape("w_down", w_down, (d.E, d.F, d.H))
        check(lib().moe_decode(_ref(d), *p, _p(w_gate, _bf), _p(w_up, _bf), _p(w_down, _bf), _mask(token_mask, d),
                               *self._b, _on(x, stream, w_r, w_gate, w_up, w_down, token_mask, self.y)))
        return self._out(d.T)


class MoEDecodeI8(MoEDecode):
    """The same with the experts in 8 bits."""

    _bytes = staticmethod(moe_decode_i8_workspace_bytes)

    def forward(self, x, w_r, w: MoeI8Experts, token_mask=None, stream=None):
        """The layer's output for x [t, H], t <= T."""
        d, p = self._args(x, w_r)
        _check_weights(w, d.E, d.H, d.F)
        check(lib().moe_decode_i8(_ref(d), *p, _ref(w), _mask(token_mask, d), *self._b,
                                  _on(x, stream, w_r, token_mask, self.y, *_tensors(w))))
        return self._out(d.T)


# ------------------------------------------------------------------ sampling
def sample_dims(B, V, fp32=True) -> MoeSampleDims:
    return MoeSampleDims(B, V, MOE_F_LOGITS_FP32 if fp32 else 0)


def moe_sample_workspace_bytes(d: MoeSampleDims) -> int:
    return lib().moe_sample_workspace_bytes(_ref(d))


def _settings(B, temperature, top_k, top_p, min_p, u):
    held = []
    for name, t, dtype in (("temperature", temperature, _f32), ("top_k", top_k, _i32), ("top_p", top_p, _f32),
                           ("min_p", min_p, _f32), ("u", u, _f32)):
        if t is not None:
            _shape(name, t, (B,))
        held.append(_p(t, dtype))
    return held


def moe_sample(d, logits, temperature, top_k, top_p, min_p, u, token, logprob, ws, stream=None):
    """token [B] int32 and, or None, logprob [B] of logits [B, V] (fp32 or bf16 as
    the dims say, rows may be strided); the settings are [B] tensors or None."""
    _shape("logits", logits, (d.B, d.V))
    _shape("token", token, (d.B,))
    if logprob is not None:
        _shape("logprob", logprob, (d.B,))
    check(lib().moe_sample(_ref(d), *_rows(logits, _f32 if d.flags & MOE_F_LOGITS_FP32 else _bf),
                           *_settings(d.B, temperature, top_k, top_p, min_p, u), _p(token, _i32), _p(logprob, _f32),
                           _p(ws), ws.numel() * ws.element_size(),
                           _on(logits, stream, temperature, top_k, top_p, min_p, u, token, logprob, ws)))


class Sampler(_Held):
    """Caller-side buffers of the choice of the next token for up to B rows of V logits."""

    def __init__(self, B, V, device="cuda"):
        self.d = sample_dims(B, V)
        self._nb = _need(moe_sample_workspace_bytes(self.d))
        self.ws = _ws(self._nb, device)
        self.token = torch.empty(B, dtype=_i32, device=device)
        self.logprob = torch.empty(B, dtype=_f32, device=device)
        self._take()

    def _take(self):
        _shape("token", self.token, (self.d.B,))
        _shape("logprob", self.logprob, (self.d.B,))
        self._b = _p(self.token, _i32), _p(self.logprob, _f32), *_take_ws(self.ws, self._nb)

    def forward(self, logits, u, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
        """(token, logprob) of logits [b, V] (fp32 or bf16, rows may be strided), b <= B,
        from uniform numbers u [b] in [0, 1); the settings are [b] tensors or None (off)."""
        b = logits.shape[0]
        if not 1 <= b <= self.d.B:
            raise ValueError(f"{b} rows, made for 1 to {self.d.B}")
        _shape("logits", logits, (b, self.d.V))
        d = sample_dims(b, self.d.V, logits.dtype == _f32)
        check(lib().moe_sample(_ref(d), *_rows(logits, _f32 if logits.dtype == _f32 else _bf),
                               *_settings(b, temperature, top_k, top_p, min_p, u), *self._b,
                               _on(logits, stream, temperature, top_k, top_p, min_p, u, self.token)))
        return (self.token, self.logprob) if b == self.d.B else (self.token[:b], self.logprob[:b])
