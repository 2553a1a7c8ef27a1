"""8-bit serving: the int8 products, dense and over the experts, and attention
over a paged int8 cache (the 8-bit part of the C ABI in include/moe.h).

As in the rest of the package the functions turn tensors into pointers and the
classes own the caller-side buffers; the work runs in the library's kernels.
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib
from ._lib import (MOE_F_CAUSAL, MOE_F_OUT_FP32, MoeDims, MoeError, MoeExpertsDims, MoeI8Dims, MoeI8Experts,
                   MoeKvAttn, MoeKvBatch, MoeKvCache, MoeKvPlanDims, check, lib)

__all__ = [
    "i8_dims", "moe_i8_quant_rows", "moe_i8_quant_weight", "moe_i8_matmul", "moe_i8_linear_workspace_bytes",
    "moe_i8_linear", "i8_weights", "moe_experts_i8_workspace_bytes", "moe_experts_i8", "moe_infer_i8_workspace_bytes",
    "moe_infer_i8", "moe_kv_plan", "moe_kv_append", "moe_kv_read", "moe_kv_attention_workspace_bytes",
    "moe_kv_attention", "kv_batch", "I8Linear", "MoEExpertsI8", "MoEInferI8", "KVPlan", "KVCache", "KVAttention",
    "MOE_F_OUT_FP32", "MOE_F_CAUSAL",
]

_ref = ctypes.byref


def _p(t, dtype=None):
    if t is None:
        return t
    if not t.is_cuda:
        raise ValueError("tensor must be on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"tensor must be {dtype}, not {t.dtype}")
    return t.data_ptr()


def _rows(t, dtype=torch.bfloat16):
    """Pointer and row pitch of packed rows: contiguous but for the first dimension."""
    if not t.is_cuda:
        raise ValueError("tensor must be on the GPU")
    if t.dtype != dtype:
        raise ValueError(f"tensor must be {dtype}, not {t.dtype}")
    if t.is_contiguous() and t.shape[0]:
        return t.data_ptr(), t.numel() // t.shape[0]
    n = 1
    for size, stride in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != n:
            raise ValueError("rows must be contiguous")
        n *= size
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else n


def _shape(name, t, shape):
    if t.shape != shape:  # torch.Size compares as the tuple that it is
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")


def _least(**sizes):
    """Refuses tensors of fewer elements than the call will read or write: name=(tensor, elements)."""
    for name, (t, n) in sizes.items():
        if t.numel() < n:
            raise ValueError(f"{name} has {t.numel()} elements of {n}")


def _s(stream):
    if stream is None:
        # the handle alone: a Stream object costs as much as the launch (3 us)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _ws(n, device):
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device)


class _Held:
    """Buffers whose pointers are taken and checked once, by _take, and not at
    every call; replacing one takes them again (or, refused, leaves it)."""

    def __setattr__(self, name, value):
        d = self.__dict__
        old = d.get(name)
        d[name] = value
        if isinstance(old, torch.Tensor) and "_b" in d:
            try:
                self._take()
            except (ValueError, AttributeError):
                d[name] = old
                raise


def _take_ws(ws, nb):
    if ws.numel() * ws.element_size() < nb:
        raise ValueError(f"ws has less than {nb} bytes")
    return _p(ws), nb


# ------------------------------------------------------------------ int8 products
def i8_dims(M, N, K, out_fp32=False) -> MoeI8Dims:
    return MoeI8Dims(M, N, K, MOE_F_OUT_FP32 if out_fp32 else 0)


def moe_i8_quant_rows(x, q, scale, stream=None):
    """Rows of x [rows, K] bf16 (rows may be strided) as int8 rows q and their scales."""
    px, ldx = _rows(x)
    _shape("q", q, x.shape)
    _shape("scale", scale, x.shape[:1])
    check(lib().moe_i8_quant_rows(x.shape[0], x.shape[1], px, ldx, _p(q, torch.int8), _p(scale, torch.float32),
                                  _s(stream)))


def moe_i8_quant_weight(w, q=None, scale=None, stream=None):
    """w [..., K, N] bf16 -> (q [..., N, K] int8, scale [..., N]), one scale per output channel."""
    *lead, K, N = w.shape
    E = 1
    for n in lead:
        E *= n
    q = torch.empty((*lead, N, K), dtype=torch.int8, device=w.device) if q is None else q
    scale = torch.empty((*lead, N), dtype=torch.float32, device=w.device) if scale is None else scale
    _shape("q", q, (*lead, N, K))
    _shape("scale", scale, (*lead, N))
    check(lib().moe_i8_quant_weight(E, K, N, _p(w, torch.bfloat16), _p(q, torch.int8), _p(scale, torch.float32),
                                    _s(stream)))
    return q, scale


def _out_rows(out, M, N):
    if out.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"out must be bf16 or fp32, not {out.dtype}")
    _shape("out", out, (M, N))
    return _rows(out, out.dtype)


def moe_i8_matmul(a, a_scale, b, b_scale, out, stream=None):
    """out [M, N] (bf16 or fp32) = a_scale[m] b_scale[n] <a[m], b[n]> of int8 rows a [M, K] and b [N, K]."""
    (M, K), N = a.shape, b.shape[0]
    _shape("b", b, (N, K))
    _shape("a_scale", a_scale, (M,))
    _shape("b_scale", b_scale, (N,))
    po, ldo = _out_rows(out, M, N)
    check(lib().moe_i8_matmul(_ref(i8_dims(M, N, K, out.dtype == torch.float32)), _p(a, torch.int8),
                              _p(a_scale, torch.float32), _p(b, torch.int8), _p(b_scale, torch.float32), po, ldo,
                              _s(stream)))


def moe_i8_linear_workspace_bytes(d: MoeI8Dims) -> int:
    return lib().moe_i8_linear_workspace_bytes(_ref(d))


def moe_i8_linear(d, x, b, b_scale, out, ws, stream=None):
    _shape("x", x, (d.M, d.K))
    _least(b=(b, d.N * d.K), b_scale=(b_scale, d.N))
    px, ldx = _rows(x)
    if (out.dtype == torch.float32) != bool(d.flags & MOE_F_OUT_FP32):
        raise ValueError(f"out is {out.dtype}, which the dims do not say")
    po, ldo = _out_rows(out, d.M, d.N)
    check(lib().moe_i8_linear(_ref(d), px, ldx, _p(b, torch.int8), _p(b_scale, torch.float32), po, ldo, _p(ws),
                              ws.numel(), _s(stream)))


class I8Linear(_Held):
    """A projection with int8 weights [N, K] (moe_i8_quant_weight) for up to M
    rows: the caller-side workspace and output."""

    def __init__(self, M, weight, scale, out_fp32=False):
        N, K = weight.shape
        self.weight, self.scale = weight, scale
        self.d = i8_dims(M, N, K, out_fp32)
        nb = moe_i8_linear_workspace_bytes(self.d)
        if nb == 0:
            raise MoeError(_lib.MOE_ERR_ARG, lib().moe_last_error().decode())
        self.ws = _ws(nb, weight.device)
        self.out = torch.empty((M, N), dtype=torch.float32 if out_fp32 else torch.bfloat16, device=weight.device)
        self._nb = nb
        self._take()

    def _take(self):
        d = self.d
        _shape("weight", self.weight, (d.N, d.K))
        _shape("scale", self.scale, (d.N,))
        _shape("out", self.out, (d.M, d.N))
        self._b = (_p(self.weight, torch.int8), _p(self.scale, torch.float32),
                   _p(self.out, torch.float32 if d.flags & MOE_F_OUT_FP32 else torch.bfloat16), d.N,
                   *_take_ws(self.ws, self._nb))

    def forward(self, x, stream=None):
        """The product of x [m, K], m <= M (rows may be strided); a view of the output's first m rows."""
        d, m = self.d, x.shape[0]
        if m != d.M:
            if not 1 <= m <= d.M:
                raise ValueError(f"{m} rows, made for 1 to {d.M}")
            d = MoeI8Dims(m, d.N, d.K, d.flags)
        _shape("x", x, (m, d.K))
        check(lib().moe_i8_linear(_ref(d), *_rows(x), *self._b, _s(stream)))
        return self.out if m == self.d.M else self.out[:m]


# ------------------------------------------------------------------ experts in 8 bits
def i8_weights(w_gate, s_gate, w_up, s_up, w_down, s_down) -> MoeI8Experts:
    """The expert weights' descriptor (device tensors stay owned by the caller):
    int8 w_gate, w_up [E, F, H], w_down [E, H, F] and their channel scales."""
    E, F, H = w_gate.shape
    _shape("w_up", w_up, (E, F, H))
    _shape("w_down", w_down, (E, H, F))
    for n, t, c in (("s_gate", s_gate, F), ("s_up", s_up, F), ("s_down", s_down, H)):
        _shape(n, t, (E, c))
    w = MoeI8Experts(*(_p(t, torch.int8) for t in (w_gate, w_up, w_down)),
                     *(_p(t, torch.float32) for t in (s_gate, s_up, s_down)))
    w.shape = (E, H, F)
    w.tensors = (w_gate, w_up, w_down, s_gate, s_up, s_down)  # as long as the descriptor
    return w


def _check_weights(w, E, H, F):
    if getattr(w, "shape", (E, H, F)) != (E, H, F):  # a descriptor made by hand has none
        raise ValueError(f"weights of E, H, F = {w.shape}, not {(E, H, F)}")


def moe_experts_i8_workspace_bytes(d: MoeExpertsDims) -> int:
    return lib().moe_experts_i8_workspace_bytes(_ref(d))


def moe_experts_i8(d, xp, counts, w: MoeI8Experts, o, ws, stream=None):
    _check_weights(w, d.E, d.H, d.F)
    _least(xp=(xp, d.rows * d.H), counts=(counts, d.E), o=(o, d.rows * d.H))
    check(lib().moe_experts_i8(_ref(d), _p(xp, torch.bfloat16), _p(counts, torch.int32), _ref(w),
                               _p(o, torch.bfloat16), _p(ws), ws.numel(), _s(stream)))


def moe_infer_i8_workspace_bytes(d: MoeDims) -> int:
    return lib().moe_infer_i8_workspace_bytes(_ref(d))


def moe_infer_i8(d, x, w_r, w: MoeI8Experts, token_mask, y, ws, stream=None):
    _check_weights(w, d.E, d.H, d.F)
    _least(x=(x, d.T * d.H), w_r=(w_r, d.H * d.E), y=(y, d.T * d.H))
    if token_mask is not None:
        _least(token_mask=(token_mask, d.T))
    check(lib().moe_infer_i8(_ref(d), _p(x, torch.bfloat16), _p(w_r, torch.bfloat16), _ref(w), _p(token_mask),
                             _p(y, torch.bfloat16), _p(ws), ws.numel(), _s(stream)))


class MoEExpertsI8(_Held):
    """Caller-side buffers of one rank's local experts in 8 bits, forward only."""

    def __init__(self, rows, H, E, F, device="cuda"):
        self.d = MoeExpertsDims(rows, H, E, F, 0)
        nb = moe_experts_i8_workspace_bytes(self.d)
        if nb == 0:
            raise MoeError(_lib.MOE_ERR_ARG, lib().moe_last_error().decode())
        self.ws = _ws(nb, device)
        self.o = torch.empty((rows, H), dtype=torch.bfloat16, device=device)
        self._nb = nb
        self._take()

    def _take(self):
        _shape("o", self.o, (self.d.rows, self.d.H))
        self._b = _p(self.o, torch.bfloat16), *_take_ws(self.ws, self._nb)

    def forward(self, xp, counts, w: MoeI8Experts, stream=None):
        d = self.d
        _check_weights(w, d.E, d.H, d.F)
        _shape("xp", xp, (d.rows, d.H))
        _shape("counts", counts, (d.E,))
        check(lib().moe_experts_i8(_ref(d), _p(xp, torch.bfloat16), _p(counts, torch.int32), _ref(w), *self._b,
                                   _s(stream)))
        return self.o


class MoEInferI8:
    """Caller-side buffers of the block's forward-only pass with the experts in 8 bits."""

    def __init__(self, T, H, E, F, top_k, mask=False, device="cuda"):
        self.d = MoeDims(T, H, E, F, top_k, _lib.MOE_F_MASK if mask else 0, 0.0, 0.0)
        nb = moe_infer_i8_workspace_bytes(self.d)
        if nb == 0:
            raise MoeError(_lib.MOE_ERR_ARG, lib().moe_last_error().decode())
        self.ws = _ws(nb, device)
        self.y = torch.empty((T, H), dtype=torch.bfloat16, device=device)

    def forward(self, x, w_r, w: MoeI8Experts, token_mask=None, stream=None):
        d = self.d
        _shape("x", x, (d.T, d.H))
        _shape("w_r", w_r, (d.H, d.E))
        moe_infer_i8(d, x, w_r, w, token_mask, self.y, self.ws, stream)
        return self.y


# ------------------------------------------------------------------ the paged cache
def moe_kv_plan(d, old_len, new_len, block_table, free_ids, n_free, row_start, kv_len, positions, slots, seq, state,
                stream=None):
    _least(old_len=(old_len, d.B), new_len=(new_len, d.B), block_table=(block_table, d.B * d.W),
           free_ids=(free_ids, d.free_cap), n_free=(n_free, 1), row_start=(row_start, d.B + 1), kv_len=(kv_len, d.B),
           positions=(positions, d.T), slots=(slots, d.T), seq=(seq, d.T), state=(state, 2))
    i32 = torch.int32
    _plan(d, old_len, new_len, block_table, free_ids, n_free,
          [_p(t, i32) for t in (row_start, kv_len, positions, slots, seq, state)], stream)


def _plan(d, old_len, new_len, block_table, free_ids, n_free, written, stream):
    """The call, on pointers of what it writes but for the table."""
    i32 = torch.int32
    check(lib().moe_kv_plan(_ref(d), _p(old_len, i32), _p(new_len, i32), _p(block_table, i32), _p(free_ids, i32),
                            _p(n_free, i32), *written, _s(stream)))


def kv_batch(T, row_start, kv_len, block_table) -> MoeKvBatch:
    B, W = block_table.shape
    _shape("row_start", row_start, (B + 1,))
    _shape("kv_len", kv_len, (B,))
    i32 = torch.int32
    return MoeKvBatch(B, T, W, _p(row_start, i32), _p(kv_len, i32), _p(block_table, i32))


def moe_kv_append(cache: MoeKvCache, batch: MoeKvBatch, k, v, stream=None):
    (pk, ldk), (pv, ldv) = _rows(k), _rows(v)
    _shape("k", k, (batch.T, cache.kv_heads, cache.head_dim))
    _shape("v", v, k.shape)
    if ldk != ldv:
        raise ValueError(f"k and v have row pitches {ldk} and {ldv}")
    check(lib().moe_kv_append(_ref(cache), _ref(batch), pk, pv, ldk, _s(stream)))


def moe_kv_read(cache: MoeKvCache, block_table, kv_start, k_out, v_out, stream=None):
    B, W = block_table.shape
    _shape("kv_start", kv_start, (B + 1,))
    _shape("k_out", k_out, (k_out.shape[0], cache.kv_heads, cache.head_dim))
    _shape("v_out", v_out, k_out.shape)
    i32, bf = torch.int32, torch.bfloat16
    check(lib().moe_kv_read(_ref(cache), B, W, _p(block_table, i32), _p(kv_start, i32), k_out.shape[0], _p(k_out, bf),
                            _p(v_out, bf), _s(stream)))


def moe_kv_attention_workspace_bytes(cache: MoeKvCache, batch: MoeKvBatch, a: MoeKvAttn) -> int:
    return lib().moe_kv_attention_workspace_bytes(_ref(cache), _ref(batch), _ref(a))


def moe_kv_attention(cache: MoeKvCache, batch: MoeKvBatch, a: MoeKvAttn, q, out, ws, stream=None):
    (pq, ldq), (po, ldo) = _rows(q), _rows(out)
    _shape("q", q, (batch.T, a.heads, cache.head_dim))
    _shape("out", out, q.shape)
    check(lib().moe_kv_attention(_ref(cache), _ref(batch), _ref(a), pq, ldq, po, ldo, _p(ws), ws.numel(), _s(stream)))


class KVPlan(_Held):
    """Buffers of one step's tables for B requests of up to W blocks, up to T packed new tokens."""

    def __init__(self, B, T, W, n_blocks, block_tokens, device="cuda"):
        self.d = MoeKvPlanDims(B, T, W, n_blocks, block_tokens, 0)

        def ints(n):
            return torch.empty(n, dtype=torch.int32, device=device)

        self.row_start, self.kv_len, self.state = ints(B + 1), ints(B), ints(2)
        self.positions, self.slots, self.seq = ints(T), ints(T), ints(T)
        self._take()

    def _take(self):
        d, held = self.d, []
        for name, n in (("row_start", d.B + 1), ("kv_len", d.B), ("positions", d.T), ("slots", d.T), ("seq", d.T),
                        ("state", 2)):
            t = getattr(self, name)
            _shape(name, t, (n,))
            held.append(_p(t, torch.int32))
        self._b = held

    def build(self, old_len, new_len, block_table, free_ids, n_free, stream=None):
        """Tables of this step; takes the blocks that the requests lack into block_table.
        The last step's kv_len and state[:1] may be passed as old_len and n_free."""
        d = self.d
        _shape("old_len", old_len, (d.B,))
        _shape("new_len", new_len, (d.B,))
        _shape("block_table", block_table, (d.B, d.W))
        _shape("n_free", n_free, (1,))
        d.free_cap = free_ids.numel()
        _plan(d, old_len, new_len, block_table, free_ids, n_free, self._b, stream)


class KVCache(_Held):
    """A paged cache of keys and values in 8 bits with a scale for each block and head."""

    def __init__(self, n_blocks, block_tokens, kv_heads, head_dim, device="cuda"):
        self._own(torch.zeros((n_blocks, kv_heads, block_tokens, head_dim), dtype=torch.int8, device=device),
                  torch.zeros((n_blocks, kv_heads, head_dim, block_tokens), dtype=torch.int8, device=device),
                  torch.zeros((n_blocks, kv_heads), dtype=torch.float32, device=device),
                  torch.zeros((n_blocks, kv_heads), dtype=torch.float32, device=device))

    @classmethod
    def of(cls, k, v, k_scale, v_scale):
        """A cache over existing tensors."""
        c = cls.__new__(cls)
        c._own(k, v, k_scale, v_scale)
        return c

    def _own(self, k, v, k_scale, v_scale):
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        n, heads, bt, D = k.shape
        self.d = MoeKvCache(n, bt, heads, D, None, None, None, None)
        self._take()

    def _take(self):
        d = self.d
        n, heads, bt, D = d.n_blocks, d.kv_heads, d.block_tokens, d.head_dim
        _shape("k", self.k, (n, heads, bt, D))
        _shape("v", self.v, (n, heads, D, bt))
        _shape("k_scale", self.k_scale, (n, heads))
        _shape("v_scale", self.v_scale, (n, heads))
        self._b = (_p(self.k, torch.int8), _p(self.v, torch.int8), _p(self.k_scale, torch.float32),
                   _p(self.v_scale, torch.float32))
        d.k, d.v, d.k_scale, d.v_scale = self._b

    def append(self, k, v, row_start, kv_len, block_table, stream=None):
        """Write the packed new keys and values ([T, kv_heads, head_dim], rows may be strided)."""
        moe_kv_append(self.d, kv_batch(k.shape[0], row_start, kv_len, block_table), k, v, stream)

    def read(self, block_table, kv_start, k_out, v_out, stream=None):
        """Read the requests' first tokens back as packed bf16 rows."""
        moe_kv_read(self.d, block_table, kv_start, k_out, v_out, stream)
        return k_out, v_out


class KVAttention(_Held):
    """Caller-side buffers of the attention of up to T packed new tokens (at most
    max_q of one request) of B requests over a cache of up to max_kv tokens each."""

    def __init__(self, cache, T, heads, B, max_q, max_kv, causal=True, scale=None, device="cuda"):
        cache = getattr(cache, "d", cache)
        D, bt = cache.head_dim, cache.block_tokens
        self.a = MoeKvAttn(heads, max_q, max_kv, D ** -0.5 if scale is None else scale, MOE_F_CAUSAL if causal else 0)
        self.T, self.B, self.D = T, B, D
        nb = moe_kv_attention_workspace_bytes(cache, MoeKvBatch(B, T, -(-max_kv // bt), None, None, None), self.a)
        if nb == 0:
            raise MoeError(_lib.MOE_ERR_ARG, lib().moe_last_error().decode())
        self.ws = _ws(nb, device)
        self.out = torch.empty((T, heads, D), dtype=torch.bfloat16, device=device)
        self._nb = nb
        self._take()

    def _take(self):
        _shape("out", self.out, (self.T, self.a.heads, self.D))
        self._b = _p(self.out, torch.bfloat16), self.a.heads * self.D, *_take_ws(self.ws, self._nb)

    def forward(self, q, cache: KVCache, block_table, row_start, kv_len, stream=None):
        """Attention of the packed queries q [t, heads, head_dim], t <= T (rows may be strided)."""
        t = q.shape[0]
        if t > self.T or block_table.shape[0] != self.B:
            raise ValueError(f"{t} tokens of {block_table.shape[0]} requests, made for {self.T} of {self.B}")
        if cache.d.head_dim != self.D:
            raise ValueError(f"cache has head_dim {cache.d.head_dim}, made for {self.D}")
        _shape("q", q, (t, self.a.heads, self.D))
        check(lib().moe_kv_attention(_ref(cache.d), _ref(kv_batch(t, row_start, kv_len, block_table)), _ref(self.a),
                                     *_rows(q), *self._b, _s(stream)))
        return self.out if t == self.T else self.out[:t]
