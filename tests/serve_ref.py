"""Plain 64-bit forms of the 8-bit serving operators, one request, expert or
block at a time, on the CPU.  Where an operator is defined in fp32 steps (the
rounding of cached tokens) the same fp32 steps are taken here."""
import numpy as np


def quant_rows(x):
    """x [rows, K] (fp64) -> (q, scale)."""
    top = np.abs(x).max(axis=-1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        q = np.where(top > 0, np.rint(127.0 * x / top), 0.0)
    return q, top / 127.0


def dequant(x):
    q, s = quant_rows(x)
    return q * s


def expert(x, wg, wu, wd):
    """One expert on rows x; wg, wu [F, H], wd [H, F] as the values they stand for."""
    x = dequant(x)
    g, u = x @ wg.T, x @ wu.T
    return dequant(g / (1.0 + np.exp(-g)) * u) @ wd.T


def append_block(q, s, x, off):
    """New tokens x [n, D] (fp32) at `off` of a block q [bt, D] with scale s, in
    the cache's own fp32 steps; returns the block's (q, scale)."""
    f = np.float32
    s0 = f(s) if off else f(0)
    s1 = max(s0, f(np.abs(x).max()) / f(127))
    q = q.copy()
    if s1 == 0:
        q[off:off + len(x)] = 0
        return q, s1
    if off:
        q[:off] = np.rint(q[:off].astype(f) * (s0 / s1))
    q[off:off + len(x)] = np.clip(np.rint(x.astype(f) / s1), -127, 127)
    return q, s1


def attention(q, k, v, pos0, kv, causal, scale):
    """q [n, heads, D], k, v [L, kv_heads, D] with NaN rows where a token has no
    place; token i is at pos0 + i and sees keys [0, kv) (causal: up to itself).
    Returns (out, the same sum over |v|)."""
    n, heads, D = q.shape
    group = heads // k.shape[1]
    out, mag = np.zeros_like(q), np.zeros_like(q)
    for i in range(n):
        lim = min(kv, pos0 + i + 1) if causal else kv
        for h in range(heads):
            kk, vv = k[:max(lim, 0), h // group], v[:max(lim, 0), h // group]
            at = ~np.isnan(kk[:, 0])
            if not at.any():
                continue
            s = kk[at] @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h] = p @ vv[at]
            mag[i, h] = p @ np.abs(vv[at])
    return out, mag


def plan(old, new, table, free, n_free, T, n_blocks, bt):
    """The tables of one step; `table` is a list of lists and is changed."""
    W = len(table[0])
    left, missing = n_free, 0
    row_start, kv_len, pos, slots, seq = [0], [], [], [], []
    for b, (o, n) in enumerate(zip(old, new)):
        o, n = max(o, 0), max(n, 0)
        have, want = -(-o // bt), -(-(o + n) // bt)
        for i in range(have, want):
            if i >= W:
                missing += 1
                continue
            if left > 0:
                left -= 1
                table[b][i] = free[left] if 0 <= free[left] < n_blocks else -1
            else:
                missing += 1
                table[b][i] = -1
        for p in range(o, o + n):
            i = p // bt
            blk = table[b][i] if i < W else -1
            pos.append(p)
            slots.append(blk * bt + p % bt if 0 <= blk < n_blocks else -1)
            seq.append(b)
        row_start.append(row_start[-1] + n)
        kv_len.append(o + n)
    cut = [a[:T] + [-1] * max(0, T - len(a)) for a in (pos, slots, seq)]
    return row_start, kv_len, *cut, [left, missing]
