"""Plain 64-bit forms of a decoding step's operators on the CPU (numpy)."""
import numpy as np

from tests import serve_ref


def norm(h, w, eps):
    """h [T, H] (the stored sum) -> (v, s)."""
    s = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return h * s * w, s


def norm_bwd(h, w, dy, dh, eps):
    """(dx, dw, size of dx's terms, size of dw's terms)."""
    _, s = norm(h, w, eps)
    n, g = h * s, dy * w
    dx = s * (g - n * (g * n).mean(-1, keepdims=True)) + dh
    mag = s * (np.abs(g) + np.abs(n) * np.abs(g * n).mean(-1, keepdims=True)) + np.abs(dh)
    return dx, (dy * n).sum(0), mag, np.abs(dy * n).sum(0)


def route(x, w_r, k):
    """The k largest logits per token, ties to the lower expert; (experts, gates, gap to the next logit)."""
    z = x @ w_r
    idx = np.argsort(-z, axis=-1, kind="stable")
    top = np.take_along_axis(z, idx, -1)
    gap = top[:, k - 1] - top[:, k] if k < z.shape[1] else np.full(len(z), np.inf)
    g = np.exp(top[:, :k] - top[:, :1])
    return idx[:, :k], g / g.sum(-1, keepdims=True), gap


def experts(x, idx, gates, get, i8=False):
    """y and the size of its terms; get(e) -> (w_gate [H, F], w_up [H, F], w_down [F, H])."""
    y, mag = np.zeros_like(x), np.zeros_like(x)
    for e in np.unique(idx):
        wg, wu, wd = get(e)
        for t, j in zip(*np.nonzero(idx == e)):
            row = serve_ref.dequant(x[t:t + 1]) if i8 else x[t:t + 1]
            g = row @ wg
            a = g / (1.0 + np.exp(-g)) * (row @ wu)
            if i8:
                a = serve_ref.dequant(a)
            y[t] += gates[t, j] * (a @ wd)[0]
            mag[t] += gates[t, j] * (np.abs(a) @ np.abs(wd))[0]
    return y, mag


def sample(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob) of one row of logits (fp64)."""
    row = np.where(np.isnan(row), -np.inf, row)
    if row.max() == -np.inf:
        return -1, -np.inf
    if not temperature > 0:
        return int(np.argmax(row)), 0.0
    order = np.argsort(-row, kind="stable")
    most = row[order[0]]
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        d = np.where(row == most, 0.0, (row - most) / np.float64(temperature))
    w = np.exp(d)[order]
    if 0 < top_k < len(w):
        w[top_k:] = 0
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        w[1:] = np.where(before[1:] < top_p * w.sum(), w[1:], 0)
    if min_p > 0:
        w[w < min(min_p, 1.0)] = 0
    kept = np.zeros(len(w))
    kept[order] = w
    c = np.cumsum(kept)
    u = 0.0 if not u > 0 else float(u)
    i = int(np.searchsorted(c, u * c[-1], side="right"))
    if i >= len(c) or u >= 1:
        i = int(np.nonzero(kept)[0][-1])
    return i, float(d[i] - np.log(kept.sum()))
