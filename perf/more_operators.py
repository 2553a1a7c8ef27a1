"""Performance cases of a decoding step around the expert layer: the sum with
the residual and its root-mean-square norm (forward in bf16 and in int8 rows,
and backward), the whole expert layer for a few tokens (bf16 and int8 weights),
and the choice of the next token from the logits.

`own` chooses between the plain form (elementary torch operations in fp32, in
fp64 where a choice hangs on a sum) and the package's entry points.  A case is
a dict of plain values: `kind` names the operator, the rest are sizes and
options.  Inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

_EXPERT = dict(E=128, H=2048, F=768, k=8)  # the expert layer of a 30B-A3B model
_EPS = 1e-6


def listed():
    return [
        # The norm before the expert layer for one new token: latency.
        dict(name="norm_1", kind="norm", T=1, H=2048, residual=True, out="bf16"),
        # The same for two query groups of 8 passages x 512 tokens.
        dict(name="norm_8192", kind="norm", T=8192, H=2048, residual=True, out="bf16"),
        # A ragged batch of prompts, normed for an int8 projection.
        dict(name="norm_i8_3001", kind="norm", T=3001, H=5120, residual=True, out="i8"),
        # The gradient of a short passage's norm, without a residual path.
        dict(name="norm_bwd_300", kind="norm_bwd", T=300, H=640, dh=False, fp32=False),
        # The gradient of two query groups, the residual's gradient added.
        dict(name="norm_bwd_8192", kind="norm_bwd", T=8192, H=2048, dh=True, fp32=True),
        # Expert layer of one running request, then of sixteen.
        dict(name="decode_1", kind="decode", T=1, i8=False, mask=False, **_EXPERT),
        dict(name="decode_16", kind="decode", T=16, i8=False, mask=False, **_EXPERT),
        # The same in 8 bits: one request, and a batch of 64 slots of which some are idle.
        dict(name="decode_i8_1", kind="decode", T=1, i8=True, mask=False, **_EXPERT),
        dict(name="decode_i8_64", kind="decode", T=64, i8=True, mask=True, **_EXPERT),
        # Next token of one request: the usual top-k and top-p.
        dict(name="sample_1", kind="sample", B=1, V=131072, fp32=True, mode="top_k_p"),
        # Next tokens of 64 requests with settings of their own.
        dict(name="sample_64", kind="sample", B=64, V=131072, fp32=True, mode="mixed"),
        # A large batch over a vocabulary of odd size, bf16 logits, top-p alone.
        dict(name="sample_256", kind="sample", B=256, V=50001, fp32=False, mode="top_p"),
    ]


def draw(rng):
    """One more case: any operator over the listed cases' ranges, no costlier
    than that operator's largest of them."""
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["norm", "norm_bwd", "decode", "decode", "sample", "sample"])
        if kind in ("norm", "norm_bwd"):
            T, H = logint(1, 16384), 16 * logint(8, 1024)
            if T * H > 8192 * 2048:
                continue
            if kind == "norm":
                return dict(kind=kind, T=T, H=H, residual=rng.random() < 0.7, out=rng.choice(["bf16", "i8", "both"]))
            return dict(kind=kind, T=T, H=H, dh=rng.random() < 0.7, fp32=rng.random() < 0.5)
        if kind == "decode":
            c = dict(kind=kind, T=logint(1, 64), i8=rng.random() < 0.5, mask=rng.random() < 0.3, E=8 * logint(1, 32),
                     H=128 * logint(1, 32), F=128 * logint(1, 12), k=rng.choice([1, 2, 4, 6, 8]))
            if rng.random() < 0.4:
                c.update(_EXPERT)
            if c["E"] * c["H"] * c["F"] <= 128 * 2048 * 768:
                return c
            continue
        c = dict(kind=kind, B=logint(1, 256), V=logint(1000, 200000), fp32=rng.random() < 0.6,
                 mode=rng.choice(["greedy", "plain", "top_k", "top_p", "top_k_p", "mixed", "mixed"]))
        if c["B"] * c["V"] <= 256 * 50001:
            return c


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, std=1.0):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=g)


def _weight8(g, *shape):
    """A weight of N(0, 0.02^2) in int8, channels [..., N, K], and its scales [..., N]."""
    q = _normal(g, *shape, std=36.0).round_().clamp_(-127, 127).to(torch.int8)
    s = (0.02 / 36.0) * (0.8 + 0.4 * torch.rand(shape[:-1], device="cuda", generator=g))
    return q, s


def _stream(g, T, H):
    """Rows of a residual stream: unit size, a few channels far larger."""
    x = _normal(g, T, H)
    x[:, :: max(1, H // 8)] *= 8
    return x


def _inputs(case, seed):
    g, kind = _gen(seed), case["kind"]
    if kind in ("norm", "norm_bwd"):
        T, H = case["T"], case["H"]
        t = dict(x=_stream(g, T, H), w=1 + _normal(g, H, std=0.1))
        if kind == "norm":
            t["r"] = _stream(g, T, H) if case["residual"] else None
        else:
            t["dy"] = _normal(g, T, H)
            t["dh"] = _normal(g, T, H) if case["dh"] else None
        return t
    if kind == "decode":
        T, E, H, F, k = (case[n] for n in ("T", "E", "H", "F", "k"))
        w_r = _normal(g, H, E, std=0.02)
        x = _normal(g, T + T // 4 + 8, H)
        if k < E:
            # a token whose k-th expert hangs on the last bits of a sum has no one answer
            z = (x.double() @ w_r.double()).sort(-1, descending=True).values
            near = z[:, k - 1] - z[:, k] < 1e-3
            x = x[near.int().argsort(stable=True)]
        t = dict(x=x[:T].contiguous(), w_r=w_r, mask=None)
        if case["mask"]:
            t["mask"] = (torch.rand(T, device="cuda", generator=g) > 1 / 8).to(torch.uint8)
            t["mask"][0] = 1
        for n, (K, N) in dict(gate=(H, F), up=(H, F), down=(F, H)).items():
            if case["i8"]:
                t["w_" + n], t["s_" + n] = _weight8(g, E, N, K)
            else:
                t["w_" + n] = _normal(g, E, K, N, std=0.02)
        return t
    B, V, mode = case["B"], case["V"], case["mode"]
    logits = torch.empty((B, V), device="cuda").normal_(0.0, 2.5, generator=g)
    # a few dozen tokens that the context makes likely
    likely = torch.randint(0, V, (B, 32), device="cuda", generator=g)
    logits.scatter_add_(1, likely, 10 * torch.rand((B, 32), device="cuda", generator=g))

    def pick(*values):
        return torch.tensor(values, device="cuda")[torch.randint(0, len(values), (B,), device="cuda", generator=g)]

    def same(v):
        return torch.full((B,), v, device="cuda")

    t = dict(logits=logits if case["fp32"] else logits.bfloat16(), u=torch.rand(B, device="cuda", generator=g),
             temperature=same(0.0 if mode == "greedy" else 0.8), top_k=None, top_p=None, min_p=None)
    if mode in ("top_k", "top_k_p"):
        t["top_k"] = same(50).to(torch.int32)
    if mode in ("top_p", "top_k_p"):
        t["top_p"] = same(0.9)
    if mode == "mixed":
        t.update(temperature=pick(0.0, 0.7, 1.0, 1.3), top_k=pick(0, 20, 50, 1000).to(torch.int32),
                 top_p=pick(1.0, 0.8, 0.95), min_p=pick(0.0, 0.02, 0.1))
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    st = dict(case=case, t=t)
    if not own:
        return st
    import paper_2608_00916_amd as moe
    kind = case["kind"]
    if kind == "norm":
        st["op"] = moe.RMSNorm(case["T"], t["w"], eps=_EPS, out=case["out"])
    elif kind == "norm_bwd":
        st["op"] = moe.RMSNorm(case["T"], t["w"], eps=_EPS, dw_fp32=case["fp32"], backward=True)
    elif kind == "decode":
        shape = [case[n] for n in ("T", "H", "E", "F", "k")]
        if case["i8"]:
            st["w8"] = moe.i8_weights(*(t[n] for n in ("w_gate", "s_gate", "w_up", "s_up", "w_down", "s_down")))
            st["op"] = moe.MoEDecodeI8(*shape, mask=case["mask"])
        else:
            st["op"] = moe.MoEDecode(*shape, mask=case["mask"])
    else:
        st["op"] = moe.Sampler(case["B"], case["V"])
    return st


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    t, case, op = st["t"], st["case"], st["op"]
    kind = case["kind"]
    if kind == "norm":
        h, y, q, scale = op.forward(t["x"], t["r"])
        return _norm_outputs(case, h, y, q, scale)
    if kind == "norm_bwd":
        return op.backward(t["x"], t["dy"], t["dh"])
    if kind == "decode":
        if case["i8"]:
            return op.forward(t["x"], t["w_r"], st["w8"], t["mask"])
        return op.forward(t["x"], t["w_r"], t["w_gate"], t["w_up"], t["w_down"], t["mask"])
    return op.forward(t["logits"], t["u"], temperature=t["temperature"], top_k=t["top_k"], top_p=t["top_p"],
                      min_p=t["min_p"])


def _norm_outputs(case, h, y, q, scale):
    """The sum (where it is one), the normed rows, the values that the int8 rows stand for (in bf16)."""
    outs = dict(h=h) if case["residual"] else {}
    if case["out"] != "i8":
        outs["y"] = y
    if case["out"] != "bf16":
        outs["q"] = torch.mul(q, scale[:, None], out=torch.empty(q.shape, dtype=torch.bfloat16, device=q.device))
    return outs


# ------------------------------------------------------------------ plain form
def _quant(x):
    """Rows of x (fp32) in int8 values (held in fp32) and a scale for each."""
    top = x.abs().amax(-1, keepdim=True)
    return torch.where(top > 0, x * 127 / top, 0).round(), top / 127


def _run_plain(st):
    t, case = st["t"], st["case"]
    kind = case["kind"]
    if kind == "norm":
        h = t["x"]
        if case["residual"]:
            h = (h.float() + t["r"].float()).bfloat16()
        x = h.float()
        v = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * t["w"].float()
        q, s = _quant(v) if case["out"] != "bf16" else (None, None)
        return _norm_outputs(case, h, v.bfloat16(), q, s if s is None else s[:, 0])
    if kind == "norm_bwd":
        h, dy = t["x"].float(), t["dy"].float()
        s = torch.rsqrt((h * h).mean(-1, keepdim=True) + _EPS)
        n, g = h * s, dy * t["w"].float()
        dx = s * (g - n * (g * n).mean(-1, keepdim=True))
        if case["dh"]:
            dx = dx + t["dh"].float()
        dw = (dy * n).sum(0)
        return dx.bfloat16(), dw if case["fp32"] else dw.bfloat16()
    return _decode_plain(t, case) if kind == "decode" else _sample_plain(t, case)


def _decode_plain(t, case):
    T, E, k = case["T"], case["E"], case["k"]
    x = t["x"].float()
    z, idx = torch.sort(x @ t["w_r"].float(), dim=-1, descending=True, stable=True)
    z, idx = z[:, :k], idx[:, :k]
    gates = (z - z[:, :1]).exp()
    gates = gates / gates.sum(-1, keepdim=True)
    if t["mask"] is not None:
        gates = gates * t["mask"][:, None]
    few = T * k < E  # the slots' own experts, or every token through every expert
    pick = idx.reshape(-1) if few else slice(None)

    def product(rows, name):
        """rows [slots or E, tokens, K] through their experts' matrix."""
        w = t["w_" + name][pick].float()
        if not case["i8"]:
            return torch.bmm(rows, w)
        q, s = _quant(rows)
        return torch.bmm(q, w.transpose(1, 2)) * s * t["s_" + name][pick][:, None]

    rows = x.repeat_interleave(k, 0)[:, None] if few else x.expand(E, *x.shape)
    gate = product(rows, "gate")
    o = product(gate * torch.sigmoid(gate) * product(rows, "up"), "down")
    if few:
        return (o.view(T, k, -1) * gates[..., None]).sum(1).bfloat16()
    dense = gates.new_zeros(T, E).scatter_(1, idx, gates)
    return (o * dense.T[..., None]).sum(0).bfloat16()


def _sample_plain(t, case):
    V = case["V"]
    v, order = torch.sort(t["logits"].float(), dim=-1, descending=True, stable=True)
    rank = torch.arange(V, device=v.device)
    temp = t["temperature"].double()[:, None]
    greedy = temp <= 0
    d = (v.double() - v[:, :1].double()) / torch.where(greedy, 1.0, temp)
    w = d.exp()
    keep = ~greedy | (rank == 0)
    if t["top_k"] is not None:
        k = t["top_k"][:, None]
        keep &= (rank < k) | (k <= 0)
    w = torch.where(keep, w, 0)
    if t["top_p"] is not None:
        p, c = t["top_p"].double()[:, None], w.cumsum(-1)
        w = torch.where((c - w < p * c[:, -1:]) | (p >= 1), w, 0)
    if t["min_p"] is not None:
        w = torch.where(w >= t["min_p"].double()[:, None], w, 0)
    c = torch.zeros_like(w).scatter_(1, order, w).cumsum(-1)
    z = c[:, -1:]
    token = (c <= t["u"].double()[:, None] * z).sum(-1, keepdim=True).clamp(max=V - 1)
    at = t["logits"].gather(1, token).double()
    logprob = torch.where(greedy, 0.0, (at - v[:, :1].double()) / torch.where(greedy, 1.0, temp) - z.log())
    return token[:, 0].to(torch.int32), logprob[:, 0].float()


# ------------------------------------------------------------------ work
def work(case):
    """Bytes of every input and output once, operations of the products."""
    kind = case["kind"]
    if kind == "norm":
        n = case["T"] * case["H"]
        each = 2 + (4 if case["residual"] else 0) + dict(bf16=2, i8=1, both=3)[case["out"]]
        return dict(bytes=each * n + 2 * case["H"] + 4 * case["T"], flops=6 * n)
    if kind == "norm_bwd":
        n = case["T"] * case["H"]
        return dict(bytes=(8 if case["dh"] else 6) * n + (6 if case["fp32"] else 4) * case["H"], flops=12 * n)
    if kind == "decode":
        T, E, H, F, k = (case[n] for n in ("T", "E", "H", "F", "k"))
        rows = T * k * (7 / 8 if case["mask"] else 1)
        used = E * (1 - (1 - k / E) ** (rows / k))  # experts with a row
        expert = (3 * H * F + 8 * F + 4 * H) if case["i8"] else 6 * H * F
        return dict(bytes=used * expert + 2 * H * E + 4 * T * H, flops=6 * H * F * rows + 2 * T * H * E)
    return dict(bytes=case["B"] * (case["V"] * (4 if case["fp32"] else 2) + 28), flops=4 * case["B"] * case["V"])


# ------------------------------------------------------------------ the same in 64 bits
def _q64(x):
    """What the int8 rows of x stand for."""
    top = x.abs().max(dim=-1, keepdim=True).values
    return torch.nan_to_num((127.0 * x / top).round(), nan=0.0) * (top / 127.0)


def exact(case, seed):
    t, kind = _inputs(case, seed), case["kind"]
    if kind == "norm":
        h = t["x"].double() + (t["r"].double() if case["residual"] else 0)
        n = h.bfloat16().double()  # the norm is that of the sum as it is stored
        y = n / (n.square().mean(-1, keepdim=True) + _EPS).sqrt() * t["w"].double()
        outs = dict(h=h) if case["residual"] else {}
        if case["out"] != "i8":
            outs["y"] = y
        if case["out"] != "bf16":
            outs["q"] = _q64(y)
        return outs
    if kind == "norm_bwd":
        h, dy, w = t["x"].double(), t["dy"].double(), t["w"].double()
        H = h.shape[1]
        r = (h.square().sum(-1, keepdim=True) / H + _EPS).sqrt()
        dx = dy * w / r - h * (dy * w * h).sum(-1, keepdim=True) / (H * r ** 3)
        if case["dh"]:
            dx += t["dh"].double()
        return dx, (h / r).mul(dy).sum(0)
    if kind == "decode":
        x, k = t["x"].double(), case["k"]
        z = x @ t["w_r"].double()
        y = torch.zeros_like(x)
        top, idx = z.topk(k, -1)
        gates = torch.softmax(top, -1)
        if t["mask"] is not None:
            gates = gates * t["mask"].double()[:, None]
        for e in range(case["E"]):
            at, slot = (idx == e).nonzero(as_tuple=True)
            if at.numel() == 0:
                continue
            if case["i8"]:
                wg, wu, wd = ((t["w_" + n][e].double() * t["s_" + n][e].double()[:, None]).T for n in ("gate", "up", "down"))
                rows = _q64(x[at])
                g = rows @ wg
                a = _q64(g / (1 + (-g).exp()) * (rows @ wu))
            else:
                wg, wu, wd = (t["w_" + n][e].double() for n in ("gate", "up", "down"))
                g = x[at] @ wg
                a = g / (1 + (-g).exp()) * (x[at] @ wu)
            y.index_add_(0, at, gates[at, slot][:, None] * (a @ wd))
        return y
    tokens, logs = [], []
    settings = {n: None if t[n] is None else t[n].tolist() for n in ("temperature", "top_k", "top_p", "min_p", "u")}
    for b in range(case["B"]):
        s = {n: None if v is None else v[b] for n, v in settings.items()}
        row = t["logits"][b].double()
        if s["temperature"] <= 0:
            tokens.append(int((row == row.max()).nonzero()[0]))
            logs.append(0.0)
            continue
        order = torch.argsort(row, descending=True, stable=True)
        p = torch.softmax(row[order] / s["temperature"], 0)
        if s["top_k"]:
            p = p[: s["top_k"]] / p[: s["top_k"]].sum()
        if s["top_p"] is not None and s["top_p"] < 1:
            before = torch.cat([p.new_zeros(1), p.cumsum(0)[:-1]])
            p = p[: int((before < s["top_p"] * p.sum()).sum())]
            p = p / p.sum()
        if s["min_p"]:
            p = p[: int((p / p[0] >= s["min_p"]).sum())]
            p = p / p.sum()
        ids, place = order[: p.numel()].sort()
        p = p[place]
        i = min(int(torch.searchsorted(p.cumsum(0), torch.tensor(s["u"], dtype=p.dtype, device=p.device), right=True)), p.numel() - 1)
        tokens.append(int(ids[i]))
        logs.append(math.log(float(p[i])))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(logs, dtype=torch.float64)
