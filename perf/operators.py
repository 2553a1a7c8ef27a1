"""Performance cases of 8-bit serving: the int8 products, dense and grouped
over the experts, the tables of the paged cache, the writes into its 8-bit
blocks and the attention over them.

`own` chooses between the plain form (elementary torch operations in fp32) and
the package's entry points.  A case is a dict of plain values: `kind` names the
operator, the rest are sizes and options.  Inputs are drawn on the GPU from the
seed alone.

The cache: block i of head h holds `bt` tokens, keys k[i, h, token, :], values
v[i, h, :, token] (int8) and one scale each, ks[i, h] and vs[i, h].
"""
import math

import torch

own = False

_HEADS = dict(heads=32, kv_heads=4, D=128)  # attention heads of a 30B-A3B model
_EXPERT = dict(H=2048, F=768)  # its expert layer


def listed():
    return [
        # The fused query/key/value projection of one token: latency, and one
        # read of the weights.
        dict(name="linear_1", kind="linear", M=1, K=2048, N=5120, fp32=False),
        # The same for two query groups of 8 passages x 512 tokens.
        dict(name="linear_8192", kind="linear", M=8192, K=2048, N=5120, fp32=False),
        # A head of odd width on a ragged batch, fp32 scores.
        dict(name="linear_ragged_3001", kind="linear", M=3001, K=640, N=1001, fp32=True),
        # Expert layer, one short query-passage pair (64 tokens, top-8):
        # reading every expert's weights.
        dict(name="experts_512", kind="experts", rows=512, E=128, **_EXPERT),
        # One expert-parallel rank of eight on a training-sized batch.
        dict(name="experts_8359", kind="experts", rows=8359, E=16, **_EXPERT),
        # Expert layer on 8192 tokens, top-8.
        dict(name="experts_65536", kind="experts", rows=65536, E=128, **_EXPERT),
        # Tables of one decoding step of a small batch.
        dict(name="plan_16", kind="plan", B=16, old=4096, new=1, bt=64, pad=0, short=False),
        # Tables of a large mixed batch, many requests with a few dozen tokens.
        dict(name="plan_4096", kind="plan", B=4096, old=2048, new=64, bt=16, pad=1000, short=False),
        # One token for each of 64 running requests into blocks that are
        # partly full, and the cache read back.
        dict(name="append_64", kind="append", B=64, old=100, new=1, bt=32, kv_heads=4, D=128),
        # 16 passages of up to 512 tokens behind a short cached prefix.
        dict(name="append_16x512", kind="append", B=16, old=100, new=512, bt=64, kv_heads=4, D=128),
        # Decoding one token each for 64 requests of up to 32768 tokens.
        dict(name="attend_64x32768", kind="attend", B=64, q=1, kv=32768, bt=64, causal=True, **_HEADS),
        # 16 passages of up to 512 tokens over the cached prefix before them.
        dict(name="attend_16x512", kind="attend", B=16, q=512, kv=4096, bt=64, causal=True, **_HEADS),
    ]


def draw(rng):
    """One more case: any operator over the listed cases' ranges, no costlier
    than that operator's largest of them."""
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {}
    for c in listed():
        most.setdefault(c["kind"], [0, 0])
        w = work(c)
        most[c["kind"]] = [max(most[c["kind"]][0], w["flops"]), max(most[c["kind"]][1], w["bytes"])]
    while True:
        kind = rng.choice(["linear", "linear", "experts", "plan", "append", "attend", "attend"])
        bt = rng.choice([16, 32, 64, 128])
        kv_heads, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128])
        if kind == "linear":
            c = dict(kind=kind, M=logint(1, 8192), K=16 * logint(8, 512), N=logint(64, 16384), fp32=rng.random() < 0.3)
        elif kind == "experts":
            c = dict(kind=kind, rows=logint(1, 65536), E=logint(1, 256), H=128 * logint(1, 32), F=128 * logint(1, 12))
            if rng.random() < 0.3:
                c.update(E=128, **_EXPERT)
        elif kind == "plan":
            c = dict(kind=kind, B=logint(1, 4096), old=logint(1, 8192), new=rng.choice([1, 1, logint(2, 512)]), bt=bt,
                     pad=rng.choice([0, logint(1, 1000)]), short=rng.random() < 0.3)
            if c["B"] * c["new"] > 262144 or c["B"] * (c["old"] + c["new"]) > 16 * 4096 * 2048:
                continue
            return c
        elif kind == "append":
            c = dict(kind=kind, B=logint(1, 256), old=logint(1, 512), new=rng.choice([1, logint(2, 1024)]), bt=bt,
                     kv_heads=kv_heads, D=D)
        else:
            c = dict(kind=kind, B=logint(1, 128), q=rng.choice([1, 1, logint(2, 1024)]), kv=logint(16, 32768), bt=bt,
                     causal=rng.random() < 0.8, heads=kv_heads * rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16]),
                     kv_heads=kv_heads, D=D)
            if c["q"] > c["kv"] or c["B"] * c["heads"] * c["q"] * c["kv"] > 16 * 32 * 512 * 4096:
                continue
        w = work(c)
        if w["flops"] <= most[kind][0] and w["bytes"] <= most[kind][1] and (kind != "experts" or c["E"] * c["H"] * c["F"] <= 128 * 2048 * 768):
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


def _cache(g, n, kv_heads, bt, D):
    """A full cache of n blocks: values of about unit size in every block."""
    k = _normal(g, n, kv_heads, bt, D, std=36.0).round_().clamp_(-127, 127).to(torch.int8)
    v = _normal(g, n, kv_heads, D, bt, std=36.0).round_().clamp_(-127, 127).to(torch.int8)
    ks, vs = (1 / 36.0 * (0.5 + torch.rand((n, kv_heads), device="cuda", generator=g)) for _ in range(2))
    return dict(k=k, v=v, ks=ks, vs=vs)


def _lengths(g, B, most, least, new):
    """Ragged lengths of B requests: up to `most` cached tokens, one request
    with all of them, and up to `new` new tokens (of a single one, a few
    requests idle).  The case fixes them, the seed which request has which."""
    fixed = _gen(B * 1000003 + most * 1009 + new)
    cached = torch.randint(least, most + 1, (B,), device="cuda", generator=fixed)
    fresh = torch.randint(0, new + 1, (B,), device="cuda", generator=fixed)
    if new == 1:
        fresh = (torch.rand(B, device="cuda", generator=fixed) > 1 / 16).long()
    cached[0], fresh[0] = most, new
    order = torch.randperm(B, device="cuda", generator=g)
    return cached[order].to(torch.int32), fresh[order].to(torch.int32)


def _table(g, kv, bt, width, n_blocks):
    """Block tables over a shuffled cache, -1 past a request's last block."""
    need = (kv + bt - 1) // bt
    at = torch.arange(width, device="cuda")[None, :]
    ids = torch.randperm(n_blocks, device="cuda", generator=g).to(torch.int32)
    i = (need.cumsum(0) - need)[:, None] + at
    return torch.where(at < need[:, None], ids[i.clamp(max=n_blocks - 1)], -1).to(torch.int32).contiguous()


def _inputs(case, seed):
    g, kind = _gen(seed), case["kind"]
    if kind == "linear":
        x = _normal(g, case["M"], case["K"])
        x[:, :: max(1, case["K"] // 8)] *= 8  # a few channels of large activations
        w, s = _weight8(g, case["N"], case["K"])
        return dict(x=x, w=w, s=s)
    if kind == "experts":
        R, E, H, F = (case[n] for n in ("rows", "E", "H", "F"))
        owner = torch.randint(0, E, (R,), device="cuda", generator=g)
        counts = torch.bincount(owner, minlength=E)
        t = dict(x=_normal(g, R, H), counts=counts.to(torch.int32), cap=int(counts.max()))
        for n, shape in dict(gate=(E, F, H), up=(E, F, H), down=(E, H, F)).items():
            t["w_" + n], t["s_" + n] = _weight8(g, *shape)
        return t
    B, bt = case["B"], case["bt"]
    if kind == "attend":
        kv, q_len = _lengths(g, B, case["kv"], max(1, case["kv"] // 4), case["q"])
        q_len = torch.minimum(q_len, kv)
        start = torch.cat([q_len.new_zeros(1), q_len.cumsum(0).to(torch.int32)])
        T, width = int(start[-1]), -(-case["kv"] // bt)
        n = int(((kv + bt - 1) // bt).sum())
        q = torch.empty((T, case["heads"], case["D"]), dtype=torch.bfloat16, device="cuda").normal_(0.0, 2.0, generator=g)
        return dict(q=q, start=start, kv=kv, table=_table(g, kv, bt, width, n), **_cache(g, n, case["kv_heads"], bt, case["D"]))
    old, new = _lengths(g, B, case["old"], 0, case["new"])
    after = old + new
    T, width = int(new.sum()), -(-(case["old"] + case["new"]) // bt)
    if kind == "plan":
        used = ((old + bt - 1) // bt).sum()
        need = int(((after + bt - 1) // bt).sum() - used)
        free = max(0, need - 1 - need // 8) if case["short"] else need + 17
        n = int(used) + need + 64
        table = _table(g, old, bt, width, int(used) + 1)
        ids = (n - 1 - torch.randperm(free + 5, device="cuda", generator=g)).to(torch.int32)
        return dict(old=old, new=new, table=table, free=ids, n_free=torch.tensor([free], dtype=torch.int32, device="cuda"),
                    T=T + case["pad"], n_blocks=n + 5)
    n = int(((after + bt - 1) // bt).sum())
    start = torch.cat([new.new_zeros(1), new.cumsum(0).to(torch.int32)])
    table = _table(g, after, bt, width, n)
    kv_start = torch.cat([new.new_zeros(1), after.cumsum(0).to(torch.int32)])
    kn, vn = (1.5 * _normal(g, T, case["kv_heads"], case["D"]) for _ in range(2))
    return dict(k_new=kn, v_new=vn, old=old, start=start, kv=after, kv_start=kv_start, total=int(after.sum()),
                table=table, **_cache(g, n, case["kv_heads"], bt, case["D"]))


def prepare(case, seed):
    t = _inputs(case, seed)
    st = dict(case=case, t=t)
    if not own:
        return st
    import paper_2608_00916_amd as moe
    kind = case["kind"]
    if kind == "linear":
        st["op"] = moe.I8Linear(case["M"], t["w"], t["s"], out_fp32=case["fp32"])
    elif kind == "experts":
        st["w8"] = moe.i8_weights(*(t[n] for n in ("w_gate", "s_gate", "w_up", "s_up", "w_down", "s_down")))
        st["op"] = moe.MoEExpertsI8(case["rows"], case["H"], case["E"], case["F"])
    elif kind == "plan":
        st["op"] = moe.KVPlan(case["B"], t["T"], t["table"].shape[1], t["n_blocks"], case["bt"])
    else:
        st["cache"] = moe.KVCache.of(t["k"], t["v"], t["ks"], t["vs"])
        if kind == "append":
            st["out"] = [torch.empty((t["total"], case["kv_heads"], case["D"]), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        else:
            st["op"] = moe.KVAttention(st["cache"].d, t["q"].shape[0], case["heads"], case["B"], case["q"], case["kv"],
                                       causal=case["causal"])
    return st


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    t, kind = st["t"], st["case"]["kind"]
    if kind == "linear":
        return st["op"].forward(t["x"])
    if kind == "experts":
        return st["op"].forward(t["x"], t["counts"], st["w8"])
    if kind == "plan":
        p = st["op"]
        p.build(t["old"], t["new"], t["table"], t["free"], t["n_free"])
        return p.row_start, p.kv_len, p.positions, p.slots, p.seq, t["table"], p.state
    if kind == "append":
        st["cache"].append(t["k_new"], t["v_new"], t["start"], t["kv"], t["table"])
        return st["cache"].read(t["table"], t["kv_start"], *st["out"])
    return st["op"].forward(t["q"], st["cache"], t["table"], t["start"], t["kv"])


# ------------------------------------------------------------------ plain form
def _quant(x):
    """Rows of x (fp32) in int8 values (held in fp32) and a scale for each."""
    top = x.abs().amax(-1, keepdim=True)
    return torch.where(top > 0, x * 127 / top, 0).round(), top / 127


def _tokens(start, T):
    """Request of each packed token, and its place in the request."""
    at = torch.arange(T, device=start.device)
    b = torch.searchsorted(start[1:].contiguous(), at.to(torch.int32), right=True)
    ok = b < start.numel() - 1
    b = b.clamp(max=start.numel() - 2)
    return b, at - start[b], ok


def _run_plain(st):
    t, case = st["t"], st["case"]
    kind = case["kind"]
    if kind == "linear":
        q, s = _quant(t["x"].float())
        out = (q @ t["w"].float().T) * s * t["s"]
        return out if case["fp32"] else out.bfloat16()
    if kind == "experts":
        return _experts_plain(t, case)
    if kind == "plan":
        return _plan_plain(t, case)
    if kind == "append":
        return _append_plain(t, case)
    return _attend_plain(t, case)


def _experts_plain(t, case):
    counts = t["counts"].long()
    R, E = t["x"].shape[0], counts.numel()
    e = torch.repeat_interleave(torch.arange(E, device="cuda"), counts, output_size=R)
    i = torch.arange(R, device="cuda") - (counts.cumsum(0) - counts)[e]

    def product(rows, name):
        q, s = _quant(rows)
        per = q.new_zeros(E, t["cap"], q.shape[1])  # each expert's rows, padded to the most that one has
        per[e, i] = q
        return torch.bmm(per, t["w_" + name].float().transpose(1, 2))[e, i] * s * t["s_" + name][e]

    x = t["x"].float()
    gate = product(x, "gate")
    a = gate * torch.sigmoid(gate) * product(x, "up")
    return product(a, "down").bfloat16()


def _plan_plain(t, case):
    bt, (B, W) = case["bt"], t["table"].shape
    old, new = t["old"].long(), t["new"].long()
    have, want = ((old + bt - 1) // bt).clamp(max=W), ((old + new + bt - 1) // bt)
    need = want.clamp(max=W) - have
    first = need.cumsum(0) - need
    at = torch.arange(W, device="cuda")[None, :]
    j = first[:, None] + at - have[:, None]
    taken = (at >= have[:, None]) & (at < have[:, None] + need[:, None])
    n_free = t["n_free"].long()
    ids = t["free"][(n_free - 1 - j).clamp(0, t["free"].numel() - 1)]
    table = torch.where(taken, torch.where(j < n_free, ids, -1), t["table"]).to(torch.int32)
    start = torch.cat([new.new_zeros(1), new.cumsum(0)])
    b, i, ok = _tokens(start.to(torch.int32), t["T"])
    pos = old[b] + i
    block = table[b, (pos // bt).clamp(max=W - 1)].long()
    good = ok & (pos // bt < W) & (block >= 0)
    slots = torch.where(good, block * bt + pos % bt, -1)
    left = (n_free - need.sum()).clamp(min=0)
    missing = (need.sum() - n_free).clamp(min=0) + (want - want.clamp(max=W)).sum()
    whole = lambda x: x.to(torch.int32)  # noqa: E731
    return (whole(start), whole(old + new), whole(torch.where(ok, pos, -1)), whole(slots), whole(torch.where(ok, b, -1)),
            table, whole(torch.cat([left, missing])))


def _append_plain(t, case):
    bt, Hk, D = case["bt"], case["kv_heads"], case["D"]
    T, n = t["k_new"].shape[0], t["k"].shape[0]
    b, i, _ = _tokens(t["start"], T)
    pos = t["old"][b].long() + i
    block, off = t["table"][b, pos // bt].long(), pos % bt
    head = torch.arange(Hk, device="cuda")

    def write(x, q, s):  # x [T, Hk, D]; q [n, Hk, bt, D] as fp32
        opened = torch.zeros(n, device="cuda").index_add_(0, block, (off == 0).float()) > 0
        s0 = torch.where(opened[:, None], 0, s)
        amax = torch.zeros_like(s).index_reduce_(0, block, x.abs().amax(-1), "amax")
        s1 = torch.maximum(s0, amax / 127)
        q = (q * torch.where(s1 > 0, s0 / s1, 0)[:, :, None, None]).round()
        q[block[:, None], head[None, :], off[:, None]] = (x / s1[block].clamp(min=1e-45)[:, :, None]).round().clamp(-127, 127)
        return q, s1

    k, ks = write(t["k_new"].float(), t["k"].float(), t["ks"])
    v, vs = write(t["v_new"].float(), t["v"].float().transpose(2, 3), t["vs"])
    rb, ri, _ = _tokens(t["kv_start"], t["total"])
    blk, o = t["table"][rb, ri // bt].long(), ri % bt
    pick = lambda q, s: (q[blk[:, None], head[None, :], o[:, None]] * s[blk][:, :, None]).bfloat16()  # noqa: E731
    return pick(k, ks), pick(v, vs)


def _attend_plain(t, case):
    bt, Hk, D = case["bt"], case["kv_heads"], case["D"]
    T, Hq, _ = t["q"].shape
    B, W = t["table"].shape
    Q = case["q"]
    blk = t["table"].clamp(min=0).long()
    k = (t["k"][blk].float() * t["ks"][blk][..., None, None]).transpose(1, 2).reshape(B, Hk, W * bt, D)
    v = (t["v"][blk].float() * t["vs"][blk][..., None, None]).permute(0, 2, 1, 4, 3).reshape(B, Hk, W * bt, D)
    b, i, _ = _tokens(t["start"], T)
    q = t["q"].new_zeros(B, Q, Hq, D, dtype=torch.float32)  # each request's tokens, padded to the most
    q[b, i] = t["q"].float()
    q = q.view(B, Q, Hk, Hq // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, D)
    s = torch.matmul(q, k.transpose(2, 3)).view(B, Hk, Hq // Hk, Q, W * bt) * D ** -0.5
    kv = t["kv"].long()
    j = torch.arange(W * bt, device="cuda")
    last = kv[:, None].expand(B, Q) - 1
    if case["causal"]:
        last = kv[:, None] - (t["start"][1:] - t["start"][:-1])[:, None] + torch.arange(Q, device="cuda")
        last = torch.minimum(last, kv[:, None] - 1)
    s.masked_fill_((j > last[..., None])[:, None, None], float("-inf"))
    p = (s - s.amax(-1, keepdim=True)).exp_()
    p /= p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hk, -1, W * bt), v).view(B, Hk, Hq // Hk, Q, D).permute(0, 3, 1, 2, 4).reshape(B, Q, Hq, D)
    return o[b, i].bfloat16()


# ------------------------------------------------------------------ work
def _mean_new(most):
    return 0.5 * most if most > 1 else 15 / 16


def work(case):
    """Bytes of every input and output once (ragged lengths at their mean),
    operations of the products."""
    kind = case["kind"]
    if kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return dict(bytes=2 * M * K + N * K + 4 * N + (4 if case["fp32"] else 2) * M * N, flops=2 * M * N * K)
    if kind == "experts":
        R, E, H, F = (case[n] for n in ("rows", "E", "H", "F"))
        used = E * (1 - (1 - 1 / E) ** R)  # experts with a row
        return dict(bytes=4 * R * H + 4 * E + used * (3 * H * F + 8 * F + 4 * H), flops=6 * R * H * F)
    B = case["B"]
    if kind == "attend":
        Hq, Hk, D = case["heads"], case["kv_heads"], case["D"]
        kv = 0.625 * case["kv"]
        q = _mean_new(case["q"])
        seen = max(1.0, kv - 0.5 * q) if case["causal"] else kv
        return dict(bytes=B * (2 * kv * Hk * (D + 4 / case["bt"]) + 4 * q * Hq * D + 4 * kv / case["bt"] + 8),
                    flops=4 * B * q * seen * Hq * D)
    old, new = 0.5 * case["old"], _mean_new(case["new"])
    if kind == "plan":
        entries = B * (new / case["bt"])
        return dict(bytes=16 * B + 12 * (B * new + case["pad"]) + 12 * entries + 4 * B, flops=0)
    # append: the new tokens in, the touched blocks out; read: all of it out
    row = case["kv_heads"] * case["D"]
    touched = new + 0.5 * case["bt"]
    return dict(bytes=B * (4 * new * row + 4 * touched * row + 2 * (old + new) * row + 4 * (old + new) * row), flops=0)


# ------------------------------------------------------------------ the same in 64 bits
def _q64(x):
    top = x.abs().max(dim=-1, keepdim=True).values
    return torch.nan_to_num((127.0 * x / top).round(), nan=0.0), top / 127.0


def exact(case, seed):
    kind = case["kind"]
    if kind == "plan":
        return None  # whole numbers only
    t = _inputs(case, seed)
    if kind == "linear":
        q, s = _q64(t["x"].double())
        return (q * s) @ (t["w"].double() * t["s"].double()[:, None]).T
    if kind == "experts":
        outs = []
        for e, rows in enumerate(t["x"].split(t["counts"].tolist())):
            if rows.shape[0] == 0:
                continue
            wg, wu, wd = (t["w_" + n][e].double() * t["s_" + n][e].double()[:, None] for n in ("gate", "up", "down"))
            q, s = _q64(rows.double())
            g, u = (q * s) @ wg.T, (q * s) @ wu.T
            q, s = _q64(g / (1 + (-g).exp()) * u)
            outs.append((q * s) @ wd.T)
        return torch.cat(outs)
    bt, start = case["bt"], t["start"].tolist()
    kv, table = t["kv"].tolist(), t["table"].tolist()
    k, v, ks, vs = t["k"].double(), t["v"].double().transpose(2, 3), t["ks"].double(), t["vs"].double()
    if kind == "append":
        for new, q8, sc in ((t["k_new"], k, ks), (t["v_new"], v, vs)):
            for b, old in enumerate(t["old"].tolist()):
                p = old
                while p < kv[b]:
                    blk, o = table[b][p // bt], p % bt
                    m = min(bt - o, kv[b] - p)
                    x = new[start[b] + p - old:start[b] + p - old + m].double().transpose(0, 1)
                    s0 = sc[blk] if o else torch.zeros_like(sc[blk])
                    s1 = torch.maximum(s0, x.abs().amax((1, 2)) / 127)
                    q8[blk] = (q8[blk] * (s0 / s1)[:, None, None]).round()
                    q8[blk, :, o:o + m] = (x / s1[:, None, None]).round()
                    sc[blk] = s1
                    p += m
        rows = []
        for b in range(case["B"]):
            at = torch.arange(kv[b], device="cuda")
            blk = t["table"][b].long()[at // bt]
            rows.append((blk, at % bt))
        blk, o = (torch.cat(x) for x in zip(*rows))
        return tuple(q8[blk, :, o] * sc[blk][:, :, None] for q8, sc in ((k, ks), (v, vs)))
    Hk, Hq, D = case["kv_heads"], case["heads"], case["D"]
    out = torch.zeros(t["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        n, L = start[b + 1] - start[b], kv[b]
        if n == 0:
            continue
        blk = t["table"][b, :-(-L // bt)].long()
        kk, vv = ((x[blk] * s[blk][:, :, None, None]).transpose(0, 1).reshape(Hk, -1, D)[:, :L] for x, s in ((k, ks), (v, vs)))
        q = t["q"][start[b]:start[b + 1]].double().view(n, Hk, Hq // Hk, D).permute(1, 2, 0, 3).reshape(Hk, -1, D)
        s = (q @ kk.transpose(1, 2)).view(Hk, Hq // Hk, n, L) / math.sqrt(D)
        if case["causal"]:
            at = torch.arange(L, device="cuda")[None, :] - torch.arange(n, device="cuda")[:, None]
            s = s.masked_fill(at > L - n, float("-inf"))
        o = torch.softmax(s, -1).view(Hk, -1, L) @ vv
        out[start[b]:start[b + 1]] = o.view(Hk, Hq // Hk, n, D).permute(2, 0, 1, 3).reshape(n, Hq, D)
    return out
