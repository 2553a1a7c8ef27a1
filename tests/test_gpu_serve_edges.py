"""GPU tests of the 8-bit serving operators at the edges of what their calls
accept: bounds that are loose, tables that start late or end early, buffers
that are replaced, operands at the ends of their types."""
import numpy as np
import pytest

from tests import serve_ref as R
from tests.test_gpu_serve import Pages, attend, bf16, dev, gen, host, i32, int8_rows, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bt", [16, 128])
@pytest.mark.parametrize("first", [1, 63, 64, 1000])
def test_read_into_rows_that_start_late(bt, first):
    """kv_start need not begin at 0: the rows before it are left alone, the others are those of a
    read that begins at 0."""
    import torch
    say("read late", bt, first)
    lens = [70, 0, 5, 200]
    pg = Pages(gen(31), lens, bt, 2, 64)
    start = np.concatenate([[0], np.cumsum(lens)])
    total = int(start[-1])
    want = [torch.empty((total, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pg.cache.read(dev(pg.table), i32(start), *want)
    got = [torch.full((first + total + 3, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pg.cache.read(dev(pg.table), i32(start + first), *got)
    for x, y in zip(got, want):
        assert torch.equal(x[first:first + total], y)
        assert (x[:first] == 9).all() and (x[first + total:] == 9).all()


@pytest.mark.parametrize("max_q", [2 ** 29, 2 ** 29 + 1, 2 ** 31 - 1])
def test_a_loose_max_q(max_q):
    """max_q only bounds a request's new tokens: times the heads of a group it may pass 32 bits."""
    say("loose max_q", max_q)
    pg = Pages(gen(32), [5000, 9, 2600], 64, 1, 128)
    attend(pg, [1, 1, 0], [5000, 9, 2600], 8, max_q=max_q)
    attend(pg, [1, 2, 4], [5000, 9, 2600], 8, max_q=max_q)
    attend(pg, [40, 2, 3], [5000, 9, 2600], 8, max_q=max_q)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("T", [0, 4, 5, 23, 24, 60])
def test_fewer_rows_than_new_tokens(T, causal):
    """Rows past T do not exist, and what there is of a request are its first new tokens: the cache
    and the output are those of a batch that has only these."""
    import torch
    import paper_2608_00916_amd as moe
    say("short T", T, causal)
    g = gen(33)
    bt, heads, D, W = 16, 2, 64, 8
    old, new = [0, 35, 3, 20], [4, 20, 100, 1]
    fit = np.clip(T - (np.cumsum(new) - new), 0, new)
    kv = bf16(g.standard_normal((2, 140, heads, D)))
    k, v = bf16(g.standard_normal((125, heads, D))), bf16(g.standard_normal((125, heads, D)))
    q = bf16(2 * g.standard_normal((125, 4, D)))
    free = dev(g.permutation(40).astype(np.int32))
    got = []
    for step in (np.array(new), fit):
        cache = moe.KVCache(40, bt, heads, D)
        cache.k.fill_(77), cache.v.fill_(-55), cache.k_scale.fill_(3.0), cache.v_scale.fill_(2.0)
        table = i32(np.full((4, W), -1))
        n_free = i32([40])
        if sum(old):
            plan = moe.KVPlan(4, sum(old), W, 40, bt)
            plan.build(i32([0] * 4), i32(old), table, free, n_free)
            cache.append(kv[0, :sum(old)], kv[1, :sum(old)], plan.row_start, plan.kv_len, table)
            n_free = plan.state[:1].clone()
        plan = moe.KVPlan(4, T, W, 40, bt)
        plan.build(i32(old), i32(step), table, free, n_free)
        cache.append(k[:T], v[:T], plan.row_start, plan.kv_len, table)
        op = moe.KVAttention(cache, T, 4, 4, 100, W * bt, causal=causal)
        op.out.fill_(3.0)
        out = op.forward(q[:T], cache, table, plan.row_start, plan.kv_len).clone()
        after = np.array(old) + fit
        start = np.concatenate([[0], np.cumsum(after)])
        ko, vo = (torch.empty((int(start[-1]), heads, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        cache.read(table, i32(start), ko, vo)
        got.append((plan.positions.clone(), out, ko, vo))
    for x, y in zip(*got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("B,W", [(3, 40), (256, 6), (700, 6), (9000, 5)])
def test_plan_in_place(B, W):
    """A step's lengths and stack are the next one's: passed as they are, the tables are those of copies."""
    import torch
    import paper_2608_00916_amd as moe
    say("plan in place", B)
    g = gen(34)
    bt, n = 16, 5 * B + 50
    free = dev(g.permutation(n).astype(np.int32))
    steps = [g.integers(-1, 30, B) * (g.random(B) > 0.2) for _ in range(4)]
    T = max(int(np.maximum(s, 0).sum()) for s in steps) + 3
    a, b = (moe.KVPlan(B, T, W, n, bt) for _ in range(2))
    ta, tb = (i32(np.full((B, W), -1)) for _ in range(2))
    a.kv_len.zero_(), a.state.fill_(n)
    length, n_free = i32(np.zeros(B)), i32([n])
    for s in steps:
        a.build(a.kv_len, i32(s), ta, free, a.state[:1])
        b.build(length, i32(s), tb, free, n_free)
        length, n_free = b.kv_len.clone(), b.state[:1].clone()
        for name in ("row_start", "kv_len", "positions", "slots", "seq", "state"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
        assert torch.equal(ta, tb)
    # the new tokens' own tensor may take the lengths as well
    s = i32(steps[0])
    want = moe.KVPlan(B, T, W, n, bt)
    want.build(length, s, tb, free, n_free)
    a.kv_len.copy_(s)
    a.build(length, a.kv_len, ta, free, n_free)
    for name in ("row_start", "kv_len", "positions", "slots", "seq", "state"):
        assert torch.equal(getattr(a, name), getattr(want, name)), name


def test_plan_from_an_empty_stack():
    """No stack at all: requests that need no block go on, the others get none."""
    import torch
    import paper_2608_00916_amd as moe
    say("plan without a stack")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    table = i32([[4, -1], [5, -1]])
    plan = moe.KVPlan(2, 5, 2, 10, 16)
    plan.build(i32([3, 15]), i32([2, 3]), table, none, i32([7]))
    assert plan.slots.tolist() == [67, 68, 95, -1, -1] and plan.state.tolist() == [0, 1]
    assert table.tolist() == [[4, -1], [5, -1]]


def test_attention_over_another_cache():
    """What is made for one cache takes another of its head size, and refuses the rest."""
    import torch
    import paper_2608_00916_amd as moe
    say("attention over another cache")
    wide, narrow = (Pages(gen(35), [100], 16, 2, D) for D in (128, 64))
    op = moe.KVAttention(wide.cache, 1, 4, 1, 1, 100)
    args = dev(narrow.table), i32([0, 1]), i32([100])
    with pytest.raises(ValueError, match="head_dim"):
        op.forward(bf16(gen(36).standard_normal((1, 4, 64))), narrow.cache, *args)
    other = Pages(gen(37), [100], 32, 2, 128)
    q = bf16(gen(38).standard_normal((1, 4, 128)))
    got = op.forward(q, other.cache, dev(other.table), i32([0, 1]), i32([100]))
    assert torch.equal(got, moe.KVAttention(other.cache, 1, 4, 1, 1, 100).forward(q, other.cache, dev(other.table),
                                                                                 i32([0, 1]), i32([100])))


@pytest.mark.parametrize("M,N", [(1, 5), (20, 40), (33, 40), (300, 500), (1000, 1001), (2000, 1500), (4096, 4104)])
def test_matmul_of_the_lowest_values(M, N):
    """-128 in both operands at the largest K: the sum is 2^31 itself.  Every tile shape."""
    import torch
    import paper_2608_00916_amd as moe
    say("i8 matmul lowest", M, N)
    K = moe._lib.MOE_I8_MAX_K
    a = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    b = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    b[1], b[2] = 127, 0
    b[0, 5] = -127
    one = torch.ones(max(M, N), device="cuda")
    want = torch.full((N,), 2.0 ** 31, device="cuda")
    want[0], want[1], want[2] = 2.0 ** 31 - 128, -128.0 * 127 * K, 0
    for fp32 in (True, False):
        out = torch.empty((M, N), dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
        moe.moe_i8_matmul(a, one[:M], b, one[:N], out)
        assert (out == want.to(out.dtype)).all()


@pytest.mark.parametrize("rows", [3, 200, 3000])
def test_experts_closed_gates_of_huge_values(rows):
    """silu(G) U is 0 where the gate is far below 0, also where G U passes fp32."""
    import paper_2608_00916_amd as moe
    say("experts closed gates", rows)
    g = gen(39)
    H = F = 128
    x = bf16(np.abs(g.standard_normal((rows, H))) * 1e10)
    w = [g.integers(-127, 128, s).astype(np.int8) for s in ((1, F, H), (1, F, H), (1, H, F))]
    s = [np.full(n, 1.0, np.float32) for n in ((1, F), (1, F), (1, H))]
    w[0][:, 1::2] = -np.abs(w[0][:, 1::2])  # these gates are closed
    w[0][:, ::2] = 0
    w[0][:, ::2, 0] = 1
    s[0][:, 1::2] = 1e10
    s[1][:, 1::2] = 1e20
    s[0][:, ::2] = s[1][:, ::2] = 1e-12
    w8 = moe.i8_weights(*(dev(t) for p in zip(w, s) for t in p))
    got = host(moe.MoEExpertsI8(rows, H, 1, F).forward(x, i32([rows]), w8))
    assert np.isfinite(got).all()
    v = [t[0].astype(np.float64) * sc[0].astype(np.float64)[:, None] for t, sc in zip(w, s)]
    v[0], v[1], v[2] = v[0][::2], v[1][::2], v[2][:, ::2]
    ref = R.expert(host(x), *v)
    assert np.linalg.norm(got - ref) <= (2.0 ** -8 + 0.0005) * np.linalg.norm(ref)


def test_buffers_may_be_replaced():
    """The classes run on the tensors they hold at the time of the call."""
    import torch
    import paper_2608_00916_amd as moe
    say("buffers replaced")
    g = gen(40)
    (w, s), (w2, s2) = ([dev(t) for t in int8_rows(g, 64, 128)] for _ in range(2))
    x = bf16(g.standard_normal((5, 128)))
    lin = moe.I8Linear(5, w, s)
    lin.forward(x)
    lin.weight, lin.scale = w2, s2
    first, lin.out = lin.out, torch.empty_like(lin.out)
    want = moe.I8Linear(5, w2, s2).forward(x)
    assert torch.equal(lin.forward(x), want) and not torch.equal(first, want)
    with pytest.raises(ValueError):
        lin.weight = w2[:32]
    with pytest.raises(ValueError):
        lin.scale = s2.double()
    assert torch.equal(lin.forward(x), want)

    pg, other = (Pages(gen(n), [50], 16, 2, 64) for n in (41, 42))
    q = bf16(g.standard_normal((1, 4, 64)))
    at = dev(other.table), i32([0, 1]), i32([50])
    want = moe.KVAttention(other.cache, 1, 4, 1, 1, 50).forward(q, other.cache, *at)
    op = moe.KVAttention(pg.cache, 1, 4, 1, 1, 50)
    cache = pg.cache
    cache.k, cache.v, cache.k_scale, cache.v_scale = (getattr(other.cache, n) for n in ("k", "v", "k_scale", "v_scale"))
    op.out, op.ws = torch.empty_like(op.out), torch.empty_like(op.ws)
    assert torch.equal(op.forward(q, cache, *at), want)
    with pytest.raises(ValueError):
        cache.v = cache.v[:1]
    with pytest.raises(ValueError):
        op.ws = op.ws[:16]
    assert torch.equal(op.forward(q, cache, *at), want)

    ex = moe.MoEExpertsI8(4, 128, 1, 128)
    t = [dev(y) for shape in ((128, 128),) * 3 for y in int8_rows(g, *shape)]
    w8 = moe.i8_weights(*(y[None] for y in t))
    x = bf16(g.standard_normal((4, 128)))
    want = ex.forward(x, i32([4]), w8).clone()
    ex.o = torch.zeros_like(ex.o)
    assert torch.equal(ex.forward(x, i32([4]), w8), want)

    plan = moe.KVPlan(2, 3, 2, 10, 16)
    plan.slots = torch.full_like(plan.slots, 9)
    plan.build(i32([0, 0]), i32([1, 1]), i32([[-1, -1]] * 2), i32([4, 5]), i32([2]))
    assert plan.slots.tolist() == [80, 64, -1]


def test_attention_over_many_keys_without_values():
    """70000 keys whose values are all 0 before a block with values: the sum of their weights, which
    grow after the first block, stays in fp32."""
    import torch
    import paper_2608_00916_amd as moe
    say("zero values")
    L, bt, D, T, heads = 70016, 64, 64, 4096, 16
    n = L // bt
    cache = moe.KVCache(n, bt, 1, D)
    cache.k[1:] = 127
    cache.k_scale.fill_(1 / 127)
    cache.v[-1] = dev(gen(43).integers(-127, 128, (1, D, bt)).astype(np.int8))
    cache.v_scale[-1] = 0.01
    q = torch.full((T, heads, D), 1 / 16, dtype=torch.bfloat16, device="cuda")
    scale = 5.4 * 16 / D  # scores 0 in the first block, 5.4 from there on: below 8 in base 2
    table, kv = i32(np.arange(n)[None]), i32([L])
    v = host(cache.v[-1, 0]) * 0.01
    want = v.sum(1) / (L - bt + bt * np.exp(-5.4))
    for t, h in ((T, heads), (1, heads), (1, 4), (2, heads)):
        op = moe.KVAttention(cache, t, h, 1, t, L, causal=False, scale=scale)
        got = host(op.forward(q[:t, :h], cache, table, i32([0, t]), kv))
        bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -14) * np.abs(v).sum(1) / (L - bt)
        assert (np.abs(got - want) <= bound * 1.01).all(), (t, h)
