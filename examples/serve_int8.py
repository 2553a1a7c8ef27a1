"""One decoder layer served in 8 bits: prompts in one pass, then single tokens.

    python examples/serve_int8.py [--requests 16] [--tokens 512] [--steps 4]

Every step builds its tables from the request lengths on the GPU (KVPlan),
projects with int8 weights (I8Linear), writes the new keys and values into the
paged int8 cache and attends over it (KVCache, KVAttention), and runs the
expert layer with int8 weights (MoEInferI8).  Weights are random, of the
expert layer of a 30B-A3B MoE model by default; norms and rotary positions are
left out.  The last step is checked against the same layer in fp32, without a
cache, from the unrounded weights.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_00916_amd as moe  # noqa: E402


class Layer:
    """Weights in bf16 and, laid out once, in int8."""

    def __init__(self, H, heads, kv_heads, D, E, F, k, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape):
            return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.02, generator=g)

        self.H, self.heads, self.kv_heads, self.D, self.E, self.F, self.k = H, heads, kv_heads, D, E, F, k
        self.qkv, self.out = w(H, (heads + 2 * kv_heads) * D), w(heads * D, H)
        self.w_r, self.gate, self.up, self.down = w(H, E), w(E, H, F), w(E, H, F), w(E, F, H)
        self.qkv8, self.out8 = moe.moe_i8_quant_weight(self.qkv), moe.moe_i8_quant_weight(self.out)
        self.experts8 = moe.i8_weights(*(t for m in (self.gate, self.up, self.down) for t in moe.moe_i8_quant_weight(m)))


class Server:
    """Cache, block tables and free stack of up to B running requests."""

    def __init__(self, layer, B, max_kv, block_tokens=64):
        self.layer, self.B, self.max_kv, self.bt = layer, B, max_kv, block_tokens
        W = -(-max_kv // block_tokens)
        n = B * W
        self.cache = moe.KVCache(n, block_tokens, layer.kv_heads, layer.D)
        self.table = torch.full((B, W), -1, dtype=torch.int32, device="cuda")
        self.free = torch.arange(n, dtype=torch.int32, device="cuda")
        self.n_free = torch.tensor([n], dtype=torch.int32, device="cuda")
        self.length = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.ops = {}

    def _ops(self, T, max_q):
        """Buffers of a step of T packed tokens, at most max_q of one request."""
        if (T, max_q) not in self.ops:
            m = self.layer
            self.ops[T, max_q] = (
                moe.KVPlan(self.B, T, self.table.shape[1], self.cache.d.n_blocks, self.bt), moe.I8Linear(T, *m.qkv8),
                moe.KVAttention(self.cache, T, m.heads, self.B, max_q, self.max_kv), moe.I8Linear(T, *m.out8),
                moe.MoEInferI8(T, m.H, m.E, m.F, m.k))
        return self.ops[T, max_q]

    def step(self, x, new_len, max_q):
        """x [T, H]: the new tokens of all requests, packed in request order; returns the layer's output."""
        m = self.layer
        plan, qkv, attn, out, experts = self._ops(x.shape[0], max_q)
        plan.build(self.length, new_len, self.table, self.free, self.n_free)
        y = qkv.forward(x).view(-1, m.heads + 2 * m.kv_heads, m.D)
        q, k, v = y[:, :m.heads], y[:, m.heads:m.heads + m.kv_heads], y[:, m.heads + m.kv_heads:]
        self.cache.append(k, v, plan.row_start, plan.kv_len, self.table)
        a = attn.forward(q, self.cache, self.table, plan.row_start, plan.kv_len)
        h = x + out.forward(a.view(-1, m.heads * m.D))
        h = h + experts.forward(h, m.w_r, m.experts8)
        self.length, self.n_free = plan.kv_len, plan.state[:1]  # the next step's, also where it has the same plan
        return h


def reference(m, xs):
    """The layer on one request's tokens xs [n, H] in fp32; the last token's output."""
    x = xs.float()
    q, k, v = (x @ m.qkv.float()).view(len(x), -1, m.D).split([m.heads, m.kv_heads, m.kv_heads], 1)
    g = m.heads // m.kv_heads
    k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    p = torch.softmax((q[-1:] * k).sum(-1) * m.D ** -0.5, 0)
    h = x[-1] + (p[..., None] * v).sum(0).reshape(1, -1) @ m.out.float()
    z = (h @ m.w_r.float())[0]
    top, idx = z.topk(m.k)
    y = sum(gate * ((torch.nn.functional.silu(h @ m.gate[e].float()) * (h @ m.up[e].float())) @ m.down[e].float())
            for gate, e in zip(torch.softmax(top, 0), idx))
    return (h + y)[0]


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=512, help="longest prompt")
    ap.add_argument("--steps", type=int, default=4, help="single-token steps after the prompts")
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--experts", type=int, default=128)
    args = ap.parse_args(argv)
    B, H = args.requests, args.hidden
    layer = Layer(H, heads=32, kv_heads=4, D=128, E=args.experts, F=768, k=8)
    g = torch.Generator(device="cuda").manual_seed(1)

    def tokens(n):
        return torch.empty((n, H), dtype=torch.bfloat16, device="cuda").normal_(generator=g)

    lens = torch.randint(max(1, args.tokens // 2), args.tokens + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
    prompts = [tokens(n) for n in lens.tolist()]
    server = Server(layer, B, args.tokens + args.steps)

    def timed(name, *step):
        torch.cuda.synchronize()
        t = time.perf_counter()
        h = server.step(*step)
        torch.cuda.synchronize()
        print(f"{name}: {step[0].shape[0]} tokens, {(time.perf_counter() - t) * 1e3:.2f} ms", flush=True)
        return h

    timed("prompts", torch.cat(prompts), lens, args.tokens)
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    for i in range(args.steps):
        x = tokens(B)
        h = timed(f"token {i + 1}", x, one, 1)
        prompts = [torch.cat([p, x[b:b + 1]]) for b, p in enumerate(prompts)]
    errs = []
    for b in range(min(B, 4)):
        ref = reference(layer, prompts[b])
        errs.append(float((h[b].float() - ref).norm() / ref.norm()))
    print(f"against fp32 without a cache: relative error {max(errs):.4f}")
    return max(errs)


if __name__ == "__main__":
    main()
