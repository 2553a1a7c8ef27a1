"""One decoder layer and a head served in 8 bits: prompts in one pass, then single tokens.

    python examples/serve_int8.py [--requests 16] [--tokens 512] [--steps 4]

Every step builds its tables from the request lengths on the GPU (KVPlan),
norms its rows into int8 (RMSNorm) and projects them with int8 weights, writes
the new keys and values into the paged int8 cache and attends over it (KVCache,
KVAttention), sums with the residual and norms (RMSNorm), and runs the expert
layer with int8 weights (MoEInferI8, for up to 64 tokens MoEDecodeI8).  The head
norms each request's last row, projects it and draws the next token (Sampler).
Weights are random, of the expert layer of a 30B-A3B MoE model by default;
rotary positions are left out.  The last step is checked against the same layer
in fp32, without a cache, from the unrounded weights.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_00916_amd as moe  # noqa: E402


class Layer:
    """Weights in bf16 and, laid out once, in int8; without `norms` the rows go in as they are."""

    def __init__(self, H, heads, kv_heads, D, E, F, k, seed=0, norms=False):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape):
            return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.02, generator=g)

        self.H, self.heads, self.kv_heads, self.D, self.E, self.F, self.k = H, heads, kv_heads, D, E, F, k
        self.qkv, self.out = w(H, (heads + 2 * kv_heads) * D), w(heads * D, H)
        self.w_r, self.gate, self.up, self.down = w(H, E), w(E, H, F), w(E, H, F), w(E, F, H)
        self.n1, self.n2 = (1 + 5 * w(H), 1 + 5 * w(H)) if norms else (None, None)
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
            experts = moe.MoEDecodeI8 if T <= moe.MOE_DECODE_MAX_T else moe.MoEInferI8
            norms = None
            if m.n1 is not None:
                norms = moe.RMSNorm(T, m.n1, out="i8"), moe.RMSNorm(T, m.n2)
            self.ops[T, max_q] = (
                moe.KVPlan(self.B, T, self.table.shape[1], self.cache.d.n_blocks, self.bt), moe.I8Linear(T, *m.qkv8),
                moe.KVAttention(self.cache, T, m.heads, self.B, max_q, self.max_kv), moe.I8Linear(T, *m.out8),
                experts(T, m.H, m.E, m.F, m.k), norms)
        return self.ops[T, max_q]

    def step(self, x, new_len, max_q):
        """x [T, H]: the new tokens of all requests, packed in request order; returns the layer's output."""
        m = self.layer
        plan, qkv, attn, out, experts, norms = self._ops(x.shape[0], max_q)
        plan.build(self.length, new_len, self.table, self.free, self.n_free)
        if norms:
            _, _, q, s = norms[0].forward(x)  # already the product's int8 rows
            moe.moe_i8_matmul(q, s, *m.qkv8, qkv.out)
            y = qkv.out
        else:
            y = qkv.forward(x)
        y = y.view(-1, m.heads + 2 * m.kv_heads, m.D)
        q, k, v = y[:, :m.heads], y[:, m.heads:m.heads + m.kv_heads], y[:, m.heads + m.kv_heads:]
        self.cache.append(k, v, plan.row_start, plan.kv_len, self.table)
        a = attn.forward(q, self.cache, self.table, plan.row_start, plan.kv_len)
        a = out.forward(a.view(-1, m.heads * m.D))
        if norms:
            h, y, _, _ = norms[1].forward(a, x)
        else:
            h = y = x + a
        h = h + experts.forward(y, m.w_r, m.experts8)
        self.length, self.n_free = plan.kv_len, plan.state[:1]  # the next step's, also where it has the same plan
        return h


class Head:
    """Norm, vocabulary projection and draw of B requests' next tokens."""

    def __init__(self, B, H, vocab, seed=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.weight = torch.empty((H, vocab), dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.1, generator=g)
        self.weight8 = moe.moe_i8_quant_weight(self.weight)
        self.norm = moe.RMSNorm(B, torch.ones(H, dtype=torch.bfloat16, device="cuda"), out="i8")
        self.sampler = moe.Sampler(B, vocab)
        self.logits = torch.empty((B, vocab), device="cuda")

    def step(self, h, u, **settings):
        """Next tokens and their log probabilities from the requests' last rows h [B, H]."""
        _, _, q, s = self.norm.forward(h)
        moe.moe_i8_matmul(q, s, *self.weight8, self.logits)
        return self.sampler.forward(self.logits, u, **settings)


def normed(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()


def reference(m, xs):
    """The layer on one request's tokens xs [n, H] in fp32; the last token's output."""
    x = xs.float()
    q, k, v = (normed(x, m.n1) @ m.qkv.float()).view(len(x), -1, m.D).split([m.heads, m.kv_heads, m.kv_heads], 1)
    g = m.heads // m.kv_heads
    k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    p = torch.softmax((q[-1:] * k).sum(-1) * m.D ** -0.5, 0)
    h = x[-1] + (p[..., None] * v).sum(0).reshape(1, -1) @ m.out.float()
    n = normed(h, m.n2)
    z = (n @ m.w_r.float())[0]
    top, idx = z.topk(m.k)
    y = sum(gate * ((torch.nn.functional.silu(n @ m.gate[e].float()) * (n @ m.up[e].float())) @ m.down[e].float())
            for gate, e in zip(torch.softmax(top, 0), idx))
    return (h + y)[0]


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=512, help="longest prompt")
    ap.add_argument("--steps", type=int, default=4, help="single-token steps after the prompts")
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--experts", type=int, default=128)
    ap.add_argument("--vocab", type=int, default=32000)
    args = ap.parse_args(argv)
    B, H = args.requests, args.hidden
    layer = Layer(H, heads=32, kv_heads=4, D=128, E=args.experts, F=768, k=8, norms=True)
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
    head = Head(B, H, args.vocab)
    full = lambda v: torch.full((B,), v, device="cuda")  # noqa: E731
    token, logprob = head.step(h, torch.rand(B, device="cuda", generator=g), temperature=full(0.8), top_p=full(0.9))
    print("next tokens: " + ", ".join(f"{t} ({p:.2f})" for t, p in zip(token.tolist()[:4], logprob.tolist())))
    errs = []
    for b in range(min(B, 4)):
        ref = reference(layer, prompts[b])
        errs.append(float((h[b].float() - ref).norm() / ref.norm()))
    print(f"against fp32 without a cache: relative error {max(errs):.4f}")
    return max(errs)


if __name__ == "__main__":
    main()
