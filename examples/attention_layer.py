"""One attention layer on MXFP4 products and an MXFP4 cache: ragged prompts, a beam forked off, decoding, pages given back.

    x -> Q(x R) . Q(W_qkv R)^T -> norm and rotation of the heads, keys and values into the cache -> attention
      -> Q(.) . Q(W_o R_v)^T

Values are rotated on their way into the cache, so attention's output is already what the output projection's quantizer takes.

    python examples/attention_layer.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_04214_amd as brq  # noqa: E402

PAGE = brq.KV4_PAGE


class Cache:
    """The pages of one layer, and which sequence has which."""

    def __init__(self, pages, sequences, tokens, Hk, D, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.pool = torch.zeros((pages, brq.kv4_page_bytes(Hk, D)), dtype=torch.uint8, device=device)
        self.table = torch.full((sequences, -(-tokens // PAGE)), -1, **i32)
        self.lens = torch.zeros((sequences,), **i32)
        self.refs = torch.zeros((pages,), **i32)

    def grow(self, seqs, tokens):
        """Room for tokens[i] more tokens of sequences seqs[i] (int32); returns every new token's (position, slot)."""
        old = self.lens[seqs.long()]
        if int(brq.kv4_pages_reserve(self.table, self.refs, seqs, old + tokens)):
            raise RuntimeError("the cache is full")
        rows = torch.repeat_interleave(torch.arange(len(seqs), device=seqs.device), tokens.long())
        start = (tokens.cumsum(0) - tokens).long()
        positions = old.long()[rows] + torch.arange(len(rows), device=seqs.device) - start[rows]
        self.lens[seqs.long()] = old + tokens
        return positions, self.table[seqs.long()[rows], positions // PAGE].long() * PAGE + positions % PAGE

    def fork(self, parents, children):
        if int(brq.kv4_pages_fork(self.pool, self.table, self.lens, self.refs, parents, children)):
            raise RuntimeError("the cache is full")

    def free(self, seqs):
        brq.kv4_pages_free(self.table, self.lens, self.refs, seqs)

    def compact(self):
        return int(brq.kv4_pages_compact(self.pool, self.table, self.refs))


class Attention:
    """Grouped-query attention with normalised heads; weights bfloat16 [(Hq + 2 Hk) D, C] and [C, Hq D], quantized once."""

    def __init__(self, w_qkv, w_o, wq, wk, Hq, Hk, D, tokens, B=32, theta=10000.0):
        self.Hq, self.Hk, self.D, self.B, self.wq, self.wk = Hq, Hk, D, B, wq, wk
        self.qkv, self.o = brq.rotate_quantize_fused(w_qkv, B), brq.rotate_quantize_fused(w_o, B)
        angle = torch.arange(tokens, device=w_qkv.device)[:, None] * theta ** (-torch.arange(D // 2, device=w_qkv.device) * 2.0 / D)
        self.cos, self.sin = angle.cos().contiguous(), angle.sin().contiguous()

    def project(self, x):
        """Queries, keys and values of x [T, C]: views of one product's result, [T, heads, D]."""
        y = brq.mxfp4_gemm(*brq.rotate_quantize_fused(x, self.B), *self.qkv, out_dtype=torch.bfloat16)
        return y.view(len(x), self.Hq + 2 * self.Hk, self.D).split((self.Hq, self.Hk, self.Hk), 1)

    def __call__(self, x, cache, seqs, tokens, max_q, max_kv):
        """The layer's output for tokens[i] new tokens of sequences seqs[i], x [sum(tokens), C]."""
        positions, slots = cache.grow(seqs, tokens)
        q, k, v = self.project(x)
        q = brq.kv4_append(cache.pool, slots, k, v, q, self.wq, self.wk, cos=self.cos, sin=self.sin, positions=positions, B=self.B, Bv=self.B)
        cu = None if max_q == 1 else torch.nn.functional.pad(tokens.cumsum(0), (1, 0)).to(torch.int32)
        o = brq.kv4_attention(q, cache.pool, cache.table[seqs.long()], cache.lens[seqs.long()], cu_q=cu, max_q=max_q, max_kv=max_kv)
        return brq.mxfp4_gemm(*brq.mxfp4_quantize(o.view(len(x), -1)), *self.o, out_dtype=torch.bfloat16)


class HeadNorms(torch.autograd.Function):
    """The layer's head pass for training: gradients of queries, keys and both norms' weights."""

    @staticmethod
    def forward(ctx, q, k, wq, wk, cos, sin, positions, B):
        ctx.save_for_backward(q, k, wq, wk, cos, sin, positions)
        ctx.B = B
        return brq.qk_norm_rope(q, k, wq, wk, cos=cos, sin=sin, positions=positions, B=B)

    @staticmethod
    def backward(ctx, gq, gk):
        q, k, wq, wk, cos, sin, positions = ctx.saved_tensors
        return (*brq.qk_norm_rope_backward(q, k, gq.contiguous(), gk.contiguous(), wq, wk, cos=cos, sin=sin, positions=positions, B=ctx.B),
                None, None, None, None)


def main(C=1024, Hq=8, Hk=2, D=128, steps=20):
    g = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")                                   # noqa: E731
    ids = lambda *n: torch.tensor(n, dtype=torch.int32, device="cuda")                                     # noqa: E731
    layer = Attention((rand((Hq + 2 * Hk) * D, C) / C ** 0.5).bfloat16(), (rand(C, Hq * D) / (Hq * D) ** 0.5).bfloat16(),
                      1 + 0.1 * rand(D), 1 + 0.1 * rand(D), Hq, Hk, D, 1024)
    cache = Cache(40, 4, 1024, Hk, D)
    x = rand(430, C).bfloat16()
    y = layer(x, cache, ids(0, 1, 2), ids(100, 300, 30), 300, 1024)                    # three prompts at once
    cache.fork(ids(1), ids(3))                                                         # two ways on from the second
    y = y[[99, 399, 429, 399]]
    for _ in range(steps):
        y = layer(y + rand(4, C).bfloat16(), cache, ids(0, 1, 2, 3), ids(1, 1, 1, 1), 1, 1024)
    cache.free(ids(0, 1))
    live = cache.compact()
    y = layer(y[2:], cache, ids(2, 3), ids(1, 1), 1, 1024)
    print("lengths %s, %d pages in use, outputs %s" % (cache.lens.tolist(), live, "finite" if y.isfinite().all() else "not finite"))

    # one step of tuning the norms' weights
    q, k, _ = layer.project(x)
    wq, wk = (w.clone().requires_grad_() for w in (layer.wq, layer.wk))
    q2, k2 = HeadNorms.apply(q, k, wq, wk, layer.cos, layer.sin, torch.arange(len(x), device="cuda"), layer.B)
    loss = (q2.float().pow(2).mean() + k2.float().pow(2).mean())
    loss.backward()
    print("loss %.4f, gradients %.4f %.4f" % (float(loss.detach()), float(wq.grad.norm()), float(wk.grad.norm())))
    return cache, y


if __name__ == "__main__":
    main()
