"""One decoder layer of a language model with block-pruned weights, as a serving program runs it: prompts of uneven length into a
paged cache, then answers token by token from one captured graph.

    y = norm(h)                                    ubp_rmsnorm
    qkv = P y                                      ubp_linear
    q = rotate(head norm(q)); k, v -> pages        ubp_rotate_append
    o = attention(q, pages)                        ubp_attention
    h = O o + h                                    ubp_linear onto the residual stream
    h = h + feed-forward(h)                        (pruned_feed_forward.py)

Compared with the same layer in float64 on all tokens at once.
    python examples/pruned_decoder_layer.py [--width 512] [--heads 8] [--kv-heads 2] [--head-size 64] [--window 0] [--sparsity 70]
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2407_19644_b200 as ubp  # noqa: E402
import ubp_synth  # noqa: E402
from examples.pruned_feed_forward import PrunedFeedForward  # noqa: E402

BF16 = torch.bfloat16
EPS = 1e-5


class PagedCache:
    """Keys and values of one layer in pages of a pool, and each sequence's list of pages."""

    def __init__(self, sequences, longest, heads, size, page=16, pages=None):
        self.page = page
        per = -(-longest // page)
        pages = pages or sequences * per
        self.k, self.v = (torch.empty(pages, heads, page, size, dtype=BF16, device="cuda") for _ in range(2))
        order = torch.randperm(pages, device="cuda")[:sequences * per].to(torch.int32)      # (a server hands them out as they are needed)
        self.table = order.view(sequences, per).contiguous()
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device="cuda")


class PrunedDecoderLayer:
    def __init__(self, weights, masks, block, heads, kv_heads, size, positions, window=0, sinks=0):
        self.heads, self.size, self.window, self.sinks = heads, size, window, sinks
        self.qkv = ubp.LinearPlan(ubp.ubp_pack(weights["qkv"], masks["qkv"], block), BF16)
        self.out = ubp.LinearPlan(ubp.ubp_pack(weights["out"], masks["out"], block), BF16)
        width = weights["out"].shape[0]
        one = torch.ones(width, device="cuda", dtype=BF16)
        self.norm, self.q_norm, self.k_norm = one, torch.full((size,), 1.1, device="cuda", dtype=BF16), torch.full((size,), 0.9, device="cuda", dtype=BF16)
        self.rotation = ubp.rotation_table(positions, size)
        self.feed_forward = PrunedFeedForward(weights["gate_up"], weights["down"], masks["gate_up"], masks["down"], block, one, BF16, EPS)

    def __call__(self, h, cache, starts=None, max_new=None):
        """h: residual stream of the new tokens, bf16 [T][width], updated in place; cache.lengths already counts them."""
        where = (cache.k, cache.v, cache.table, cache.lengths)
        y = ubp.ubp_rmsnorm(h, self.norm, EPS)[0]
        q = ubp.ubp_rotate_append(ubp.ubp_linear(self.qkv, y), self.heads, *where, starts=starts, rotation=self.rotation, q_gamma=self.q_norm,
                                  k_gamma=self.k_norm, eps=EPS)
        o = ubp.ubp_attention(q, *where, starts=starts, window=self.window, sinks=self.sinks, max_new=max_new)
        ubp.ubp_linear(self.out, o.flatten(1), residual=h, out=h)
        return self.feed_forward(torch.zeros_like(h), h)


def reference(h, w, heads, kv_heads, size, window=0, sinks=0):
    """The layer in float64 on all tokens of one sequence."""
    def norm(x, g):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * torch.tensor(g, dtype=BF16).double()

    h = h.double()
    n, g = h.shape[0], heads // kv_heads
    x = (norm(h, 1.0) @ w["qkv"].t()).view(n, heads + 2 * kv_heads, size)
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    p = torch.arange(n, device="cuda", dtype=torch.float64)
    angle = p[:, None] * 10000.0 ** (-torch.arange(0, size, 2, device="cuda", dtype=torch.float64) / size)
    c, s = angle.cos()[:, None], angle.sin()[:, None]

    def turn(u):
        a, b = u[..., :size // 2], u[..., size // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    q, k = turn(norm(q, 1.1)), turn(norm(k, 0.9)).repeat_interleave(g, 1)
    z = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(size)
    seen = p[None] <= p[:, None]
    if window:
        seen &= (p[None] > p[:, None] - window) | (p[None] < sinks)
    o = torch.einsum("hij,jhd->ihd", torch.softmax(z.masked_fill(~seen, -math.inf), -1), v.repeat_interleave(g, 1))
    h = h + o.reshape(n, -1) @ w["out"].t()
    a, b = (norm(h, 1.0) @ w["gate_up"].t()).chunk(2, dim=1)
    return h + (a * torch.sigmoid(a) * b) @ w["down"].t()


def make_weights(width, hidden, heads, kv_heads, size, block, sparsity, seed=1):
    shapes = {"qkv": ((heads + 2 * kv_heads) * size, width), "out": (width, heads * size), "gate_up": (2 * hidden, width), "down": (width, hidden)}
    weights, masks = {}, {}
    for i, (name, (M, C)) in enumerate(shapes.items()):
        L = ubp_synth.make_layer("layer", M, C, block, sparsity, seed + i, Nc=1, make_x=False)
        weights[name] = np.random.default_rng(seed + i).standard_normal((M, C)).astype(np.float32) * L.mask / np.sqrt(C * (100 - sparsity) / 100)
        masks[name] = L.mask
    return weights, masks


def run(prompts, tokens, width=512, hidden=1024, heads=8, kv_heads=2, size=64, window=0, sinks=0, block=4, sparsity=70, page=16, timing=False):
    """Prompts of these lengths, then `tokens` answers each; the largest relative error of a sequence against float64."""
    weights, masks = make_weights(width, hidden, heads, kv_heads, size, block, sparsity)
    B, longest = len(prompts), max(prompts) + tokens
    layer = PrunedDecoderLayer(weights, masks, block, heads, kv_heads, size, longest, window, sinks)
    cache = PagedCache(B, longest, kv_heads, size, page)
    g = torch.Generator(device="cuda").manual_seed(0)
    inputs = [torch.randn(n + tokens, width, device="cuda", generator=g).to(BF16) for n in prompts]
    got = [torch.empty_like(x) for x in inputs]
    # the prompts, one call for all of them
    starts = torch.tensor([0] + prompts, device="cuda").cumsum(0).to(torch.int32)
    cache.lengths += torch.tensor(prompts, dtype=torch.int32, device="cuda")
    h = layer(torch.cat([x[:n] for x, n in zip(inputs, prompts)]), cache, starts)
    for b, n in enumerate(prompts):
        got[b][:n] = h[starts[b]:starts[b + 1]]
    # the answers, a token a sequence and step, from one graph (a warm-up step first: it appends what step 0 appends again)
    h = torch.empty(B, width, dtype=BF16, device="cuda")
    step = torch.cuda.CUDAGraph()
    cache.lengths += 1
    h.copy_(torch.stack([x[n] for x, n in zip(inputs, prompts)]))
    layer(h, cache, max_new=1)
    with torch.cuda.graph(step):
        layer(h, cache, max_new=1)
    for i in range(tokens):
        h.copy_(torch.stack([x[n + i] for x, n in zip(inputs, prompts)]))
        step.replay()
        for b, n in enumerate(prompts):
            got[b][n + i] = h[b]
        if i + 1 < tokens:
            cache.lengths += 1
    ubp.attention_check()
    if timing:
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        ev[0].record()
        for _ in range(50):
            step.replay()
        ev[1].record()
        torch.cuda.synchronize()
        print(f"{B} sequences of {[n + tokens for n in prompts]} tokens: {ev[0].elapsed_time(ev[1]) * 20:.1f} us a step")
    w64 = {k: torch.from_numpy(v).cuda().double() for k, v in weights.items()}
    worst = 0.0
    for x, y in zip(inputs, got):
        want = reference(x, w64, heads, kv_heads, size, window, sinks)
        worst = max(worst, float((y.double() - want).norm() / want.norm()))
    return worst


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("width", 512), ("hidden", 1024), ("heads", 8), ("kv-heads", 2), ("head-size", 64), ("window", 0), ("sinks", 0), ("sparsity", 70), ("block", 4)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--prompts", type=int, nargs="+", default=[300, 17, 129])
    ap.add_argument("--tokens", type=int, default=8)
    a = ap.parse_args()
    err = run(a.prompts, a.tokens, a.width, a.hidden, a.heads, a.kv_heads, a.head_size, a.window, a.sinks, a.block, a.sparsity, timing=True)
    print(f"relative error against float64 on unrounded weights: {err:.4f}")
    assert err < 0.02, err
    print("pruned decoder layer ok")


if __name__ == "__main__":
    main()
