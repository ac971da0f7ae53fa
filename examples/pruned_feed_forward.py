"""One feed-forward block of a language model with block-pruned weights, as a serving program runs it.

    h = x + r                       the residual stream, updated in place
    q, s = norm(h)                  8-bit rows with a scale each           ubp_rmsnorm
    a = silu(G q) * (U q)           gate and up in one product             ubp_linear, gated plan
    p, t = a in 8 bits                                                     ubp_quant_rows
    h = D p + h                     down product onto the residual stream  ubp_linear

run for a prompt and then token by token, in 8 bits and in bf16, and compared with the same block in float64.
    python examples/pruned_feed_forward.py [--width 1024] [--hidden 4096] [--sparsity 80] [--block 4]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2407_19644_b200 as ubp  # noqa: E402
import ubp_synth  # noqa: E402

F8 = torch.float8_e4m3fn


class PrunedFeedForward:
    """Plans and calls of one block. dtype: torch.float8_e4m3fn (8-bit rows and weights) or torch.bfloat16."""

    def __init__(self, gate_up, down, gate_up_mask, down_mask, block, gamma, dtype, eps=1e-5):
        self.dtype, self.gamma, self.eps = dtype, gamma, eps
        self.gate_up = ubp.LinearPlan(ubp.ubp_pack(gate_up, gate_up_mask, block), dtype, gated=True)
        self.down = ubp.LinearPlan(ubp.ubp_pack(down, down_mask, block), dtype)

    def __call__(self, x, h):
        """h (the residual stream, bf16 [T][width]) <- h + x + the block's output; returns h."""
        if self.dtype == F8:
            q, s, _ = ubp.ubp_rmsnorm(x, self.gamma, self.eps, residual=h, residual_out=h, out_dtype=F8)
            p, t = ubp.ubp_quant_rows(ubp.ubp_linear(self.gate_up, q, activation="silu", x_scales=s))
            return ubp.ubp_linear(self.down, p, residual=h, x_scales=t, out=h)
        y, _, _ = ubp.ubp_rmsnorm(x, self.gamma, self.eps, residual=h, residual_out=h)
        return ubp.ubp_linear(self.down, ubp.ubp_linear(self.gate_up, y, activation="silu"), residual=h, out=h)


def reference(x, h, gate_up, down, gamma, eps=1e-5):
    """The block in float64 on unquantised weights."""
    h = h.double() + x.double()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + eps) * gamma.double()
    g, u = (y @ gate_up.double().t()).chunk(2, dim=1)
    return h + (g * torch.sigmoid(g) * u) @ down.double().t()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--sparsity", type=int, default=80)
    ap.add_argument("--block", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=300)
    ap.add_argument("--tokens", type=int, default=8)
    a = ap.parse_args()

    def layer(M, C, seed):
        L = ubp_synth.make_layer("ff", M, C, a.block, a.sparsity, seed, Nc=1, make_x=False)
        scale = 1.0 / np.sqrt(C * (100 - a.sparsity) / 100)
        W = np.random.default_rng(seed).standard_normal((M, C)).astype(np.float32) * scale * L.mask
        return W, L.mask

    (gu, gum), (dn, dnm) = layer(2 * a.hidden, a.width, 1), layer(a.width, a.hidden, 2)
    g = torch.Generator(device="cuda").manual_seed(0)
    gamma = (1 + 0.1 * torch.randn(a.width, device="cuda", generator=g)).to(torch.bfloat16)
    gu64, dn64 = torch.from_numpy(gu).cuda(), torch.from_numpy(dn).cuda()
    for dtype, limit in ((torch.bfloat16, 0.02), (F8, 0.12)):
        block = PrunedFeedForward(gu, dn, gum, dnm, a.block, gamma, dtype)
        worst = 0.0
        for T in [a.prompt] + [1] * a.tokens:                       # a prompt, then one token at a time
            x, h = (torch.randn(T, a.width, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
            want = reference(x, h, gu64, dn64, gamma)
            got = block(x, h)
            worst = max(worst, float((got.double() - want).norm() / want.norm()))
        block.gate_up.check()
        block.down.check()
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        for T in (1, a.prompt):
            x, h = (torch.randn(T, a.width, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
            for _ in range(10):
                block(x, h)
            ev[0].record()
            for _ in range(50):
                block(x, h)
            ev[1].record()
            torch.cuda.synchronize()
            print(f"{str(dtype):24s} {T:5d} tokens  {ev[0].elapsed_time(ev[1]) * 20:8.1f} us a block  "
                  f"kernels {block.gate_up.choice(T)} {block.down.choice(T)}")
        print(f"{str(dtype):24s} relative error against float64 on unquantised weights: {worst:.4f}")
        assert worst < limit, worst
    print("pruned feed-forward ok")


if __name__ == "__main__":
    main()
