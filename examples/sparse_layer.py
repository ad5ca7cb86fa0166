"""A sparse feed-forward layer with 4-bit experts: norm with the residual, router, plan, experts' products, next norm.

    python examples/sparse_layer.py [--tokens 64]

The router's logits are a product in the library's 4-bit form like any other; experts' weights are quantized with the MSE-based
choice of dialects and laid out once.  The layer has random weights.  At the end its result is computed again in float32 from the
weights' and rows' 4-bit values.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2501_01144_amd import dfp4, synth  # noqa: E402


class SparseLayer:
    def __init__(self, hidden, inner, experts, k, seed=0):
        self.experts, self.k = experts, k
        quantized = lambda rows, cols, s: dfp4.quantize_mse(synth.gaussian(rows, cols, cols ** -0.5, seed + s).cuda())  # noqa: E731
        self.gate, self.up, self.down = quantized(experts * inner, hidden, 1), quantized(experts * inner, hidden, 2), quantized(experts * hidden, inner, 3)
        self.router = dfp4.native_pack(quantized(-(-experts // 32) * 32, hidden, 4))
        self.w_up, self.w_down = dfp4.expert_weights(self.gate, experts, up=self.up), dfp4.expert_weights(self.down, experts)
        self.norm = torch.ones(hidden, device="cuda")

    def __call__(self, y, residual):
        """y: what the block before gives; returns this block's result, the residual with y added, and what was computed on the way."""
        residual, x = dfp4.add_norm(y, residual, self.norm)
        logits = dfp4.gemm_native_packed(dfp4.quantize_native(x), self.router)[:, :self.experts]
        ids, weights = dfp4.route(logits, self.k)
        plan = dfp4.expert_plan(ids, self.experts)
        h = dfp4.experts_up(x, plan, self.w_up)
        return dfp4.experts_down(h, plan, self.w_down, weights), residual, (x, ids, weights, plan, h)


def run(tokens=64, hidden=512, inner=256, experts=16, k=4, layers=2, steps=20):
    """Returns how far the last layer's result is from float32 on the 4-bit values, relative to its size, and the seconds a step."""
    stack = [SparseLayer(hidden, inner, experts, k, seed=10 * i) for i in range(layers)]
    start = synth.gaussian(tokens, hidden, 1.0, 5).cuda()
    for step in range(steps):
        if step == steps // 2:                        # (the first ones load kernels)
            torch.cuda.synchronize()
            began = time.perf_counter()
        y, residual = torch.zeros_like(start), start
        for layer in stack:
            y, residual, seen = layer(y, residual)
    torch.cuda.synchronize()
    seconds = (time.perf_counter() - began) / (steps - steps // 2)

    x, ids, weights, plan, h = seen
    values = lambda q: dfp4.dequantize(q, dtype=torch.float32).view(experts, -1, q.K)  # noqa: E731
    gate, up, down = values(layer.gate), values(layer.up), values(layer.down)
    four_bits = lambda t: dfp4.dequantize(dfp4.quantize(t), dtype=torch.float32)  # noqa: E731
    xq, hq, want = four_bits(x), four_bits(h), torch.zeros(tokens, hidden, device="cuda")
    offsets, worst = plan.offsets.tolist(), 0.0
    for e in range(experts):
        pairs = plan.order[offsets[e]:offsets[e + 1]].long()
        if len(pairs):
            a = xq[pairs // k]
            mine, own = h[offsets[e]:offsets[e + 1]].float(), torch.nn.functional.silu(a @ gate[e].T) * (a @ up[e].T)
            worst = max(worst, float((mine - own).norm() / own.norm()))
            want.index_add_(0, pairs // k, weights.flatten()[pairs, None] * (hq[offsets[e]:offsets[e + 1]] @ down[e].T))
    return max(worst, float((y.float() - want).norm() / want.norm())), seconds


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--tokens", type=int, default=64)
    args = parser.parse_args()
    off, seconds = run(tokens=args.tokens)
    print("%.1e from float32 on the 4-bit values; %.0f us for two layers" % (off, seconds * 1e6))
