"""One attention layer with 4-bit weights and a paged 4-bit cache: prompts of several sequences, then tokens one at a time.

    python examples/paged_decode.py [--tokens 32]

Per step: hidden states are quantized and multiplied with packed weights (queries, keys and values in one product), queries and keys
are normalized per head and rotated by position in one pass, keys and values are written to the cache, the new tokens attend to
their sequences' pages, and the result goes through the output projection.  The layer has random weights.  At the end the cache is
read back and the last step's attention computed again in float32 from what it stands for.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2501_01144_amd import dfp4, kvcache, synth  # noqa: E402


class Layer:
    def __init__(self, hidden, heads, kv_heads, head_dim, seed=0):
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        pack = lambda rows, cols, s: dfp4.native_pack(dfp4.quantize_mse(synth.gaussian(rows, cols, cols ** -0.5, seed + s).cuda()))  # noqa: E731
        self.w_qkv, self.w_out = pack((heads + 2 * kv_heads) * head_dim, hidden, 1), pack(hidden, heads * head_dim, 2)
        self.q_norm, self.k_norm = torch.ones(head_dim, device="cuda"), torch.ones(head_dim, device="cuda")
        self.inv_freq = (1.0 / 500000.0 ** (torch.arange(0, head_dim, 2, device="cuda", dtype=torch.float64) / head_dim)).float()

    def __call__(self, x, positions, cache, batch):
        qkv = dfp4.gemm_native_packed(dfp4.quantize_native(x), self.w_qkv, dtype=torch.bfloat16).view(x.shape[0], -1, self.head_dim)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
        q, k = dfp4.norm_rope(q, k, positions, self.inv_freq, self.q_norm, self.k_norm)
        dfp4.paged_write(k, v, cache, batch)
        o = dfp4.paged_attention(q, cache, batch)
        return dfp4.gemm_native_packed(dfp4.quantize_native(o.flatten(1)), self.w_out, dtype=torch.bfloat16), q, o


def run(prompts=(300, 33, 1000, 128), tokens=32, hidden=1024, heads=16, kv_heads=4, head_dim=64, page=64):
    """Returns how far the last step's attention is from float32 on the cached values, relative to their size, and the seconds a step."""
    n = len(prompts)
    layer = Layer(hidden, heads, kv_heads, head_dim)
    width = -(-(max(prompts) + tokens) // page)
    cache = kvcache.PagedCache(n * width, page, kv_heads, head_dim, n, torch.device("cuda"))
    table = torch.randperm(n * width, device="cuda", dtype=torch.int32).view(n, width)
    slots = torch.arange(n, device="cuda", dtype=torch.int32)
    whole = lambda t: torch.tensor(t, device="cuda", dtype=torch.int32)  # noqa: E731

    # prompts: all of their tokens at once
    cu = [sum(prompts[:b]) for b in range(n + 1)]
    lengths = whole(prompts)
    x = synth.gaussian(cu[-1], hidden, 1.0, 5).cuda()
    positions = torch.cat([torch.arange(p, device="cuda", dtype=torch.int32) for p in prompts])
    y, _, _ = layer(x, positions, cache, kvcache.PagedBatch(whole(cu), lengths, table, slots, max_new=max(prompts)))
    x = y[[c - 1 for c in cu[1:]]]

    # tokens: one a sequence and step; the batch's lengths are device memory that a step counts up
    batch = kvcache.PagedBatch(torch.arange(n + 1, device="cuda", dtype=torch.int32), lengths, table, slots, max_new=1)
    for step in range(tokens):
        if step == tokens // 2:                       # (the first ones load kernels)
            torch.cuda.synchronize()
            began = time.perf_counter()
        positions = lengths.clone()
        lengths += 1
        x, q, o = layer(x, positions, cache, batch)
    torch.cuda.synchronize()
    seconds = (time.perf_counter() - began) / (tokens - tokens // 2)

    every = kvcache.PagedBatch(torch.cat([lengths.new_zeros(1), lengths.cumsum(0).int()]), lengths, table, slots)
    k, v = dfp4.paged_read(cache, every, dtype=torch.float32)
    worst, at = 0.0, 0
    for b, length in enumerate(lengths.tolist()):
        kb, vb = (t[at:at + length].repeat_interleave(heads // kv_heads, 1) for t in (k, v))
        at += length
        p = torch.softmax((kb * q[b].float()).sum(-1) * head_dim ** -0.5, 0)
        want = (p[..., None] * vb).sum(0)
        worst = max(worst, float((o[b].float() - want).norm() / want.norm()))
    return worst, seconds


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--tokens", type=int, default=32)
    args = parser.parse_args()
    off, seconds = run(tokens=args.tokens)
    print("attention of the last step: %.1e from float32 on the cached values; %.0f us a step" % (off, seconds * 1e6))
