"""A decode step of one transformer block as a program runs it: projections (torch), keys and values into the paged 8-bit cache with the
rotary positions applied on the way, attention over it, and the compressed MoE layer behind it.  Several sequences with prompts of
different length are written in one call, then decoded together; the decode step is captured into a graph, with the lengths on the
device.

    python examples/decode_block.py [--tokens N] [--batch B] [--format int8|e4m3]

Weights are random, so the tokens mean nothing; what is printed is the time of a step and where the cache stands."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_05950_amd as F  # noqa: E402


class Block:
    """Attention with grouped heads and an MoE layer of compressed experts, for up to `batch` sequences of up to `max_len` tokens."""

    def __init__(self, batch, max_len, fmt, d=2048, q_heads=16, kv_heads=4, dim=128, f=1408, experts=8, top_k=2, block=64, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weights(*shape, scale=0.02):
            return (torch.randn(shape, generator=g, device="cuda") * scale).half()
        self.d, self.q_heads, self.kv_heads, self.dim, self.batch, self.max_len = d, q_heads, kv_heads, dim, batch, max_len
        self.w_qkv, self.w_out = weights(d, (q_heads + 2 * kv_heads) * dim), weights(q_heads * dim, d)
        blocks = -(-max_len // block)
        self.cache = F.KVCache(batch * blocks, kv_heads, dim, block, fmt, torch.float16)
        # every sequence gets its pages at the start; a server would hand them out as sequences grow
        self.table = torch.randperm(batch * blocks, generator=g, device="cuda").to(torch.int32).view(batch, blocks)
        self.rope = F.Rope(F.floe_rope_table(max_len, dim))
        packed = []
        for _ in range(experts):
            codes, scale, zero = F.floe_quantize_expert(weights(f, d), 2, 64)
            packed.append(F.Expert(d, f, 2, 64, codes, scale, zero, weights(f, 2, d)))
        tau = torch.full((experts,), 1.0, device="cuda")  # about 70 % of the channels stay out for inputs of unit variance
        self.moe = F.Layer(packed, 0, top_k, True, weights(experts, d), tau, False)

    def __call__(self, x, cu_rows, before, after, max_rows, max_len):
        """x [rows][d]: rows of the sequences one behind the other, behind before[s] tokens each."""
        rows = x.shape[0]
        qkv = (_norm(x) @ self.w_qkv).view(rows, -1, self.dim)
        q, k, v = qkv.split([self.q_heads, self.kv_heads, self.kv_heads], dim=1)
        q = F.floe_kv_append(self.cache, k, v, cu_rows, before, self.table, max_rows, q=q, rope=self.rope)
        o = F.floe_kv_attention(self.cache, q, cu_rows, after, self.table, max_rows, max_len)
        x = x + o.view(rows, -1) @ self.w_out
        return x + torch.cat([F.floe_moe_layer_decode(self.moe, part) for part in _norm(x).split(4096)])  # (a layer call takes 4096 tokens)


def _norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).half()


def main(tokens=32, batch=4, fmt="int8", verbose=True):
    prompts = [37 + 211 * s for s in range(batch)]
    max_len = max(prompts) + tokens + 3
    block = Block(batch, max_len, F.KV_INT8 if fmt == "int8" else F.KV_E4M3)
    g = torch.Generator(device="cuda").manual_seed(1)

    def i32(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")
    # the prompts, in one call
    ends = [0]
    for n in prompts:
        ends.append(ends[-1] + n)
    x = torch.randn((ends[-1], block.d), generator=g, device="cuda").half()
    y = block(x, i32(ends), i32([0] * batch), i32(prompts), max(prompts), max(prompts))
    x = y[i32(ends[1:]).long() - 1].clone()  # each sequence goes on from its last row
    # one token of every sequence per step: lengths live on the device, so the captured step serves all of them
    cu, before, after = i32(list(range(batch + 1))), i32(prompts), i32([n + 1 for n in prompts])

    def step():
        y = block(x, cu, before, after, 1, max_len)
        x.copy_(_norm(y))
        before.add_(1)
        after.add_(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(tokens - 2):
        graph.replay()
    stop.record()
    torch.cuda.synchronize()
    if verbose:
        us = 1e3 * start.elapsed_time(stop) / max(1, tokens - 2)
        print(f"{batch} sequences, {before.tolist()} tokens in the {fmt} cache, {us:.1f} us per block and step")
    return x, before


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--tokens", type=int, default=32)
    p.add_argument("--batch", type=int, default=4)
    p.add_argument("--format", default="int8", choices=("int8", "e4m3"))
    a = p.parse_args()
    if a.tokens < 3 or a.batch < 1:
        p.error("at least three tokens and one sequence")
    main(a.tokens, a.batch, a.format)
