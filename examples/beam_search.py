"""Beam search over the paged 8-bit cache as a program runs it: the block of decode_block.py with an output layer behind it, a pool that hands
out the cache's pages, and per step the selection, the tables that follow their parents, and the pages that a beam needs for itself.
Prompts are written once; their beams share the pages.  The step is captured into a graph: nothing of it looks at a result on the host.

    python examples/beam_search.py [--tokens N] [--groups G] [--beams W] [--format int8|e4m3]

Weights are random, so the tokens mean nothing; what is printed is the time of a step, the pages in use and the scores."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path[:0] = [os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(os.path.abspath(__file__))]
import paper_2505_05950_amd as F  # noqa: E402
from decode_block import Block, _norm  # noqa: E402


class Search:
    """Beams of several prompts: their tables and lengths, scores, and which tokens came from where."""

    def __init__(self, block, vocab, groups, beams, steps, eos=2, seed=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.block, self.groups, self.beams, self.eos = block, groups, beams, eos
        self.embed = (torch.randn((vocab, block.d), generator=g, device="cuda")).half()
        self.pool = F.KVPool(block.cache.n_pages, block.cache.block)
        n = groups * beams
        self.cu = torch.arange(n + 1, dtype=torch.int32, device="cuda")
        self.steps, self.at = steps, torch.zeros((1,), dtype=torch.int64, device="cuda")
        self.tokens, self.parents = (torch.full((steps, n), -1, dtype=torch.int32, device="cuda") for _ in range(2))
        self.missing = torch.zeros((1,), dtype=torch.int32, device="cuda")

    def logits(self, y):
        return _norm(y) @ self.embed.t() * (4.0 / self.block.d ** 0.5)

    def start(self, x, ends, prompts):
        """Writes the prompts (rows x, one behind the other up to ends[s]) and opens the beams from their last rows."""
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        block, width = self.block, -(-self.block.max_len // self.block.cache.block)
        table, before, cu = torch.full((self.groups, width), -1, dtype=torch.int32, device="cuda"), i32([0] * self.groups), i32(ends)
        _, missing = F.floe_kv_reserve(self.pool, table, before, cu)
        self.missing += missing
        block.table = table
        y = block(x, cu, before, i32(prompts), max(prompts), max(prompts))
        first = torch.zeros((self.groups, 1), device="cuda")
        self.score, parent, token, self.done = F.floe_beam_select(self.logits(y[cu[1:].long() - 1]), first, take=self.beams, eos=self.eos)
        self.table, self.length = F.floe_kv_reorder(self.pool, table, i32(prompts), parent.view(-1))
        block.table = self.table
        self._keep(parent, token)

    def _keep(self, parent, token):
        self.token = token.view(-1).clone()
        self.tokens.index_copy_(0, self.at, token.view(1, -1))
        self.parents.index_copy_(0, self.at, parent.view(1, -1))
        self.at += 1

    def step(self):
        """A token of every beam: everything in place, so that it can be captured."""
        block = self.block
        pairs, missing = F.floe_kv_reserve(self.pool, self.table, self.length, self.cu)
        F.floe_kv_copy_pages(block.cache, pairs)
        y = block(self.embed[self.token.clamp(min=0).long()], self.cu, self.length, self.length + 1, 1, block.max_len)
        self.length.add_(1)
        score, parent, token, done = F.floe_beam_select(self.logits(y), self.score, done=self.done, eos=self.eos)
        table, length = F.floe_kv_reorder(self.pool, self.table, self.length, parent.view(-1))
        for old, new in ((self.table, table), (self.length, length), (self.score, score), (self.done, done), (self.token, token.view(-1))):
            old.copy_(new)
        self.missing += missing
        self.tokens.index_copy_(0, self.at, token.view(1, -1))
        self.parents.index_copy_(0, self.at, parent.view(1, -1))
        self.at += 1

    def sequences(self):
        """Tokens of every beam, from its first to its last, by walking back over the parents (on the host)."""
        tokens, parents, out = self.tokens.tolist(), self.parents.tolist(), []
        for beam in range(self.groups * self.beams):
            row, at = [], beam
            for t in reversed(range(int(self.at))):
                row.append(tokens[t][at])
                at = parents[t][at]
                if at < 0:
                    break
            out.append(row[::-1])
        return out


def main(tokens=24, groups=2, beams=4, fmt="int8", vocab=8000, captured=True, verbose=True):
    prompts = [45 + 90 * s for s in range(groups)]
    max_len = max(prompts) + tokens + 3
    n = groups * beams
    block = Block(n, max_len, F.KV_INT8 if fmt == "int8" else F.KV_E4M3)
    search = Search(block, vocab, groups, beams, tokens)
    ends = [0]
    for p in prompts:
        ends.append(ends[-1] + p)
    x = torch.randn((ends[-1], block.d), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").half()
    search.start(x, ends, prompts)
    if not captured:
        for _ in range(tokens - 1):
            search.step()
        torch.cuda.synchronize()
        return search
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        search.step()
        search.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        search.step()
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(tokens - 3):
        graph.replay()
    stop.record()
    torch.cuda.synchronize()
    if verbose:
        us = 1e3 * start.elapsed_time(stop) / max(1, tokens - 3)
        used = int((search.pool.refs > 0).sum())
        print(f"{groups} x {beams} beams, {us:.1f} us per block and step, {used} pages in use ({n * -(-max_len // block.cache.block)} without sharing)")
        print("scores", [[round(s, 2) for s in row] for row in search.score.tolist()])
    return search


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--tokens", type=int, default=24)
    p.add_argument("--groups", type=int, default=2)
    p.add_argument("--beams", type=int, default=4)
    p.add_argument("--format", default="int8", choices=("int8", "e4m3"))
    a = p.parse_args()
    if a.tokens < 4 or a.groups < 1 or not 1 <= a.beams <= 64:
        p.error("at least four tokens, one group, and one to 64 beams")
    main(a.tokens, a.groups, a.beams, a.format)
