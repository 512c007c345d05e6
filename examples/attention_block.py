#!/usr/bin/env python3
"""The attention half of a transformer block on this library's calls: quantized q|k|v projection, prompt attention, the 8-bit
cache, attention over it token by token with an account of the attention given, eviction under a budget, quantized output
projection.  Random weights; prints what a prompt and a token take.

    python examples/attention_block.py [--model qwen2-7b] [--prompts 517,64,1200] [--tokens 64] [--budget 1024]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2506_10443_amd import binding as B, synth  # noqa: E402


PROMPT_QUERIES = 32     # of a prompt that goes to eviction: how many of the last ones say what was attended to


class Blocks:
    """A pool of cache blocks and the blocks that nobody holds."""

    def __init__(self, blocks, kv_heads, block_tokens, head_dim, k_type, v_type):
        shape = (blocks, kv_heads, block_tokens, head_dim)
        self.k_codes = torch.empty(shape, dtype=k_type, device="cuda")
        self.v_codes = torch.empty(shape, dtype=v_type, device="cuda")
        self.k_range = torch.empty(shape[:2], device="cuda")
        self.v_range = torch.empty(shape[:2], device="cuda")
        self.block_tokens, self.free = block_tokens, list(range(blocks))

    def arrays(self):
        return self.k_codes, self.k_range, self.v_codes, self.v_range

    def take(self, n):
        if n > len(self.free):
            raise RuntimeError("the pool has %d free blocks, %d are needed" % (len(self.free), n))
        taken, self.free = self.free[:n], self.free[n:]
        return taken


class AttentionBlock:
    """q|k|v, attention and output projection of one layer, for a batch of sequences that grow together."""

    def __init__(self, hidden, heads, kv_heads, head_dim, sequences, max_tokens, budget=None, recent=64, block_tokens=64,
                 k_type=torch.int8, v_type=torch.float8_e4m3fn, seed=0):
        if budget is not None and budget + block_tokens > max_tokens:
            raise ValueError("a budget leaves room for a block of new tokens")
        self.hidden, self.heads, self.kv_heads, self.head_dim = hidden, heads, kv_heads, head_dim
        self.budget, self.recent = budget, recent
        rows = (heads + 2 * kv_heads) * head_dim
        gen = torch.Generator(device="cuda").manual_seed(seed)
        weights = lambda n, k: torch.randn((n, k), generator=gen, device="cuda") * 0.02
        self.qkv, self.o = B.mnnq_pack_weights(weights(rows, hidden)), B.mnnq_pack_weights(weights(hidden, heads * head_dim))
        per = -(-max_tokens // block_tokens)
        # (while tokens move to new blocks the old ones are still held)
        spare = 0 if budget is None else sequences * -(-budget // block_tokens)
        self.pool = Blocks(sequences * per + spare, kv_heads, block_tokens, head_dim, k_type, v_type)
        self.held = [self.pool.take(per) for _ in range(sequences)]
        self.table = torch.tensor(self.held, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.longest = 0
        self.given = torch.zeros((sequences, kv_heads, per * block_tokens), device="cuda")

    def project(self, x):
        """x fp16 [tokens, hidden] -> q, k, v: column ranges of the projection's result."""
        rows = (self.heads + 2 * self.kv_heads) * self.head_dim
        if x.shape[0] == 1:
            y = B.mnnq_linear_decode_f16_o16(self.qkv, rows, self.hidden, x[0])
        else:
            y = B.mnnq_linear_prefill_f16_o16(self.qkv, rows, self.hidden, x)
        y = y.view(x.shape[0], -1, self.head_dim)
        return y[:, :self.heads], y[:, self.heads:self.heads + self.kv_heads], y[:, self.heads + self.kv_heads:]

    def output(self, a):
        a = a.view(a.shape[0], -1)
        if a.shape[0] == 1:
            return B.mnnq_linear_decode_f16_o16(self.o, self.hidden, a.shape[1], a[0]).view(1, -1)
        return B.mnnq_linear_prefill_f16_o16(self.o, self.hidden, a.shape[1], a)

    def prompt(self, x, counts):
        """x fp16 [sum of counts, hidden], the sequences' prompts one behind the other; the cache is empty."""
        if self.longest:
            raise RuntimeError("prompt attention looks at the prompt only: the cache must be empty")
        if max(counts) > self.table.shape[1] * self.pool.block_tokens:
            raise RuntimeError("a sequence has no room for its prompt")
        starts = [0]
        for n in counts:
            starts.append(starts[-1] + n)
        start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        q, k, v = self.project(x)
        B.mnnq_kv_append(k, v, *self.pool.arrays(), self.table, self.lengths, start=start)
        self.lengths += start[1:] - start[:-1]
        self.longest += max(counts)
        out = self.output(B.mnnq_attn_prefill(q, k, v, start))
        if self.beyond_budget():
            self.account(q, starts)
            self.evict()
        return out

    def account(self, q, starts):
        """Prompt attention keeps no account: a prompt that is beyond the budget at once is judged by the attention that its last
        queries give, asked of the cache again."""
        for s in range(len(starts) - 1):
            first, last = max(starts[s], starts[s + 1] - PROMPT_QUERIES), starts[s + 1]
            if last > first:
                B.mnnq_attn_decode(q[first:last], *self.pool.arrays(), self.table[s:s + 1], self.lengths[s:s + 1],
                                   max_length=last - starts[s], weights=self.given[s:s + 1])

    def step(self, x):
        """x fp16 [sequences, hidden]: one token of every sequence."""
        if self.longest + 1 > self.table.shape[1] * self.pool.block_tokens:
            raise RuntimeError("a sequence has no room for another token")
        q, k, v = self.project(x)
        B.mnnq_kv_append(k, v, *self.pool.arrays(), self.table, self.lengths)
        self.lengths += 1
        self.longest += 1
        a = B.mnnq_attn_decode(q, *self.pool.arrays(), self.table, self.lengths, max_length=self.longest, weights=self.given)
        out = self.output(a)
        self.evict()
        return out

    def beyond_budget(self):
        """Whether the longest sequence is a block beyond it."""
        return self.budget is not None and self.longest >= self.budget + self.pool.block_tokens

    def evict(self):
        """Back to the budget where it is exceeded."""
        block = self.pool.block_tokens
        if not self.beyond_budget():
            return None
        need = -(-self.budget // block)
        fresh = [self.pool.take(need) for _ in self.held]
        table = torch.tensor(fresh, dtype=torch.int32, device="cuda")
        given = torch.empty_like(self.given)
        kept, self.lengths = B.mnnq_kv_evict(*self.pool.arrays(), self.table, self.lengths, self.given, self.budget, self.recent,
                                             table, given)
        for old in self.held:                # (blocks are used again behind the call on the same stream)
            self.pool.free += old
        per = self.table.shape[1]
        self.held = [f + self.pool.take(per - need) for f in fresh]
        self.table = torch.tensor(self.held, dtype=torch.int32, device="cuda")
        self.given, self.longest = given, self.budget
        return kept


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--model", choices=sorted(synth.MODELS), default="qwen2-7b")
    ap.add_argument("--prompts", default="517,64,1200")
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--budget", type=int, default=1024)
    a = ap.parse_args()
    layers, dim = synth.MODELS[a.model]["layers"], 128
    hidden = layers["q"][1]
    counts = [int(n) for n in a.prompts.split(",")]
    block = AttentionBlock(hidden, layers["q"][0] // dim, layers["k"][0] // dim, dim, len(counts),
                           max(max(counts) + a.tokens, a.budget + 64), budget=a.budget)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((sum(counts), hidden), generator=gen, device="cuda").half()
    tokens = torch.randn((a.tokens, len(counts), hidden), generator=gen, device="cuda").half()
    torch.cuda.synchronize()
    t = time.perf_counter()
    block.prompt(x, counts)
    torch.cuda.synchronize()
    print("prompts of %s tokens: %.3f ms" % (a.prompts, 1e3 * (time.perf_counter() - t)))
    t = time.perf_counter()
    for i in range(a.tokens):
        block.step(tokens[i])
    torch.cuda.synchronize()
    print("%d tokens of %d sequences: %.1f us each, longest cache %d tokens"
          % (a.tokens, len(counts), 1e6 * (time.perf_counter() - t) / a.tokens, block.longest))


if __name__ == "__main__":
    main()
