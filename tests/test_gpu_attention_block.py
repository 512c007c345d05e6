"""The attention half of a block, prompt to eviction, against the same steps in 64 bits.

The projections have tests of their own; here the reference takes what they give (the same call on the same row gives the same bits)
and follows the attention in between.  Tolerance: as for the attention calls, one unit of float16, 2^-11 (2-norm)."""
import os
import sys

import torch
import pytest

import attn_reference as R
from paper_2506_10443_amd import binding as B

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from attention_block import AttentionBlock  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k_type,v_type", [(torch.int8, torch.float8_e4m3fn), (torch.float8_e4m3fn, torch.int8)])
def test_a_prompt_and_tokens_under_a_budget(k_type, v_type):
    hidden, heads, kv_heads, dim, counts, budget, recent = 256, 8, 2, 64, [90, 17, 129], 100, 16
    block = AttentionBlock(hidden, heads, kv_heads, dim, 3, 200, budget=budget, recent=recent, block_tokens=32, k_type=k_type,
                           v_type=v_type, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    cache = R.Cache(block.pool.k_codes.shape[0], kv_heads, 32, dim, k_type, v_type)
    lengths, given = [0, 0, 0], torch.zeros(3, kv_heads, 400, dtype=torch.float64)
    seen = {}

    def watch(name):
        inner = getattr(B, name)

        def call(*args, **kwargs):
            seen[name] = inner(*args, **kwargs)
            return seen[name]
        return inner, call

    patched = {name: watch(name) for name in ("mnnq_attn_prefill", "mnnq_attn_decode", "mnnq_kv_evict")}
    for name, (_, call) in patched.items():
        setattr(B, name, call)
    try:
        evictions = 0
        for turn in range(45):
            print("turn", turn, lengths, flush=True)
            n = counts if turn == 0 else [1, 1, 1]
            x = torch.randn((sum(n), hidden), generator=gen, device="cuda").half()
            q, k, v = (t.cpu() for t in block.project(x))
            table, before = block.table.cpu(), list(lengths)
            seen.clear()
            out = block.prompt(x, n) if turn == 0 else block.step(x)
            assert out.shape == (sum(n), hidden) and bool(torch.isfinite(out).all())
            at = 0
            for s, m in enumerate(n):
                cache.append("k", table[s], lengths[s], k[at:at + m])
                cache.append("v", table[s], lengths[s], v[at:at + m])
                lengths[s] += m
                at += m
            if turn == 0:
                want = R.prompt(q, k, v, n, n)
                assert R.error(seen["mnnq_attn_prefill"].cpu(), want) <= 2.0 ** -11
            else:
                want, w = R.decode(cache, table, lengths, q, 1)
                assert R.error(seen["mnnq_attn_decode"].cpu(), want) <= 2.0 ** -11
                given[..., :w.shape[2]] += w
            assert max(before) < budget + 32
            if "mnnq_kv_evict" in seen:
                evictions += 1
                kept = seen["mnnq_kv_evict"][0].cpu()
                # which tokens went: by sums that the call's own agree with to fp32; the places are the call's
                weights = torch.zeros(3, kv_heads, 400, dtype=torch.float64)
                for s in range(3):
                    m = min(lengths[s], budget)
                    for h in range(kv_heads):
                        places = [int(p) for p in kept[s, h] if p >= 0]
                        assert len(places) == m and places == sorted(set(places)) and places[-1] == lengths[s] - 1
                        last = set(range(lengths[s] - min(recent, m), lengths[s]))
                        assert last <= set(places)
                        gone = [t for t in range(lengths[s]) if t not in places]
                        stay = [t for t in places if t not in last]
                        if gone and stay:
                            assert float(given[s, h, gone].max()) <= float(given[s, h, stay].min()) + 1e-4
                        weights[s, h, :m] = given[s, h, places]
                        # the reference follows the same choice
                        rank = torch.zeros(400, dtype=torch.float64)
                        rank[stay] = 1.0
                        one = R.Cache(cache.codes["k"].shape[0], kv_heads, 32, dim, k_type, v_type)
                        one.codes, one.range = ({y: z[y].clone() for y in "kv"} for z in (cache.codes, cache.range))
                        fresh = block.table.cpu()[s:s + 1]
                        ranks = torch.zeros(1, kv_heads, 400, dtype=torch.float64)
                        ranks[0, h] = rank
                        R.evict(one, table[s:s + 1], [lengths[s]], ranks, budget, recent, fresh)
                        for b in range(-(-m // 32)):
                            to = int(fresh[0, b])
                            for y in "kv":
                                block_codes = getattr(block.pool, y + "_codes").view(torch.uint8)[to, h].cpu()
                                got = block_codes.view(cache.type[y]).double()
                                used = min(32, m - 32 * b)
                                assert torch.equal(got[:used], one.codes[y][to, h, :used])
                given = weights
                lengths = [min(m, budget) for m in lengths]
                # (from here the reference's cache is what the call wrote, just compared)
                for y in "kv":
                    cache.codes[y] = getattr(block.pool, y + "_codes").view(torch.uint8).cpu().view(cache.type[y]).double()
                    cache.range[y] = getattr(block.pool, y + "_range").cpu().double()
            assert block.lengths.tolist() == lengths and block.longest >= max(lengths)
        assert evictions >= 2
    finally:
        for name, (inner, _) in patched.items():
            setattr(B, name, inner)
