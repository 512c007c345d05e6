"""The account that mnnq_attn_decode keeps of the attention given: a query adds to the tokens that it sees and to no other."""
import os
import sys

import pytest
import torch

import attn_reference as R
from paper_2506_10443_amd import binding as B
from test_gpu_attn_decode import filled, rows
from test_gpu_kv_cache import F8, I8

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from attention_block import AttentionBlock  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("lengths", [[20, 3], [300, 40], [1500, 700]])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_query_that_is_no_number_spoils_what_it_sees_only(bad, lengths, dtype):
    gen = torch.Generator().manual_seed(sum(lengths))
    c = filled(gen, lengths, 2, 16, 64, I8, F8, dtype)
    q = rows(gen, 5 * 2, 8, 64, dtype)
    q[1, 6, 2] = q[6, 1, 2] = bad                           # the second query of the first sequence, and of the second
    base = torch.rand((2, 2, c.table.shape[1] * 16), device="cuda")
    w = base.clone()
    B.mnnq_attn_decode(q.cuda(), *c.args(), weights=w)
    _, want = R.decode(c.ref, c.table, lengths, q, 5)
    got = (w - base)[..., :max(lengths)].cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.isnan(want[0, 1, :lengths[0] - 3]).all() and torch.isfinite(want[0, 1, lengths[0] - 3:]).all()
    assert R.error(got.nan_to_num(0.0), want.nan_to_num(0.0)) <= 1e-5 + 2.0 ** -24 * float(base.norm()) / float(want.nan_to_num(0.0).norm())


def test_tokens_of_missing_blocks_are_given_nothing():
    gen = torch.Generator().manual_seed(7)
    c = filled(gen, [700], 1, 16, 64)
    table = c.table.clone()
    table[0, 2] = -1
    q = rows(gen, 3, 4, 64, torch.float16)
    q[0, 2] = float("nan")
    w = torch.zeros((1, 1, table.shape[1] * 16), device="cuda")
    B.mnnq_attn_decode(q.cuda(), *c.args(table=table), weights=w)
    assert not w[0, 0, 32:48].any() and not w[0, 0, 700:].any()
    assert torch.isnan(w[0, 0, :32]).all() and torch.isnan(w[0, 0, 48:698]).all() and torch.isfinite(w[0, 0, 698:]).all()


def test_a_prompt_beyond_the_budget_is_judged_by_its_attention(monkeypatch):
    """The example evicts behind a prompt: by the attention of the prompt's last queries, not by position."""
    hidden, heads, kv_heads, dim, counts, budget, recent = 256, 8, 2, 64, [180, 17, 260], 100, 16
    block = AttentionBlock(hidden, heads, kv_heads, dim, 3, 300, budget=budget, recent=recent, block_tokens=32, seed=5)
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((sum(counts), hidden), generator=gen, device="cuda").half() * 4
    q, k, v = (t.cpu() for t in block.project(x))
    cache = R.Cache(block.pool.k_codes.shape[0], kv_heads, 32, dim, block.pool.k_codes.dtype, block.pool.v_codes.dtype)
    table, seen = block.table.cpu(), {}
    inner = B.mnnq_kv_evict

    def call(*args):
        seen["given"] = args[6].clone()
        seen["kept"], lengths = inner(*args)
        return seen["kept"], lengths

    monkeypatch.setattr(B, "mnnq_kv_evict", call)
    out = block.prompt(x, counts)
    assert out.shape == (sum(counts), hidden) and bool(torch.isfinite(out).all())
    assert block.lengths.tolist() == [100, 17, 100]
    given, kept, at, by_place = seen["given"].cpu().double(), seen["kept"].cpu(), 0, True
    for s, n in enumerate(counts):
        for y, rows_of in (("k", k), ("v", v)):
            cache.append(y, table[s], 0, rows_of[at:at + n])
        tokens = min(n, 32)
        _, want = R.decode(cache, table[s:s + 1], [n], q[at + n - tokens:at + n], tokens)
        assert R.error(given[s:s + 1, :, :n], want) <= 1e-5
        at += n
        for h in range(kv_heads):
            places = [int(p) for p in kept[s, h] if p >= 0]
            assert len(places) == min(n, budget) and places[-1] == n - 1
            last = set(range(n - min(recent, len(places)), n))
            assert last <= set(places)
            gone, stay = [t for t in range(n) if t not in places], [t for t in places if t not in last]
            if gone:
                assert float(want[0, h, gone].max()) <= float(want[0, h, stay].min()) + 1e-4
                by_place &= stay == list(range(len(stay)))
    assert not by_place
    assert bool(torch.isfinite(block.step(x[:3])).all())


def test_the_example_refuses_what_it_cannot_do():
    block = AttentionBlock(256, 8, 2, 64, 1, 64, block_tokens=32)
    x = torch.zeros((65, 256), dtype=torch.float16, device="cuda")
    with pytest.raises(RuntimeError, match="room"):
        block.prompt(x, [65])
    block.prompt(x[:10], [10])
    with pytest.raises(RuntimeError, match="empty"):
        block.prompt(x[:10], [10])
