"""mnnq_attn_decode where ranges lie far apart: what tells of a row's result is what the row sees, however great its neighbours.

Tolerance: that of test_gpu_attn_decode.py, one unit of the result's type (2-norm), row by row."""
import pytest
import torch

import attn_reference as R
from paper_2506_10443_amd import binding as B
from test_gpu_attn_decode import TOL, filled, rows
from test_gpu_kv_cache import F8, I8, Pair

pytestmark = pytest.mark.gpu


def close(out, want, dtype):
    """Every row of every head by itself."""
    off, norm = (out.cpu().double() - want).norm(dim=-1), want.norm(dim=-1)
    assert bool(torch.isfinite(out).all()) and bool((off <= TOL[dtype] * norm).all()), float((off / norm).max())


@pytest.mark.parametrize("n", [1, 16, 33, 200])
@pytest.mark.parametrize("what", [1e30, -1e30, float("inf")])
@pytest.mark.parametrize("dtype,k_type,v_type", [(torch.float16, I8, F8), (torch.bfloat16, F8, I8)])
def test_entries_behind_the_last_token_may_name_any_block(n, what, dtype, k_type, v_type):
    """A block of nobody's with ranges that are none of this sequence's: in the table's rest, and where max_length cuts."""
    gen = torch.Generator().manual_seed(n)
    c = filled(gen, [n], 2, 16, 64, k_type, v_type, dtype, extra=16)
    held = -(-n // 16)
    stranger = int(c.table[0, -1])
    for x in "kv":
        c.gpu[x + "_range"][stranger] = what
    q = rows(gen, 2, 8, 64, dtype)
    outs = []
    for entry in (-1, stranger):
        table = c.table.clone()
        table[0, held:] = entry
        w = torch.zeros((1, 2, table.shape[1] * 16), device="cuda")
        outs.append((B.mnnq_attn_decode(q.cuda(), *c.args(table=table), weights=w), w))
    want, want_w = R.decode(c.ref, c.table, [n], q, 2)
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert R.error(outs[1][0].cpu(), want) <= TOL[dtype]
    assert R.error(outs[1][1][..., :n].cpu(), want_w) <= 1e-5
    # the same blocks behind the bound of the call
    table = c.table.clone()
    table[0, held:] = stranger
    out = B.mnnq_attn_decode(q.cuda(), *c.args(lengths=[n + 100], table=table), max_length=n)
    assert torch.equal(out, outs[0][0])


@pytest.mark.parametrize("n", [1, 300, 3000])
@pytest.mark.parametrize("v_type", [I8, F8])
def test_values_near_the_greatest_number(n, v_type):
    """The result is a mean of values that bfloat16 has; sums on the way must not pass it."""
    gen = torch.Generator().manual_seed(n)
    c = Pair(1, -(-n // 64), 1, 64, 64, I8, v_type)
    v = (2.9e38 + 4e37 * torch.rand((n, 1, 64), generator=gen)).to(torch.bfloat16)
    c.append(rows(gen, n, 1, 64, torch.bfloat16), v, [n])
    q = rows(gen, 1, 4, 64, torch.bfloat16)
    want, _ = R.decode(c.ref, c.table, [n], q, 1)
    close(B.mnnq_attn_decode(q.cuda(), *c.args()), want, torch.bfloat16)


def one_great_block(order, apart, dtype, scores, blocks=12, dim=64, block=16, heads=4, seed=1):
    """A cache of one sequence whose blocks `order` have values 2^apart times the others'; token j's score is scores[its kind]."""
    gen = torch.Generator().manual_seed(seed)
    n = blocks * block
    c = Pair(1, blocks, 1, block, dim, I8, I8)
    great = torch.zeros(n, dtype=torch.bool)
    for b in order:
        great[b * block:(b + 1) * block] = True
    k = torch.zeros(n, 1, dim)
    k[:, 0, 0] = torch.where(great, scores[1], scores[0]) * dim ** 0.5      # (a constant in a block: 127 times a step exactly)
    v = rows(gen, n, 1, dim, torch.float32) * torch.where(great, 2.0 ** apart, 1.0)[:, None, None]
    if dtype == torch.float16:
        v *= 2.0 ** -6
    c.append(k.to(dtype), v.to(dtype), [n])
    q = torch.zeros(1, heads, dim)
    q[:, :, 0] = 1.0
    return c, q.to(dtype), n


@pytest.mark.parametrize("order", [[0], [5], [11], [4, 9], [3, 4, 5, 6]])
@pytest.mark.parametrize("dtype,apart", [(torch.float16, a) for a in (5, 12, 18)] +
                         [(torch.bfloat16, a) for a in (5, 22, 28, 36, 60, 100, 120)])
@pytest.mark.parametrize("given", ["none", "even", "all"])
@pytest.mark.parametrize("block", [16, 64])
def test_great_blocks_with_little_attention(order, dtype, apart, given, block):
    """Blocks 2^apart times as great that get next to no attention, as much of the result as the others, or all of it."""
    less = {"none": 200.0, "even": min(apart, 110) * 0.6931, "all": 0.0}[given]
    print(order, dtype, apart, given, block, flush=True)
    c, q, n = one_great_block(order, apart, dtype, (0.0, -less), block=block)
    want, _ = R.decode(c.ref, c.table, [n], q, 1)
    close(B.mnnq_attn_decode(q.cuda(), *c.args()), want, dtype)
    close(B.mnnq_attn_decode(q.cuda(), *c.args(), weights=torch.zeros((1, 1, n), device="cuda")), want, dtype)


@pytest.mark.parametrize("n", [48, 41, 700])
@pytest.mark.parametrize("great", [1e10, 1e30, 3e38])
@pytest.mark.parametrize("types", [(I8, I8), (I8, F8)])
def test_a_great_value_behind_a_query_is_not_its_concern(n, great, types):
    """Two queries; the last token, which the first does not see, opens a block (48 tokens before it) or shares one."""
    gen = torch.Generator().manual_seed(n)
    c = Pair(1, 48, 1, 16, 64, *types)
    k, v = rows(gen, n + 1, 1, 64, torch.bfloat16), rows(gen, n + 1, 1, 64, torch.bfloat16)
    v[n, 0, 5] = great
    c.append(k, v, [n + 1])
    q = rows(gen, 2, 8, 64, torch.bfloat16)
    want, _ = R.decode(c.ref, c.table, [n + 1], q, 2)
    close(B.mnnq_attn_decode(q.cuda(), *c.args()), want, torch.bfloat16)


def test_ranges_apart_and_an_undefined_block():
    """Ranges far apart beside one that is no number: only the rows that see it get it."""
    c, q, n = one_great_block([2, 5], 40, torch.bfloat16, (0.0, -100.0))
    c.gpu["v_range"][int(c.table[0, 11])] = float("nan")
    q = q.repeat(18, 1, 1)
    out = B.mnnq_attn_decode(q.cuda(), *c.args())
    want, _ = R.decode(c.ref, c.table, [n], q, 18)
    close(out[:2], want[:2], torch.bfloat16)                 # (the last block has 16 tokens: queries 0 and 1 see none of them)
    assert bool(torch.isnan(out[2:]).all())


