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


