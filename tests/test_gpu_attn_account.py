"""The account that mnnq_attn_decode keeps of the attention given: a query adds to the tokens that it sees and to no other."""
import pytest
import torch

import attn_reference as R
from paper_2506_10443_amd import binding as B
from test_gpu_attn_decode import filled, rows
from test_gpu_kv_cache import F8, I8

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


