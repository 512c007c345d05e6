"""Rows whose scores are all -inf: they see keys, but their softmax is 0 / 0.  A row of zeros is one that sees nothing."""
import pytest
import torch

import attn_reference as R
from paper_2506_10443_amd import binding as B
from test_gpu_attn_decode import TOL, filled, rows
from test_gpu_attn_prefill import starts
from test_gpu_kv_cache import F8, I8

pytestmark = pytest.mark.gpu


def agrees(out, want, dtype):
    """NaN where the definition has it, and the other rows as always."""
    out = out.cpu()
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    rest = ~torch.isnan(want).any(-1)
    assert R.error(out[rest], want[rest]) <= TOL[dtype]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,dim,lens", [(2, 64, [70, 90]), (8, 128, [200, 333]), (64, 64, [1100]), (64, 128, [300, 600]), (8, 256, [150])])
def test_prompt_rows_of_infinite_scores(dtype, heads, dim, lens):
    """A query with -inf in a channel where all keys are positive, and a first key that gives its only row -inf."""
    gen = torch.Generator().manual_seed(heads)
    n = sum(lens)
    print(dtype, heads, dim, lens, flush=True)
    q, k, v = rows(gen, n, heads, dim, dtype), rows(gen, n, 2, dim, dtype), rows(gen, n, 2, dim, dtype)
    k[:, :, 3] = k[:, :, 3].abs() + 0.5
    for at in (0, 33, n - 1):
        q[at, :, 3] = float("-inf")
    q[:, :, 7] = q[:, :, 7].abs() + 0.5
    q[lens[0] - 1, 0, 7] = float("-inf")
    k[:, :, 7] = k[:, :, 7].abs() + 0.5
    agrees(B.mnnq_attn_prefill(q.cuda(), k.cuda(), v.cuda(), starts(lens)), R.prompt(q, k, v, lens, lens), dtype)
    # a key of -inf: the first row sees nothing else, the others do
    q[:, :, 3] = rows(gen, n, heads, dim, dtype)[:, :, 3].abs() + 0.5
    k[0, :, 3] = float("-inf")
    want = R.prompt(q, k, v, lens, lens)
    assert torch.isnan(want[0]).all() and torch.isfinite(want[1:lens[0] - 1]).all()
    agrees(B.mnnq_attn_prefill(q.cuda(), k.cuda(), v.cuda(), starts(lens)), want, dtype)


def test_prompt_rows_that_see_nothing_beside_them():
    gen = torch.Generator().manual_seed(3)
    q, k, v = (rows(gen, n, 2, 64, torch.float16) for n in (40, 30, 30))
    k[:, :, 3] = k[:, :, 3].abs() + 0.5
    q[:, 0, 3] = float("-inf")
    want = R.prompt(q, k, v, [40], [30])
    assert not want[:10].any() and torch.isnan(want[10:, 0]).all()
    agrees(B.mnnq_attn_prefill(q.cuda(), k.cuda(), v.cuda(), starts([40]), starts([30])), want, torch.float16)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("k_type,v_type", [(I8, F8), (F8, I8)])
@pytest.mark.parametrize("lengths,dim", [([1, 40, 3], 64), ([300, 17, 0], 256), ([2600, 700, 1], 64)])
def test_cache_rows_of_infinite_scores(dtype, k_type, v_type, lengths, dim):
    """One wave, several, several parts; two queries each, of which the first sees nothing where there is one token."""
    gen = torch.Generator().manual_seed(sum(lengths))
    c = filled(gen, [0] * len(lengths), 2, 64, dim, k_type, v_type, extra=-(-max(lengths) // 64))
    n = sum(lengths)
    k = rows(gen, n, 2, dim, dtype)
    k[:, :, 3] = k[:, :, 3].abs() + 0.5                     # (a code of at least one step in every token)
    c.append(k, rows(gen, n, 2, dim, dtype), lengths)
    q = rows(gen, 2 * len(lengths), 8, dim, dtype)
    q[:, 1, 3] = q[3, 6, 3] = float("-inf")
    want, want_w = R.decode(c.ref, c.table, lengths, q, 2)
    w = torch.zeros((len(lengths), 2, c.table.shape[1] * 64), device="cuda")
    agrees(B.mnnq_attn_decode(q.cuda(), *c.args()), want, dtype)
    agrees(B.mnnq_attn_decode(q.cuda(), *c.args(), weights=w), want, dtype)
    got = w[..., :max(lengths)].cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want_w))
    assert R.error(got.nan_to_num(0.0), want_w.nan_to_num(0.0)) <= 1e-5


def test_a_cache_without_any_of_its_blocks_gives_zeros():
    gen = torch.Generator().manual_seed(4)
    for n in (40, 900):
        c = filled(gen, [n], 1, 16, 64)
        table = torch.full_like(c.table, -1)
        w = torch.zeros((1, 1, table.shape[1] * 16), device="cuda")
        for q in (rows(gen, 1, 4, 64, torch.float16), torch.full((1, 4, 64), float("-inf"), dtype=torch.float16)):
            assert not B.mnnq_attn_decode(q.cuda(), *c.args(table=table)).any()
            assert not B.mnnq_attn_decode(q.cuda(), *c.args(table=table), weights=w).any()
        assert not w.any()


