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


