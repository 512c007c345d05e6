"""mnnq_attn_prefill on values near both ends of bfloat16: means that the type holds come out as numbers.  Tolerance as in
test_gpu_attn_prefill.py."""
import pytest
import torch

from test_gpu_attn_prefill import check, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,lens", [(2, [70, 300]), (8, [500]), (64, [300]), (40, [1030])])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("least", [2.9e38, 1e-30])
def test_great_and_small_values(heads, lens, dim, least):
    gen = torch.Generator().manual_seed(heads + dim)
    n = sum(lens)
    print("prompt", heads, lens, dim, least, flush=True)
    v = (least * (1 + 0.1 * torch.rand((n, 2, dim), generator=gen))).to(torch.bfloat16)
    q, k = rows(gen, n, heads, dim, torch.bfloat16), rows(gen, n, 2, dim, torch.bfloat16)
    out = check(q, k, v, lens, lens)
    assert bool(torch.isfinite(out).all())
