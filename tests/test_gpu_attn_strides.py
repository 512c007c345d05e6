"""Rows of q, k and v that share memory: one row for all tokens or heads (distance 0), rows that overlap."""
import pytest
import torch

from paper_2506_10443_amd import binding as B
from test_gpu_attn_decode import filled, rows
from test_gpu_attn_prefill import starts
from test_gpu_kv_cache import Pair

pytestmark = pytest.mark.gpu


def shared(gen, tokens, heads, dim, dtype, how):
    """A view and its copy."""
    if how == "tokens":
        x = rows(gen, 1, heads, dim, dtype).cuda().expand(tokens, heads, dim)
    elif how == "heads":
        x = rows(gen, tokens, 1, dim, dtype).cuda().expand(tokens, heads, dim)
    else:
        flat = rows(gen, 1, 1, 8 * tokens + 16 * heads + dim, dtype).cuda().view(-1)
        x = flat.as_strided((tokens, heads, dim), (8, 16, 1))
    return x, x.contiguous()


@pytest.mark.parametrize("how", ["tokens", "heads", "overlap"])
@pytest.mark.parametrize("heads,lens", [(4, [70, 33]), (16, [300]), (64, [500])])
@pytest.mark.parametrize("bad", [None, float("nan")])
def test_prompt(how, heads, lens, bad):
    gen = torch.Generator().manual_seed(heads)
    n = sum(lens)
    (q, qc), (k, kc), (v, vc) = (shared(gen, n, h, 64, torch.bfloat16, how) for h in (heads, 2, 2))
    if bad is not None:
        v[n // 2, 0, 5] = bad
        vc = v.contiguous()
    out, want = B.mnnq_attn_prefill(q, k, v, starts(lens)), B.mnnq_attn_prefill(qc, kc, vc, starts(lens))
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("how", ["tokens", "heads", "overlap"])
def test_cache(how):
    gen = torch.Generator().manual_seed(1)
    (k, kc), (v, vc) = (shared(gen, 70, 2, 64, torch.float16, how) for _ in range(2))
    caches = [Pair(1, 3, 2, 32, 64) for _ in range(2)]
    for c, kk, vv in zip(caches, (k, kc), (v, vc)):
        B.mnnq_kv_append(kk, vv, *c.args(lengths=[0]))
    for x in ("k_codes", "v_codes", "k_range", "v_range"):
        a, b = (c.gpu[x].view(torch.uint8) for c in caches)
        assert torch.equal(a, b)
    c = filled(gen, [90, 20], 2, 32, 64)
    q, qc = shared(gen, 2 * 3, 8, 64, torch.float16, how)
    assert torch.equal(B.mnnq_attn_decode(q, *c.args()), B.mnnq_attn_decode(qc, *c.args()))
