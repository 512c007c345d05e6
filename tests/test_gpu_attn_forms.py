"""Forms of the attention kernels that a call's sizes choose: widths with several parts, two row tiles with wide rows, long evictions."""
import pytest
import torch

from paper_2506_10443_amd import binding as B
from test_gpu_attn_decode import check, filled, rows
from test_gpu_kv_cache import F8, I8, Pair, run_evict, sums
from test_gpu_kv_cache import rows as spread_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [80, 144, 192, 256])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("k_type,v_type,dtype", [(I8, F8, torch.float16), (F8, I8, torch.bfloat16)])
def test_several_parts_of_wide_rows(dim, weights, k_type, v_type, dtype):
    gen = torch.Generator().manual_seed(dim)
    print("decode", dim, weights, dtype, flush=True)
    c = filled(gen, [1300, 40, 700], 2, 64, dim, k_type, v_type, dtype)
    check(c, rows(gen, 3, 8, dim, dtype), weights=weights)
    check(c, rows(gen, 2 * 3, 4, dim, dtype), 2, weights=weights)


@pytest.mark.parametrize("dim", [80, 128, 192, 256])
@pytest.mark.parametrize("heads,tokens", [(17, 1), (40, 1), (12, 3), (5, 8)])
@pytest.mark.parametrize("lengths", [[90, 300], [900, 33]])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_more_rows_than_a_tile(dim, heads, tokens, lengths, dtype):
    gen = torch.Generator().manual_seed(dim + heads)
    print("decode", dim, heads, tokens, lengths, dtype, flush=True)
    c = filled(gen, lengths, 1, 32, dim, I8, F8, dtype)
    check(c, rows(gen, 2 * tokens, heads, dim, dtype), tokens, weights=True)


@pytest.mark.parametrize("keep,recent", [(300, 100), (9000, 64), (20100, 0)])
def test_evict_more_tokens_than_are_held(keep, recent):
    gen = torch.Generator().manual_seed(keep)
    lengths = [20000, 700]
    more = -(-keep // 128)
    c = Pair(2, 157, 1, 128, 16, I8, F8, spare=2 * more)
    k = spread_rows(gen, sum(lengths), 1, 16, torch.float16)
    c.append(k, k, lengths)
    run_evict(c, sums(gen, (2, 1, 157 * 128)), keep, recent, c.free.view(2, more), keep)
