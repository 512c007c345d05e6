"""mnnq_attn_prefill against attention in 64 bits.

Tolerance (2-norm of the difference over that of the result): the result and the probabilities are each rounded once to the type, to
2^-12 of a value at most for float16 and 2^-9 for bfloat16; independent roundings of uniform mantissas have about 0.4 of that as root
mean square, two of them 0.57, and probabilities' roundings average out over keys at best - the bound is the full unit, 2^-11 and 2^-8,
which also covers the fp32 sums (2^-20)."""
import itertools

import numpy as np
import pytest
import torch

import attn_reference as R
from paper_2506_10443_amd import binding as B

pytestmark = pytest.mark.gpu

TOL = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def starts(lens):
    return torch.tensor([0] + list(itertools.accumulate(lens)), dtype=torch.int32, device="cuda")


def rows(gen, tokens, heads, dim, dtype, spread=1.0):
    return (torch.randn((tokens, heads, dim), generator=gen) * spread).to(dtype)


def check(q, k, v, q_lens, k_lens, scale=None, views=lambda t: t.cuda()):
    out = B.mnnq_attn_prefill(views(q), views(k), views(v), starts(q_lens), starts(k_lens), scale=scale)
    want = R.prompt(q, k, v, q_lens, k_lens, scale)
    assert out.shape == q.shape and out.dtype == q.dtype
    assert R.error(out.cpu(), want) <= TOL[q.dtype]
    # no single row is far off either: rows have norms of the same order, a row's error is a few times the average at most
    off = (out.cpu().double() - want).norm(dim=-1)
    assert float(off.max()) <= 8 * TOL[q.dtype] * float(want.norm(dim=-1).max())
    return out


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [16, 64, 80, 128, 144, 256])
@pytest.mark.parametrize("lens", [[1], [2], [31], [33], [64], [65], [127, 1, 130], [300]])
def test_lengths_and_widths(dtype, dim, lens):
    gen = torch.Generator().manual_seed(dim + sum(lens))
    n = sum(lens)
    print("prompt", dtype, dim, lens, flush=True)
    check(rows(gen, n, 4, dim, dtype), rows(gen, n, 2, dim, dtype), rows(gen, n, 2, dim, dtype), lens, lens)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [48, 96, 112, 176, 192, 208])
@pytest.mark.parametrize("heads,lens", [(2, [130]), (8, [200, 333]), (64, [600])])
def test_widths_between_the_powers_of_two(dtype, dim, heads, lens):
    gen = torch.Generator().manual_seed(dim + heads)
    n = sum(lens)
    print("prompt", dtype, dim, heads, lens, flush=True)
    check(rows(gen, n, heads, dim, dtype), rows(gen, n, 2, dim, dtype), rows(gen, n, 2, dim, dtype), lens, lens)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (7, 1), (8, 8), (12, 2), (28, 4)])
def test_grouped_heads(heads, kv_heads):
    gen = torch.Generator().manual_seed(heads)
    lens = [97, 40]
    n = sum(lens)
    check(rows(gen, n, heads, 64, torch.float16), rows(gen, n, kv_heads, 64, torch.float16),
          rows(gen, n, kv_heads, 64, torch.float16), lens, lens)


@pytest.mark.parametrize("q_lens,k_lens", [([5], [200]), ([64, 1], [65, 300]), ([200], [200 + 77]), ([1, 1, 1], [1, 64, 129])])
def test_keys_before_the_first_query(q_lens, k_lens):
    gen = torch.Generator().manual_seed(sum(k_lens))
    check(rows(gen, sum(q_lens), 4, 128, torch.bfloat16), rows(gen, sum(k_lens), 2, 128, torch.bfloat16),
          rows(gen, sum(k_lens), 2, 128, torch.bfloat16), q_lens, k_lens)


@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("q_lens,k_lens", [([600], [1100]), ([1055], [1055]), ([513], [1024]), ([1, 300, 40], [2500, 300, 700]),
                                           ([300, 260], [2000, 100])])
def test_many_heads_and_keys(dim, dtype, q_lens, k_lens):
    """Enough tiles of queries for every CU: two waves share the keys of a tile, one of them without any in the first rows."""
    gen = torch.Generator().manual_seed(dim + sum(q_lens))
    print("prompt", dim, dtype, q_lens, k_lens, flush=True)
    check(rows(gen, sum(q_lens), 64, dim, dtype), rows(gen, sum(k_lens), 2, dim, dtype), rows(gen, sum(k_lens), 2, dim, dtype),
          q_lens, k_lens)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["k", "v", "q"])
def test_what_is_masked_has_no_part_with_many_heads(bad, where):
    gen = torch.Generator().manual_seed(10)
    n, dim, dtype, at = 1100, 64, torch.bfloat16, 555
    x = {"q": rows(gen, n, 64, dim, dtype), "k": rows(gen, n, 1, dim, dtype), "v": rows(gen, n, 1, dim, dtype)}
    clean = B.mnnq_attn_prefill(x["q"].cuda(), x["k"].cuda(), x["v"].cuda(), starts([n]))
    x[where][at, :, 3] = bad
    out = B.mnnq_attn_prefill(x["q"].cuda(), x["k"].cuda(), x["v"].cuda(), starts([n]))
    assert torch.equal(out[:at], clean[:at])
    if where == "q":
        assert torch.equal(out[at + 1:], clean[at + 1:])
    if where == "v":
        assert not torch.isfinite(out[at:, :, 3]).any()


def test_rows_that_see_nothing_are_zero():
    # fewer keys than queries: the first ones see none; a sequence without keys; a sequence without queries
    gen = torch.Generator().manual_seed(5)
    q_lens, k_lens = [100, 70, 0, 40], [30, 0, 50, 40]
    q, k, v = (rows(gen, n, h, 64, torch.float16) for n, h in ((sum(q_lens), 4), (sum(k_lens), 2), (sum(k_lens), 2)))
    out = check(q, k, v, q_lens, k_lens)
    assert not out[:70].any() and not out[100:170].any() and out[70:100].any()


def test_projection_views_and_head_major_rows():
    gen = torch.Generator().manual_seed(6)
    n, heads, kv, dim = 150, 6, 2, 64
    q, k, v = rows(gen, n, heads, dim, torch.float16), rows(gen, n, kv, dim, torch.float16), rows(gen, n, kv, dim, torch.float16)
    plain = check(q, k, v, [n], [n])
    # columns of one q|k|v result
    whole = torch.cat([q, k, v], 1).cuda()
    out = B.mnnq_attn_prefill(whole[:, :heads], whole[:, heads:heads + kv], whole[:, heads + kv:], starts([n]))
    assert torch.equal(out, plain)
    # [heads, tokens, dim] in memory, the output too, with room between the heads that is not written
    major = lambda t: t.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    room = torch.full((heads, n + 3, dim), 7.0, dtype=torch.float16, device="cuda")
    out = B.mnnq_attn_prefill(major(q), major(k), major(v), starts([n]), out=room[:, :n].transpose(0, 1))
    assert torch.equal(out, plain) and torch.equal(room[:, n:], torch.full_like(room[:, n:], 7.0))


def test_rows_of_no_sequence_stay_as_they_are():
    gen = torch.Generator().manual_seed(7)
    q, k, v = (rows(gen, 100, h, 64, torch.float16) for h in (2, 1, 1))
    at = torch.tensor([10, 60, 60, 90], dtype=torch.int32, device="cuda")
    out = torch.full((100, 2, 64), 3.0, dtype=torch.float16, device="cuda")
    B.mnnq_attn_prefill(q.cuda(), k.cuda(), v.cuda(), at, out=out)
    want = R.prompt(q[10:90], k[10:90], v[10:90], [50, 30], [50, 30])
    assert R.error(out[10:90].cpu(), want) <= TOL[torch.float16]
    assert bool((out[:10] == 3).all()) and bool((out[90:] == 3).all())


def test_starts_outside_the_rows_are_clamped():
    gen = torch.Generator().manual_seed(8)
    q, k, v = (rows(gen, 64, h, 64, torch.float16) for h in (2, 1, 1))
    at = torch.tensor([-5, 40, 1000], dtype=torch.int32, device="cuda")
    out = B.mnnq_attn_prefill(q.cuda(), k.cuda(), v.cuda(), at)
    assert R.error(out.cpu(), R.prompt(q, k, v, [40, 24], [40, 24])) <= TOL[torch.float16]


def test_great_and_small_scores():
    """Scores of several hundred: one key takes all, and the running maximum moves from tile to tile."""
    gen = torch.Generator().manual_seed(9)
    n = 200
    q, k, v = rows(gen, n, 2, 128, torch.bfloat16, 12.0), rows(gen, n, 2, 128, torch.bfloat16, 12.0), rows(gen, n, 2, 128, torch.bfloat16)
    check(q, k, v, [n], [n])
    check(q * 0, k, v, [n], [n])                       # all keys the same
    rising = k * (torch.arange(n)[:, None, None] / n).to(torch.bfloat16)
    check(q, rising, v, [n], [n])
    check(q, k, v, [n], [n], scale=1e-4)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("where", ["k", "v", "q"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_what_is_masked_has_no_part(bad, where, dtype):
    """A NaN or an infinity at one token reaches the rows that see it and no other: not the earlier rows of the same tile, not the
    sequence before."""
    gen = torch.Generator().manual_seed(10)
    lens, dim = [70, 90], 64
    n = sum(lens)
    x = {"q": rows(gen, n, 2, dim, dtype), "k": rows(gen, n, 1, dim, dtype), "v": rows(gen, n, 1, dim, dtype)}
    clean = B.mnnq_attn_prefill(x["q"].cuda(), x["k"].cuda(), x["v"].cuda(), starts(lens))
    at = 70 + 41
    x[where][at, :, 3] = bad
    out = B.mnnq_attn_prefill(x["q"].cuda(), x["k"].cuda(), x["v"].cuda(), starts(lens))
    assert torch.equal(out[:at], clean[:at])
    if where == "q":
        assert torch.equal(out[at + 1:], clean[at + 1:])
    elif where == "v":
        assert not torch.isfinite(out[at:, :, 3]).any()
        keep = [d for d in range(dim) if d != 3]
        assert torch.equal(out[:, :, keep], clean[:, :, keep])


def test_another_stream_and_a_graph():
    gen = torch.Generator().manual_seed(11)
    lens = [130, 70]
    n = sum(lens)
    q, k, v = (rows(gen, n, h, 128, torch.bfloat16).cuda() for h in (4, 2, 2))
    at, out = starts(lens), torch.empty_like(q)
    want = B.mnnq_attn_prefill(q, k, v, at).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.mnnq_attn_prefill(q, k, v, at, out=out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.mnnq_attn_prefill(q, k, v, at, out=out)
    for i in range(3):
        q.copy_(rows(gen, n, 4, 128, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, B.mnnq_attn_prefill(q, k, v, at))


def test_long_prompt_rows_at_the_far_end():
    """The last rows of a long sequence see every tile."""
    gen = torch.Generator().manual_seed(12)
    n, dim = 5000, 128
    q, k, v = (rows(gen, n, h, dim, torch.float16) for h in (2, 1, 1))
    out = B.mnnq_attn_prefill(q.cuda(), k.cuda(), v.cuda(), starts([n])).cpu()
    for i in (0, 63, 64, 2047, 4095, 4999):
        for h in range(2):
            want, _ = R.attend(q[i:i + 1, h], k[:, 0], v[:, 0], [i + 1], dim ** -0.5)
            assert R.error(out[i:i + 1, h], want) <= 2 * TOL[torch.float16]
