"""mnnq_attn_decode against attention in 64 bits over the values that the cache's codes stand for.

Tolerance (2-norm of the difference over that of the result): the result is rounded once, to 2^-12 of a value at most for float16 and
2^-9 for bfloat16, the probabilities to halves; queries, codes and products are exact and the sums fp32.  As for the prompt the bound is
a full unit, 2^-11 and 2^-8.  Attention weights are fp32 throughout: scores up to a few tens carry 2^-24 of themselves into the exponent
and as much from their sums, 64 terms' worth and more at most: 1e-5."""
import pytest
import torch

import attn_reference as R
from paper_2506_10443_amd import binding as B
from test_gpu_kv_cache import F8, I8, Pair

pytestmark = pytest.mark.gpu

TOL = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def rows(gen, tokens, heads, dim, dtype, spread=1.0):
    return (torch.randn((tokens, heads, dim), generator=gen) * spread).to(dtype)


def filled(gen, lengths, kv_heads, block, dim, k_type=I8, v_type=F8, dtype=torch.float16, extra=1):
    most = max(max(lengths), 1)
    c = Pair(len(lengths), -(-most // block) + extra, kv_heads, block, dim, k_type, v_type)
    n = sum(lengths)
    if n:
        c.append(rows(gen, n, kv_heads, dim, dtype), rows(gen, n, kv_heads, dim, dtype), lengths)
    return c


def check(c, q, tokens=1, weights=False, max_length=None, scale=None):
    want, want_w = R.decode(c.ref, c.table, c.lengths, q, tokens, scale)
    w = None
    if weights:
        base = torch.rand((len(c.lengths), c.ref.kv_heads, c.table.shape[1] * c.ref.block), device="cuda")
        w = base.clone()
    out = B.mnnq_attn_decode(q.cuda(), *c.args(), max_length=max_length, weights=w, scale=scale)
    assert R.error(out.cpu(), want) <= TOL[q.dtype]
    off = (out.cpu().double() - want).norm(dim=-1)
    assert float(off.max()) <= 8 * TOL[q.dtype] * float(want.norm(dim=-1).max())
    if weights:
        n = want_w.shape[2]
        assert R.error((w - base)[..., :n].cpu(), want_w) <= 1e-5 + 2.0 ** -24 * float(base[..., :n].norm()) / float(want_w.norm())
        for s, m in enumerate(c.lengths):
            assert torch.equal(w[s, :, m:], base[s, :, m:])
    return out


@pytest.mark.parametrize("k_type,v_type", [(I8, I8), (I8, F8), (F8, I8), (F8, F8)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,block", [(128, 64), (64, 16), (80, 32), (256, 128), (16, 16), (192, 64)])
def test_forms_and_widths(k_type, v_type, dtype, dim, block):
    gen = torch.Generator().manual_seed(dim)
    print("decode", k_type, v_type, dtype, dim, block, flush=True)
    c = filled(gen, [1, 17, 200, 333, 0], 2, block, dim, k_type, v_type)
    out = check(c, rows(gen, 5, 8, dim, dtype))
    assert not out[4].any()                                    # an empty cache: zeros


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000])
def test_lengths(n):
    gen = torch.Generator().manual_seed(n)
    check(filled(gen, [n], 1, 16, 64), rows(gen, 1, 4, 64, torch.float16))


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (7, 1), (16, 1), (17, 1), (40, 1), (28, 4), (8, 8)])
@pytest.mark.parametrize("tokens", [1, 2, 5])
def test_groups_and_tokens(heads, kv_heads, tokens):
    gen = torch.Generator().manual_seed(heads + tokens)
    lengths = [150, 5, 2]                                      # (fewer tokens than queries: the first see nothing)
    c = filled(gen, lengths, kv_heads, 32, 64)
    out = check(c, rows(gen, 3 * tokens, heads, 64, torch.float16), tokens, weights=True)
    if tokens == 5:
        assert not out[2 * tokens:2 * tokens + 3].any() and out[-1].any()


@pytest.mark.parametrize("weights", [False, True])
def test_parts_of_long_sequences(weights):
    """Long enough for many parts, with short sequences beside; a bound above the lengths, and one that cuts them."""
    gen = torch.Generator().manual_seed(1)
    c = filled(gen, [2600, 3, 700], 1, 128, 64)
    q = rows(gen, 3, 4, 64, torch.float16)
    check(c, q, weights=weights, max_length=2600)
    check(c, q, weights=weights)
    full = c.lengths
    c.lengths = [500, 3, 500]
    want, _ = R.decode(c.ref, c.table, c.lengths, q, 1)
    c.lengths = full
    out = B.mnnq_attn_decode(q.cuda(), *c.args(), max_length=500)
    assert R.error(out.cpu(), want) <= TOL[torch.float16]


def test_ranges_far_apart():
    """Blocks of very different magnitudes, greatest first, last and between; queries near both ends of bfloat16."""
    gen = torch.Generator().manual_seed(2)
    c = Pair(1, 20, 1, 16, 64, I8, F8)
    n = 300
    k = rows(gen, n, 1, 64, torch.bfloat16, 0.05)
    v = rows(gen, n, 1, 64, torch.bfloat16)
    size = torch.tensor([1e-6, 1.0, 1e4, 1e-20, 30.0])
    v = (v.float() * size[(torch.arange(n) // 16) % 5][:, None, None]).to(torch.bfloat16)
    c.append(k, v, [n])
    check(c, rows(gen, 1, 4, 64, torch.bfloat16))
    check(c, rows(gen, 1, 4, 64, torch.bfloat16, 1e30), scale=1e-30)
    check(c, rows(gen, 1, 4, 64, torch.bfloat16, 1e-30), scale=1e30)
    check(c, rows(gen, 1, 4, 64, torch.bfloat16) * 0, weights=True)
    small = Pair(1, 20, 1, 16, 64, I8, F8)
    small.append(k, (v.float() * 1e-12).to(torch.bfloat16), [n])
    check(small, rows(gen, 1, 4, 64, torch.bfloat16))


def test_great_scores():
    gen = torch.Generator().manual_seed(3)
    c = Pair(1, 10, 1, 32, 64, I8, I8)
    k = rows(gen, 300, 1, 64, torch.float16, 10.0)
    c.append(k, rows(gen, 300, 1, 64, torch.float16), [300])
    check(c, rows(gen, 1, 4, 64, torch.float16, 10.0))


def test_blocks_that_are_not_there_are_masked():
    gen = torch.Generator().manual_seed(4)
    c = filled(gen, [100], 1, 16, 64)
    q = rows(gen, 1, 4, 64, torch.float16)
    table = c.table.clone()
    table[0, 2], table[0, 5] = -1, 10000
    w = torch.zeros((1, 1, 128), device="cuda")
    out = B.mnnq_attn_decode(q.cuda(), *c.args(table=table), weights=w)
    seen = [t for t in range(100) if t // 16 not in (2, 5)]
    for h in range(4):
        k, v = c.ref.values("k", c.table[0], 100, 0)[seen], c.ref.values("v", c.table[0], 100, 0)[seen]
        want, p = R.attend(q[:, h], k, v, [len(seen)], 0.125)
        assert R.error(out[:, h].cpu(), want) <= 2 * TOL[torch.float16]
    assert not w[0, 0, 32:48].any() and not w[0, 0, 80:96].any() and not w[0, 0, 100:].any()
    assert abs(float(w.sum()) - 4) < 1e-4


def test_another_heads_undefined_block_does_no_harm():
    """A NaN appended for one head leaves the other heads' results as they are; rows that do not see it too."""
    gen = torch.Generator().manual_seed(5)
    c = filled(gen, [80], 2, 16, 64, I8, F8)
    q = rows(gen, 2, 8, 64, torch.float16)
    clean = B.mnnq_attn_decode(q.cuda(), *c.args())
    for x in "kv":
        c.gpu[x + "_range"][int(c.table[0, 2]), 1] = float("nan")
    out = B.mnnq_attn_decode(q.cuda(), *c.args())
    assert torch.equal(out[:, :4], clean[:, :4]) and torch.isnan(out[:, 4:]).all()


@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("k_type,v_type", [(I8, I8), (I8, F8), (F8, I8), (F8, F8)])
@pytest.mark.parametrize("evicted", [False, True])
def test_queries_before_an_undefined_block_do_not_see_it(what, k_type, v_type, evicted):
    """Two queries, the last token opens a block: only the second one sees what is no number there."""
    outs = []
    for value in (0.0, what):
        gen = torch.Generator().manual_seed(11)
        c = Pair(1, 8, 2, 16, 64, k_type, v_type, spare=8)
        c.append(rows(gen, 48, 2, 64, torch.bfloat16), rows(gen, 48, 2, 64, torch.bfloat16), [48])
        k, v = rows(gen, 1, 2, 64, torch.bfloat16), rows(gen, 1, 2, 64, torch.bfloat16)
        k[:, 1] = v[:, 1] = 0
        k[0, 1, 3] = v[0, 1, 5] = value
        B.mnnq_kv_append(k.cuda(), v.cuda(), *c.args())
        q = rows(gen, 2, 8, 64, torch.bfloat16).cuda()
        table, lengths = c.table, [49]
        if evicted:
            table = c.free.view(1, 8)
            B.mnnq_kv_evict(*c.args(lengths=lengths), torch.ones((1, 2, 128), device="cuda"), 128, 0, table.cuda(),
                            torch.empty((1, 2, 128), device="cuda"))
        outs.append(B.mnnq_attn_decode(q, *c.args(lengths=lengths, table=table)))
    clean, out = outs
    assert torch.equal(out[0], clean[0]) and torch.isfinite(clean).all()
    assert torch.equal(out[1, :4], clean[1, :4]) and torch.isnan(out[1, 4:]).all()


def test_strided_queries_and_output():
    gen = torch.Generator().manual_seed(6)
    c = filled(gen, [90, 20], 2, 32, 64)
    q = rows(gen, 2, 8, 64, torch.bfloat16)
    plain = check(c, q)
    whole = torch.zeros((2, 12, 64), dtype=torch.bfloat16, device="cuda")
    whole[:, 2:10] = q.cuda()
    out = torch.full((8, 5, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    B.mnnq_attn_decode(whole[:, 2:10], *c.args(), out=out[:, 1:3].transpose(0, 1))
    assert torch.equal(out[:, 1:3].transpose(0, 1), plain)
    assert bool((out[:, 0] == 2).all()) and bool((out[:, 3:] == 2).all())


def test_workspace_and_another_stream():
    gen = torch.Generator().manual_seed(7)
    c = filled(gen, [2000], 1, 64, 128)
    q = rows(gen, 1, 4, 128, torch.float16).cuda()
    args = c.args()
    want = B.mnnq_attn_decode(q, *args)
    need = B.mnnq_attn_decode_workspace_size(q, args[0], args[4])
    ws = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")    # (NaN everywhere)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.mnnq_attn_decode(q, *args, out=out, workspace=ws[:need])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want) and bool((ws[need:] == 0xff).all())


def test_a_graph_follows_the_lengths():
    """Appending and attending, recorded once: lengths and rows change on the device between the replays."""
    gen = torch.Generator().manual_seed(8)
    c = filled(gen, [250, 40], 2, 64, 128, extra=1)
    k_codes, k_range, v_codes, v_range, table, lengths = c.args()
    q, k, v = (rows(gen, 2, h, 128, torch.float16).cuda() for h in (4, 2, 2))
    out, w = torch.empty_like(q), torch.zeros((2, 2, table.shape[1] * 64), device="cuda")
    need = B.mnnq_attn_decode_workspace_size(q, k_codes, table, 0, True)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step():
        B.mnnq_kv_append(k, v, k_codes, k_range, v_codes, v_range, table, lengths)
        lengths.add_(1)
        B.mnnq_attn_decode(q, k_codes, k_range, v_codes, v_range, table, lengths, out=out, weights=w, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    c.ref.append("k", c.table[0], 250, k[:1].cpu()), c.ref.append("v", c.table[0], 250, v[:1].cpu())
    c.ref.append("k", c.table[1], 40, k[1:].cpu()), c.ref.append("v", c.table[1], 40, v[1:].cpu())
    c.lengths = [251, 41]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for t, h in ((q, 4), (k, 2), (v, 2)):
            t.copy_(rows(gen, 2, h, 128, torch.float16))
        w.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for s in range(2):
            c.ref.append("k", c.table[s], c.lengths[s], k[s:s + 1].cpu())
            c.ref.append("v", c.table[s], c.lengths[s], v[s:s + 1].cpu())
        c.lengths = [n + 1 for n in c.lengths]
        assert lengths.tolist() == c.lengths
        c.check()
        want, want_w = R.decode(c.ref, c.table, c.lengths, q.cpu(), 1)
        assert R.error(out.cpu(), want) <= TOL[torch.float16]
        assert R.error(w[..., :want_w.shape[2]].cpu(), want_w) <= 1e-5


def test_the_same_call_twice_gives_the_same_bits():
    gen = torch.Generator().manual_seed(9)
    c = filled(gen, [1500, 900], 2, 64, 128)
    q = rows(gen, 2, 8, 128, torch.float16).cuda()
    args = c.args()
    results = []
    for _ in range(3):
        w = torch.zeros((2, 2, c.table.shape[1] * 64), device="cuda")
        results.append((B.mnnq_attn_decode(q, *args, weights=w), w))
    assert all(torch.equal(a, results[0][0]) and torch.equal(b, results[0][1]) for a, b in results)
