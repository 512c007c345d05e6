"""mnnq_kv_evict: tokens whose blocks the cache does not have, weights shorter than a sequence, the newest tokens' weights."""
import pytest
import torch

import attn_reference as R
from paper_2506_10443_amd import binding as B
from test_gpu_attn_decode import TOL
from test_gpu_kv_cache import F8, I8, Pair, rows, sums

pytestmark = pytest.mark.gpu


def chosen(w, there, keep, recent):
    """Places kept of a row of weights, `there` the places that can be."""
    newest = there[len(there) - min(recent, keep, len(there)):]
    others = there[:len(there) - len(newest)]
    best = sorted(others, key=lambda i: (-float(w[i]), i))[:min(keep, len(there)) - len(newest)]
    return sorted(best) + newest

def test_the_newest_tokens_weights_are_written_like_the_others():
    """-0 as 0, every NaN as the same one."""
    gen = torch.Generator().manual_seed(4)
    c = Pair(1, 4, 1, 16, 16, I8, I8, spare=2)
    k = rows(gen, 60, 1, 16, torch.float16)
    c.append(k, k, [60])
    w = torch.full((1, 1, 64), -0.0)
    odd = torch.tensor([0x7f800001, -1, 0x7fc00000, -0x80000000], dtype=torch.int64).to(torch.int32).view(torch.float32)
    w[0, 0, 10:14] = odd
    w[0, 0, 56:60] = odd
    nw = torch.empty((1, 1, 20), device="cuda")
    kept, _ = B.mnnq_kv_evict(*c.args(), w.cuda(), 20, 8, c.free.view(1, 2).cuda(), nw)
    places = kept[0, 0].tolist()
    assert places == list(range(9)) + [10, 11, 12] + list(range(52, 60))
    bits = nw[0, 0].cpu().view(torch.int32).tolist()
    assert bits == [0x7fc00000 if p in (10, 11, 12, 56, 57, 58) else 0 for p in places]


@pytest.mark.parametrize("n", [200, 5000])
@pytest.mark.parametrize("stride", [1, 100, 150])
def test_weights_shorter_than_the_sequence(n, stride):
    """Tokens behind the weights have a weight of zero; the newest ones stay."""
    gen = torch.Generator().manual_seed(n + stride)
    c = Pair(1, n // 16 + 1, 2, 16, 16, I8, I8, spare=4)
    k = rows(gen, n, 2, 16, torch.float16)
    c.append(k, k, [n])
    w = sums(gen, (1, 2, stride))
    whole = torch.cat([w, torch.zeros(1, 2, n - stride)], -1)
    for keep, recent in ((60, 20), (64, 0), (5, 5)):
        nw = torch.empty((1, 2, 64), device="cuda")
        kept, left = B.mnnq_kv_evict(*c.args(), w.cuda(), keep, recent, c.free.view(1, 4).cuda(), nw)
        assert left.tolist() == [keep]
        for h in range(2):
            places = chosen(whole[0, h], list(range(n)), keep, recent)
            assert kept[0, h].tolist() == places
            assert torch.equal(nw[0, h, :keep].cpu(), whole[0, h][torch.tensor(places)]) and not nw[0, h, keep:].any()



@pytest.mark.parametrize("k_type,v_type,dim,block", [(I8, F8, 64, 16), (F8, I8, 80, 64)])
@pytest.mark.parametrize("keep,recent", [(1, 1), (40, 8), (64, 64), (150, 100), (400, 0), (400, 300)])
def test_tokens_of_missing_blocks_are_not_kept(k_type, v_type, dim, block, keep, recent):
    """They count as masked before; they must not come back as tokens that are seen."""
    gen = torch.Generator().manual_seed(keep)
    lengths = [300, 64, 33, 130, 0]
    print("evict", dim, block, keep, recent, flush=True)
    per, more = -(-max(lengths) // block), -(-keep // block)
    c = Pair(5, per, 2, block, dim, k_type, v_type, spare=5 * more)
    c.append(rows(gen, sum(lengths), 2, dim, torch.float16), rows(gen, sum(lengths), 2, dim, torch.float16), lengths)
    table = c.table.clone()
    table[0, 1] = table[0, 3] = -1                          # between, and the newest tokens of the second
    table[1, (lengths[1] - 1) // block] = 1 << 30
    table[2] = -5                                           # all of the third
    there = [[t for t in range(n) if 0 <= int(table[s, t // block]) < c.gpu["k_codes"].shape[0]] for s, n in enumerate(lengths)]
    w, fresh = sums(gen, (5, 2, per * block)), c.free.view(5, more)
    nw = torch.full((5, 2, keep + 3), 9.0, device="cuda")
    source = {x: (c.ref.codes[x].clone(), c.ref.range[x].clone()) for x in "kv"}
    kept, left = B.mnnq_kv_evict(*c.args(table=table), w.cuda(), keep, recent, fresh.cuda(), nw)
    lens = [min(len(x), keep) for x in there]
    assert left.tolist() == lens
    for s in range(5):
        for h in range(2):
            places = chosen(w[s, h], there[s], keep, recent)
            assert kept[s, h].tolist() == places + [-1] * (keep - len(places)), (s, h)
            assert torch.equal(nw[s, h, :len(places)].cpu(), w[s, h][torch.tensor(places, dtype=torch.long)])
            assert not nw[s, h, len(places):].any()
            for x in "kv":
                codes, ranges = source[x]
                for b in range(-(-len(places) // block)):
                    part = places[b * block:(b + 1) * block]
                    at, to = [int(table[s, t // block]) for t in part], int(fresh[s, b])
                    r = max(float(ranges[i, h]) for i in at)
                    c.ref.range[x][to, h] = r
                    for j, (t, i) in enumerate(zip(part, at)):
                        old, code = float(ranges[i, h]), codes[i, h, t % block]
                        c.ref.codes[x][to, h, j] = code if old == r else R.nearest(code * old / r, c.ref.type[x])
    c.check(fresh, lens)


def test_attention_after_missing_tokens_went_is_what_it_was():
    gen = torch.Generator().manual_seed(1)
    c = Pair(1, 20, 2, 16, 64, I8, F8, spare=20)
    c.append(rows(gen, 300, 2, 64, torch.float16), rows(gen, 300, 2, 64, torch.float16), [300])
    for x in "kv":
        c.gpu[x + "_range"][:] = 3.0                        # (the same range everywhere: codes move as they are)
    table = c.table.clone()
    table[0, 4] = table[0, 18] = -1
    q = rows(gen, 1, 8, 64, torch.float16).cuda()
    before = B.mnnq_attn_decode(q, *c.args(table=table))
    nw = torch.empty((1, 2, 320), device="cuda")
    _, left = B.mnnq_kv_evict(*c.args(table=table), torch.ones((1, 2, 320), device="cuda"), 320, 20, c.free.view(1, 20).cuda(), nw)
    assert left.tolist() == [272]
    after = B.mnnq_attn_decode(q, *c.args(lengths=[272], table=c.free.view(1, 20)))
    assert R.error(after.cpu(), before.cpu().double()) <= 2 * TOL[torch.float16]


def test_missing_blocks_among_many_tokens():
    gen = torch.Generator().manual_seed(2)
    c = Pair(1, 160, 1, 128, 16, I8, I8, spare=70)
    k = rows(gen, 20000, 1, 16, torch.float16)
    c.append(k, k, [20000])
    table = c.table.clone()
    table[0, 3::5] = -1
    table[0, 150:156] = -1
    there = [t for t in range(20000) if int(table[0, t // 128]) >= 0]
    w = sums(gen, (1, 1, 160 * 128))
    for keep, recent in ((8900, 3000), (100, 0), (5000, 5000)):
        nw = torch.empty((1, 1, 9000), device="cuda")
        kept, left = B.mnnq_kv_evict(*c.args(table=table), w.cuda(), keep, recent, c.free.view(1, 70).cuda(), nw)
        assert left.tolist() == [keep] and kept[0, 0].tolist() == chosen(w[0, 0], there, keep, recent)


