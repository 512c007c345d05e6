"""Attention beside the quantized linear layer: what a program calls between the q|k|v and the output projection.

A prompt is attended to as a whole, on the projections' 16-bit results; its keys and values go into a cache of 8-bit codes,
one range for each block of tokens and head; every further token appends one row and attends to the cache; a program with
a budget drops the tokens that have had the least attention.  Four operators, one for each step:

  op "prompt": causal attention over packed prompts of different lengths, grouped heads; `history` keys stand before each
               sequence's first query (a prompt that goes on after a prefix).
  op "append": new keys and values into the cache; `lengths` tokens are there before, `tokens` are new (a number for each
               sequence).  The range of a block and head is the greatest magnitude in it; where a new token raises it, the
               block's older codes are rounded to the new range.
  op "decode": attention over the cache, `tokens` queries for each sequence (the last tokens in the cache are theirs);
               with `weights` the attention that each cached token received is added to a running sum as well.
  op "evict":  of every sequence and head the last `recent` tokens and the others with the greatest sums are kept, `keep`
               in all, and written to new blocks.

Head counts are those of `paper_2506_10443_amd.synth.MODELS` (Qwen2-1.5B 12 query and 2 key heads, Qwen2-7B 28 and 4,
Llama-3-8B 32 and 8, 128 wide); `draw` fills the ranges between them, other widths included.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
CODES = {"int8": torch.int8, "fp8": torch.float8_e4m3fn}
TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def _case(name, op, lengths, heads, kv_heads, **more):
    return {"name": name, "op": op, "lengths": lengths, "heads": heads, "kv_heads": kv_heads, "dim": 128, **more}


def listed():
    cache = {"k_codes": "int8", "v_codes": "int8", "block": 64}
    fp8 = {"k_codes": "fp8", "v_codes": "fp8", "block": 64}
    mixed = {"k_codes": "int8", "v_codes": "fp8", "block": 64}
    return [
        # one short prompt through the smallest model: latency
        _case("prompt 512 1.5b", "prompt", "512", 12, 2, type="f16", history=0),
        # prompts that arrived together, from one token to a page of text, packed without padding
        _case("prompts packed 7b", "prompt", "1,17,1024,333,64,777,129,1500,5,250", 28, 4, type="bf16", history=0),
        # the largest: one long document
        _case("prompt 8192 8b", "prompt", "8192", 32, 8, type="bf16", history=0),
        # what one generated token adds to the cache: the smallest call there is
        _case("append token 7b", "append", "713", 28, 4, tokens="1", type="f16", **cache),
        # the same for 48 sequences at once
        _case("append 48 tokens 8b", "append", ",".join(str(61 + 37 * i) for i in range(48)), 32, 8,
              tokens=",".join(["1"] * 48), type="bf16", **fp8),
        # a prompt's keys and values, behind a prefix that ends inside a block
        _case("append prompt 8b", "append", "100", 32, 8, tokens="8192", type="bf16", **mixed),
        # one token of one sequence, a short cache: latency
        _case("decode 1001 7b", "decode", "1001", 28, 4, tokens=1, type="f16", weights=False, **cache),
        # batched decoding, lengths as they come
        _case("decode batch 8b", "decode", ",".join(str(1 + (i * i * 547) % 8191) for i in range(32)), 32, 8, tokens=1,
              type="bf16", weights=False, **fp8),
        # one token of one sequence with a long cache
        _case("decode 131072 7b", "decode", "131072", 28, 4, tokens=1, type="f16", weights=False, **mixed),
        # a few tokens at once (speculative decoding) that keep account of the attention given
        _case("decode 4 tokens weights 1.5b", "decode", "4000,2999,1999,1500,1024,800,333,77", 12, 2, tokens=4, type="f16",
              weights=True, **cache),
        # a sequence that has outgrown its budget
        _case("evict 4097 7b", "evict", "4097", 28, 4, keep=1024, recent=128, **cache),
        # a batch of them, some still below it
        _case("evict batch 8b", "evict", ",".join(str(1000 + 1021 * i) for i in range(16)), 32, 8, keep=4096, recent=256,
              **fp8),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prompt", "append", "decode", "evict"])
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 4, 5, 7, 8])
    dim = rng.choice([64, 128, 128, 128, 80, 256])
    case = {"op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim}
    cache = {"k_codes": rng.choice(["int8", "fp8"]), "v_codes": rng.choice(["int8", "fp8"]),
             "block": rng.choice([16, 32, 64, 128])}
    kind = rng.choice(["f16", "bf16"])
    if op == "prompt":
        # the total bounds what the products of all pairs take
        count = rng.choice([1, 1, _log_uniform(rng, 2, 64)])
        most = 8192 if heads * dim <= 4096 else 4096
        total = _log_uniform(rng, 64, most)
        lengths = [total] if count == 1 else [_log_uniform(rng, 1, max(1, 3 * total // count)) for _ in range(count)]
        while sum(lengths) > most:
            lengths = [(n + 1) // 2 for n in lengths]
        history = rng.choice([0, 0, _log_uniform(rng, 1, 2048)]) if count <= 4 and sum(lengths) <= 2048 else 0
        case.update(type=kind, history=history)
    elif op == "append":
        count = rng.choice([1, _log_uniform(rng, 2, 64)])
        lengths = [_log_uniform(rng, 1, 2048) - 1 for _ in range(count)]
        if rng.random() < 0.5:
            tokens = [1] * count
        else:
            tokens = [_log_uniform(rng, 1, 8192 // count) for _ in range(count)]
        case.update(tokens=",".join(map(str, tokens)), type=kind, **cache)
    elif op == "decode":
        count = rng.choice([1, _log_uniform(rng, 2, 64)])
        most = min(131072, 2 ** 26 // (count * kv_heads * dim))
        lengths = [_log_uniform(rng, 1, most) for _ in range(count)]
        case.update(tokens=rng.choice([1, 1, 1, rng.randint(2, 8)]), type=kind, weights=rng.random() < 0.3, **cache)
    else:
        count = rng.choice([1, _log_uniform(rng, 2, 16)])
        lengths = [_log_uniform(rng, 256, 16384) for _ in range(count)]
        keep = _log_uniform(rng, 64, 4096)
        case.update(keep=keep, recent=rng.randint(0, keep // 4), **cache)
    case["lengths"] = ",".join(map(str, lengths))
    return case


def _numbers(text):
    return [int(n) for n in text.split(",")]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(counts):
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    return starts


def _rows(gen, tokens, heads, dim, dtype, spread, mean):
    """Rows of a projection: every channel of a head has a spread and a mean of its own."""
    s = torch.rand((heads, dim), generator=gen, device="cuda") * spread + 0.3
    m = torch.randn((heads, dim), generator=gen, device="cuda") * mean
    return (torch.randn((tokens, heads, dim), generator=gen, device="cuda") * s + m).to(dtype)


def _codes(gen, shape, dtype):
    values = torch.randn(shape, generator=gen, device="cuda") * (TOP[dtype] / 3)
    values = values.clamp_(-TOP[dtype], TOP[dtype])
    return values.round_().to(dtype) if dtype == torch.int8 else values.to(dtype)


def _cache(gen, case, capacities):
    """Blocks with room for `capacities` tokens of each sequence, in no order, and a few that are nobody's."""
    block, heads, dim = case["block"], case["kv_heads"], case["dim"]
    need = [-(-n // block) for n in capacities]
    blocks = sum(need) + 3
    order = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(need), max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    for i, (n, at) in enumerate(zip(need, _starts(need))):
        table[i, :n] = order[at:at + n]
    cache = {"block_table": table}
    for x in ("k", "v"):
        cache[x + "_codes"] = _codes(gen, (blocks, heads, block, dim), CODES[case[x + "_codes"]])
        # ranges are magnitudes of 16-bit numbers
        r = torch.rand((blocks, heads), generator=gen, device="cuda") * 2 + 3
        cache[x + "_range"] = r.to(TYPES[case.get("type", "bf16")]).float()
    return cache


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, heads, kv_heads, dim = case["op"], case["heads"], case["kv_heads"], case["dim"]
    lengths = _numbers(case["lengths"])
    state = {"op": op}
    if op == "prompt":
        dtype, keys = TYPES[case["type"]], [n + case["history"] for n in lengths]
        state["q_start"], state["k_start"] = _ints(_starts(lengths)), _ints(_starts(keys))
        # without history the three are column ranges of one projection's result
        rows = sum(lengths)
        state["q"] = _rows(gen, rows, heads, dim, dtype, 1.4, 0.2)
        state["k"] = _rows(gen, sum(keys), kv_heads, dim, dtype, 1.4, 0.5)
        state["v"] = _rows(gen, sum(keys), kv_heads, dim, dtype, 1.0, 0.3)
        if not case["history"]:
            whole = torch.cat([state["q"], state["k"], state["v"]], dim=1)
            state["q"], state["k"], state["v"] = whole[:, :heads], whole[:, heads:heads + kv_heads], whole[:, heads + kv_heads:]
        return state
    state["lengths"] = _ints(lengths)
    if op == "append":
        tokens = _numbers(case["tokens"])
        state.update(_cache(gen, case, [a + b for a, b in zip(lengths, tokens)]))
        state["start"] = _ints(_starts(tokens)) if max(tokens) > 1 else None
        state["k"] = _rows(gen, sum(tokens), kv_heads, dim, TYPES[case["type"]], 1.4, 0.5)
        state["v"] = _rows(gen, sum(tokens), kv_heads, dim, TYPES[case["type"]], 1.0, 0.3)
    elif op == "decode":
        state.update(_cache(gen, case, lengths))
        state["q"] = _rows(gen, len(lengths) * case["tokens"], heads, dim, TYPES[case["type"]], 1.0, 0.2)
        state["max_length"] = max(lengths)
        state["weights"] = None
        if case["weights"]:
            state["weights"] = torch.rand((len(lengths), kv_heads, max(lengths)), generator=gen, device="cuda")
    else:
        state.update(_cache(gen, case, lengths))
        kept = [min(n, case["keep"]) for n in lengths]
        # the new blocks: a second table into the same pool
        pool = _cache(gen, case, kept)
        pool["block_table"] += torch.where(pool["block_table"] >= 0, state["k_codes"].shape[0], 0).to(torch.int32)
        state["new_table"] = pool["block_table"]
        for x in ("k_codes", "k_range", "v_codes", "v_range"):
            state[x] = torch.cat([state[x].view(torch.uint8), pool[x].view(torch.uint8)]).view(state[x].dtype)
        # sums of attention: a few tokens have had most of it, many the same little, some none
        w = torch.exp(2 * torch.randn((len(lengths), kv_heads, max(lengths)), generator=gen, device="cuda") - 4)
        few = torch.rand(w.shape, generator=gen, device="cuda")
        state["weights"] = torch.where(few < 0.1, 0.0, torch.where(few < 0.2, 2.0 ** -9, w))
        state["new_weights"] = torch.empty((len(lengths), kv_heads, case["keep"] + 64), device="cuda")
        state["keep"], state["recent"] = case["keep"], case["recent"]
    return state


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _softmax(scores, seen):
    """Rows of attention; a row that sees nothing is all zeros."""
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, 1.0)


def _prompt(s):
    q, k, v = (s[x].float().transpose(0, 1).contiguous() for x in ("q", "k", "v"))
    group, dim = q.shape[0] // k.shape[0], q.shape[2]
    rows, keys = (torch.arange(x.shape[1], device="cuda", dtype=torch.int32) for x in (q, k))
    # sequence of every query and key, and the place in it, counted from the sequence's end
    q_seq = torch.searchsorted(s["q_start"], rows, right=True) - 1
    k_seq = torch.searchsorted(s["k_start"], keys, right=True) - 1
    q_at, k_at = rows - s["q_start"][q_seq + 1], keys - s["k_start"][k_seq + 1]
    seen = (q_seq[:, None] == k_seq) & (k_at <= q_at[:, None])
    q = q.view(k.shape[0], -1, dim)
    scores = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(1 / math.sqrt(dim))
    p = _softmax(scores.view(k.shape[0], group, len(rows), len(keys)), seen)
    out = torch.bmm(p.view(k.shape[0], -1, len(keys)), v)
    return out.view(-1, len(rows), dim).transpose(0, 1).contiguous().to(s["q"].dtype)


def _append(s):
    count, block = s["lengths"].shape[0], s["k_codes"].shape[2]
    rows = torch.arange(s["k"].shape[0], device="cuda", dtype=torch.int32)
    if s["start"] is None:
        seq, at = rows, s["lengths"]
    else:
        seq = torch.searchsorted(s["start"], rows, right=True) - 1
        at = s["lengths"][seq] + rows - s["start"][seq]
    place, slot = s["block_table"][seq, at // block], at % block
    # a block that begins with a new token has no range yet; the block that a sequence's tokens end in keeps its own
    partly = s["lengths"] % block > 0
    first = s["block_table"].gather(1, (s["lengths"] // block).clamp(max=s["block_table"].shape[1] - 1)[:, None].long())[:, 0]
    first = torch.where(partly, first, s["k_codes"].shape[0])  # (a block that does not exist where nothing is partly full)
    for x in ("k", "v"):
        codes, ranges, values = s[x + "_codes"], s[x + "_range"], s[x].float()
        top = TOP[codes.dtype]
        old = torch.cat([ranges, ranges.new_zeros(1, ranges.shape[1])])
        new = old.index_fill(0, place.long(), 0.0)
        new[first.long()] = old[first.long()]
        new.index_reduce_(0, place, values.abs().amax(-1), "amax")
        # older codes of the blocks that are partly full
        older = torch.where(partly, first, 0).long()
        before, after = old[older][:, :, None, None], new[older][:, :, None, None]
        raw = codes.view(torch.uint8)
        c = raw[older].view(codes.dtype).float()
        c = c * torch.where(after > 0, before, 0.0) / torch.where(after > 0, after, 1.0)
        c = c.round() if codes.dtype == torch.int8 else c
        there = torch.arange(block, device="cuda") < (s["lengths"] % block)[:, None]
        there = (there & partly[:, None])[:, None, :, None]
        kept = torch.where(there, c.to(codes.dtype).view(torch.uint8), raw[older])
        where = older[partly]
        raw[where] = kept[partly]
        # the new rows
        r = new[place.long()][:, :, None]
        c = values * top / torch.where(r > 0, r, 1.0)
        c = c.round() if codes.dtype == torch.int8 else c
        raw[place.long(), :, slot.long()] = c.to(codes.dtype).view(torch.uint8)
        ranges.copy_(new[:-1])
    return [s[x] for x in ("k_codes", "k_range", "v_codes", "v_range")]


def _values(s, x, table):
    """[sequences, heads, tokens, dim] of the cache in 32 bits."""
    codes, at = s[x + "_codes"], table.clamp(min=0).long()
    c = codes.view(torch.uint8)[at].view(codes.dtype).float()  # [sequences, blocks, heads, tokens, dim]
    c = c * (s[x + "_range"][at] / TOP[codes.dtype])[..., None, None]
    return c.transpose(1, 2).reshape(at.shape[0], codes.shape[1], -1, codes.shape[3])


def _decode(s):
    k, v = _values(s, "k", s["block_table"]), _values(s, "v", s["block_table"])
    count, heads, dim = k.shape[0], s["q"].shape[1], k.shape[3]
    tokens, group = s["q"].shape[0] // count, heads // k.shape[1]
    q = s["q"].float().view(count, tokens, k.shape[1], group, dim).permute(0, 2, 1, 3, 4).reshape(count * k.shape[1], -1, dim)
    scores = torch.bmm(q, k.view(-1, k.shape[2], dim).transpose(1, 2).contiguous()) * (1 / math.sqrt(dim))
    row = torch.arange(tokens, device="cuda")[:, None].expand(tokens, group).reshape(-1)
    limit = s["lengths"][:, None] - tokens + row + 1
    seen = (torch.arange(k.shape[2], device="cuda") < limit[:, :, None])[:, None]
    p = _softmax(scores.view(count, k.shape[1], -1, k.shape[2]), seen)
    out = torch.bmm(p.view(-1, p.shape[2], p.shape[3]), v.view(-1, v.shape[2], dim))
    out = out.view(count, k.shape[1], tokens, group, dim).permute(0, 2, 1, 3, 4).reshape(-1, heads, dim).to(s["q"].dtype)
    if s["weights"] is None:
        return out
    s["weights"] += p.sum(2)[..., :s["weights"].shape[2]]
    return out, s["weights"]


def _evict(s):
    block, keep, w = s["k_codes"].shape[2], s["keep"], s["weights"]
    lengths, at = s["lengths"][:, None, None], torch.arange(w.shape[2], device="cuda")
    rank = torch.where(at >= lengths - s["recent"], math.inf, w)
    rank = torch.where(at < lengths, rank, -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    order = torch.cat([order, order.new_zeros(*order.shape[:2], keep - order.shape[2])], -1)
    places = torch.arange(keep, device="cuda")
    left = torch.minimum(s["lengths"], torch.full_like(s["lengths"], keep))
    there = (places < left[:, None, None]).expand(order.shape)
    kept = torch.where(there, order, w.shape[2]).sort(-1).values
    source = torch.where(there, kept, 0)
    s["new_weights"].zero_()
    s["new_weights"][..., :keep] = torch.where(there, w.gather(-1, source), 0.0)
    seq = torch.arange(w.shape[0], device="cuda")[:, None, None]
    head = torch.arange(w.shape[1], device="cuda")[None, :, None]
    old = s["block_table"][seq, source // block].long()
    blocks = -(-keep // block)
    table = s["new_table"][:, :blocks]
    table = torch.cat([table, table.new_full((w.shape[0], blocks - table.shape[1]), -1)], 1)
    to = table[seq, places // block].long().expand(order.shape)
    h, slots = head.expand(order.shape), (places % block).expand(order.shape)
    for x in ("k", "v"):
        codes, ranges = s[x + "_codes"], s[x + "_range"]
        raw = codes.view(torch.uint8)
        before = torch.where(there, ranges[old, head], 0.0)
        pad = torch.cat([before, before.new_zeros(*before.shape[:2], blocks * block - keep)], -1)
        new = pad.view(*pad.shape[:2], blocks, block).amax(-1)
        after = new.repeat_interleave(block, -1)[..., :keep]
        c = raw[old, head, source % block].view(codes.dtype).float()
        c = c * before[..., None] / torch.where(after > 0, after, 1.0)[..., None]
        c = c.round() if codes.dtype == torch.int8 else c
        raw[to[there], h[there], slots[there]] = c[there].to(codes.dtype).view(torch.uint8)
        used = (table >= 0)[:, None].expand(new.shape)
        ranges[table[:, None].expand(new.shape)[used].long(), head.expand(new.shape)[used]] = new[used]
    kept = torch.where(there, kept, -1).to(torch.int32)
    return [kept, left, s["new_weights"]] + [s[x] for x in ("k_codes", "k_range", "v_codes", "v_range")]


def run(state):
    s, op = state, state["op"]
    if not own:
        return {"prompt": _prompt, "append": _append, "decode": _decode, "evict": _evict}[op](s)
    from paper_2506_10443_amd import binding as B
    if op == "prompt":
        return B.mnnq_attn_prefill(s["q"], s["k"], s["v"], s["q_start"], s["k_start"])
    cache = (s["k_codes"], s["k_range"], s["v_codes"], s["v_range"], s["block_table"], s["lengths"])
    if op == "append":
        B.mnnq_kv_append(s["k"], s["v"], *cache, start=s["start"])
        return list(cache[:4])
    if op == "decode":
        out = B.mnnq_attn_decode(s["q"], *cache, max_length=s["max_length"], weights=s["weights"])
        return out if s["weights"] is None else (out, s["weights"])
    kept, left = B.mnnq_kv_evict(*cache, s["weights"], s["keep"], s["recent"], s["new_table"], s["new_weights"])
    return [kept, left, s["new_weights"]] + list(cache[:4])


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    op, heads, kv_heads, dim = case["op"], case["heads"], case["kv_heads"], case["dim"]
    lengths = _numbers(case["lengths"])
    if op == "prompt":
        keys = [n + case["history"] for n in lengths]
        pairs = sum(n * (n + 1) // 2 + n * case["history"] for n in lengths)
        return {"bytes": 2 * dim * (2 * heads * sum(lengths) + 2 * kv_heads * sum(keys)), "flops": 4 * dim * heads * pairs}
    if op == "append":
        tokens = sum(_numbers(case["tokens"]))
        return {"bytes": tokens * kv_heads * dim * 2 * (2 + 1) + 8 * kv_heads * len(lengths), "flops": 0}
    if op == "decode":
        rows, total = case["tokens"] * len(lengths), sum(lengths)
        more = 8 * kv_heads * total if case["weights"] else 0
        return {"bytes": 2 * total * kv_heads * dim + 4 * rows * heads * dim + more,
                "flops": 4 * dim * heads * case["tokens"] * total}
    kept = sum(min(n, case["keep"]) for n in lengths)
    # the sums are read, the kept tokens' codes read and written, their places and sums written
    return {"bytes": kv_heads * (4 * sum(lengths) + kept * (4 * dim + 8)), "flops": 0}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _attend(q, k, v, visible):
    """One head of one sequence: q [rows, dim], row i sees the keys below visible[i]."""
    z = q @ k.t() / math.sqrt(q.shape[1])
    hidden = torch.arange(k.shape[0], device=z.device)[None, :] >= visible[:, None]
    z.masked_fill_(hidden, -math.inf)
    z = torch.nan_to_num(torch.softmax(z, dim=1), nan=0.0)  # (a row of nothing)
    return z @ v, z


def _to_grid(values, dtype):
    """Nearest code, ties to even: a whole number, or a number of three fraction bits from 2^-6 on."""
    if dtype == torch.int8:
        return values.round()
    part, _ = torch.frexp(values)  # 0.5 <= |part| < 1
    power = torch.where(values != 0, values / (2 * part), 0.0).clamp(min=2.0 ** -6)
    return (values / power * 8).round() * power / 8


def _exact_append(case, s):
    block, lengths, tokens = case["block"], _numbers(case["lengths"]), _numbers(case["tokens"])
    table, starts, result = s["block_table"].tolist(), _starts(_numbers(case["tokens"])), []
    for x in ("k", "v"):
        codes, dtype = s[x + "_codes"].double(), s[x + "_codes"].dtype
        ranges, rows = s[x + "_range"].double(), s[x].double()
        for i, (n, t) in enumerate(zip(lengths, tokens)):
            for b in range(n // block, (n + t - 1) // block + 1):
                lo, hi = max(n, b * block), min(n + t, (b + 1) * block)
                new, at, first = rows[starts[i] + lo - n:starts[i] + hi - n].transpose(0, 1), table[i][b], lo - b * block
                r = new.abs().amax((1, 2))
                if first > 0:
                    r = torch.maximum(r, ranges[at])
                    codes[at, :, :first] = _to_grid(codes[at, :, :first] * (ranges[at] / r)[:, None, None], dtype)
                codes[at, :, first:first + hi - lo] = _to_grid(new * TOP[dtype] / r[:, None, None], dtype)
                ranges[at] = r
        result += [codes if dtype != torch.int8 else None, ranges]
    return result


def _exact_decode(case, s):
    tokens, group = case["tokens"], case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    sums = s["weights"].double() if case["weights"] else None
    for i, n in enumerate(_numbers(case["lengths"])):
        places = s["block_table"][i, :-(-n // case["block"])].long()
        sees = torch.arange(tokens, device="cuda") + n - tokens + 1
        rows = slice(i * tokens, (i + 1) * tokens)
        for h in range(case["kv_heads"]):
            k, v = ((s[x + "_codes"].view(torch.uint8)[places, h].view(s[x + "_codes"].dtype).double()
                     * s[x + "_range"][places, h].double()[:, None, None] / TOP[s[x + "_codes"].dtype]).flatten(0, 1)[:n]
                    for x in ("k", "v"))
            for j in range(h * group, (h + 1) * group):
                out[rows, j], p = _attend(s["q"][rows, j].double(), k, v, sees)
                if sums is not None:
                    sums[i, h, :n] += p.sum(0)
    return out if sums is None else (out, sums)


def _exact_evict(case, s):
    block, keep, recent = case["block"], case["keep"], case["recent"]
    weights = torch.zeros(s["new_weights"].shape, dtype=torch.float64, device="cuda")
    after = {x: s[x].double() for x in ("k_codes", "k_range", "v_codes", "v_range")}
    for i, n in enumerate(_numbers(case["lengths"])):
        for h in range(case["kv_heads"]):
            w = s["weights"][i, h, :n].double()
            last = min(recent, n, keep)
            # by falling sum, then by place
            best = torch.argsort(-w[:n - last], stable=True)[:min(keep, n) - last]
            chosen = torch.cat([best, torch.arange(n - last, n, device="cuda")]).sort().values
            weights[i, h, :len(chosen)] = w[chosen]
            source = s["block_table"][i][chosen // block].long()
            for x in ("k", "v"):
                dtype, ranges = s[x + "_codes"].dtype, s[x + "_range"].double()[source, h]
                c = s[x + "_codes"].view(torch.uint8)[source, h, chosen % block].view(dtype).double()
                for b in range(-(-len(chosen) // block)):
                    part, to = slice(b * block, min((b + 1) * block, len(chosen))), int(s["new_table"][i, b])
                    r = ranges[part].max()
                    after[x + "_range"][to, h] = r
                    after[x + "_codes"][to, h, :part.stop - part.start] = _to_grid(c[part] * (ranges[part] / r)[:, None], dtype)
    for x in ("k_codes", "v_codes"):
        after[x] = after[x] if s[x].dtype != torch.int8 else None
    return [None, None, weights] + [after[x] for x in ("k_codes", "k_range", "v_codes", "v_range")]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(case, s)
    if case["op"] == "decode":
        return _exact_decode(case, s)
    if case["op"] == "evict":
        return _exact_evict(case, s)
    lengths, group = _numbers(case["lengths"]), case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for i, n in enumerate(lengths):
        before = at + i * case["history"]
        keys = slice(before, before + n + case["history"])
        for h in range(case["heads"]):
            out[at:at + n, h] = _attend(s["q"][at:at + n, h].double(), s["k"][keys, h // group].double(),
                                        s["v"][keys, h // group].double(),
                                        torch.arange(n, device="cuda") + case["history"] + 1)[0]
        at += n
    return out
