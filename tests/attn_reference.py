"""Attention and its 8-bit cache in 64 bits on the CPU, written from the definitions: the oracle of the attention tests."""
import math

import torch

TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def attend(q, k, v, visible, scale):
    """q [rows, dim], k and v [keys, dim], row i sees the keys below visible[i] -> (out, probabilities), 64 bits.  What a row does
    not see has no part in it, whatever its value."""
    q, k, v = q.double(), k.double(), v.double()
    out = torch.zeros(q.shape[0], v.shape[1], dtype=torch.float64)
    prob = torch.zeros(q.shape[0], k.shape[0], dtype=torch.float64)
    for i in range(q.shape[0]):
        n = max(0, min(int(visible[i]), k.shape[0]))
        if n:
            s = (k[:n] @ q[i]) * scale
            e = torch.exp(s - s.max())
            prob[i, :n] = e / e.sum()
            out[i] = prob[i, :n] @ v[:n]
    return out, prob


def prompt(q, k, v, q_lens, k_lens, scale=None):
    """Packed causal attention; [tokens, heads, dim] on the CPU -> 64 bits."""
    heads, dim = q.shape[1:]
    group = heads // k.shape[1]
    scale = 1 / math.sqrt(dim) if scale is None else scale
    out = torch.zeros(q.shape, dtype=torch.float64)
    qa = ka = 0
    for nq, nk in zip(q_lens, k_lens):
        sees = torch.arange(nq) + nk - nq + 1
        for h in range(heads):
            out[qa:qa + nq, h], _ = attend(q[qa:qa + nq, h], k[ka:ka + nk, h // group], v[ka:ka + nk, h // group], sees, scale)
        qa, ka = qa + nq, ka + nk
    return out


def nearest(values, dtype):
    """Codes of 64-bit values: nearest whole number, or nearest number with three fraction bits from 2^-6 on; ties to even."""
    if dtype == torch.int8:
        return values.round()
    _, e = torch.frexp(values)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return (values / step).round() * step


class Cache:
    """A cache on the CPU: codes as 64-bit numbers, ranges in 64 bits."""

    def __init__(self, blocks, kv_heads, block, dim, k_type, v_type):
        self.type = {"k": k_type, "v": v_type}
        self.block, self.kv_heads, self.dim = block, kv_heads, dim
        self.codes = {x: torch.zeros(blocks, kv_heads, block, dim, dtype=torch.float64) for x in "kv"}
        self.range = {x: torch.zeros(blocks, kv_heads, dtype=torch.float64) for x in "kv"}

    def append(self, x, table, length, rows):
        """rows [tokens, kv_heads, dim] of one sequence behind its first `length` tokens."""
        top, dtype, at = TOP[self.type[x]], self.type[x], 0
        while at < rows.shape[0]:
            place = length + at
            b, first = int(table[place // self.block]), place % self.block
            n = min(self.block - first, rows.shape[0] - at)
            part = rows[at:at + n].double()
            for h in range(self.kv_heads):
                codes = self.codes[x][b, h]
                old = float(self.range[x][b, h]) if first else 0.0
                new = max(old, float(part[:, h].abs().max()))
                if first and new != old:
                    codes[:first] = nearest(codes[:first] * old / new, dtype)
                codes[first:first + n] = nearest(part[:, h] * top / new, dtype) if new else 0.0
                self.range[x][b, h] = new
            at += n

    def values(self, x, table, length, head):
        """[length, dim] in 64 bits."""
        n = -(-length // self.block)
        b = table[:n].long()
        v = self.codes[x][b, head] * (self.range[x][b, head] / TOP[self.type[x]])[:, None, None]
        return v.reshape(-1, self.dim)[:length]


def decode(cache, tables, lengths, q, tokens, scale=None):
    """q [sequences * tokens, heads, dim] -> (out, weights [sequences, kv_heads, longest]) in 64 bits."""
    heads, dim = q.shape[1:]
    group = heads // cache.kv_heads
    scale = 1 / math.sqrt(dim) if scale is None else scale
    out = torch.zeros(q.shape, dtype=torch.float64)
    weights = torch.zeros(len(lengths), cache.kv_heads, max(max(lengths), 1), dtype=torch.float64)
    for s, n in enumerate(lengths):
        rows = slice(s * tokens, (s + 1) * tokens)
        sees = torch.arange(tokens) + n - tokens + 1
        for h in range(cache.kv_heads):
            k, v = cache.values("k", tables[s], n, h), cache.values("v", tables[s], n, h)
            for j in range(h * group, (h + 1) * group):
                out[rows, j], p = attend(q[rows, j], k, v, sees, scale)
                weights[s, h, :n] += p.sum(0)
    return out, weights


def evict(cache, tables, lengths, weights, keep, recent, new_tables):
    """Kept places and weights of every (sequence, head); moves the codes."""
    result = {}
    source = {x: (cache.codes[x].clone(), cache.range[x].clone()) for x in "kv"}
    for s, n in enumerate(lengths):
        for h in range(cache.kv_heads):
            last = min(recent, n, keep)
            w = weights[s, h, :n - last]
            best = sorted(range(n - last), key=lambda i: (-float(w[i]), i))[:min(keep, n) - last]
            chosen = sorted(best) + list(range(n - last, n))
            result[s, h] = chosen
            for x in "kv":
                codes, ranges = source[x]
                for b in range(-(-len(chosen) // cache.block)):
                    part = chosen[b * cache.block:(b + 1) * cache.block]
                    at = [int(tables[s][t // cache.block]) for t in part]
                    to = int(new_tables[s][b])
                    r = max(float(ranges[i, h]) for i in at)
                    cache.range[x][to, h] = r
                    for j, (t, i) in enumerate(zip(part, at)):
                        old = float(ranges[i, h])
                        c = codes[i, h, t % cache.block]
                        cache.codes[x][to, h, j] = c if old == r else nearest(c * old / r, cache.type[x])
    return result


def error(got, want):
    """2-norm of the difference over 2-norm of the result."""
    norm = float(want.norm())
    return float((got.double() - want).norm()) / norm if norm else float(got.double().norm())
