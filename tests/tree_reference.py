"""Plain 64-bit implementations of the operators of tree drafts and of a bounded
cache, one tree, row or head at a time, on CPU tensors."""
import math

import torch

from tests.layer_reference import PAGE, tokens


def masks(parents):
    """[n] Python integers: bit j of entry i for node i itself and the nodes above it,
    0 for rows that are not part of the tree."""
    words = []
    for i, p in enumerate(parents):
        if p < -1 or p >= i or (p >= 0 and not words[p]):
            words.append(0)
        else:
            words.append(1 << i | (words[p] if p >= 0 else 0))
    return words


def signed(word):
    return word - (1 << 64) if word >> 63 else word


def path(parents, node_tokens, sampled):
    """The nodes that the target's tokens lead through, from node 0."""
    out = [0]
    while True:
        at = out[-1]
        more = [c for c in range(at + 1, len(parents)) if parents[c] == at and node_tokens[c] == sampled[at]]
        if not more:
            return out
        out.append(more[0])


def sees(i, before, n, word):
    """Positions that row i of n sees behind a context of `before` tokens."""
    return list(range(before)) + [before + j for j in range(n) if word >> j & 1]


def attention(q, k_cache, v_cache, block_table, seq_lens, mask, scale=None):
    """(out, lse, spread) in fp64; mask [B][n] of Python integers; spread = sum_t p_t
    |v_t|, the size that relative errors of the weights are multiplied by."""
    B, n, H, d = q.shape
    kv = k_cache.shape[1]
    scale = scale or 1 / math.sqrt(d)
    out, spread = torch.zeros(2, B, n, H, d, dtype=torch.float64)
    lse = torch.full((B, n, H), -math.inf, dtype=torch.float64)
    for b in range(B):
        T = int(seq_lens[b])
        if T == 0:
            continue
        k, v = (tokens(c, block_table[b], T) for c in (k_cache, v_cache))
        for i in range(n):
            at = sees(i, T - n, n, mask[b][i])
            if not at:
                continue
            for h in range(H):
                kk, vv = k[h * kv // H, at], v[h * kv // H, at]
                s = scale * (kk @ q[b, i, h].double())
                lse[b, i, h] = torch.logsumexp(s, 0)
                w = torch.softmax(s, 0)
                out[b, i, h] = w @ vv
                spread[b, i, h] = w @ vv.abs()
    return out, lse, spread


def mass(q, lse, k_cache, block_table, seq_lens, weights=None, scale=None):
    """(sums [B][kv][tokens of the longest context] in fp64, error bound of fp32 scores
    and sums).  A score is off by at most d 2^-23 sum |q_e k_e| scale (sums of d
    products in any order, each step's rounding 2^-23 at most), its way through the
    exponent by 2^-22 |score - lse| + 2^-20, which is the relative error of its weight;
    adding up R of them costs R 2^-24 of the sum."""
    B, n, H, d = q.shape
    kv = k_cache.shape[1]
    g = H // kv
    scale = scale or 1 / math.sqrt(d)
    longest = max(1, max(int(t) for t in seq_lens) - n)
    total, bound = torch.zeros(2, B, kv, longest, dtype=torch.float64)
    for b in range(B):
        before = int(seq_lens[b]) - n
        if before <= 0:
            continue
        k = tokens(k_cache, block_table[b], before)
        for i in range(n):
            w = 1.0 if weights is None else float(weights[b, i])
            if w == 0:
                continue
            for h in range(H):
                if lse[b, i, h] == -math.inf:
                    continue
                x = q[b, i, h].double()
                s = scale * (k[h // g] @ x) - lse[b, i, h].double()
                p = w * s.exp()
                total[b, h // g, :before] += p
                off = d * 2.0 ** -23 * scale * (k[h // g].abs() @ x.abs()) + (s.abs() + lse[b, i, h].abs()) * 2.0 ** -22 + 2.0 ** -20
                bound[b, h // g, :before] += p * (off + n * g * 2.0 ** -24)
    return total, bound


def kept(mass_row, length, budget, first, recent):
    """Positions that stay of one head's `length` tokens."""
    if length <= budget:
        return list(range(length))
    must = [t for t in range(length) if t < first or t >= length - recent]
    rest = [t for t in range(length) if first <= t < length - recent]
    value = [-math.inf if math.isnan(x) else x for x in mass_row[:length]]
    rest = sorted(rest, key=lambda t: (-value[t], t))[:budget - len(must)]
    return sorted(must + rest)


def place(table_row, position):
    return int(table_row[position // PAGE]), position % PAGE
