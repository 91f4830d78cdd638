"""Plain 64-bit implementations of the decoder-layer operators, one row, pair or
key at a time where that is short enough, on CPU tensors."""
import math

import torch

PAGE = 16


def rms_norm(x, weight, residual, eps):
    """(y, h) in fp64."""
    h = x.double() if residual is None else x.double() + residual.double()
    y = torch.empty_like(h)
    for t in range(h.shape[0]):
        y[t] = h[t] * weight.double() / math.sqrt(float((h[t] ** 2).sum()) / h.shape[1] + eps) \
            if torch.isfinite(h[t]).all() else h[t] * weight.double() / ((h[t] ** 2).sum() / h.shape[1] + eps).sqrt()
    return y, h


def scales(y, group):
    """Per row or per `group` columns: max|y| / 448, at least 2^-126."""
    width = group or y.shape[1]
    s = torch.stack([part.abs().amax(1) for part in y.split(width, 1)], 1) / 448
    return torch.where(s < 2.0 ** -126, torch.full_like(s, 2.0 ** -126), s)


def rotate(x, positions, inv_freq, axis, interleaved, amplitude=1.0):
    """x [T][H][d] rotated by positions [axes][T] in fp64."""
    y = x.double().clone()
    n = inv_freq.shape[0]
    for j in range(n):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + n)
        angle = positions[int(axis[j]) if axis is not None else 0].double() * inv_freq[j]
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        u, w = x[:, :, a].double(), x[:, :, b].double()
        y[:, :, a], y[:, :, b] = amplitude * (u * c - w * s), amplitude * (u * s + w * c)
    return y


def places(T, B, seq_lens, row_starts, block_table):
    """(page, slot) of every row, None for rows that are not appended."""
    out = [None] * T
    starts = [b * (T // B) for b in range(B + 1)] if row_starts is None else [int(v) for v in row_starts]
    for b in range(B):
        n = starts[b + 1] - starts[b]
        for i in range(n):
            at = int(seq_lens[b]) - n + i
            if int(seq_lens[b]) != 0 and 0 <= at < block_table.shape[1] * PAGE:
                out[starts[b] + i] = (int(block_table[b, at // PAGE]), at % PAGE)
    return out


def tokens(cache, pages, length):
    """The first `length` tokens of a page list: [H_kv][length][d] in fp64."""
    n = -(-length // PAGE)
    x = [cache[int(p)].double() if 0 <= int(p) < cache.shape[0] else torch.zeros(cache.shape[1:], dtype=torch.float64)
         for p in pages[:n]]
    if not x:
        return torch.zeros(cache.shape[1], 0, cache.shape[3], dtype=torch.float64)
    return torch.cat(x, 1)[:, :length]


def shared_prefix(q, k_cache, v_cache, prefix_table, prefix_lens, group_starts, block_table, seq_lens, scale=None):
    """(out, lse, spread) in fp64; spread = sum_t p_t |v_t|, the size that
    relative errors of the weights p_t are multiplied by."""
    B, n, H, d = q.shape
    kv = k_cache.shape[1]
    g_of = {b: g for g in range(len(group_starts) - 1) for b in range(int(group_starts[g]), int(group_starts[g + 1]))}
    scale = scale or 1 / math.sqrt(d)
    out, spread = torch.zeros(2, B, n, H, d, dtype=torch.float64)
    lse = torch.full((B, n, H), -math.inf, dtype=torch.float64)
    for b in range(B):
        L = int(seq_lens[b])
        if L == 0:
            continue
        g = g_of.get(b)
        P = 0 if g is None else int(prefix_lens[g])
        own = [tokens(c, block_table[b], L) for c in (k_cache, v_cache)]
        pre = [tokens(c, prefix_table[g or 0], P) for c in (k_cache, v_cache)]
        k, v = (torch.cat([a, c], 1) for a, c in zip(pre, own))
        for i in range(n):
            end = P + L - n + i + 1
            for h in range(H):
                s = scale * (k[h * kv // H, :end] @ q[b, i, h].double())
                lse[b, i, h] = torch.logsumexp(s, 0)
                w = torch.softmax(s, 0)
                out[b, i, h] = w @ v[h * kv // H, :end]
                spread[b, i, h] = w @ v[h * kv // H, :end].abs()
    return out, lse, spread


def bf16_half_ulp(x):
    """Half the spacing of bf16 values at |x|."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -126)))
    return torch.exp2(e - 8)


def e4m3_half_ulp(x):
    """Half the spacing of e4m3 values at |x| (subnormals below 2^-6)."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    return torch.exp2(e - 4)
