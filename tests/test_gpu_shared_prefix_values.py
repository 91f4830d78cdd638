"""sf_shared_prefix_attention where inputs hold NaN or a few weights carry a row (GPU)."""
import math

import pytest
import torch

from tests import layer_reference as ref
from tests.gpu_helpers import require_gpu
from tests.test_gpu_shared_prefix import check, close, make, run

pytestmark = pytest.mark.gpu


def rows_of_head(args, h):
    """The query heads of KV head h."""
    g = args[0].shape[2] // args[1].shape[1]
    return slice(h * g, (h + 1) * g)


def check_nan(args, nan):
    """Rows marked in nan [B][n][H_q] are NaN in out and lse; the others are those of the
    same inputs without NaN."""
    require_gpu()
    out, lse, status = run(args)
    assert status == 0
    out, lse = out.cpu(), lse.cpu()
    assert out[nan].isnan().all() and lse[nan].isnan().all()
    o, l, spread = ref.shared_prefix(*(a.nan_to_num() if a.is_floating_point() else a for a in args))
    close(torch.where(nan[..., None], o, out.double()), torch.where(nan, l, lse.double()), (o, l, spread))


# One own token behind a prefix of 8 to 31 key tiles: its partial stands at every place
# of a list that several threads take in batches, alone in a batch at some.
@pytest.mark.parametrize("tiles", range(8, 32))
@pytest.mark.parametrize("H_q, H_kv, d", [(1, 1, 128), (4, 2, 64), (8, 4, 128)])
def test_nan_in_the_key_of_the_only_own_token(tiles, H_q, H_kv, d):
    args = make([1], [tiles * 128], [1], 1, H_q, H_kv, d, seed=tiles, spare=tiles % 2 * 64)
    nan = torch.zeros(1, 1, H_q, dtype=torch.bool)
    args[1][args[6][0, 0], H_kv - 1, 0, 3] = math.nan
    nan[:, :, rows_of_head(args, H_kv - 1)] = True
    check_nan(args, nan)


@pytest.mark.parametrize("prefix, lens", [(0, [9, 40]), (300, [130, 20]), (5000, [8, 300])])
@pytest.mark.parametrize("H_q, H_kv, d", [(3, 3, 128), (8, 2, 64)])
def test_nan_in_q(prefix, lens, H_q, H_kv, d):
    args = make([2], [prefix], lens, 4, H_q, H_kv, d, seed=prefix + H_q)
    nan = torch.zeros(2, 4, H_q, dtype=torch.bool)
    nan[0, 1, 0] = nan[1, 3, H_q - 1] = True
    args[0][0, 1, 0, 5] = args[0][1, 3, H_q - 1, d - 1] = math.nan
    check_nan(args, nan)


@pytest.mark.parametrize("prefix, lens", [([0, 40], [9, 40, 12]), ([700, 129], [130, 20, 300]), ([3000, 0], [4, 5, 600])])
@pytest.mark.parametrize("H_q, H_kv, d", [(3, 3, 128), (8, 2, 64)])
def test_nan_in_keys_reaches_the_rows_that_see_it(prefix, lens, H_q, H_kv, d):
    # one prefix token (its whole group), a token in front of the draft rows, a draft
    # row (itself and the later ones), and every key of a whole tile
    for place in ("prefix", "own", "draft", "tile"):
        args = make([2, 1], prefix, lens, 4, H_q, H_kv, d, seed=sum(lens) + d)
        nan = torch.zeros(3, 4, H_q, dtype=torch.bool)
        h = H_kv - 1
        heads = rows_of_head(args, h)
        kc, pt, bt = args[1], args[3], args[6]
        if place == "prefix":
            if prefix[0] == 0:
                continue
            kc[pt[0, (prefix[0] - 1) // 16], h, (prefix[0] - 1) % 16, 0] = math.nan
            nan[:2, :, heads] = True
        elif place == "own":
            if lens[1] <= 4:
                continue
            kc[bt[1, 0], h, 0, d - 1] = math.nan
            nan[1, :, heads] = True
        elif place == "draft":
            at = lens[2] - 4 + 2
            kc[bt[2, at // 16], h, at % 16, 7] = math.nan
            nan[2, 2:, heads] = True
        else:
            if prefix[0] < 300:
                continue
            kc[pt[0, 8:16].long(), h] = math.nan  # the prefix's second key tile
            nan[:2, :, heads] = True
        check_nan(args, nan)


def weights(args):
    """Softmax weights in fp64: one [n][H_q][prefix + own keys] per sequence, over its prefix
    and own tokens, and their values [H_kv][keys][d]."""
    q, kc, vc, pt, pl, gs, bt, sl = args
    n, H, d = q.shape[1:]
    kv = kc.shape[1]
    for b, L in enumerate(sl.tolist()):
        g = max(i for i in range(len(gs) - 1) if int(gs[i]) <= b < int(gs[i + 1]))
        P = int(pl[g])
        k, v = (torch.cat([ref.tokens(c, pt[g], P), ref.tokens(c, bt[b], L)], 1) for c in (kc, vc))
        s = torch.einsum("nhd,hkd->nhk", q[b].double(), k.repeat_interleave(H // kv, 0)) / math.sqrt(d)
        hidden = torch.arange(P + L) > (P + L - n + torch.arange(n))[:, None]
        yield torch.softmax(s.masked_fill(hidden[:, None], -math.inf), 2), v


def attract(args, tokens, score):
    """Keys `tokens` (table row, position, whether of the prefix) get `score` more from every
    q, in natural units: q has 4 in its first column, a key what that takes."""
    q, kc, pt, bt = args[0], args[1], args[3], args[6]
    d = q.shape[3]
    q[..., 0] = 4.0
    kc[..., 0] = torch.where(kc[..., 0].isnan(), kc[..., 0], torch.zeros_like(kc[..., 0]))
    for i, (row, at, prefix) in enumerate(tokens):
        page = (pt if prefix else bt)[row, at // 16]
        kc[page, :, at % 16, 0] = (score if isinstance(score, float) else score[i]) * math.sqrt(d) / 4


# A few first keys that carry nearly all of the weight, as attention sinks do: in the
# prefix, in the own tokens where there is no prefix, and in both where it is short.
# The first 128 keys' weights come with 16 bits, so of the error only the output's own
# rounding, that of the scores (|q| . |k| below 250 products' size 1 here and the sinks'
# 20 units: 3e-4 of a weight and as much of their sum), and 2^-8 of the later keys' part
# remain.
@pytest.mark.parametrize("prefix, own, at", [(700, 40, [(0, 0, 1), (0, 1, 1), (0, 2, 1), (0, 5, 1)]),
                                             (3000, 300, [(0, 3, 1), (0, 90, 1), (0, 127, 1)]),
                                             (0, 900, [(0, 0, 0), (0, 1, 0), (0, 3, 0), (0, 100, 0)]),
                                             (50, 700, [(0, 0, 0), (0, 7, 0), (0, 20, 1), (0, 77, 0)])])
@pytest.mark.parametrize("H_q, H_kv, d", [(8, 8, 64), (28, 4, 128), (3, 3, 128)])
def test_first_keys_that_carry_the_weight(prefix, own, at, H_q, H_kv, d):
    require_gpu()
    args = make([1], [prefix], [own], 8, H_q, H_kv, d, seed=prefix + own + d)
    attract(args, at, 14.0)
    out, lse, status = run(args)
    assert status == 0
    o, l, _ = ref.shared_prefix(*args)
    (w, v), = weights(args)
    size = v.abs().repeat_interleave(H_q // H_kv, 0)
    first, later = (torch.einsum("nhk,hkd->nhd", w[..., part], size[:, part]) for part in (slice(0, 128), slice(128, None)))
    tol = ref.bf16_half_ulp(o[0]) * (1 + 2.0 ** -6) + 2 * 3e-4 * (first + later) + 2.0 ** -8 * later
    err = (out[0].double().cpu() - o[0]).abs()
    assert (err <= tol).all(), ((err > tol).sum(), (err - tol).max())
    assert (lse.double().cpu() - l).abs().max() <= 3e-3  # (scores of 14 and more: their fp32 error grows with them)


@pytest.mark.parametrize("prefix, lens", [(0, [9, 40]), (900, [130, 20])])
def test_an_infinite_score_makes_its_rows_nan(prefix, lens):
    require_gpu()
    args = make([2], [prefix], lens, 4, 4, 2, 64, seed=prefix + 3)
    args[0][..., 0] = 1.0
    args[1][args[6][0, 0], 1, 2, 0] = math.inf  # own token 2 of sequence 0: all of its rows see it
    out, lse, status = run(args)
    assert status == 0
    assert out[0, :, 2:].isnan().all() and lse[0, :, 2:].isnan().all()
    assert out[0, :, :2].isfinite().all() and out[1].isfinite().all() and lse[1].isfinite().all()


# One key of a later tile that outweighs all others, 3 to 8 base-2 units above the first
# tile's largest score, so that its weight is no power of two and its rounding (2^-8 of it)
# would be the row's.  With p_t the weights, * that key and |delta_t| <= 2^-8 the weights'
# roundings, a result that is divided by a sum with the rounding of each tile's largest
# weight in it is off by at most 2^-8 (1 + 2^-7) times
#     p_* |v_* - out| + sum over the other keys of p_t (|v_t| + |out|),
# beside the scores' 3e-4 and the output's own rounding.
@pytest.mark.parametrize("groups, prefix, own, n, H_q, H_kv, d", [
    ([1] * 16, 1024, 3, 2, 8, 8, 128), ([1] * 16, 0, 1024, 2, 8, 8, 64), ([20], 2048, 9, 8, 32, 32, 64),
    ([9, 12], 1500, 300, 4, 28, 4, 128)])
@pytest.mark.parametrize("excess", [3.4, 5.3, 7.3])
def test_one_key_that_outweighs_all_others(groups, prefix, own, n, H_q, H_kv, d, excess):
    require_gpu()
    B = sum(groups)
    args = make(groups, [prefix] * len(groups), [own] * B, n, H_q, H_kv, d, seed=int(10 * excess) + d, q_scale=0.1)
    at, score = [], []
    for i in range(len(groups) if prefix else B):
        later = 130 + (i * 97) % ((prefix or own) - 140)
        at += [(i, 5, prefix > 0), (i, later, prefix > 0)]
        score += [12.0, 12.0 + excess * math.log(2)]
    attract(args, at, score)
    out, lse, status = run(args)
    assert status == 0
    out, lse = out.double().cpu(), lse.double().cpu()
    for b, (w, v) in enumerate(weights(args)):
        v = v.repeat_interleave(H_q // H_kv, 0)
        o = torch.einsum("nhk,hkd->nhd", w, v)
        size = torch.einsum("nhk,hkd->nhd", w, v.abs())
        top, key = w.max(2)
        assert (top > 0.85).all()
        mine = v.gather(1, key.t()[..., None].expand(-1, -1, d)).transpose(0, 1)
        p = top[..., None]
        rest = p * (mine - o).abs() + (size - p * mine.abs()) + (1 - p) * o.abs()
        tol = ref.bf16_half_ulp(o) * (1 + 2.0 ** -6) + 2 * 3e-4 * size + 2.0 ** -8 * (1 + 2.0 ** -7) * rest
        err = (out[b] - o).abs()
        assert (err <= tol).all(), ((err > tol).sum(), (err - tol).max())


# 128-wide heads with batches whose plan leaves four ring slots (88 sequences of one
# group and more), beside the largest that leave five
@pytest.mark.parametrize("groups", [[87], [88], [40, 60], [1] * 19, [1] * 18, [3, 297]])
def test_batches_on_both_sides_of_the_ring(groups):
    check(groups, [(171 * (g + 2)) % 700 for g in range(len(groups))], [3 + (53 * b) % 290 for b in range(sum(groups))], 3, 4, 2,
          128, seed=len(groups) + sum(groups))
