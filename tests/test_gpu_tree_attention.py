"""sf_tree_attention against the 64-bit softmax over the keys that a row sees (GPU).

Tolerances.  Each weight is rounded to bf16 for its product with V, off by at most
2^-8 of itself (half a step of bf16); the fp32 scores, sums of d products, are off by
at most d 2^-23 sum |q_e k_e| scale, below 2^-12 for the N(0, 1) inputs used here (d =
128, sum |q_e k_e| scale below 16), which the weights and the LSE inherit; exp2 adds
2^-21.  So |out - exact| <= (2^-8 + 2^-11) sum_t p_t |v_t| + half a bf16 step of the
output, and |lse - exact| <= 2^-11."""
import math

import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import layer_reference, tree_reference as ref
from tests.gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu


def random_tree(n, g, width=4):
    return [-1] + [int(torch.randint(max(0, i - width), i, (1,), generator=g)) for i in range(1, n)]


def make(before, n, H_q, H_kv, d, seed, masks=None, q_scale=1.0, spare=0):
    """before: the contexts' lengths (None: an idle slot).  Caches over a permuted pool;
    the tails of the pages past every length, and the spare pages, hold NaN."""
    g = torch.Generator().manual_seed(seed)
    lens = [0 if x is None else x + n for x in before]
    pages = [-(-x // 16) for x in lens]
    pool = sum(pages) + 2
    ids = torch.randperm(pool, generator=g).int()
    bt = torch.full((len(lens), max(1, max(pages)) + spare), -1, dtype=torch.int32)
    kc, vc = torch.randn(2, pool, H_kv, 16, d, generator=g).bfloat16()
    at = 0
    for r, (c, size) in enumerate(zip(pages, lens)):
        bt[r, :c] = ids[at:at + c]
        at += c
        if size % 16:
            kc[bt[r, c - 1], :, size % 16:] = math.nan
            vc[bt[r, c - 1], :, size % 16:] = math.nan
    kc[ids[at:].long()] = math.nan
    vc[ids[at:].long()] = math.nan
    q = (q_scale * torch.randn(len(lens), n, H_q, d, generator=g)).bfloat16()
    if masks is None:
        masks = [ref.masks(random_tree(n, g)) for _ in lens]
    words = torch.tensor([[ref.signed(w) for w in row] for row in masks], dtype=torch.int64)
    return [q, kc, vc, bt, torch.tensor(lens, dtype=torch.int32), words], masks


def run(args, **kw):
    q, kc, _, bt = args[:4]
    ws = sfv.new_workspace(sfv.tree_attention_workspace_size(*q.shape[:3], kc.shape[1], q.shape[3], bt.shape[1]))
    out, lse = sfv.tree_attention(*(a.cuda() for a in args), workspace=ws, **kw)
    return out, lse, sfv.read_device_status(ws)


def close(out, lse, want, lse_atol=2.0 ** -11):
    o, l, spread = want
    out, lse = out.double().cpu(), lse.double().cpu()
    tol = layer_reference.bf16_half_ulp(o) * (1 + 2.0 ** -6) + spread * (2.0 ** -8 + 2.0 ** -11)
    err = (out - o).abs()
    assert (err <= tol).all(), ((err - tol).max(), (err > tol).sum())
    none = torch.isinf(l)
    assert torch.equal(lse[none], l[none])
    assert not out[none].any()
    assert (lse - l)[~none].abs().max() <= lse_atol if (~none).any() else True


def check(*a, **kw):
    require_gpu()
    scale = kw.pop("softmax_scale", 0.0)
    args, masks = make(*a, **kw)
    out, lse, status = run(args, softmax_scale=scale)
    assert status == 0
    close(out, lse, ref.attention(*args[:5], masks, scale=scale or None))


HEADS = [(8, 8, 64), (28, 4, 128), (4, 4, 128), (8, 1, 64), (6, 2, 128), (5, 1, 128), (3, 3, 64), (9, 3, 128), (8, 1, 128)]


@pytest.mark.parametrize("H_q, H_kv, d", HEADS)
@pytest.mark.parametrize("n", [1, 2, 15, 17, 26, 33, 64])
def test_head_layouts_and_tree_sizes(H_q, H_kv, d, n):
    check([0, 40, 130], n, H_q, H_kv, d, seed=n * 1000 + d)


# context lengths around pages and 128-key tiles, so that the tree's rows begin, end
# and lie across them
@pytest.mark.parametrize("before", [0, 1, 15, 16, 17, 63, 64, 65, 100, 111, 112, 113, 127, 128, 129, 240, 255, 256, 300])
@pytest.mark.parametrize("n", [1, 5, 16, 40])
def test_lengths_around_pages_and_tiles(before, n):
    check([before], n, 4, 2, 64, seed=100 * before + n)
    check([before, 3], n, 2, 1, 128, seed=100 * before + n + 1)


def test_idle_slots_and_many_sequences():
    check([None, 50, None, 0, 130, None], 7, 4, 2, 64, seed=5)
    check([None, None], 3, 4, 2, 64, seed=6)
    check([(31 * b) % 170 if b % 7 else None for b in range(150)], 3, 2, 1, 64, seed=7)
    check([(7 * b) % 33 for b in range(1024)], 1, 1, 1, 64, seed=8)


def test_more_heads_than_ctas_and_more_sequences_than_lanes():
    # pairs of heads (an odd number of them too) once every SM has a head; plans of more
    # than 32 sequences; up to four row tiles a head
    check([(37 * b) % 150 if b % 11 else None for b in range(60)], 6, 3, 3, 64, seed=70)
    check([(53 * b) % 300 for b in range(100)], 9, 4, 2, 128, seed=71)
    check([(29 * b) % 200 for b in range(40)], 20, 14, 2, 128, seed=72)
    check([(29 * b) % 140 for b in range(33)], 64, 8, 1, 64, seed=73)
    check([500, 3, 200], 40, 7, 1, 128, seed=74)
    check([(31 * b) % 90 for b in range(32)], 50, 8, 2, 64, seed=75)


def test_long_contexts_in_many_pieces():
    check([5000], 20, 4, 2, 128, seed=9)
    check([3000, 70, 1200], 30, 7, 1, 128, seed=10)
    check([9000], 2, 2, 1, 64, seed=11)


def test_masks_that_are_no_trees():
    n = 40
    g = torch.Generator().manual_seed(12)
    wild = [[int(torch.randint(0, 1 << 40, (1,), generator=g)) for _ in range(n)] for _ in range(3)]
    wild[0] = [0] * n                                    # nobody sees a new row
    wild[1] = [(1 << 64) - 1] * n                        # everybody sees all, and bits that mean nothing
    for before in (0, 1, 90):
        args, masks = make([before] * 3, n, 7, 1, 128, seed=13, masks=wild)
        require_gpu()
        out, lse, status = run(args)
        assert status == 0
        close(out, lse, ref.attention(*args[:5], [[w & (1 << n) - 1 for w in r] for r in masks]))


def test_rows_that_see_nothing():
    n = 6
    masks = [[0, 0b10, 0, 0b1000, 0b11000, 0], [0] * n]
    check([0, 0], n, 8, 2, 64, seed=14, masks=masks)
    check([0, 5], 6, 28, 4, 128, seed=15, masks=masks)


def test_one_tree_for_all_sequences_and_strided_masks():
    require_gpu()
    args, masks = make([40, 3, 200], 12, 6, 2, 128, seed=16)
    masks = [masks[0]] * 3
    want = ref.attention(*args[:5], masks)
    q, kc, vc, bt, sl, words = (a.cuda() for a in args)
    row = words[0].contiguous()
    for m in (row, row.expand(3, 12), torch.cat([row.expand(3, 12), words], 1)[:, :12]):
        out, lse = sfv.tree_attention(q, kc, vc, bt, sl, m)
        close(out, lse, want)


def test_chain_masks_agree_with_verify_attention():
    require_gpu()
    n = 8
    args, masks = make([70, 500, 8], n, 28, 4, 128, seed=17, masks=[[(2 << i) - 1 for i in range(n)]] * 3)
    out, lse, _ = run(args)
    q, kc, vc, bt, sl, _ = (a.cuda() for a in args)
    o2, l2 = sfv.verify_attention(q, kc.nan_to_num(), vc.nan_to_num(), bt, sl)
    assert (out.float() - o2.float()).abs().max() <= 2e-2 and (lse - l2).abs().max() <= 1e-3


def test_sharp_scores_and_scale():
    check([400, 30], 9, 4, 2, 64, seed=18, softmax_scale=0.5)
    # growing scores: the running maximum moves at every tile
    args, masks = make([700, 40], 4, 4, 2, 64, seed=19)
    for r, size in enumerate((704, 44)):
        for t in range(size):
            args[1][int(args[3][r, t // 16]), :, t % 16] = (args[0][0, 0, 0].float() * (t / 200)).bfloat16()
    require_gpu()
    out, lse, status = run(args)
    assert status == 0
    # |k| grows to 3.5 |q|: scores off by 64 2^-23 sum |q_e k_e| / 8 <= 64 2^-23 64 3.5 / 8 16 = 0.0034
    close(out, lse, ref.attention(*args[:5], masks), lse_atol=4e-3)


def test_a_late_key_that_outweighs_all_others():
    require_gpu()
    args, masks = make([700], 20, 4, 2, 128, seed=20)
    for h in range(2):
        page, slot = ref.place(args[3][0], 600)
        args[1][page, h, slot] = 2 * args[0][0, 3, 2 * h]
    out, lse, status = run(args)
    assert status == 0
    # |k| is 2 |q|: sum |q_e k_e| scale <= 2 |q|^2 scale < 32, twice the header's
    close(out, lse, ref.attention(*args[:5], masks), lse_atol=2.0 ** -10)


def test_infinities_and_nan_of_new_rows_reach_only_the_rows_that_see_them():
    require_gpu()
    for H_q, H_kv, d, n, spare in ((8, 8, 64, 20, 0), (28, 4, 128, 30, 0), (3, 3, 128, 7, 0), (8, 1, 64, 60, 0), (2, 2, 64, 9, 100)):
        for before in (0, 100, 250):
            args, masks = make([before, before + 9] + [4] * spare, n, H_q, H_kv, d, seed=21 + before)
            words = [[w | 1 << i for i, w in enumerate(row)] for row in masks]
            clean = ref.attention(*args[:5], words)
            bad = (n - 2, n // 2)
            for c, row in zip((1, 2), bad):
                for b in range(2):
                    page, slot = ref.place(args[3][b], before + 9 * b + row)
                    args[c][page, :, slot, 5] = math.nan if c == 1 else math.inf
            out, lse, status = run(args)
            assert status == 0
            out, lse = out.cpu(), lse.cpu()
            for b in range(2):
                for i in range(n):
                    hit = [bool(words[b][i] >> row & 1) for row in bad]
                    part = [x[b:b + 1, i:i + 1] for x in clean]
                    if not any(hit):
                        close(out[b:b + 1, i:i + 1], lse[b:b + 1, i:i + 1], part)
                    elif hit[0]:
                        assert out[b, i].isnan().all() and lse[b, i].isnan().all()
                    else:  # V alone: its column (an infinity under a weight of two terms is NaN)
                        assert not out[b, i, :, 5].isfinite().any()
                        out[b, i, :, 5] = part[0][0, 0, :, 5].to(out.dtype)
                        close(out[b:b + 1, i:i + 1], lse[b:b + 1, i:i + 1], part)


# more segments than CTAs: most lie in one piece; pairs of heads (the last alone), one row
# tile, two, three and four
@pytest.mark.parametrize("H_q, H_kv, d, n, B", [(3, 3, 64, 9, 90), (4, 2, 64, 5, 100), (2, 1, 128, 12, 170), (8, 1, 128, 20, 90),
                                                (8, 1, 64, 40, 90), (8, 1, 64, 60, 90)])
def test_segments_of_one_piece(H_q, H_kv, d, n, B):
    require_gpu()
    before = [None if b % 13 == 5 else 0 if b % 5 == 1 else (37 * b) % 170 for b in range(B)]
    g = torch.Generator().manual_seed(76)
    masks = [ref.masks(random_tree(n, g)) for _ in before]
    for b in range(0, B, 4):
        masks[b][n // 3] = 0
    args, _ = make(before, n, H_q, H_kv, d, seed=77, masks=masks)
    clean = ref.attention(*args[:5], masks)
    out, lse, status = run(args)
    assert status == 0
    close(out, lse, clean)
    for c, row in ((1, n - 2), (2, n // 2)):
        for b in range(0, B, 3):
            if before[b] is not None:
                page, slot = ref.place(args[3][b], before[b] + row)
                args[c][page, :, slot, 5] = math.nan if c == 1 else -math.inf
    out, lse, status = run(args)
    assert status == 0
    out, lse = out.cpu(), lse.cpu()
    for b in range(0, B, 3):
        for i in range(n) if before[b] is not None else ():
            if masks[b][i] >> n - 2 & 1:
                assert out[b, i].isnan().all() and lse[b, i].isnan().all()
                out[b, i], lse[b, i] = clean[0][b, i].to(out.dtype), clean[1][b, i].to(lse.dtype)
            elif masks[b][i] >> n // 2 & 1:
                assert not out[b, i, :, 5].isfinite().any()
                out[b, i, :, 5] = clean[0][b, i, :, 5].to(out.dtype)
    close(out, lse, clean)


def test_infinities_and_nan_of_the_context_reach_all_rows():
    require_gpu()
    args, masks = make([300], 10, 6, 2, 64, seed=22)
    page, slot = ref.place(args[3][0], 40)
    args[2][page, 1, slot, 7] = math.nan
    out, lse, _ = run(args)
    assert out[0, :, 3:, 7].isnan().all() and out[0, :, :3].isfinite().all() and lse.isfinite().all()
    args[1][page, 0, slot, 7] = math.nan
    out, lse, _ = run(args)
    assert out[0, :, :3].isnan().all() and lse[0, :, :3].isnan().all() and lse[0, :, 3:].isfinite().all()


def test_device_data_errors_are_flagged():
    require_gpu()
    args, masks = make([100, 40], 9, 4, 2, 64, seed=23, spare=1)
    bad = [a.clone() for a in args]
    bad[3][0, 2], bad[3][1, 0] = -5, 1 << 20
    out, lse, status = run(bad)
    assert status == sfv.SF_DEVICE_BAD_PAGE
    close(out, lse, ref.attention(*bad[:5], masks))
    for value, clamped in ((5, 9), (1 << 20, 16 * args[3].shape[1]), (-3, 9)):
        bad = [a.clone() for a in args]
        bad[3][1] = bad[3][0]
        bad[3][:, -1] = bad[3][0, 0]
        bad[1], bad[2] = bad[1].nan_to_num(0.5), bad[2].nan_to_num(0.5)
        bad[4][1] = value
        out, lse, status = run(bad)
        assert status == sfv.SF_DEVICE_BAD_SEQLEN
        bad[4][1] = clamped
        close(out, lse, ref.attention(*bad[:5], masks))


def test_calls_in_a_row_are_bit_identical_without_lse_and_with_a_default_workspace():
    require_gpu()
    sets = [[a.cuda() for a in make(*s)[0]] for s in (
        ([900, 3, None, 400], 30, 8, 2, 128, 24), ([5], 3, 8, 2, 128, 25), ([2000] * 6, 64, 28, 4, 128, 26),
        ([700] * 3, 8, 16, 16, 64, 27))]
    size = max(sfv.tree_attention_workspace_size(*a[0].shape[:3], a[1].shape[1], a[0].shape[3], a[3].shape[1]) for a in sets)
    ws = sfv.new_workspace(size)
    first = [sfv.tree_attention(*a) for a in sets]
    for _ in range(30):
        for a, (o, l) in zip(sets, first):
            o2, l2 = sfv.tree_attention(*a, workspace=ws)
            assert torch.equal(o, o2) and torch.equal(l, l2)
    assert sfv.read_device_status(ws) == 0
    o2, none = sfv.tree_attention(*sets[0], with_lse=False)
    assert none is None and torch.equal(o2, first[0][0])


def test_captured_and_replayed_and_on_another_stream():
    require_gpu()
    args, masks = make([300, 20], 12, 8, 2, 64, seed=28)
    q, kc, vc, bt, sl, words = (a.cuda() for a in args)
    want = sfv.tree_attention(q, kc, vc, bt, sl, words)
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    ws = sfv.new_workspace(sfv.tree_attention_workspace_size(2, 12, 8, 2, 64, bt.shape[1]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sfv.tree_attention(q, kc, vc, bt, sl, words, out=out, lse=lse, workspace=ws)
    out.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    words.copy_(torch.ones_like(words))  # what a replay reads is what is there then
    graph.replay()
    o2, l2 = sfv.tree_attention(q, kc, vc, bt, sl, words)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    o3, l3 = sfv.tree_attention(q, kc, vc, bt, sl, words, stream=side)
    side.synchronize()
    assert torch.equal(o3, o2) and torch.equal(l3, l2)
