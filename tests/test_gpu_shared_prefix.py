"""sf_shared_prefix_attention against the 64-bit softmax over all visible tokens (GPU).

Tolerances.  The weights are rounded to bf16 (2^-9 relative) before they are
multiplied with V; the fp32 scores of |q| . |k| ~ d products are off by at most
d * 2^-24 * sum |q_e k_e| * scale < 2e-4 for the N(0, 1) inputs used here, which a
weight and the LSE inherit, and exp2 is within 2^-21.  So |out - exact| <= (2^-9 +
2^-11) * sum_t p_t |v_t| + half a bf16 ulp of the output, and |lse - exact| <= 3e-4."""
import math

import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import layer_reference as ref
from tests.gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu


def make(groups, prefix, lens, n, H_q, H_kv, d, seed, spare=0, q_scale=1.0):
    """groups: sequences per group.  Caches over a permuted pool; tails of the
    pages past every length, and the spare pages, hold NaN."""
    g = torch.Generator().manual_seed(seed)
    B = sum(groups)
    pp, op = [-(-x // 16) for x in prefix], [-(-x // 16) for x in lens]
    pool = sum(pp) + sum(op) + 2
    ids = torch.randperm(pool, generator=g).int()
    pt = torch.full((len(groups), max(1, max(pp)) + spare), -1, dtype=torch.int32)
    bt = torch.full((B, max(1, max(op)) + spare), -1, dtype=torch.int32)
    kc, vc = torch.randn(2, pool, H_kv, 16, d, generator=g).bfloat16()
    at = 0
    for table, counts, sizes in ((pt, pp, prefix), (bt, op, lens)):
        for r, (c, size) in enumerate(zip(counts, sizes)):
            table[r, :c] = ids[at:at + c]
            at += c
            if size % 16:
                kc[table[r, c - 1], :, size % 16:] = math.nan
                vc[table[r, c - 1], :, size % 16:] = math.nan
    kc[ids[at:].long()] = math.nan
    vc[ids[at:].long()] = math.nan
    q = (q_scale * torch.randn(B, n, H_q, d, generator=g)).bfloat16()
    starts = [0]
    for m in groups:
        starts.append(starts[-1] + m)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return [q, kc, vc, pt, i32(prefix), i32(starts), bt, i32(lens)]


def run(args, **kw):
    ws = sfv.new_workspace(sfv.shared_prefix_attention_workspace_size(
        *args[0].shape[:3], args[1].shape[1], args[0].shape[3], args[3].shape[0], args[3].shape[1], args[6].shape[1]))
    out, lse = sfv.shared_prefix_attention(*(a.cuda() for a in args), workspace=ws, **kw)
    return out, lse, sfv.read_device_status(ws)


def close(out, lse, want, lse_atol=3e-4):
    o, l, spread = want
    out, lse = out.double().cpu(), lse.double().cpu()
    tol = ref.bf16_half_ulp(o) * (1 + 2.0 ** -6) + spread * (2.0 ** -9 + 2.0 ** -11)
    err = (out - o).abs()
    assert (err <= tol).all(), ((err - tol).max(), (err > tol).sum())
    idle = torch.isinf(l)
    assert torch.equal(lse[idle], l[idle])
    assert (lse - l)[~idle].abs().max() <= lse_atol if (~idle).any() else True


def check(*a, **kw):
    require_gpu()
    scale = kw.pop("softmax_scale", 0.0)
    args = make(*a, **kw)
    out, lse, status = run(args, softmax_scale=scale)
    assert status == 0
    close(out, lse, ref.shared_prefix(*args, scale=scale or None))


HEADS = [(8, 8, 64), (28, 4, 128), (4, 4, 128), (8, 1, 64), (6, 2, 128), (5, 1, 128)]


@pytest.mark.parametrize("H_q, H_kv, d", HEADS)
@pytest.mark.parametrize("n", [1, 5, 8, 16])
def test_head_layouts_and_draft_lengths(H_q, H_kv, d, n):
    check([2, 1], [200, 77], [n, n + 40, 130 + n], n, H_q, H_kv, d, seed=n * 1000 + d)


# prefix lengths around pages, 64- and 128-key tiles; own lengths likewise
@pytest.mark.parametrize("P", [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 300])
@pytest.mark.parametrize("L", [3, 16, 64, 65, 127, 129, 260])
def test_lengths_around_pages_and_tiles(P, L):
    check([2], [P], [L, 3], 3, 4, 2, 64, seed=1000 * P + L)
    check([1], [P], [L], 3, 2, 1, 128, seed=1000 * P + L + 1)


@pytest.mark.parametrize("groups", [[1], [1, 1, 1], [5], [0, 3, 0, 2], [17, 1], [0, 0, 4], [40], [3, 33, 20]])
def test_groups(groups):
    prefix = [(90 * (g + 1)) % 401 for g in range(len(groups))]
    B = sum(groups)
    while len(groups) > B:
        groups = groups[:-1]
    check(groups, prefix[:len(groups)], [8 + (37 * b) % 90 for b in range(B)], 8, 7, 1, 128, seed=sum(groups))


def test_idle_slots():
    check([3, 2, 1], [50, 0, 130], [0, 9, 40, 0, 5, 0], 4, 4, 2, 64, seed=5)
    check([2], [50], [0, 0], 4, 4, 2, 64, seed=6)


def test_long_prefix_in_many_pieces():
    check([2], [5000], [30, 100], 2, 4, 2, 128, seed=7)
    check([3], [70], [3000, 2, 900], 2, 4, 2, 64, seed=8)


def test_many_sequences():
    n = [1, 60, 2, 137]
    check(n, [300, 40, 0, 129], [2 + (31 * b) % 70 for b in range(200)], 2, 2, 1, 64, seed=9)


def test_more_groups_and_sequences_than_threads():
    check([1] * 600 + [400], [(7 * g) % 40 for g in range(601)], [1 + b % 20 for b in range(1000)], 1, 1, 1, 64, seed=10)


def test_sharp_scores_and_scale():
    check([3], [400], [20, 30, 300], 4, 4, 2, 64, seed=11, softmax_scale=0.5)
    # growing scores: the running maximum moves at every tile
    args = make([2], [700], [200, 40], 4, 4, 2, 64, seed=12)
    for table, lens in ((args[3], [700, ]), (args[6], [200, 40])):
        for r, size in enumerate(lens):
            for t in range(size):
                page = int(table[r, t // 16])
                args[1][page, :, t % 16] = (args[0][0, 0, 0].float() * (t / 200)).bfloat16()
    require_gpu()
    out, lse, status = run(args)
    assert status == 0
    # scores reach 60: their fp32 error grows with them (64 products of up to 60 / 64)
    close(out, lse, ref.shared_prefix(*args), lse_atol=3e-3)


def test_without_lse_and_with_default_workspace():
    require_gpu()
    args = [a.cuda() for a in make([2, 2], [100, 30], [9, 20, 33, 4], 4, 4, 2, 64, seed=13)]
    out, lse, _ = run(args)
    o2, none = sfv.shared_prefix_attention(*args, with_lse=False)
    assert none is None and torch.equal(out, o2)


def test_calls_in_a_row_and_repeats_are_bit_identical():
    # one workspace for shapes that grow and shrink, then each again
    require_gpu()
    sets = [[a.cuda() for a in make([3, 1], [900, 30], [9, 20, 33, 400], 4, 8, 2, 128, seed=14)],
            [a.cuda() for a in make([1], [3], [5], 5, 8, 2, 128, seed=15)],
            [a.cuda() for a in make([20], [2000], list(range(8, 28)), 8, 8, 2, 128, seed=16)]]
    size = max(sfv.shared_prefix_attention_workspace_size(*a[0].shape[:3], a[1].shape[1], a[0].shape[3], a[3].shape[0],
                                                          a[3].shape[1], a[6].shape[1]) for a in sets)
    ws = sfv.new_workspace(size)
    first = [sfv.shared_prefix_attention(*a, workspace=ws) for a in sets]
    for _ in range(3):
        for a, (o, l) in zip(sets, first):
            o2, l2 = sfv.shared_prefix_attention(*a, workspace=ws)
            assert torch.equal(o, o2) and torch.equal(l, l2)
    assert sfv.read_device_status(ws) == 0
    for a, (o, l) in zip(sets, first):
        close(o, l, ref.shared_prefix(*(t.cpu() for t in a)))


def test_many_calls_close_behind_each_other():
    # pieces of one and two row tiles, of one key tile and of many, in turn: the
    # streams of a CTA run ahead of each other by amounts that vary from call to call
    require_gpu()
    sets = [[a.cuda() for a in make([9, 3, 15, 5], [4800, 700, 4100, 130], [8 + (67 * b) % 500 for b in range(32)], 8, 28, 4,
                                    128, seed=30)],
            [a.cuda() for a in make([2, 1, 4, 1], [900, 40, 0, 3000], [2 + (91 * b) % 300 for b in range(8)], 2, 8, 8, 64,
                                    seed=31)]]
    first = [sfv.shared_prefix_attention(*a) for a in sets]
    ws = [sfv.new_workspace(sfv.shared_prefix_attention_workspace_size(
        *a[0].shape[:3], a[1].shape[1], a[0].shape[3], a[3].shape[0], a[3].shape[1], a[6].shape[1])) for a in sets]
    outs = [[torch.empty_like(o), torch.empty_like(l)] for o, l in first]
    for a, w, (o, l) in zip(sets, ws, outs):
        for _ in range(400):
            sfv.shared_prefix_attention(*a, out=o, lse=l, workspace=w)
    for _ in range(400):
        for a, w, (o, l) in zip(sets, ws, outs):
            sfv.shared_prefix_attention(*a, out=o, lse=l, workspace=w)
    for (o, l), (o2, l2), w in zip(first, outs, ws):
        assert sfv.read_device_status(w) == 0
        assert torch.equal(o, o2) and torch.equal(l, l2)
    close(*first[1], ref.shared_prefix(*(t.cpu() for t in sets[1])))


def test_agrees_with_verify_attention_where_nothing_is_shared():
    require_gpu()
    args = make([1, 1, 1], [0, 0, 0], [70, 500, 8], 8, 28, 4, 128, seed=17)
    out, lse, _ = run(args)
    q, kc, vc, _, _, _, bt, sl = (a.cuda() for a in args)
    kc, vc = kc.nan_to_num(), vc.nan_to_num()
    o2, l2 = sfv.verify_attention(q, kc, vc, bt, sl)
    assert (out.float() - o2.float()).abs().max() <= 2e-2 and (lse - l2).abs().max() <= 1e-3


def test_device_data_errors_are_flagged():
    require_gpu()
    base = make([2, 1], [100, 40], [20, 50, 30], 4, 4, 2, 64, seed=18, spare=1)

    def call(**kw):
        args = [a.clone() for a in base]
        for name, f in kw.items():
            f(args[["q", "k", "v", "pt", "pl", "gs", "bt", "sl"].index(name)])
        return args, run(args)

    def put(at, value):
        def f(t):
            t[at] = value
        return f

    # a page outside the pool reads as zeros
    for value in (-7, 10 ** 6, 2 ** 31 - 1):
        args, (out, lse, status) = call(pt=put((0, 2), value))
        assert status == sfv.SF_DEVICE_BAD_PAGE
        close(out, lse, ref.shared_prefix(*args))
        args, (out, lse, status) = call(bt=put((1, 0), value))
        assert status == sfv.SF_DEVICE_BAD_PAGE
        close(out, lse, ref.shared_prefix(*args))
    # lengths are clamped (short ones to n_q, long ones to the table, whose pages are -1 there)
    args, (out, lse, status) = call(sl=put(0, 3))
    assert status == sfv.SF_DEVICE_BAD_SEQLEN
    args[7][0] = 4
    close(out, lse, ref.shared_prefix(*args))
    args, (out, lse, status) = call(sl=put(1, -9))
    assert status == sfv.SF_DEVICE_BAD_SEQLEN
    args, (out, lse, status) = call(pl=put(1, -1))
    assert status == sfv.SF_DEVICE_BAD_SEQLEN
    args[4][1] = 0
    close(out, lse, ref.shared_prefix(*args))
    _, (_, _, status) = call(pl=put(0, 10 ** 9), sl=put(2, 2 ** 31 - 1))
    assert status == sfv.SF_DEVICE_BAD_SEQLEN | sfv.SF_DEVICE_BAD_PAGE
    # malformed groups: no sequence has a prefix
    for at, value in ((0, 1), (2, 2), (1, -1), (1, 4), (2, 2 ** 31 - 1), (0, -(2 ** 31))):
        args, (out, lse, status) = call(gs=put(at, value))
        assert status == sfv.SF_DEVICE_BAD_INDEX
        args[5] = [0, 0, 0]
        close(out, lse, ref.shared_prefix(*args))


def test_append_then_attention_back_to_back():
    # the append of a prompt and of draft rows directly in front of the attention
    require_gpu()
    B, n, H_q, H_kv, d, P = 3, 4, 8, 2, 128, 333
    g = torch.Generator().manual_seed(19)
    args = make([3], [P], [n, n + 30, n + 77], n, H_q, H_kv, d, seed=20)
    prompt = torch.randn(2, P, H_kv, d, generator=g).bfloat16()
    pos = torch.arange(P, dtype=torch.int32)[None]
    f = 10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))
    q, kc, vc, pt, pl, gs, bt, sl = (a.cuda() for a in args)
    f, prompt, pos = f.cuda(), prompt.cuda(), pos.cuda()
    rows = torch.randn(3, B * n, H_q, d, generator=g).bfloat16().cuda()
    rpos = (P + torch.arange(B * n, dtype=torch.int32))[None].cuda()
    ws = sfv.new_workspace(sfv.kv_append_workspace_size())
    sfv.kv_append(None, prompt[0], prompt[1], pos, f, kc, vc, pt, pl, workspace=ws)
    rq = sfv.kv_append(rows[0], rows[1][:, :H_kv], rows[2][:, :H_kv], rpos, f, kc, vc, bt, sl, workspace=ws)
    out, lse = sfv.shared_prefix_attention(rq.view(B, n, H_q, d), kc, vc, pt, pl, gs, bt, sl)
    assert sfv.read_device_status(ws) == 0
    close(out, lse, ref.shared_prefix(rq.view(B, n, H_q, d).cpu(), kc.cpu(), vc.cpu(), *args[3:]))


def test_refusals():
    require_gpu()
    args = [a.cuda() for a in make([2], [40], [9, 20], 4, 4, 2, 64, seed=21)]

    def call(**kw):
        a = dict(zip(["q", "k", "v", "pt", "pl", "gs", "bt", "sl"], args)) | kw
        return sfv.shared_prefix_attention(*a.values())

    with pytest.raises(TypeError, match="q must be"):
        call(q=args[0].float())
    with pytest.raises(ValueError, match="v_cache has shape"):
        call(v=args[2][:1].contiguous())
    with pytest.raises(ValueError, match="prefix_lens has shape"):
        call(pl=args[7])
    with pytest.raises(ValueError, match="group_starts has shape"):
        call(gs=args[7][:1])
    with pytest.raises(ValueError, match="block_table has shape"):
        call(bt=args[6][:1])
    with pytest.raises(TypeError, match="seq_lens must be"):
        call(sl=args[7].long())
    with pytest.raises(ValueError, match="contiguous"):
        call(q=args[0].transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(sfv.SFError) as e:
        sfv.shared_prefix_attention(*args, workspace=sfv.new_workspace(128))
    assert e.value.status == 4
    with pytest.raises(sfv.SFError, match="softmax_scale"):
        sfv.shared_prefix_attention(*args, softmax_scale=-1.0)


# few rows, long parts: many partials a row (lists over several threads), an odd and a
# single KV head among them, the long part shared or a sequence's own
@pytest.mark.parametrize("prefix, own, n, H_q, H_kv, d", [
    (9000, 15, 6, 16, 4, 64), (6100, 9, 1, 3, 3, 128), (5003, 20, 3, 8, 1, 128), (70, 6007, 4, 6, 2, 64), (0, 7011, 16, 5, 5, 128)])
def test_many_partials_a_row(prefix, own, n, H_q, H_kv, d):
    check([1], [prefix], [own], n, H_q, H_kv, d, seed=prefix + own)
    check([2], [prefix], [own, 0], n, H_q, H_kv, d, seed=prefix + own + 1)


# own tokens of two KV heads side by side: one, two and many key tiles, with an odd
# number of heads, cut between and inside the pairs
@pytest.mark.parametrize("H_q, H_kv, d", [(3, 3, 128), (2, 2, 64), (10, 5, 64), (7, 1, 128), (32, 32, 64)])
@pytest.mark.parametrize("lens", [[128, 140], [129, 1, 300], [127, 640, 16, 255, 1000, 17]])
def test_own_tokens_of_pairs_of_heads(H_q, H_kv, d, lens):
    check([len(lens)], [0], lens, 1, H_q, H_kv, d, seed=sum(lens))
    check([1, len(lens) - 1], [40, 260], [x + 3 for x in lens], 4, H_q, H_kv, d, seed=sum(lens) + 1)


# NaN and infinities in V of a draft token reach its own row and the later ones, in
# their columns: one key tile and several, drafts across the line between two tiles, an
# odd head, two-term weights, pieces of one and of two heads
@pytest.mark.parametrize("H_q, H_kv, d", [(3, 3, 128), (8, 2, 64), (7, 1, 128), (16, 8, 64)])
@pytest.mark.parametrize("prefix, lens, n", [
    (0, [9, 40], 8), (300, [130, 128, 131], 8), (40, [1000, 16, 257], 16), (500, [263, 640], 4), (0, [2000], 3)])
def test_draft_values_reach_the_rows_that_see_them(prefix, lens, n, H_q, H_kv, d):
    require_gpu()
    args = make([len(lens)], [prefix], lens, n, H_q, H_kv, d, seed=prefix + sum(lens) + d)
    vc, bt = args[2], args[6]
    bad = vc.clone()
    nan = torch.zeros(len(lens), n, H_q, d, dtype=torch.bool)
    up, down = nan.clone(), nan.clone()
    g = H_q // H_kv
    for b, size in enumerate(lens):
        for j, marks in ((1, [(nan, 3, math.nan), (up, 5, math.inf)]), (n - 1, [(down, d - 1, -math.inf), (down, 5, -math.inf)])):
            pos = size - n + j
            for h in range(b % 2, H_kv, 2):  # every other head
                for mask, col, value in marks:
                    bad[bt[b, pos // 16], h, pos % 16, col] = value
                    vc[bt[b, pos // 16], h, pos % 16, col] = 0.0
                    mask[b, j:, h * g:(h + 1) * g, col] = True
    want = ref.shared_prefix(*args)  # what the rows before see, and the other columns
    args[2] = bad
    out, lse, status = run(args)
    assert status == 0
    out = out.cpu()
    nan |= up & down  # inf - inf
    assert out[nan].isnan().all()
    assert (out[up & ~nan] == math.inf).all() and (out[down & ~nan] == -math.inf).all()
    seen = nan | up | down
    o, l, spread = want
    out = torch.where(seen, o, out.double())
    close(out, lse, want)
