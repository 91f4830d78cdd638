"""sf_attention_mass and sf_kv_evict against 64 bits and plain Python (GPU).  The bound
of a mass is that of fp32 scores and sums (tests/tree_reference.py); what is evicted,
kept and moved has to be equal."""
import math

import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import tree_reference as ref
from tests.gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu

i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731


def pages_of(lens, g, spare=0):
    pages = [-(-x // 16) for x in lens]
    pool = sum(pages) + 2
    ids = torch.randperm(pool, generator=g).int()
    bt = torch.full((len(lens), max(1, max(pages)) + spare), -1, dtype=torch.int32)
    at = 0
    for r, c in enumerate(pages):
        bt[r, :c] = ids[at:at + c]
        at += c
    return bt, pool


def make(before, n, H_q, H_kv, d, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    lens = [0 if x is None else x + n for x in before]
    bt, pool = pages_of(lens, g)
    kc = torch.randn(pool, H_kv, 16, d, generator=g).bfloat16()
    for r, x in enumerate(before):  # nothing past the context matters
        for t in range(x or 0, bt.shape[1] * 16):
            if bt[r, t // 16] >= 0:
                kc[bt[r, t // 16], :, t % 16] = math.nan
    q = (spread * torch.randn(len(lens), n, H_q, d, generator=g)).bfloat16()
    lse = 4 + torch.randn(len(lens), n, H_q, generator=g)
    return [q, lse, kc, bt, i32(lens)]


def run_mass(args, **kw):
    ws = sfv.new_workspace(sfv.attention_mass_workspace_size())
    out = sfv.attention_mass(*(a.cuda() for a in args), workspace=ws, **kw)
    return out, sfv.read_device_status(ws)


def close(got, args, weights=None, scale=None, add=None):
    want, bound = ref.mass(*args, weights=weights, scale=scale)
    B, kv, longest = want.shape
    got = got.cpu().double()
    n = args[0].shape[1]
    if add is not None:
        want, bound = want + add[..., :longest].double(), bound + (want + add[..., :longest].double().abs()) * 2.0 ** -23
    for b in range(B):
        x = max(0, int(args[4][b]) - n)
        err = (got[b, :, :x] - want[b, :, :x]).abs()
        assert (err <= bound[b, :, :x]).all(), (err - bound[b, :, :x]).max()
        if add is None:
            assert not got[b, :, x:].any()
        else:
            assert torch.equal(got[b, :, x:], add[b, :, x:].double())


HEADS = [(8, 8, 64), (28, 4, 128), (4, 4, 128), (8, 1, 64), (6, 2, 128), (5, 1, 128), (3, 3, 64), (8, 1, 128)]


@pytest.mark.parametrize("H_q, H_kv, d", HEADS)
@pytest.mark.parametrize("n", [1, 2, 16, 26, 33, 64])
def test_mass_of_head_layouts_and_rows(H_q, H_kv, d, n):
    require_gpu()
    args = make([0, 40, 130], n, H_q, H_kv, d, seed=n * 1000 + d)
    got, status = run_mass(args)
    assert status == 0
    close(got, args)


@pytest.mark.parametrize("before", [0, 1, 15, 16, 17, 63, 127, 128, 129, 240, 255, 256, 257, 300, 2000])
def test_mass_of_lengths_around_pages_and_tiles(before):
    require_gpu()
    for H_q, H_kv, d, n in ((4, 2, 64, 3), (2, 1, 128, 20)):
        args = make([before, 3], n, H_q, H_kv, d, seed=before + d)
        got, status = run_mass(args)
        assert status == 0
        close(got, args)


def test_mass_of_many_and_idle_sequences():
    require_gpu()
    for before, n in (([None, 50, None, 0, 130], 7), ([None], 3), ([(31 * b) % 170 if b % 7 else None for b in range(150)], 2),
                      ([(5 * b) % 20 for b in range(1024)], 1)):
        args = make(before, n, 2, 1, 64, seed=len(before))
        got, status = run_mass(args)
        assert status == 0
        close(got, args)


def test_mass_weights_addition_scale_and_in_place():
    require_gpu()
    n = 12
    args = make([200, 70], n, 6, 2, 128, seed=1)
    g = torch.Generator().manual_seed(2)
    weights = torch.rand(2, n, generator=g) * (torch.rand(2, n, generator=g) < 0.6)
    add = torch.rand(2, 2, args[3].shape[1] * 16 + 5, generator=g)
    got, status = run_mass(args, mass=add.cuda(), row_weights=weights.cuda(), softmax_scale=0.05)
    assert status == 0
    close(got, args, weights=weights, scale=0.05, add=add)
    again = add.cuda()
    same, _ = run_mass(args, mass=again, row_weights=weights.cuda(), softmax_scale=0.05, out=again)
    assert same is again and torch.equal(same, got)
    # an output that holds something: nothing from the context's end on is written
    held = torch.full_like(add, 7.0).cuda()
    into, _ = run_mass(args, mass=None, row_weights=weights.cuda(), out=held)
    assert (into[0, :, 200:] == 7).all() and (into[1, :, 70:] == 7).all() and (into[0, :, :200] < 7).all()


def test_mass_rows_that_do_not_count():
    require_gpu()
    for H_q, H_kv, d in ((8, 2, 64), (28, 4, 128)):
        args = make([300, 20], 9, H_q, H_kv, d, seed=3)
        weights = torch.ones(2, 9)
        weights[0, 4] = weights[1, 0] = weights[1, 8] = 0
        want, _ = run_mass(args, row_weights=weights.cuda())
        args[0][0, 4], args[1][0, 4] = math.nan, math.nan
        args[0][1, 0], args[1][1, 8] = math.inf, -math.inf
        got, _ = run_mass(args, row_weights=weights.cuda())
        assert torch.equal(got, want)
        args = make([300, 20], 9, H_q, H_kv, d, seed=3)
        args[1][0, 2:5] = -math.inf  # rows that saw nothing
        args[0][0, 3] = math.nan
        got, _ = run_mass(args)
        weights = torch.ones(2, 9)
        weights[0, 2:5] = 0
        args[0][0, 3] = 0
        close(got, args, weights=weights)


def test_mass_nan_and_infinities_reach_their_keys_and_heads_only():
    require_gpu()
    args = make([300, 150], 5, 8, 2, 64, seed=4)
    want, _ = run_mass(args)
    page, slot = ref.place(args[3][0], 77)
    args[2][page, 1, slot, 3] = math.nan
    got, _ = run_mass(args)
    assert got[0, 1, 77].isnan()
    got[0, 1, 77] = want[0, 1, 77]
    assert torch.equal(got, want)
    args[2][page, 1, slot, 3] = 0
    args[0][1, 2, 1, 9] = math.nan  # a query of KV head 0 of the second sequence
    got, _ = run_mass(args)
    assert got[1, 0, :150].isnan().all() and torch.equal(got[1, 1], want[1, 1])


def test_mass_device_data_errors_are_flagged():
    require_gpu()
    args = make([100, 40], 6, 4, 2, 64, seed=5)
    bad = [a.clone() for a in args]
    bad[3][0, 2] = -5
    got, status = run_mass(bad)
    assert status == sfv.SF_DEVICE_BAD_PAGE
    close(got, bad)
    width = 50
    held = torch.zeros(2, 2, width, device="cuda")
    got, status = run_mass(args, out=held)  # the first context is longer than the output
    assert status == sfv.SF_DEVICE_BAD_SEQLEN
    full, _ = run_mass(args)
    assert torch.equal(got, full[..., :width].clone().masked_fill(torch.arange(width, device="cuda") >= i32([50, 40]).cuda()[:, None, None], 0))
    bad = [a.clone() for a in args]
    bad[4][1] = 3  # shorter than its rows
    got, status = run_mass(bad)
    assert status == sfv.SF_DEVICE_BAD_SEQLEN and not got[1].any() and torch.equal(got[0], full[0])


def test_mass_of_an_attention_call_adds_up_to_its_rows():
    require_gpu()
    g = torch.Generator().manual_seed(6)
    n, before = 10, 3000
    bt, pool = pages_of([before + n], g)
    kc, vc = torch.randn(2, pool, 4, 16, 128, generator=g).bfloat16().cuda()
    q = torch.randn(1, n, 28, 128, generator=g).bfloat16().cuda()
    sl, bt = i32([before + n]).cuda(), bt.cuda()
    none = torch.zeros(1, n, dtype=torch.int64, device="cuda")
    _, lse = sfv.tree_attention(q, kc, vc, bt, sl, none)  # no row sees a new one
    total = sfv.attention_mass(q, lse, kc, bt, sl).double().sum(2)
    assert (total - 7 * n).abs().max() <= 7 * n * (2.0 ** -11 + 2.0 ** -12)  # the LSE's bound, and the scores'


# ---- eviction ----

def evict_case(before, layers, H_kv, d, seed, n=0, ties=False, width=None):
    g = torch.Generator().manual_seed(seed)
    lens = [0 if x is None else x + n for x in before]
    bt, pool = pages_of(lens, g, spare=1)
    kc, vc = torch.randn(2, layers, pool, H_kv, 16, d, generator=g).bfloat16()
    mass = torch.randn(layers, len(lens), H_kv, width or bt.shape[1] * 16, generator=g)
    mass = (mass * 2).round() / 2 if ties else (2 * mass).exp()
    return mass, kc, vc, bt, lens


def check_evict(case, budget, first=0, recent=0, n=0, in_place=False, as_list=False, stack=None):
    require_gpu()
    mass, kc, vc, bt, lens = case
    layers, B, kv, width = mass.shape
    m, k, v, table, sl = mass.cuda(), kc.cuda(), vc.cuda(), bt.cuda(), i32(lens).cuda()
    m_out, sl_out = (None, None) if in_place else (torch.full_like(m, 9.0), torch.full_like(sl, -5))
    kept = torch.full((layers, B, kv, budget), -7, dtype=torch.int32, device="cuda")
    ws = sfv.new_workspace(sfv.kv_evict_workspace_size(layers, B, kv, budget))
    split = (lambda t: None if t is None else list(t)) if as_list else (lambda t: t)
    free = dict(free_pages=stack[0], free_count=stack[1]) if stack else {}
    got, got_len, got_kept = sfv.kv_evict(split(m), split(k), split(v), table, sl, budget, first=first, recent=recent, n_q=n,
                                          mass_out=split(m_out), seq_lens_out=sl_out, kept=split(kept), workspace=ws, **free)
    status = sfv.read_device_status(ws)
    m_out = m if in_place else m_out
    want_k, want_v, want_m = kc.clone(), vc.clone(), torch.zeros_like(mass)
    want_kept = torch.full_like(kept, -1).cpu()
    for b in range(B):
        L = max(0, lens[b] - n)
        for l in range(layers):
            for h in range(kv):
                stay = ref.kept(mass[l, b, h].tolist(), L, budget, first, recent)
                want_kept[l, b, h, :len(stay)] = i32(stay)
                want_m[l, b, h, :len(stay)] = mass[l, b, h, stay]
                if L > budget:
                    to = [ref.place(bt[b], j) for j in range(budget)]
                    source = [ref.place(bt[b], t) for t in stay]
                    tp, ts = (torch.tensor(x) for x in zip(*to))
                    sp, ss = (torch.tensor(x) for x in zip(*source))
                    want_k[l, tp, h, ts] = kc[l, sp, h, ss]
                    want_v[l, tp, h, ts] = vc[l, sp, h, ss]
    assert torch.equal(kept.cpu(), want_kept)
    assert torch.equal(m_out.cpu(), want_m) if not mass.isnan().any() else torch.equal(m_out.cpu().nan_to_num(-3), want_m.nan_to_num(-3))
    assert torch.equal(k.cpu(), want_k) and torch.equal(v.cpu(), want_v)
    new = [min(x - n, budget) + n if x else 0 for x in lens]
    assert (sl if in_place else sl_out).tolist() == new
    if not stack:
        assert torch.equal(table.cpu(), bt)
    return status, table, new


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("budget, first, recent", [(1, 0, 0), (1, 1, 0), (16, 0, 0), (33, 4, 10), (100, 0, 100), (100, 60, 40),
                                                   (129, 3, 0), (299, 1, 1), (300, 0, 5), (500, 2, 2)])
def test_evict_budgets(budget, first, recent, in_place):
    case = evict_case([300, 100, None, 0, 17, 301], 2, 3, 64, seed=budget)
    assert check_evict(case, budget, first, recent, in_place=in_place)[0] == 0


@pytest.mark.parametrize("before, layers, H_kv, d, budget", [
    ([5000], 1, 1, 128, 700), ([5000], 1, 2, 64, 4999), ([3000, 2000], 3, 8, 128, 1024), ([700] * 8, 16, 4, 64, 333),
    ([200, 90], 2, 3, 24, 61), ([200], 1, 2, 256, 100), ([150], 2, 1, 8, 40), ([20000], 1, 1, 64, 64),
    ([40] * 300, 1, 2, 64, 17), ([600], 128, 1, 64, 200),
    # clusters of eight, four and two, and of each where CTAs share an SM
    ([2000], 1, 3, 256, 800), ([2000, 1900], 1, 10, 256, 800), ([2500], 1, 60, 128, 900), ([2500], 1, 60, 24, 900),
    ([4500, 3600], 1, 20, 8, 3501), ([3000], 3, 30, 8, 2400), ([5200], 4, 40, 8, 4400), ([700, 4000], 2, 15, 16, 640)])
def test_evict_shapes(before, layers, H_kv, d, budget):
    case = evict_case(before, layers, H_kv, d, seed=budget + d)
    assert check_evict(case, budget, 2, min(16, budget - 2), in_place=True, as_list=layers == 3)[0] == 0


@pytest.mark.parametrize("L", [511, 512, 513, 1024, 1500, 4095, 4096, 4097])
def test_evict_lengths_around_a_round(L):
    for budget in (L - 1, L // 2, 127, 128):
        assert check_evict(evict_case([L], 1, 2, 128, seed=L), budget, 1, 5, in_place=True)[0] == 0


# both sides of the widths up to which one warp has all weights, few heads and many
@pytest.mark.parametrize("width, layers", [(256, 2), (256, 12), (257, 2), (257, 12), (512, 2), (512, 12), (513, 12)])
@pytest.mark.parametrize("budget, first, recent, d, ties", [(1, 0, 1, 128, False), (31, 3, 8, 64, True), (32, 0, 0, 8, False),
                                                            (100, 40, 60, 24, False), (129, 1, 2, 256, True), (255, 0, 9, 128, True)])
def test_evict_short_contexts(width, layers, budget, first, recent, d, ties):
    long = min(width, 512)
    before = [256, 255, None, 1, 0, 31, 33, 128, 130, 200, 101, long, long - 1, long - 130]
    for in_place in (False, True):
        case = evict_case(before, layers, 3, d, seed=budget + d, n=0 if in_place else 4, ties=ties, width=width)
        case[0][0, 0, 0, 5:9], case[0][1, 1, 2, 200:] = math.nan, -math.inf
        assert check_evict(case, budget, first, recent, n=0 if in_place else 4, in_place=in_place)[0] == 0


def test_evict_ties_zeros_infinities_and_nan():
    case = evict_case([900, 333], 2, 2, 64, seed=1, ties=True)
    case[0][0, 0, 0] = 0
    case[0][0, 0, 1, ::3] = -0.0
    case[0][0, 1, 0, 5::7] = math.nan
    case[0][1, 0, 0, ::11] = math.inf
    case[0][1, 0, 1, ::2] = -math.inf
    case[0][1, 1, 1] = math.nan
    case[0][1, 1, 0] = torch.linspace(1, 1 + 2.0 ** -12, case[0].shape[3])  # neighbours in fp32
    for budget in (1, 100, 332, 600):
        assert check_evict(case, budget, 0, 0)[0] == 0
        assert check_evict(case, budget, 1, 0, in_place=True)[0] == 0


def test_evict_leaves_room_for_rows_to_come_and_wide_weights():
    case = evict_case([300, 40, None, 100], 2, 2, 64, seed=2, n=9, width=1000)
    assert check_evict(case, 64, 1, 8, n=9)[0] == 0
    assert check_evict(case, 64, 1, 8, n=9, in_place=True)[0] == 0


def test_evict_gives_pages_back():
    case = evict_case([300, 40, None, 100, 200], 1, 2, 64, seed=3, n=5)
    mass, kc, vc, bt, lens = case
    ids = sorted(set(range(kc.shape[1])) - set(bt[bt >= 0].tolist()))
    free = torch.full((64,), -9, dtype=torch.int32)
    free[:len(ids)] = i32(ids)
    free, count = free.cuda(), i32([len(ids)]).cuda()
    status, table, new = check_evict(case, 64, 1, 8, n=5, in_place=True, stack=(free, count))
    assert status == 0
    freed = []
    for b in range(5):
        need, had = -(-new[b] // 16), -(-lens[b] // 16)
        want = bt[b].tolist()
        freed += want[need:had]
        want[need:had] = [-1] * (had - need)
        assert table[b].tolist() == want
    assert free[:int(count)].tolist() == ids + freed


def test_evict_with_a_full_stack_keeps_the_pages_mapped():
    case = evict_case([300, 400, 64], 1, 1, 64, seed=4)
    bt = case[3]
    free, count = torch.full((20,), -9, dtype=torch.int32).cuda(), i32([2]).cuda()
    status, table, new = check_evict(case, 64, in_place=True, stack=(free, count))
    # 300 tokens: 19 pages, 15 of them freed; 400: 25 pages, 21 freed, which is too many
    assert status == sfv.SF_DEVICE_OUT_OF_PAGES and int(count) == 17
    assert free[2:17].tolist() == bt[0, 4:19].tolist() and torch.equal(table[1:].cpu(), bt[1:])


# more sequences than a CTA has threads, of which some give pages back, some are cut
# inside their last page, some stay; `room`: of the pages that all of them would give
@pytest.mark.parametrize("room", [1.0, 0.9, 0.45, 0.0])
def test_evict_gives_back_the_pages_of_many(room):
    before = [[None, 20, 33, 70, 0, 36, 150][b % 7] for b in range(600)]
    case = evict_case(before, 1, 1, 8, seed=6)
    bt, lens = case[3], case[4]
    had, need = ([-(-(min(x, cut) if x else 0) // 16) for x in lens] for cut in (1000, 32))
    free = torch.full((7 + int(room * (sum(had) - sum(need))),), -9, dtype=torch.int32)
    room = len(free) - 7
    free, count = free.cuda(), i32([7]).cuda()
    status, table, _ = check_evict(case, 32, in_place=True, stack=(free, count))
    freed, want, full = [], bt.clone(), False
    for b, x in enumerate(lens):
        full |= x > 32 and len(freed) + had[b] - need[b] > room
        if x > 32 and not full:
            freed += bt[b, need[b]:had[b]].tolist()
            want[b, need[b]:had[b]] = -1
    assert status == (sfv.SF_DEVICE_OUT_OF_PAGES if full else 0)
    assert int(count) == 7 + len(freed) and free[7:int(count)].tolist() == freed
    assert free[:7].tolist() == [-9] * 7 and torch.equal(table.cpu(), want)


def test_evict_bad_lengths_and_pages_are_flagged():
    require_gpu()
    mass, kc, vc, bt, lens = evict_case([300, 200, 100], 1, 2, 64, seed=5)
    bt[0, 3] = -1
    lens = [300, 5, 1 << 20]
    k, v, sl, m = kc.cuda(), vc.cuda(), i32(lens).cuda(), mass.cuda()
    ws = sfv.new_workspace(sfv.kv_evict_workspace_size(1, 3, 2, 50))
    m_out, sl_out, _ = sfv.kv_evict(m, k, v, bt.cuda(), sl, 50, n_q=9, seq_lens_out=torch.empty_like(sl),
                                    mass_out=torch.empty_like(m), workspace=ws)
    assert sfv.read_device_status(ws) == sfv.SF_DEVICE_BAD_SEQLEN | sfv.SF_DEVICE_BAD_PAGE
    assert sl_out.tolist() == [59, 5, 1 << 20]
    for h in range(2):
        stay = ref.kept(mass[0, 0, h].tolist(), 291, 50, 0, 0)
        for j, t in enumerate(stay):
            to, source = ref.place(bt[0], j), ref.place(bt[0], t)
            if to[0] >= 0 and source[0] >= 0:
                assert torch.equal(k[0, to[0], h, to[1]].cpu(), kc[0, source[0], h, source[1]])
    others = [p for p in range(kc.shape[1]) if p not in bt[0].tolist()]
    assert torch.equal(k[0, others].cpu(), kc[0, others]) and torch.equal(v[0, others].cpu(), vc[0, others])


def test_evict_repeats_and_replays():
    require_gpu()
    mass, kc, vc, bt, lens = evict_case([900, 500], 4, 4, 64, seed=6)
    m, table, sl = mass.cuda(), bt.cuda(), i32(lens).cuda()
    k, v = kc.cuda(), vc.cuda()
    out, sl_out = torch.empty_like(m), torch.empty_like(sl)
    kept = torch.empty(4, 2, 4, 200, dtype=torch.int32, device="cuda")
    ws = sfv.new_workspace(sfv.kv_evict_workspace_size(4, 2, 4, 200))
    call = lambda: sfv.kv_evict(m, k, v, table, sl, 200, first=1, recent=9, mass_out=out, seq_lens_out=sl_out,  # noqa: E731
                                kept=kept, workspace=ws)
    call()
    want = [t.clone() for t in (k, v, out, sl_out, kept)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(20):
        k.copy_(kc)
        v.copy_(vc)
        graph.replay()
        for x, y in zip((k, v, out, sl_out, kept), want):
            assert torch.equal(x, y)
