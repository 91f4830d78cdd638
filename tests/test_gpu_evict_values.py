"""sf_kv_evict where it is easy to go wrong (GPU): lengths that it refuses on the device,
calls in which a CTA gave up, and long contexts of whose weights more fall into one bin of
the choice's first digit than shared memory has room for.  Everything has to be equal."""
import math

import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import tree_reference as ref
from tests.gpu_helpers import require_gpu
from tests.test_gpu_bounded_cache import evict_case

pytestmark = pytest.mark.gpu

i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731

# The word of the workspace in which CTAs that gave up on a copy say so.
GAVE_UP = slice(192, 196)


# Kernels: one warp a head (tables of up to 256 tokens), one CTA a head, clusters of eight.
@pytest.mark.parametrize("longest, layers, H_kv, width", [(200, 2, 3, 256), (700, 2, 3, 900), (4000, 1, 2, 4100)])
@pytest.mark.parametrize("in_place", [False, True])
def test_weights_of_sequences_with_bad_lengths_stay(longest, layers, H_kv, width, in_place):
    require_gpu()
    n, budget = 9, 50
    mass, kc, vc, bt, lens = evict_case([longest, 30, 30, longest, 30, None, 20], layers, H_kv, 64, seed=longest, n=n, width=width)
    most = bt.shape[1] * 16
    # shorter than the rows to come, negative, far and just past the pages
    bad = {1: 5, 2: -3, 3: 1 << 20, 4: most + 1}
    lens = [bad.get(b, x) for b, x in enumerate(lens)]
    m, k, v, table, sl = mass.cuda(), kc.cuda(), vc.cuda(), bt.cuda(), i32(lens).cuda()
    m_out = m if in_place else torch.full_like(m, 9.0)
    kept = torch.full((layers, 7, H_kv, budget), -7, dtype=torch.int32, device="cuda")
    free, count = torch.full((600,), -9, dtype=torch.int32, device="cuda"), i32([0]).cuda()
    ws = sfv.new_workspace(sfv.kv_evict_workspace_size(layers, 7, H_kv, budget))
    _, sl_out, _ = sfv.kv_evict(m, k, v, table, sl, budget, n_q=n, mass_out=m_out, kept=kept, free_pages=free,
                                free_count=count, workspace=ws)
    assert sfv.read_device_status(ws) == sfv.SF_DEVICE_BAD_SEQLEN
    assert sl_out.tolist() == [budget + n] + [bad[b] for b in (1, 2, 3, 4)] + [0, 20 + n]
    for b in bad:
        assert torch.equal(m_out[:, b].cpu(), mass[:, b]), b
        assert torch.equal(table[b].cpu(), bt[b])
        pages = bt[b][bt[b] >= 0].long()
        assert torch.equal(k[:, pages].cpu(), kc[:, pages]) and torch.equal(v[:, pages].cpu(), vc[:, pages])
    want = torch.zeros(layers, H_kv, width)
    for l in range(layers):
        for h in range(H_kv):
            stay = ref.kept(mass[l, 0, h].tolist(), longest, budget, 0, 0)
            assert kept[l, 0, h].tolist() == stay
            want[l, h, :budget] = mass[l, 0, h, stay]
    assert torch.equal(m_out[:, 0].cpu(), want)
    assert torch.equal(m_out[:, 6, :, :20].cpu(), mass[:, 6, :, :20])
    assert not m_out[:, 6, :, 20:].any() and not m_out[:, 5].any()


def test_a_length_of_more_than_the_weights_leaves_them():
    require_gpu()
    for width in (100, 600):  # (the pages would hold 1008)
        mass, kc, vc, bt, lens = evict_case([1000, 60], 1, 2, 64, seed=width, width=width)
        m, sl = mass.cuda(), i32(lens).cuda()
        ws = sfv.new_workspace(sfv.kv_evict_workspace_size(1, 2, 2, 50))
        sfv.kv_evict(m, kc.cuda(), vc.cuda(), bt.cuda(), sl, 50, workspace=ws)
        assert sfv.read_device_status(ws) == sfv.SF_DEVICE_BAD_SEQLEN and sl.tolist() == [1000, 50]
        assert torch.equal(m[0, 0].cpu(), mass[0, 0])


@pytest.mark.parametrize("longest, H_kv", [(200, 2), (700, 2), (4000, 2)])
def test_lengths_and_pages_stay_where_a_cta_gave_up(longest, H_kv):
    # Rows that did not arrive make the cache useless; a length or a page that says otherwise
    # would hand it on.  The failure is made here, by the word in which such a CTA says so.
    require_gpu()
    mass, kc, vc, bt, lens = evict_case([longest, 100], 1, H_kv, 64, seed=longest + 1, n=4)
    m, k, v, table, sl = mass.cuda(), kc.cuda(), vc.cuda(), bt.cuda(), i32(lens).cuda()
    free, count = torch.full((600,), -9, dtype=torch.int32, device="cuda"), i32([3]).cuda()
    sl_out = torch.full_like(sl, -1)
    ws = sfv.new_workspace(sfv.kv_evict_workspace_size(1, 2, H_kv, 40))
    ws[GAVE_UP] = 1
    call = lambda: sfv.kv_evict(m, k, v, table, sl, 40, n_q=4, mass_out=torch.empty_like(m), seq_lens_out=sl_out,  # noqa: E731
                                free_pages=free, free_count=count, workspace=ws)
    call()
    assert sl_out.tolist() == lens and torch.equal(table.cpu(), bt)
    assert int(count) == 3 and (free == -9).all()
    assert not ws[GAVE_UP].any()  # the next call starts anew
    k.copy_(kc)
    v.copy_(vc)
    call()
    assert sl_out.tolist() == [44, 44] and int(count) == 3 + sum(-(-x // 16) - 3 for x in lens)


@pytest.mark.parametrize("longest", [200, 700])
def test_places_of_the_kept_ones_need_no_room_in_the_workspace(longest):
    require_gpu()
    mass, kc, vc, bt, lens = evict_case([longest, 90], 2, 3, 64, seed=longest)
    got = []
    for size in (256, sfv.kv_evict_workspace_size(2, 2, 3, 64), None):
        m, k, v, sl = mass.cuda(), kc.cuda(), vc.cuda(), i32(lens).cuda()
        kept = torch.full((2, 2, 3, 64), -7, dtype=torch.int32, device="cuda")
        room = None if size is None else sfv.new_workspace(size + 256)  # nothing behind is written
        ws = None if size is None else room[:size]
        sfv.kv_evict(m, k, v, bt.cuda(), sl, 64, kept=kept, workspace=ws)
        assert room is None or not room[256:].any()
        got.append([m, k, v, sl, kept])
    for other in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(got[0], other))
    with pytest.raises(sfv.SFError) as e:
        sfv.kv_evict(mass.cuda(), kc.cuda(), vc.cuda(), bt.cuda(), i32(lens).cuda(), 64, workspace=sfv.new_workspace(256))
    assert e.value.status == 4


def weights(kind, shape, g):
    x = torch.rand(shape, generator=g, device="cuda")
    if kind == "uniform":
        return x
    if kind == "equal":
        return torch.full_like(x, 0.75)
    if kind == "half zeros":
        return torch.where(torch.rand(shape, generator=g, device="cuda") < 0.5, 0.0, x)
    if kind == "neighbours":  # a few hundred steps of fp32 above 1: ties, too
        return 1 + (x * 700).floor() * 2.0 ** -23
    if kind == "two digits":  # one value of the first digit, many of the second, ties in the third
        return 1 + (x * 2 ** 20).floor() * 2.0 ** -22
    assert kind == "special"
    x = torch.where(x < 0.3, -math.inf, torch.where(x < 0.6, math.nan, torch.where(x < 0.8, -0.0, 0.0)))
    x[..., ::501] = math.inf
    return x


# heads of one CTA each (three and four an SM), and in clusters of two, four and eight
@pytest.mark.parametrize("heads, L", [(500, 12000), (320, 9000), (120, 10000), (30, 20000), (9, 30000), (1, 30001)])
@pytest.mark.parametrize("kind", ["uniform", "equal", "half zeros", "neighbours", "two digits", "special"])
def test_more_keys_in_a_bin_than_shared_memory_has_room_for(heads, L, kind):
    require_gpu()
    g = torch.Generator("cuda").manual_seed(heads + L)
    d, pages = 8, -(-L // 16)
    mass = weights(kind, (1, 1, heads, pages * 16), g)
    first_k, first_v = torch.randn(2, 1, pages, heads, 16, d, generator=g, device="cuda").bfloat16()
    table = torch.randperm(pages, generator=g, device="cuda").int()[None]
    value = mass[0, 0, :, :L].nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    for budget, first, recent in ((L // 3, 0, 0), (L * 7 // 10, 3, 60), (700, 4, 32)):
        best = torch.sort(value[:, first:L - recent], dim=1, descending=True, stable=True)[1][:, :budget - first - recent] + first
        ends = torch.cat([torch.arange(first, device="cuda"), torch.arange(L - recent, L, device="cuda")])
        stay = torch.sort(torch.cat([best, ends.expand(heads, -1)], 1), 1)[0]
        m, k, v, sl = mass.clone(), first_k.clone(), first_v.clone(), i32([L]).cuda()
        kept = torch.empty(1, 1, heads, budget, dtype=torch.int32, device="cuda")
        ws = sfv.new_workspace(256 + 4 * heads * budget + 256)
        sfv.kv_evict(m, k, v, table, sl, budget, first=first, recent=recent, kept=kept, workspace=ws)
        assert sfv.read_device_status(ws) == 0 and sl.tolist() == [budget]
        assert torch.equal(kept[0, 0].long(), stay)
        want = torch.zeros_like(mass[0, 0])
        want[:, :budget] = mass[0, 0].gather(1, stay)
        assert torch.equal(m[0, 0].nan_to_num(-3), want.nan_to_num(-3))
        for new, old in ((k, first_k), (v, first_v)):
            rows, before = (c[0, table[0].long()].transpose(0, 1).reshape(heads, pages * 16, d) for c in (new, old))
            assert torch.equal(rows[:, :budget], before.gather(1, stay[..., None].expand(-1, -1, d)))
            assert torch.equal(rows[:, budget:], before[:, budget:])
