"""sf_kv_evict where it is easy to go wrong (GPU): lengths that it refuses on the device,
and calls in which a CTA gave up.  Everything has to be equal."""
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
