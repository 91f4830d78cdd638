"""sf_attention_mass where it is easy to go wrong (GPU): infinite keys beside rows that do
not count, and contexts of many key tiles a CTA, in which the ring of keys, the buffers of
queries and those of scores come round several times."""
import math

import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import tree_reference as ref
from tests.gpu_helpers import require_gpu
from tests.test_gpu_bounded_cache import make, run_mass

pytestmark = pytest.mark.gpu


# rows a KV head: 5 and 27 (padded to 16 and 32), 16 (none), 264 (three chunks of 96)
@pytest.mark.parametrize("H_q, H_kv, d, n", [(2, 2, 64, 5), (3, 1, 128, 9), (2, 2, 128, 16), (8, 1, 128, 33)])
def test_infinite_keys_that_no_counted_row_looks_at_get_nothing(H_q, H_kv, d, n):
    require_gpu()
    args = make([300, 150], n, H_q, H_kv, d, seed=n + d)
    args[0][..., 3] = args[0][..., 3].abs() + 0.5  # every row has a positive element there,
    args[0][..., 7] = -args[0][..., 7].abs() - 0.5  # and a negative one here
    page, slot = ref.place(args[3][0], 140)
    for counted in (torch.ones(2, n), (torch.arange(n) % 3 != 1).float().expand(2, n).contiguous(), torch.zeros(2, n)):
        counted = counted.cuda()
        clean, _ = run_mass(args, row_weights=counted)
        for element, value in ((3, -math.inf), (7, math.inf)):  # scores of -inf: exp(-inf - lse) = 0
            bad = [a.clone() for a in args]
            bad[2][page, H_kv - 1, slot, element] = value
            if not bool(counted.all()):
                bad[0][:, 1] = math.nan  # what a row of weight 0 holds has no effect
            got, status = run_mass(bad, row_weights=counted)
            assert status == 0 and float(got[0, H_kv - 1, 140]) == 0.0
            got[0, H_kv - 1, 140] = clean[0, H_kv - 1, 140]
            assert torch.equal(got, clean)
        if bool(counted.any()):
            bad = [a.clone() for a in args]
            bad[2][page, H_kv - 1, slot, 3] = math.inf  # scores of +inf: exp(inf - lse) = inf
            got, _ = run_mass(bad, row_weights=counted)
            assert float(got[0, H_kv - 1, 140]) == math.inf
            bad[2][page, H_kv - 1, slot, 7] = math.inf  # inf - inf
            got, _ = run_mass(bad, row_weights=counted)
            assert got[0, H_kv - 1, 140].isnan()
            bad[2][page, H_kv - 1, slot, 7] = 0
            bad[1][0, 0, H_q - 1] = math.inf  # a row that saw that key: inf - inf
            got, _ = run_mass(bad, row_weights=counted)
            assert got[0, H_kv - 1, 140].isnan() and got[0, H_kv - 1, :140].isfinite().all()


def test_infinite_keys_and_rows_that_saw_nothing():
    require_gpu()
    args = make([200], 4, 4, 2, 64, seed=8)
    args[0][..., 3] = args[0][..., 3].abs() + 0.5
    args[1][0, 2] = -math.inf
    want, _ = run_mass(args)
    page, slot = ref.place(args[3][0], 50)
    args[2][page, 1, slot, 3] = -math.inf
    got, _ = run_mass(args)
    assert float(got[0, 1, 50]) == 0.0
    got[0, 1, 50] = want[0, 1, 50]
    assert torch.equal(got, want)


def reference(args, weights):
    """As tree_reference.mass, on the GPU, one sequence and KV head at a time."""
    q, lse, kc, bt, lens = (a.cuda() for a in args)
    B, n, H, d = q.shape
    kv, scale = kc.shape[1], 1 / math.sqrt(d)
    g = H // kv
    for b in range(B):
        before = int(lens[b]) - n
        if before <= 0:
            continue
        pages = bt[b, :-(-before // 16)].long()
        for h in range(kv):
            k = kc[pages, h].reshape(-1, d)[:before].double()
            x = q[b, :, h * g:(h + 1) * g].reshape(n * g, d).double()
            m = lse[b, :, h * g:(h + 1) * g].reshape(n * g, 1).double()
            w = weights[b].cuda().double().repeat_interleave(g)[:, None]
            s = scale * (x @ k.T) - m
            p = w * s.exp()
            off = d * 2.0 ** -23 * scale * (x.abs() @ k.abs().T) + (s.abs() + m.abs()) * 2.0 ** -22 + 2.0 ** -20
            yield b, h, before, p.sum(0), (p * (off + n * g * 2.0 ** -24)).sum(0)


# 224 rows: two q buffers, three ring slots, two chunks; 512: one q buffer, two slots, four
# chunks, several segments a CTA; few rows: the deepest rings, with 64-wide heads as well
@pytest.mark.parametrize("lens, n, H_q, H_kv, d", [
    ([16000] * 16, 32, 28, 4, 128), ([200 + (37 * b) % 401 for b in range(200)], 64, 8, 1, 128),
    ([40000, 39999, 17, 30001], 5, 8, 8, 64), ([20000] * 4, 5, 8, 8, 128), ([9000, None, 12000], 64, 16, 2, 64),
    ([6000] * 12, 33, 6, 6, 128)])
def test_many_key_tiles_a_cta(lens, n, H_q, H_kv, d):
    require_gpu()
    args = make(lens, n, H_q, H_kv, d, seed=len(lens) + n)
    g = torch.Generator().manual_seed(9)
    weights = (torch.rand(len(lens), n, generator=g) < 0.8).float() * torch.rand(len(lens), n, generator=g)
    got, status = run_mass(args, row_weights=weights.cuda())
    assert status == 0
    again, _ = run_mass(args, row_weights=weights.cuda())
    assert torch.equal(got, again)
    for b, h, before, want, bound in reference(args, weights):
        err = (got[b, h, :before].double() - want).abs()
        assert (err <= bound).all(), (b, h, (err - bound).max())
        assert not got[b, h, before:].any()
