"""sf_shared_prefix_attention where inputs hold NaN or a few weights carry a row (GPU)."""
import math

import pytest
import torch

from tests import layer_reference as ref
from tests.gpu_helpers import require_gpu
from tests.test_gpu_shared_prefix import close, make, run

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
