"""The workspace that sf_tree_attention asks for (GPU): no more than its partial results
take, and nothing behind it is touched."""
import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import tree_reference as ref
from tests.gpu_helpers import require_gpu
from tests.test_gpu_tree_attention import close, make

pytestmark = pytest.mark.gpu


# An fp32 row of head_dim and two more words a partial row; n_q * group rows a KV head of a
# sequence (one more head where their number is odd), and 256 for each SM.
@pytest.mark.parametrize("B, n, H_q, H_kv, d", [(64, 8, 32, 32, 128), (256, 16, 32, 32, 128), (1024, 8, 32, 32, 128),
                                                (1, 5, 8, 8, 64), (512, 18, 28, 4, 128), (300, 1, 3, 3, 64)])
def test_rows_of_a_tile_that_no_query_has_take_no_room(B, n, H_q, H_kv, d):
    require_gpu()
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    rows = B * (H_kv + 1) * n * (H_q // H_kv) + 256 * sms
    need = rows * 4 * (d + 2) + 64 * B
    assert sfv.tree_attention_workspace_size(B, n, H_q, H_kv, d, 64) <= need + 1024


# one row tile (pairs of heads, an odd head, a head at a time), two, three and four
@pytest.mark.parametrize("before, n, H_q, H_kv, d", [
    ([(37 * b) % 150 if b % 11 else None for b in range(60)], 6, 3, 3, 64), ([(53 * b) % 300 for b in range(100)], 16, 8, 2, 128),
    ([700, 0, 1300], 16, 8, 1, 128), ([3000, 64], 5, 8, 8, 64), ([(29 * b) % 200 for b in range(40)], 20, 14, 2, 128),
    ([500, 3, 2000], 45, 7, 1, 128), ([1500, 300], 64, 8, 1, 64), ([(31 * b) % 90 for b in range(200)], 3, 2, 1, 64)])
def test_nothing_behind_the_workspace_is_written(before, n, H_q, H_kv, d):
    require_gpu()
    args, masks = make(before, n, H_q, H_kv, d, seed=n + d)
    size = sfv.tree_attention_workspace_size(len(before), n, H_q, H_kv, d, args[3].shape[1])
    room = torch.zeros(size + 65536, dtype=torch.uint8, device="cuda")
    room[size:] = 0x5a
    out, lse = sfv.tree_attention(*(a.cuda() for a in args), workspace=room[:size])
    assert (room[size:] == 0x5a).all()
    assert sfv.read_device_status(room[:size]) == 0
    close(out, lse, ref.attention(*args[:5], masks))
    with pytest.raises(sfv.SFError) as e:
        sfv.tree_attention(*(a.cuda() for a in args), workspace=sfv.new_workspace(size - 256))
    assert e.value.status == 4
