"""sf_tree_commit of sequences whose node 0 is not part of the tree (GPU): sf_tree_mask
gives such a tree masks of 0, and the commit no path."""
import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import tree_reference as ref
from tests.gpu_helpers import require_gpu
from tests.test_gpu_tree_draft import expect, make

pytestmark = pytest.mark.gpu

i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731


def rootless(seed, nodes):
    """A batch of five trees, of which 1 and 3 have no root; what it should become."""
    case = make([30, 5, 40, 160, None], 20, 2, 2, 64, seed=seed, agree=1.0)
    tokens, sampled, trees, kc, vc, bt, lens = case
    accepted, out, path, weights, k, v = expect(*case)
    for b in (1, 3):
        trees[b][0] = nodes[b]
        if len(ref.path(trees[b], tokens[b].tolist(), sampled[b].tolist())) < 2:  # a child that could be taken
            trees[b][1], tokens[b, 1] = 0, sampled[b, 0]
        accepted[b], out[b], path[b], weights[b] = 0, -1, -1, 0
        pages = bt[b][bt[b] >= 0].long()
        k[:, pages], v[:, pages] = kc[:, pages], vc[:, pages]
    return case, (accepted, out, path, weights, k, v)


@pytest.mark.parametrize("nodes, status", [({1: -2, 3: -7}, 0), ({1: 0, 3: -2}, "index"), ({1: 5, 3: 2 ** 31 - 1}, "index")])
def test_a_tree_without_a_root_has_no_path(nodes, status):
    require_gpu()
    (tokens, sampled, trees, kc, vc, bt, lens), want = rootless(11, nodes)
    k, v, ws = kc.cuda(), vc.cuda(), sfv.new_workspace(sfv.tree_commit_workspace_size())
    mask, _ = sfv.tree_mask(i32(trees).cuda())
    assert not mask[1, 0] and not mask[3, 0]
    got = sfv.tree_commit(tokens.cuda(), sampled.cuda(), i32(trees).cuda(), k, v, bt.cuda(), i32(lens).cuda(), workspace=ws)
    for x, y in zip((*got, k, v), want):
        assert torch.equal(x.cpu(), y)
    assert sfv.read_device_status(ws) == (sfv.SF_DEVICE_BAD_INDEX if status else 0)


def test_its_context_stays_as_long_as_it_was():
    require_gpu()
    (tokens, sampled, trees, kc, vc, bt, lens), want = rootless(12, {1: -2, 3: -2})
    n, nxt = 20, 9
    ids = sorted(set(range(kc.shape[1])) - set(bt[bt >= 0].tolist()))
    stack = torch.full((64,), -9, dtype=torch.int32)
    stack[:len(ids)] = i32(ids)
    k, v, table, sl, free, count = kc.cuda(), vc.cuda(), bt.cuda(), i32(lens).cuda(), stack.cuda(), i32([len(ids)]).cuda()
    ws = sfv.new_workspace(sfv.tree_commit_workspace_size())
    got = sfv.tree_commit(tokens.cuda(), sampled.cuda(), i32(trees).cuda(), k, v, table, sl, n_q_next=nxt, free_pages=free,
                          free_count=count, workspace=ws)
    for x, y in zip((*got, k, v), want):
        assert torch.equal(x.cpu(), y)
    assert sfv.read_device_status(ws) == 0
    rows = [0 if b in (1, 3) else int(want[0][b]) + 1 for b in range(5)]
    new = [T - n + r + nxt if T else 0 for T, r in zip(lens, rows)]
    assert sl.tolist() == new
    mapped = []
    for b in range(5):
        row, need = table[b].tolist(), -(-new[b] // 16)
        assert all(x >= 0 for x in row[:need]) and all(x == -1 for x in row[need:])
        mapped += row[:need]
    assert sorted(mapped + free[:int(count)].tolist()) == list(range(kc.shape[1]))


def test_an_idle_slot_has_no_tree_to_look_at():
    require_gpu()
    (tokens, sampled, trees, kc, vc, bt, lens), want = rootless(13, {1: -2, 3: -2})
    trees[4][0] = -2
    got = sfv.tree_commit(tokens.cuda(), sampled.cuda(), i32(trees).cuda(), kc.cuda(), vc.cuda(), bt.cuda(), i32(lens).cuda())
    for x, y in zip(got, want):
        assert torch.equal(x.cpu(), y)
