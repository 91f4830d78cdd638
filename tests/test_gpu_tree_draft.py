"""sf_tree_mask and sf_tree_commit against plain Python (GPU).  Whole numbers and moved
bits: everything has to be equal."""
import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import tree_reference as ref
from tests.gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu

i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731


def random_parents(n, g, width=4, unused=0.0, deep=False):
    p = [-1]
    for i in range(1, n):
        lo = i - 1 if deep else max(0, i - width)
        p.append(int(torch.randint(lo, i, (1,), generator=g)))
        if float(torch.rand(1, generator=g)) < unused:
            p[-1] = [-2, -1, -7][int(torch.randint(0, 3, (1,), generator=g))]
    return p


@pytest.mark.parametrize("n", [1, 2, 3, 31, 32, 33, 61, 63, 64])
@pytest.mark.parametrize("B", [1, 3, 9])
def test_masks_and_positions(n, B):
    require_gpu()
    g = torch.Generator().manual_seed(n * 10 + B)
    trees = [random_parents(n, g, width=1 + 7 * b, unused=0.1 * (b % 3), deep=b == 1) for b in range(B)]
    start = torch.randint(-5, 40000, (B,), generator=g).int()
    want = [ref.masks(t) for t in trees]
    depth = [[max(0, bin(w).count("1") - 1) for w in row] for row in want]
    ws = sfv.new_workspace(sfv.tree_mask_workspace_size())
    for s in (start.cuda(), None):
        mask, positions = sfv.tree_mask(i32(trees).cuda(), s, workspace=ws)
        assert mask.tolist() == [[ref.signed(w) for w in row] for row in want]
        assert torch.equal(positions.cpu(), i32(depth) + (start[:, None] if s is not None else 0))
    assert sfv.read_device_status(ws) == 0


def test_entries_that_are_not_below_their_row_are_flagged():
    require_gpu()
    trees = [[-1, 0, 1, 3, 3, 2], [0, 0, 1, 2, 2 ** 31 - 1, 4], [-1, 0, 0, 0, 0, 0]]
    ws = sfv.new_workspace(sfv.tree_mask_workspace_size())
    mask, positions = sfv.tree_mask(i32(trees).cuda(), workspace=ws)
    assert mask.tolist() == [ref.masks(t) for t in trees]
    assert mask[1].tolist() == [0] * 6 and mask[0, 3:].tolist() == [0, 0, 0b100111]
    assert sfv.read_device_status(ws) == sfv.SF_DEVICE_BAD_INDEX


def make(before, n, layers, H_kv, d, seed, agree=0.7):
    """before: the contexts' lengths (None: idle).  Siblings share tokens now and then."""
    g = torch.Generator().manual_seed(seed)
    B = len(before)
    lens = [0 if x is None else x + n for x in before]
    pages = [-(-x // 16) for x in lens]
    pool = sum(pages) + 2
    ids = torch.randperm(pool, generator=g).int()
    bt = torch.full((B, max(1, max(pages)) + 1), -1, dtype=torch.int32)
    at = 0
    for r, c in enumerate(pages):
        bt[r, :c] = ids[at:at + c]
        at += c
    kc, vc = torch.randn(2, layers, pool, H_kv, 16, d, generator=g).bfloat16()
    trees = [random_parents(n, g, width=3, unused=0.05, deep=b % 4 == 1) for b in range(B)]
    tokens = torch.randint(0, 3, (B, n), generator=g).int()
    sampled = torch.randint(0, 3, (B, n), generator=g).int()
    for b in range(B):
        for i in range(n):
            children = [c for c in range(n) if trees[b][c] == i]
            if children and float(torch.rand(1, generator=g)) < agree:
                sampled[b, i] = tokens[b, children[int(torch.randint(0, len(children), (1,), generator=g))]]
    return tokens, sampled, trees, kc, vc, bt, lens


def expect(tokens, sampled, trees, kc, vc, bt, lens):
    B, n = tokens.shape
    kc, vc = kc.clone(), vc.clone()
    old_k, old_v = kc.clone(), vc.clone()
    accepted, out, paths, weights = [], [], [], torch.zeros(B, n)
    for b in range(B):
        path = ref.path(trees[b], tokens[b].tolist(), sampled[b].tolist()) if lens[b] else []
        accepted.append(max(0, len(path) - 1))
        out.append([int(sampled[b, i]) for i in path] + [-1] * (n - len(path)))
        paths.append(path + [-1] * (n - len(path)))
        weights[b, path] = 1
        for r, i in enumerate(path):
            to, source = (ref.place(bt[b], lens[b] - n + x) for x in (r, i))
            for new, old in ((kc, old_k), (vc, old_v)):
                new[:, to[0], :, to[1]] = old[:, source[0], :, source[1]]
    return i32(accepted), i32(out), i32(paths), weights, kc, vc


@pytest.mark.parametrize("before, n, layers, H_kv, d", [
    ([30], 1, 1, 1, 64), ([30, 0, None, 7], 20, 2, 3, 64), ([15, 100, 16], 33, 3, 4, 128), ([3, 250], 64, 2, 2, 128),
    ([40] * 9, 64, 1, 1, 8), ([9, 1, 40], 40, 2, 5, 24), ([5, 77], 50, 1, 2, 256), ([None, None], 5, 2, 2, 64),
    ([1000], 26, 32, 8, 128)])
def test_paths_and_moves(before, n, layers, H_kv, d):
    require_gpu()
    case = make(before, n, layers, H_kv, d, seed=n + d, agree=0.9)
    tokens, sampled, trees, kc, vc, bt, lens = case
    want = expect(*case)
    for as_list in (False, True):
        k, v = kc.cuda(), vc.cuda()
        ws = sfv.new_workspace(sfv.tree_commit_workspace_size())
        table, sl = bt.cuda(), i32(lens).cuda()
        got = sfv.tree_commit(tokens.cuda(), sampled.cuda(), i32(trees).cuda(), list(k) if as_list else k,
                              list(v) if as_list else v, table, sl, workspace=ws)
        for x, y in zip((*got, k, v), want):
            assert torch.equal(x.cpu(), y)
        assert torch.equal(table.cpu(), bt) and torch.equal(sl.cpu(), i32(lens))
        assert sfv.read_device_status(ws) == 0


def test_a_chain_that_is_accepted_whole_moves_nothing():
    require_gpu()
    n = 64
    tokens = torch.arange(n).int()[None]
    sampled = tokens + 1
    k = torch.randn(2, 9, 2, 16, 64).bfloat16().cuda()
    before = k.clone()
    bt = torch.arange(9).int()[None].cuda()
    got = sfv.tree_commit(tokens.cuda(), sampled.cuda(), i32([list(range(-1, n - 1))]).cuda(), k, k.clone(), bt,
                          i32([70 + n]).cuda())
    assert got[0].tolist() == [n - 1] and got[1][0].tolist() == list(range(1, n + 1))
    assert got[2][0].tolist() == list(range(n)) and torch.equal(k, before)


def test_interleaved_caches_and_no_layers():
    require_gpu()
    case = make([30, 5], 20, 3, 2, 64, seed=3, agree=1.0)
    tokens, sampled, trees, kc, vc, bt, lens = case
    want = expect(*case)
    both = torch.stack([kc, vc], 1).cuda()  # [layers][2][pages]..
    args = tokens.cuda(), sampled.cuda(), i32(trees).cuda()
    rest = bt.cuda(), i32(lens).cuda()
    got = sfv.tree_commit(*args, both[:, 0], both[:, 1], *rest)
    assert torch.equal(both[:, 0].cpu(), want[4]) and torch.equal(both[:, 1].cpu(), want[5])
    none = sfv.tree_commit(*args, [], [], *rest)
    for x, y, z in zip(got, none, want):
        assert torch.equal(x.cpu(), z) and torch.equal(y.cpu(), z)


def test_lengths_and_pages_for_the_next_tree():
    require_gpu()
    n, nxt = 40, 9
    case = make([30, 5, None, 160], n, 1, 2, 64, seed=4, agree=0.8)
    tokens, sampled, trees, kc, vc, bt, lens = case
    accepted = expect(*case)[0].tolist()
    ids = set(range(kc.shape[1])) - set(bt[bt >= 0].tolist())
    stack = torch.full((64,), -9, dtype=torch.int32)
    stack[:len(ids)] = i32(sorted(ids))
    table, sl, free, count = bt.cuda(), i32(lens).cuda(), stack.cuda(), i32([len(ids)]).cuda()
    ws = sfv.new_workspace(sfv.tree_commit_workspace_size())
    sfv.tree_commit(tokens.cuda(), sampled.cuda(), i32(trees).cuda(), kc.cuda(), vc.cuda(), table, sl, n_q_next=nxt,
                    free_pages=free, free_count=count, workspace=ws)
    assert sfv.read_device_status(ws) == 0
    new = [T - n + a + 1 + nxt if T else 0 for T, a in zip(lens, accepted)]
    assert sl.tolist() == new
    mapped = []
    for b in range(4):
        row, need = table[b].tolist(), -(-new[b] // 16)
        assert all(x >= 0 for x in row[:need]) and all(x == -1 for x in row[need:])
        assert row[:min(need, -(-lens[b] // 16))] == bt[b, :min(need, -(-lens[b] // 16))].tolist()
        mapped += row[:need]
    left = free[:int(count)].tolist()
    assert sorted(mapped + left) == list(range(kc.shape[1]))


def test_bad_lengths_pages_and_parents_are_flagged():
    require_gpu()
    case = make([30, 5, 40], 20, 2, 2, 64, seed=5, agree=1.0)
    tokens, sampled, trees, kc, vc, bt, lens = case
    lens = [lens[0], 19, lens[2]]  # shorter than the tree: counts as idle
    bt[2, 3] = 1 << 30             # rows 8 .. 19 of the third tree
    trees[0][7] = 9                # not below its row
    clean = [[p if p < i else -2 for i, p in enumerate(t)] for t in trees]
    k, v = kc.cuda(), vc.cuda()
    ws = sfv.new_workspace(sfv.tree_commit_workspace_size())
    got = sfv.tree_commit(tokens.cuda(), sampled.cuda(), i32(trees).cuda(), k, v, bt.cuda(), i32(lens).cuda(), workspace=ws)
    status = sfv.read_device_status(ws)
    assert status & sfv.SF_DEVICE_BAD_SEQLEN and status & sfv.SF_DEVICE_BAD_INDEX
    paths = [ref.path(clean[b], tokens[b].tolist(), sampled[b].tolist()) if b != 1 else [] for b in range(3)]
    assert [[i for i in row if i >= 0] for row in got[2].tolist()] == paths
    assert got[0].tolist() == [max(0, len(p) - 1) for p in paths]
    for b, path in enumerate(paths):
        for r, i in enumerate(path):
            to, source = (ref.place(bt[b], lens[b] - 20 + x) for x in (r, i))
            if max(to[0], source[0]) < k.shape[1]:
                assert torch.equal(k[:, to[0], :, to[1]].cpu(), kc[:, source[0], :, source[1]])
    moved = any(ref.place(bt[2], 40 + i)[0] == 1 << 30 and i != r for r, i in enumerate(paths[2]))
    assert bool(status & sfv.SF_DEVICE_BAD_PAGE) == moved


def test_captured_and_replayed():
    require_gpu()
    case = make([30, 5], 20, 2, 2, 64, seed=6, agree=1.0)
    tokens, sampled, trees, kc, vc, bt, lens = case
    want = expect(*case)
    k, v, par = kc.cuda(), vc.cuda(), i32(trees).cuda()
    args = tokens.cuda(), sampled.cuda(), par, k, v, bt.cuda(), i32(lens).cuda()
    outs = [torch.empty_like(w, device="cuda") for w in want[:4]]
    mask, pos = torch.empty(2, 20, dtype=torch.int64, device="cuda"), torch.empty(2, 20, dtype=torch.int32, device="cuda")
    ws = sfv.new_workspace(256)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sfv.tree_mask(par, mask=mask, positions=pos, workspace=ws)
        sfv.tree_commit(*args, num_accepted=outs[0], out_tokens=outs[1], path=outs[2], row_weights=outs[3], workspace=ws)
    for _ in range(2):
        k.copy_(kc)
        v.copy_(vc)
        graph.replay()
        for x, y in zip((*outs, k, v), want):
            assert torch.equal(x.cpu(), y)
        assert mask.tolist() == [[ref.signed(w) for w in ref.masks(t)] for t in trees]
