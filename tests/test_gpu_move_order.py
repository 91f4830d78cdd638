"""sf_verify_attention directly behind sf_tree_commit and sf_kv_evict (GPU): it reads the
lengths, the block table and the keys in front of its draft rows before it waits for the
kernel in front of it, so those two let it start only once their stores can be read."""
import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests.gpu_helpers import require_gpu
from tests.test_gpu_bounded_cache import evict_case
from tests.test_gpu_tree_draft import expect, make

pytestmark = pytest.mark.gpu
LAYERS = 6  # calls close behind each other


def follow(moves, caches, first, table, lens, H_q, n_q, reset):
    """moves(i) and then the attention over caches[i], some times over, as calls and as a
    graph, against the same with a wait between."""
    kc, vc = caches
    layers, _, H_kv, _, d = kc.shape
    B = table.shape[0]
    q = torch.randn(B, n_q, H_q, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    outs = [torch.empty_like(q) for _ in range(layers)]
    ws = sfv.new_workspace(sfv.verify_attention_workspace_size(B, n_q, H_q, H_kv, d, table.shape[1]))

    def run(wait):
        for i in range(layers):
            moves(i)
            if wait:
                torch.cuda.synchronize()
            sfv.verify_attention(q, kc[i], vc[i], table, lens[i], out=outs[i], workspace=ws, with_lse=False)

    def again(call):
        for o in outs:
            o.zero_()
        kc.copy_(first[0])
        vc.copy_(first[1])
        reset()
        torch.cuda.synchronize()
        call()
        torch.cuda.synchronize()
        return [o.clone() for o in outs]

    stale = again(lambda: [sfv.verify_attention(q, kc[i], vc[i], table, lens[i], out=outs[i], workspace=ws, with_lse=False)
                           for i in range(layers)])
    want = again(lambda: run(True))
    assert all(o.isfinite().all() for o in want)
    assert not any(torch.equal(a, b) for a, b in zip(want, stale))  # what comes too early would be seen
    for _ in range(4):
        assert all(torch.equal(a, b) for a, b in zip(again(lambda: run(False)), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(False)
    for _ in range(4):
        assert all(torch.equal(a, b) for a, b in zip(again(graph.replay), want))
    assert sfv.read_device_status(ws) == 0


# both attention kernels (5 and 28 rows a KV head)
@pytest.mark.parametrize("H_q, H_kv, d, n_q", [(8, 8, 128, 5), (28, 4, 128, 4), (4, 4, 64, 5)])
@pytest.mark.parametrize("before", [[600, 33, 400], [20], [90] * 40])
def test_attention_directly_behind_the_commit(H_q, H_kv, d, n_q, before):
    require_gpu()
    n = 40
    tokens, sampled, trees, kc, vc, bt, lens = case = make(before, n, LAYERS, H_kv, d, seed=d + len(before), agree=1.0)
    accepted = expect(*case)[0]
    # the context with the path, and n_q rows behind it that are there already
    after = (torch.tensor([min(x + int(a) + 1, x + n - n_q) for x, a in zip(before, accepted)]) + n_q).int().cuda()
    first = kc.cuda(), vc.cuda()
    k, v = (t.clone() for t in first)
    args = [t.cuda() for t in (tokens, sampled, torch.tensor(trees, dtype=torch.int32))]
    table, sl = bt.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    ws = sfv.new_workspace(sfv.tree_commit_workspace_size())
    outs = dict(num_accepted=torch.empty(len(before), dtype=torch.int32, device="cuda"), out_tokens=torch.empty_like(args[0]),
                path=torch.empty_like(args[0]), row_weights=torch.empty(args[0].shape, device="cuda"))
    follow(lambda i: sfv.tree_commit(*args, k[i:i + 1], v[i:i + 1], table, sl, workspace=ws, **outs), (k, v), first, table,
           [after] * LAYERS, H_q, n_q, lambda: None)
    assert sfv.read_device_status(ws) == 0


# one warp a head, one CTA a head, clusters
@pytest.mark.parametrize("H_q, H_kv, d, n_q", [(8, 8, 128, 5), (28, 4, 128, 4), (4, 4, 64, 5)])
@pytest.mark.parametrize("before, budget", [([220, 40, 180], 64), ([60] * 90, 30), ([900, 300], 200), ([5000], 3000),
                                            ([1500] * 60, 700)])
def test_attention_directly_behind_the_eviction(H_q, H_kv, d, n_q, before, budget):
    require_gpu()
    mass, kc, vc, bt, lens = evict_case(before, LAYERS, H_kv, d, seed=d + budget, n=n_q)
    first = kc.cuda(), vc.cuda()
    k, v = (t.clone() for t in first)
    m, table, sl = mass.cuda(), bt.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    after = [torch.empty_like(sl) for _ in range(LAYERS)]
    ws = sfv.new_workspace(sfv.kv_evict_workspace_size(1, len(before), H_kv, budget))
    m_out = torch.empty_like(m[:1])

    def reset():
        for t in after:
            t.fill_(n_q + 1)

    follow(lambda i: sfv.kv_evict(m[i:i + 1], k[i:i + 1], v[i:i + 1], table, sl, budget, n_q=n_q, mass_out=m_out,
                                  seq_lens_out=after[i], workspace=ws), (k, v), first, table, after, H_q, n_q, reset)
    assert sfv.read_device_status(ws) == 0
