"""sf_verify_attention directly behind the append of its prefix (GPU): it copies the
keys in front of its draft rows before it waits for the kernel in front of it."""
import math

import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests.gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32


# sequences of one length (the rows counted from T / B) and of several (row_starts), both
# attention kernels (5 and 28 rows a KV head), 16-byte rows and rows one element off
@pytest.mark.parametrize("lens, ragged", [([600] * 3, False), ([17], False), ([600] * 3, True), ([2100, 700, 33, 1400], True),
                                          ([5] * 40, True)])
@pytest.mark.parametrize("H_q, H_kv, d, n_q", [(8, 8, 128, 5), (28, 4, 128, 4)])
@pytest.mark.parametrize("off", [0, 1])
def test_attention_directly_behind_the_append_of_its_prefix(lens, ragged, H_q, H_kv, d, n_q, off):
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(len(lens) + d + off)
    B, T = len(lens), sum(lens)
    wide = torch.randn(T, (H_q + 2 * H_kv) * d + off, generator=g, device="cuda").to(BF)[:, off:]
    q, k, v = (t.unflatten(1, (-1, d)) for t in wide.split([H_q * d, H_kv * d, H_kv * d], 1))
    pages = [-(-n // 16) for n in lens]
    table = torch.full((B, max(pages)), -1, dtype=I32)
    ids, at = torch.randperm(sum(pages), generator=torch.Generator().manual_seed(1)).int(), 0
    for b, n in enumerate(pages):
        table[b, :n] = ids[at:at + n]
        at += n
    table, sl = table.cuda(), torch.tensor(lens, dtype=I32).cuda()
    starts = torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=I32).cuda()
    pos = torch.arange(T, dtype=I32, device="cuda")[None]
    freq = 10000.0 ** (-torch.arange(d // 2, dtype=torch.float64, device="cuda") / (d // 2))
    draft = torch.cat([starts[b + 1].long() - n_q + torch.arange(n_q, device="cuda") for b in range(B)])
    query = q[draft].view(B, n_q, H_q, d).contiguous()
    caches = torch.empty(6, 2, sum(pages), H_kv, 16, d, dtype=BF, device="cuda")
    ws = sfv.new_workspace(sfv.kv_append_workspace_size())
    wa = sfv.new_workspace(sfv.verify_attention_workspace_size(B, n_q, H_q, H_kv, d, table.shape[1]))
    outs = [torch.empty_like(query) for _ in range(6)]
    qo = torch.empty(T, H_q, d, dtype=BF, device="cuda")

    def layer(i, wait):
        kc, vc = caches[i]
        sfv.kv_append(q, k, v, pos, freq, kc, vc, table, sl, row_starts=starts if ragged else None, q_out=qo, workspace=ws)
        if wait:
            torch.cuda.synchronize()
        sfv.verify_attention(query, kc, vc, table, sl, out=outs[i], workspace=wa, with_lse=False)

    caches.fill_(math.nan)
    layer(0, True)
    want = outs[0].clone()
    assert want.isfinite().all()
    for _ in range(3):
        caches.fill_(math.nan)  # what a copy that comes too early reads
        torch.cuda.synchronize()
        for i in range(6):
            layer(i, False)
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs)
    caches.fill_(math.nan)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for i in range(6):
            layer(i, False)
    for _ in range(3):
        caches.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs)
    assert sfv.read_device_status(ws) == 0 and sfv.read_device_status(wa) == 0
