"""Forms in which the decoder-layer operators' arguments come (GPU): a single row whose
stride means nothing, strides of 0, another stream, a captured graph."""
import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests.gpu_helpers import require_gpu
from tests.test_gpu_layer_calls import OPS

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


# A tensor of one row is contiguous whatever its row stride says: the transposed column
# (1), a row of an expanded tensor (0), a slice of a wider one.
@pytest.mark.parametrize("rows", [lambda t: t.new_empty(t.shape[1], 1).copy_(t.t()).t(), lambda t: t[0].expand(3, -1)[:1],
                                  lambda t: torch.cat([t, t], 1)[:, :t.shape[1]]])
@pytest.mark.parametrize("kind", [BF, torch.float32])
@pytest.mark.parametrize("out_dtype", [BF, torch.float8_e4m3fn])
def test_norm_of_a_single_row(rows, kind, out_dtype, monkeypatch):
    require_gpu()
    d = 512
    g = torch.Generator(device="cuda").manual_seed(3)
    x, r = torch.randn(2, 1, d, generator=g, device="cuda").to(kind)
    w = torch.ones(d, dtype=BF, device="cuda")
    scales = torch.empty(1, 1, device="cuda") if out_dtype is not BF else None
    want = sfv.add_rms_norm(x, w, r, out_dtype=out_dtype)

    def call():
        return sfv.add_rms_norm(rows(x), w, rows(r), out=rows(torch.empty(1, d, dtype=out_dtype, device="cuda")),
                                residual_out=rows(torch.empty_like(r)), scales=scales)

    direct = call()
    monkeypatch.setattr(sfv, "_calls", None)
    for got in (direct, call()):
        assert torch.equal(got[0].float(), want[0].float()) and torch.equal(got[1], want[1])


# One key and value for all heads, one query for all rows: strides of 0, on 16-byte
# boundaries and one element off, against the same values written out.
@pytest.mark.parametrize("kind", [BF, torch.float32])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T", [6, 300])
def test_append_of_broadcast_tensors(kind, off, interleaved, T):
    require_gpu()
    H_q, H_kv, d, B = 4, 3, 64, 2
    g = torch.Generator(device="cuda").manual_seed(off + T)
    q, k, v = (torch.randn(T, d + off, generator=g, device="cuda").to(kind)[:, off:] for _ in range(3))
    q = q[:1, None].expand(T, H_q, d)
    k, v = (t[:, None].expand(T, H_kv, d) for t in (k, v))
    assert v.stride(1) == 0 and q.stride()[:2] == (0, 0)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")[None]
    freq = torch.linspace(1, 0.01, 32, dtype=torch.float64, device="cuda")
    pages = -(-T // B // 16) + 1
    table = torch.arange(B * pages, dtype=torch.int32, device="cuda").view(B, pages)
    lens = torch.full((B,), T // B + 3, dtype=torch.int32, device="cuda")

    def call(q, k, v):
        kc, vc = torch.zeros(2, B * pages, H_kv, 16, d, dtype=BF, device="cuda")
        return sfv.kv_append(q, k, v, pos, freq, kc, vc, table, lens, interleaved=interleaved), kc, vc

    for a, b in zip(call(q, k, v), call(q.contiguous(), k.contiguous(), v.contiguous())):
        assert torch.equal(a, b) and bool((b != 0).any())


def tensors(kw):
    return {n: t.clone() for n, t in kw.items() if isinstance(t, torch.Tensor) and n != "workspace"}


def same(a, b):
    return a.keys() == b.keys() and all(torch.equal(a[n].nan_to_num(), b[n].nan_to_num()) for n in a)


@pytest.mark.parametrize("direct", [True, False])
@pytest.mark.parametrize("name, args", OPS)
def test_on_another_stream(name, args, direct, monkeypatch):
    # outputs and workspace given, and left to the call
    require_gpu()
    if not direct:
        monkeypatch.setattr(sfv, "_calls", None)
    want, kw = args(), args()
    getattr(sfv, name)(**want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    getattr(sfv, name)(**kw, stream=side)
    side.synchronize()
    assert same(tensors(kw), tensors(want))
    outputs = ("out", "q_out", "lse", "residual_out")
    kw = {n: t for n, t in args().items() if n not in outputs and n not in ("workspace", "scales")}
    side.wait_stream(torch.cuda.current_stream())
    got = getattr(sfv, name)(**kw, stream=side)
    side.synchronize()
    got = [t for t in (got if isinstance(got, tuple) else (got,)) if t is not None]
    expected = [want[n] for n in outputs if want.get(n) is not None]
    assert len(got) == len(expected) and all(torch.equal(a, b) for a, b in zip(got, expected))


@pytest.mark.parametrize("direct", [True, False])
@pytest.mark.parametrize("name, args", OPS)
def test_in_a_captured_graph(name, args, direct, monkeypatch):
    # three calls of one workspace in a graph, replayed on new contents of the same tensors
    require_gpu()
    if not direct:
        monkeypatch.setattr(sfv, "_calls", None)
    kw = args()
    getattr(sfv, name)(**kw)  # (once outside: the library looks up its kernels)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            getattr(sfv, name)(**kw)
    first = next(n for n in ("x", "q") if n in kw)
    for scale in (1.0, -0.5):
        fresh = args()
        for n, t in fresh.items():
            if isinstance(t, torch.Tensor) and n != "workspace":
                kw[n].copy_(t)
        fresh[first].mul_(scale)
        kw[first].mul_(scale)
        getattr(sfv, name)(**fresh)
        graph.replay()
        torch.cuda.synchronize()
        assert same(tensors(kw), tensors(fresh))
    if "workspace" in kw:
        assert sfv.read_device_status(kw["workspace"]) == 0
