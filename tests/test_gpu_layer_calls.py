"""The direct calls of the decoder-layer operators (csrc/layer_calls.cpp) against the
binding's own way through the same arguments (GPU): the same results bit for bit,
the same errors, and no argument that they let through and the binding refuses."""
import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests.gpu_helpers import require_gpu
from tests.test_gpu_shared_prefix import make

pytestmark = pytest.mark.gpu
BF, I32, F32 = torch.bfloat16, torch.int32, torch.float32


def norm_args():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g).to(BF).cuda()  # noqa: E731
    return dict(x=r(6, 256), weight=r(256), residual=r(6, 256), eps=1e-6, group=0,
                out=torch.empty(6, 256, dtype=BF, device="cuda"), residual_out=torch.empty(6, 256, dtype=BF, device="cuda"),
                scales=None)


def append_args():
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=g).to(BF).cuda()  # noqa: E731
    i = lambda v: torch.tensor(v, dtype=I32).cuda()  # noqa: E731
    return dict(q=r(6, 4, 64), k=r(6, 2, 64), v=r(6, 2, 64), positions=i([[3, 4, 5, 9, 10, 11]]),
                inv_freq=torch.linspace(1, 0.01, 32, dtype=torch.float64).cuda(), k_cache=r(4, 2, 16, 64),
                v_cache=r(4, 2, 16, 64), block_table=i([[0, 1], [2, 3]]), seq_lens=i([6, 20]), axis=None, row_starts=None,
                interleaved=False, amplitude=1.0, q_out=torch.empty(6, 4, 64, dtype=BF, device="cuda"),
                workspace=sfv.new_workspace(256))


def shared_args():
    a = [t.cuda() for t in make([2, 1], [40, 3], [9, 20, 33], 4, 4, 2, 64, seed=22)]
    names = ["q", "k_cache", "v_cache", "prefix_table", "prefix_lens", "group_starts", "block_table", "seq_lens"]
    ws = sfv.new_workspace(sfv.shared_prefix_attention_workspace_size(3, 4, 4, 2, 64, 2, a[3].shape[1], a[6].shape[1]))
    return dict(zip(names, a)) | dict(softmax_scale=0.0, out=torch.empty_like(a[0]),
                                      lse=torch.empty(3, 4, 4, device="cuda"), workspace=ws)


OPS = [("add_rms_norm", norm_args), ("kv_append", append_args), ("shared_prefix_attention", shared_args)]


@pytest.fixture
def calls():
    require_gpu()
    assert sfv._calls is not None, "csrc/layer_calls.cpp was not built"
    return sfv._calls


def outputs(kw):
    return {n: t.clone() for n, t in kw.items() if isinstance(t, torch.Tensor)}


@pytest.mark.parametrize("name, args", OPS)
def test_the_same_results(calls, name, args, monkeypatch):
    one, two = args(), args()
    assert getattr(calls, name)(*one.values()) == 0  # taken, without the binding's help
    monkeypatch.setattr(sfv, "_calls", None)
    getattr(sfv, name)(**two)
    torch.cuda.synchronize()
    a, b = outputs(one), outputs(two)
    assert a.keys() == b.keys() and all(torch.equal(a[n].nan_to_num(), b[n].nan_to_num()) for n in a)


@pytest.mark.parametrize("name, args", OPS)
def test_leaves_what_is_not_as_it_should_be_to_the_binding(calls, name, args):
    # each tensor in turn: missing, on the host, of another type, with a dimension
    # less, of another size, not contiguous
    good = args()
    direct = getattr(calls, name)
    for at, (key, value) in enumerate(good.items()):
        if not isinstance(value, torch.Tensor):
            continue
        wrong = [object(), value.cpu(), value.to(torch.float16 if value.dtype.is_floating_point else torch.int64), value[0]]
        # (the library compares a workspace with what it needs; two rows of positions are
        # two axes, and twice the frequencies are its to refuse)
        if key not in ("workspace", "positions", "inv_freq"):
            wrong.append(torch.cat([value, value]))
        if value.dim() > 1 and value.shape[0] > 1:
            wrong.append(value.transpose(0, -1).contiguous().transpose(0, -1))
        for bad in wrong:
            v = list(good.values())
            v[at] = bad
            assert direct(*v) is None, (key, getattr(bad, "shape", bad))
    torch.cuda.synchronize()


def test_status_of_the_library_comes_through(calls):
    kw = shared_args()
    kw["workspace"] = kw["workspace"][:256].clone()
    with pytest.raises(sfv.SFError) as e:
        sfv.shared_prefix_attention(**kw)
    assert e.value.status == 4
    kw = norm_args()
    kw["eps"] = -1.0
    with pytest.raises(sfv.SFError, match="eps"):
        sfv.add_rms_norm(**kw)
    kw = append_args()
    kw["block_table"] = kw["block_table"].view(4, 1)
    kw["seq_lens"] = torch.zeros(4, dtype=I32, device="cuda")
    with pytest.raises(sfv.SFError, match="multiple of B"):
        sfv.kv_append(**kw)


def test_parameters_and_current_stream(calls):
    kw = norm_args()
    want = sfv.add_rms_norm(**kw)[0].clone()
    kw["weight"] = torch.nn.Parameter(kw["weight"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kw["out"].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        sfv.add_rms_norm(**kw)
    side.synchronize()
    assert torch.equal(kw["out"], want)
