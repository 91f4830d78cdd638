"""Calls of the tree and eviction operators in other forms (GPU): the direct calls
(csrc/layer_calls.cpp) against the binding's own way, calls on two streams at once,
kernels close behind each other, and a step of all of them captured into a graph."""
import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import tree_reference as ref
from tests.gpu_helpers import require_gpu
from tests.test_gpu_bounded_cache import evict_case, make as mass_make
from tests.test_gpu_tree_attention import make as attention_make
from tests.test_gpu_tree_draft import make as commit_make

pytestmark = pytest.mark.gpu
I32 = torch.int32


def cuda(v):
    return torch.tensor(v, dtype=I32, device="cuda")


def mask_args():
    return dict(parents=cuda([[-1, 0, 0, 2], [-1, 0, 1, -2]]), start=cuda([7, 100]),
                mask=torch.empty(2, 4, dtype=torch.int64, device="cuda"), positions=torch.empty(2, 4, dtype=I32, device="cuda"),
                workspace=sfv.new_workspace(256))


def attention_args():
    a = [t.cuda() for t in attention_make([40, 3, 200], 12, 6, 2, 128, seed=1)[0]]
    ws = sfv.new_workspace(sfv.tree_attention_workspace_size(3, 12, 6, 2, 128, a[3].shape[1]))
    return dict(zip(["q", "k_cache", "v_cache", "block_table", "seq_lens", "mask"], a)) | dict(
        softmax_scale=0.0, out=torch.empty_like(a[0]), lse=torch.empty(3, 12, 6, device="cuda"), workspace=ws)


def commit_args():
    tokens, sampled, trees, kc, vc, bt, lens = commit_make([30, 5, None], 20, 2, 2, 64, seed=2, agree=0.9)
    out = [torch.empty_like(tokens, device="cuda") for _ in range(2)]
    return dict(tokens=tokens.cuda(), sampled=sampled.cuda(), parents=cuda(trees), k_caches=kc.cuda(), v_caches=vc.cuda(),
                block_table=bt.cuda(), seq_lens=cuda(lens), num_accepted=torch.empty(3, dtype=I32, device="cuda"),
                out_tokens=out[0], path=out[1], row_weights=torch.empty(3, 20, device="cuda"), n_q_next=None,
                free_pages=None, free_count=None, workspace=sfv.new_workspace(256))


def mass_args():
    a = [t.cuda() for t in mass_make([40, 3, 200], 12, 6, 2, 128, seed=3)]
    width = a[3].shape[1] * 16
    return dict(zip(["q", "lse", "k_cache", "block_table", "seq_lens"], a)) | dict(
        mass=torch.rand(3, 2, width, device="cuda", generator=torch.Generator("cuda").manual_seed(1)),
        row_weights=torch.ones(3, 12, device="cuda"), softmax_scale=0.0, out=torch.zeros(3, 2, width, device="cuda"),
        workspace=sfv.new_workspace(256))


def evict_args(longest=300):
    mass, kc, vc, bt, lens = evict_case([longest, 40, None], 2, 2, 64, seed=4)
    return dict(mass=mass.cuda(), k_caches=kc.cuda(), v_caches=vc.cuda(), block_table=bt.cuda(), seq_lens=cuda(lens),
                budget=64, first=1, recent=8, n_q=0, mass_out=torch.empty_like(mass, device="cuda"),
                seq_lens_out=torch.empty(3, dtype=I32, device="cuda"),
                kept=torch.empty(2, 3, 2, 64, dtype=I32, device="cuda"), free_pages=None, free_count=None,
                workspace=sfv.new_workspace(sfv.kv_evict_workspace_size(2, 3, 2, 64)))


OPS = [("tree_mask", mask_args), ("tree_attention", attention_args), ("tree_commit", commit_args),
       ("attention_mass", mass_args), ("kv_evict", evict_args)]


@pytest.fixture
def calls():
    require_gpu()
    assert sfv._calls is not None, "csrc/layer_calls.cpp was not built"
    return sfv._calls


@pytest.mark.parametrize("name, args", OPS)
def test_the_same_results(calls, name, args, monkeypatch):
    one, two = args(), args()
    assert getattr(calls, name)(*one.values()) == 0  # taken, without the binding's help
    monkeypatch.setattr(sfv, "_calls", None)
    getattr(sfv, name)(**two)
    torch.cuda.synchronize()
    for key, value in one.items():
        if isinstance(value, torch.Tensor):
            assert torch.equal(value.nan_to_num(), two[key].nan_to_num()), key


@pytest.mark.parametrize("name, args", OPS)
def test_leaves_what_is_not_as_it_should_be_to_the_binding(calls, name, args):
    # each tensor in turn: missing, on the host, of another type, with a dimension
    # less, of another size, not contiguous
    good = args()
    direct = getattr(calls, name)
    for at, (key, value) in enumerate(good.items()):
        if not isinstance(value, torch.Tensor):
            continue
        wrong = [object(), value.cpu(), value.to(torch.float64 if value.dtype.is_floating_point else torch.int16)]
        if key != "mask" or name == "tree_mask":
            wrong.append(value[0])  # (one mask is a tree for all sequences)
        # (the library compares a workspace with what it needs; twice the pages of the only
        # cache are a larger pool)
        if key != "workspace" and (name, key) != ("attention_mass", "k_cache"):
            wrong.append(torch.cat([value, value]))
        if value.dim() > 1 and value.shape[0] > 1:
            wrong.append(value.transpose(0, -1).contiguous().transpose(0, -1))
        for bad in wrong:
            v = list(good.values())
            v[at] = bad
            assert direct(*v) is None, (key, getattr(bad, "shape", bad))
    torch.cuda.synchronize()


def test_errors_of_the_binding_and_of_the_library(calls):
    kw = attention_args()
    kw["workspace"] = kw["workspace"][:256].clone()
    with pytest.raises(sfv.SFError) as e:
        sfv.tree_attention(**kw)
    assert e.value.status == 4
    kw = attention_args()
    with pytest.raises(ValueError, match="mask has shape"):
        sfv.tree_attention(**(kw | dict(mask=kw["mask"][:, :5])))
    with pytest.raises(TypeError, match="mask must be"):
        sfv.tree_attention(**(kw | dict(mask=kw["mask"].float())))
    kw = evict_args()
    with pytest.raises(sfv.SFError, match="first"):
        sfv.kv_evict(**(kw | dict(recent=64)))
    with pytest.raises(ValueError, match="numbers of layers"):
        sfv.kv_evict(**(kw | dict(v_caches=kw["v_caches"][:1])))
    with pytest.raises(ValueError, match="kept has layers of shape"):
        sfv.kv_evict(**(kw | dict(budget=65)))
    with pytest.raises(ValueError, match="belong together"):
        sfv.kv_evict(**(kw | dict(free_pages=cuda([0]))))
    kw = commit_args()
    with pytest.raises(ValueError, match="layers of shape"):
        sfv.tree_commit(**(kw | dict(v_caches=list(kw["v_caches"][:, 1:]))))
    with pytest.raises(sfv.SFError, match="n_q_next"):
        sfv.tree_commit(**(kw | dict(n_q_next=65, free_pages=cuda([0]), free_count=cuda([1]))))
    kw = mass_args()
    with pytest.raises(ValueError, match="out has shape"):
        sfv.attention_mass(**(kw | dict(out=kw["out"][..., :-1].contiguous())))
    with pytest.raises(ValueError, match="lse has shape"):
        sfv.attention_mass(**(kw | dict(lse=kw["lse"][:2])))


def test_two_streams_at_once(calls):
    # the same operators on two streams, each with its own workspace and outputs
    sets = [[args() for _, args in OPS] for _ in range(2)]
    for kw in sets[0]:
        for key, value in kw.items():
            if isinstance(value, torch.Tensor) and value.dtype is torch.bfloat16 and key == "q":
                value.mul_(0.5)
    want = []
    for group in sets:
        copies = [{k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in kw.items()} for kw in group]
        for (name, _), kw in zip(OPS, copies):
            getattr(sfv, name)(**kw)
        want.append(copies)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for stream, group in zip(streams, sets):
        with torch.cuda.stream(stream):
            for _ in range(20):
                for (name, _), kw in zip(OPS, group):
                    if name in ("tree_mask", "tree_attention", "attention_mass"):  # (the others change their caches)
                        getattr(sfv, name)(**kw)
            for (name, _), kw in zip(OPS, group):
                if name in ("tree_commit", "kv_evict"):
                    getattr(sfv, name)(**kw)
    torch.cuda.synchronize()
    for copies, group in zip(want, sets):
        for a, b in zip(copies, group):
            for key, value in a.items():
                if isinstance(value, torch.Tensor):
                    assert torch.equal(value.nan_to_num(), b[key].nan_to_num()), key


def test_a_step_captured_and_replayed(calls):
    """Masks, append, attention, commit, weights and eviction in one graph: every replay
    starts from the same state and ends in the same one as the calls themselves."""
    n, before, H_q, H_kv, d, layers = 14, [200, 37], 8, 2, 64, 2
    g = torch.Generator("cuda").manual_seed(5)
    pages = -(-(max(before) + 2 * n) // 16)
    k, v = torch.randn(2, layers, 2 * pages, H_kv, 16, d, device="cuda", generator=g).bfloat16()
    table = torch.arange(2 * pages, dtype=I32, device="cuda").view(2, pages)
    qkv = torch.randn(layers, 2 * n, H_q + 2 * H_kv, d, device="cuda", generator=g).bfloat16()
    parents = cuda([[-1, 0, 0, 0, 1, 1, 2, 2, 4, 4, 6, 8, 8, 11]] * 2)
    tokens = torch.arange(n, dtype=I32, device="cuda").expand(2, n).contiguous()
    sampled = cuda([[2, 0, 6, 0, 0, 0, 10, 0, 0, 0, 50, 0, 0, 0], [1, 4, 0, 0, 9, 0, 0, 0, 0, 60, 0, 0, 0, 0]])
    lens0 = cuda([x + n for x in before])
    free0, count0 = torch.full((8,), -1, dtype=I32, device="cuda"), cuda([0])
    freq = torch.linspace(1, 0.01, d // 2, dtype=torch.float64, device="cuda")
    mass = torch.zeros(layers, 2, H_kv, pages * 16, device="cuda")
    state = [t.clone() for t in (k, v, table, lens0, mass, free0, count0)]
    kc, vc, bt, lens, m, free, count = state
    lens_old, bt_old = torch.empty_like(lens), torch.empty_like(bt)
    outs = []

    def step():
        outs.clear()
        lens_old.copy_(lens)
        bt_old.copy_(bt)
        mask, positions = sfv.tree_mask(parents, lens_old - n)
        seen = []
        for layer in range(layers):
            q, kk, vv = qkv[layer].split([H_q, H_kv, H_kv], 1)
            q = sfv.kv_append(q, kk, vv, positions.view(1, -1), freq, kc[layer], vc[layer], bt, lens).view(2, n, H_q, d)
            out, lse = sfv.tree_attention(q, kc[layer], vc[layer], bt, lens, mask)
            seen.append((q, lse))
            outs.append(out)
        got = sfv.tree_commit(tokens, sampled, parents, kc, vc, bt, lens, n_q_next=n, free_pages=free, free_count=count)
        for layer, (q, lse) in enumerate(seen):
            sfv.attention_mass(q, lse, kc[layer], bt_old, lens_old, m[layer], row_weights=got[3], out=m[layer])
        sfv.kv_evict(m, kc, vc, bt, lens, 128, first=2, recent=16, n_q=n, free_pages=free, free_count=count)
        outs.extend(got)

    def reset():
        for a, b in zip(state, (k, v, table, lens0, mass, free0, count0)):
            a.copy_(b)

    step()
    want = [t.clone() for t in (*outs, *state)]
    assert want[2].tolist() == [3, 3] and want[4][0, :4].tolist() == [0, 2, 6, 10] and want[4][1, :4].tolist() == [0, 1, 4, 9]
    assert lens.tolist() == [128 + n, 37 + 4 + n] and int(count) > 0
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        reset()
        graph.replay()
        for a, b in zip((*outs, *state), want):
            assert torch.equal(a, b)


def test_attention_over_what_eviction_left(calls):
    # what was kept, moved to the front, gives what attention over the kept keys gives
    mass, kc, vc, bt, lens = evict_case([300, 90], 1, 2, 64, seed=7, n=5)
    n, budget = 5, 80
    for b in range(2):
        for j in range(n):  # rows that are still to come
            page, slot = ref.place(bt[b], lens[b] - n + j)
            kc[0, page, :, slot] = vc[0, page, :, slot] = 0
    k, v, sl, table, m = kc.cuda(), vc.cuda(), cuda(lens), bt.cuda(), mass.cuda()
    kept = torch.empty(1, 2, 2, budget, dtype=I32, device="cuda")
    sfv.kv_evict(m, k, v, table, sl, budget, recent=10, n_q=n, kept=kept)
    assert sl.tolist() == [85, 85]
    q = torch.randn(2, n, 4, 64, generator=torch.Generator().manual_seed(8)).bfloat16()
    rows = torch.randn(2, 2 * n, 2, 64, generator=torch.Generator().manual_seed(9)).bfloat16()
    sfv.kv_append(None, rows[0].cuda(), rows[1].cuda(), None, None, k[0], v[0], table, sl)
    words = [ref.masks([-1, 0, 0, 1, 3])] * 2
    out, lse = sfv.tree_attention(q.cuda(), k[0], v[0], table, sl, torch.tensor(words, device="cuda"))
    for b in range(2):
        for h in range(2):
            stay = kept[0, b, h].tolist()
            old = [ref.place(bt[b], t) for t in stay]
            keys, values = (torch.stack([c[0, p, h, s] for p, s in old] + list(x[b * n:(b + 1) * n, h])).double()
                            for c, x in ((kc, rows[0]), (vc, rows[1])))
            for i in range(n):
                at = ref.sees(i, budget, n, words[b][i])
                for j in range(2):
                    s = keys[at] @ q[b, i, 2 * h + j].double() / 8
                    w = torch.softmax(s, 0)
                    # (as in test_gpu_tree_attention.py)
                    tol = (w @ values[at].abs()) * (2.0 ** -8 + 2.0 ** -11) + (w @ values[at]).abs() * 2.0 ** -8 * (1 + 2.0 ** -6)
                    assert ((out[b, i, 2 * h + j].cpu().double() - w @ values[at]).abs() <= tol).all()
                    assert abs(float(lse[b, i, 2 * h + j]) - float(torch.logsumexp(s, 0))) <= 2.0 ** -11


@pytest.mark.parametrize("name, args", OPS[1:] + [("kv_evict", lambda: evict_args(200))])
def test_pages_more_than_32_bits_away(name, args):
    # the same pages at the end of a pool of 2^31 elements and more
    require_gpu()
    one, two = args(), args()
    pools = [k for k in two if k.endswith(("k_cache", "v_cache", "k_caches", "v_caches"))]
    small = one[pools[0]].shape[-4]
    many = 2 ** 31 // one[pools[0]].shape[-3:].numel() + 2 * small
    if name == "tree_attention":  # infinities are looked up in the cache
        for a in (one, two):
            t = int(a["seq_lens"][0]) - 2
            a["v_cache"][int(a["block_table"][0, t // 16]), :, t % 16, 3] = float("inf")
    for k in pools:
        shape = list(two[k].shape)
        shape[-4] = many
        big = torch.empty(shape, dtype=two[k].dtype, device="cuda")
        big[..., -small:, :, :, :] = two[k]
        two[k] = big
    two["block_table"] = torch.where(two["block_table"] >= 0, two["block_table"] + many - small, -1).to(I32)
    for a in (one, two):
        getattr(sfv, name)(**a)
        assert sfv.read_device_status(a["workspace"]) == 0
    for key, a in one.items():
        if isinstance(a, torch.Tensor) and key not in ("block_table", "workspace"):
            b = two[key][..., -small:, :, :, :] if key in pools else two[key]
            assert torch.equal(a.nan_to_num(-3), b.nan_to_num(-3)), key
