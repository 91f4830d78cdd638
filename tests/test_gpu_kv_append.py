"""sf_kv_append against the 64-bit rotation and a row-by-row append (GPU).

Tolerance of a rotated element u = a cos - b sin: the fixed-point turn is exact
but for 2^-32 turns and 2^-53 * position of the step's rounding (below 2^-28 at
the positions used here); its rounding to fp32 is 2^-24 of the angle (pi at
most), and sincospif is within 2 ulp, so cos and sin are within 2^-21; the
products and their sum add 2 * 2^-24.  |u - exact| <= (|a| + |b|) * 2^-20, and half a
bf16 ulp of the output.  Copied elements are equal bit for bit (bf16) or rounded
once (fp32)."""
import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import layer_reference as ref
from tests.gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu


def make(T, H_q, H_kv, d, pairs, axes, kind, seed, fused=True, top=40000):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(T, (H_q + 2 * H_kv) * d, generator=g).to(kind)
    pos = torch.randint(-50, top, (max(axes, 1), T), generator=g, dtype=torch.int32)
    f = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))
    axis = torch.randint(0, axes, (pairs,), generator=g, dtype=torch.int32) if axes > 1 else None
    return qkv, pos, f, axis


def split(qkv, H_q, H_kv, d):
    return [t.unflatten(1, (-1, d)) for t in qkv.split([H_q * d, H_kv * d, H_kv * d], 1)]


def tables(B, lens, max_pages, seed):
    """Block table over a permuted pool with a few spare pages; -1 past the ends."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // 16) for n in lens]
    pool = sum(need) + 3
    ids = torch.randperm(pool, generator=g).int()
    t, at = torch.full((B, max_pages), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        t[b, :n] = ids[at:at + n]
        at += n
    return t, pool


def check_rotated(got, x, want, pairs, inter):
    """got bf16 against want fp64; x the input."""
    x = x.double().abs()
    tol = ref.bf16_half_ulp(want) * (1 + 2.0 ** -8)
    size = torch.zeros_like(x)
    n = pairs
    if inter:
        s = x[..., 0:2 * n:2] + x[..., 1:2 * n:2]
        size[..., 0:2 * n:2] = size[..., 1:2 * n:2] = s
    else:
        s = x[..., :n] + x[..., n:2 * n]
        size[..., :n] = size[..., n:2 * n] = s
    err = (got.double() - want).abs()
    assert (err <= tol + size * 2.0 ** -20).all(), (err - tol).max()


def run_and_check(T, B, lens, row_starts, H_q, H_kv, d, pairs, axes, kind, inter, seed, max_pages=None, amplitude=1.0,
                  views=None):
    require_gpu()
    qkv, pos, f, axis = make(T, H_q, H_kv, d, pairs, axes, kind, seed)
    q, k, v = split(qkv, H_q, H_kv, d)
    dq, dk, dv = (views or split)(qkv.cuda(), H_q, H_kv, d)
    max_pages = max_pages or max(1, max(-(-n // 16) for n in lens) + 1)
    table, pool = tables(B, lens, max_pages, seed)
    g = torch.Generator().manual_seed(seed + 1)
    kc, vc = torch.randn(2, pool, H_kv, 16, d, generator=g).bfloat16()
    dkc, dvc = kc.cuda(), vc.cuda()
    starts = None if row_starts is None else torch.tensor(row_starts, dtype=torch.int32)
    ws = sfv.new_workspace(sfv.kv_append_workspace_size())
    out = sfv.kv_append(dq if H_q else None, dk, dv, pos.cuda() if pairs else None, f.cuda() if pairs else None, dkc, dvc,
                        table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                        axis=None if axis is None else axis.cuda(), row_starts=None if starts is None else starts.cuda(),
                        interleaved=inter, amplitude=amplitude, workspace=ws)
    assert sfv.read_device_status(ws) == 0
    if H_q:
        check_rotated(out.cpu(), q, ref.rotate(q, pos, f, axis, inter, amplitude), pairs, inter)
    else:
        assert out is None
    want_k = ref.rotate(k, pos, f, axis, inter, amplitude)
    got_k, got_v = dkc.cpu(), dvc.cpu()
    touched = torch.zeros(pool, 16, dtype=torch.bool)
    for t, place in enumerate(ref.places(T, B, lens, row_starts, table)):
        if place is None:
            continue
        page, slot = place
        assert not touched[page, slot]
        touched[page, slot] = True
        check_rotated(got_k[page, :, slot], k[t], want_k[t], pairs, inter)
        assert torch.equal(got_v[page, :, slot], v[t].bfloat16())
    same = ~touched[:, None, :, None]
    assert torch.equal(got_k * same, kc * same) and torch.equal(got_v * same, vc * same)


HEADS = [(8, 8, 64), (28, 4, 128), (1, 1, 8), (6, 2, 80), (5, 5, 256), (0, 3, 64), (32, 32, 128)]


@pytest.mark.parametrize("H_q, H_kv, d", HEADS)
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
def test_uniform_rows(H_q, H_kv, d, kind, inter):
    # full rotation, half of the head, an odd number of pairs, none
    for n, pairs in enumerate((d // 2, d // 4, 3, 0)):
        run_and_check(T=12, B=3, lens=[4, 37, 16], row_starts=None, H_q=H_q, H_kv=H_kv, d=d, pairs=pairs,
                      axes=(1, 3, 4, 1)[n], kind=kind, inter=inter, seed=100 * d + n, amplitude=(1.0, 1.25, 1.0, 1.0)[n])


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33])
def test_numbers_of_rows(rows):
    run_and_check(T=2 * rows, B=2, lens=[rows, rows + 21], row_starts=None, H_q=4, H_kv=2, d=64, pairs=32, axes=1,
                  kind=torch.bfloat16, inter=False, seed=rows)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_ragged_prompts_with_empty_sequences_and_padding(kind):
    # sequence 1 brings no rows, 3 appends behind 40 tokens, rows 100.. are padding
    run_and_check(T=107, B=5, lens=[63, 20, 1, 49, 27], row_starts=[0, 63, 63, 64, 73, 100], H_q=28, H_kv=4, d=128,
                  pairs=64, axes=3, kind=kind, inter=False, seed=11)


def test_many_rows_and_sequences():
    n = [1 + (7 * b) % 29 for b in range(200)]
    starts = [0]
    for m in n:
        starts.append(starts[-1] + m)
    run_and_check(T=starts[-1], B=200, lens=[m + 5 * b % 40 for b, m in enumerate(n)], row_starts=starts, H_q=3, H_kv=1,
                  d=64, pairs=32, axes=1, kind=torch.bfloat16, inter=False, seed=12)


def test_idle_slots_are_left_out():
    run_and_check(T=12, B=4, lens=[0, 18, 0, 3], row_starts=None, H_q=4, H_kv=2, d=64, pairs=32, axes=1,
                  kind=torch.bfloat16, inter=False, seed=13)


def test_strides_and_alignments():
    def heads_first(qkv, H_q, H_kv, d):  # [heads][T][d] memory
        return [t.transpose(0, 1).contiguous().transpose(0, 1) for t in split(qkv, H_q, H_kv, d)]

    def odd_offset(qkv, H_q, H_kv, d):  # rows that start one element off, an odd row stride
        out = []
        for t in split(qkv, H_q, H_kv, d):
            big = torch.zeros(t.shape[0], t.shape[1] * d + 3, dtype=t.dtype, device=t.device)
            view = big[:, 1:1 + t.shape[1] * d].unflatten(1, (-1, d))
            view.copy_(t)
            out.append(view)
        return out

    def broadcast_rows(qkv, H_q, H_kv, d):  # one v for every head: a stride of 0
        q, k, v = split(qkv, H_q, H_kv, d)
        return q, k, v

    for n, views in enumerate((heads_first, odd_offset, broadcast_rows)):
        for kind in (torch.bfloat16, torch.float32):
            run_and_check(T=10, B=2, lens=[5, 19], row_starts=None, H_q=6, H_kv=3, d=64, pairs=16, axes=2, kind=kind,
                          inter=bool(n % 2), seed=20 + n, views=views)


def test_q_in_place():
    require_gpu()
    for inter in (False, True):
        qkv, pos, f, _ = make(9, 4, 2, 128, 64, 1, torch.bfloat16, 30)
        q, k, v = (t.contiguous().cuda() for t in split(qkv, 4, 2, 128))
        kc = torch.zeros(2, 2, 16, 128, dtype=torch.bfloat16, device="cuda")
        args = (k, v, pos.cuda(), f.cuda(), kc, kc.clone(), torch.tensor([[0, 1]], dtype=torch.int32).cuda(),
                torch.tensor([9], dtype=torch.int32).cuda())
        a = sfv.kv_append(q, *args, interleaved=inter)
        b = sfv.kv_append(q, *args, interleaved=inter, q_out=q)
        assert b is q and torch.equal(a, b)


def test_far_positions():
    # fixed-point turns: the error does not grow with the position
    require_gpu()
    pos = torch.tensor([[2 ** 24 - 3, -(2 ** 24), 1 << 20, 0]], dtype=torch.int32)
    f = 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)
    k = torch.randn(4, 2, 64, generator=torch.Generator().manual_seed(5)).bfloat16()
    kc = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    sfv.kv_append(None, k.cuda(), k.cuda(), pos.cuda(), f.cuda(), kc, kc.clone(), torch.zeros(1, 1, dtype=torch.int32).cuda(),
                  torch.tensor([4], dtype=torch.int32).cuda())
    check_rotated(kc[0, :, :4].transpose(0, 1).cpu(), k, ref.rotate(k, pos, f, None, False), 32, False)


def test_device_data_errors_are_flagged_and_skipped():
    require_gpu()
    k = torch.ones(8, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(1, 8, dtype=torch.int32, device="cuda")
    f = torch.ones(32, dtype=torch.float64, device="cuda")

    def call(table, lens, row_starts=None, axis=None):
        kc = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
        ws = sfv.new_workspace(sfv.kv_append_workspace_size())
        i = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        sfv.kv_append(None, k, k, pos, f, kc, kc.clone(), i(table), i(lens), row_starts=i(row_starts),
                      axis=None if axis is None else torch.full((32,), axis, dtype=torch.int32, device="cuda"), workspace=ws)
        return sfv.read_device_status(ws), int((kc != 0).any(3).any(1).sum())

    assert call([[0, 1], [2, 3]], [4, 32]) == (0, 8)
    assert call([[4, 1], [2, -1]], [4, 32]) == (sfv.SF_DEVICE_BAD_PAGE, 0)
    assert call([[0, 1], [2, 3]], [3, 34]) == (sfv.SF_DEVICE_BAD_SEQLEN, 5)
    assert call([[0, 1], [2, 3]], [-5, 2 ** 31 - 1]) == (sfv.SF_DEVICE_BAD_SEQLEN, 0)
    assert call([[0, 1], [2, 3]], [4, 4], row_starts=[2, 5, 8]) == (sfv.SF_DEVICE_BAD_INDEX, 6)
    assert call([[0, 1], [2, 3]], [4, 4], axis=1) == (sfv.SF_DEVICE_BAD_INDEX, 8)
    assert call([[0, 1], [2, 3]], [4, 4], axis=-1) == (sfv.SF_DEVICE_BAD_INDEX, 8)


def test_no_rows_and_refusals():
    require_gpu()
    kc = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    bt, sl = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    pos, f = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda")
    e = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert sfv.kv_append(e, e, e, pos[:, :0], f, kc, kc, bt, sl).shape == (0, 2, 64)
    k = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="v has shape"):
        sfv.kv_append(None, k, k[:, :1], pos, f, kc, kc, bt, sl)
    with pytest.raises(TypeError, match="v must be"):
        sfv.kv_append(None, k, k.float(), pos, f, kc, kc, bt, sl)
    with pytest.raises(ValueError, match="positions"):
        sfv.kv_append(None, k, k, pos[:, :3].contiguous(), f, kc, kc, bt, sl)
    with pytest.raises(ValueError, match="positions"):
        sfv.kv_append(None, k, k, None, f, kc, kc, bt, sl)
    with pytest.raises(ValueError, match="need inv_freq"):
        sfv.kv_append(None, k, k, pos, None, kc, kc, bt, sl)
    with pytest.raises(TypeError, match="float64"):
        sfv.kv_append(None, k, k, pos, f.float(), kc, kc, bt, sl)
    with pytest.raises(ValueError, match="axis has shape"):
        sfv.kv_append(None, k, k, pos, f, kc, kc, bt, sl, axis=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="k_cache has shape"):
        sfv.kv_append(None, k, k, pos, f, kc[:, :1].contiguous(), kc, bt, sl)
    with pytest.raises(ValueError, match="row_starts has shape"):
        sfv.kv_append(None, k, k, pos, f, kc, kc, bt, sl, row_starts=sl)
    with pytest.raises(ValueError, match="q_out needs"):
        sfv.kv_append(None, k, k, pos, f, kc, kc, bt, sl, q_out=k)
    with pytest.raises(sfv.SFError, match="rotary_dim"):
        sfv.kv_append(None, k, k, pos, torch.ones(33, dtype=torch.float64, device="cuda"), kc, kc, bt, sl)
    with pytest.raises(sfv.SFError, match="multiple of B"):
        sfv.kv_append(None, k[:3], k[:3], pos[:, :3].contiguous(), f, kc, kc, bt, sl)


def test_attention_reads_what_was_appended():
    # append then verify_attention of the same draft rows, back to back on the stream
    require_gpu()
    H_q, H_kv, d, n_q, lens = 8, 2, 64, 4, [100, 37]
    qkv, pos, f, _ = make(2 * n_q, H_q, H_kv, d, 32, 1, torch.bfloat16, 40)
    q, k, v = split(qkv, H_q, H_kv, d)
    table, pool = tables(2, lens, 8, 41)
    kc, vc = torch.randn(2, pool, H_kv, 16, d, generator=torch.Generator().manual_seed(42)).bfloat16()
    dk, dv = kc.cuda(), vc.cuda()
    sl = torch.tensor(lens, dtype=torch.int32)
    rq = sfv.kv_append(*(t.cuda() for t in (q, k, v)), pos.cuda(), f.cuda(), dk, dv, table.cuda(), sl.cuda())
    out, lse = sfv.verify_attention(rq.view(2, n_q, H_q, d), dk, dv, table.cuda(), sl.cuda())
    want, want_lse, spread = ref.shared_prefix(rq.cpu().view(2, n_q, H_q, d), dk.cpu(), dv.cpu(), table, [0, 0], [0, 1, 2],
                                               table, lens)
    assert ((out.double().cpu() - want).abs() <= ref.bf16_half_ulp(want) * 1.01 + spread * 2.0 ** -8).all()
    assert (lse.double().cpu() - want_lse).abs().max() <= 1e-3
