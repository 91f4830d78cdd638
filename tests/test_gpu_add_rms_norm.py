"""sf_add_rms_norm against the 64-bit norm (GPU).

Tolerances.  y is an fp32 product of h, the inverse root mean square and the
weight.  h itself is rounded once (2^-24).  The sum of d <= 32768 squares is
taken in at most 128 sequential and 15 tree additions per term, so its relative
error stays below 150 * 2^-24, half of it through the root; with the roundings
of the root, the division and the two products y is within 2^-17 of exact.  The
output adds half a bf16 ulp, or half an e4m3 ulp of y / scale times the scale
(the division and the scale's own rounding are part of the 2^-17)."""
import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests import layer_reference as ref
from tests.gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu
REL = 2.0 ** -17


def make(T, d, kind, seed, residual=True, wkind=torch.bfloat16, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (scale * torch.randn(T, d, generator=g)).to(kind)
    r = (3 * scale * torch.randn(T, d, generator=g)).to(kind) if residual else None
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(wkind)
    return x, r, w


def check(got, x, r, w, eps, group):
    out, r_out, scales = got
    y, h = ref.rms_norm(x, w, r, eps)
    if r is None:
        assert r_out is None
    else:
        err = (r_out.double().cpu() - h).abs()
        half = ref.bf16_half_ulp(h) if x.dtype is torch.bfloat16 else h.abs() * 2.0 ** -24
        assert (err <= half * (1 + 2.0 ** -12) + h.abs() * 2.0 ** -23).all()
    if scales is None:
        assert out.dtype is torch.bfloat16
        err, tol = (out.double().cpu() - y).abs(), ref.bf16_half_ulp(y) * (1 + 2.0 ** -8) + y.abs() * REL
    else:
        s = ref.scales(y, group)
        assert ((scales.double().cpu() - s).abs() <= s * REL).all()
        s = scales.double().cpu().repeat_interleave(group or y.shape[1], 1)[:, :y.shape[1]]
        err = (out.float().double().cpu() * s - y).abs()
        tol = ref.e4m3_half_ulp(y / s) * s * (1 + 2.0 ** -8) + y.abs() * REL
    assert (err <= tol).all(), (err / tol).max()


# widths around vectors, warps, groups and blocks; rows from one
SIZES = [(1, 1), (3, 7), (2, 64), (5, 100), (3, 128), (4, 129), (7, 1000), (2, 1155), (5, 2048), (9, 3584), (16, 4096),
         (3, 8192), (2, 8200), (3, 16384), (2, 20001), (1, 32768), (300, 256)]


@pytest.mark.parametrize("T, d", SIZES)
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("out, group", [("bf16", 0), ("e4m3", 0), ("e4m3", 128)])
def test_norm_matches(T, d, kind, out, group):
    require_gpu()
    for residual in (True, False):
        x, r, w = make(T, d, kind, seed=T * 100000 + d, residual=residual)
        got = sfv.add_rms_norm(x.cuda(), w.cuda(), None if r is None else r.cuda(), eps=1e-5, group=group,
                               out_dtype=torch.float8_e4m3fn if out == "e4m3" else torch.bfloat16)
        check(got, x, r, w, 1e-5, group)


@pytest.mark.parametrize("pad, offset", [(8, 0), (8, 8), (1, 0), (3, 1), (4, 2)])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_strided_rows_and_unaligned_bases(pad, offset, kind):
    require_gpu()
    T, d = 6, 640

    def strided(t):
        big = torch.full((T, d + pad + offset), 7.0, dtype=t.dtype, device="cuda")
        view = big[:, offset:offset + d]
        view.copy_(t)
        return big, view

    x, r, w = make(T, d, kind, seed=pad * 10 + offset, wkind=torch.float32)
    (_, xs), (_, rs) = strided(x), strided(r)
    for out_dtype, group in ((torch.bfloat16, 0), (torch.float8_e4m3fn, 128)):
        ob, o = strided(torch.zeros(T, d, dtype=out_dtype))
        rb, ro = strided(torch.zeros(T, d, dtype=kind))
        got = sfv.add_rms_norm(xs, w.cuda(), rs, eps=0.0, group=group, out=o, residual_out=ro)
        check(got, x, r, w, 0.0, group)
        for big in (ob, rb):  # nothing past the rows is written
            side = torch.ones(d + pad + offset, dtype=torch.bool, device="cuda")
            side[offset:offset + d] = False
            assert (big[:, side].float() == 7.0).all()


def test_in_place_forms_equal_the_separate_ones():
    require_gpu()
    for d in (512, 515):
        x, r, w = make(33, d, torch.bfloat16, seed=d)
        a, ra, _ = sfv.add_rms_norm(x.cuda(), w.cuda(), r.cuda())
        xs, rs = x.cuda(), r.cuda()
        b, rb, _ = sfv.add_rms_norm(xs, w.cuda(), rs, residual_out=rs, out=xs)
        assert b is xs and rb is rs
        assert torch.equal(a, b) and torch.equal(ra, rb)


def test_zero_rows_tiny_and_huge_values():
    require_gpu()
    x = torch.zeros(4, 256)
    x[1] = 1e-30
    x[2] = 1e18
    x[3, 5] = 1.0
    w = torch.ones(256)
    for group in (0, 128):
        out, _, s = sfv.add_rms_norm(x.cuda(), w.cuda(), None, eps=1e-6, out_dtype=torch.float8_e4m3fn, group=group)
        check((out, None, s), x, None, w, 1e-6, group)
        assert (s[0] == 2.0 ** -126).all() and (out[0].float() == 0).all()
    out, _, _ = sfv.add_rms_norm(torch.zeros(1, 256, device="cuda"), w.cuda(), None, eps=0.0)
    assert out.isnan().all()  # 0 / 0, as the formula says


def test_nan_and_infinity_stay_in_their_rows():
    require_gpu()
    x, r, w = make(5, 384, torch.float32, seed=3)
    x[1, 200] = float("nan")
    x[3, 7] = float("inf")
    out, r_out, s = sfv.add_rms_norm(x.cuda(), w.cuda(), r.cuda(), eps=1e-6, out_dtype=torch.float8_e4m3fn, group=128)
    keep = [0, 2, 4]
    check((out[keep], r_out[keep], s[keep]), x[keep], r[keep], w, 1e-6, 128)
    assert out[1].float().isnan().all() and s[1].isnan().all()
    # h / inf = 0 but for the infinity itself, whose group's scale is NaN
    assert (out[3, 128:].float() == 0).all() and s[3, 0].isnan() and out[3, 7].float().isnan()


def test_no_rows_and_refusals():
    require_gpu()
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out, r, s = sfv.add_rms_norm(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), w)
    assert out.shape == (0, 64)
    x = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="residual has shape"):
        sfv.add_rms_norm(x, w, x[:2])
    with pytest.raises(TypeError, match="residual must be"):
        sfv.add_rms_norm(x, w, x.float())
    with pytest.raises(ValueError, match="weight has shape"):
        sfv.add_rms_norm(x, w[:32])
    with pytest.raises(ValueError, match="last dimension"):
        sfv.add_rms_norm(torch.ones(64, 4, dtype=torch.bfloat16, device="cuda").t(), w)
    with pytest.raises(ValueError, match="scales and group"):
        sfv.add_rms_norm(x, w, group=128)
    with pytest.raises(ValueError, match="group=64"):
        sfv.add_rms_norm(x, w, group=64, out_dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="needs a residual"):
        sfv.add_rms_norm(x, w, residual_out=x)
    with pytest.raises(TypeError, match="out must be"):
        sfv.add_rms_norm(x, w, out=x.float())
    with pytest.raises(sfv.SFError) as e:
        sfv.add_rms_norm(x, w, eps=-1.0)
    assert e.value.status == 1


def test_on_another_stream():
    require_gpu()
    x, r, w = make(64, 4096, torch.bfloat16, seed=9)
    xs, rs, ws = x.cuda(), r.cuda(), w.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = sfv.add_rms_norm(xs, ws, rs, eps=1e-6, out_dtype=torch.float8_e4m3fn, stream=side)
    side.synchronize()
    check(got, x, r, w, 1e-6, 0)


# rows that start anywhere between 16-byte boundaries, in all tensors alike or not;
# one row a CTA, several, and two chunks a thread
@pytest.mark.parametrize("T, d, stride, offset, apart", [
    (2600, 1, 1, 0, 0), (2600, 9, 11, 3, 0), (3000, 129, 129, 0, 0), (1300, 777, 777, 5, 0), (5, 5001, 5002, 7, 0),
    (700, 3589, 3589, 1, 0), (1300, 640, 643, 5, 0), (700, 333, 333, 2, 1), (40, 4097, 4097, 0, 3), (3, 20001, 20001, 6, 0)])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("out_dtype, group", [(torch.bfloat16, 0), (torch.float8_e4m3fn, 0), (torch.float8_e4m3fn, 128)])
def test_rows_between_boundaries(T, d, stride, offset, apart, kind, out_dtype, group):
    require_gpu()

    def rows(t, at):
        big = torch.full((at + T * stride + 16,), 7.0, device="cuda").to(t.dtype)
        view = big.as_strided((T, d), (stride, 1), at)
        view.copy_(t)
        return big, view

    x, r, w = make(T, d, kind, seed=T + d)
    bad = T // 2  # its neighbours share 16 bytes with it and keep their values
    x[bad] = float("nan")
    (_, xs), (_, rs) = rows(x, offset), rows(r, offset + apart)
    ob, o = rows(torch.zeros(T, d, dtype=out_dtype), offset)
    rb, ro = rows(torch.zeros(T, d, dtype=kind), offset)
    out, r_out, sc = sfv.add_rms_norm(xs, w.cuda(), rs, eps=1e-6, group=group, out=o, residual_out=ro)
    good = torch.arange(T) != bad
    check((out[good.cuda()], r_out[good.cuda()], None if sc is None else sc[good.cuda()]), x[good], r[good], w, 1e-6, group)
    assert out[bad].float().isnan().all() and r_out[bad].isnan().all()
    inside = torch.zeros(ob.numel(), dtype=torch.bool, device="cuda")
    inside.as_strided((T, d), (stride, 1), offset).fill_(True)
    for big in (ob, rb):
        assert (big.float()[~inside] == 7.0).all()


# narrow rows in number: a warp each, the last CTA not full
@pytest.mark.parametrize("T, d", [(1217, 256), (1220, 248), (1301, 249), (4999, 64), (2001, 136), (1999, 255)])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("out_dtype, group", [(torch.bfloat16, 0), (torch.float8_e4m3fn, 0), (torch.float8_e4m3fn, 128)])
def test_many_narrow_rows(T, d, kind, out_dtype, group):
    require_gpu()
    for residual in (True, False):
        x, r, w = make(T, d, kind, seed=T + d, residual=residual, wkind=torch.float32)
        got = sfv.add_rms_norm(x.cuda(), w.cuda(), None if r is None else r.cuda(), eps=1e-5, group=group,
                               out_dtype=out_dtype)
        check(got, x, r, w, 1e-5, group)
