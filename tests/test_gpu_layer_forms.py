"""Forms in which the decoder-layer operators' arguments come (GPU): a single row whose
stride means nothing."""
import pytest
import torch

from paper_2505_12728_gb300 import specflash_verify as sfv
from tests.gpu_helpers import require_gpu

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
