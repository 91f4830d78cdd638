"""Pins of the plain 64-bit implementations that the decoder-layer operators are
tested against (CPU)."""
import math

import torch

from tests import layer_reference as ref


def test_norm_of_equal_values_is_the_weight():
    x = torch.full((1, 7), -3.0)
    w = torch.arange(1, 8).double()
    y, h = ref.rms_norm(x, w, None, 0.0)
    assert torch.allclose(y, -w[None]) and torch.equal(h, x.double())
    y, h = ref.rms_norm(x, w, torch.full((1, 7), 4.0), 0.0)
    assert torch.allclose(y, w[None]) and torch.equal(h, torch.ones(1, 7).double())


def test_scales_reach_448_and_never_0():
    y = torch.tensor([[0.0] * 130, [896.0] + [1.0] * 129]).double()
    assert ref.scales(y, 0).tolist() == [[2.0 ** -126], [2.0]]
    assert torch.allclose(ref.scales(y, 128)[1], torch.tensor([2.0, 1 / 448]).double())


def test_rotation_keeps_scores_of_equal_distances():
    g = torch.Generator().manual_seed(0)
    q, k = torch.randn(2, 1, 1, 8, generator=g).unbind(0)
    f = torch.tensor([1.0, 0.5, 0.1, 0.01]).double()
    for inter in (False, True):
        at = lambda p: torch.tensor([[p]])  # noqa: E731
        dot = [(ref.rotate(q, at(a), f, None, inter) * ref.rotate(k, at(b), f, None, inter)).sum()
               for a, b in ((5, 3), (105, 103), (-7, -9))]
        assert abs(dot[0] - dot[1]) < 1e-12 and abs(dot[0] - dot[2]) < 1e-12
    one = ref.rotate(torch.tensor([[[1.0, 0.0]]]), torch.tensor([[1]]), torch.tensor([math.pi / 2], dtype=torch.float64), None, False)
    assert torch.allclose(one, torch.tensor([[[0.0, 1.0]]]).double())


def test_attention_over_a_prefix_is_the_softmax_over_all_tokens():
    g = torch.Generator().manual_seed(1)
    kc, vc = torch.randn(2, 4, 1, 16, 8, generator=g)
    q = torch.randn(2, 2, 2, 8, generator=g)
    out, lse, _ = ref.shared_prefix(q, kc, vc, torch.tensor([[3, 1]]), [20], [0, 2], torch.tensor([[0], [2]]), [2, 5])
    for b, L in ((0, 2), (1, 5)):
        own = 0 if b == 0 else 2
        k = torch.cat([kc[3, 0], kc[1, 0, :4], kc[own, 0, :L]]).double()
        v = torch.cat([vc[3, 0], vc[1, 0, :4], vc[own, 0, :L]]).double()
        for i in range(2):
            n = 20 + L - 1 + i
            s = (q[b, i].double() @ k[:n].T) / math.sqrt(8)
            assert torch.allclose(out[b, i], torch.softmax(s, 1) @ v[:n])
            assert torch.allclose(lse[b, i], s.exp().sum(1).log())
    out, lse, _ = ref.shared_prefix(q, kc, vc, torch.tensor([[3, 1]]), [20], [0, 2], torch.tensor([[0], [2]]), [0, 5])
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
