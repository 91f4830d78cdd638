"""The plain implementations of the tree and eviction operators, by hand-worked and
closed-form cases."""
import math

import torch

from tests import tree_reference as ref


def table_of(pages):
    return torch.arange(pages, dtype=torch.int32)[None]


def test_masks_of_a_hand_worked_tree():
    #        0 -> 1 -> 3, 0 -> 2 -> 4 -> 5; 6 is a root of its own; 7 and 8 are not part of the tree
    assert ref.masks([-1, 0, 0, 1, 2, 4, -1, -2, 7]) == [1, 0b11, 0b101, 0b1011, 0b10101, 0b110101, 1 << 6, 0, 0]
    assert ref.masks([-1, 1, 5, 0]) == [1, 0, 0, 0b1001]  # entries that are not below their row
    assert ref.signed(1 << 63) == -(1 << 63) and ref.signed(5) == 5


def test_path_takes_the_lowest_matching_child_and_stops():
    parents = [-1, 0, 0, 0, 1, 2, 2, 6]
    tokens = [9, 4, 7, 7, 1, 3, 5, 8]
    assert ref.path(parents, tokens, [7, 0, 5, 0, 0, 0, 8, 2]) == [0, 2, 6, 7]
    assert ref.path(parents, tokens, [4, 2, 5, 0, 0, 0, 8, 2]) == [0, 1]
    assert ref.path(parents, tokens, [6, 2, 5, 0, 0, 0, 8, 2]) == [0]


def test_attention_of_equal_keys_is_the_mean_of_what_is_seen():
    n, d = 3, 64
    v = torch.randn(1, 1, 16, d).bfloat16()
    k = torch.zeros(1, 1, 16, d).bfloat16()
    q = torch.randn(1, n, 1, d).bfloat16()
    out, lse, _ = ref.attention(q, k, v, table_of(1), torch.tensor([8]), [[0b001, 0b011, 0b101]])
    for i, at in enumerate(([0, 1, 2, 3, 4, 5], [0, 1, 2, 3, 4, 5, 6], [0, 1, 2, 3, 4, 5, 7])):
        assert (out[0, i, 0] - v[0, 0, at].double().mean(0)).abs().max() < 1e-12
        assert abs(lse[0, i, 0] - math.log(len(at))) < 1e-12
    out, lse, _ = ref.attention(q, k, v, table_of(1), torch.tensor([3]), [[0, 0b011, 0b101]])
    assert not out[0, 0].any() and lse[0, 0, 0] == -math.inf


def test_chain_masks_give_causal_attention():
    g = torch.Generator().manual_seed(1)
    n, d = 4, 64
    k, v = torch.randn(2, 2, 1, 16, d, generator=g).bfloat16()
    q = torch.randn(1, n, 1, d, generator=g).bfloat16()
    out, _, _ = ref.attention(q, k, v, table_of(2), torch.tensor([20]), [[(2 << i) - 1 for i in range(n)]])
    kk, vv = k.reshape(-1, d).double(), v.reshape(-1, d).double()
    for i in range(n):
        w = torch.softmax(kk[:17 + i] @ q[0, i, 0].double() / 8, 0)
        assert (out[0, i, 0] - w @ vv[:17 + i]).abs().max() < 1e-12


def test_mass_of_a_context_sums_to_the_rows_share_of_it():
    g = torch.Generator().manual_seed(2)
    n, d = 3, 64
    k, v = torch.randn(2, 2, 2, 16, d, generator=g).bfloat16()
    q = torch.randn(1, n, 4, d, generator=g).bfloat16()
    _, lse, _ = ref.attention(q, k, v, table_of(2), torch.tensor([20]), [[0, 0, 0]])
    total, bound = ref.mass(q, lse, k, table_of(2), torch.tensor([20]), torch.tensor([[1.0, 0.0, 0.5]]))
    # no row sees an own key, so each of a KV head's two query heads gives its weight away
    assert (total.sum(2) - 3.0).abs().max() < 1e-12 and (bound < 1e-3).all()


def test_kept_positions():
    row = [0.5, 0.1, 0.9, 0.1, math.nan, 0.3, -1.0, 0.2]
    assert ref.kept(row, 8, 8, 0, 0) == list(range(8)) and ref.kept(row, 3, 5, 0, 0) == [0, 1, 2]
    assert ref.kept(row, 8, 3, 0, 0) == [0, 2, 5]
    assert ref.kept(row, 8, 4, 0, 2) == [0, 2, 6, 7]
    assert ref.kept(row, 8, 6, 0, 0) == [0, 1, 2, 3, 5, 7]  # the first of two equal ones, then the second
    assert ref.kept(row, 8, 5, 0, 0) == [0, 1, 2, 5, 7]
    assert ref.kept(row, 8, 2, 1, 1) == [0, 7]
    assert ref.kept(row, 8, 7, 0, 0) == [0, 1, 2, 3, 5, 6, 7]
