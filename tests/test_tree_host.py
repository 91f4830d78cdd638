"""Refusals of the tree and eviction operators that need no GPU: the library checks
its arguments before it touches the device, the binding before the library."""
import ctypes

import pytest
import torch

from paper_2505_12728_gb300 import build_lib
from paper_2505_12728_gb300 import specflash_verify as sfv

FAKE = ctypes.c_void_p(256)
ODD = ctypes.c_void_p(257)


def pointers(*values):
    return (ctypes.c_void_p * max(1, len(values)))(*values)


TWO = pointers(256, 512)


@pytest.fixture(scope="module")
def lib():
    build_lib.build()
    return sfv.load_library()


def mask_args(**kw):
    a = dict(parents=FAKE, start=FAKE, B=2, n=5, mask=FAKE, positions=FAKE, workspace=FAKE, bytes=256, stream=None)
    assert not kw.keys() - a.keys()
    return [*(a | kw).values()]


@pytest.mark.parametrize("bad, status", [
    (dict(B=0), 1), (dict(B=1025), 1), (dict(n=0), 1), (dict(n=65), 1), (dict(parents=None), 1), (dict(mask=None), 1),
    (dict(mask=ctypes.c_void_p(260)), 1), (dict(parents=ODD), 1), (dict(start=ODD), 1), (dict(positions=ODD), 1),
    (dict(workspace=None), 4), (dict(workspace=ctypes.c_void_p(128)), 4), (dict(bytes=255), 4)])
def test_tree_mask_refuses(lib, bad, status):
    assert lib.sf_tree_mask(*mask_args(**bad)) == status
    assert lib.sf_last_error()


def attention_args(**kw):
    a = dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, block_table=FAKE, seq_lens=FAKE, mask=FAKE, mask_stride=4, B=2, n_q=4,
             H_q=8, H_kv=8, head_dim=64, page_size=16, num_pages=10, max_pages=4, softmax_scale=0.0, out=FAKE, lse=None,
             workspace=FAKE, bytes=1 << 40, stream=None)
    assert not kw.keys() - a.keys()
    return [*(a | kw).values()]


SHAPES = [
    (dict(B=0), 1), (dict(B=1025), 1), (dict(n_q=0), 1), (dict(n_q=65), 1), (dict(H_q=7, H_kv=2), 1), (dict(H_kv=0), 1),
    (dict(H_q=18, H_kv=2), 2), (dict(head_dim=96), 2), (dict(page_size=8), 2), (dict(max_pages=0), 1),
    (dict(max_pages=1 << 27), 1), (dict(num_pages=0), 1), (dict(num_pages=1 << 25), 2), (dict(softmax_scale=-1.0), 1),
    (dict(softmax_scale=float("nan")), 1), (dict(softmax_scale=float("inf")), 1), (dict(q=None), 1),
    (dict(k_cache=None), 1), (dict(block_table=None), 1), (dict(seq_lens=None), 1), (dict(q=ctypes.c_void_p(264)), 1),
    (dict(k_cache=ctypes.c_void_p(264)), 1), (dict(seq_lens=ODD), 1), (dict(block_table=ODD), 1), (dict(lse=ODD), 1),
    (dict(workspace=None), 4), (dict(workspace=ctypes.c_void_p(16)), 4)]


@pytest.mark.parametrize("bad, status", SHAPES + [
    (dict(v_cache=None), 1), (dict(mask=None), 1), (dict(out=None), 1), (dict(mask=ctypes.c_void_p(260)), 1),
    (dict(mask_stride=3), 1), (dict(mask_stride=-4), 1), (dict(out=ctypes.c_void_p(264)), 1)])
def test_tree_attention_refuses(lib, bad, status):
    assert lib.sf_tree_attention(*attention_args(**bad)) == status
    assert lib.sf_last_error()


def mass_args(**kw):
    a = dict(q=FAKE, lse=FAKE, k_cache=FAKE, block_table=FAKE, seq_lens=FAKE, mass=None, weights=None, B=2, n_q=4, H_q=8,
             H_kv=8, head_dim=64, page_size=16, num_pages=10, max_pages=4, width=64, softmax_scale=0.0, out=FAKE,
             workspace=FAKE, bytes=1 << 40, stream=None)
    assert not kw.keys() - a.keys()
    return [*(a | kw).values()]


@pytest.mark.parametrize("bad, status", SHAPES + [
    (dict(lse=None), 1), (dict(out=None), 1), (dict(width=0), 1), (dict(width=(1 << 30) + 1), 1), (dict(mass=ODD), 1),
    (dict(weights=ODD), 1), (dict(out=ODD), 1)])
def test_attention_mass_refuses(lib, bad, status):
    assert lib.sf_attention_mass(*mass_args(**bad)) == status
    assert lib.sf_last_error()


def commit_args(**kw):
    a = dict(tokens=FAKE, sampled=FAKE, parents=FAKE, k=TWO, v=TWO, layers=2, block_table=FAKE, seq_lens=FAKE, B=2, n_q=5,
             H_kv=8, head_dim=64, page_size=16, num_pages=10, max_pages=4, accepted=FAKE, out_tokens=FAKE, path=FAKE,
             weights=FAKE, n_q_next=5, free_pages=None, free_count=None, capacity=0, workspace=FAKE, bytes=256,
             stream=None)
    assert not kw.keys() - a.keys()
    return [*(a | kw).values()]


@pytest.mark.parametrize("bad, status", [
    (dict(B=0), 1), (dict(B=1025), 1), (dict(n_q=0), 1), (dict(n_q=65), 1), (dict(layers=-1), 1), (dict(layers=129), 1),
    (dict(H_kv=0), 1), (dict(H_kv=1025), 1), (dict(head_dim=60), 2), (dict(head_dim=264), 2), (dict(page_size=32), 2),
    (dict(num_pages=0), 1), (dict(max_pages=0), 1), (dict(max_pages=1 << 27), 1), (dict(tokens=None), 1),
    (dict(sampled=None), 1), (dict(parents=None), 1), (dict(block_table=None), 1), (dict(seq_lens=None), 1),
    (dict(accepted=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(k=pointers(256, 264)), 1),
    (dict(v=pointers(0, 256)), 1), (dict(tokens=ODD), 1), (dict(path=ODD), 1), (dict(weights=ODD), 1),
    (dict(free_pages=FAKE), 1), (dict(free_count=FAKE), 1),
    (dict(free_pages=FAKE, free_count=FAKE, n_q_next=0), 1), (dict(free_pages=FAKE, free_count=FAKE, n_q_next=65), 1),
    (dict(free_pages=FAKE, free_count=FAKE, capacity=-1), 1), (dict(workspace=None), 4),
    (dict(workspace=ctypes.c_void_p(128)), 4), (dict(bytes=255), 4)])
def test_tree_commit_refuses(lib, bad, status):
    assert lib.sf_tree_commit(*commit_args(**bad)) == status
    assert lib.sf_last_error()


def evict_args(**kw):
    a = dict(mass=TWO, k=TWO, v=TWO, layers=2, block_table=FAKE, seq_lens=FAKE, B=2, H_kv=8, head_dim=64, page_size=16,
             num_pages=10, max_pages=4, width=64, budget=32, first=2, recent=4, n_q=0, mass_out=TWO, lens_out=FAKE,
             kept=None, free_pages=None, free_count=None, capacity=0, workspace=FAKE, bytes=1 << 30, stream=None)
    assert not kw.keys() - a.keys()
    return [*(a | kw).values()]


@pytest.mark.parametrize("bad, status", [
    (dict(layers=0), 1), (dict(layers=129), 1), (dict(B=0), 1), (dict(B=1025), 1), (dict(H_kv=0), 1),
    (dict(H_kv=1025), 1), (dict(head_dim=60), 2), (dict(head_dim=264), 2), (dict(page_size=32), 2),
    (dict(num_pages=0), 1), (dict(max_pages=0), 1), (dict(width=0), 1), (dict(budget=0), 1), (dict(first=-1), 1),
    (dict(recent=-1), 1), (dict(first=20, recent=13), 1), (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), 1),
    (dict(n_q=-1), 1), (dict(n_q=65), 1), (dict(mass=None), 1),
    (dict(k=None), 1), (dict(v=None), 1), (dict(mass_out=None), 1), (dict(lens_out=None), 1), (dict(seq_lens=None), 1),
    (dict(block_table=None), 1), (dict(k=pointers(256, 0)), 1), (dict(v=pointers(256, 264)), 1),
    (dict(mass=pointers(256, 258)), 1), (dict(kept=pointers(0, 256)), 1), (dict(lens_out=ODD), 1),
    (dict(free_pages=FAKE), 1), (dict(free_count=FAKE), 1), (dict(capacity=-1), 1), (dict(workspace=None), 4),
    (dict(workspace=ctypes.c_void_p(128)), 4), (dict(bytes=256), 4)])
def test_kv_evict_refuses(lib, bad, status):
    assert lib.sf_kv_evict(*evict_args(**bad)) == status
    assert lib.sf_last_error()


def test_workspace_sizes_refuse_shapes_that_the_calls_refuse(lib):
    assert lib.sf_tree_mask_workspace_size() >= 4 and lib.sf_tree_commit_workspace_size() >= 4
    assert lib.sf_tree_attention_workspace_size(0, 4, 8, 8, 64, 4, 16) == 0
    assert lib.sf_tree_attention_workspace_size(1, 65, 8, 8, 64, 4, 16) == 0
    assert lib.sf_kv_evict_workspace_size(0, 1, 8, 16) == 0 and lib.sf_kv_evict_workspace_size(1, 1, 8, 0) == 0
    with pytest.raises(sfv.SFError, match="n_q"):
        sfv.tree_attention_workspace_size(1, 65, 8, 8, 64, 4)
    with pytest.raises(sfv.SFError, match="budget"):
        sfv.kv_evict_workspace_size(1, 1, 8, 0)


def test_binding_refuses_host_tensors_and_wrong_shapes_before_the_library(monkeypatch):
    def no_library():
        raise AssertionError("the library must not be reached")

    monkeypatch.setattr(sfv, "load_library", no_library)
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    rows, ones = torch.zeros(1, 4, dtype=i32), torch.zeros(1, dtype=i32)
    cache, q = torch.zeros(4, 8, 16, 64, dtype=bf), torch.zeros(1, 4, 8, 64, dtype=bf)
    with pytest.raises(ValueError, match="CUDA"):
        sfv.tree_mask(rows)
    with pytest.raises(ValueError, match="parents must be"):
        sfv.tree_mask(ones)
    with pytest.raises(ValueError, match="CUDA"):
        sfv.tree_attention(q, cache, cache, rows, ones, torch.zeros(1, 4, dtype=torch.int64))
    with pytest.raises(ValueError, match="head_dim"):
        sfv.tree_attention(q, cache[..., :32], cache, rows, ones, torch.zeros(1, 4, dtype=torch.int64))
    with pytest.raises(ValueError, match="q must be"):
        sfv.attention_mass(q[0], torch.zeros(1, 4, 8), cache, rows, ones)
    with pytest.raises(ValueError, match="CUDA"):
        sfv.tree_commit(rows, rows, rows, cache[None], cache[None], rows, ones)
    with pytest.raises(ValueError, match="CUDA"):
        sfv.kv_evict(torch.zeros(1, 1, 8, 64, dtype=f32), cache[None], cache[None], rows, ones, 16)
    with pytest.raises(ValueError, match="layers first"):
        sfv._layer_pointers(cache, "k_caches", bf, 4)
    with pytest.raises(ValueError, match="CUDA"):
        sfv._layer_pointers([cache], "k_caches", bf, 4)
    with pytest.raises(ValueError, match="numbers of layers"):
        sfv._same_count({"k_caches": 2, "v_caches": 1})
