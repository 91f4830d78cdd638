"""Refusals of the decoder-layer operators that need no GPU: the library checks
its arguments before it touches the device, the binding before the library."""
import ctypes

import pytest
import torch

from paper_2505_12728_gb300 import build_lib
from paper_2505_12728_gb300 import specflash_verify as sfv

FAKE = ctypes.c_void_p(256)
ODD = ctypes.c_void_p(257)


@pytest.fixture(scope="module")
def lib():
    build_lib.build()
    return sfv.load_library()


def norm_args(**kw):
    a = dict(x=FAKE, residual=FAKE, weight=FAKE, dtype=0, weight_dtype=0, T=4, d=64, x_stride=64, residual_stride=64,
             eps=1e-6, residual_out=FAKE, residual_out_stride=64, out=FAKE, out_dtype=0, out_stride=64, group=0,
             scales=None, stream=None)
    assert not kw.keys() - a.keys()
    return [*(a | kw).values()]


@pytest.mark.parametrize("bad, status", [
    (dict(T=-1), 1), (dict(d=0), 1), (dict(d=32769), 1), (dict(dtype=2), 2), (dict(weight_dtype=7), 2),
    (dict(out_dtype=1), 2), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1),
    (dict(group=128), 1), (dict(out_dtype=2, group=64, scales=FAKE), 1), (dict(out_dtype=2), 1),
    (dict(scales=FAKE), 1), (dict(x=None), 1), (dict(weight=None), 1), (dict(out=None), 1), (dict(residual=None), 1),
    (dict(residual_out=None), 1), (dict(x_stride=63), 1), (dict(out_stride=0), 1), (dict(residual_stride=-64), 1),
    (dict(residual_out_stride=63), 1), (dict(x=ODD), 1), (dict(weight=ODD), 1),
    (dict(dtype=1, x=ctypes.c_void_p(258)), 1), (dict(out=ODD), 1)])
def test_norm_refuses(lib, bad, status):
    assert lib.sf_add_rms_norm(*norm_args(**bad)) == status
    assert lib.sf_last_error()


def test_norm_of_no_rows_does_nothing(lib):
    assert lib.sf_add_rms_norm(*norm_args(T=0, x=None, out=None)) == 0


def append_args(**kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, dtype=0, q_row=512, q_head=64, k_row=512, k_head=64, v_row=512, v_head=64,
             positions=FAKE, axes=1, inv_freq=FAKE, freq_axis=None, rotary_dim=64, interleaved=0, amplitude=1.0,
             block_table=FAKE, seq_lens=FAKE, row_starts=None, T=8, B=2, H_q=8, H_kv=8, head_dim=64, page_size=16,
             num_pages=10, max_pages=4, q_out=FAKE, k_cache=FAKE, v_cache=FAKE, workspace=FAKE, workspace_bytes=256,
             stream=None)
    assert not kw.keys() - a.keys()
    return [*(a | kw).values()]


@pytest.mark.parametrize("bad, status", [
    (dict(dtype=2), 2), (dict(T=-2), 1), (dict(T=7), 1), (dict(B=0), 1), (dict(B=1025), 1), (dict(H_q=-1), 1),
    (dict(H_kv=0), 1), (dict(H_kv=1025), 1), (dict(head_dim=60), 2), (dict(head_dim=264), 2), (dict(page_size=32), 2),
    (dict(max_pages=0), 1), (dict(max_pages=1 << 27), 1), (dict(num_pages=0), 1), (dict(rotary_dim=63), 1),
    (dict(rotary_dim=66), 1), (dict(rotary_dim=-2), 1), (dict(axes=0), 1), (dict(axes=5), 1),
    (dict(amplitude=float("nan")), 1), (dict(q=None), 1), (dict(q_out=None), 1), (dict(k=None), 1), (dict(v=None), 1),
    (dict(positions=None), 1), (dict(inv_freq=None), 1), (dict(block_table=None), 1), (dict(seq_lens=None), 1),
    (dict(k_cache=None), 1), (dict(v_cache=None), 1), (dict(k=ODD), 1), (dict(q_out=ctypes.c_void_p(264)), 1),
    (dict(k_cache=ctypes.c_void_p(264)), 1), (dict(inv_freq=ctypes.c_void_p(260)), 1), (dict(workspace=None), 4),
    (dict(workspace=ctypes.c_void_p(128)), 4), (dict(workspace_bytes=255), 4)])
def test_append_refuses(lib, bad, status):
    assert lib.sf_kv_append(*append_args(**bad)) == status
    assert lib.sf_last_error()


def test_append_of_no_rows_does_nothing(lib):
    assert lib.sf_kv_append(*append_args(T=0, k=None, workspace=None)) == 0


def shared_args(**kw):
    a = dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, prefix_table=FAKE, prefix_lens=FAKE, group_starts=FAKE,
             block_table=FAKE, seq_lens=FAKE, B=2, n_q=4, H_q=8, H_kv=8, head_dim=64, page_size=16, num_pages=10,
             num_groups=1, max_prefix_pages=4, max_pages=4, softmax_scale=0.0, out=FAKE, lse=None, workspace=FAKE,
             workspace_bytes=1 << 30, stream=None)
    assert not kw.keys() - a.keys()
    return [*(a | kw).values()]


@pytest.mark.parametrize("bad, status", [
    (dict(B=0), 1), (dict(B=1025), 1), (dict(n_q=0), 1), (dict(n_q=17), 1), (dict(H_q=7, H_kv=2), 1), (dict(H_kv=0), 1),
    (dict(H_q=32, H_kv=2), 2), (dict(head_dim=96), 2), (dict(page_size=8), 2), (dict(num_groups=0), 1),
    (dict(num_groups=3), 1), (dict(max_pages=0), 1), (dict(max_prefix_pages=0), 1), (dict(max_prefix_pages=1 << 27), 1),
    (dict(num_pages=0), 1), (dict(num_pages=1 << 25), 2), (dict(softmax_scale=-1.0), 1),
    (dict(softmax_scale=float("nan")), 1), (dict(q=None), 1), (dict(k_cache=None), 1), (dict(v_cache=None), 1),
    (dict(prefix_table=None), 1), (dict(prefix_lens=None), 1), (dict(group_starts=None), 1), (dict(block_table=None), 1),
    (dict(seq_lens=None), 1), (dict(out=None), 1), (dict(q=ctypes.c_void_p(264)), 1), (dict(seq_lens=ODD), 1),
    (dict(lse=ODD), 1), (dict(workspace=None), 4), (dict(workspace=ctypes.c_void_p(16)), 4)])
def test_shared_prefix_refuses(lib, bad, status):
    assert lib.sf_shared_prefix_attention(*shared_args(**bad)) == status
    assert lib.sf_last_error()


def test_workspace_sizes_refuse_shapes_that_the_calls_refuse(lib):
    assert lib.sf_kv_append_workspace_size() >= 4
    assert lib.sf_shared_prefix_attention_workspace_size(0, 4, 8, 8, 64, 1, 4, 4, 16) == 0
    assert lib.sf_shared_prefix_attention_workspace_size(2, 4, 8, 8, 64, 3, 4, 4, 16) == 0
    with pytest.raises(sfv.SFError, match="num_groups"):
        sfv.shared_prefix_attention_workspace_size(2, 4, 8, 8, 64, 3, 4, 4)


def test_binding_refuses_host_tensors_and_wrong_shapes_before_the_library(monkeypatch):
    def no_library():
        raise AssertionError("the library must not be reached")

    monkeypatch.setattr(sfv, "load_library", no_library)
    bf, i32 = torch.bfloat16, torch.int32
    x, w = torch.zeros(4, 64, dtype=bf), torch.zeros(64, dtype=bf)
    with pytest.raises(ValueError, match="CUDA"):
        sfv.add_rms_norm(x, w)
    with pytest.raises(TypeError, match="x must be"):
        sfv.add_rms_norm(x.half(), w)
    with pytest.raises(ValueError, match="shape"):
        sfv.add_rms_norm(x[0], w)
    k = torch.zeros(4, 8, 64, dtype=bf)
    cache, bt, sl = torch.zeros(4, 8, 16, 64, dtype=bf), torch.zeros(1, 4, dtype=i32), torch.zeros(1, dtype=i32)
    with pytest.raises(ValueError, match="CUDA"):
        sfv.kv_append(k, k, k, None, None, cache, cache, bt, sl)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        sfv.kv_append(None, k.half(), k, None, None, cache, cache, bt, sl)
    with pytest.raises(ValueError, match="k must be"):
        sfv.kv_append(None, k[0], k, None, None, cache, cache, bt, sl)
    q = torch.zeros(1, 4, 8, 64, dtype=bf)
    with pytest.raises(ValueError, match="CUDA"):
        sfv.shared_prefix_attention(q, cache, cache, bt, sl, torch.zeros(2, dtype=i32), bt, sl)
    with pytest.raises(ValueError, match="head_dim"):
        sfv.shared_prefix_attention(q, cache[..., :32], cache, bt, sl, torch.zeros(2, dtype=i32), bt, sl)
    with pytest.raises(ValueError, match="q must be"):
        sfv.shared_prefix_attention(q[0], cache, cache, bt, sl, torch.zeros(2, dtype=i32), bt, sl)


def test_norm_refuses_rows_that_a_step_of_the_grid_would_take_past_an_int(lib):
    assert lib.sf_add_rms_norm(*norm_args(T=0x7fff0001)) == 2
    assert b"T=" in lib.sf_last_error()
