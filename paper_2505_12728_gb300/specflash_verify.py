"""Python binding of the C ABI in include/specflash_verify.h (ctypes).

Argument marshalling only: tensors are checked for dtype, device, shape and
contiguity, their device pointers and the current CUDA stream are passed to
the library, and outputs/workspaces are allocated with torch when the caller
does not supply them.  Every step of the computation runs in the library's
CUDA kernels; there is no fallback.  If the compiled library is missing the
first call raises.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import threading

import torch

from . import build_lib

SF_OK = 0
SF_DEVICE_BAD_PAGE = 0x1
SF_DEVICE_BAD_TOKEN = 0x2
SF_DEVICE_TIMEOUT = 0x4
SF_DEVICE_BAD_SEQLEN = 0x8
SF_DEVICE_OUT_OF_PAGES = 0x10
SF_DEVICE_BAD_INDEX = 0x20
PAGE_SIZE = 16

EXPORTED_SYMBOLS = (
    "sf_status_string", "sf_last_error", "sf_version", "sf_workspace_init",
    "sf_read_device_status", "sf_selftest_bounded_wait",
    "sf_verify_attention_workspace_size", "sf_verify_attention",
    "sf_verify_attention_noalloc", "sf_verify_attention_kernel_launches",
    "sf_accept_workspace_size", "sf_accept", "sf_accept_kernel_launches",
    "sf_kv_commit_workspace_size", "sf_kv_commit",
    "sf_draft_tail_workspace_size", "sf_lm_head", "sf_sample", "sf_draft_sample",
    "sf_visual_compress_workspace_size", "sf_visual_compress",
    "sf_verify_lm_head_accept_workspace_size", "sf_verify_lm_head_accept",
    "sf_add_rms_norm", "sf_kv_append_workspace_size", "sf_kv_append",
    "sf_shared_prefix_attention_workspace_size", "sf_shared_prefix_attention",
    "sf_tree_mask_workspace_size", "sf_tree_mask", "sf_tree_attention_workspace_size", "sf_tree_attention",
    "sf_tree_commit_workspace_size", "sf_tree_commit", "sf_attention_mass_workspace_size", "sf_attention_mass",
    "sf_kv_evict_workspace_size", "sf_kv_evict",
)

_lock = threading.Lock()
_lib = None
_calls = None  # csrc/layer_calls.cpp, once the library is loaded (and if it was built)


class SFError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(message)
        self.status = status


def library_path() -> str:
    return build_lib.LIB


def load_library(path: str | None = None):
    """Load (once) the compiled library; raises if it has not been built."""
    global _lib
    if _lib is not None:  # the lock guards the loading only
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        path = path or library_path()
        if not os.path.exists(path):
            raise RuntimeError(
                f"{path} is missing: build it with paper_2505_12728_gb300.build_lib.build() "
                "(nvcc for sm_103a); the verification step has no CPU implementation")
        lib = ctypes.CDLL(path)
        P, I, F = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
        S = ctypes.c_size_t
        lib.sf_status_string.argtypes = [I]
        lib.sf_status_string.restype = ctypes.c_char_p
        lib.sf_last_error.argtypes = []
        lib.sf_last_error.restype = ctypes.c_char_p
        lib.sf_version.argtypes = []
        lib.sf_version.restype = I
        lib.sf_workspace_init.argtypes = [P, S, P]
        lib.sf_workspace_init.restype = I
        lib.sf_read_device_status.argtypes = [P, ctypes.POINTER(ctypes.c_uint32)]
        lib.sf_read_device_status.restype = I
        lib.sf_selftest_bounded_wait.argtypes = [P, S, P]
        lib.sf_selftest_bounded_wait.restype = I
        lib.sf_verify_attention_workspace_size.argtypes = [I, I, I, I, I, I, I, I]
        lib.sf_verify_attention_workspace_size.restype = S
        lib.sf_verify_attention.argtypes = [P, P, P, P, P, I, I, I, I, I, I, I, I, F, I, P, P, P,
                                            S, P]
        lib.sf_verify_attention.restype = I
        lib.sf_verify_attention_noalloc.argtypes = [P, P, P, P, P, I, I, I, I, I, I, I, I, F, I,
                                                    P, P, P]
        lib.sf_verify_attention_noalloc.restype = I
        lib.sf_verify_attention_kernel_launches.argtypes = [I] * 8
        lib.sf_verify_attention_kernel_launches.restype = I
        lib.sf_accept_workspace_size.argtypes = [I, I, I]
        lib.sf_accept_workspace_size.restype = S
        lib.sf_accept_kernel_launches.argtypes = [I, I, I]
        lib.sf_accept_kernel_launches.restype = I
        lib.sf_accept.argtypes = [P, P, P, P, P, I, I, I, P, P, P, P, S, P]
        lib.sf_accept.restype = I
        lib.sf_kv_commit_workspace_size.argtypes = []
        lib.sf_kv_commit_workspace_size.restype = S
        lib.sf_kv_commit.argtypes = [P, P, P, P, P, I, I, I, I, I, I, P, S, P]
        lib.sf_kv_commit.restype = I
        lib.sf_draft_tail_workspace_size.argtypes = [I, I]
        lib.sf_draft_tail_workspace_size.restype = S
        lib.sf_lm_head.argtypes = [P, P, I, I, I, P, P, S, P]
        lib.sf_lm_head.restype = I
        lib.sf_sample.argtypes = [P, P, P, I, I, P, P, P, S, P]
        lib.sf_sample.restype = I
        lib.sf_draft_sample.argtypes = [P, P, P, P, I, I, I, P, P, P, P, S, P]
        lib.sf_draft_sample.restype = I
        lib.sf_visual_compress_workspace_size.argtypes = [I, I, I, I]
        lib.sf_visual_compress_workspace_size.restype = S
        lib.sf_visual_compress.argtypes = [P, P, I, I, I, I, P, P, S, P]
        lib.sf_visual_compress.restype = I
        lib.sf_verify_lm_head_accept_workspace_size.argtypes = [I, I, I]
        lib.sf_verify_lm_head_accept_workspace_size.restype = S
        lib.sf_verify_lm_head_accept.argtypes = [P, P, P, P, P, P, I, I, I, I, P, P, P, P, P, S, P]
        lib.sf_verify_lm_head_accept.restype = I
        L = ctypes.c_longlong
        lib.sf_add_rms_norm.argtypes = [P, P, P, I, I, I, I, L, L, F, P, L, P, I, L, I, P, P]
        lib.sf_add_rms_norm.restype = I
        lib.sf_kv_append_workspace_size.argtypes = []
        lib.sf_kv_append_workspace_size.restype = S
        lib.sf_kv_append.argtypes = [P, P, P, I, L, L, L, L, L, L, P, I, P, P, I, I, F, P, P, P, I,
                                     I, I, I, I, I, I, I, P, P, P, P, S, P]
        lib.sf_kv_append.restype = I
        lib.sf_shared_prefix_attention_workspace_size.argtypes = [I] * 9
        lib.sf_shared_prefix_attention_workspace_size.restype = S
        lib.sf_shared_prefix_attention.argtypes = [P, P, P, P, P, P, P, P, I, I, I, I, I, I, I, I,
                                                   I, I, F, P, P, P, S, P]
        lib.sf_shared_prefix_attention.restype = I
        lib.sf_tree_mask_workspace_size.argtypes = []
        lib.sf_tree_mask_workspace_size.restype = S
        lib.sf_tree_mask.argtypes = [P, P, I, I, P, P, P, S, P]
        lib.sf_tree_mask.restype = I
        lib.sf_tree_attention_workspace_size.argtypes = [I] * 7
        lib.sf_tree_attention_workspace_size.restype = S
        lib.sf_tree_attention.argtypes = [P, P, P, P, P, P, L, I, I, I, I, I, I, I, I, F, P, P, P, S, P]
        lib.sf_tree_attention.restype = I
        lib.sf_tree_commit_workspace_size.argtypes = []
        lib.sf_tree_commit_workspace_size.restype = S
        lib.sf_tree_commit.argtypes = [P, P, P, P, P, I, P, P, I, I, I, I, I, I, I, P, P, P, P, I, P, P, I, P, S, P]
        lib.sf_tree_commit.restype = I
        lib.sf_attention_mass_workspace_size.argtypes = []
        lib.sf_attention_mass_workspace_size.restype = S
        lib.sf_attention_mass.argtypes = [P, P, P, P, P, P, P, I, I, I, I, I, I, I, I, I, F, P, P, S, P]
        lib.sf_attention_mass.restype = I
        lib.sf_kv_evict_workspace_size.argtypes = [I] * 4
        lib.sf_kv_evict_workspace_size.restype = S
        lib.sf_kv_evict.argtypes = [P, P, P, I, P, P, I, I, I, I, I, I, I, I, I, I, I, P, P, P, P, P, I, P, S, P]
        lib.sf_kv_evict.restype = I
        _load_calls(lib)
        _lib = lib
        return lib


def _load_calls(lib):
    """The decoder-layer operators' direct calls, where they were built for the
    Python and the torch that run."""
    global _calls
    path = build_lib.calls_path()
    if not os.path.exists(path):
        return
    spec = importlib.util.spec_from_file_location("_layer_calls", path)
    try:
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError:  # a library that it was linked with is gone
        return
    module.set_entries(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.sf_add_rms_norm, lib.sf_kv_append, lib.sf_shared_prefix_attention, lib.sf_tree_mask, lib.sf_tree_attention,
        lib.sf_tree_commit, lib.sf_attention_mass, lib.sf_kv_evict)))
    _calls = module


def _check(status: int):
    if status != SF_OK:
        lib = load_library()
        raise SFError(status, f"{lib.sf_status_string(status).decode()}: "
                              f"{lib.sf_last_error().decode()}")


# The marshalling of a call is host time that a small call waits for (17
# tensors and two calls for one layer and its acceptance): pointers go to ctypes
# as integers, the current stream is read without building a Stream object
# (2.8 us a call), and a tensor that is as it should be takes one expression.
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream_handle(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(_device())
    return torch.cuda.current_stream().cuda_stream


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _need_workspace(workspace):
    """A caller-supplied workspace must be a contiguous uint8 CUDA tensor (its
    numel() is the byte count passed to the library)."""
    _need(workspace, "workspace", torch.uint8)


def _need(t, name, dtype, shape=None):
    if (type(t) is torch.Tensor and t.dtype is dtype and t.is_cuda and t.is_contiguous()
            and (shape is None or t.shape == shape)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


# --------------------------------------------------------------------------- #
# workspaces                                                                  #
# --------------------------------------------------------------------------- #
def verify_attention_workspace_size(B, n_q, H_q, H_kv, head_dim, max_pages_per_seq,
                                    page_size=PAGE_SIZE, num_splits=0) -> int:
    n = load_library().sf_verify_attention_workspace_size(B, n_q, H_q, H_kv, head_dim,
                                                          max_pages_per_seq, page_size,
                                                          num_splits)
    if n == 0:
        raise SFError(1, "invalid verify-attention shape: " + load_library().sf_last_error().decode())
    return int(n)


def accept_workspace_size(B, k, V) -> int:
    n = load_library().sf_accept_workspace_size(B, k, V)
    if n == 0:
        raise SFError(1, "invalid acceptance shape: " + load_library().sf_last_error().decode())
    return int(n)


def verify_attention_kernel_launches(B, n_q, H_q, H_kv, head_dim, max_pages_per_seq,
                                     num_splits=0) -> int:
    """Kernels one verify_attention call with these shapes launches (1 or 2)."""
    n = load_library().sf_verify_attention_kernel_launches(B, n_q, H_q, H_kv, head_dim,
                                                           max_pages_per_seq, PAGE_SIZE, num_splits)
    if n == 0:
        raise SFError(1, "no attention launch plan: " + load_library().sf_last_error().decode())
    return int(n)


def accept_kernel_launches(B, k, V) -> int:
    """Kernels one accept call with these shapes launches (1 or 2)."""
    n = load_library().sf_accept_kernel_launches(B, k, V)
    if n == 0:
        raise SFError(1, "no acceptance launch plan: " + load_library().sf_last_error().decode())
    return int(n)


def new_workspace(nbytes: int, device=None) -> torch.Tensor:
    """A zero-filled uint8 device buffer (the library's counters start at 0)."""
    return torch.zeros(int(nbytes), dtype=torch.uint8, device=device or "cuda")


def workspace_init(workspace: torch.Tensor, stream=None):
    _need_workspace(workspace)
    _check(load_library().sf_workspace_init(_ptr(workspace), workspace.numel(),
                                            _stream_handle(stream)))


def read_device_status(workspace: torch.Tensor) -> int:
    _need_workspace(workspace)
    v = ctypes.c_uint32(0)
    _check(load_library().sf_read_device_status(_ptr(workspace), ctypes.byref(v)))
    return int(v.value)


def selftest_bounded_wait(workspace: torch.Tensor, stream=None) -> None:
    """sf_selftest_bounded_wait: a wait that nothing completes gives up after
    about a second and sets SF_DEVICE_TIMEOUT in the workspace's status word
    (read it with read_device_status)."""
    _need_workspace(workspace)
    _check(load_library().sf_selftest_bounded_wait(_ptr(workspace), workspace.numel(),
                                                   _stream_handle(stream)))


# --------------------------------------------------------------------------- #
# verification attention                                                      #
# --------------------------------------------------------------------------- #
def verify_attention(q, k_cache, v_cache, block_table, seq_lens, *, out=None, lse=None,
                     workspace=None, softmax_scale=0.0, num_splits=0, stream=None,
                     with_lse=True):
    """sf_verify_attention: q bf16 [B][n_q][H_q][d]; k/v_cache bf16
    [pages][H_kv][16][d]; block_table int32 [B][max_pages]; seq_lens int32 [B]
    (prefix + n_q).  Returns (out bf16 [B][n_q][H_q][d], lse fp32 [B][n_q][H_q]
    or None).

    The keys and values in front of the n_q draft rows, the block table and the
    lengths are read before the kernel waits for the previous one on the stream: a
    kernel that lets its successor start early must not write them (kv_append says
    which of its calls may precede this one; tree_commit without free_pages and
    kv_evict may)."""
    B, n_q, H_q, d = q.shape
    num_pages, H_kv, page, d2 = k_cache.shape
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError(f"block_table has shape {tuple(block_table.shape)}, expected ({B}, max_pages)")
    if d2 != d:
        raise ValueError("head_dim of q and caches differ")
    _need(q, "q", torch.bfloat16)
    _need(k_cache, "k_cache", torch.bfloat16)
    _need(v_cache, "v_cache", torch.bfloat16, k_cache.shape)
    _need(block_table, "block_table", torch.int32)
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    max_pages = block_table.shape[1]
    if out is None:
        out = torch.empty_like(q)
    _need(out, "out", torch.bfloat16, q.shape)
    if lse is None and with_lse:
        lse = torch.empty((B, n_q, H_q), dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse, "lse", torch.float32, (B, n_q, H_q))
    if workspace is None:
        workspace = new_workspace(verify_attention_workspace_size(
            B, n_q, H_q, H_kv, d, max_pages, page, num_splits), q.device)
    _need_workspace(workspace)
    _check(load_library().sf_verify_attention(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(seq_lens), B, n_q, H_q,
        H_kv, d, page, num_pages, max_pages, float(softmax_scale), int(num_splits), _ptr(out),
        _ptr(lse), _ptr(workspace), workspace.numel(), _stream_handle(stream)))
    return out, lse


def verify_attention_noalloc(q, k_cache, v_cache, block_table, seq_lens, *, out=None, lse=None,
                             softmax_scale=0.0, num_splits=0, stream=None, with_lse=True):
    """sf_verify_attention_noalloc: the same computation as verify_attention
    for callers that cannot allocate device memory while verifying; the
    library's own 16 MiB device scratch replaces the workspace (calls that
    overlap on the GPU race on it).  Outputs may still be allocated here when
    not supplied."""
    B, n_q, H_q, d = q.shape
    num_pages, H_kv, page, d2 = k_cache.shape
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError(f"block_table has shape {tuple(block_table.shape)}, expected ({B}, max_pages)")
    if d2 != d:
        # the library sizes the caches' tensor maps from q's head_dim: a
        # narrower cache would let the copies read past its end
        raise ValueError("head_dim of q and caches differ")
    _need(q, "q", torch.bfloat16)
    _need(k_cache, "k_cache", torch.bfloat16)
    _need(v_cache, "v_cache", torch.bfloat16, k_cache.shape)
    _need(block_table, "block_table", torch.int32)
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    if out is None:
        out = torch.empty_like(q)
    _need(out, "out", torch.bfloat16, q.shape)
    if lse is None and with_lse:
        lse = torch.empty((B, n_q, H_q), dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse, "lse", torch.float32, (B, n_q, H_q))
    _check(load_library().sf_verify_attention_noalloc(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(seq_lens), B, n_q, H_q,
        H_kv, d, page, num_pages, block_table.shape[1], float(softmax_scale), int(num_splits),
        _ptr(out), _ptr(lse), _stream_handle(stream)))
    return out, lse


# --------------------------------------------------------------------------- #
# acceptance                                                                  #
# --------------------------------------------------------------------------- #
def accept(target_logits, draft_probs, draft_tokens, uniforms, temperature, *,
           num_accepted=None, out_tokens=None, accept_ratio=None, workspace=None, stream=None,
           with_ratio=True):
    """sf_accept: target_logits fp32 [B][k+1][V], draft_probs fp32 [B][k][V],
    draft_tokens int32 [B][k], uniforms fp32 [B][k+1], temperature fp32 [B]
    (<= 0 greedy).  Returns (num_accepted int32 [B], out_tokens int32 [B][k+1],
    accept_ratio fp32 [B][k] or None)."""
    B, k1, V = target_logits.shape
    k = k1 - 1
    _need(target_logits, "target_logits", torch.float32)
    _need(draft_probs, "draft_probs", torch.float32, (B, k, V))
    _need(draft_tokens, "draft_tokens", torch.int32, (B, k))
    _need(uniforms, "uniforms", torch.float32, (B, k + 1))
    _need(temperature, "temperature", torch.float32, (B,))
    dev = target_logits.device
    if num_accepted is None:
        num_accepted = torch.empty(B, dtype=torch.int32, device=dev)
    if out_tokens is None:
        out_tokens = torch.empty((B, k + 1), dtype=torch.int32, device=dev)
    if accept_ratio is None and with_ratio:
        accept_ratio = torch.empty((B, k), dtype=torch.float32, device=dev)
    _need(num_accepted, "num_accepted", torch.int32, (B,))
    _need(out_tokens, "out_tokens", torch.int32, (B, k + 1))
    if accept_ratio is not None:
        _need(accept_ratio, "accept_ratio", torch.float32, (B, k))
    if workspace is None:
        workspace = new_workspace(accept_workspace_size(B, k, V), dev)
    _need_workspace(workspace)
    _check(load_library().sf_accept(
        _ptr(target_logits), _ptr(draft_probs), _ptr(draft_tokens), _ptr(uniforms),
        _ptr(temperature), B, k, V, _ptr(num_accepted), _ptr(out_tokens), _ptr(accept_ratio),
        _ptr(workspace), workspace.numel(), _stream_handle(stream)))
    return num_accepted, out_tokens, accept_ratio


def verify_lm_head_accept_workspace_size(B, k, V) -> int:
    n = load_library().sf_verify_lm_head_accept_workspace_size(B, k, V)
    if n == 0:
        raise SFError(1, "invalid fused acceptance shape")
    return int(n)


def verify_lm_head_accept(hidden, weight, draft_probs, draft_tokens, uniforms, temperature, *,
                          logits=None, num_accepted=None, out_tokens=None, accept_ratio=None,
                          workspace=None, stream=None, with_ratio=True):
    """sf_verify_lm_head_accept: hidden bf16 [B][k+1][d] (the target's final
    hidden states of the verified positions), weight bf16 [V][d], then the
    acceptance rule as in accept().  Returns (logits fp32 [B][k+1][V],
    num_accepted int32 [B], out_tokens int32 [B][k+1], accept_ratio or None)."""
    B, k1, d = hidden.shape
    k = k1 - 1
    V = weight.shape[0]
    _need(hidden, "hidden", torch.bfloat16)
    _need(weight, "weight", torch.bfloat16, (V, d))
    _need(draft_probs, "draft_probs", torch.float32, (B, k, V))
    _need(draft_tokens, "draft_tokens", torch.int32, (B, k))
    _need(uniforms, "uniforms", torch.float32, (B, k + 1))
    _need(temperature, "temperature", torch.float32, (B,))
    dev = hidden.device
    if logits is None:
        logits = torch.empty((B, k + 1, V), dtype=torch.float32, device=dev)
    if num_accepted is None:
        num_accepted = torch.empty(B, dtype=torch.int32, device=dev)
    if out_tokens is None:
        out_tokens = torch.empty((B, k + 1), dtype=torch.int32, device=dev)
    if accept_ratio is None and with_ratio:
        accept_ratio = torch.empty((B, k), dtype=torch.float32, device=dev)
    _need(logits, "logits", torch.float32, (B, k + 1, V))
    _need(num_accepted, "num_accepted", torch.int32, (B,))
    _need(out_tokens, "out_tokens", torch.int32, (B, k + 1))
    if accept_ratio is not None:
        _need(accept_ratio, "accept_ratio", torch.float32, (B, k))
    if workspace is None:
        workspace = new_workspace(verify_lm_head_accept_workspace_size(B, k, V), dev)
    _need_workspace(workspace)
    _check(load_library().sf_verify_lm_head_accept(
        _ptr(hidden), _ptr(weight), _ptr(draft_probs), _ptr(draft_tokens), _ptr(uniforms),
        _ptr(temperature), B, k, V, d, _ptr(logits), _ptr(num_accepted), _ptr(out_tokens),
        _ptr(accept_ratio), _ptr(workspace), workspace.numel(), _stream_handle(stream)))
    return logits, num_accepted, out_tokens, accept_ratio


def kv_commit_workspace_size() -> int:
    return int(load_library().sf_kv_commit_workspace_size())


def kv_commit(seq_lens, block_table, free_pages, free_count, num_accepted, n_q, n_q_next, *,
              workspace=None, stream=None):
    """sf_kv_commit, in place: seq_lens int32 [B], block_table int32
    [B][max_pages], free_pages int32 [capacity] (a stack of free page ids),
    free_count int32 [1], num_accepted int32 [B] (from accept).  Keeps the
    first min(a + 1, n_q) verified rows of each sequence, prepares seq_lens
    for the next n_q_next rows and maps exactly their pages."""
    B, max_pages = block_table.shape
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    _need(block_table, "block_table", torch.int32)
    _need(free_pages, "free_pages", torch.int32)
    _need(free_count, "free_count", torch.int32, (1,))
    _need(num_accepted, "num_accepted", torch.int32, (B,))
    if workspace is None:
        workspace = new_workspace(kv_commit_workspace_size(), seq_lens.device)
    _need_workspace(workspace)
    _check(load_library().sf_kv_commit(
        _ptr(seq_lens), _ptr(block_table), _ptr(free_pages), _ptr(free_count), _ptr(num_accepted),
        B, n_q, n_q_next, max_pages, PAGE_SIZE, free_pages.numel(), _ptr(workspace),
        workspace.numel(), _stream_handle(stream)))


# --------------------------------------------------------------------------- #
# draft-distribution tail                                                     #
# --------------------------------------------------------------------------- #
def draft_tail_workspace_size(R, V) -> int:
    n = load_library().sf_draft_tail_workspace_size(R, V)
    if n == 0:
        raise SFError(1, "invalid draft-tail shape: " + load_library().sf_last_error().decode())
    return int(n)


def lm_head(hidden, weight, *, logits=None, workspace=None, stream=None):
    """sf_lm_head: hidden bf16 [R][hidden_size], weight bf16 [V][hidden_size].
    Returns logits fp32 [R][V] = hidden @ weight^T."""
    R, Hd = hidden.shape
    V = weight.shape[0]
    _need(hidden, "hidden", torch.bfloat16)
    _need(weight, "weight", torch.bfloat16, (V, Hd))
    if logits is None:
        logits = torch.empty((R, V), dtype=torch.float32, device=hidden.device)
    _need(logits, "logits", torch.float32, (R, V))
    if workspace is None:
        workspace = new_workspace(draft_tail_workspace_size(R, V), hidden.device)
    _need_workspace(workspace)
    _check(load_library().sf_lm_head(_ptr(hidden), _ptr(weight), R, Hd, V, _ptr(logits),
                                     _ptr(workspace), workspace.numel(), _stream_handle(stream)))
    return logits


def sample(logits, uniforms, temperature, *, probs=None, tokens=None, workspace=None,
           stream=None):
    """sf_sample: logits fp32 [R][V], uniforms fp32 [R], temperature fp32 [R]
    (<= 0 greedy).  Returns (probs fp32 [R][V], tokens int32 [R])."""
    R, V = logits.shape
    _need(logits, "logits", torch.float32)
    _need(uniforms, "uniforms", torch.float32, (R,))
    _need(temperature, "temperature", torch.float32, (R,))
    dev = logits.device
    if probs is None:
        probs = torch.empty((R, V), dtype=torch.float32, device=dev)
    if tokens is None:
        tokens = torch.empty(R, dtype=torch.int32, device=dev)
    _need(probs, "probs", torch.float32, (R, V))
    _need(tokens, "tokens", torch.int32, (R,))
    if workspace is None:
        workspace = new_workspace(draft_tail_workspace_size(R, V), dev)
    _need_workspace(workspace)
    _check(load_library().sf_sample(_ptr(logits), _ptr(uniforms), _ptr(temperature), R, V,
                                    _ptr(probs), _ptr(tokens), _ptr(workspace), workspace.numel(),
                                    _stream_handle(stream)))
    return probs, tokens


def draft_sample(hidden, weight, uniforms, temperature, *, logits=None, probs=None, tokens=None,
                 workspace=None, stream=None):
    """sf_draft_sample: the LM-head projection and sampling of the draft
    rows in two launches.  Returns (logits fp32 [R][V], probs fp32 [R][V],
    tokens int32 [R])."""
    R, Hd = hidden.shape
    V = weight.shape[0]
    _need(hidden, "hidden", torch.bfloat16)
    _need(weight, "weight", torch.bfloat16, (V, Hd))
    _need(uniforms, "uniforms", torch.float32, (R,))
    _need(temperature, "temperature", torch.float32, (R,))
    dev = hidden.device
    if logits is None:
        logits = torch.empty((R, V), dtype=torch.float32, device=dev)
    if probs is None:
        probs = torch.empty((R, V), dtype=torch.float32, device=dev)
    if tokens is None:
        tokens = torch.empty(R, dtype=torch.int32, device=dev)
    _need(logits, "logits", torch.float32, (R, V))
    _need(probs, "probs", torch.float32, (R, V))
    _need(tokens, "tokens", torch.int32, (R,))
    if workspace is None:
        workspace = new_workspace(draft_tail_workspace_size(R, V), dev)
    _need_workspace(workspace)
    _check(load_library().sf_draft_sample(
        _ptr(hidden), _ptr(weight), _ptr(uniforms), _ptr(temperature), R, Hd, V, _ptr(logits),
        _ptr(probs), _ptr(tokens), _ptr(workspace), workspace.numel(), _stream_handle(stream)))
    return logits, probs, tokens


# --------------------------------------------------------------------------- #
# visual token compression                                                    #
# --------------------------------------------------------------------------- #
def visual_compress_workspace_size(F, N, C, d) -> int:
    n = load_library().sf_visual_compress_workspace_size(F, N, C, d)
    if n == 0:
        raise SFError(1, "invalid compressor shape")
    return int(n)


def visual_compress(queries, features, *, out=None, workspace=None, stream=None):
    """sf_visual_compress: queries bf16 [C][d], features bf16 [F][N][d].
    Returns out bf16 [F][C][d] = softmax(Q F_V^T) F_V per frame."""
    C, d = queries.shape
    F, N, d2 = features.shape
    _need(queries, "queries", torch.bfloat16)
    _need(features, "features", torch.bfloat16)
    if d2 != d:
        raise ValueError("queries and features differ in d")
    if out is None:
        out = torch.empty((F, C, d), dtype=torch.bfloat16, device=queries.device)
    _need(out, "out", torch.bfloat16, (F, C, d))
    if workspace is None:
        workspace = new_workspace(visual_compress_workspace_size(F, N, C, d), queries.device)
    _need_workspace(workspace)
    _check(load_library().sf_visual_compress(_ptr(queries), _ptr(features), F, N, C, d, _ptr(out),
                                             _ptr(workspace), workspace.numel(),
                                             _stream_handle(stream)))
    return out


# --------------------------------------------------------------------------- #
# the decoder layer around the attention                                      #
# --------------------------------------------------------------------------- #
# Host time is most of a small call here.  A call that brings its outputs and its
# workspace goes through csrc/layer_calls.cpp, which looks at the tensors directly;
# where that finds anything missing or not as it should be (or was not built) the
# functions below go through the arguments themselves.
_Tensor, _BF16, _F32, _E4M3 = torch.Tensor, torch.bfloat16, torch.float32, torch.float8_e4m3fn
_I32, _F64 = torch.int32, torch.float64


def _refuse_rows(t, name, dtype, shape):
    """Raises what is wrong with a tensor that may be strided but for its last
    dimension."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    raise ValueError(f"{name} must be contiguous in its last dimension")


def _row_stride(t, name, dtype, shape):
    """Elements between the rows of a checked CUDA tensor [T][d]."""
    if t.__class__ is _Tensor and t.dtype is dtype and t.is_cuda and t.shape == shape:
        if t.is_contiguous():
            return shape[1]
        row, last = t.stride()
        if last == 1 or shape[1] == 1:
            return row
    elif isinstance(t, _Tensor) and t.__class__ is not _Tensor:  # a subclass, such as a Parameter
        return _row_stride(t.detach().as_subclass(_Tensor), name, dtype, shape)
    _refuse_rows(t, name, dtype, shape)


def _head_strides(t, name, dtype, shape):
    """Elements between the rows and heads of a checked CUDA tensor [T][H][d]."""
    if t.__class__ is _Tensor and t.dtype is dtype and t.is_cuda and t.shape == shape:
        row, head, last = t.stride()
        if last == 1 or shape[2] == 1:
            return row, head
    elif isinstance(t, _Tensor) and t.__class__ is not _Tensor:
        return _head_strides(t.detach().as_subclass(_Tensor), name, dtype, shape)
    _refuse_rows(t, name, dtype, shape)


def _new(shape, dtype, device, stream, zero=False):
    """A tensor for a call on `stream`: allocated (and zeroed) in its order."""
    make = torch.zeros if zero else torch.empty
    if stream is None:
        return make(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype, device=device)


def add_rms_norm(x, weight, residual=None, *, eps=1e-6, out_dtype=torch.bfloat16, group=0, out=None,
                 residual_out=None, scales=None, stream=None):
    """sf_add_rms_norm: x bf16 or fp32 [T][d] (rows may be strided), residual like
    x or None, weight bf16 or fp32 [d].  y = rms_norm(x + residual) * weight as
    bf16, or with out_dtype (or out) float8_e4m3fn as 8-bit values with fp32
    scales, one per row (group 0) or per 128 columns (group 128).
    Returns (out [T][d], residual_out like x or None, scales [T][groups] or
    None).  residual_out may be the residual itself."""
    if _calls is not None and out is not None and stream is None:
        status = _calls.add_rms_norm(x, weight, residual, eps, group, out, residual_out, scales)
        if status is not None:
            if status:
                _check(status)
            return out, residual_out, scales
    if not isinstance(x, _Tensor):
        raise TypeError("x must be a torch.Tensor")
    shape, kind = x.shape, x.dtype
    if len(shape) != 2:
        raise ValueError(f"x has shape {tuple(shape)}, expected (T, d)")
    T, d = shape
    if kind is not _BF16 and kind is not _F32:
        raise TypeError(f"x must be bfloat16 or float32, got {kind}")
    x_row = _row_stride(x, "x", kind, shape)
    if not isinstance(weight, _Tensor) or (weight.dtype is not _BF16 and weight.dtype is not _F32):
        raise TypeError("weight must be a bfloat16 or float32 torch.Tensor")
    if not (weight.is_cuda and weight.is_contiguous() and weight.shape == (d,)):
        _need(weight, "weight", weight.dtype, (d,))
    r_ptr = ro_ptr = None
    r_row = ro_row = 0
    if residual is not None:
        r_row = _row_stride(residual, "residual", kind, shape)
        if residual_out is None:
            residual_out = _new(shape, kind, x.device, stream)
        ro_row = _row_stride(residual_out, "residual_out", kind, shape)
        r_ptr, ro_ptr = residual.data_ptr(), residual_out.data_ptr()
    elif residual_out is not None:
        raise ValueError("residual_out needs a residual")
    if out is None:
        if out_dtype is not _BF16 and out_dtype is not _E4M3:
            raise TypeError(f"out_dtype must be bfloat16 or float8_e4m3fn, got {out_dtype}")
        out = _new(shape, out_dtype, x.device, stream)
    elif not isinstance(out, _Tensor) or (out.dtype is not _BF16 and out.dtype is not _E4M3):
        raise TypeError("out must be a bfloat16 or float8_e4m3fn torch.Tensor")
    o_row = _row_stride(out, "out", out.dtype, shape)
    o_type, s_ptr = 0, None
    if out.dtype is _E4M3:
        if group != 0 and group != 128:
            raise ValueError(f"group={group}: 0 (a scale per row) or 128 columns")
        groups = -(-d // group) if group else 1
        if scales is None:
            scales = _new((T, groups), _F32, x.device, stream)
        _need(scales, "scales", _F32, (T, groups))
        o_type, s_ptr = 2, scales.data_ptr()
    elif scales is not None or group:
        raise ValueError("scales and group belong to float8_e4m3fn output")
    status = (_lib or load_library()).sf_add_rms_norm(
        x.data_ptr(), r_ptr, weight.data_ptr(), kind is _F32, weight.dtype is _F32, T, d, x_row, r_row, eps, ro_ptr,
        ro_row, out.data_ptr(), o_type, o_row, group, s_ptr, _stream_handle(stream))
    if status:
        _check(status)
    return out, residual_out, scales


def kv_append_workspace_size() -> int:
    return int(load_library().sf_kv_append_workspace_size())


def kv_append(q, k, v, positions, inv_freq, k_cache, v_cache, block_table, seq_lens, *, axis=None,
              row_starts=None, interleaved=False, amplitude=1.0, q_out=None, workspace=None,
              stream=None):
    """sf_kv_append: rotates the new rows' q and k and writes k and v into the
    paged cache.  q [T][H_q][d] (None: keys and values only), k and v
    [T][H_kv][d], bf16 or fp32, views of a fused projection allowed; positions
    int32 [axes][T]; inv_freq fp64 [rotary_dim / 2] (None: no rotation, and no
    positions); axis int32 [rotary_dim / 2] (None: axis 0); caches, block_table
    and seq_lens (counting the new rows) as for verify_attention; row_starts
    int32 [B + 1] for sequences of different numbers of new rows (None: T / B
    each).  Returns q_out bf16 [T][H_q][d] or None.

    verify_attention copies the keys in front of its n_q draft rows before it waits
    for the previous kernel.  It may follow this call directly if row_starts is given,
    if a sequence has more than 16 new rows, or if they are no more than its n_q;
    shared_prefix_attention always may."""
    if _calls is not None and workspace is not None and stream is None and (q is None) == (q_out is None):
        status = _calls.kv_append(q, k, v, positions, inv_freq, k_cache, v_cache, block_table, seq_lens, axis,
                                  row_starts, interleaved, amplitude, q_out, workspace)
        if status is not None:
            if status:
                _check(status)
            return q_out
    if not isinstance(k, _Tensor) or k.dim() != 3:
        raise ValueError("k must be a tensor [T][H_kv][d]")
    shape, kind = k.shape, k.dtype
    T, H_kv, d = shape
    if kind is not _BF16 and kind is not _F32:
        raise TypeError(f"k must be bfloat16 or float32, got {kind}")
    k_row, k_head = _head_strides(k, "k", kind, shape)
    v_row, v_head = _head_strides(v, "v", kind, shape)
    H_q = q_row = q_head = 0
    q_ptr = out_ptr = pos_ptr = freq_ptr = None
    if q is not None:
        if not isinstance(q, _Tensor) or q.dim() != 3:
            raise ValueError("q must be a tensor [T][H_q][d] or None")
        H_q = q.shape[1]
        q_shape = (T, H_q, d)
        q_row, q_head = _head_strides(q, "q", kind, q_shape)
        if q_out is None:
            q_out = _new(q_shape, _BF16, k.device, stream)
        _need(q_out, "q_out", _BF16, q_shape)
        q_ptr, out_ptr = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out needs a q")
    if not isinstance(block_table, _Tensor) or block_table.dim() != 2:
        raise ValueError("block_table must be [B][max_pages]")
    B, max_pages = block_table.shape
    if not isinstance(k_cache, _Tensor) or k_cache.dim() != 4:
        raise ValueError("k_cache must be a tensor [pages][H_kv][16][d]")
    cache = k_cache.shape
    num_pages, heads, page, wide = cache
    if heads != H_kv or wide != d:
        raise ValueError(f"k_cache has shape {tuple(cache)}, expected (pages, {H_kv}, 16, {d})")
    _need(k_cache, "k_cache", _BF16)
    _need(v_cache, "v_cache", _BF16, cache)
    _need(block_table, "block_table", _I32)
    _need(seq_lens, "seq_lens", _I32, (B,))
    axes = pairs = 0
    if inv_freq is not None:
        _need(inv_freq, "inv_freq", _F64)
        if inv_freq.dim() != 1 or not isinstance(positions, _Tensor) or positions.dim() != 2:
            raise ValueError("inv_freq must be [rotary_dim / 2] and positions a tensor [axes][T]")
        pairs, axes = inv_freq.shape[0], positions.shape[0]
        _need(positions, "positions", _I32, (axes, T))
        pos_ptr, freq_ptr = positions.data_ptr(), inv_freq.data_ptr()
        if axis is not None:
            _need(axis, "axis", _I32, (pairs,))
    elif positions is not None or axis is not None:
        raise ValueError("positions and axis need inv_freq")
    if row_starts is not None:
        _need(row_starts, "row_starts", _I32, (B + 1,))
    if workspace is None:
        workspace = _new(kv_append_workspace_size(), torch.uint8, k.device, stream, zero=True)
    _need_workspace(workspace)
    status = (_lib or load_library()).sf_kv_append(
        q_ptr, k.data_ptr(), v.data_ptr(), kind is _F32, q_row, q_head, k_row, k_head, v_row, v_head,
        pos_ptr, axes, freq_ptr, None if axis is None else axis.data_ptr(), 2 * pairs, interleaved, amplitude,
        block_table.data_ptr(), seq_lens.data_ptr(), None if row_starts is None else row_starts.data_ptr(), T, B, H_q,
        H_kv, d, page, num_pages, max_pages, out_ptr, k_cache.data_ptr(), v_cache.data_ptr(),
        workspace.data_ptr(), workspace.numel(), _stream_handle(stream))
    if status:
        _check(status)
    return q_out


def shared_prefix_attention_workspace_size(B, n_q, H_q, H_kv, head_dim, num_groups,
                                           max_prefix_pages, max_pages_per_seq,
                                           page_size=PAGE_SIZE) -> int:
    n = load_library().sf_shared_prefix_attention_workspace_size(
        B, n_q, H_q, H_kv, head_dim, num_groups, max_prefix_pages, max_pages_per_seq, page_size)
    if n == 0:
        raise SFError(1, "invalid shared-prefix shape: " + load_library().sf_last_error().decode())
    return int(n)


def shared_prefix_attention(q, k_cache, v_cache, prefix_table, prefix_lens, group_starts,
                            block_table, seq_lens, *, out=None, lse=None, workspace=None,
                            softmax_scale=0.0, stream=None, with_lse=True):
    """sf_shared_prefix_attention: verification attention of a batch whose
    sequences share prefixes.  q bf16 [B][n_q][H_q][d]; k/v_cache bf16
    [pages][H_kv][16][d]; group g = sequences group_starts[g] ..
    group_starts[g + 1] - 1 (int32 [groups + 1]) with the prefix_lens[g] (int32
    [groups]) tokens of the pages prefix_table[g] (int32 [groups][pages]);
    block_table int32 [B][pages] and seq_lens int32 [B] (0: idle slot) describe
    each sequence's own tokens, draft rows included.  Returns (out bf16
    [B][n_q][H_q][d], lse fp32 [B][n_q][H_q] or None)."""
    if _calls is not None and out is not None and workspace is not None and stream is None and (
            lse is not None or not with_lse):
        status = _calls.shared_prefix_attention(q, k_cache, v_cache, prefix_table, prefix_lens, group_starts,
                                                block_table, seq_lens, softmax_scale, out, lse, workspace)
        if status is not None:
            if status:
                _check(status)
            return out, lse
    if not isinstance(q, _Tensor) or q.dim() != 4:
        raise ValueError("q must be a tensor [B][n_q][H_q][d]")
    B, n_q, H_q, d = shape = q.shape
    if not isinstance(k_cache, _Tensor) or k_cache.dim() != 4:
        raise ValueError("k_cache must be a tensor [pages][H_kv][16][d]")
    cache = k_cache.shape
    num_pages, H_kv, page, d2 = cache
    if d2 != d:
        # the library sizes the caches' tensor maps from q's head_dim
        raise ValueError("head_dim of q and caches differ")
    _need(q, "q", _BF16)
    _need(k_cache, "k_cache", _BF16)
    _need(v_cache, "v_cache", _BF16, cache)
    _need(prefix_table, "prefix_table", _I32)
    _need(block_table, "block_table", _I32)
    if prefix_table.dim() != 2 or block_table.dim() != 2:
        raise ValueError("prefix_table and block_table must be two-dimensional")
    G, max_prefix = prefix_table.shape
    rows, max_pages = block_table.shape
    if rows != B:
        raise ValueError(f"block_table has shape {tuple(block_table.shape)}, expected ({B}, max_pages)")
    _need(prefix_lens, "prefix_lens", _I32, (G,))
    _need(group_starts, "group_starts", _I32, (G + 1,))
    _need(seq_lens, "seq_lens", _I32, (B,))
    if out is None:
        out = _new(shape, _BF16, q.device, stream)
    _need(out, "out", _BF16, shape)
    if lse is None and with_lse:
        lse = _new((B, n_q, H_q), _F32, q.device, stream)
    if lse is not None:
        _need(lse, "lse", _F32, (B, n_q, H_q))
    if workspace is None:
        workspace = _new(shared_prefix_attention_workspace_size(
            B, n_q, H_q, H_kv, d, G, max_prefix, max_pages, page), torch.uint8, q.device, stream, zero=True)
    _need_workspace(workspace)
    status = (_lib or load_library()).sf_shared_prefix_attention(
        q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), prefix_table.data_ptr(),
        prefix_lens.data_ptr(), group_starts.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
        B, n_q, H_q, H_kv, d, page, num_pages, G, max_prefix, max_pages, softmax_scale,
        out.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.numel(),
        _stream_handle(stream))
    if status:
        _check(status)
    return out, lse


# --------------------------------------------------------------------------- #
# trees of drafts, and a cache held at a budget                               #
# --------------------------------------------------------------------------- #
_I64, _U8 = torch.int64, torch.uint8


def _workspace(workspace, size, device, stream):
    if workspace is None:
        workspace = _new(size, _U8, device, stream, zero=True)
    _need_workspace(workspace)
    return workspace


def _matrix(t, name, dtype):
    """The shape of a checked contiguous CUDA tensor with two dimensions."""
    if not isinstance(t, _Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a two-dimensional tensor")
    _need(t, name, dtype)
    return t.shape


def _layer_pointers(x, name, dtype, dim, shape=None):
    """(ctypes array of the layers' device pointers, a layer's shape) of one tensor
    [layers][...] or a sequence of tensors, each layer contiguous."""
    if isinstance(x, _Tensor):
        if x.dim() != dim + 1:
            raise ValueError(f"{name} must have {dim + 1} dimensions (layers first) or be a list of tensors of {dim}")
        count = x.shape[0]
        if count and not x[0].is_contiguous():
            raise ValueError(f"{name} must be contiguous within a layer")
        each, step, first = x.shape[1:], x.stride(0) * x.element_size(), x.data_ptr()
        pointers = [first + i * step for i in range(count)]
        if x.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {x.dtype}")
        if not x.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
    else:
        count = len(x)
        each = x[0].shape if count and isinstance(x[0], _Tensor) else None
        for t in x:
            _need(t, name, dtype, each)
        if count and len(each) != dim:
            raise ValueError(f"{name} must be tensors of {dim} dimensions")
        pointers = [t.data_ptr() for t in x]
    if shape is not None and count and tuple(each) != tuple(shape):
        raise ValueError(f"{name} has layers of shape {tuple(each)}, expected {tuple(shape)}")
    return (ctypes.c_void_p * max(count, 1))(*pointers), count, each


def _same_count(counts):
    if len(set(counts.values())) > 1:
        raise ValueError("different numbers of layers: " + ", ".join(f"{k} {v}" for k, v in counts.items()))


def _free_stack(free_pages, free_count):
    if (free_pages is None) != (free_count is None):
        raise ValueError("free_pages and free_count belong together")
    if free_pages is None:
        return None, None, 0
    _need(free_pages, "free_pages", _I32)
    _need(free_count, "free_count", _I32, (1,))
    return free_pages.data_ptr(), free_count.data_ptr(), free_pages.numel()


def tree_mask_workspace_size() -> int:
    return int(load_library().sf_tree_mask_workspace_size())


def tree_mask(parents, start=None, *, mask=None, positions=None, workspace=None, stream=None):
    """sf_tree_mask: parents int32 [B][n] (each below its row; -1: a root, less: not
    part of the tree), start int32 [B] or None.  Returns (mask int64 [B][n]: bit j
    of row i for node i itself and the nodes above it; positions int32 [B][n]:
    start plus the number of nodes above)."""
    if _calls is not None and mask is not None and positions is not None and workspace is not None and stream is None:
        status = _calls.tree_mask(parents, start, mask, positions, workspace)
        if status is not None:
            if status:
                _check(status)
            return mask, positions
    B, n = shape = _matrix(parents, "parents", _I32)
    if start is not None:
        _need(start, "start", _I32, (B,))
    if mask is None:
        mask = _new(shape, _I64, parents.device, stream)
    _need(mask, "mask", _I64, shape)
    if positions is None:
        positions = _new(shape, _I32, parents.device, stream)
    _need(positions, "positions", _I32, shape)
    workspace = _workspace(workspace, tree_mask_workspace_size(), parents.device, stream)
    _check(load_library().sf_tree_mask(parents.data_ptr(), _ptr(start), B, n, mask.data_ptr(), positions.data_ptr(),
                                       workspace.data_ptr(), workspace.numel(), _stream_handle(stream)))
    return mask, positions


def tree_attention_workspace_size(B, n_q, H_q, H_kv, head_dim, max_pages_per_seq, page_size=PAGE_SIZE) -> int:
    n = load_library().sf_tree_attention_workspace_size(B, n_q, H_q, H_kv, head_dim, max_pages_per_seq, page_size)
    if n == 0:
        raise SFError(1, "invalid tree-attention shape: " + load_library().sf_last_error().decode())
    return int(n)


def _attention_arguments(q, k_cache, block_table, seq_lens):
    """Shapes of a checked q, key cache, block table and lengths."""
    if not isinstance(q, _Tensor) or q.dim() != 4:
        raise ValueError("q must be a tensor [B][n_q][H_q][d]")
    B, n_q, H_q, d = q.shape
    if not isinstance(k_cache, _Tensor) or k_cache.dim() != 4:
        raise ValueError("k_cache must be a tensor [pages][H_kv][16][d]")
    num_pages, H_kv, page, d2 = k_cache.shape
    if d2 != d:
        # the library sizes the caches' tensor maps from q's head_dim
        raise ValueError("head_dim of q and caches differ")
    _need(q, "q", _BF16)
    _need(k_cache, "k_cache", _BF16)
    rows, max_pages = _matrix(block_table, "block_table", _I32)
    if rows != B:
        raise ValueError(f"block_table has shape {tuple(block_table.shape)}, expected ({B}, max_pages)")
    _need(seq_lens, "seq_lens", _I32, (B,))
    return B, n_q, H_q, H_kv, d, page, num_pages, max_pages


def tree_attention(q, k_cache, v_cache, block_table, seq_lens, mask, *, out=None, lse=None, workspace=None,
                   softmax_scale=0.0, stream=None, with_lse=True):
    """sf_tree_attention: verification attention of n_q <= 64 nodes of a tree.  q,
    caches, block_table and seq_lens as for verify_attention (seq_lens 0: an idle
    slot); mask int64 [B][n_q], or [n_q] for one tree in all sequences: bit j of
    row i where it sees new row j (tree_mask makes it).  Rows that see nothing get
    0 and an lse of -inf.  Returns (out bf16 [B][n_q][H_q][d], lse fp32
    [B][n_q][H_q] or None)."""
    if _calls is not None and out is not None and workspace is not None and stream is None and (
            lse is not None or not with_lse):
        status = _calls.tree_attention(q, k_cache, v_cache, block_table, seq_lens, mask, softmax_scale, out, lse,
                                       workspace)
        if status is not None:
            if status:
                _check(status)
            return out, lse
    B, n_q, H_q, H_kv, d, page, num_pages, max_pages = _attention_arguments(q, k_cache, block_table, seq_lens)
    _need(v_cache, "v_cache", _BF16, k_cache.shape)
    stride = 0
    if isinstance(mask, _Tensor) and mask.dim() == 1:
        _need(mask, "mask", _I64, (n_q,))
    else:
        stride = _row_stride(mask, "mask", _I64, (B, n_q))
    if out is None:
        out = _new(q.shape, _BF16, q.device, stream)
    _need(out, "out", _BF16, q.shape)
    if lse is None and with_lse:
        lse = _new((B, n_q, H_q), _F32, q.device, stream)
    if lse is not None:
        _need(lse, "lse", _F32, (B, n_q, H_q))
    if workspace is None:
        workspace = _new(tree_attention_workspace_size(B, n_q, H_q, H_kv, d, max_pages, page), _U8, q.device, stream,
                         zero=True)
    _need_workspace(workspace)
    _check(load_library().sf_tree_attention(
        q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
        mask.data_ptr(), stride, B, n_q, H_q, H_kv, d, page, num_pages, max_pages, softmax_scale, out.data_ptr(),
        _ptr(lse), workspace.data_ptr(), workspace.numel(), _stream_handle(stream)))
    return out, lse


def tree_commit_workspace_size() -> int:
    return int(load_library().sf_tree_commit_workspace_size())


def tree_commit(tokens, sampled, parents, k_caches, v_caches, block_table, seq_lens, *, num_accepted=None,
                out_tokens=None, path=None, row_weights=None, n_q_next=None, free_pages=None, free_count=None,
                workspace=None, stream=None):
    """sf_tree_commit: the path that the target's tokens take through a tree, and its
    keys and values moved to follow the context.  tokens (the nodes'), sampled (the
    target's after each node) and parents int32 [B][n]; k_caches and v_caches bf16
    [layers][pages][H_kv][16][d] or lists of the layers' caches; block_table and
    seq_lens as for tree_attention.  Where node 0 is no root (parents not -1) there is
    no path: path and out_tokens -1, the rest 0.  With free_pages and free_count, seq_lens and
    block_table are then prepared for the next tree of n_q_next nodes (None: n), as
    by kv_commit.  Returns (num_accepted int32 [B], out_tokens int32 [B][n], path
    int32 [B][n], row_weights fp32 [B][n])."""
    if (_calls is not None and workspace is not None and stream is None and num_accepted is not None
            and out_tokens is not None and path is not None and row_weights is not None):
        status = _calls.tree_commit(tokens, sampled, parents, k_caches, v_caches, block_table, seq_lens, num_accepted,
                                    out_tokens, path, row_weights, n_q_next, free_pages, free_count, workspace)
        if status is not None:
            if status:
                _check(status)
            return num_accepted, out_tokens, path, row_weights
    B, n = shape = _matrix(tokens, "tokens", _I32)
    _need(sampled, "sampled", _I32, shape)
    _need(parents, "parents", _I32, shape)
    k_ptrs, layers, cache = _layer_pointers(k_caches, "k_caches", _BF16, 4)
    v_ptrs, v_layers, _ = _layer_pointers(v_caches, "v_caches", _BF16, 4, cache)
    _same_count({"k_caches": layers, "v_caches": v_layers})
    num_pages, H_kv, page, d = cache if layers else (1, 1, PAGE_SIZE, 64)
    rows, max_pages = _matrix(block_table, "block_table", _I32)
    if rows != B:
        raise ValueError(f"block_table has shape {tuple(block_table.shape)}, expected ({B}, max_pages)")
    _need(seq_lens, "seq_lens", _I32, (B,))
    device = tokens.device
    if num_accepted is None:
        num_accepted = _new((B,), _I32, device, stream)
    if out_tokens is None:
        out_tokens = _new(shape, _I32, device, stream)
    if path is None:
        path = _new(shape, _I32, device, stream)
    if row_weights is None:
        row_weights = _new(shape, _F32, device, stream)
    _need(num_accepted, "num_accepted", _I32, (B,))
    _need(out_tokens, "out_tokens", _I32, shape)
    _need(path, "path", _I32, shape)
    _need(row_weights, "row_weights", _F32, shape)
    free, count, capacity = _free_stack(free_pages, free_count)
    workspace = _workspace(workspace, tree_commit_workspace_size(), device, stream)
    _check(load_library().sf_tree_commit(
        tokens.data_ptr(), sampled.data_ptr(), parents.data_ptr(), k_ptrs, v_ptrs, layers, block_table.data_ptr(),
        seq_lens.data_ptr(), B, n, H_kv, d, page, num_pages, max_pages, num_accepted.data_ptr(), out_tokens.data_ptr(),
        path.data_ptr(), row_weights.data_ptr(), n if n_q_next is None else n_q_next, free, count, capacity,
        workspace.data_ptr(), workspace.numel(), _stream_handle(stream)))
    return num_accepted, out_tokens, path, row_weights


def attention_mass_workspace_size() -> int:
    return int(load_library().sf_attention_mass_workspace_size())


def attention_mass(q, lse, k_cache, block_table, seq_lens, mass=None, *, row_weights=None, out=None,
                   softmax_scale=0.0, workspace=None, stream=None):
    """sf_attention_mass: the attention weight that the n_q rows of an attention call
    gave each key of the context, per KV head.  q, k_cache, block_table and seq_lens
    are that call's, lse what it returned; mass fp32 [B][H_kv][width] is added to
    (None: 0), row_weights fp32 [B][n_q] weighs the rows (None: 1).  Returns out fp32
    [B][H_kv][width], which may be mass; its entries from a sequence's context on
    (seq_lens - n_q) are not written (a new one has zeros there, or mass's)."""
    if _calls is not None and out is not None and workspace is not None and stream is None:
        status = _calls.attention_mass(q, lse, k_cache, block_table, seq_lens, mass, row_weights, softmax_scale, out,
                                       workspace)
        if status is not None:
            if status:
                _check(status)
            return out
    B, n_q, H_q, H_kv, d, page, num_pages, max_pages = _attention_arguments(q, k_cache, block_table, seq_lens)
    _need(lse, "lse", _F32, (B, n_q, H_q))
    if mass is not None:
        if not isinstance(mass, _Tensor) or mass.dim() != 3 or mass.shape[:2] != (B, H_kv):
            raise ValueError(f"mass must be a tensor [{B}][{H_kv}][width]")
        _need(mass, "mass", _F32)
    if row_weights is not None:
        _need(row_weights, "row_weights", _F32, (B, n_q))
    if out is None:
        shape = (B, H_kv, max_pages * page) if mass is None else mass.shape
        out = _new(shape, _F32, q.device, stream, zero=True)
        if mass is not None:
            with torch.cuda.stream(stream):
                out.copy_(mass)
    if not isinstance(out, _Tensor) or out.dim() != 3 or out.shape[:2] != (B, H_kv):
        raise ValueError(f"out must be a tensor [{B}][{H_kv}][width]")
    _need(out, "out", _F32, out.shape if mass is None else mass.shape)
    workspace = _workspace(workspace, attention_mass_workspace_size(), q.device, stream)
    _check(load_library().sf_attention_mass(
        q.data_ptr(), lse.data_ptr(), k_cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), _ptr(mass),
        _ptr(row_weights), B, n_q, H_q, H_kv, d, page, num_pages, max_pages, out.shape[2], softmax_scale,
        out.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream_handle(stream)))
    return out


def kv_evict_workspace_size(num_layers, B, H_kv, budget) -> int:
    n = load_library().sf_kv_evict_workspace_size(num_layers, B, H_kv, budget)
    if n == 0:
        raise SFError(1, "invalid eviction shape: " + load_library().sf_last_error().decode())
    return int(n)


def kv_evict(mass, k_caches, v_caches, block_table, seq_lens, budget, *, first=0, recent=0, n_q=0, mass_out=None,
             seq_lens_out=None, kept=None, free_pages=None, free_count=None, workspace=None, stream=None):
    """sf_kv_evict: cuts every sequence of more than `budget` tokens (seq_lens - n_q) to
    its budget.  Per layer and KV head the `first` tokens, the last `recent` ones and
    those of largest mass stay, in their order; K, V and mass are compacted.  mass
    fp32 [layers][B][H_kv][width], k_caches and v_caches bf16
    [layers][pages][H_kv][16][d], mass_out (None: mass itself) and kept int32
    [layers][B][H_kv][budget] (the kept positions; None: not wanted): one tensor, or
    a list of the layers'.  seq_lens_out None: seq_lens itself.  With free_pages and
    free_count the pages that are no longer needed go back to that stack.  Returns
    (mass_out, seq_lens_out, kept)."""
    if mass_out is None:
        mass_out = mass
    if seq_lens_out is None:
        seq_lens_out = seq_lens
    if _calls is not None and workspace is not None and stream is None:
        status = _calls.kv_evict(mass, k_caches, v_caches, block_table, seq_lens, budget, first, recent, n_q, mass_out,
                                 seq_lens_out, kept, free_pages, free_count, workspace)
        if status is not None:
            if status:
                _check(status)
            return mass_out, seq_lens_out, kept
    B, max_pages = _matrix(block_table, "block_table", _I32)
    _need(seq_lens, "seq_lens", _I32, (B,))
    _need(seq_lens_out, "seq_lens_out", _I32, (B,))
    k_ptrs, layers, cache = _layer_pointers(k_caches, "k_caches", _BF16, 4)
    v_ptrs, v_layers, _ = _layer_pointers(v_caches, "v_caches", _BF16, 4, cache)
    m_ptrs, m_layers, m = _layer_pointers(mass, "mass", _F32, 3)
    o_ptrs, o_layers, _ = _layer_pointers(mass_out, "mass_out", _F32, 3, m)
    counts = {"mass": m_layers, "k_caches": layers, "v_caches": v_layers, "mass_out": o_layers}
    _same_count(counts)
    if not layers:
        raise ValueError("no layers")
    num_pages, H_kv, page, d = cache
    if tuple(m[:2]) != (B, H_kv):
        raise ValueError(f"mass has layers of shape {tuple(m)}, expected ({B}, {H_kv}, width)")
    kept_ptrs = None
    if kept is not None:
        kept_ptrs, counts["kept"], _ = _layer_pointers(kept, "kept", _I32, 3, (B, H_kv, budget))
        _same_count(counts)
    free, count, capacity = _free_stack(free_pages, free_count)
    if workspace is None:
        size = kv_evict_workspace_size(layers, B, H_kv, budget) if kept is None else 256
        workspace = _new(size, _U8, block_table.device, stream, zero=True)
    _need_workspace(workspace)
    _check(load_library().sf_kv_evict(
        m_ptrs, k_ptrs, v_ptrs, layers, block_table.data_ptr(), seq_lens.data_ptr(), B, H_kv, d, page, num_pages,
        max_pages, m[2], budget, first, recent, n_q, o_ptrs, seq_lens_out.data_ptr(), kept_ptrs, free, count, capacity,
        workspace.data_ptr(), workspace.numel(), _stream_handle(stream)))
    return mass_out, seq_lens_out, kept
