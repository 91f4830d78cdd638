// kv_append.cu -- rotary position encoding of a layer's new rows, and their
// keys' and values' way into the paged cache.
//
// Angles: pair j of row t turns by positions[axis_j][t] * inv_freq[j] radians.
// The turn is taken in 64-bit fixed point: step_j = the fraction of one turn per
// position, as round(2^64 * frac(inv_freq[j] / 2 pi)); position * step_j modulo
// 2^64 is the exact fraction of a turn for every int32 position, negative ones
// included, and its upper 32 bits go through sincospif.  (fp32 angles are off by
// 2^-24 of the angle, 2e-3 radians at position 32768.)
//
// One CTA per row.
#include <cmath>

#include "sf_device.cuh"
#include "sf_host.h"

namespace sf {

constexpr int kAppendThreads = 256;
constexpr int kMaxHeadDim = 256;
constexpr int kMaxHeads = 1024;

struct AppendParams {
  const void *q, *k, *v;
  long long q_row, q_head, k_row, k_head, v_row, v_head;
  const int32_t *positions;
  const double *inv_freq;
  const int32_t *freq_axis;
  const int32_t *block_table;
  const int32_t *seq_lens;
  const int32_t *row_starts;
  __nv_bfloat16 *q_out, *k_cache, *v_cache;
  uint32_t *status;
  int T, B, H_q, H_kv, D, num_pages, max_pages, axes, pairs, interleaved, wide, rows;
  float amplitude;
};

// cos and sin (times the amplitude) of pair j of row t
__device__ __forceinline__ float2 pair_turn(const AppendParams &p, int t, int j) {
  int axis = p.freq_axis ? p.freq_axis[j] : 0;
  if (axis < 0 || axis >= p.axes) {
    set_status(p.status, SF_DEVICE_BAD_INDEX);
    axis = 0;
  }
  double turns = p.inv_freq[j] * 0.15915494309189535;  // 1 / (2 pi)
  turns -= floor(turns);
  const unsigned long long step = __double2ull_rn(turns * 18446744073709551616.0);
  const long long pos = p.positions[static_cast<size_t>(axis) * p.T + t];
  const int hi = static_cast<int>(static_cast<unsigned long long>(pos) * step >> 32);
  float s, c;
  sincospif(static_cast<float>(hi) * 4.656612873077393e-10f, &s, &c);  // 2^-31: half turns
  return make_float2(c * p.amplitude, s * p.amplitude);
}

// The cache page and slot of row t: -1 where the row is not appended.
__device__ __forceinline__ int row_place(const AppendParams &p, int t, int &slot) {
  int b, i, n;
  if (p.row_starts) {
    int lo = 0, hi = p.B;  // last sequence that starts at or before t
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (p.row_starts[mid] <= t) lo = mid + 1; else hi = mid;
    }
    b = lo - 1;
    if (b < 0) {
      set_status(p.status, SF_DEVICE_BAD_INDEX);
      return -1;
    }
    const int first = p.row_starts[b], end = p.row_starts[b + 1];
    if (t >= end) {
      if (b != p.B - 1) set_status(p.status, SF_DEVICE_BAD_INDEX);
      return -1;  // padding
    }
    i = t - first;
    n = end - first;
  } else {
    b = t / p.rows;
    i = t - b * p.rows;
    n = p.rows;
  }
  const int len = p.seq_lens[b];
  if (len == 0) return -1;  // idle slot
  const long long at = static_cast<long long>(len) - n + i;
  if (at < 0 || at >= static_cast<long long>(p.max_pages) * SF_PAGE_SIZE) {
    set_status(p.status, SF_DEVICE_BAD_SEQLEN);
    return -1;
  }
  slot = static_cast<int>(at % SF_PAGE_SIZE);
  const int page = p.block_table[static_cast<size_t>(b) * p.max_pages + at / SF_PAGE_SIZE];
  if (page < 0 || page >= p.num_pages) {
    set_status(p.status, SF_DEVICE_BAD_PAGE);
    return -1;
  }
  return page;
}

__device__ __forceinline__ float load_as_float(const void *p, long long i, int wide) {
  return wide ? static_cast<const float *>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(const __grid_constant__ AppendParams p) {
  __shared__ float2 s_turn[kMaxHeadDim / 2];
  __shared__ int s_place[2];
  const int tid = threadIdx.x, t = blockIdx.x;
  grid_dependency_wait();
  for (int j = tid; j < p.pairs; j += kAppendThreads) s_turn[j] = pair_turn(p, t, j);
  if (tid == 0) {
    int slot = 0;
    s_place[0] = row_place(p, t, slot);
    s_place[1] = slot;
  }
  __syncthreads();
  const int page = s_place[0], slot = s_place[1];
  const int per = p.D - p.pairs;  // items of a rotated head: its pairs, then the single elements
  const int heads = p.H_q + (page >= 0 ? p.H_kv : 0);
  for (int x = tid; x < heads * per; x += kAppendThreads) {
    const int h = x / per, e = x - h * per;
    const bool is_q = h < p.H_q;
    const void *src = is_q ? p.q : p.k;
    const long long so = is_q ? t * p.q_row + h * p.q_head : t * p.k_row + (h - p.H_q) * p.k_head;
    __nv_bfloat16 *dst = is_q ? p.q_out + (static_cast<size_t>(t) * p.H_q + h) * p.D
                              : p.k_cache + ((static_cast<size_t>(page) * p.H_kv + h - p.H_q) * SF_PAGE_SIZE + slot) * p.D;
    if (e < p.pairs) {
      const int i0 = p.interleaved ? 2 * e : e, i1 = p.interleaved ? 2 * e + 1 : e + p.pairs;
      const float a = load_as_float(src, so + i0, p.wide), b = load_as_float(src, so + i1, p.wide);
      const float2 w = s_turn[e];
      dst[i0] = __float2bfloat16_rn(a * w.x - b * w.y);
      dst[i1] = __float2bfloat16_rn(a * w.y + b * w.x);
    } else {
      const int i = e + p.pairs;
      dst[i] = __float2bfloat16_rn(load_as_float(src, so + i, p.wide));
    }
  }
  if (page < 0) return;
  for (int x = tid; x < p.H_kv * p.D; x += kAppendThreads) {
    const int h = x / p.D, e = x - h * p.D;
    p.v_cache[((static_cast<size_t>(page) * p.H_kv + h) * SF_PAGE_SIZE + slot) * p.D + e] =
        __float2bfloat16_rn(load_as_float(p.v, t * p.v_row + h * p.v_head + e, p.wide));
  }
}

}  // namespace sf

extern "C" {

size_t sf_kv_append_workspace_size(void) { return 256; }

int sf_kv_append(const void *q, const void *k, const void *v, int dtype, long long q_row_stride,
                 long long q_head_stride, long long k_row_stride, long long k_head_stride,
                 long long v_row_stride, long long v_head_stride, const int32_t *positions,
                 int axes, const double *inv_freq, const int32_t *freq_axis, int rotary_dim,
                 int interleaved, float amplitude, const int32_t *block_table,
                 const int32_t *seq_lens, const int32_t *row_starts, int T, int B, int H_q,
                 int H_kv, int head_dim, int page_size, int num_pages, int max_pages_per_seq,
                 void *q_out, void *k_cache, void *v_cache, void *workspace,
                 size_t workspace_bytes, cudaStream_t stream) {
  using namespace sf;
  clear_error();
  if (dtype != SF_BF16 && dtype != SF_F32) return fail(SF_ERR_UNSUPPORTED, "dtype=%d (built: bf16, fp32)", dtype);
  if (T < 0) return fail(SF_ERR_INVALID_ARG, "T=%d is negative", T);
  if (B < 1 || B > SF_MAX_BATCH) return fail(SF_ERR_INVALID_ARG, "B=%d outside [1, %d]", B, SF_MAX_BATCH);
  if (H_q < 0 || H_q > kMaxHeads || H_kv < 1 || H_kv > kMaxHeads)
    return fail(SF_ERR_INVALID_ARG, "H_q=%d, H_kv=%d outside [0, %d], [1, %d]", H_q, H_kv, kMaxHeads, kMaxHeads);
  if (head_dim < 8 || head_dim > kMaxHeadDim || head_dim % 8 != 0)
    return fail(SF_ERR_UNSUPPORTED, "head_dim=%d (built: multiples of 8 in [8, %d])", head_dim, kMaxHeadDim);
  if (page_size != SF_PAGE_SIZE) return fail(SF_ERR_UNSUPPORTED, "page_size=%d (built: 16)", page_size);
  if (max_pages_per_seq < 1 || (long long)max_pages_per_seq * page_size > (1LL << 30))
    return fail(SF_ERR_INVALID_ARG, "max_pages_per_seq=%d", max_pages_per_seq);
  if (num_pages < 1) return fail(SF_ERR_INVALID_ARG, "num_pages=%d", num_pages);
  if (rotary_dim < 0 || rotary_dim > head_dim || rotary_dim % 2 != 0)
    return fail(SF_ERR_INVALID_ARG, "rotary_dim=%d must be even and in [0, head_dim]", rotary_dim);
  if (rotary_dim > 0 && (axes < 1 || axes > SF_MAX_AXES))
    return fail(SF_ERR_INVALID_ARG, "axes=%d outside [1, %d]", axes, SF_MAX_AXES);
  if (!std::isfinite(amplitude)) return fail(SF_ERR_INVALID_ARG, "amplitude must be finite");
  if (!row_starts && T % B != 0) return fail(SF_ERR_INVALID_ARG, "T=%d is no multiple of B=%d (give row_starts)", T, B);
  if (T == 0) return SF_OK;
  if (!k || !v || !k_cache || !v_cache || !block_table || !seq_lens || (H_q > 0 && (!q || !q_out)) ||
      (rotary_dim > 0 && (!positions || !inv_freq)))
    return fail(SF_ERR_INVALID_ARG, "a required pointer is NULL");
  const size_t e = dtype == SF_F32 ? 4 : 2;
  if ((H_q > 0 && (!aligned(q, e) || !aligned(q_out, 16))) || !aligned(k, e) || !aligned(v, e) ||
      !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(block_table, 4) || !aligned(seq_lens, 4) ||
      (row_starts && !aligned(row_starts, 4)) || (positions && !aligned(positions, 4)) ||
      (inv_freq && !aligned(inv_freq, 8)) || (freq_axis && !aligned(freq_axis, 4)))
    return fail(SF_ERR_INVALID_ARG, "q_out and caches must be 16-byte aligned, other arrays to their elements");
  if (!workspace || !aligned(workspace, 256))
    return fail(SF_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
  if (workspace_bytes < sf_kv_append_workspace_size())
    return fail(SF_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes,
                sf_kv_append_workspace_size());
  AppendParams p;
  p.q = q;
  p.k = k;
  p.v = v;
  p.q_row = q_row_stride;
  p.q_head = q_head_stride;
  p.k_row = k_row_stride;
  p.k_head = k_head_stride;
  p.v_row = v_row_stride;
  p.v_head = v_head_stride;
  p.positions = positions;
  p.inv_freq = inv_freq;
  p.freq_axis = freq_axis;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.row_starts = row_starts;
  p.q_out = static_cast<__nv_bfloat16 *>(q_out);
  p.k_cache = static_cast<__nv_bfloat16 *>(k_cache);
  p.v_cache = static_cast<__nv_bfloat16 *>(v_cache);
  p.status = static_cast<uint32_t *>(workspace);
  p.T = T;
  p.B = B;
  p.H_q = H_q;
  p.H_kv = H_kv;
  p.D = head_dim;
  p.num_pages = num_pages;
  p.max_pages = max_pages_per_seq;
  p.axes = axes;
  p.pairs = rotary_dim / 2;
  p.interleaved = interleaved != 0;
  p.wide = dtype == SF_F32;
  p.rows = T / B;
  p.amplitude = amplitude;
  kv_append_kernel<<<T, kAppendThreads, 0, stream>>>(p);
  const cudaError_t err = cudaGetLastError();
  if (err != cudaSuccess) return fail(SF_ERR_CUDA, "kv append launch: %s", cudaGetErrorString(err));
  return SF_OK;
}

}  // extern "C"
