// shared_prefix.cu -- verification attention of a batch whose sequences share
// long prefixes.  Row i of sequence b sees the prefix of its group and its own
// tokens 0 .. L_b + i.
//
// One warp per query row and head: each lane holds head_dim / 32 elements of q
// and of the output, keys come one at a time, with the running maximum and sum
// of the softmax.
#include <cmath>

#include "sf_device.cuh"
#include "sf_host.h"

namespace sf {

constexpr int kSpThreads = 128;

struct SpParams {
  const __nv_bfloat16 *q, *k_cache, *v_cache;
  const int32_t *prefix_table, *prefix_lens, *group_starts, *block_table, *seq_lens;
  __nv_bfloat16 *out;
  float *lse;
  uint32_t *status;
  int B, n_q, H_q, H_kv, group, num_pages, num_groups, max_prefix_pages, max_pages;
  float scale_log2;
};

template <int D>
__global__ void __launch_bounds__(kSpThreads) shared_prefix_kernel(const __grid_constant__ SpParams p) {
  constexpr int E = D / 32;
  constexpr float kLn2 = 0.6931471805599453f;
  __shared__ int s_bad;
  grid_dependency_wait();
  if (threadIdx.x == 0) s_bad = p.group_starts[0] != 0 || p.group_starts[p.num_groups] != p.B;
  __syncthreads();
  for (int g = threadIdx.x; g < p.num_groups; g += kSpThreads)
    if (p.group_starts[g + 1] < p.group_starts[g]) s_bad = 1;
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * (kSpThreads / 32) + warp;
  if (row >= static_cast<long long>(p.B) * p.n_q * p.H_q) return;
  const int hq = static_cast<int>(row % p.H_q), h = hq / p.group;
  const int bi = static_cast<int>(row / p.H_q), b = bi / p.n_q, i = bi - b * p.n_q;
  int L = p.seq_lens[b];
  const int most = p.max_pages * SF_PAGE_SIZE;
  if (L != 0 && (L < p.n_q || L > most)) {
    set_status(p.status, SF_DEVICE_BAD_SEQLEN);
    L = L < p.n_q ? p.n_q : most;
  }
  int P = 0, g = 0;
  if (s_bad) {
    set_status(p.status, SF_DEVICE_BAD_INDEX);
  } else {
    int lo = 0, hi = p.num_groups;  // the group: last g with starts[g] <= b
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (p.group_starts[mid] <= b) lo = mid + 1; else hi = mid;
    }
    g = lo - 1;
    P = p.prefix_lens[g];
    const int most_prefix = p.max_prefix_pages * SF_PAGE_SIZE;
    if (P < 0 || P > most_prefix) {
      set_status(p.status, SF_DEVICE_BAD_SEQLEN);
      P = P < 0 ? 0 : most_prefix;
    }
  }
  float q[E], o[E];
  for (int e = 0; e < E; ++e) {
    q[e] = __bfloat162float(p.q[row * D + lane * E + e]);
    o[e] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  for (int part = 0; part < 2 && L > 0; ++part) {
    const int32_t *table = part ? p.block_table + static_cast<size_t>(b) * p.max_pages
                                : p.prefix_table + static_cast<size_t>(g) * p.max_prefix_pages;
    const int keys = part ? L - p.n_q + i + 1 : P;
    for (int t = 0; t < keys; ++t) {
      const int page = table[t / SF_PAGE_SIZE];
      const bool in = page >= 0 && page < p.num_pages;
      if (!in && t % SF_PAGE_SIZE == 0) set_status(p.status, SF_DEVICE_BAD_PAGE);
      const size_t at = ((static_cast<size_t>(in ? page : 0) * p.H_kv + h) * SF_PAGE_SIZE + t % SF_PAGE_SIZE) * D + lane * E;
      float s = 0.f, v[E];
      for (int e = 0; e < E; ++e) {
        s += in ? q[e] * __bfloat162float(p.k_cache[at + e]) : 0.f;
        v[e] = in ? __bfloat162float(p.v_cache[at + e]) : 0.f;
      }
      for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
      s *= p.scale_log2;
      const float top = fmaxf(m, s), w = exp2f(s - top), a = exp2f(m - top);
      l = l * a + w;
      for (int e = 0; e < E; ++e) o[e] = o[e] * a + w * v[e];
      m = top;
    }
  }
  for (int e = 0; e < E; ++e) p.out[row * D + lane * E + e] = __float2bfloat16_rn(L > 0 ? o[e] / l : 0.f);
  if (p.lse && lane == 0) p.lse[row] = L > 0 ? (m + log2f(l)) * kLn2 : -INFINITY;
}

static int check_sp_shapes(int B, int n_q, int H_q, int H_kv, int D, int num_groups, int max_prefix_pages,
                           int max_pages, int page_size) {
  if (B < 1 || B > SF_MAX_BATCH) return fail(SF_ERR_INVALID_ARG, "B=%d outside [1, %d]", B, SF_MAX_BATCH);
  if (n_q < 1 || n_q > SF_MAX_QUERY_ROWS)
    return fail(SF_ERR_INVALID_ARG, "n_q=%d outside [1, %d]", n_q, SF_MAX_QUERY_ROWS);
  if (H_kv < 1 || H_q < 1 || H_q % H_kv != 0)
    return fail(SF_ERR_INVALID_ARG, "H_q=%d must be a positive multiple of H_kv=%d", H_q, H_kv);
  if (H_q / H_kv > SF_MAX_GROUP)
    return fail(SF_ERR_UNSUPPORTED, "group H_q/H_kv=%d above %d", H_q / H_kv, SF_MAX_GROUP);
  if (D != 64 && D != 128) return fail(SF_ERR_UNSUPPORTED, "head_dim=%d (built: 64, 128)", D);
  if (page_size != SF_PAGE_SIZE) return fail(SF_ERR_UNSUPPORTED, "page_size=%d (built: 16)", page_size);
  if (num_groups < 1 || num_groups > B)
    return fail(SF_ERR_INVALID_ARG, "num_groups=%d outside [1, B=%d]", num_groups, B);
  if (max_pages < 1 || (long long)max_pages * page_size > (1LL << 30))
    return fail(SF_ERR_INVALID_ARG, "max_pages_per_seq=%d", max_pages);
  if (max_prefix_pages < 1 || (long long)max_prefix_pages * page_size > (1LL << 30))
    return fail(SF_ERR_INVALID_ARG, "max_prefix_pages=%d", max_prefix_pages);
  return SF_OK;
}

}  // namespace sf

extern "C" {

size_t sf_shared_prefix_attention_workspace_size(int B, int n_q, int H_q, int H_kv, int head_dim,
                                                 int num_groups, int max_prefix_pages,
                                                 int max_pages_per_seq, int page_size) {
  if (sf::check_sp_shapes(B, n_q, H_q, H_kv, head_dim, num_groups, max_prefix_pages, max_pages_per_seq,
                          page_size) != SF_OK)
    return 0;
  return 256;
}

int sf_shared_prefix_attention(const void *q, const void *k_cache, const void *v_cache,
                               const int32_t *prefix_table, const int32_t *prefix_lens,
                               const int32_t *group_starts, const int32_t *block_table,
                               const int32_t *seq_lens, int B, int n_q, int H_q, int H_kv,
                               int head_dim, int page_size, int num_pages, int num_groups,
                               int max_prefix_pages, int max_pages_per_seq, float softmax_scale,
                               void *out, float *lse, void *workspace, size_t workspace_bytes,
                               cudaStream_t stream) {
  using namespace sf;
  clear_error();
  int st = check_sp_shapes(B, n_q, H_q, H_kv, head_dim, num_groups, max_prefix_pages, max_pages_per_seq, page_size);
  if (st != SF_OK) return st;
  if (!q || !k_cache || !v_cache || !prefix_table || !prefix_lens || !group_starts || !block_table || !seq_lens || !out)
    return fail(SF_ERR_INVALID_ARG, "a required pointer is NULL");
  if (num_pages < 1) return fail(SF_ERR_INVALID_ARG, "num_pages=%d", num_pages);
  if ((long long)num_pages * H_kv * SF_PAGE_SIZE >= (1LL << 31))
    return fail(SF_ERR_UNSUPPORTED, "KV pool of %d pages x %d heads too large", num_pages, H_kv);
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16) ||
      !aligned(prefix_table, 4) || !aligned(prefix_lens, 4) || !aligned(group_starts, 4) || !aligned(block_table, 4) ||
      !aligned(seq_lens, 4) || (lse && !aligned(lse, 4)))
    return fail(SF_ERR_INVALID_ARG, "q, caches and out must be 16-byte aligned, other arrays 4-byte aligned");
  if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale))
    return fail(SF_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0");
  if (!workspace || !aligned(workspace, 256))
    return fail(SF_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
  const size_t need = sf_shared_prefix_attention_workspace_size(B, n_q, H_q, H_kv, head_dim, num_groups,
                                                                max_prefix_pages, max_pages_per_seq, page_size);
  if (need == 0) return SF_ERR_CUDA;  // (sf_last_error says why)
  if (workspace_bytes < need)
    return fail(SF_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, need);
  SpParams p;
  p.q = static_cast<const __nv_bfloat16 *>(q);
  p.k_cache = static_cast<const __nv_bfloat16 *>(k_cache);
  p.v_cache = static_cast<const __nv_bfloat16 *>(v_cache);
  p.prefix_table = prefix_table;
  p.prefix_lens = prefix_lens;
  p.group_starts = group_starts;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.out = static_cast<__nv_bfloat16 *>(out);
  p.lse = lse;
  p.status = static_cast<uint32_t *>(workspace);
  p.B = B;
  p.n_q = n_q;
  p.H_q = H_q;
  p.H_kv = H_kv;
  p.group = H_q / H_kv;
  p.num_pages = num_pages;
  p.num_groups = num_groups;
  p.max_prefix_pages = max_prefix_pages;
  p.max_pages = max_pages_per_seq;
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim);
  p.scale_log2 = scale * 1.4426950408889634f;
  const long long rows = static_cast<long long>(B) * n_q * H_q;
  const unsigned grid = static_cast<unsigned>((rows + kSpThreads / 32 - 1) / (kSpThreads / 32));
  if (head_dim == 128) shared_prefix_kernel<128><<<grid, kSpThreads, 0, stream>>>(p);
  else shared_prefix_kernel<64><<<grid, kSpThreads, 0, stream>>>(p);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(SF_ERR_CUDA, "shared-prefix attention launch: %s", cudaGetErrorString(e));
  return SF_OK;
}

}  // extern "C"
