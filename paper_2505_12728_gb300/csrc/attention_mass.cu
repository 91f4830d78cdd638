// attention_mass.cu -- the attention weight that each cached key got.
//
//   out[b][h][t] = in[b][h][t] + sum_i w_i sum_j exp(scale <q_ij, k_t> - lse_ij)
//
// over the query rows i of sequence b, with weight w_i, and the query heads j of KV
// head h, for the L_b = seq_lens[b] - n_q keys of the context.
//
// A warp takes 32 keys of one KV head, a key a lane, and the rows one by one.
#include <cmath>

#include "sf_device.cuh"
#include "sf_host.h"

namespace sf {

struct MassParams {
  const __nv_bfloat16 *q, *k_cache;
  const float *lse, *mass, *weights;
  const int32_t *block_table, *seq_lens;
  float *out;
  uint32_t *status;
  int n_q, H_q, H_kv, group, num_pages, max_pages, width, D;
  float scale_log2;
};

constexpr int kMassThreads = 128;

__global__ void __launch_bounds__(kMassThreads) attention_mass_kernel(const __grid_constant__ MassParams p) {
  const int t = blockIdx.x * kMassThreads + threadIdx.x, h = blockIdx.y, b = blockIdx.z;
  grid_dependency_wait();
  grid_launch_dependents();
  const int T = p.seq_lens[b];
  int before = T - p.n_q;
  if (T != 0 && (before < 0 || T > p.max_pages * SF_PAGE_SIZE || before > p.width)) {
    if (threadIdx.x == 0) set_status(p.status, SF_DEVICE_BAD_SEQLEN);
    before = min(max(before, 0), min(p.width, p.max_pages * SF_PAGE_SIZE - p.n_q));
  }
  if (t >= before) return;
  const int page = p.block_table[static_cast<size_t>(b) * p.max_pages + t / SF_PAGE_SIZE];
  const bool in = page >= 0 && page < p.num_pages;
  if (!in) set_status(p.status, SF_DEVICE_BAD_PAGE);
  const __nv_bfloat16 *k = p.k_cache + ((static_cast<size_t>(in ? page : 0) * p.H_kv + h) * SF_PAGE_SIZE + t % SF_PAGE_SIZE) * p.D;
  float sum = 0.f;
  for (int i = 0; i < p.n_q; ++i) {
    const float w = p.weights ? p.weights[static_cast<size_t>(b) * p.n_q + i] : 1.f;
    if (w == 0.f) continue;
    for (int j = 0; j < p.group; ++j) {
      const size_t row = (static_cast<size_t>(b) * p.n_q + i) * p.H_q + h * p.group + j;
      const float lse = p.lse[row];
      if (lse == -INFINITY) continue;
      float s = 0.f;
      for (int e = 0; e < p.D; ++e) s = fmaf(__bfloat162float(p.q[row * p.D + e]), in ? __bfloat162float(k[e]) : 0.f, s);
      sum += w * exp2f(s * p.scale_log2 - lse * 1.4426950408889634f);
    }
  }
  const size_t at = (static_cast<size_t>(b) * p.H_kv + h) * p.width + t;
  p.out[at] = (p.mass ? p.mass[at] : 0.f) + sum;
}

}  // namespace sf

extern "C" {

size_t sf_attention_mass_workspace_size(void) { return 256; }

int sf_attention_mass(const void *q, const float *lse, const void *k_cache, const int32_t *block_table,
                      const int32_t *seq_lens, const float *mass, const float *row_weights, int B, int n_q, int H_q,
                      int H_kv, int head_dim, int page_size, int num_pages, int max_pages_per_seq, int mass_width,
                      float softmax_scale, float *mass_out, void *workspace, size_t workspace_bytes,
                      cudaStream_t stream) {
  using namespace sf;
  clear_error();
  if (B < 1 || B > SF_MAX_BATCH) return fail(SF_ERR_INVALID_ARG, "B=%d outside [1, %d]", B, SF_MAX_BATCH);
  if (n_q < 1 || n_q > SF_MAX_TREE_ROWS)
    return fail(SF_ERR_INVALID_ARG, "n_q=%d outside [1, %d]", n_q, SF_MAX_TREE_ROWS);
  if (H_kv < 1 || H_q < 1 || H_q % H_kv != 0)
    return fail(SF_ERR_INVALID_ARG, "H_q=%d must be a positive multiple of H_kv=%d", H_q, H_kv);
  if (H_q / H_kv > SF_MAX_GROUP)
    return fail(SF_ERR_UNSUPPORTED, "group H_q/H_kv=%d above %d", H_q / H_kv, SF_MAX_GROUP);
  if (head_dim != 64 && head_dim != 128) return fail(SF_ERR_UNSUPPORTED, "head_dim=%d (built: 64, 128)", head_dim);
  if (page_size != SF_PAGE_SIZE) return fail(SF_ERR_UNSUPPORTED, "page_size=%d (built: 16)", page_size);
  if (max_pages_per_seq < 1 || (long long)max_pages_per_seq * page_size > (1LL << 30))
    return fail(SF_ERR_INVALID_ARG, "max_pages_per_seq=%d", max_pages_per_seq);
  if (mass_width < 1 || mass_width > (1 << 30)) return fail(SF_ERR_INVALID_ARG, "mass_width=%d", mass_width);
  if (!q || !lse || !k_cache || !block_table || !seq_lens || !mass_out)
    return fail(SF_ERR_INVALID_ARG, "a required pointer is NULL");
  if (num_pages < 1) return fail(SF_ERR_INVALID_ARG, "num_pages=%d", num_pages);
  if ((long long)num_pages * H_kv * SF_PAGE_SIZE >= (1LL << 31))
    return fail(SF_ERR_UNSUPPORTED, "KV pool of %d pages x %d heads too large", num_pages, H_kv);
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(lse, 4) || !aligned(block_table, 4) ||
      !aligned(seq_lens, 4) || !aligned(mass, 4) || !aligned(row_weights, 4) || !aligned(mass_out, 4))
    return fail(SF_ERR_INVALID_ARG, "q and k_cache must be 16-byte aligned, other arrays 4-byte aligned");
  if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale))
    return fail(SF_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0");
  if (!workspace || !aligned(workspace, 256))
    return fail(SF_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
  if (workspace_bytes < 256) return fail(SF_ERR_WORKSPACE, "workspace has %zu bytes, needs 256", workspace_bytes);
  MassParams p;
  p.q = static_cast<const __nv_bfloat16 *>(q);
  p.k_cache = static_cast<const __nv_bfloat16 *>(k_cache);
  p.lse = lse;
  p.mass = mass;
  p.weights = row_weights;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.out = mass_out;
  p.status = static_cast<uint32_t *>(workspace);
  p.n_q = n_q;
  p.H_q = H_q;
  p.H_kv = H_kv;
  p.group = H_q / H_kv;
  p.num_pages = num_pages;
  p.max_pages = max_pages_per_seq;
  p.width = mass_width;
  p.D = head_dim;
  p.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim)) * 1.4426950408889634f;
  const int most = max_pages_per_seq * page_size;
  const dim3 grid((most + kMassThreads - 1) / kMassThreads, H_kv, B);
  attention_mass_kernel<<<grid, kMassThreads, 0, stream>>>(p);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(SF_ERR_CUDA, "attention mass launch: %s", cudaGetErrorString(e));
  return SF_OK;
}

}  // extern "C"
