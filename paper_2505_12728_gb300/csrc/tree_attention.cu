// tree_attention.cu -- verification attention of a tree of drafted tokens.
//
// Row i of sequence b sees the L_b = seq_lens[b] - n_q tokens of the context and
// those of the n_q new rows whose bit its mask has:
//   s_t = scale <q, k_t>,  lse = ln sum_t exp(s_t),  out = sum_t exp(s_t - lse) v_t.
//
// A block takes one query row of one head; its warps take the keys in turn, each
// with a running maximum, sum and output, and are joined at the end.
#include <cmath>

#include "sf_device.cuh"
#include "sf_host.h"

namespace sf {

struct TreeAttnParams {
  const __nv_bfloat16 *q, *k_cache, *v_cache;
  const int32_t *block_table, *seq_lens;
  const unsigned long long *mask;
  long long mask_stride;
  __nv_bfloat16 *out;
  float *lse;
  uint32_t *status;
  int n_q, H_q, H_kv, group, num_pages, max_pages;
  float scale_log2;
};

constexpr int kTreeAttnWarps = 4;

template <int D>
__global__ void __launch_bounds__(32 * kTreeAttnWarps) tree_attention_kernel(const __grid_constant__ TreeAttnParams p) {
  constexpr int E = D / 32;  // elements of a row a lane has
  __shared__ float s_o[kTreeAttnWarps][D], s_m[kTreeAttnWarps], s_l[kTreeAttnWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z;
  grid_dependency_wait();
  grid_launch_dependents();
  int T = p.seq_lens[b];
  if (T != 0 && (T < p.n_q || T > p.max_pages * SF_PAGE_SIZE)) {
    if (threadIdx.x == 0) set_status(p.status, SF_DEVICE_BAD_SEQLEN);
    T = T < p.n_q ? p.n_q : p.max_pages * SF_PAGE_SIZE;
  }
  const int before = T - p.n_q;
  const unsigned long long mask = p.mask[b * p.mask_stride + i];
  const size_t row = (static_cast<size_t>(b) * p.n_q + i) * p.H_q + h;
  float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) q[e] = __bfloat162float(p.q[row * D + lane + 32 * e]);
  for (int t = warp; t < T; t += kTreeAttnWarps) {
    if (t >= before && !((mask >> (t - before)) & 1ull)) continue;
    const int page = p.block_table[static_cast<size_t>(b) * p.max_pages + t / SF_PAGE_SIZE];
    const bool in = page >= 0 && page < p.num_pages;
    if (!in && lane == 0) set_status(p.status, SF_DEVICE_BAD_PAGE);
    const size_t at = ((static_cast<size_t>(in ? page : 0) * p.H_kv + h / p.group) * SF_PAGE_SIZE + t % SF_PAGE_SIZE) * D + lane;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(q[e], in ? __bfloat162float(p.k_cache[at + 32 * e]) : 0.f, s);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= p.scale_log2;
    const float top = fmaxf(m, s), a = top == -INFINITY ? 0.f : exp2f(m - top), w = s == -INFINITY ? 0.f : exp2f(s - top);
    l = l * a + w;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * a + w * (in ? __bfloat162float(p.v_cache[at + 32 * e]) : 0.f);
    m = top;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) s_o[warp][lane + 32 * e] = o[e];
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
  __syncthreads();
  float M = -INFINITY, L = 0.f;
  for (int w = 0; w < kTreeAttnWarps; ++w) M = fmaxf(M, s_m[w]);
  if (M == -INFINITY) M = 0.f;
  for (int w = 0; w < kTreeAttnWarps; ++w) L += s_l[w] * exp2f(s_m[w] - M);
  for (int c = threadIdx.x; c < D; c += 32 * kTreeAttnWarps) {
    float x = 0.f;
    for (int w = 0; w < kTreeAttnWarps; ++w) x += s_o[w][c] * exp2f(s_m[w] - M);
    p.out[row * D + c] = __float2bfloat16_rn(L == 0.f ? 0.f : x / L);
  }
  if (p.lse && threadIdx.x == 0) p.lse[row] = (M + log2f(L)) * 0.6931471805599453f;
}

static int check_tree_attention(int B, int n_q, int H_q, int H_kv, int D, int max_pages, int page_size) {
  if (B < 1 || B > SF_MAX_BATCH) return fail(SF_ERR_INVALID_ARG, "B=%d outside [1, %d]", B, SF_MAX_BATCH);
  if (n_q < 1 || n_q > SF_MAX_TREE_ROWS)
    return fail(SF_ERR_INVALID_ARG, "n_q=%d outside [1, %d]", n_q, SF_MAX_TREE_ROWS);
  if (H_kv < 1 || H_q < 1 || H_q % H_kv != 0)
    return fail(SF_ERR_INVALID_ARG, "H_q=%d must be a positive multiple of H_kv=%d", H_q, H_kv);
  if (H_q / H_kv > SF_MAX_GROUP)
    return fail(SF_ERR_UNSUPPORTED, "group H_q/H_kv=%d above %d", H_q / H_kv, SF_MAX_GROUP);
  if (D != 64 && D != 128) return fail(SF_ERR_UNSUPPORTED, "head_dim=%d (built: 64, 128)", D);
  if (page_size != SF_PAGE_SIZE) return fail(SF_ERR_UNSUPPORTED, "page_size=%d (built: 16)", page_size);
  if (max_pages < 1 || (long long)max_pages * page_size > (1LL << 30))
    return fail(SF_ERR_INVALID_ARG, "max_pages_per_seq=%d", max_pages);
  return SF_OK;
}

}  // namespace sf

extern "C" {

size_t sf_tree_attention_workspace_size(int B, int n_q, int H_q, int H_kv, int head_dim, int max_pages_per_seq,
                                        int page_size) {
  return sf::check_tree_attention(B, n_q, H_q, H_kv, head_dim, max_pages_per_seq, page_size) == SF_OK ? 256 : 0;
}

int sf_tree_attention(const void *q, const void *k_cache, const void *v_cache, const int32_t *block_table,
                      const int32_t *seq_lens, const uint64_t *tree_mask, long long mask_stride, int B, int n_q,
                      int H_q, int H_kv, int head_dim, int page_size, int num_pages, int max_pages_per_seq,
                      float softmax_scale, void *out, float *lse, void *workspace, size_t workspace_bytes,
                      cudaStream_t stream) {
  using namespace sf;
  clear_error();
  const int st = check_tree_attention(B, n_q, H_q, H_kv, head_dim, max_pages_per_seq, page_size);
  if (st != SF_OK) return st;
  if (!q || !k_cache || !v_cache || !block_table || !seq_lens || !tree_mask || !out)
    return fail(SF_ERR_INVALID_ARG, "a required pointer is NULL");
  if (num_pages < 1) return fail(SF_ERR_INVALID_ARG, "num_pages=%d", num_pages);
  if ((long long)num_pages * H_kv * SF_PAGE_SIZE >= (1LL << 31))
    return fail(SF_ERR_UNSUPPORTED, "KV pool of %d pages x %d heads too large", num_pages, H_kv);
  if (mask_stride != 0 && mask_stride < n_q)
    return fail(SF_ERR_INVALID_ARG, "mask_stride=%lld: 0 (one tree for all) or at least n_q", mask_stride);
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16) ||
      !aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(tree_mask, 8) || !aligned(lse, 4))
    return fail(SF_ERR_INVALID_ARG,
                "q, caches and out must be 16-byte aligned, tree_mask 8-byte, other arrays 4-byte aligned");
  if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale))
    return fail(SF_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0");
  if (!workspace || !aligned(workspace, 256))
    return fail(SF_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
  if (workspace_bytes < 256) return fail(SF_ERR_WORKSPACE, "workspace has %zu bytes, needs 256", workspace_bytes);
  TreeAttnParams p;
  p.q = static_cast<const __nv_bfloat16 *>(q);
  p.k_cache = static_cast<const __nv_bfloat16 *>(k_cache);
  p.v_cache = static_cast<const __nv_bfloat16 *>(v_cache);
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.mask = reinterpret_cast<const unsigned long long *>(tree_mask);
  p.mask_stride = mask_stride;
  p.out = static_cast<__nv_bfloat16 *>(out);
  p.lse = lse;
  p.status = static_cast<uint32_t *>(workspace);
  p.n_q = n_q;
  p.H_q = H_q;
  p.H_kv = H_kv;
  p.group = H_q / H_kv;
  p.num_pages = num_pages;
  p.max_pages = max_pages_per_seq;
  p.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim)) * 1.4426950408889634f;
  const dim3 grid(H_q, n_q, B);
  if (head_dim == 128) tree_attention_kernel<128><<<grid, 32 * kTreeAttnWarps, 0, stream>>>(p);
  else tree_attention_kernel<64><<<grid, 32 * kTreeAttnWarps, 0, stream>>>(p);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(SF_ERR_CUDA, "tree attention launch: %s", cudaGetErrorString(e));
  return SF_OK;
}

}  // extern "C"
