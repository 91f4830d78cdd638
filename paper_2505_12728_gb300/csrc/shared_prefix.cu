// shared_prefix.cu -- verification attention of a batch whose sequences share long
// prefixes: checks, workspace and launch of shared_prefix_kernel.cuh's kernels.
#include "shared_prefix_kernel.cuh"

namespace sf {

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

// Upper bounds over all groupings of B sequences into num_groups groups.
static SpBounds sp_bounds(int B, int n_q, int H_q, int H_kv, int num_groups, int max_prefix_pages, int max_pages, int G) {
  const long long group = H_q / H_kv, per_tile = kSpTile / group, tokens = (long long)B * n_q;
  const long long prefix_tiles = ((long long)max_prefix_pages + kSpTilePages - 1) / kSpTilePages;
  const long long own_tiles = ((long long)max_pages + kSpTilePages - 1) / kSpTilePages;
  // a group of t tokens has ceil(t / per_tile) <= t / per_tile + 1 row tiles, and
  // at most half of that plus one pairs, of at most 2 * kSpTile partial rows each
  const long long tiles = tokens / per_tile + num_groups, pairs = tokens / (2 * per_tile) + num_groups;
  SpBounds b;
  b.cost = H_kv * (pairs * (kSpCostSegTwo + kSpCostFew) + tiles * prefix_tiles * kSpCostOne + B * (kSpCostSegOne + own_tiles * kSpCostOne));
  b.rows = H_kv * pairs * 2 * kSpTile + (H_kv + 1) * tokens * group + 2LL * kSpTile * G;
  return b;
}

}  // namespace sf

extern "C" {

size_t sf_shared_prefix_attention_workspace_size(int B, int n_q, int H_q, int H_kv, int head_dim,
                                                 int num_groups, int max_prefix_pages,
                                                 int max_pages_per_seq, int page_size) {
  using namespace sf;
  int G = 0;
  if (check_sp_shapes(B, n_q, H_q, H_kv, head_dim, num_groups, max_prefix_pages, max_pages_per_seq, page_size) != SF_OK ||
      sp_grid(&G) != SF_OK)
    return 0;
  return sp_layout(sp_bounds(B, n_q, H_q, H_kv, num_groups, max_prefix_pages, max_pages_per_seq, G), head_dim, B)
      .total;
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
  DeviceInfo dev;
  int G = 0;
  if ((st = sp_grid(&G)) != SF_OK || (st = current_device(&dev)) != SF_OK) return st;
  const SpBounds bounds = sp_bounds(B, n_q, H_q, H_kv, num_groups, max_prefix_pages, max_pages_per_seq, G);
  if (bounds.cost >= (1LL << 31) || bounds.rows >= (1LL << 31))
    return fail(SF_ERR_UNSUPPORTED, "up to %lld tiles and %lld partial rows (limits 2^31)", bounds.cost, bounds.rows);
  const SpLayout lay = sp_layout(bounds, head_dim, B);
  if (workspace_bytes < lay.total)
    return fail(SF_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, lay.total);
  if ((st = sp_setup<false>(dev.ordinal)) != SF_OK) return st;

  const uint64_t rows = (uint64_t)num_pages * H_kv * SF_PAGE_SIZE;
  SpParams p{};
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  p.prefix_table = prefix_table;
  p.prefix_lens = prefix_lens;
  p.group_starts = group_starts;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.v_cache = static_cast<const __nv_bfloat16 *>(v_cache);
  p.out = static_cast<__nv_bfloat16 *>(out);
  p.lse = lse;
  p.status = reinterpret_cast<uint32_t *>(ws);
  p.plan = reinterpret_cast<SpRecord *>(ws + lay.plan_off);
  p.part_ml = reinterpret_cast<float2 *>(ws + lay.ml_off);
  p.part_o = reinterpret_cast<float *>(ws + lay.o_off);
  p.B = B;
  p.n_q = n_q;
  p.H_q = H_q;
  p.H_kv = H_kv;
  p.group = H_q / H_kv;
  p.num_pages = num_pages;
  p.num_groups = num_groups;
  p.max_prefix_pages = max_prefix_pages;
  p.max_pages = max_pages_per_seq;
  p.tokens_per_tile = kSpTile / p.group;
  p.tile_magic = static_cast<uint32_t>(((1ull << 32) + p.tokens_per_tile - 1) / p.tokens_per_tile);
  p.oob_row = static_cast<int>(rows);
  p.G = G;
  p.per_cta = 1.f / static_cast<float>(G);
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim);
  p.scale_log2 = scale * 1.4426950408889634f;
  CUtensorMap m[4];
  if ((st = sp_maps(m, k_cache, v_cache, q, rows, B, n_q, H_q, H_kv, head_dim, p.tokens_per_tile)) != SF_OK) return st;

  auto partials = [&](int pages, int segments) { return std::min((pages + kSpTilePages - 1) / kSpTilePages, G / segments + 1); };
  return sp_launch<false, false>(m, p, B, std::max(partials(max_prefix_pages, num_groups * H_kv), partials(max_pages_per_seq, B * H_kv)),
                          head_dim, stream);
}

}  // extern "C"
