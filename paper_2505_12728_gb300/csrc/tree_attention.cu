// tree_attention.cu -- verification attention of a tree of drafted tokens.
//
// Row i of sequence b sees the L_b = seq_lens[b] - n_q tokens of the context and
// those of the n_q new rows whose bit its mask has:
//   s_t = scale <q, k_t>,  lse = ln sum_t exp(s_t),  out = sum_t exp(s_t - lse) v_t.
//
// The kernels are those of shared_prefix_kernel.cuh with one segment list: a sequence's
// rows for one KV head (n_q nodes x g query heads) are packed into row tiles of whole
// nodes, up to four; two tiles a segment share each key tile that is copied, and where
// all rows fit one tile two KV heads make a segment, a stream each.  A row's mask is one
// 64-bit word.  Only the key tiles that hold new rows look at it: the word, shifted to
// where the tile begins, gives a bit per key.  Masked rows of K drop out as -infinity
// before the maximum is taken, infinities and NaN in masked rows of V are taken out of
// the tile and added to the rows that see them.
//
// What bounds it.  Many rows (16 sequences of 8192 to 32768 tokens, 61 nodes, 28 / 4 heads:
// 242 us, 1.08 PFLOP/s, 1.29 with the rows that fill the four tiles up): the MMAs and the
// softmax between them, tensor pipe active 67 %; neighbouring CTAs take the two pairs of row
// tiles of the same keys, so that K and V come from memory once (271 of 536 MB at 4 x 32768
// tokens).  Few rows and keys: the chain.  Of the 17 us of 26 nodes, 3008 tokens, 32 heads
// (7.4 for the bytes) 2.1 go by from the lengths to the first copy, 2.4 to the first keys,
// 7.5 to the last, 1.8 to the last CTA's end, 1.3 to the merge kernel, 2 in it.  Not kept:
// the merge by whichever CTA ends last (21.9 us; with 224 rows 59 for 23.3: 1.3 MB of partials
// for one SM), clusters that join in shared memory (18.7, 9.8 for 9.3 with 5 nodes and 640
// tokens, 29.5 for 23.2 with 224 rows), a CTA for every short segment (7.1 for 8.9 with one key
// tile, but 11.6 for 10.1 with six), the block table fetched to L2 ahead (no change).
#include "shared_prefix_kernel.cuh"

namespace sf {

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

// Upper bounds over all lengths of B sequences.
static SpBounds tree_bounds(int B, int n_q, int H_q, int H_kv, int max_pages, int G) {
  const long long key_tiles = ((long long)max_pages + kSpTilePages - 1) / kSpTilePages;
  SpBounds b;
  b.cost = (long long)B * H_kv * (kSpCostSegTwo + kSpCostFew + std::max(kSpCostTwo, 2 * kSpCostOne) * key_tiles);
  b.rows = sp_tree_rows(B, n_q, H_q / H_kv, H_kv, G);
  return b;
}

}  // namespace sf

extern "C" {

size_t sf_tree_attention_workspace_size(int B, int n_q, int H_q, int H_kv, int head_dim, int max_pages_per_seq,
                                        int page_size) {
  using namespace sf;
  int G = 0;
  if (check_tree_attention(B, n_q, H_q, H_kv, head_dim, max_pages_per_seq, page_size) != SF_OK || sp_grid(&G) != SF_OK)
    return 0;
  return sp_layout(tree_bounds(B, n_q, H_q, H_kv, max_pages_per_seq, G), head_dim, B).total;
}

int sf_tree_attention(const void *q, const void *k_cache, const void *v_cache, const int32_t *block_table,
                      const int32_t *seq_lens, const uint64_t *tree_mask, long long mask_stride, int B, int n_q,
                      int H_q, int H_kv, int head_dim, int page_size, int num_pages, int max_pages_per_seq,
                      float softmax_scale, void *out, float *lse, void *workspace, size_t workspace_bytes,
                      cudaStream_t stream) {
  using namespace sf;
  clear_error();
  int st = check_tree_attention(B, n_q, H_q, H_kv, head_dim, max_pages_per_seq, page_size);
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
  DeviceInfo dev;
  int G = 0;
  if ((st = sp_grid(&G)) != SF_OK || (st = current_device(&dev)) != SF_OK) return st;
  const SpBounds bounds = tree_bounds(B, n_q, H_q, H_kv, max_pages_per_seq, G);
  if (bounds.cost >= (1LL << 31) || bounds.rows >= (1LL << 31))
    return fail(SF_ERR_UNSUPPORTED, "up to %lld tiles and %lld partial rows (limits 2^31)", bounds.cost, bounds.rows);
  const SpLayout lay = sp_layout(bounds, head_dim, B);
  if (workspace_bytes < lay.total)
    return fail(SF_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, lay.total);
  if ((st = sp_setup<true>(dev.ordinal)) != SF_OK) return st;

  const uint64_t rows = (uint64_t)num_pages * H_kv * SF_PAGE_SIZE;
  SpParams p{};
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.mask = reinterpret_cast<const unsigned long long *>(tree_mask);
  p.mask_stride = mask_stride;
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
  p.max_pages = max_pages_per_seq;
  p.tokens_per_tile = kSpTile / p.group;
  p.row_tiles = (n_q + p.tokens_per_tile - 1) / p.tokens_per_tile;
  // A stream a head where every SM has a whole head and more (8 sequences of 700 to 900
  // tokens, 32 heads: 32.7 us, with a head at a time 36.8), else a head's key tiles over
  // both streams, which leaves half as many partial results (4 sequences of 4864 tokens,
  // 4 heads, 112 rows: 22.2 -> 19.5).
  p.paired = p.row_tiles == 1 && B * H_kv >= G;
  p.tile_magic = static_cast<uint32_t>(((1ull << 32) + p.tokens_per_tile - 1) / p.tokens_per_tile);
  p.oob_row = static_cast<int>(rows);
  p.folds = (p.row_tiles + 1) / 2;
  p.fold_rows = static_cast<uint32_t>(bounds.rows / p.folds);
  p.G = G / p.folds;
  p.per_cta = 1.f / static_cast<float>(p.G);
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim);
  p.scale_log2 = scale * 1.4426950408889634f;
  CUtensorMap m[4];
  if ((st = sp_maps(m, k_cache, v_cache, q, rows, B, n_q, H_q, H_kv, head_dim, p.tokens_per_tile)) != SF_OK) return st;
  const int most = std::min((max_pages_per_seq + kSpTilePages - 1) / kSpTilePages, G / (B * H_kv) + 1);
  // With a segment and more for each CTA most segments are one piece (256 sequences of 508
  // tokens, 4 heads, 56 rows: 91.5 -> 80.2 us; of 216 tokens, 32 heads, 16 rows 367 -> 317), and
  // all are where a table has one key tile (6 sequences of 5 to 67 tokens, 3 heads, 4 to 252
  // rows: 9.1 -> 8.6 to 15.6 -> 13.2).  Otherwise hardly any are, and the code for them costs
  // (2 sequences of 645 tokens, 8 heads, 5 rows: 8.8 us, with it 9.1; 16 of 8 to 32 K tokens,
  // 4 heads, 427 rows: 233, 237).
  return B * H_kv >= p.G || max_pages_per_seq <= kSpTilePages ? sp_launch<true, true>(m, p, B, most, head_dim, stream)
                                                              : sp_launch<true, false>(m, p, B, most, head_dim, stream);
}

}  // extern "C"
