// tree_draft.cu -- drafts that are trees of tokens: the nodes' ancestor masks
// and positions, and, after the target has scored all nodes, the path that it
// takes through the tree.
//
// Node i of a tree of at most 64 hangs below node parents[i] < i; node 0 is the
// root, the token that the previous step emitted.  Both kernels keep a tree in a
// warp, two nodes a lane, and are latency-bound: some loads, a few rounds of
// shuffles, a store.  On the GPU (calls in a graph) the masks of one tree of 26 nodes
// take 0.9 us and those of 256 trees of 61 1.6, the commit of one sequence in 32 layers
// with 32 heads 3.7 (three dependent loads: the tree, the page, the row) and of 16
// sequences in 28 layers with 4 heads 4.3; called from Python 2.4, 2.8, 3.9 and 4.6.  The
// lengths and pages of the next tree are a second launch of one CTA: one sequence in 32 layers
// 6.2 us in a graph and 8.3 called, 3.8 and 4.1 without.
//
// tree_mask: mask[i] = bit i | mask[parents[i]].  Not node by node, but by
// doubling: every node knows the part of its ancestors that the last round
// found, and the node where that part ends; each round adds that node's part,
// so a tree of depth t takes log2(t) rounds, at most six.
//
// tree_commit: from the root, as long as a child carries the token that the
// target gives at its parent, the lowest such child is next (a sequence whose node
// 0 is no root has no path: its masks are 0).  The rows of the
// path then follow the context: row path[r] of keys and values moves to row r.
// path[r] >= r and ascends, so rows that are written never hold what a later row
// still has to be read from, and a warp that moves one KV head's rows of one layer
// in order (a batch's loads in front of its stores) needs nothing but its own order.
// Every warp takes the walk for itself: that is a few hundred cycles beside
// loads that every one of them needs anyway, and a second launch costs more.
#include "layer_device.cuh"
#include "sf_host.h"

namespace sf {

// kv_commit.cu: the pages and lengths after n_q verified rows (sf_kv_commit), where
// a length of 0 marks an idle slot and none of the rows stay where parents [B][n_q]
// has no root at node 0.
int launch_kv_commit(int32_t *seq_lens, int32_t *block_table, int32_t *free_pages, int32_t *free_count,
                     const int32_t *num_accepted, int B, int n_q, int n_q_next, int max_pages, int capacity,
                     const int32_t *parents, uint32_t *status, cudaStream_t stream);

constexpr int kTreeWarps = 4;
constexpr int kTreeBatch = 8;  // 16-byte loads of a thread in flight

// The value that node `at` has; a and b are this lane's nodes lane and lane + 32.
template <typename T>
__device__ __forceinline__ T of_node(T a, T b, int at) {
  const T x = __shfl_sync(0xffffffffu, a, at & 31), y = __shfl_sync(0xffffffffu, b, at & 31);
  return at & 32 ? y : x;
}

__global__ void __launch_bounds__(32 * kTreeWarps)
tree_mask_kernel(const int32_t *parents, const int32_t *start, int B, int n, unsigned long long *mask,
                 int32_t *positions, uint32_t *status) {
  const int lane = threadIdx.x & 31, b = blockIdx.x * kTreeWarps + uniform_warp_id();
  grid_dependency_wait();
  grid_launch_dependents();
  if (b >= B) return;
  const size_t row = static_cast<size_t>(b) * n;
  unsigned long long m[2];
  int up[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int i = lane + 32 * s;
    up[s] = i < n ? parents[row + i] : -2;
    if (up[s] >= i) {
      set_status(status, SF_DEVICE_BAD_INDEX);
      up[s] = -2;
    }
    m[s] = up[s] >= -1 ? 1ull << i : 0ull;  // 0: not part of the tree
  }
  while (__any_sync(0xffffffffu, up[0] >= 0 || up[1] >= 0)) {
    unsigned long long more[2];
    int next[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int at = up[s] < 0 ? 0 : up[s];
      more[s] = of_node(m[0], m[1], at);
      next[s] = of_node(up[0], up[1], at);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (up[s] < 0) continue;
      m[s] = more[s] ? m[s] | more[s] : 0ull;  // below a node that is not part of the tree
      up[s] = more[s] ? next[s] : -2;
    }
  }
  const int base = start && positions ? start[b] : 0;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int i = lane + 32 * s;
    if (i >= n) continue;
    mask[row + i] = m[s];
    if (positions) positions[row + i] = base + (m[s] ? __popcll(m[s]) - 1 : 0);
  }
}

struct TreeCommitParams {
  const int32_t *tokens, *sampled, *parents, *block_table, *seq_lens;
  int32_t *num_accepted, *out_tokens, *path;
  float *row_weights;
  uint32_t *status;
  int B, n, H_kv, D, num_pages, max_pages, layers;
  uint4 *caches[2 * SF_MAX_LAYERS];  // K, then V, of each layer
};

// What one warp does: KV head h of cache c (K, then V, of each layer) of sequence b;
// the sequence's first warp (at_head = 0) writes its results.
__device__ __forceinline__ void commit_rows(const TreeCommitParams &p, int b, int at_head, int c, int h, int lane) {
  const size_t row = static_cast<size_t>(b) * p.n;
  const int T = p.seq_lens[b], before = T - p.n;
  int parent[2], token[2], target[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int i = lane + 32 * s;
    parent[s] = i < p.n ? p.parents[row + i] : -2;
    token[s] = i < p.n ? p.tokens[row + i] : 0;
    target[s] = i < p.n ? p.sampled[row + i] : 0;
    if (parent[s] >= i) {
      if (at_head == 0) set_status(p.status, SF_DEVICE_BAD_INDEX);
      parent[s] = -2;
    }
  }
  bool live = T != 0;
  if (live && (before < 0 || T > p.max_pages * SF_PAGE_SIZE)) {
    if (at_head == 0 && lane == 0) set_status(p.status, SF_DEVICE_BAD_SEQLEN);
    live = false;
  }
  if (__shfl_sync(0xffffffffu, parent[0], 0) != -1) live = false;  // node 0 is no root
  // path[r] of r = lane and r = lane + 32, its node's target token
  int path[2] = {-1, -1}, out[2] = {-1, -1};
  unsigned long long on = 0ull;
  int rows = 0;
  if (live) {
    int cur = 0;
    while (true) {
      const int want = of_node(target[0], target[1], cur);
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (rows == lane + 32 * s) {
          path[s] = cur;
          out[s] = want;
        }
      on |= 1ull << cur;
      ++rows;
      const unsigned lo = __ballot_sync(0xffffffffu, parent[0] == cur && token[0] == want);
      const unsigned hi = __ballot_sync(0xffffffffu, parent[1] == cur && token[1] == want);
      if (!(lo | hi)) break;
      cur = lo ? __ffs(lo) - 1 : 31 + __ffs(hi);
    }
  }
  if (at_head == 0) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int i = lane + 32 * s;
      if (i >= p.n) continue;
      if (p.out_tokens) p.out_tokens[row + i] = out[s];
      if (p.path) p.path[row + i] = path[s];
      if (p.row_weights) p.row_weights[row + i] = static_cast<float>((on >> i) & 1ull);
    }
    if (lane == 0) p.num_accepted[b] = rows > 0 ? rows - 1 : 0;
  }
  // rows that are in place already: path[r] == r for all up to the first that is not
  const int first = ~on ? __ffsll(~on) - 1 : 64;
  if (c >= 2 * p.layers || first >= rows) return;
  uint4 *cache = p.caches[c];
  const int wide = p.D / 8;  // 16-byte pieces of a row
  const int total = (rows - first) * wide;
  const int32_t *table = p.block_table + static_cast<size_t>(b) * p.max_pages;
  auto place = [&](int pos) -> long long {  // in 16-byte pieces; -1: a page outside the pool
    const int page = table[pos / SF_PAGE_SIZE];
    if (page < 0 || page >= p.num_pages) {
      set_status(p.status, SF_DEVICE_BAD_PAGE);
      return -1;
    }
    return ((static_cast<long long>(page) * p.H_kv + h) * SF_PAGE_SIZE + pos % SF_PAGE_SIZE) * wide;
  };
  for (int base = 0; base < total; base += 32 * kTreeBatch) {
    uint4 v[kTreeBatch];
    long long to[kTreeBatch];
#pragma unroll
    for (int u = 0; u < kTreeBatch; ++u) {
      const int x = base + 32 * u + lane, r = first + x / wide, piece = x % wide;
      const int node = of_node(path[0], path[1], r & 63);
      to[u] = -1;
      if (x < total) {
        const long long from = place(before + node);
        to[u] = place(before + r);
        if (from < 0) to[u] = -1;
        if (to[u] >= 0) {
          to[u] += piece;
          v[u] = cache[from + piece];
        }
      }
    }
    __syncwarp();
#pragma unroll
    for (int u = 0; u < kTreeBatch; ++u)
      if (to[u] >= 0) cache[to[u]] = v[u];
    __syncwarp();
  }
}

__global__ void __launch_bounds__(32 * kTreeWarps)
tree_commit_kernel(const __grid_constant__ TreeCommitParams p) {
  const int lane = threadIdx.x & 31;
  const int item = blockIdx.x * kTreeWarps + uniform_warp_id();  // KV head of a cache of a layer of a sequence
  const int heads = 2 * p.layers * p.H_kv, per = heads > 0 ? heads : 1;
  const int b = item / per, at_head = item - b * per, c = at_head / p.H_kv, h = at_head - c * p.H_kv;
  grid_dependency_wait();
  if (b < p.B) commit_rows(p, b, at_head, c, h, lane);
  launch_dependents_after_stores();
}

static int check_tree(int B, int n) {
  if (B < 1 || B > SF_MAX_BATCH) return fail(SF_ERR_INVALID_ARG, "B=%d outside [1, %d]", B, SF_MAX_BATCH);
  if (n < 1 || n > SF_MAX_TREE_ROWS) return fail(SF_ERR_INVALID_ARG, "n=%d nodes outside [1, %d]", n, SF_MAX_TREE_ROWS);
  return SF_OK;
}

static int check_workspace(const void *workspace, size_t bytes, size_t need) {
  if (!workspace || !aligned(workspace, 256))
    return fail(SF_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
  if (bytes < need) return fail(SF_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", bytes, need);
  return SF_OK;
}

}  // namespace sf

extern "C" {

size_t sf_tree_mask_workspace_size(void) { return 256; }

int sf_tree_mask(const int32_t *parents, const int32_t *start, int B, int n, uint64_t *mask, int32_t *positions,
                 void *workspace, size_t workspace_bytes, cudaStream_t stream) {
  using namespace sf;
  clear_error();
  int st = check_tree(B, n);
  if (st != SF_OK) return st;
  if (!parents || !mask) return fail(SF_ERR_INVALID_ARG, "a required pointer is NULL");
  if (!aligned(parents, 4) || !aligned(start, 4) || !aligned(positions, 4) || !aligned(mask, 8))
    return fail(SF_ERR_INVALID_ARG, "mask must be 8-byte aligned, int32 arrays 4-byte aligned");
  if ((st = check_workspace(workspace, workspace_bytes, sf_tree_mask_workspace_size())) != SF_OK) return st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((B + kTreeWarps - 1) / kTreeWarps);
  cfg.blockDim = dim3(32 * kTreeWarps);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, tree_mask_kernel, parents, start, B, n,
                                           reinterpret_cast<unsigned long long *>(mask), positions,
                                           static_cast<uint32_t *>(workspace));
  if (e != cudaSuccess) return fail(SF_ERR_CUDA, "tree mask launch: %s", cudaGetErrorString(e));
  return SF_OK;
}

size_t sf_tree_commit_workspace_size(void) { return 256; }

int sf_tree_commit(const int32_t *tokens, const int32_t *sampled, const int32_t *parents, void *const *k_caches,
                   void *const *v_caches, int num_layers, int32_t *block_table, int32_t *seq_lens, int B, int n_q,
                   int H_kv, int head_dim, int page_size, int num_pages, int max_pages_per_seq, int32_t *num_accepted,
                   int32_t *out_tokens, int32_t *path, float *row_weights, int n_q_next, int32_t *free_pages,
                   int32_t *free_count, int capacity, void *workspace, size_t workspace_bytes, cudaStream_t stream) {
  using namespace sf;
  clear_error();
  int st = check_tree(B, n_q);
  if (st != SF_OK) return st;
  if (num_layers < 0 || num_layers > SF_MAX_LAYERS)
    return fail(SF_ERR_INVALID_ARG, "num_layers=%d outside [0, %d]", num_layers, SF_MAX_LAYERS);
  if (H_kv < 1 || H_kv > 1024) return fail(SF_ERR_INVALID_ARG, "H_kv=%d outside [1, 1024]", H_kv);
  if (head_dim < 8 || head_dim > 256 || head_dim % 8 != 0)
    return fail(SF_ERR_UNSUPPORTED, "head_dim=%d (a multiple of 8 in [8, 256])", head_dim);
  if (page_size != SF_PAGE_SIZE) return fail(SF_ERR_UNSUPPORTED, "page_size=%d (built: 16)", page_size);
  if (num_pages < 1) return fail(SF_ERR_INVALID_ARG, "num_pages=%d", num_pages);
  if (max_pages_per_seq < 1 || (long long)max_pages_per_seq * page_size > (1LL << 30))
    return fail(SF_ERR_INVALID_ARG, "max_pages_per_seq=%d", max_pages_per_seq);
  if (!tokens || !sampled || !parents || !block_table || !seq_lens || !num_accepted ||
      (num_layers > 0 && (!k_caches || !v_caches)))
    return fail(SF_ERR_INVALID_ARG, "a required pointer is NULL");
  if (!aligned(tokens, 4) || !aligned(sampled, 4) || !aligned(parents, 4) || !aligned(block_table, 4) ||
      !aligned(seq_lens, 4) || !aligned(num_accepted, 4) || !aligned(out_tokens, 4) || !aligned(path, 4) ||
      !aligned(row_weights, 4) || !aligned(free_pages, 4) || !aligned(free_count, 4))
    return fail(SF_ERR_INVALID_ARG, "arrays of tokens, lengths and pages must be 4-byte aligned");
  if ((free_pages == nullptr) != (free_count == nullptr))
    return fail(SF_ERR_INVALID_ARG, "free_pages and free_count belong together");
  if (free_pages && (n_q_next < 1 || n_q_next > SF_MAX_TREE_ROWS || capacity < 0))
    return fail(SF_ERR_INVALID_ARG, "n_q_next=%d outside [1, %d] or capacity=%d", n_q_next, SF_MAX_TREE_ROWS, capacity);
  if ((st = check_workspace(workspace, workspace_bytes, sf_tree_commit_workspace_size())) != SF_OK) return st;
  TreeCommitParams p;
  for (int l = 0; l < num_layers; ++l) {
    if (!k_caches[l] || !v_caches[l] || !aligned(k_caches[l], 16) || !aligned(v_caches[l], 16))
      return fail(SF_ERR_INVALID_ARG, "the caches of layer %d must be non-NULL and 16-byte aligned", l);
    p.caches[2 * l] = static_cast<uint4 *>(k_caches[l]);
    p.caches[2 * l + 1] = static_cast<uint4 *>(v_caches[l]);
  }
  const long long items = (long long)B * (num_layers > 0 ? 2LL * num_layers * H_kv : 1LL);
  p.tokens = tokens;
  p.sampled = sampled;
  p.parents = parents;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.num_accepted = num_accepted;
  p.out_tokens = out_tokens;
  p.path = path;
  p.row_weights = row_weights;
  p.status = static_cast<uint32_t *>(workspace);
  p.B = B;
  p.n = n_q;
  p.H_kv = H_kv;
  p.D = head_dim;
  p.num_pages = num_pages;
  p.max_pages = max_pages_per_seq;
  p.layers = num_layers;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((items + kTreeWarps - 1) / kTreeWarps));
  cfg.blockDim = dim3(32 * kTreeWarps);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, tree_commit_kernel, p);
  if (e != cudaSuccess) return fail(SF_ERR_CUDA, "tree commit launch: %s", cudaGetErrorString(e));
  if (!free_pages) return SF_OK;
  return launch_kv_commit(seq_lens, block_table, free_pages, free_count, num_accepted, B, n_q, n_q_next,
                          max_pages_per_seq, capacity, parents, p.status, stream);
}

}  // extern "C"
