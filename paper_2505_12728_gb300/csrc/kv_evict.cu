// kv_evict.cu -- a paged cache back to its budget: of each sequence that is longer,
// each layer and KV head keeps the `budget` keys of most accumulated attention
// weight (the first and the last ones in any case), in their order, and its rows of
// K, V and weights are compacted in place.
//
// One cluster of CTAs per (layer, sequence, KV head); nothing is shared between
// them but the pages, of which each has rows of its own.
//
// Which keys.  The weights' bits, ordered as unsigned integers (positive values above
// negative ones, NaN as -infinity, the keys that stay in any case above all), in
// three rounds of 11, 11 and 10 bits from the top: a histogram of the keys that agree
// with the digits found so far, the bin in which the budget's last key lies, the
// same again inside that bin.  That gives the last kept key's value exactly, and how
// many of its equals are kept (the lowest positions).  A second pass in order of the
// positions counts the larger and the equal keys in front of each, which is the place
// that a kept key moves to.
//
// In place.  Row j of the result comes from position kept[j] >= j, and the positions
// ascend.  So rows are moved in rounds of ascending j, each round's loads (into
// registers) in front of a barrier and its stores behind it: a store overwrites rows
// at or below its own j only, which later rounds do not read.
//
// The last cluster to finish writes the lengths and, if asked to, gives the pages
// that are no longer needed back to the free-page stack.
#include "sf_device.cuh"
#include "sf_host.h"

namespace sf {

constexpr int kEvictThreads = 512;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kEvictBins = 2048;
constexpr int kEvictBatch = 8;         // 16-byte loads of a thread in flight
constexpr int kEvictMaxCluster = 8;

struct EvictLayer {
  const float *mass;
  float *mass_out;
  uint4 *k, *v;
  int32_t *kept;
};

struct EvictParams {
  const int32_t *seq_lens;
  int32_t *block_table, *seq_lens_out, *free_pages, *free_count;
  uint32_t *status, *ticket;
  int B, H_kv, D, num_pages, max_pages, width, budget, first, recent, n_q, capacity;
  EvictLayer layers[SF_MAX_LAYERS];
};

// What is left of sequence b: the tokens of its context, and whether it is cut.
__device__ __forceinline__ int evict_length(const EvictParams &p, int b, bool &cut, bool flag) {
  const int T = p.seq_lens[b], n = T - p.n_q;
  cut = false;
  if (T == 0) return 0;
  if (n < 0 || T > p.max_pages * SF_PAGE_SIZE || n > p.width) {
    if (flag) set_status(p.status, SF_DEVICE_BAD_SEQLEN);
    return n < 0 ? 0 : n > p.width ? p.width : n;
  }
  cut = n > p.budget;
  return n;
}

// Larger weights have larger keys; -0 counts as 0, NaN as -infinity.
__device__ __forceinline__ uint32_t evict_key(float w) {
  const uint32_t u = __float_as_uint(w == w ? w + 0.f : -INFINITY);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ uint32_t ld_dsmem_u32(uint32_t local, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(dsmem_addr(local, rank)) : "memory");
  return v;
}

// Exclusive sum over the block's threads; *total is all of them.
__device__ __forceinline__ uint32_t evict_scan(uint32_t v, uint32_t *s_warp, uint32_t *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  uint32_t off = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kEvictWarps; ++w) {
    const uint32_t x = s_warp[w];
    if (w < warp) off += x;
    sum += x;
  }
  __syncthreads();
  *total = sum;
  return off + incl - v;
}

template <int C>
__global__ void __launch_bounds__(kEvictThreads) kv_evict_kernel(const __grid_constant__ EvictParams p) {
  __shared__ uint32_t s_hist[3][kEvictBins];
  __shared__ uint32_t s_warp[kEvictWarps], s_pick[2], s_count[2];
  __shared__ uint32_t s_last;
  const int tid = threadIdx.x, lane = tid & 31;
  const int rank = C > 1 ? static_cast<int>(blockIdx.x % C) : 0, task = blockIdx.x / C;
  const int h = task % p.H_kv, lb = task / p.H_kv, b = lb % p.B;
  const EvictLayer &layer = p.layers[lb / p.B];
  const size_t bh = static_cast<size_t>(b) * p.H_kv + h;
  auto sync_all = [&]() {
    if constexpr (C > 1) cluster_sync();
    else __syncthreads();
  };
  for (int i = tid; i < 3 * kEvictBins; i += kEvictThreads) s_hist[0][i] = 0u;
  grid_dependency_wait();
  bool cut;
  const int L = evict_length(p, b, cut, task / p.H_kv < p.B && h == 0 && rank == 0 && tid == 0);
  const float *mass = layer.mass + bh * p.width;
  float *mass_out = layer.mass_out + bh * p.width;
  int32_t *kept = layer.kept + bh * p.budget;
  __syncthreads();
  if (!cut) {
    // nothing moves
    const int all = C * kEvictThreads, me = rank * kEvictThreads + tid;
    for (int t = me; t < p.width; t += all)
      if (t >= L) mass_out[t] = 0.f;
      else if (mass != mass_out) mass_out[t] = mass[t];
    for (int j = me; j < p.budget; j += all) kept[j] = j < L ? j : -1;
  } else {
    const int per = (L + C - 1) / C, from = min(rank * per, L), to = min(from + per, L);
    const int late = L - p.recent;
    auto key_at = [&](int t) -> uint32_t {
      return t < p.first || t >= late ? 0xffffffffu : evict_key(mass[t]);
    };
    uint32_t found = 0u, left = static_cast<uint32_t>(p.budget);
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
      const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, width = round == 2 ? 10 : 11;
      uint32_t *hist = s_hist[round];
      for (int t0 = from; t0 < to; t0 += kEvictThreads) {
        const int t = t0 + tid;
        const uint32_t key = t < to ? key_at(t) : 0u;
        const bool in = t < to && (round == 0 || (key >> (shift + width)) == (found >> (shift + width)));
        const uint32_t bin = in ? (key >> shift) & ((1u << width) - 1u) : kEvictBins;
        // one add for the lanes that agree with the first: weights cluster, and equal
        // addresses are served one after the other
        const unsigned any = __ballot_sync(0xffffffffu, in);
        if (!any) continue;
        const int lead = __ffs(any) - 1;
        const uint32_t common = __shfl_sync(0xffffffffu, bin, lead);
        const unsigned same = __ballot_sync(0xffffffffu, bin == common);
        if (lane == lead) atomicAdd(&hist[common], static_cast<uint32_t>(__popc(same)));
        else if (in && bin != common) atomicAdd(&hist[bin], 1u);
      }
      sync_all();
      // the bin that holds the left-th key from the top
      constexpr int kPer = kEvictBins / kEvictThreads;
      uint32_t n[kPer], sum = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int bin = kEvictBins - 1 - (tid * kPer + i);
        n[i] = 0;
        if constexpr (C > 1) {
#pragma unroll
          for (int r = 0; r < C; ++r) n[i] += ld_dsmem_u32(smem_addr(&hist[bin]), r);
        } else {
          n[i] = hist[bin];
        }
        sum += n[i];
      }
      uint32_t total, above = evict_scan(sum, s_warp, &total);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (above < left && left <= above + n[i]) {
          s_pick[0] = kEvictBins - 1 - (tid * kPer + i);
          s_pick[1] = left - above;
        }
        above += n[i];
      }
      __syncthreads();
      found |= s_pick[0] << shift;
      left = s_pick[1];
      __syncthreads();
    }
    // keys above `found` are kept, and the first `left` of those equal to it
    uint32_t larger = 0, equal = 0;
    if constexpr (C > 1) {
      uint32_t mine = 0;
      for (int t = from + tid; t < to; t += kEvictThreads) {
        const uint32_t key = key_at(t);
        mine += key > found ? 1u : 0u;
        equal += key == found ? 1u : 0u;
      }
      uint32_t sum_l, sum_e;
      (void)evict_scan(mine, s_warp, &sum_l);
      (void)evict_scan(equal, s_warp, &sum_e);
      if (tid == 0) {
        s_count[0] = sum_l;
        s_count[1] = sum_e;
      }
      cluster_sync();
      larger = equal = 0;
      for (int r = 0; r < rank; ++r) {
        larger += ld_dsmem_u32(smem_addr(&s_count[0]), r);
        equal += ld_dsmem_u32(smem_addr(&s_count[1]), r);
      }
    }
    for (int t0 = from; t0 < to; t0 += kEvictThreads) {
      const int t = t0 + tid;
      const uint32_t key = t < to ? key_at(t) : 0u;
      const bool gt = t < to && key > found, eq = t < to && key == found;
      uint32_t total;
      const uint32_t before = evict_scan((gt ? 1u : 0u) | (eq ? 0x10000u : 0u), s_warp, &total);
      const uint32_t l = larger + (before & 0xffffu), e = equal + (before >> 16);
      if (gt || (eq && e < left)) kept[l + min(e, left)] = t;
      larger += total & 0xffffu;
      equal += total >> 16;
    }
    sync_all();
    // rows in rounds of ascending places
    const int wide = p.D / 8, kv_wide = 2 * wide;  // 16-byte pieces of a row of K, and of K and V
    const int rows = min(kEvictThreads * kEvictBatch / kv_wide, kEvictThreads);  // of a CTA and round
    const int32_t *table = p.block_table + static_cast<size_t>(b) * p.max_pages;
    auto place = [&](int pos) -> long long {
      const int page = table[pos / SF_PAGE_SIZE];
      if (page < 0 || page >= p.num_pages) {
        set_status(p.status, SF_DEVICE_BAD_PAGE);
        return -1;
      }
      return ((static_cast<long long>(page) * p.H_kv + h) * SF_PAGE_SIZE + pos % SF_PAGE_SIZE) * wide;
    };
    for (int j0 = 0; j0 < p.budget; j0 += C * rows) {
      const int base = j0 + rank * rows;
      uint4 v[kEvictBatch];
      uint4 *dst[kEvictBatch];
      float w = 0.f;
      if (tid < rows && base + tid < p.budget) w = mass[kept[base + tid]];
#pragma unroll
      for (int u = 0; u < kEvictBatch; ++u) {
        const int x = u * kEvictThreads + tid, r = x / kv_wide, piece = x - r * kv_wide, j = base + r;
        dst[u] = nullptr;
        if (r < rows && j < p.budget) {
          const int pos = kept[j];
          if (pos != j) {
            const long long src = place(pos), at = place(j);
            uint4 *cache = piece < wide ? layer.k : layer.v;
            const int c = piece < wide ? piece : piece - wide;
            if (src >= 0 && at >= 0) {
              v[u] = cache[src + c];
              dst[u] = cache + at + c;
            }
          }
        }
      }
      sync_all();
#pragma unroll
      for (int u = 0; u < kEvictBatch; ++u)
        if (dst[u]) *dst[u] = v[u];
      if (tid < rows && base + tid < p.budget) mass_out[base + tid] = w;
    }
    sync_all();
    for (int t = p.budget + rank * kEvictThreads + tid; t < p.width; t += C * kEvictThreads) mass_out[t] = 0.f;
  }

  // the last CTA: lengths and pages
  __syncthreads();
  if (tid == 0) s_last = atom_add_acq_rel_gpu(p.ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  if (s_last) {
    if (tid == 0) *p.ticket = 0u;
    uint32_t freed = p.free_count ? static_cast<uint32_t>(*p.free_count) : 0u;
    const int fc0 = static_cast<int>(freed);
    bool full = fc0 < 0;
    for (int b1 = 0; b1 < p.B; ++b1) {
      bool c1;
      (void)evict_length(p, b1, c1, false);
      const int T = p.seq_lens[b1], now = c1 ? p.budget + p.n_q : T;
      __syncthreads();  // (seq_lens_out may be seq_lens)
      if (tid == 0) p.seq_lens_out[b1] = now;
      if (!p.free_count || !c1) continue;
      const int need = (now + SF_PAGE_SIZE - 1) / SF_PAGE_SIZE, had = (T + SF_PAGE_SIZE - 1) / SF_PAGE_SIZE;
      int32_t *table = p.block_table + static_cast<size_t>(b1) * p.max_pages;
      // a stack without room: the pages stay mapped
      if (full || static_cast<long long>(freed) + (had - need) > p.capacity) {
        full = true;
        continue;
      }
      for (int i = tid; i < had - need; i += kEvictThreads) {
        p.free_pages[freed + i] = table[need + i];
        table[need + i] = -1;
      }
      freed += had - need;
    }
    if (tid == 0 && p.free_count) {
      if (!(fc0 < 0)) *p.free_count = static_cast<int32_t>(freed);
      if (full) set_status(p.status, SF_DEVICE_OUT_OF_PAGES);
    }
  }
  launch_dependents_after_stores();
}

// `kept` of all layers for a call that does not ask for it lies behind the header.
static size_t evict_bytes(int layers, int B, int H_kv, int budget) {
  return 256 + round_up(static_cast<size_t>(layers) * B * H_kv * budget * sizeof(int32_t), 256);
}

static int check_evict(int layers, int B, int H_kv, int budget) {
  if (layers < 1 || layers > SF_MAX_LAYERS)
    return fail(SF_ERR_INVALID_ARG, "num_layers=%d outside [1, %d]", layers, SF_MAX_LAYERS);
  if (B < 1 || B > SF_MAX_BATCH) return fail(SF_ERR_INVALID_ARG, "B=%d outside [1, %d]", B, SF_MAX_BATCH);
  if (H_kv < 1 || H_kv > 1024) return fail(SF_ERR_INVALID_ARG, "H_kv=%d outside [1, 1024]", H_kv);
  if (budget < 1 || budget > (1 << 30)) return fail(SF_ERR_INVALID_ARG, "budget=%d", budget);
  return SF_OK;
}

static int evict_cluster(int tasks, int sms) {
  int C = 1;
  while (C < kEvictMaxCluster && static_cast<long long>(tasks) * C < 2LL * sms) C *= 2;
  return C;
}

}  // namespace sf

extern "C" {

size_t sf_kv_evict_workspace_size(int num_layers, int B, int H_kv, int budget) {
  return sf::check_evict(num_layers, B, H_kv, budget) == SF_OK ? sf::evict_bytes(num_layers, B, H_kv, budget) : 0;
}

int sf_kv_evict(const float *const *mass, void *const *k_caches, void *const *v_caches, int num_layers,
                int32_t *block_table, const int32_t *seq_lens, int B, int H_kv, int head_dim, int page_size,
                int num_pages, int max_pages_per_seq, int mass_width, int budget, int first, int recent, int n_q,
                float *const *mass_out, int32_t *seq_lens_out, int32_t *const *kept, int32_t *free_pages,
                int32_t *free_count, int capacity, void *workspace, size_t workspace_bytes, cudaStream_t stream) {
  using namespace sf;
  clear_error();
  int st = check_evict(num_layers, B, H_kv, budget);
  if (st != SF_OK) return st;
  if (head_dim < 8 || head_dim > 256 || head_dim % 8 != 0)
    return fail(SF_ERR_UNSUPPORTED, "head_dim=%d (a multiple of 8 in [8, 256])", head_dim);
  if (page_size != SF_PAGE_SIZE) return fail(SF_ERR_UNSUPPORTED, "page_size=%d (built: 16)", page_size);
  if (num_pages < 1) return fail(SF_ERR_INVALID_ARG, "num_pages=%d", num_pages);
  if (max_pages_per_seq < 1 || (long long)max_pages_per_seq * page_size > (1LL << 30))
    return fail(SF_ERR_INVALID_ARG, "max_pages_per_seq=%d", max_pages_per_seq);
  if (mass_width < 1 || mass_width > (1 << 30)) return fail(SF_ERR_INVALID_ARG, "mass_width=%d", mass_width);
  if (first < 0 || recent < 0 || (long long)first + recent > budget)
    return fail(SF_ERR_INVALID_ARG, "first=%d and recent=%d must be >= 0 and fit the budget=%d", first, recent, budget);
  if (n_q < 0 || n_q > SF_MAX_TREE_ROWS)
    return fail(SF_ERR_INVALID_ARG, "n_q=%d outside [0, %d]", n_q, SF_MAX_TREE_ROWS);
  if (!mass || !k_caches || !v_caches || !block_table || !seq_lens || !mass_out || !seq_lens_out)
    return fail(SF_ERR_INVALID_ARG, "a required pointer is NULL");
  if (!aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(seq_lens_out, 4) || !aligned(free_pages, 4) ||
      !aligned(free_count, 4))
    return fail(SF_ERR_INVALID_ARG, "int32 arrays must be 4-byte aligned");
  if ((free_pages == nullptr) != (free_count == nullptr) || capacity < 0)
    return fail(SF_ERR_INVALID_ARG, "free_pages and free_count belong together, capacity=%d", capacity);
  if ((long long)num_layers * B * H_kv * kEvictMaxCluster >= (1LL << 31))
    return fail(SF_ERR_UNSUPPORTED, "%d layers of %d sequences with %d heads", num_layers, B, H_kv);
  if (!workspace || !aligned(workspace, 256))
    return fail(SF_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
  if (workspace_bytes < evict_bytes(num_layers, B, H_kv, budget))
    return fail(SF_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes,
                evict_bytes(num_layers, B, H_kv, budget));
  EvictParams p;
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  for (int l = 0; l < num_layers; ++l) {
    EvictLayer &x = p.layers[l];
    x.mass = mass[l];
    x.mass_out = mass_out[l];
    x.k = static_cast<uint4 *>(k_caches[l]);
    x.v = static_cast<uint4 *>(v_caches[l]);
    x.kept = kept ? kept[l] : reinterpret_cast<int32_t *>(ws + 256) + static_cast<size_t>(l) * B * H_kv * budget;
    if (!x.mass || !x.mass_out || !x.k || !x.v || !x.kept)
      return fail(SF_ERR_INVALID_ARG, "a required pointer of layer %d is NULL", l);
    if (!aligned(x.mass, 4) || !aligned(x.mass_out, 4) || !aligned(x.k, 16) || !aligned(x.v, 16) || !aligned(x.kept, 4))
      return fail(SF_ERR_INVALID_ARG, "the caches of layer %d must be 16-byte aligned, its other arrays 4-byte", l);
  }
  DeviceInfo dev;
  if ((st = current_device(&dev)) != SF_OK) return st;
  p.seq_lens = seq_lens;
  p.block_table = block_table;
  p.seq_lens_out = seq_lens_out;
  p.free_pages = free_pages;
  p.free_count = free_count;
  p.status = reinterpret_cast<uint32_t *>(ws);
  p.ticket = reinterpret_cast<uint32_t *>(ws + 128);
  p.B = B;
  p.H_kv = H_kv;
  p.D = head_dim;
  p.num_pages = num_pages;
  p.max_pages = max_pages_per_seq;
  p.width = mass_width;
  p.budget = budget;
  p.first = first;
  p.recent = recent;
  p.n_q = n_q;
  p.capacity = capacity;
  const int tasks = num_layers * B * H_kv, C = evict_cluster(tasks, dev.sm_count);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = C;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(tasks * C));
  cfg.blockDim = dim3(kEvictThreads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = C > 1 ? 2 : 1;
  auto kernel = C == 1 ? kv_evict_kernel<1> : C == 2 ? kv_evict_kernel<2> : C == 4 ? kv_evict_kernel<4> : kv_evict_kernel<8>;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
  if (e != cudaSuccess) return fail(SF_ERR_CUDA, "eviction launch: %s", cudaGetErrorString(e));
  return SF_OK;
}

}  // extern "C"
