// kv_evict.cu -- a paged cache back to its budget: of each sequence that is longer,
// each layer and KV head keeps the `budget` keys of most accumulated attention
// weight (the first and the last ones in any case), in their order, and its rows of
// K, V and weights are compacted in place.
//
// One CTA, or a cluster, per (layer, sequence, KV head); nothing is shared between
// them but the pages, of which each has rows of its own.  Where the weights' width or the
// table, whichever is less, has room for at most 256 or 512 tokens, contexts have a kernel of
// their own, kv_evict_short_kernel; the rest of this is about kv_evict_kernel.
//
// Which keys.  The first and the last ones stay in any case; of those between, the
// weights' bits, ordered as unsigned integers (positive values above negative ones, NaN
// as -infinity), in three rounds of 11, 11 and 10 bits from the top: a histogram of the keys that agree
// with the digits found so far, the bin in which the budget's last key lies, the
// same again inside that bin.  That gives the last kept key's value exactly, and how
// many of its equals are kept (the lowest positions).  A second pass in order of the
// positions counts the larger and the equal keys in front of each, which is the place
// that a kept key moves to.
//
// In place.  Row j of the result comes from position kept[j] >= j, and the positions
// ascend.  So rows are moved in rounds of ascending j, each round's copies into shared
// memory in front of a barrier and those out of it behind it: they overwrite rows at
// or below their own j only, which later rounds do not read.
//
// What bounds it: the rows' way out and in, 256 bytes at a time from all over the cache.  32
// layers of 32 heads, 3008 -> 1024 keys: 195 us, 5.6 TB/s, 82 % of the copy rate (with 16-byte
// loads and a barrier a round 350); 28 layers of 4 sequences and 4 heads, 8192 to 32768 ->
// 4096 keys: 340 us, 83 % (770).  Three CTAs a SM with two rounds of 32 KB each in flight, or
// four with 24 KB (evict_launch), so that one's choice of keys runs beside another's rows (five
// with 16 KB: 219 and 436).  The choice reads the weights three times, the second and third
// time from L2: the first digit's histogram, the few keys of its bin to shared memory, where
// the other digits are found, and the places.  It is bound by its instructions: 448 heads of
// 30000 keys to 1000 took 148 us with a test of every key for its place and two compares
// for ties in all cases, 132 without, 129 with plain adds to the histogram.
//
// The last CTA to finish writes the lengths and, if asked to, gives the pages that are no
// longer needed back to the free-page stack: a thread a sequence, then a thread a page (one
// sequence after the other took 37.6 us for 256 sequences of which none is cut, 10.2 so;
// 256 sequences of 4 pages back 123 -> 38).
#include <algorithm>
#include <mutex>

#include "layer_device.cuh"
#include "sf_host.h"

namespace sf {

constexpr int kEvictThreads = 256;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kEvictBins = 2048;
constexpr int kEvictKeys = 8;          // keys of a thread in flight
constexpr int kEvictMaxCluster = 8;
constexpr size_t kEvictHeader = 256;   // status, ticket, word of the CTAs that gave up
constexpr int kShortBatch = 4;         // 16-byte loads of a thread in flight
// With `blocks` CTAs per SM: bytes of a warp's rows of a round, and of shared memory.
constexpr int evict_slot(int blocks) { return 12 * 1024 / blocks; }
constexpr int evict_smem(int blocks) {
  return 2 * kEvictWarps * evict_slot(blocks) > 5 * kEvictBins * 4 ? 2 * kEvictWarps * evict_slot(blocks) : 5 * kEvictBins * 4;
}

struct EvictLayer {
  const float *mass;
  float *mass_out;
  uint4 *k, *v;
  int32_t *kept;
};

struct EvictParams {
  const int32_t *seq_lens;
  int32_t *block_table, *seq_lens_out, *free_pages, *free_count;
  uint32_t *status, *ticket, *gave_up;
  int B, H_kv, D, num_pages, max_pages, width, budget, first, recent, n_q, capacity;
  EvictLayer layers[SF_MAX_LAYERS];
};

// What is left of sequence b: the tokens of its context, whether it is cut, and whether its
// length cannot be (then nothing of it changes).
__device__ __forceinline__ int evict_length(const EvictParams &p, int b, bool &cut, bool &bad) {
  const int T = p.seq_lens[b], n = T < p.n_q ? 0 : T - p.n_q;
  bad = T != 0 && (T < p.n_q || T > p.max_pages * SF_PAGE_SIZE || n > p.width);
  cut = !bad && n > p.budget;
  return min(n, p.width);
}

// A head of which nothing moves, by `all` threads: what lies behind the context has no weight
// (that of a bad length says nothing about where that is).
__device__ __forceinline__ void evict_nothing(const EvictParams &p, const float *mass, float *mass_out, int32_t *kept, int L,
                                              bool bad, int me, int all) {
  for (int t = me; t < p.width; t += all)
    if (t >= L && !bad) mass_out[t] = 0.f;
    else if (mass != mass_out) mass_out[t] = mass[t];
  for (int j = me; j < p.budget; j += all) kept[j] = j < L ? j : -1;
}

// Larger weights have larger keys; -0 counts as 0, NaN as -infinity.
__device__ __forceinline__ uint32_t evict_key(float w) {
  const int u = __float_as_int(fmaxf(w, -INFINITY) + 0.f);
  return static_cast<uint32_t>(u ^ (u >> 31 | static_cast<int>(0x80000000u)));
}

// Bulk copies of rows back to global memory, in groups of the issuing thread.
__device__ __forceinline__ void bulk_copy_s2g(void *dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(reinterpret_cast<uint64_t>(dst)), "r"(src),
               "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ uint32_t ld_dsmem_u32(uint32_t local, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(dsmem_addr(local, rank)) : "memory");
  return v;
}

// Exclusive sum over the block's threads; *total is all of them.
template <int WARPS, typename T>
__device__ __forceinline__ T evict_scan(T v, T *s_warp, T *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  T off = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    const T x = s_warp[w];
    if (w < warp) off += x;
    sum += x;
  }
  __syncthreads();
  *total = sum;
  return off + incl - v;
}

// The last CTA to come here writes the lengths and gives the pages back.  If one gave up
// on a row they stay as they were: what is in the cache is nobody's context.
template <int THREADS>
__device__ __forceinline__ void evict_finish(const EvictParams &p) {
  __shared__ uint32_t s_last, s_stop;
  __shared__ long long s_wide[THREADS / 32];
  __shared__ uint32_t s_plan[2 * THREADS];
  const int tid = threadIdx.x;
  __syncthreads();
  if (tid == 0) {
    s_last = atom_add_acq_rel_gpu(p.ticket, 1u) == gridDim.x - 1;
    s_stop = s_last ? *p.gave_up : 0u;
  }
  __syncthreads();
  if (s_last) {
    if (tid == 0) {
      *p.ticket = 0u;
      if (s_stop) *p.gave_up = 0u;
    }
    if (s_stop) {
      for (int b = tid; b < p.B; b += THREADS) p.seq_lens_out[b] = p.seq_lens[b];
      return;
    }
    // A thread a sequence; then the pages of all of them, found by their places on the stack.
    const int fc0 = p.free_count ? *p.free_count : 0;
    long long freed = fc0;
    bool full = fc0 < 0;
    uint32_t *s_off = s_plan, *s_need = s_plan + THREADS;
    for (int b0 = 0; b0 < p.B; b0 += THREADS) {
      const int b1 = b0 + tid;
      bool c1 = false, bad;
      int need = 0;
      long long gone = 0, total;
      if (b1 < p.B) {
        const int T = p.seq_lens[b1];
        (void)evict_length(p, b1, c1, bad);
        const int now = c1 ? p.budget + p.n_q : T;
        p.seq_lens_out[b1] = now;  // (may be seq_lens)
        need = (now + SF_PAGE_SIZE - 1) / SF_PAGE_SIZE;
        if (c1) gone = (T + SF_PAGE_SIZE - 1) / SF_PAGE_SIZE - need;
      }
      if (!p.free_count) continue;
      const long long off = evict_scan<THREADS / 32>(gone, s_wide, &total);
      // sequences that the stack has no room for: their pages stay mapped
      const bool stays = c1 && (full || freed + off + gone > p.capacity);
      s_off[tid] = static_cast<uint32_t>(off > p.capacity ? p.capacity : off);
      s_need[tid] = need;
      if (__syncthreads_or(stays)) {
        full = true;
        (void)evict_scan<THREADS / 32>(stays ? 0ll : gone, s_wide, &total);
      }
      for (long long f0 = 0; f0 < total; f0 += kEvictKeys * THREADS) {
        int32_t *from[kEvictKeys], page[kEvictKeys];
#pragma unroll
        for (int u = 0; u < kEvictKeys; ++u) {
          const long long f = f0 + u * THREADS + tid;
          if (f >= total) continue;
          int at = 0;  // the last sequence whose pages start at or before f
#pragma unroll
          for (int step = THREADS / 2; step > 0; step >>= 1)
            if (s_off[at + step] <= f) at += step;
          from[u] = p.block_table + static_cast<size_t>(b0 + at) * p.max_pages + s_need[at] + (f - s_off[at]);
          page[u] = *from[u];
        }
#pragma unroll
        for (int u = 0; u < kEvictKeys; ++u) {
          const long long f = f0 + u * THREADS + tid;
          if (f >= total) continue;
          p.free_pages[freed + f] = page[u];
          *from[u] = -1;
        }
      }
      freed += total;
      __syncthreads();
    }
    if (tid == 0 && p.free_count) {
      if (!(fc0 < 0)) *p.free_count = static_cast<int32_t>(freed);
      if (full) set_status(p.status, SF_DEVICE_OUT_OF_PAGES);
    }
  }
}

template <int C, int BLOCKS>
__global__ void __launch_bounds__(kEvictThreads, BLOCKS) kv_evict_kernel(const __grid_constant__ EvictParams p) {
  constexpr int kSlot = evict_slot(BLOCKS);
  extern __shared__ __align__(128) uint8_t smem[];
  // while the keys are chosen; then the slots of the rows on their way, two a warp
  uint32_t(*s_hist)[kEvictBins] = reinterpret_cast<uint32_t(*)[kEvictBins]>(smem);
  uint32_t *s_total = s_hist[3];  // a histogram of all CTAs
  uint32_t *s_few = s_hist[4];    // keys in the first digit's bin
  __shared__ __align__(8) uint64_t s_bar[kEvictWarps][2];
  __shared__ uint32_t s_rows[2][kEvictWarps];
  __shared__ uint32_t s_found, s_warp[kEvictWarps], s_pick[3], s_count[2];
  const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp_id();
  const int rank = C > 1 ? static_cast<int>(blockIdx.x % C) : 0, task = blockIdx.x / C;
  const int h = task % p.H_kv, lb = task / p.H_kv, b = lb % p.B;
  const EvictLayer &layer = p.layers[lb / p.B];
  const size_t bh = static_cast<size_t>(b) * p.H_kv + h;
  auto sync_all = [&]() {
    if constexpr (C > 1) cluster_sync();
    else __syncthreads();
  };
  for (int i = tid; i < 3 * kEvictBins; i += kEvictThreads) s_hist[0][i] = 0u;
  if (tid == 0) {
    s_found = 0u;
    for (int i = 0; i < 2 * kEvictWarps; ++i) mbar_init(smem_addr(&s_bar[0][0]) + 8 * i, 1);
    fence_mbar_init();
  }
  grid_dependency_wait();
  bool cut, bad;
  const int L = evict_length(p, b, cut, bad);
  if (bad && lb < p.B && h == 0 && rank == 0 && tid == 0) set_status(p.status, SF_DEVICE_BAD_SEQLEN);
  const float *mass = layer.mass + bh * p.width;
  float *mass_out = layer.mass_out + bh * p.width;
  int32_t *kept = layer.kept + bh * p.budget;
  __syncthreads();
  if (!cut) {
    evict_nothing(p, mass, mass_out, kept, L, bad, rank * kEvictThreads + tid, C * kEvictThreads);
  } else {
    // the first and the last ones stay; of the `inner` others, `left` do
    const int late = L - p.recent, inner = late - p.first;
    const int per = (inner + C - 1) / C, from = p.first + min(rank * per, inner), to = min(from + per, late);
    for (int i = rank * kEvictThreads + tid; i < p.first + p.recent; i += C * kEvictThreads) {
      if (i < p.first) kept[i] = i;
      else kept[p.budget - p.recent + i - p.first] = late + i - p.first;
    }
    uint32_t found = 0u, left = static_cast<uint32_t>(p.budget - p.first - p.recent);
    uint32_t mine = 0u;  // keys of this thread's bins above `found`, of this CTA
    // (an add a lane; one for all lanes of the first one's bin was slower whatever the weights:
    // 448 heads of 30000 keys 135 us against 131, uniform ones 183, 159, all equal 133, 105)
    auto count_keys = [&](uint32_t *hist, bool in, uint32_t bin) {
      if (in) atomicAdd(&hist[bin], 1u);
    };
    // all keys of this CTA's positions, kEvictKeys of a thread at a time
    constexpr int kStep = kEvictThreads * kEvictKeys;
    auto each_key = [&](auto &&f) {
      float next[kEvictKeys];
      auto load = [&](int t0) {
        const float *at = mass + t0 + tid;
        if (t0 + kStep <= to) {
#pragma unroll
          for (int u = 0; u < kEvictKeys; ++u) next[u] = at[u * kEvictThreads];
        } else {
#pragma unroll
          for (int u = 0; u < kEvictKeys; ++u) next[u] = t0 + u * kEvictThreads + tid < to ? at[u * kEvictThreads] : 0.f;
        }
      };
      load(from);
#pragma unroll 1
      for (int t0 = from; t0 < to; t0 += kStep) {
        float now[kEvictKeys];
#pragma unroll
        for (int u = 0; u < kEvictKeys; ++u) now[u] = next[u];
        load(t0 + kStep);
        if (t0 + kStep <= to) {
#pragma unroll
          for (int u = 0; u < kEvictKeys; ++u) f(true, evict_key(now[u]));
        } else {
#pragma unroll
          for (int u = 0; u < kEvictKeys; ++u) f(t0 + u * kEvictThreads + tid < to, evict_key(now[u]));
        }
      }
    };
    if (left) each_key([&](bool in, uint32_t key) { count_keys(s_hist[0], in, key >> 21); });
#pragma unroll 1
    for (int round = 0; round < 3 && left; ++round) {
      uint32_t *hist = s_hist[round];
      sync_all();
      // the bin that holds the left-th key from the top
      constexpr int kPer = kEvictBins / kEvictThreads;
      if constexpr (C > 1) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          uint32_t n = 0;
#pragma unroll
          for (int r = 0; r < C; ++r) n += ld_dsmem_u32(smem_addr(&hist[i * kEvictThreads + tid]), r);
          s_total[i * kEvictThreads + tid] = n;
        }
        __syncthreads();
      }
      const uint32_t *bins = C > 1 ? s_total : hist;
      const int top = kEvictBins - kPer * (tid + 1);  // the thread's bins top .. top + kPer - 1
      uint32_t n[kPer], sum = 0;
#pragma unroll
      for (int i = 0; i < kPer; i += 4) {
        const uint4 x = *reinterpret_cast<const uint4 *>(bins + top + i);
        n[i] = x.x;
        n[i + 1] = x.y;
        n[i + 2] = x.z;
        n[i + 3] = x.w;
        sum += x.x + x.y + x.z + x.w;
      }
      uint32_t total, above = evict_scan<kEvictWarps>(sum, s_warp, &total);
#pragma unroll
      for (int i = kPer - 1; i >= 0; --i) {
        if (above < left && left <= above + n[i]) {
          s_pick[0] = top + i;
          s_pick[1] = left - above;
          s_pick[2] = n[i];
        }
        above += n[i];
      }
      __syncthreads();
      const uint32_t pick = s_pick[0];
      if constexpr (C > 1) {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (static_cast<uint32_t>(top + i) > pick) mine += hist[top + i];
      }
      found |= pick << (round == 0 ? 21 : round == 1 ? 10 : 0);
      left = s_pick[1];
      if (round == 2) break;
      if (round == 0) {
        // the keys of that bin, which the other digits are taken from
        each_key([&](bool in, uint32_t key) {
          const bool take = in && (key ^ found) < 1u << 21;
          const unsigned who = __ballot_sync(0xffffffffu, take);
          if (!who) return;
          uint32_t at = 0;
          if (lane == 0) at = atomicAdd(&s_found, static_cast<uint32_t>(__popc(who)));
          at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1u));
          if (take && at < kEvictBins) s_few[at] = key;
        });
      }
      __syncthreads();
      const int few = s_found;
      if (few <= kEvictBins) {
        for (int i = tid; i < (few + 31) / 32 * 32; i += kEvictThreads) {
          const uint32_t key = i < few ? s_few[i] : 0u;
          if (round == 0) count_keys(s_hist[1], i < few, (key >> 10) & 2047u);
          else count_keys(s_hist[2], i < few && (key >> 10) == (found >> 10), key & 1023u);
        }
      } else if (round == 0) {
        each_key([&](bool in, uint32_t key) { count_keys(s_hist[1], in && (key >> 21) == (found >> 21), (key >> 10) & 2047u); });
      } else {
        each_key([&](bool in, uint32_t key) { count_keys(s_hist[2], in && (key >> 10) == (found >> 10), key & 1023u); });
      }
    }
    // Keys above `found` are kept, and the first `left` of those equal to it (mostly that
    // is one, or all).  In front of this CTA's positions:
    const bool all = left && left == s_pick[2];
    uint32_t larger = 0, equal = 0;
    if (C > 1 && left) {
      uint32_t sum;
      (void)evict_scan<kEvictWarps>(mine, s_warp, &sum);
      if (tid == 0) {
        s_count[0] = sum;
        s_count[1] = s_hist[2][found & 1023u];
      }
      cluster_sync();
      for (int r = 0; r < rank; ++r) {
        larger += ld_dsmem_u32(smem_addr(&s_count[0]), r);
        equal += ld_dsmem_u32(smem_addr(&s_count[1]), r);
      }
    }
    if (all) larger += equal;
    float coming[kEvictKeys];
    auto load_row = [&](int t0) {  // a warp has 32 * kEvictKeys positions in a row
      const int t1 = t0 + warp * 32 * kEvictKeys + lane;
#pragma unroll
      for (int u = 0; u < kEvictKeys; ++u) coming[u] = t1 + 32 * u < to ? mass[t1 + 32 * u] : 0.f;
    };
    const unsigned lower = (1u << lane) - 1u;
    int32_t *const others = kept + p.first;
    int turn = 0;
    load_row(from);
#pragma unroll 1
    for (int t0 = from; t0 < to && left; t0 += kStep, turn ^= 1) {
      const int t1 = t0 + warp * 32 * kEvictKeys + lane;
      unsigned who[kEvictKeys], same[kEvictKeys];
      uint32_t count = 0;
#pragma unroll
      for (int u = 0; u < kEvictKeys; ++u) {
        const uint32_t key = evict_key(coming[u]);
        const bool in = t1 + 32 * u < to;
        who[u] = __ballot_sync(0xffffffffu, in && (all ? key >= found : key > found));
        count += __popc(who[u]);
        same[u] = 0u;
        if (!all) {
          same[u] = __ballot_sync(0xffffffffu, in && key == found);
          count += __popc(same[u]) << 16;
        }
      }
      load_row(t0 + kStep);
      if (lane == 0) s_rows[turn][warp] = count;
      __syncthreads();
      uint32_t l = larger, e = equal;
#pragma unroll
      for (int w = 0; w < kEvictWarps; ++w) {
        const uint32_t x = s_rows[turn][w];
        if (w < warp) {
          l += x & 0xffffu;
          e += x >> 16;
        }
        larger += x & 0xffffu;
        equal += x >> 16;
      }
#pragma unroll
      for (int u = 0; u < kEvictKeys; ++u) {
        const uint32_t before = all ? 0u : e + __popc(same[u] & lower);
        if ((who[u] >> lane & 1u) || ((same[u] >> lane & 1u) && before < left))
          others[l + __popc(who[u] & lower) + (all ? 0u : min(before, left))] = t1 + 32 * u;
        l += __popc(who[u]);
        e += __popc(same[u]);
      }
    }
    sync_all();
    // Rows in rounds of ascending places, by asynchronous copies: a warp has some rows of
    // every round and two slots of shared memory, so that a round's rows are on their way
    // in while the round before waits for its barrier and goes out.  Where they come from
    // and go to is looked up a round ahead of that.  One of two CTAs has K and the other V, so
    // that neither waits for the other (11 ns a row, with rows of both 19); of more each has
    // rows of both (a CTA's copies are bound by their number: 128-byte parts of rows
    // took as long as whole ones).
    constexpr int kSheets = C == 2 ? 1 : 2, kGroups = C == 2 ? 1 : C;
    const int row_bytes = p.D * 2, R = min(32 / kSheets, kSlot / (kSheets * row_bytes));
    const int32_t *table = p.block_table + static_cast<size_t>(b) * p.max_pages;
    auto place = [&](int pos) -> int {
      const int page = table[pos / SF_PAGE_SIZE];
      if (page < 0 || page >= p.num_pages) {
        set_status(p.status, SF_DEVICE_BAD_PAGE);
        return -1;
      }
      return (page * p.H_kv + h) * SF_PAGE_SIZE + pos % SF_PAGE_SIZE;
    };
    const int r = lane % R, sheet = lane / R;  // the lane's row of the warp's
    const int side = C == 2 ? rank : sheet;    // K or V
    const bool works = sheet < kSheets;
    const int group = C == 2 ? 0 : rank, first_row = (group * kEvictWarps + warp) * R + r, rows = kGroups * kEvictWarps * R;
    const int rounds = (p.budget + rows - 1) / rows;
    char *cache = reinterpret_cast<char *>(side == 0 ? layer.k : layer.v);
    const uint32_t slot = smem_addr(smem) + warp * 2 * kSlot + lane * row_bytes;
    const uint32_t bar = smem_addr(&s_bar[warp][0]);
    struct Row {
      int src, dst;  // cache rows, dst < 0: stays
      float w;
    };
    auto look_up = [&](int round) -> Row {
      Row x{-1, -1, 0.f};
      const int j = round * rows + first_row;
      if (works && j < p.budget) {
        const int pos = kept[j];
        if (side == 0) x.w = mass[pos];
        if (pos != j) {
          x.src = place(pos);
          x.dst = place(j);
          if (x.src < 0) x.dst = -1;
        }
      }
      return x;
    };
    bool ok = true;
    int asked = 0;  // rounds whose rows were asked for
    auto copy_in = [&](int round, const Row &x) {
      asked = round + 1;
      const unsigned who = __ballot_sync(0xffffffffu, x.dst >= 0);
      const uint32_t full = bar + 8 * (round & 1);
      if (lane == 0) mbar_arrive_expect_tx(full, static_cast<uint32_t>(__popc(who) * row_bytes));
      __syncwarp();
      if (x.dst >= 0)
        bulk_copy_g2s(slot + (round & 1) * kSlot, cache + static_cast<long long>(x.src) * row_bytes, row_bytes, full);
    };
    asm volatile("fence.proxy.async;" ::: "memory");  // the slots held the histograms
    __syncthreads();
    Row now = look_up(0), next = look_up(1);
    copy_in(0, now);
#pragma unroll 1
    for (int round = 0; round < rounds; ++round) {
      if (ok && round + 1 < rounds) {
        bulk_wait_read();  // this lane's rows of the round before have left the slot
        __syncwarp();
        copy_in(round + 1, next);
      }
      const Row then = look_up(round + 2);
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait_bounded(bar + 8 * (round & 1), (round >> 1) & 1));
      if constexpr (kGroups > 1) cluster_sync();  // every row of this round and of those before is in
      else __syncthreads();
      if (ok && now.dst >= 0) {
        bulk_copy_s2g(cache + static_cast<long long>(now.dst) * row_bytes, slot + (round & 1) * kSlot, row_bytes);
        bulk_commit();
      }
      const int j = round * rows + first_row;
      if (works && side == 0 && j < p.budget) mass_out[j] = now.w;
      now = next;
      next = then;
    }
    bulk_wait_all();
    if (!ok) {  // the copies still in flight land (bounded) before shared memory is left
      for (int round = max(asked - 2, 0); round < asked; ++round)
        (void)mbar_wait_bounded(bar + 8 * (round & 1), (round >> 1) & 1);
      if (lane == 0) {
        set_status(p.status, SF_DEVICE_TIMEOUT);
        atomicOr(p.gave_up, 1u);
      }
      __syncwarp();
    }
    sync_all();
    for (int t = p.budget + rank * kEvictThreads + tid; t < p.width; t += C * kEvictThreads) mass_out[t] = 0.f;
  }

  evict_finish<kEvictThreads>(p);
  launch_dependents_after_stores();
}

// Contexts of at most 32 * KEYS keys: one CTA a (layer, sequence, KV head).  Its first
// warp has all weights in registers and finds the value of the last kept key bit by bit,
// by counting.  Then each warp moves some columns of K or of V, in the order of the rows, a
// batch's loads in front of its stores, as tree_commit does: it needs no barrier.
template <int KEYS, int WARPS, int BLOCKS>
__global__ void __launch_bounds__(32 * WARPS, BLOCKS) kv_evict_short_kernel(const __grid_constant__ EvictParams p) {
  constexpr int THREADS = 32 * WARPS, PARTS = WARPS / 2, MOST = 32 * KEYS;
  __shared__ int32_t s_page[MOST / SF_PAGE_SIZE];
  __shared__ uint16_t s_pos[MOST];
  __shared__ int s_first;
  const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp_id();
  const int task = blockIdx.x, h = task % p.H_kv, lb = task / p.H_kv, b = lb % p.B;
  const EvictLayer &layer = p.layers[lb / p.B];
  const size_t bh = static_cast<size_t>(b) * p.H_kv + h;
  grid_dependency_wait();
  bool cut, bad;
  const int L = evict_length(p, b, cut, bad);
  if (bad && lb < p.B && h == 0 && tid == 0) set_status(p.status, SF_DEVICE_BAD_SEQLEN);
  const float *mass = layer.mass + bh * p.width;
  float *mass_out = layer.mass_out + bh * p.width;
  int32_t *kept = layer.kept + bh * p.budget;
  if (!cut) {
    evict_nothing(p, mass, mass_out, kept, L, bad, tid, THREADS);
  } else {
    if (warp == 1 && lane < MOST / SF_PAGE_SIZE)
      s_page[lane] = lane * SF_PAGE_SIZE < L ? p.block_table[static_cast<size_t>(b) * p.max_pages + lane] : -1;
    if (warp == 0) {
      float w[KEYS];
      uint32_t key[KEYS];
#pragma unroll
      for (int u = 0; u < KEYS; ++u) w[u] = 32 * u + lane < L ? mass[32 * u + lane] : 0.f;
#pragma unroll
      for (int u = 0; u < KEYS; ++u) {
        const int t = 32 * u + lane;
        key[u] = t >= L ? 0u : t < p.first || t >= L - p.recent ? 0xffffffffu : evict_key(w[u]);  // (no weight's is 0)
      }
      // the largest value that `budget` keys reach; once as many do, it need not be exact
      const int budget = p.budget;
      uint32_t found = 0u;
      int reach = L;
      for (uint32_t bit = 1u << 31; bit && reach != budget; bit >>= 1) {
        int n = 0;
#pragma unroll
        for (int u = 0; u < KEYS; ++u) n += key[u] >= (found | bit);
        n = __reduce_add_sync(0xffffffffu, n);
        if (n >= budget) {
          found |= bit;
          reach = n;
        }
      }
      // all above, and the first of those equal to it
      int above = 0;
#pragma unroll
      for (int u = 0; u < KEYS; ++u) above += key[u] > found;
      int left = reach == budget ? MOST : budget - __reduce_add_sync(0xffffffffu, above);
      int at = 0, in_place = MOST;
#pragma unroll
      for (int u = 0; u < KEYS; ++u) {
        const unsigned lower = (1u << lane) - 1u;
        const bool eq = key[u] == found && 32 * u + lane < L;
        const unsigned equal = __ballot_sync(0xffffffffu, eq);
        const bool stays = key[u] > found || (eq && __popc(equal & lower) < left);
        left -= __popc(equal);
        const unsigned who = __ballot_sync(0xffffffffu, stays);
        if (in_place == MOST && ~who) in_place = 32 * u + __ffs(~who) - 1;
        if (stays) {
          const int j = at + __popc(who & lower);
          kept[j] = 32 * u + lane;
          s_pos[j] = static_cast<uint16_t>(32 * u + lane);
          mass_out[j] = w[u];
        }
        at += __popc(who);
      }
      for (int t = budget + lane; t < p.width; t += 32) mass_out[t] = 0.f;
      if (lane == 0) s_first = in_place;
    }
    __syncthreads();
    uint4 *cache = warp & 1 ? layer.v : layer.k;
    const int wide = p.D / 8, from = (warp >> 1) * wide / PARTS, columns = ((warp >> 1) + 1) * wide / PARTS - from;
    const int first = s_first, total = (p.budget - first) * columns;
    auto place = [&](int pos) -> long long {  // in 16-byte pieces; -1: a page outside the pool
      const int page = s_page[pos / SF_PAGE_SIZE];
      if (page < 0 || page >= p.num_pages) {
        set_status(p.status, SF_DEVICE_BAD_PAGE);
        return -1;
      }
      return ((static_cast<long long>(page) * p.H_kv + h) * SF_PAGE_SIZE + pos % SF_PAGE_SIZE) * wide + from;
    };
    for (int base = 0; base < total; base += 32 * kShortBatch) {
      uint4 v[kShortBatch];
      long long to[kShortBatch];
#pragma unroll
      for (int u = 0; u < kShortBatch; ++u) {
        const int x = base + 32 * u + lane;
        to[u] = -1;
        if (x < total) {
          const int r = x / columns, piece = x - r * columns;
          const long long source = place(s_pos[first + r]);
          to[u] = place(first + r);
          if (source < 0) to[u] = -1;
          if (to[u] >= 0) {
            to[u] += piece;
            v[u] = cache[source + piece];
          }
        }
      }
      __syncwarp();
#pragma unroll
      for (int u = 0; u < kShortBatch; ++u)
        if (to[u] >= 0) cache[to[u]] = v[u];
      __syncwarp();
    }
  }
  evict_finish<THREADS>(p);
  launch_dependents_after_stores();
}

// `kept` of all layers for a call that does not ask for it lies behind the header.
static size_t evict_bytes(int layers, int B, int H_kv, int budget) {
  return kEvictHeader + round_up(static_cast<size_t>(layers) * B * H_kv * budget * sizeof(int32_t), 256);
}

static int check_evict(int layers, int B, int H_kv, int budget) {
  if (layers < 1 || layers > SF_MAX_LAYERS)
    return fail(SF_ERR_INVALID_ARG, "num_layers=%d outside [1, %d]", layers, SF_MAX_LAYERS);
  if (B < 1 || B > SF_MAX_BATCH) return fail(SF_ERR_INVALID_ARG, "B=%d outside [1, %d]", B, SF_MAX_BATCH);
  if (H_kv < 1 || H_kv > 1024) return fail(SF_ERR_INVALID_ARG, "H_kv=%d outside [1, 1024]", H_kv);
  if (budget < 1 || budget > (1 << 30)) return fail(SF_ERR_INVALID_ARG, "budget=%d", budget);
  return SF_OK;
}

static int evict_setup(int device) {
  static std::mutex mu;
  static bool done[64] = {};
  if (device < 0 || device >= 64) return fail(SF_ERR_UNSUPPORTED, "device ordinal %d", device);
  std::lock_guard<std::mutex> lock(mu);
  if (done[device]) return SF_OK;
  for (auto fn : {kv_evict_kernel<1, 3>, kv_evict_kernel<1, 4>, kv_evict_kernel<2, 3>, kv_evict_kernel<4, 3>, kv_evict_kernel<8, 3>}) {
    const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, evict_smem(3));
    if (e != cudaSuccess) return fail(SF_ERR_CUDA, "cudaFuncSetAttribute (eviction): %s", cudaGetErrorString(e));
  }
  done[device] = true;
  return SF_OK;
}

// CTAs per (layer, sequence, KV head).  One CTA takes 10 us, 24 ns a row and 2.5 a key, so
// `rows` says how long; a cluster starts 6 to 9 us later, more yet where CTAs share an SM, and
// takes 11 ns a row with two CTAs, 10 with four and 5 with eight.  In us, one / two / four /
// eight CTAs (152 SMs):
//     heads    500 to 400      1000 to 900     3000 to 1024    10000 to 6000
//         8  17 / 20 / 19 / 19  29 / 26 / 23 / 21  36 / 28 / 24 / 22  173 / 96 / 72 / 45
//        18  18 / 20 / 18 / 25  29 / 26 / 23 / 28  36 / 28 / 25 / 28  177 / 97 / 72 / 58
//        40  18 / 20 / 22 / 31  29 / 26 / 27 / 35  36 / 29 / 29 / 36  209 / 110 / 98 / 78
//       100  18 / 23 / 26 / 65  29 / 31 / 33 / 71  38 / 35 / 36 / 74  228 / 150 / 133 / 168
//       200  22 / 26 / 50 / 126  41 / 41 / 70 / 147  57 / 52 / 82 / 154  283 / 226 / 295 / 354
static int evict_cluster(int tasks, int budget, int width, int sms) {
  const long long rows = budget + 3LL * width / 20, slots = 3LL * sms;
  if (rows < 640) return 1;
  if (8LL * tasks <= slots && (9LL * tasks <= sms || rows >= 3400)) return 8;
  if (4LL * tasks <= slots && (4LL * tasks <= sms || rows >= 2400)) return 4;
  if (2LL * tasks <= slots && (2LL * tasks <= sms || rows >= 1400)) return 2;
  return 1;
}

struct EvictLaunch {
  void (*kernel)(const EvictParams);
  int cluster, threads, smem;
};

// The lengths are on the device, so `width` bounds them: the weights' or the table's, whichever
// is less.  Of at most 256 tokens a head: 16 warps where no SM has more than two heads (8
// heads of 250 tokens to 200: 11.9 us, with kv_evict_kernel 13.1),
// else four, which leave room for eight heads an SM (2400 heads of 85 tokens to 12: 12.2 us, with
// 16 warps 43; in a table of 4096 tokens, which takes kv_evict_kernel, 27; of 250 to
// 200: 90, with 16 warps 131, 120).  Of at most 512, many heads: 2400 of 500 tokens to 64 47 us, with
// kv_evict_kernel 75, to 400 173 and 193 (but 128 heads to 400 21, 17.5).
static EvictLaunch evict_launch(int tasks, int budget, int width, int sms) {
  const bool many = tasks > 2 * sms;
  if (width <= 256)
    return many ? EvictLaunch{kv_evict_short_kernel<8, 4, 8>, 1, 128, 0} : EvictLaunch{kv_evict_short_kernel<8, 16, 2>, 1, 512, 0};
  if (width <= 512 && many) return {kv_evict_short_kernel<16, 4, 8>, 1, 128, 0};
  const int C = evict_cluster(tasks, budget, width, sms);
  // Four CTAs an SM with smaller slots where three leave more of the last wave empty (1024
  // heads of 3008 tokens to 1024: 195 us, with three 210; 600 of 3000 to 1000 122, 134; 3584
  // of 1000 to 200 164, 178; but 680 of 3000 to 2500 345, 305).
  const int three = (tasks + 3 * sms - 1) / (3 * sms) * 3, four = (tasks + 4 * sms - 1) / (4 * sms) * 4;
  if (C == 1 && four <= three) return {kv_evict_kernel<1, 4>, 1, kEvictThreads, evict_smem(4)};
  return {C == 1 ? kv_evict_kernel<1, 3> : C == 2 ? kv_evict_kernel<2, 3> : C == 4 ? kv_evict_kernel<4, 3> : kv_evict_kernel<8, 3>, C,
          kEvictThreads, evict_smem(3)};
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
  if ((long long)num_pages * H_kv * SF_PAGE_SIZE >= (1LL << 31))
    return fail(SF_ERR_UNSUPPORTED, "KV pool of %d pages x %d heads too large", num_pages, H_kv);
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
  const size_t need = kept ? kEvictHeader : evict_bytes(num_layers, B, H_kv, budget);
  if (workspace_bytes < need) return fail(SF_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, need);
  EvictParams p;
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  for (int l = 0; l < num_layers; ++l) {
    EvictLayer &x = p.layers[l];
    x.mass = mass[l];
    x.mass_out = mass_out[l];
    x.k = static_cast<uint4 *>(k_caches[l]);
    x.v = static_cast<uint4 *>(v_caches[l]);
    x.kept = kept ? kept[l] : reinterpret_cast<int32_t *>(ws + kEvictHeader) + static_cast<size_t>(l) * B * H_kv * budget;
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
  p.gave_up = reinterpret_cast<uint32_t *>(ws + 192);
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
  const int tasks = num_layers * B * H_kv;
  const EvictLaunch launch = evict_launch(tasks, budget, std::min(mass_width, max_pages_per_seq * SF_PAGE_SIZE), dev.sm_count);
  const int C = launch.cluster;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = C;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(tasks * C));
  cfg.blockDim = dim3(launch.threads);
  cfg.dynamicSmemBytes = launch.smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = C > 1 ? 2 : 1;
  if ((st = evict_setup(dev.ordinal)) != SF_OK) return st;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, launch.kernel, p);
  if (e != cudaSuccess) return fail(SF_ERR_CUDA, "eviction launch: %s", cudaGetErrorString(e));
  return SF_OK;
}

}  // extern "C"
