// shared_prefix.cu -- verification attention of a batch whose sequences share
// long prefixes, on the 5th-generation tensor cores.
//
// Row i of sequence b sees the prefix of its group and its own tokens
// 0 .. L_b + i.  The softmax over both parts is the merge of the softmaxes over
// the parts (running maximum, sum and unnormalised output), so the work is a
// list of segments, each a product of up to 256 query rows with a run of keys:
//  * prefix segments (group, KV head, pair of row tiles): the rows of all of a
//    group's sequences for one KV head, packed into tiles of 128 rows (whole
//    tokens: floor(128 / g) tokens of g query heads), two tiles a segment.  The
//    prefix's keys and values are copied to shared memory once for 256 rows.
//  * own segments (sequence, pair of KV heads): the sequence's n_q * g rows of each
//    head against its own tokens, with the causal mask of the draft block.  Their key
//    tiles alternate between the heads.
// The segments' key tiles (128 keys) lie on one axis, which is cut into one
// equal range per SM by a cost rule (below); a CTA works through the pieces of
// its range and leaves one partial result (maximum, sum, O in fp32) per piece
// and row tile; shared_prefix_merge_kernel joins the partials of every row.
//
// The CTA has two streams, each with 128 softmax threads (one TMEM lane, one
// query row a thread), a score buffer and an accumulator:
//     TMEM columns  S_0 [0, 128)  S_1 [128, 256)  O_0 [256, 384)  O_1 [384, 512).
// A piece with two row tiles gives one to each stream, and so does one with two heads
// (59 sequences of 212 to 916 own tokens, 32 heads, a prefix of 140: 122 us; a piece per
// head took a quarter more); a piece with one row tile gives its even key tiles to stream 0 and
// its odd ones to stream 1, whose results are joined in the CTA, or, with one key
// tile, goes to the streams in turn.  So while one stream's softmax runs, the tensor
// cores work for the other.
// P = exp2(S') goes back over the scores as bf16 (the A operand of O += P V), so
// a stream's next Q K^T is issued behind its P V; tcgen05 MMAs of one thread
// execute in issue order.  Each stream has a warp that issues its MMAs (one warp
// for both, looking for what is ready, left the tensor cores idle for some 300
// cycles before every operation); one warp copies K and V, and one publishes the
// pieces and copies Q, which has to wait for the stream's previous job while keys of
// the next can be copied ahead.  K and V tiles go through one ring of 32 KB slots (16
// KB with 64-wide heads), which both streams pass in order.
//
// What bounds it.  Many rows (64 sequences of 8 rows, 28 / 4 heads of 128, a prefix of
// 32768 tokens: 184 to 199 us by box, 1.2 to 1.3 PFLOP/s, 13 of them the merge): the MMAs.  A
// key tile of two row tiles is 32 of them; they take 74 cycles each, not the 64 of the
// tensor cores' rate, as Q, K, V and the copies together read and write shared memory
// at its full 128 bytes a cycle; a tile takes 2,880 cycles with what the turns leave
// idle.  One row tile (8 sequences of 5 rows, 32 / 32 heads, 3008 tokens: 25 us for 62.5
// MB, 2.5 TB/s) and few keys: the start (the cut of the axis takes 3 us from cold
// instructions, the first keys 2), the partials' way through L2 and the merge kernel
// (5 us behind the last piece).
//
// The running maximum is a reference that moves when a row's new maximum
// exceeds it by more than kSpRescaleLog2, so rescaling O is rare.  The row sums
// are sums of the fp32 weights.  P V takes the weights rounded to bf16 (up to 2^-8
// of a weight, which averages out over many keys), and on the key tiles that hold a
// sequence's first 128 keys also what that rounding left, as a second bf16 term: rows
// that see few keys, and rows whose weight lies on their first keys, as with attention
// sinks, have no others to average with (8 sequences of 5 rows over 3008 tokens: 24.4 ->
// 24.9 us, 64 over 32768 183 -> 184).  On the other tiles the sum that O is divided by
// takes each tile's largest weight as it was rounded (the LSE's does not): a later key
// that outweighs all others may be up to 2^kSpRescaleLog2 in units of the reference, and
// its rounding would be the row's (1 %: 24.9 -> 25.2 us, 34.0 -> 34.3 for 4 videos).
// Every wait is bounded; a timeout sets SF_DEVICE_TIMEOUT and stops every role.
#include <algorithm>
#include <cmath>
#include <mutex>
#include <type_traits>

#include "attn_common.cuh"
#include "sf_host.h"
#include "shared_prefix_layout.h"

namespace sf {

constexpr int kSpTilePages = kSpTile / SF_PAGE_SIZE;
constexpr int kSpThreads = 384;  // two softmax warpgroups, two MMA warps, two copy warps
constexpr int kSpMmaWarp = 8, kSpCopyWarp = 10, kSpQueryWarp = 11;
constexpr int kSpMaxRegs = 168;  // three warps share a sub-partition's 16K registers
constexpr uint32_t kSpTmemCols = 512;
constexpr float kSpRescaleLog2 = 8.f;
constexpr int kSpMergeThreads = 256;
// Cost of a segment on the partition's axis: kSpCostOne or kSpCostTwo for each of its
// key tiles (one row tile, or two), and kSpCostSegOne or kSpCostSegTwo for itself (its Q
// copy, pipeline start and epilogue; two row tiles leave 128 KB of partial results),
// with kSpCostFew more for a prefix's first key tile in two terms (with 0, 1 or 2 the same
// within 3 %).  Measured, least squares over the CTAs
// of three workloads: 1.3 to 1.5 us for a key tile of two row tiles, 0.9 to 1.8 of one,
// 2 to 4 for a piece.  With one unit for every row tile's key tile and two a segment the
// longest CTA of the workload of 64 sequences took 18 % more than the mean (225 us, with
// the costs 195); with 5 for either kind of segment, 59 sequences of some 560 tokens with a prefix
// of 8 took 174 us (119 with 10): a few CTAs had all the prefix's segments.
constexpr uint32_t kSpCostSegOne = 5, kSpCostSegTwo = 10, kSpCostFew = 4, kSpCostOne = 3, kSpCostTwo = 4;
constexpr int kSpFirstPages = 4; // pages of a key tile in the first part of P V (the rest follows while that runs)

// What the merge kernel has to know about a sequence: where its own segments and
// its group's lie on the partition's axis.
struct __align__(16) SpRecord {
  uint32_t cost, slot;  // axis and partial rows before the own segments
  int keys;             // own keys (0: idle)
  uint32_t chunk;       // axis per CTA
  uint32_t pre_cost, pre_slot;
  int pre_keys;         // 0: no prefix
  int first, sequences; // of the group
  int pad[3];
};

struct SpParams {
  const int32_t *prefix_table, *prefix_lens, *group_starts, *block_table, *seq_lens;
  const __nv_bfloat16 *v_cache;
  __nv_bfloat16 *out;
  float *lse;
  uint32_t *status;
  float *part_o;   // unnormalised outputs, [D / 4][rows] float4 per piece and row tile
  float2 *part_ml; // maximum (base-2 units) and sum of every row of a partial
  SpRecord *plan;  // [B], for the merge kernel
  int B, n_q, H_q, H_kv, group, num_pages, num_groups, max_prefix_pages, max_pages;
  int tokens_per_tile;  // floor(128 / group), at least 16
  uint32_t tile_magic;
  int oob_row;          // a tensor-map row beyond the pool: loads as zeros
  int G;                // CTAs of the split kernel
  float per_cta;        // 1 / G
  float scale_log2;
};

// The segments: entity e < num_groups is a group's prefix, entity num_groups + b
// sequence b's own tokens.  `tokens` query tokens from token0 on, in `tiles` row
// tiles, against `keys` keys.
struct SpEntity {
  int keys, token0, tokens, tiles, pairs, key_tiles;
  int units;           // KV heads, or (own) pairs of KV heads, the last perhaps a single one
  uint32_t head_cost;  // per unit
  uint32_t cost;       // of all units
  uint32_t slot_rows;  // partial rows of one piece
  uint32_t few;        // the first key tile's second term
  // of a segment: its start, and its length for key tiles of which some may be other heads'
  __device__ __forceinline__ uint32_t start(int dual) const { return (dual ? kSpCostSegTwo : kSpCostSegOne) + few; }
  __device__ __forceinline__ uint32_t length(int dual, int tiles_) const {
    return start(dual) + (dual ? kSpCostTwo : kSpCostOne) * static_cast<uint32_t>(tiles_);
  }
  // its first key tile at or behind position at of the axis
  __device__ __forceinline__ int tile_at(uint32_t at, uint32_t base, int dual, int tiles_) const {
    const uint32_t b = base + start(dual);
    if (at <= b) return 0;
    const uint32_t t = dual ? (at - b + kSpCostTwo - 1) / kSpCostTwo : (at - b + kSpCostOne - 1) / kSpCostOne;
    return t < static_cast<uint32_t>(tiles_) ? static_cast<int>(t) : tiles_;
  }
};

// n / tokens_per_tile for n < 2^25 (tile_magic = ceil(2^32 / tokens_per_tile))
__device__ __forceinline__ int sp_tiles(const SpParams &p, int n) {
  return static_cast<int>(__umulhi(static_cast<uint32_t>(n), p.tile_magic));
}

__device__ __forceinline__ SpEntity sp_entity(const SpParams &p, bool own, int first, int sequences, int keys) {
  SpEntity x;
  x.keys = keys;
  x.token0 = first * p.n_q;
  x.tokens = sequences * p.n_q;
  x.tiles = own ? 1 : sp_tiles(p, x.tokens + p.tokens_per_tile - 1);
  x.pairs = (x.tiles + 1) >> 1;
  x.key_tiles = (keys + kSpTile - 1) / kSpTile;
  x.few = own ? 0u : kSpCostFew;
  if (own) {
    x.units = (p.H_kv + 1) >> 1;
    x.head_cost = x.length(0, 2 * x.key_tiles);
    x.cost = x.units * x.head_cost - (p.H_kv & 1) * kSpCostOne * static_cast<uint32_t>(x.key_tiles);
    x.slot_rows = 2u * static_cast<uint32_t>(x.tokens * p.group);
  } else {
    x.units = p.H_kv;
    x.head_cost = static_cast<uint32_t>(x.tiles >> 1) * x.length(1, x.key_tiles) + (x.tiles & 1) * x.length(0, x.key_tiles);
    x.cost = x.units * x.head_cost;
    x.slot_rows = x.tiles > 1 ? 2u * kSpTile : static_cast<uint32_t>(x.tokens * p.group);
  }
  if (keys == 0) x.head_cost = x.cost = 0u;
  return x;
}

// The axis in ranges of `chunk`, one per CTA (the last ones shorter or empty: the
// longest is what counts).  At least ceil(Tot / G), and hardly more.
__device__ __forceinline__ uint32_t sp_chunk(const SpParams &p, uint32_t Tot) {
  const uint32_t q = static_cast<uint32_t>(static_cast<float>(Tot) * p.per_cta + 0.999f);
  return q + (q >> 20) + (Tot > q * static_cast<uint32_t>(p.G));
}

// a / b for quotients below 2^20
__device__ __forceinline__ uint32_t sp_div(uint32_t a, uint32_t b) {
  uint32_t q = static_cast<uint32_t>(__fdividef(static_cast<float>(a), static_cast<float>(b)));
  if (q * b > a) --q;
  if ((q + 1u) * b <= a) ++q;
  return q;
}

__device__ __forceinline__ int sp_rows(const SpParams &p, const SpEntity &x, int tile) {
  const int left = x.tokens - tile * p.tokens_per_tile;
  return (left < p.tokens_per_tile ? left : p.tokens_per_tile) * p.group;
}

// max of three in one instruction (a NaN is ignored, as by fmaxf)
__device__ __forceinline__ float sp_max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Two fp32 values in one 64-bit register: one instruction for both.
__device__ __forceinline__ unsigned long long sp_pair(float x, float y) {
  unsigned long long v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
  return v;
}
__device__ __forceinline__ void sp_unpair(unsigned long long v, float &x, float &y) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
}
__device__ __forceinline__ unsigned long long sp_fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ unsigned long long sp_add2(unsigned long long a, unsigned long long b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

template <int D, int STAGES>
__global__ void __maxnreg__(kSpMaxRegs)
shared_prefix_split_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                           const __grid_constant__ CUtensorMap tmap_q_tile,
                           const __grid_constant__ CUtensorMap tmap_q_own,
                           const __grid_constant__ SpParams p) {
  using L = SpSmem<D, STAGES>;
  constexpr int HALVES = D / 64;
  constexpr int kPageBytes = SF_PAGE_SIZE * D * 2;
  constexpr int kPageHalfBytes = SF_PAGE_SIZE * kRowBytes;
  constexpr int kHalfTileBytes = kSpTile * kRowBytes;       // 64 columns of a Q tile
  constexpr uint32_t kKSbo = HALVES == 2 ? 2048u : 1024u;   // 8-key atoms of a K tile
  constexpr uint32_t kIdescQK = idesc_bf16_f32(128, kSpTile, 0, 0);
  constexpr uint32_t kIdescPV = idesc_bf16_f32(128, D, 0, 1);
  constexpr int FULL = 0, EMPTY = STAGES, QFULL = 2 * STAGES, QEMPTY = QFULL + 2, SFULL = QEMPTY + 2,
                PFULL = SFULL + 2, ODONE = PFULL + 4, FIN = ODONE + 2, TURN = FIN + 2,
                IFULL = TURN + 2, IEMPTY = IFULL + kSpItems, JOINT = IEMPTY + kSpItems, READ = JOINT + 2;

  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t ring = smem_addr(smem);
  auto bar = [&](int i) -> uint32_t { return ring + L::kBarOffset + 8u * static_cast<uint32_t>(i); };
  int *s_misc = reinterpret_cast<int *>(smem + L::kMiscOffset);
  volatile int *s_abort = s_misc + 1;
  int *s_info = reinterpret_cast<int *>(smem + L::kInfoOffset);
  // per stream and parity of its job (a warp may be a job ahead of another): the last
  // piece with infinities or NaN among the draft's V
  volatile int *s_bad = s_info + 8 * kSpInfo;
  const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp_id();

  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(bar(FULL + s), 1);
      mbar_init(bar(EMPTY + s), 2);  // one arrival per stream
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar(QFULL + s), 1);
      mbar_init(bar(QEMPTY + s), 1);
      mbar_init(bar(SFULL + s), 1);
      mbar_init(bar(PFULL + 2 * s), 4);
      mbar_init(bar(PFULL + 2 * s + 1), 4);
      mbar_init(bar(ODONE + s), 1);
      mbar_init(bar(FIN + s), 1);
      mbar_init(bar(TURN + s), 1);
      mbar_init(bar(JOINT + s), 4);
      mbar_init(bar(READ + s), 4);
    }
    for (int i = 0; i < kSpItems; ++i) {
      mbar_init(bar(IFULL + i), 1);
      mbar_init(bar(IEMPTY + i), kSpThreads / 32 - 1);  // every warp but the publishing one
    }
    fence_mbar_init();
    prefetch_tensormap(&tmap_k);
    prefetch_tensormap(&tmap_v);
    prefetch_tensormap(&tmap_q_tile);
    prefetch_tensormap(&tmap_q_own);
    s_misc[1] = 0;
    for (int i = 0; i < 4; ++i) s_bad[i] = 0;
  }
  __syncthreads();
  grid_dependency_wait();
  grid_launch_dependents();
  SpItem *items = reinterpret_cast<SpItem *>(smem + L::kItemOffset);
  uint32_t seen = 0;  // pieces read
  // tensor memory: allocated (behind the wait: a kernel that waits for its
  // predecessor must not hold what that may need) by the first MMA warp
  uint32_t tmem = 0;
  if (warp < kSpCopyWarp) {
    if (warp == kSpMmaWarp) {
      tmem_alloc(smem_addr(s_misc), kSpTmemCols);
      tmem_relinquish_alloc_permit();
      tc_fence_before_sync();
    }
    named_bar_sync(1, 32 * kSpCopyWarp);
    tc_fence_after_sync();
    tmem = static_cast<uint32_t>(s_misc[0]);
  }
  // The next piece; null behind the last one (or after a timeout).  The warp
  // gives the entry back with release_item.
  auto next_item = [&]() -> const SpItem * {
    const uint32_t i = seen % kSpItems;
    const bool w = mbar_wait_or_abort(bar(IFULL + i), (seen / kSpItems) & 1u, s_abort);
    ++seen;
    return __all_sync(0xffffffffu, w) && items[i].n > 0 ? items + i : nullptr;
  };
  auto release_item = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(IEMPTY + (seen - 1) % kSpItems));
  };

  if (warp == kSpQueryWarp) {
    // ------------------------------------------------------------------
    // The CTA's pieces, published one after the other, each followed by the
    // copies of its Q tiles as soon as the streams' last Q K^T have read theirs.
    // Loops up to the first piece stay loops: their instructions come from L2, and
    // unrolled they cost a call of few keys 0.3 to 0.6 us of some 14.
    // ------------------------------------------------------------------
    const int E = p.num_groups + p.B;
    int *s_len = reinterpret_cast<int *>(smem + L::kPlanOffset), *s_start = s_len + E;
    uint32_t *s_cost = reinterpret_cast<uint32_t *>(s_start + p.num_groups + 1), *s_slot = s_cost + p.num_groups;
    bool bad = false;
#pragma unroll 1
    for (int e = lane; e <= E; e += 32) {
      const bool own = e >= p.num_groups;
      int n = 0, s = 0;
      if (e < E) n = own ? p.seq_lens[e - p.num_groups] : p.prefix_lens[e];
      if (e <= p.num_groups) s = p.group_starts[e];
      const int least = own ? p.n_q : 0, most = (own ? p.max_pages : p.max_prefix_pages) * SF_PAGE_SIZE;
      if ((n < least || n > most) && n != 0) {
        set_status(p.status, SF_DEVICE_BAD_SEQLEN);
        n = n < least ? least : most;
      }
      if (e < E) s_len[e] = n;
      if (e <= p.num_groups) {
        s_start[e] = s;
        bad |= (e == 0 && s != 0) || (e == p.num_groups && s != p.B);
      }
    }
    __syncwarp();
#pragma unroll 1
    for (int g = lane; g < p.num_groups; g += 32) bad |= s_start[g + 1] < s_start[g];
    if (__any_sync(0xffffffffu, bad)) {  // malformed groups: no sequence has a prefix
      for (int g = lane; g <= p.num_groups; g += 32) s_start[g] = 0;
      if (lane == 0) set_status(p.status, SF_DEVICE_BAD_INDEX);
      __syncwarp();
    }
    auto entity = [&](int e) -> SpEntity {
      const bool own = e >= p.num_groups;
      const int first = own ? e - p.num_groups : s_start[e];
      return sp_entity(p, own, first, own ? 1 : s_start[e + 1] - first, s_len[e]);
    };
    auto group_of = [&](int b) -> int {  // the last group that starts at or before sequence b
      int lo = 0, hi = p.num_groups;
#pragma unroll 1
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_start[mid] <= b) lo = mid; else hi = mid;
      }
      return lo;
    };
    uint32_t sum = 0;
#pragma unroll 1
    for (int e = lane; e < E; e += 32) sum += entity(e).cost;
    const uint32_t Tot = __reduce_add_sync(0xffffffffu, sum), chunk = sp_chunk(p, Tot);
    const uint32_t c = blockIdx.x;
    const bool writes = c == gridDim.x - 1;  // this CTA (with the least to do) leaves the plan for the merge kernel
    const uint32_t at = min(c * chunk, Tot), end = min(at + chunk, Tot);
    // the entity that position `at` lies in, with the costs and partial rows before it
    int e = E;
    uint32_t e_cost = 0, e_slot = 0, cost = 0, slot = 0;
#pragma unroll 1
    for (int e0 = 0; e0 < E && (e == E || writes); e0 += 32) {
      const int k = e0 + lane;
      SpEntity x{};
      if (k < E) x = entity(k);
      uint32_t ci = x.cost, si = x.cost ? x.slot_rows * x.pairs * x.units : 0u;
      const uint32_t mine = ci, rows = si;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, ci, o), v = __shfl_up_sync(0xffffffffu, si, o);
        if (lane >= o) {
          ci += u;
          si += v;
        }
      }
      const uint32_t before = cost + ci - mine, slots = slot + si - rows;
      const unsigned in = __ballot_sync(0xffffffffu, mine > 0 && before <= at && at < before + mine);
      if (in) {
        const int l = __ffs(in) - 1;
        e = e0 + l;
        e_cost = __shfl_sync(0xffffffffu, before, l);
        e_slot = __shfl_sync(0xffffffffu, slots, l);
      }
      if (writes && k < p.num_groups) {
        s_cost[k] = before;
        s_slot[k] = slots;
      }
      __syncwarp();
      if (writes && k >= p.num_groups && k < E) {
        SpRecord rec;
        const int g = group_of(k - p.num_groups);
        rec.cost = before;
        rec.slot = slots;
        rec.keys = x.keys;
        rec.chunk = chunk;
        rec.pre_cost = s_cost[g];
        rec.pre_slot = s_slot[g];
        rec.first = s_start[g];
        rec.sequences = s_start[g + 1] - rec.first;
        rec.pre_keys = rec.sequences > 0 ? s_len[g] : 0;
        p.plan[k - p.num_groups] = rec;
      }
      cost += __shfl_sync(0xffffffffu, ci, 31);
      slot += __shfl_sync(0xffffffffu, si, 31);
    }
    SpEntity x{};
    int h = 0, pair = 0;
    uint32_t base = 0;
    slot = 0;
    if (e < E) {
      x = entity(e);
      const uint32_t in = at - e_cost;
      h = static_cast<int>(sp_div(in, x.head_cost));
      pair = x.pairs > 1 ? static_cast<int>(sp_div(in - h * x.head_cost, x.length(1, x.key_tiles))) : 0;
      base = e_cost + h * x.head_cost + pair * x.length(1, x.key_tiles);
      slot = e_slot + (h * x.pairs + pair) * x.slot_rows + 2u * kSpTile * c;
    }
    const uint64_t again = l2_policy_evict_last();
    uint32_t published = 0, jobs[2] = {0, 0};
    int turn = 0;
    bool ok = true, more = true;
    auto wait = [&](uint32_t b, uint32_t parity) -> bool {
      int w = 1;
      if (lane == 0) w = mbar_wait_or_abort(b, parity, s_abort);
      return __shfl_sync(0xffffffffu, w, 0) != 0;
    };
    while (ok && more) {
      SpItem it;
      it.n = 0;
      while (it.n == 0 && e < E && base < end) {
        const bool own = e >= p.num_groups;
        const int dual = 2 * pair + 1 < x.tiles, duo = own && 2 * h + 1 < p.H_kv, key_tiles = x.key_tiles << duo;
        it.t0 = x.tile_at(at, base, dual, key_tiles);
        it.n = x.tile_at(end, base, dual, key_tiles) - it.t0;
        if (it.n > 0) {
          it.keys = x.keys;
          it.own = own;
          it.row = own ? e - p.num_groups : e;
          it.h = own ? 2 * h : h;
          it.dual = dual;
          it.duo = duo;
          it.again = x.pairs > 1;
          // Among a sequence's first keys lie those of rows that see few, and those that
          // may carry a row alone (attention sinks): there the roundings of the weights
          // do not average out.
          bool first_keys = true;
          if (own) {
            const int g = group_of(it.row);
            first_keys = s_start[g + 1] == s_start[g] || s_len[g] < kSpTile;
          }
          const int rows0 = sp_rows(p, x, 2 * pair), tok0 = x.token0 + 2 * pair * p.tokens_per_tile;
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            auto &j = it.s[s];
            j.token = tok0;
            j.rows = rows0;
            j.slot = slot;
            j.first = 0;
            j.step = 1;
            j.n = it.n;
            if (dual) {  // a row tile each
              if (s == 1) {
                j.token += p.tokens_per_tile;
                j.rows = sp_rows(p, x, 2 * pair + 1);
                j.slot += kSpTile;
              }
            } else if (duo) {  // a head each
              j.first = (it.t0 ^ s) & 1;
              j.step = 2;
              j.n = (it.n + 1 - j.first) >> 1;
              j.slot += s * rows0;
            } else if (it.n > 1) {  // even and odd key tiles
              j.first = s;
              j.step = 2;
              j.n = (it.n + 1 - s) >> 1;
            } else {  // one key tile: the streams in turn
              j.n = turn == s;
            }
            j.two = first_keys && (it.t0 + j.first) >> duo == 0;
          }
          if (!dual && !duo && it.n == 1) turn ^= 1;
        }
        // the next segment
        base += x.length(dual, key_tiles);
        slot += x.slot_rows;
        if (++pair == x.pairs) {
          pair = 0;
          if (++h == x.units) {
            h = 0;
#pragma unroll 1
            do x = ++e < E ? entity(e) : x;
            while (e < E && x.head_cost == 0);  // entities without keys or rows
          }
        }
      }
      more = it.n > 0;
      const uint32_t i = published % kSpItems;
      if (published >= kSpItems && !(ok = wait(bar(IEMPTY + i), (published / kSpItems - 1) & 1u))) break;
      if (lane == 0) {
        items[i] = it;
        mbar_arrive(bar(IFULL + i));
      }
      ++published;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (!more || !ok || it.s[s].n == 0) continue;
        if (jobs[s] > 0 && !(ok = wait(bar(QEMPTY + s), (jobs[s] - 1) & 1u))) continue;
        if (lane == 0) {
          mbar_arrive_expect_tx(bar(QFULL + s),
                                static_cast<uint32_t>((it.own ? p.n_q : p.tokens_per_tile) * p.group * D * 2));
          for (int hf = 0; hf < HALVES; ++hf)
            tma_load_4d(ring + L::kQOffset + s * L::kTileBytes + hf * kHalfTileBytes, it.own ? &tmap_q_own : &tmap_q_tile,
                        64 * hf, 0, it.h + (it.duo & s), it.s[s].token, bar(QFULL + s), again);
        }
        __syncwarp();
        ++jobs[s];
      }
    }
    if (*s_abort && lane == 0) {  // stopped: the copies in flight land (bounded) before shared memory is left
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (jobs[s]) (void)mbar_wait_bounded(bar(QFULL + s), (jobs[s] - 1) & 1u);
    }
    __syncwarp();
  } else if (warp == kSpCopyWarp) {
    // ------------------------------------------------------------------
    // K and V of the pieces' key tiles, one box a page
    // ------------------------------------------------------------------
    const uint64_t once = l2_policy_evict_first(), again = l2_policy_evict_last();
    uint32_t pos = 0;  // ring slots filled
    bool ok = true;
    // every lane gets the answer of lane 0's bounded wait
    auto wait = [&](uint32_t b, uint32_t parity) -> bool {
      int w = 1;
      if (lane == 0) w = mbar_wait_or_abort(b, parity, s_abort);
      return __shfl_sync(0xffffffffu, w, 0) != 0;
    };
    while (ok) {
      const SpItem *item = next_item();
      if (!item) break;
      const int n = item->n, t0 = item->t0, keys = item->keys, h = item->h, duo = item->duo;
      const int32_t *table = item->own ? p.block_table + static_cast<size_t>(item->row) * p.max_pages
                                       : p.prefix_table + static_cast<size_t>(item->row) * p.max_prefix_pages;
      const uint64_t policy = item->again ? again : once;
      release_item();
      int ids = kBeyondEnd;
      for (int it = 0; it < n; ++it) {
        if ((it & 3) == 0) {  // page ids of the next four tiles, one a lane
          const int lt = it + (lane >> 3), page = ((t0 + lt) >> duo) * kSpTilePages + (lane & 7);
          ids = lt < n && page * SF_PAGE_SIZE < keys ? table[page] : kBeyondEnd;
        }
        const int phys = __shfl_sync(0xffffffffu, ids, ((it & 3) << 3) + (lane & 7));
        int row = p.oob_row;  // pages past the end or outside the pool load as zeros
        if (phys != kBeyondEnd) {
          if (phys < 0 || phys >= p.num_pages) {
            if (lane < kSpTilePages) set_status(p.status, SF_DEVICE_BAD_PAGE);
          } else {
            row = (phys * p.H_kv + h + (duo & (t0 + it))) * SF_PAGE_SIZE;
          }
        }
        int rows[kSpTilePages];  // the same in every lane: the copies' operands are warp-uniform
#pragma unroll
        for (int j = 0; j < kSpTilePages; ++j) rows[j] = __shfl_sync(0xffffffffu, row, j);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv, ++pos) {
          const uint32_t slot = pos % STAGES;
          if (pos >= STAGES && !(ok = wait(bar(EMPTY + slot), (pos / STAGES - 1) & 1u))) break;
          const uint32_t dst = ring + slot * L::kTileBytes, full = bar(FULL + slot);
          if (elect_one()) {
            mbar_arrive_expect_tx(full, L::kTileBytes);
#pragma unroll
            for (int j = 0; j < kSpTilePages; ++j) {
              if (kv == 0) {
                if constexpr (HALVES == 2) tma_load_4d(dst + j * kPageBytes, &tmap_k, 0, 0, 0, rows[j] / 8, full, policy);
                else tma_load_2d(dst + j * kPageBytes, &tmap_k, 0, rows[j], full, policy);
              } else {
                if constexpr (HALVES == 2) tma_load_3d(dst + j * kPageBytes, &tmap_v, 0, rows[j], 0, full, policy);
                else tma_load_2d(dst + j * kPageBytes, &tmap_v, 0, rows[j], full, policy);
              }
            }
          }
          __syncwarp();
        }
        if (!ok) break;
      }
    }
    if (*s_abort && lane == 0) {
      for (uint32_t x = pos > STAGES ? pos - STAGES : 0; x < pos; ++x)
        (void)mbar_wait_bounded(bar(FULL + x % STAGES), (x / STAGES) & 1u);
    }
    __syncwarp();
  } else if (warp >= kSpMmaWarp) {
    // ------------------------------------------------------------------
    // MMAs of one stream, in order: Q K^T of a key tile (its K tile copied, and
    // Q for a job's first tile), then P V of its first and second 64 keys
    // (those weights written, V copied).  What the issuing branch needs is made
    // warp-uniform outside of it.
    // Two row tiles of one piece take turns: a stream issues P V of a tile and
    // Q K^T of the next, then the other does.  Left to themselves both streams
    // fall into step (the tensor cores serve them alternately, so both finish
    // together) and the softmaxes run side by side while the tensor cores wait.
    // ------------------------------------------------------------------
    const int s = warp - kSpMmaWarp;
    const uint32_t ts = __shfl_sync(0xffffffffu, tmem, 0) + s * 128u, to = ts + 256u;
    const uint64_t q0 = smem_desc_sw128(ring + L::kQOffset + s * L::kTileBytes, 16, 1024);
    auto wait = [&](uint32_t b, uint32_t parity) -> bool {
      const bool w = mbar_wait_or_abort(b, parity, s_abort);
      return __all_sync(0xffffffffu, w);
    };
    uint32_t pos = 0, tiles = 0, jobs = 0, turns = 0;  // pos: ring slots passed
    bool ok = true;
    // one thread issues: Q K^T of a tile ..
    auto issue_qk = [&](uint64_t k0) {
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        tc_mma_ss(ts, q0 + (((kk >> 2) * kHalfTileBytes + (kk & 3) * 32) >> 4),
                  k0 + (((kk >> 2) * 1024 + (kk & 3) * 32) >> 4), kIdescQK, kk > 0 ? 1u : 0u);
      tc_commit(bar(SFULL + s));
    };
    // .. and P V of a part of a tile's keys (`more`: not the job's first tile)
    auto issue_pv = [&](uint64_t v0, int part, uint32_t more, bool two) {
#pragma unroll
      for (int j = part ? kSpFirstPages : 0; j < (part ? kSpTilePages : kSpFirstPages); ++j) {
        const uint64_t v = v0 + (j * kPageBytes >> 4);
        tc_mma_ts(to, ts + j * 8, v, kIdescPV, j == 0 ? more : 1u);
        if (two) tc_mma_ts(to, ts + 64 + j * 8, v, kIdescPV, 1u);
      }
    };
    // stream 1's i-th turn follows stream 0's, stream 0's next follows that
    auto take_turn = [&]() -> bool {
      const bool w = s == 0 ? (turns == 0 || wait(bar(TURN), (turns - 1) & 1u)) : wait(bar(TURN + 1), turns & 1u);
      ++turns;
      return w;
    };
    while (ok) {
      const SpItem *item = next_item();
      if (!item) break;
      const int total = __shfl_sync(0xffffffffu, item->n, 0), n = __shfl_sync(0xffffffffu, item->s[s].n, 0);
      const int step = __shfl_sync(0xffffffffu, item->s[s].step, 0);
      const bool dual = __shfl_sync(0xffffffffu, item->dual, 0) != 0;
      int mine = n > 0 ? __shfl_sync(0xffffffffu, item->s[s].first, 0) : total;  // the stream's next key tile
      bool two = __shfl_sync(0xffffffffu, item->s[s].two, 0) != 0;  // P_hi + P_lo on the segment's first key tile
      int left = n;
      bool ahead = false;  // the tile's Q K^T is issued already
      release_item();
      for (int t = 0; t < total; ++t, pos += 2) {
        uint32_t slot = pos % STAGES;
        if (!(ok = wait(bar(FULL + slot), (pos / STAGES) & 1u))) break;
        if (t != mine) {
          // The other stream's tile: this stream gives its slots back too.  Both
          // streams pass every tile, so neither is ever two rounds of the ring
          // from the copies, where the parity of a slot's barrier says nothing.
          const uint32_t slot_v = (pos + 1) % STAGES;
          if (lane == 0) mbar_arrive(bar(EMPTY + slot));
          if (!(ok = wait(bar(FULL + slot_v), ((pos + 1) / STAGES) & 1u))) break;
          if (lane == 0) mbar_arrive(bar(EMPTY + slot_v));
          continue;
        }
        const bool first = left == n, last = left == 1;
        mine += step;
        --left;
        if (first) {
          if (!(ok = wait(bar(QFULL + s), jobs & 1u))) break;
          ++jobs;
          if (dual && !(ok = take_turn())) break;
        }
        if (!ahead) {
          tc_fence_after_sync();
          const uint64_t k0 = smem_desc_sw128(ring + slot * L::kTileBytes, 16, kKSbo);
          if (elect_one()) {
            issue_qk(k0);
            tc_commit(bar(EMPTY + slot));
            if (last) tc_commit(bar(QEMPTY + s));
            if (dual) mbar_arrive(bar(TURN + 1 - s));
          }
          __syncwarp();
        }
        ahead = false;
        slot = (pos + 1) % STAGES;
        if (!(ok = wait(bar(FULL + slot), ((pos + 1) / STAGES) & 1u))) break;
        const uint64_t v0 = smem_desc_sw128(ring + slot * L::kTileBytes, kPageHalfBytes, 1024);
        const uint32_t more = first ? 0u : 1u;
        if (!(ok = wait(bar(PFULL + 2 * s), tiles & 1u))) break;
        if (dual && !(ok = take_turn())) break;
        tc_fence_after_sync();
        if (elect_one()) issue_pv(v0, 0, more, two);
        __syncwarp();
        // of two row tiles the next Q K^T goes along where its K tile is there
        const uint32_t slot_n = (pos + 2) % STAGES;
        if (dual && !last) ahead = mbar_test_wait(bar(FULL + slot_n), ((pos + 2) / STAGES) & 1u);
        ahead = __all_sync(0xffffffffu, ahead);
        const bool last_n = left == 1;
        const uint64_t kn = smem_desc_sw128(ring + slot_n * L::kTileBytes, 16, kKSbo);
        if (!(ok = wait(bar(PFULL + 2 * s + 1), tiles & 1u))) break;
        tc_fence_after_sync();
        if (elect_one()) {
          issue_pv(v0, 1, more, two);
          tc_commit(bar(EMPTY + slot));
          if (last) tc_commit(bar(ODONE + s));
          if (last && dual) mbar_arrive(bar(TURN + 1 - s));
          if (ahead) {
            issue_qk(kn);
            tc_commit(bar(EMPTY + slot_n));
            if (last_n) tc_commit(bar(QEMPTY + s));
            mbar_arrive(bar(TURN + 1 - s));
          }
        }
        __syncwarp();
        two = false;
        ++tiles;
      }
    }
    // every MMA issued has completed once this arrives
    if (elect_one()) tc_commit(bar(FIN + s));
    __syncwarp();
    (void)mbar_wait_bounded(bar(FIN + s), 0);
  } else {
    // ------------------------------------------------------------------
    // softmax and partial results: stream s = warpgroup, thread = query row
    // ------------------------------------------------------------------
    const int s = warp >> 2, r = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + s * 128 + lanes, to = tmem + 256 + s * 128 + lanes;
    auto wwait = [&](uint32_t b, uint32_t parity) -> bool {
      const bool w = mbar_wait_or_abort(b, parity, s_abort);
      return __all_sync(0xffffffffu, w);
    };
    uint32_t base = 0, tiles = 0, jobs = 0, joints = 0;
    bool ok = true;
    while (ok) {
      const SpItem *item = next_item();
      if (!item) break;
      const int n = item->s[s].n, step = item->s[s].step, rows = item->s[s].rows, keys = item->keys;
      const uint32_t slot0 = item->s[s].slot;
      const int duo = item->duo;
      const bool joint = !item->dual && !duo && item->n > 1;  // the other stream has a part of the same row tile
      bool two = item->s[s].two != 0;
      uint32_t ring_tile = base + item->s[s].first;
      int tile_pos = ((item->t0 + item->s[s].first) >> duo) * kSpTile;  // position of the tile's first key
      base += item->n;
      const bool valid = r < rows;
      int *info = s_info + kSpInfo * warp;
      if (lane == 0) {
        info[0] = item->own ? p.n_q - 1 : 0;  // draft rows that are masked for some rows
        info[1] = item->row;
        info[2] = item->h + (duo & s);
        info[3] = tile_pos - (joint ? s * kSpTile : 0);  // the piece's first key, and the one behind its last
        info[4] = joint ? (item->t0 + item->n) * kSpTile : tile_pos + n * kSpTile;
      }
      // last visible key of this row (rows past the tile's end see every key:
      // their scores are not used)
      const int lim = !valid ? 0x7fffff00 : item->own ? keys - p.n_q + r / p.group : keys - 1;
      release_item();
      if (n == 0) continue;
      float ref = -INFINITY, l_run = 0.f, off = 0.f;
      for (int k = 0; k < n; ++k, ++tiles, ring_tile += step, tile_pos += (step >> duo) * kSpTile) {
        if (!(ok = wwait(bar(SFULL + s), tiles & 1u))) break;
        tc_fence_after_sync();
        uint32_t sv[128];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t part[64];
          tmem_ld_32x32b_x64(ts + 64 * q, part);
#pragma unroll
          for (int i = 0; i < 64; ++i) sv[64 * q + i] = part[i];
        }
        // What must not meet a weight of 0 (0 * NaN) is taken out of V: the rows of the
        // last page past the end, which hold whatever the page holds (whole pages past
        // the end are zeros already), and infinities and NaN of draft rows that are
        // masked for the rows before them (spread_bad gives them to those that see
        // them; 3 % of the time for many rows, 4 % where all keys are own ones).  In
        // front of the weights' release, as V may come behind the scores.
        const int valid_keys = keys - tile_pos;
        auto clean_v = [&]() -> bool {
          if (valid_keys >= kSpTile + SF_MAX_QUERY_ROWS - 1) return true;
          // rows from .. behind - 1 of the tile: hidden draft rows, then those past the end
          const int from = max(valid_keys - info[0], 0), behind = min((valid_keys + SF_PAGE_SIZE - 1) / SF_PAGE_SIZE * SF_PAGE_SIZE, kSpTile);
          if (from >= behind) return true;
          const uint32_t pos = 2u * ring_tile + 1u, slot = pos % STAGES;
          if (!wwait(bar(FULL + slot), (pos / STAGES) & 1u)) return false;
          uint8_t *vt = smem + slot * L::kTileBytes;
#pragma unroll 1
          for (int idx = r; idx < (behind - from) * HALVES * 8; idx += 128) {
            // 16 bytes of a row (in the order that the copy's swizzle leaves)
            const int tok = from + idx / (HALVES * 8), rem = idx % (HALVES * 8);
            uint4 *at = reinterpret_cast<uint4 *>(vt + (tok / SF_PAGE_SIZE) * kPageBytes + (rem >> 3) * kPageHalfBytes +
                                                  (tok % SF_PAGE_SIZE) * kRowBytes + (rem & 7) * 16);
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            uint32_t out = 0u;
            if (tok < valid_keys) {
              v = *at;
              auto finite = [&](uint32_t w) -> uint32_t {
                const uint32_t m = __vcmpeq2(w & 0x7f807f80u, 0x7f807f80u);
                out |= m;
                return w & ~m;
              };
              v = make_uint4(finite(v.x), finite(v.y), finite(v.z), finite(v.w));
              if (out) s_bad[2 * s + (jobs & 1u)] = static_cast<int>(seen);
            }
            if (out || tok >= valid_keys) *at = v;
          }
          fence_proxy_async_smem();
          return true;
        };
        if (tile_pos + kSpTile - 1 > lim) {
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (tile_pos + i > lim) sv[i] = __float_as_uint(-INFINITY);
        }
        float mu = ref == -INFINITY ? 0.f : ref;
        float a0 = __uint_as_float(sv[0]), a1 = __uint_as_float(sv[1]), a2 = __uint_as_float(sv[2]),
              a3 = __uint_as_float(sv[3]);
#pragma unroll
        for (int i = 4; i < 124; i += 8) {
          a0 = sp_max3(a0, __uint_as_float(sv[i]), __uint_as_float(sv[i + 1]));
          a1 = sp_max3(a1, __uint_as_float(sv[i + 2]), __uint_as_float(sv[i + 3]));
          a2 = sp_max3(a2, __uint_as_float(sv[i + 4]), __uint_as_float(sv[i + 5]));
          a3 = sp_max3(a3, __uint_as_float(sv[i + 6]), __uint_as_float(sv[i + 7]));
        }
        a0 = sp_max3(a0, __uint_as_float(sv[124]), __uint_as_float(sv[125]));
        a1 = sp_max3(a1, __uint_as_float(sv[126]), __uint_as_float(sv[127]));
        const float raw = fmaxf(fmaxf(a0, a1), fmaxf(a2, a3)), mx = raw * p.scale_log2;
        float alpha = 1.f;
        if (mx > ref + kSpRescaleLog2) {
          if (ref != -INFINITY) alpha = exp2f(ref - mx);
          ref = mx;
        }
        if (__any_sync(0xffffffffu, alpha != 1.f)) {
          // O *= alpha: the P V before this tile's Q K^T has completed with it
#pragma unroll 1
          for (int ch = 0; ch < D / 16; ++ch) {
            uint32_t ov[16];
            tmem_ld_32x32b_x16(to + ch * 16, ov);
#pragma unroll
            for (int i = 0; i < 16; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * alpha);
            tmem_st_32x32b_x16(to + ch * 16, ov);
          }
        }
        mu = ref == -INFINITY ? 0.f : ref;
        const unsigned long long scale2 = sp_pair(p.scale_log2, p.scale_log2), mu2 = sp_pair(-mu, -mu);
        unsigned long long sum = 0ull;
        // The tile's weights, and with `rest` what their rounding left, as a second term,
        // to columns [64, 128): two loops, as the branch inside of one made the tiles
        // without it 5 % slower.
        auto put_weights = [&](auto rest) {
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int k0 = 32 * ch + 2 * i;
              float x0, x1;
              sp_unpair(sp_fma2(sp_pair(__uint_as_float(sv[k0]), __uint_as_float(sv[k0 + 1])), scale2, mu2), x0, x1);
              const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
              if constexpr (decltype(rest)::value) {
                sv[k0] = __float_as_uint(p0);
                sv[k0 + 1] = __float_as_uint(p1);
              }
              w[i] = pack_bf16x2(p0, p1);
              sum = sp_add2(sum, sp_pair(p0, p1));
            }
            tmem_st_32x32b_x16(ts + 16 * ch, w);
            if constexpr (decltype(rest)::value) {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int k0 = 32 * ch + 2 * i;
                w[i] = pack_bf16x2(__uint_as_float(sv[k0]) - __uint_as_float(w[i] << 16),
                                   __uint_as_float(sv[k0 + 1]) - __uint_as_float(w[i] & 0xffff0000u));
              }
              tmem_st_32x32b_x16(ts + 64 + 16 * ch, w);
            }
            if (ch == 1) {  // P V of the first 64 keys may begin
              if (!(ok = clean_v())) return;
              tmem_wait_st();
              tc_fence_before_sync();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar(PFULL + 2 * s));
            }
          }
        };
        if (two) put_weights(std::true_type());
        else put_weights(std::false_type());
        if (!ok) break;
        float sum0, sum1;
        sp_unpair(sum, sum0, sum1);
        l_run = l_run * alpha + (sum0 + sum1);
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(PFULL + 2 * s + 1));
        // what rounding made of the tile's largest weight, for the same score in the same steps
        const float most = fast_exp2(fmaf(raw, p.scale_log2, -mu));
        off = off * alpha + (two ? 0.f : __bfloat162float(__float2bfloat16_rn(most)) - most);
        two = false;
      }
      if (ok) ok = wwait(bar(ODONE + s), jobs & 1u);
      if (!ok) break;
      ++jobs;
      tc_fence_after_sync();
      // Where every visible score is NaN the sum is NaN and no maximum was found; -inf
      // would tell the joins that the row saw no key.
      if (ref == -INFINITY && l_run != 0.f) ref = 0.f;
      // One weight may be nearly all of the sum, and O has it as it was rounded.  So O is
      // divided by the sum with that rounding in it, l_run + off, and the unit of both is
      // moved so that the part counts with its unrounded sum, l_run 2^ref, as before.
      if (l_run > fabsf(off)) {
        const float rounded = l_run + off;
        ref += __log2f(__fdividef(l_run, rounded));  // (near 1: within 2^-21)
        l_run = rounded;
      }
      float4 *dst = reinterpret_cast<float4 *>(p.part_o + static_cast<size_t>(slot0) * D) + r;
      // spread_bad: the infinities and NaN that this row sees among the piece's draft
      // rows of V, added to its results of `columns` columns from `first` on.
      auto is_bad = [&](int stream) {
        return s_bad[2 * stream] == static_cast<int>(seen) || s_bad[2 * stream + 1] == static_cast<int>(seen);
      };
      auto spread_bad = [&](int first, int columns) {
        if (!valid) return;
        const int32_t *table = p.block_table + static_cast<size_t>(info[1]) * p.max_pages;
#pragma unroll 1
        for (int col = first; col < first + columns; ++col) {
          float f = 0.f;
#pragma unroll 1
          for (int pos = max(keys - info[0], info[3]); pos < min(keys, info[4]) && pos <= lim; ++pos) {
            const int page = table[pos / SF_PAGE_SIZE];
            if (page < 0 || page >= p.num_pages) continue;  // (zeros)
            const float v = __bfloat162float(
                p.v_cache[((static_cast<size_t>(page) * p.H_kv + info[2]) * SF_PAGE_SIZE + pos % SF_PAGE_SIZE) * D + col]);
            if (!isfinite(v)) f += v;
          }
          if (f != 0.f) reinterpret_cast<float *>(dst + static_cast<size_t>(col / 4) * rows)[col % 4] += f;
        }
      };
      if (!joint) {
#pragma unroll 1
        for (int ch = 0; ch < D / 32; ++ch) {
          uint32_t ov[32];
          tmem_ld_32x32b_x32(to + ch * 32, ov);
          if (valid) {
#pragma unroll
            for (int q4 = 0; q4 < 8; ++q4)
              dst[static_cast<size_t>(ch * 8 + q4) * rows] =
                  make_float4(__uint_as_float(ov[4 * q4]), __uint_as_float(ov[4 * q4 + 1]),
                              __uint_as_float(ov[4 * q4 + 2]), __uint_as_float(ov[4 * q4 + 3]));
          }
        }
        if (valid) p.part_ml[slot0 + r] = make_float2(ref, l_run);
        if (is_bad(s)) spread_bad(0, D);
      } else {
        // Both streams' accumulators of a row are in this thread's lane, and its
        // maximum and sum come through shared memory: each stream joins and writes
        // half of the columns, when both are done, and goes on when both have read.
        float2 *s_ml = reinterpret_cast<float2 *>(smem + L::kMlOffset);
        s_ml[s * kSpTile + r] = make_float2(ref, l_run);
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(JOINT + s));
        if (!(ok = wwait(bar(JOINT + 1 - s), joints & 1u))) break;
        tc_fence_after_sync();
        const float2 ml = s_ml[(1 - s) * kSpTile + r];
        const float top = fmaxf(ref, ml.x);
        const float w = ref == -INFINITY ? 0.f : fast_exp2(ref - top), wo = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - top);
        const uint32_t half = s * (D / 2), other = to + 128 - 256 * s;  // (O_0, O_1 are 128 columns apart)
#pragma unroll 1
        for (int ch = 0; ch < D / 32; ++ch) {
          uint32_t a[16], b[16];
          tmem_ld_32x32b_x16(to + half + ch * 16, a);
          tmem_ld_32x32b_x16(other + half + ch * 16, b);
          if (valid) {
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
              float v[4];
#pragma unroll
              for (int i = 0; i < 4; ++i)
                v[i] = __uint_as_float(a[4 * q4 + i]) * w + __uint_as_float(b[4 * q4 + i]) * wo;
              dst[static_cast<size_t>(half / 4 + ch * 4 + q4) * rows] = make_float4(v[0], v[1], v[2], v[3]);
            }
          }
        }
        if (valid && s == 0) p.part_ml[slot0 + r] = make_float2(top, l_run * w + ml.y * wo);
        if (is_bad(0) || is_bad(1)) spread_bad(s * (D / 2), D / 2);
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(READ + s));
        if (!(ok = wwait(bar(READ + 1 - s), joints & 1u))) break;
        ++joints;
      }
      tc_fence_before_sync();
    }
    tc_fence_before_sync();
  }

  __syncthreads();
  if (*s_abort && tid == 0) set_status(p.status, SF_DEVICE_TIMEOUT);
  if (warp == kSpMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, kSpTmemCols);
  }
}

// --------------------------------------------------------------------------
// The partials of every row, joined in piece order (deterministic):
//   M = max_q m_q,  L = sum_q l_q 2^(m_q - M),  O = sum_q 2^(m_q - M) O_q / L,
//   lse = (M + log2 L) ln 2.
// A block takes one sequence and KV head (or a part of its rows): two warps list
// where the partials of its rows lie -- the prefix's for the one or two row tiles
// its tokens are in, then the own segment's -- and its threads walk the lists,
// kSpJoinBatch partials in flight.  One item per output quad (row, 4 columns);
// consecutive threads take consecutive rows of one quad, as the partials lie.
// --------------------------------------------------------------------------
constexpr int kSpJoinBatch = 8;
constexpr int kSpMaxSms = 512;                // CTAs of the split kernel at most
constexpr int kSpListMax = 2 * kSpMaxSms;     // a partial per CTA from the prefix, one from the own segment

struct SpJoin {
  float M, L;
  float4 acc;
  // one batch: its weights relative to the new maximum
  __device__ __forceinline__ void add(const float2 (&ml)[kSpJoinBatch], const float4 (&o)[kSpJoinBatch]) {
    float top = M;
#pragma unroll
    for (int u = 0; u < kSpJoinBatch; ++u) top = fmaxf(top, ml[u].x);
    if (top == -INFINITY) return;  // no visible key so far
    const float a = fast_exp2(M - top);
    L *= a;
    acc.x *= a; acc.y *= a; acc.z *= a; acc.w *= a;
#pragma unroll
    for (int u = 0; u < kSpJoinBatch; ++u) {
      const float w = fast_exp2(ml[u].x - top);
      L += ml[u].y * w;
      acc.x += o[u].x * w; acc.y += o[u].y * w; acc.z += o[u].z * w; acc.w += o[u].w * w;
    }
    M = top;
  }
  // what the lanes at distance `lanes` have joined, too (both sides alike)
  __device__ __forceinline__ void add_lanes(int lanes) {
    const float m = __shfl_xor_sync(0xffffffffu, M, lanes), l = __shfl_xor_sync(0xffffffffu, L, lanes);
    const float x = __shfl_xor_sync(0xffffffffu, acc.x, lanes), y = __shfl_xor_sync(0xffffffffu, acc.y, lanes);
    const float z = __shfl_xor_sync(0xffffffffu, acc.z, lanes), w = __shfl_xor_sync(0xffffffffu, acc.w, lanes);
    const float top = fmaxf(M, m);
    if (top == -INFINITY) return;
    const float a = fast_exp2(M - top), b = fast_exp2(m - top);
    L = L * a + l * b;
    acc.x = acc.x * a + x * b;
    acc.y = acc.y * a + y * b;
    acc.z = acc.z * a + z * b;
    acc.w = acc.w * a + w * b;
    M = top;
  }
};

// Appends the first partial rows of a row tile's partials of one segment to
// list[n ..]; returns the new length.  A whole warp calls it.
__device__ __forceinline__ int sp_list(uint32_t chunk, const SpParams &p, uint32_t cost, uint32_t slot, const SpEntity &x,
                                       bool own, int h, int tile, uint32_t *list, int n) {
  if (x.head_cost == 0) return n;
  const int lane = threadIdx.x & 31, pair = tile >> 1, dual = 2 * pair + 1 < x.tiles;
  const int duo = own && (h | 1) < p.H_kv, second = h & 1, unit = own ? h >> 1 : h, key_tiles = x.key_tiles << duo;
  const uint32_t base = cost + unit * x.head_cost + pair * x.length(1, x.key_tiles);
  slot += (unit * x.pairs + pair) * x.slot_rows + (dual ? (tile & 1) * kSpTile : duo ? second * x.tokens * p.group : 0);
  const int last = static_cast<int>(sp_div(base + x.length(dual, key_tiles) - 1, chunk));
  for (int c0 = static_cast<int>(sp_div(base, chunk)); c0 <= last; c0 += 32) {
    const int c = c0 + lane;
    // (a range's end may lie past the axis' end: no tile does)
    const int t0 = x.tile_at(c * chunk, base, dual, key_tiles);
    // (of a pair of heads: a tile of this one)
    const bool piece = c <= last && x.tile_at((c + 1) * chunk, base, dual, key_tiles) > t0 + (duo ? (t0 ^ second) & 1 : 0);
    const unsigned in = __ballot_sync(0xffffffffu, piece);
    if (piece) list[n + __popc(in & ((1u << lane) - 1u))] = slot + 2u * kSpTile * c;
    n += __popc(in);
  }
  return n;
}

// kWays threads an output quad, every kWays-th batch of its partials each.
template <int D, int kWays>
__global__ void __launch_bounds__(kSpMergeThreads) shared_prefix_merge_kernel(const __grid_constant__ SpParams p) {
  constexpr float kLn2 = 0.6931471805599453f;
  constexpr int C4 = D / 4;
  __shared__ uint32_t s_list[2][kSpListMax];
  __shared__ int s_pre[2], s_all[2], s_rows[2];  // list lengths (prefix, all) and rows of the prefix's row tiles
  const int tid = threadIdx.x, warp = tid >> 5;
  const int b = blockIdx.x / p.H_kv, h = blockIdx.x - b * p.H_kv;
  const int R = p.n_q * p.group, per = R * C4;
  grid_dependency_wait();
  grid_launch_dependents();
  const SpRecord rec = p.plan[b];
  int tok0 = 0, tile0 = 0;  // the sequence's first token within its group's, and that token's row tile
  if (rec.keys > 0) {
    tok0 = (b - rec.first) * p.n_q;
    tile0 = sp_tiles(p, tok0);
    if (warp < 2) {
      const int tile = tile0 + warp;
      int n = 0, rows = 0;
      if (rec.pre_keys > 0) {
        const SpEntity px = sp_entity(p, false, rec.first, rec.sequences, rec.pre_keys);
        if (tile < px.tiles) {
          n = sp_list(rec.chunk, p, rec.pre_cost, rec.pre_slot, px, false, h, tile, s_list[warp], 0);
          rows = sp_rows(p, px, tile);
        }
      }
      const int all = sp_list(rec.chunk, p, rec.cost, rec.slot, sp_entity(p, true, b, 1, rec.keys), true, h, 0, s_list[warp], n);
      s_pre[warp] = n;
      s_all[warp] = all;
      s_rows[warp] = rows;
    }
    __syncthreads();
  }
  constexpr int kItems = kSpMergeThreads / kWays, kLanes = 32 / kWays;  // quads of a block, and of a warp, at a time
  const int way = (tid & 31) / kLanes;
  for (int first = blockIdx.y * kItems; first < per; first += gridDim.y * kItems) {
    const int item = first + warp * kLanes + (tid & (kLanes - 1));
    const bool live = item < per;
    if (kWays == 1 && !live) break;
    const int c4 = item / R, r = item - c4 * R, i = r / p.group, j = r - i * p.group;
    const size_t row = (static_cast<size_t>(b) * p.n_q + i) * p.H_q + static_cast<size_t>(h) * p.group + j;
    SpJoin jn;
    jn.M = -INFINITY;
    jn.L = 0.f;
    jn.acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float inv = 0.f;
    if (rec.keys > 0) {
      const int sel = (tok0 + i >= (tile0 + 1) * p.tokens_per_tile);
      const int row_pre = (tok0 + i - (tile0 + sel) * p.tokens_per_tile) * p.group + j;
      const int pre = s_pre[sel], all = live ? s_all[sel] : 0, rows_pre = s_rows[sel];
      for (int k0 = way * kSpJoinBatch; k0 < all; k0 += kWays * kSpJoinBatch) {
        float2 ml[kSpJoinBatch];
        float4 o[kSpJoinBatch];
#pragma unroll
        for (int u = 0; u < kSpJoinBatch; ++u) {
          ml[u] = make_float2(-INFINITY, 0.f);
          o[u] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (k0 + u < all) {
            const bool in_pre = k0 + u < pre;
            const uint32_t at = s_list[sel][k0 + u];
            const int rr = in_pre ? row_pre : r, rows = in_pre ? rows_pre : R;
            ml[u] = p.part_ml[at + rr];
            o[u] = (reinterpret_cast<const float4 *>(p.part_o) + static_cast<size_t>(at) * C4 + rr)[static_cast<size_t>(c4) * rows];
          }
        }
        jn.add(ml, o);
      }
#pragma unroll
      for (int lanes = kLanes; lanes < 32; lanes *= 2) jn.add_lanes(lanes);
      inv = 1.f / jn.L;
    }
    if (kWays > 1 && (!live || way > 0)) continue;
    uint2 packed;
    packed.x = pack_bf16x2(jn.acc.x * inv, jn.acc.y * inv);
    packed.y = pack_bf16x2(jn.acc.z * inv, jn.acc.w * inv);
    *reinterpret_cast<uint2 *>(p.out + row * D + 4 * c4) = packed;
    if (p.lse && c4 == 0) p.lse[row] = rec.keys > 0 ? (jn.M + log2f(jn.L)) * kLn2 : -INFINITY;
  }
}

// --------------------------------------------------------------------------
// host side
// --------------------------------------------------------------------------
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
struct SpBounds {
  long long cost;  // length of the partition's axis
  long long rows;  // partial rows
};

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

struct SpLayout {
  size_t plan_off, ml_off, o_off, total;
};

static SpLayout sp_layout(const SpBounds &b, int D, int B) {
  SpLayout l;
  l.plan_off = 256;
  l.ml_off = round_up(l.plan_off + static_cast<size_t>(B) * sizeof(SpRecord), 256);
  l.o_off = round_up(l.ml_off + static_cast<size_t>(b.rows) * sizeof(float2), 256);
  l.total = l.o_off + static_cast<size_t>(b.rows) * D * sizeof(float);
  return l;
}

static int sp_grid(int *G) {
  DeviceInfo dev;
  const int st = current_device(&dev);
  if (st != SF_OK) return st;
  if (dev.max_smem_optin < kSpSmemMax)
    return fail(SF_ERR_UNSUPPORTED, "needs %d B shared memory, device allows %d", kSpSmemMax, dev.max_smem_optin);
  *G = dev.sm_count < kSpMaxSms ? dev.sm_count : kSpMaxSms;
  return SF_OK;
}

using SpKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const SpParams);

// The kernel with the deepest ring that leaves room for the plan of B sequences.
static void sp_select(int D, int B, int num_groups, SpKernel *fn, int *smem) {
  const int stages = sp_stages(D, B, num_groups);
  if (D == 128) {
    *fn = stages == 5 ? shared_prefix_split_kernel<128, 5> : shared_prefix_split_kernel<128, 4>;
    *smem = stages == 5 ? sp_smem_bytes<128, 5>(B, num_groups) : sp_smem_bytes<128, 4>(B, num_groups);
  } else {
    *fn = stages == 10 ? shared_prefix_split_kernel<64, 10> : shared_prefix_split_kernel<64, 8>;
    *smem = stages == 10 ? sp_smem_bytes<64, 10>(B, num_groups) : sp_smem_bytes<64, 8>(B, num_groups);
  }
}

static int sp_setup(int device) {
  static std::mutex mu;
  static bool done[64] = {};
  if (device < 0 || device >= 64) return fail(SF_ERR_UNSUPPORTED, "device ordinal %d", device);
  std::lock_guard<std::mutex> lock(mu);
  if (done[device]) return SF_OK;
  for (SpKernel fn : {static_cast<SpKernel>(shared_prefix_split_kernel<128, 5>),
                      static_cast<SpKernel>(shared_prefix_split_kernel<128, 4>),
                      static_cast<SpKernel>(shared_prefix_split_kernel<64, 10>),
                      static_cast<SpKernel>(shared_prefix_split_kernel<64, 8>)}) {
    const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kSpSmemMax);
    if (e != cudaSuccess) return fail(SF_ERR_CUDA, "cudaFuncSetAttribute (shared prefix): %s", cudaGetErrorString(e));
  }
  done[device] = true;
  return SF_OK;
}

// Tensor maps of one call: a page of K as [8-token group][half][8 tokens][128 B],
// a page of V as [half][16 tokens][128 B], 64 columns of a row tile of Q.
static int sp_maps(CUtensorMap (&m)[4], const void *k, const void *v, const void *q, uint64_t rows, int B, int n_q,
                   int H_q, int H_kv, int D, int tokens_per_tile) {
  int st;
  if (D == 128) {
    const uint64_t kd[4] = {64, 8, 2, rows / 8}, ks[3] = {256, 128, 2048};
    const uint32_t kb[4] = {64, 8, 2, 2};
    if ((st = encode_tensor_map_bf16(&m[0], k, 4, kd, ks, kb)) != SF_OK) return st;
    const uint64_t vd[3] = {64, rows, 2}, vs[2] = {256, 128};
    const uint32_t vb[3] = {64, SF_PAGE_SIZE, 2};
    if ((st = encode_tensor_map_bf16(&m[1], v, 3, vd, vs, vb)) != SF_OK) return st;
  } else {
    const uint64_t d[2] = {64, rows}, s[1] = {128};
    const uint32_t b[2] = {64, SF_PAGE_SIZE};
    if ((st = encode_tensor_map_bf16(&m[0], k, 2, d, s, b)) != SF_OK) return st;
    if ((st = encode_tensor_map_bf16(&m[1], v, 2, d, s, b)) != SF_OK) return st;
  }
  const uint64_t group = H_q / H_kv, e = 2ull * D;
  const uint64_t qd[4] = {(uint64_t)D, group, (uint64_t)H_kv, (uint64_t)B * n_q}, qs[3] = {e, group * e, H_q * e};
  const uint32_t qb[4] = {64, (uint32_t)group, 1, (uint32_t)tokens_per_tile};
  if ((st = encode_tensor_map_bf16(&m[2], q, 4, qd, qs, qb)) != SF_OK) return st;
  const uint32_t ob[4] = {64, (uint32_t)group, 1, (uint32_t)n_q};
  return encode_tensor_map_bf16(&m[3], q, 4, qd, qs, ob);
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
  if ((st = sp_setup(dev.ordinal)) != SF_OK) return st;

  const uint64_t rows = (uint64_t)num_pages * H_kv * SF_PAGE_SIZE;
  SpParams p;
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

  SpKernel fn;
  int smem;
  sp_select(head_dim, B, num_groups, &fn, &smem);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(G);
  cfg.blockDim = dim3(kSpThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, fn, m[0], m[1], m[2], m[3], p);
  if (e != cudaSuccess) return fail(SF_ERR_CUDA, "shared-prefix attention launch: %s", cudaGetErrorString(e));
  // one block per sequence and KV head, its rows over several where that leaves
  // SMs without one
  // and, where its rows may have more than two batches of partials and four threads an
  // output quad still leave SMs without a second block, each list over four threads
  // (one sequence of 6 rows, 4 KV heads of 64, 14000 tokens, 38 partials a row: 18.7 ->
  // 15.5 us; with at most 8 partials 10.9 -> 11.9, with more blocks, as for 8 sequences of
  // 5 rows and 32 heads, 24.8 -> 27.7).
  const int quads = n_q * p.group * (head_dim / 4);
  auto partials = [&](int pages, int segments) { return std::min((pages + kSpTilePages - 1) / kSpTilePages, G / segments + 1); };
  const bool wide = std::max(partials(max_prefix_pages, num_groups * H_kv), partials(max_pages_per_seq, B * H_kv)) >
                        2 * kSpJoinBatch &&
                    static_cast<long long>(B) * H_kv * ((quads * 4 + kSpMergeThreads - 1) / kSpMergeThreads) <= 2 * G;
  const int per = ((wide ? 4 : 1) * quads + kSpMergeThreads - 1) / kSpMergeThreads;
  int parts = (4 * G + B * H_kv - 1) / (B * H_kv);
  if (parts > per) parts = per;
  cfg.gridDim = dim3(static_cast<unsigned>(B * H_kv), static_cast<unsigned>(parts));
  cfg.blockDim = dim3(kSpMergeThreads);
  cfg.dynamicSmemBytes = 0;
  e = head_dim == 128 ? (wide ? cudaLaunchKernelEx(&cfg, shared_prefix_merge_kernel<128, 4>, p)
                              : cudaLaunchKernelEx(&cfg, shared_prefix_merge_kernel<128, 1>, p))
                      : (wide ? cudaLaunchKernelEx(&cfg, shared_prefix_merge_kernel<64, 4>, p)
                              : cudaLaunchKernelEx(&cfg, shared_prefix_merge_kernel<64, 1>, p));
  if (e != cudaSuccess) return fail(SF_ERR_CUDA, "shared-prefix merge launch: %s", cudaGetErrorString(e));
  return SF_OK;
}

}  // extern "C"
