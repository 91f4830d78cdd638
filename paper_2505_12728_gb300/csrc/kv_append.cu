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
// Bound by HBM for prompts (q, k and v are read once, written once) and by latency
// for a few draft rows.  A CTA takes up to kAppendRows rows: it computes their
// cosines and sines once for all heads and finds their cache places (one warp a
// row: a 32-ary search in row_starts), then its threads walk the heads, each with
// one 16-byte chunk of a head (and, for pairs (j, j + n), the chunk of the partners)
// in kBatch rows at a time.  A row's place is three loads that wait for each other:
// the first rows' elements and the positions are loaded in front of them.  35k rows
// of 28 + 8 bf16 heads of 128: 110 us, 5.9 TB/s (6 of them for the order of the stores
// and the next kernel; without that 117 us with the sines in the order of the pairs,
// four-way bank conflicts, and 148 with four rows at a time and three CTAs an SM).
// Few rows are spread over more CTAs by heads.  Tensors that 16-byte accesses
// cannot reach take kv_append_any_kernel, one pair of elements at a time (16000 rows
// of 28 + 8 heads of 128, 2 bytes off: 174 us, 52 on the boundary).
#include <cmath>

#include "sf_device.cuh"
#include "sf_host.h"

namespace sf {

constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 8;      // rows of a CTA at most, one per warp for their places
constexpr int kAppendResident = 4; // CTAs of an SM
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
  int late;  // the next kernel on the stream starts behind the stores, not beside them
  float amplitude;
};

// The fraction of a turn per position of pair j, and the axis of its positions.
__device__ __forceinline__ unsigned long long pair_step(const AppendParams &p, int j, int &axis) {
  axis = p.freq_axis ? p.freq_axis[j] : 0;
  if (axis < 0 || axis >= p.axes) {
    set_status(p.status, SF_DEVICE_BAD_INDEX);
    axis = 0;
  }
  double turns = p.inv_freq[j] * 0.15915494309189535;  // 1 / (2 pi)
  turns -= floor(turns);
  return __double2ull_rn(turns * 18446744073709551616.0);
}

// cos and sin (times the amplitude) at a position
__device__ __forceinline__ float2 pair_turn(const AppendParams &p, unsigned long long step, int position) {
  const int hi = static_cast<int>(static_cast<unsigned long long>(static_cast<long long>(position)) * step >> 32);
  float s, c;
  sincospif(static_cast<float>(hi) * 4.656612873077393e-10f, &s, &c);  // 2^-31: half turns
  return make_float2(c * p.amplitude, s * p.amplitude);
}

// Lets the next kernel on the stream start once all stores of the grid can be read by
// it, also by bulk copies that it issues before it waits for this one.  All threads of
// the block call it, behind their stores.  (A block stays until its stores have arrived:
// 35k rows 104 -> 110 us.)
__device__ __forceinline__ void launch_dependents_after_stores() {
  asm volatile("fence.proxy.async.global;" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    grid_launch_dependents();
  }
}

// The cache row (page * H_kv * 16 + slot; head h adds h * 16) of row t, or -1
// where the row is not appended.  A whole warp calls it.
__device__ __forceinline__ long long row_place(const AppendParams &p, int t) {
  const int lane = threadIdx.x & 31;
  int b, i, n;
  if (p.row_starts) {
    // the last sequence that starts at or before t: starts[b] <= t, by 32nds
    int lo = 0, width = p.B + 1;  // candidates lo .. lo + width - 1
    while (width > 1) {
      const int step = (width + 31) >> 5, k = lo + lane * step;
      const unsigned le = __ballot_sync(0xffffffffu, lane * step < width && p.row_starts[k < p.B ? k : p.B] <= t);
      if (!(le & 1u)) break;  // (row_starts[0] > t, or not ascending)
      const int hit = 31 - __clz(le);
      width = min(step, width - hit * step);
      lo += hit * step;
    }
    b = lo;
    const int first = p.row_starts[b], end = b < p.B ? p.row_starts[b + 1] : first;
    if (b == p.B) return -1;  // padding
    if (t < first || t >= end) {
      if (lane == 0) set_status(p.status, SF_DEVICE_BAD_INDEX);
      return -1;
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
    if (lane == 0) set_status(p.status, SF_DEVICE_BAD_SEQLEN);
    return -1;
  }
  const int page = p.block_table[static_cast<size_t>(b) * p.max_pages + at / SF_PAGE_SIZE];
  if (page < 0 || page >= p.num_pages) {
    if (lane == 0) set_status(p.status, SF_DEVICE_BAD_PAGE);
    return -1;
  }
  return static_cast<long long>(page) * p.H_kv * SF_PAGE_SIZE + at % SF_PAGE_SIZE;
}

__device__ __forceinline__ float load_as_float(const void *p, long long i, int wide) {
  return wide ? static_cast<const float *>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

// 8 neighbouring elements as they lie in memory, as fp32, and back as bf16
template <bool kWide>
struct Chunk {
  uint4 v[kWide ? 2 : 1];
  __device__ __forceinline__ void load(const void *base, long long at) {
    const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const char *>(base) + at * (kWide ? 4 : 2));
    v[0] = src[0];
    if constexpr (kWide) v[1] = src[1];
  }
  __device__ __forceinline__ void floats(float (&f)[8]) const {
    if constexpr (kWide) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f[4 * i] = __uint_as_float(v[i].x);
        f[4 * i + 1] = __uint_as_float(v[i].y);
        f[4 * i + 2] = __uint_as_float(v[i].z);
        f[4 * i + 3] = __uint_as_float(v[i].w);
      }
    } else {
      const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
};

__device__ __forceinline__ void store8(__nv_bfloat16 *dst, const float (&v)[8]) {
  *reinterpret_cast<uint4 *>(dst) =
      make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

// `rows` rows per CTA; blockIdx.y of gridDim.y takes every gridDim.y-th pass over
// the heads.  With few heads, row_groups groups of threads take the rows in turn
// (15000 rows of 12 + 3 bf16 heads of 128: 35 -> 30 us).
template <bool kWide, bool kInterleaved>
__global__ void __launch_bounds__(kAppendThreads, kAppendResident) kv_append_kernel(const __grid_constant__ AppendParams p, int rows, int row_groups) {
  // a row's cosines and sines, two pairs of every chunk in turn: the chunks' threads
  // read 16 neighbouring bytes each
  __shared__ float4 s_turn[kAppendRows][kMaxHeadDim / 4];
  __shared__ long long s_place[kAppendRows];
  const int tid = threadIdx.x, warp = tid >> 5;
  const int t0 = blockIdx.x * rows, nr = min(rows, p.T - t0);
  grid_dependency_wait();
  if (!p.late) grid_launch_dependents();
  // units of a head: its rotated chunks (or pairs of chunks), then the others.  A
  // thread has one unit of a head and takes the CTA's rows kBatch at a time, all their
  // loads in flight: 64 bytes (16000 rows of 36 interleaved bf16 heads: 60 us with 32).
  constexpr int kBatch = (kWide ? 1 : 2) * (kInterleaved ? 2 : 1);
  const int turned = kInterleaved ? p.pairs / 4 : p.pairs / 8, rest = (p.D - 2 * p.pairs) / 8, units = turned + rest;
  const int u = tid % units, lane_head = tid / units, heads_at_once = kAppendThreads / units;
  const bool turn = u < turned, both = turn && !kInterleaved;
  const int at = turn ? 8 * u : 2 * p.pairs + (u - turned) * 8;
  Chunk<kWide> a[kBatch], b[kBatch];
  auto load = [&](int h, int r0) {
    const bool is_q = h < p.H_q;
    const long long row = is_q ? p.q_row : p.k_row;
    const long long first = (is_q ? h * p.q_head : (h - p.H_q) * p.k_head) + (t0 + r0) * row + at;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (r0 + i >= nr) continue;
      a[i].load(is_q ? p.q : p.k, first + i * row);
      if (both) b[i].load(is_q ? p.q : p.k, first + i * row + p.pairs);
    }
  };
  // The places are three loads that wait for each other; the first rows' elements and
  // the positions are on their way meanwhile.
  const int heads = p.H_q + p.H_kv;
  int h = lane_head + static_cast<int>(blockIdx.y) * heads_at_once, r_start = 0;
  if (row_groups > 1) {
    r_start = lane_head / heads * kBatch;
    h = r_start < row_groups * kBatch ? lane_head % heads : heads;
  }
  if (lane_head >= heads_at_once) h = heads;
  const int h_first = h;
  if (h < heads) load(h, r_start);
  constexpr int kTurns = kAppendRows * (kMaxHeadDim / 2) / kAppendThreads;  // positions of a thread at most
  const int j = p.pairs > 0 ? tid % p.pairs : 0, each = p.pairs > 0 ? kAppendThreads / p.pairs : 0;
  const int r_first = p.pairs > 0 && tid < each * p.pairs ? tid / p.pairs : nr;
  int position[kTurns];
  unsigned long long step_j = 0;
  if (r_first < nr) {
    int axis;
    step_j = pair_step(p, j, axis);
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
      if (r_first + i * each < nr) position[i] = p.positions[static_cast<size_t>(axis) * p.T + t0 + r_first + i * each];
  }
  // (the last warps first: of a few rows the first warps take the angles)
  const int r_place = kAppendThreads / 32 - 1 - warp;
  if (r_place < nr) {
    const long long place = row_place(p, t0 + r_place);
    if ((tid & 31) == 0) s_place[r_place] = place;
  }
#pragma unroll
  for (int i = 0; i < kTurns; ++i)
    if (r_first + i * each < nr) {
      constexpr int kPairs = kInterleaved ? 4 : 8;  // of a chunk
      reinterpret_cast<float2 *>(s_turn[r_first + i * each])[(j % kPairs / 2 * turned + j / kPairs) * 2 + j % 2] =
          pair_turn(p, step_j, position[i]);
    }
  __syncthreads();
  for (; h < heads; h += heads_at_once * gridDim.y) {
    const bool is_q = h < p.H_q;
    const int hk = h - p.H_q;
    for (int r0 = r_start; r0 < nr; r0 += row_groups * kBatch) {
      if (r0 > r_start || h > h_first) load(h, r0);  // (the first is there)
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int r = r0 + i;
        if (r >= nr) continue;
        const long long place = s_place[r];
        if (!is_q && place < 0) continue;
        __nv_bfloat16 *dst = is_q ? p.q_out + (static_cast<size_t>(t0 + r) * p.H_q + h) * p.D
                                  : p.k_cache + static_cast<size_t>(place + hk * SF_PAGE_SIZE) * p.D;
        float x[8], y[8];
        a[i].floats(x);
        if (turn) {
          const float4 *w = s_turn[r] + u;
          if constexpr (kInterleaved) {
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
              const float4 c = w[e / 4 * turned];
              const float x0 = x[e], x1 = x[e + 1], x2 = x[e + 2], x3 = x[e + 3];
              x[e] = x0 * c.x - x1 * c.y;
              x[e + 1] = x0 * c.y + x1 * c.x;
              x[e + 2] = x2 * c.z - x3 * c.w;
              x[e + 3] = x2 * c.w + x3 * c.z;
            }
          } else {
            b[i].floats(y);
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const float4 c = w[e / 2 * turned];
              const float x0 = x[e], y0 = y[e], x1 = x[e + 1], y1 = y[e + 1];
              x[e] = x0 * c.x - y0 * c.y;
              y[e] = x0 * c.y + y0 * c.x;
              x[e + 1] = x1 * c.z - y1 * c.w;
              y[e + 1] = x1 * c.w + y1 * c.z;
            }
            store8(dst + at + p.pairs, y);
          }
        }
        store8(dst + at, x);
      }
    }
  }
  // values
  const int chunks = p.D / 8, per_row = p.H_kv * chunks, step = kAppendThreads * gridDim.y;
  for (int x0 = tid + blockIdx.y * kAppendThreads; x0 < nr * per_row; x0 += kBatch * step) {
    Chunk<kWide> a[kBatch];
    long long dst[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int x = x0 + i * step;
      dst[i] = -1;
      if (x >= nr * per_row) continue;
      const int r = x / per_row, c = x - r * per_row, h = c / chunks, e = (c - h * chunks) * 8;
      const long long place = s_place[r];
      if (place < 0) continue;
      dst[i] = (place + h * SF_PAGE_SIZE) * p.D + e;
      a[i].load(p.v, (t0 + r) * p.v_row + h * p.v_head + e);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (dst[i] < 0) continue;
      if constexpr (kWide) {
        float f[8];
        a[i].floats(f);
        store8(p.v_cache + dst[i], f);
      } else {
        *reinterpret_cast<uint4 *>(p.v_cache + dst[i]) = a[i].v[0];
      }
    }
  }
  if (p.late) launch_dependents_after_stores();
}

// The same for any alignment, strides and number of pairs: one row per CTA, one
// pair or element per thread.
__global__ void __launch_bounds__(kAppendThreads) kv_append_any_kernel(const __grid_constant__ AppendParams p) {
  __shared__ float2 s_turn[kMaxHeadDim / 2];
  __shared__ long long s_place;
  const int tid = threadIdx.x, t = blockIdx.x;
  grid_dependency_wait();
  if (!p.late) grid_launch_dependents();
  for (int j = tid; j < p.pairs; j += kAppendThreads) {
    int axis;
    const unsigned long long step = pair_step(p, j, axis);
    s_turn[j] = pair_turn(p, step, p.positions[static_cast<size_t>(axis) * p.T + t]);
  }
  if (tid >= kAppendThreads - 32) {
    const long long place = row_place(p, t);
    if (tid == kAppendThreads - 1) s_place = place;
  }
  __syncthreads();
  const long long place = s_place;
  // A thread keeps its item of a head (a pair, or an element that is not turned) over
  // the heads: one division for all of them.
  const int per = p.D - p.pairs, at_once = kAppendThreads / per, e = tid % per;
  const bool turn = e < p.pairs;
  const int i0 = !turn ? e + p.pairs : p.interleaved ? 2 * e : e, i1 = p.interleaved ? 2 * e + 1 : e + p.pairs;
  const float2 w = turn ? s_turn[e] : make_float2(1.f, 0.f);
  const int heads = tid < at_once * per ? p.H_q + (place >= 0 ? p.H_kv : 0) : 0;
#pragma unroll 2
  for (int h = tid / per; h < heads; h += at_once) {
    const bool is_q = h < p.H_q;
    const void *src = is_q ? p.q : p.k;
    const long long so = is_q ? t * p.q_row + h * p.q_head : t * p.k_row + (h - p.H_q) * p.k_head;
    __nv_bfloat16 *dst = is_q ? p.q_out + (static_cast<size_t>(t) * p.H_q + h) * p.D
                              : p.k_cache + static_cast<size_t>(place + (h - p.H_q) * SF_PAGE_SIZE) * p.D;
    const float a = load_as_float(src, so + i0, p.wide);
    if (turn) {
      const float b = load_as_float(src, so + i1, p.wide);
      dst[i0] = __float2bfloat16_rn(a * w.x - b * w.y);
      dst[i1] = __float2bfloat16_rn(a * w.y + b * w.x);
    } else {
      dst[i0] = __float2bfloat16_rn(a);
    }
  }
  const int v_at_once = kAppendThreads / p.D, i = tid % p.D;
  const int v_heads = place >= 0 && tid < v_at_once * p.D ? p.H_kv : 0;
  for (int h = tid / p.D; h < v_heads; h += v_at_once)
    p.v_cache[static_cast<size_t>(place + h * SF_PAGE_SIZE) * p.D + i] =
        __float2bfloat16_rn(load_as_float(p.v, t * p.v_row + h * p.v_head + i, p.wide));
  if (p.late) launch_dependents_after_stores();
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
  // sf_verify_attention copies the keys in front of its n_q draft rows before it waits for
  // this kernel, so it starts beside it only where all rows are such draft rows (late
  // always: append and attention 17.6 us a layer, 15.7 so, for 5 rows, 32 heads, 3008
  // tokens).
  p.late = row_starts != nullptr || p.rows > SF_MAX_QUERY_ROWS;
  p.amplitude = amplitude;
  DeviceInfo dev;
  const int st = current_device(&dev);
  if (st != SF_OK) return st;
  // 16-byte accesses: whole chunks of 8 rotated elements, strides of whole chunks
  const bool vec = p.pairs % (p.interleaved ? 4 : 8) == 0 && aligned(k, 16) && aligned(v, 16) && k_row_stride % 8 == 0 &&
                   k_head_stride % 8 == 0 && v_row_stride % 8 == 0 && v_head_stride % 8 == 0 &&
                   (H_q == 0 || (aligned(q, 16) && q_row_stride % 8 == 0 && q_head_stride % 8 == 0));
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kAppendThreads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t err;
  if (vec) {
    // Full waves of CTAs, with the fewest that kAppendRows allows (3250 rows of 16 + 4
    // fp32 heads of 64: 7.2 us with one wave of 6 rows, 9.7 with 2.7 waves of 2); few
    // rows are cut by heads.
    const long long wave = static_cast<long long>(kAppendResident) * dev.sm_count;
    const long long ctas = wave * ((T + wave * kAppendRows - 1) / (wave * kAppendRows));
    const int rows = static_cast<int>((T + ctas - 1) / ctas);
    const int grid = (T - 1) / rows + 1;
    const int passes = ((H_q + H_kv) * (head_dim / 8) + kAppendThreads - 1) / kAppendThreads;
    const int per_head = head_dim / 8 - (p.interleaved ? 0 : p.pairs / 8), at_once = kAppendThreads / per_head;
    const int row_groups = H_q + H_kv < at_once && rows > 1 ? at_once / (H_q + H_kv) : 1;
    int parts = dev.sm_count / grid;
    parts = parts < 1 ? 1 : parts > passes ? passes : parts;
    cfg.gridDim = dim3(grid, parts);
    if (p.wide)
      err = p.interleaved ? cudaLaunchKernelEx(&cfg, kv_append_kernel<true, true>, p, rows, row_groups)
                          : cudaLaunchKernelEx(&cfg, kv_append_kernel<true, false>, p, rows, row_groups);
    else
      err = p.interleaved ? cudaLaunchKernelEx(&cfg, kv_append_kernel<false, true>, p, rows, row_groups)
                          : cudaLaunchKernelEx(&cfg, kv_append_kernel<false, false>, p, rows, row_groups);
  } else {
    cfg.gridDim = dim3(T);
    err = cudaLaunchKernelEx(&cfg, kv_append_any_kernel, p);
  }
  if (err != cudaSuccess) return fail(SF_ERR_CUDA, "kv append launch: %s", cudaGetErrorString(err));
  return SF_OK;
}

}  // extern "C"
