// attention_mass.cu -- the attention weight that each cached key got, on the
// 5th-generation tensor cores.
//
//   out[b][h][t] = in[b][h][t] + sum_i w_i sum_j exp(scale <q_ij, k_t> - lse_ij)
//
// over the query rows i of sequence b, with weight w_i, and the query heads j of KV
// head h, for the L_b = seq_lens[b] - n_q keys of the context.
//
// The product is taken the other way round than in attention: keys are the M = 128
// side (S^T = K Q^T), so a thread that reads one TMEM lane has all rows' scores of one
// key and adds up their weights by itself; nothing crosses threads, and sums have one
// order.  The row's constant -lse log2(e) + log2(w) is one number per column, which
// makes a score one fused multiply-add and one exp2; the type's lowest value for rows that
// do not count (their q, which may hold anything, is zeroed in shared memory).  Zero times an
// infinite key is NaN all the same: where a chunk of columns makes a key's sum NaN it is added
// up again without those rows (looking for that takes 0.1 us of 8, 0.3 of 78).
//
// The key tiles (128 keys) of all (sequence, KV head) segments lie on one axis, cut
// into equal ranges, one per CTA.  Warps 0-7 are two groups of 128 summing threads
// that take the CTA's tiles in turn; warp 8 issues the MMAs, warp 9 copies K (a ring),
// warp 10 brings a segment's rows of q and its constants.  A group has two TMEM
// buffers of up to 128 columns: with more rows than that a tile's columns come in
// chunks, the next chunk's MMAs running while one is summed.
//
// What bounds it.  Up to some 128 rows K's way from memory (4 sequences of 32768 tokens, 4
// heads: 24.7 us with 112 rows, 5.6 TB/s; 4 sequences of 3008 tokens, 32 heads, 16 rows:
// 19.0, 5.4).  Then the tile's chain: 224 rows 31.4 us, 4.4 TB/s (25 without the sums and
// the MMAs, 28 with the sums alone, 30 with the MMAs alone), 448 rows 70; the tensor pipe is
// active for 41 % of it, the exponentials take 42 % of their pipe.  5 rows, 3008 tokens, 32
// heads: 5.8 us in a graph for 25 MB; from memory, called from Python, 7.9.  Not kept: page
// ids loaded four tiles ahead (no change), one q buffer and five ring slots where two and
// three fit (33 us), all scores in registers in front of the sums (34.6), 32 columns at a
// time (33.9), one TMEM buffer of 256 columns a group (31.3, and 75 with 448 rows).
#include <cmath>
#include <mutex>

#include "attn_common.cuh"
#include "layer_device.cuh"
#include "sf_host.h"

namespace sf {

constexpr int kMassTile = 128;                  // keys per tile
constexpr int kMassTilePages = kMassTile / SF_PAGE_SIZE;
constexpr int kMassChunk = 128;                 // columns of a TMEM buffer
constexpr int kMassThreads = 352;
constexpr int kMassMmaWarp = 8, kMassCopyWarp = 9, kMassQueryWarp = 10;
constexpr int kMassMaxStages = 8;
constexpr int kMassMaxRegs = 168;  // three warps share a sub-partition's 16K registers
constexpr int kMassSmemMax = 227 * 1024;
constexpr uint32_t kMassTmemCols = 512;
constexpr float kMassNoRow = -3.402823466e+38f;  // constant of a row that does not count

struct MassParams {
  const float *lse, *mass, *weights;
  const int32_t *block_table, *seq_lens;
  float *out;
  uint32_t *status;
  int B, n_q, H_q, H_kv, group, num_pages, max_pages, width;
  int R, cols, chunk, chunks;  // rows, and the same in chunks of `chunk` columns
  int stages, q_bufs;          // K ring slots, q buffers
  int oob_row;
  float scale_log2;
};

// Shared memory: K ring | q buffers | constants [2][cols] | barriers | prefix of tiles [B + 1] | lengths [B]
struct MassLayout {
  int q_off, q_bytes, c_off, bar_off, misc_off, prefix_off, total;
};
__host__ __device__ inline MassLayout mass_layout(int D, int stages, int q_bufs, int cols, int B) {
  MassLayout l;
  l.q_off = stages * kMassTile * D * 2;
  l.q_bytes = cols * D * 2;
  l.c_off = l.q_off + q_bufs * l.q_bytes;
  l.bar_off = l.c_off + q_bufs * cols * 4;
  l.misc_off = l.bar_off + 8 * (2 * kMassMaxStages + 4 + 4 + 3 * 2 + 1);
  l.prefix_off = l.misc_off + 16;
  l.total = l.prefix_off + 4 * (2 * B + 1);
  return l;
}

// A CTA's tiles in order: tile `t` of segment (b, h); every role walks them alike.
struct MassWalk {
  int b, h, t, tiles, L;
  uint32_t left;
  const int *prefix, *lens;
  int H_kv;
  __device__ __forceinline__ void enter() {
    while (prefix[b + 1] == prefix[b]) ++b;  // sequences without keys (there is a later one with some)
    tiles = prefix[b + 1] - prefix[b];
    L = lens[b];
  }
  __device__ __forceinline__ void start(uint32_t from, uint32_t to, int B) {
    left = to - from;
    if (!left) return;
    int lo = 0, hi = B;  // the last sequence that begins at or before `from`
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (static_cast<uint32_t>(prefix[mid]) * static_cast<uint32_t>(H_kv) <= from) lo = mid; else hi = mid;
    }
    b = lo;
    enter();
    const uint32_t in = from - static_cast<uint32_t>(prefix[b]) * static_cast<uint32_t>(H_kv);
    h = static_cast<int>(in / static_cast<uint32_t>(tiles));
    t = static_cast<int>(in) - h * tiles;
  }
  // tiles of this segment from here on that the CTA has
  __device__ __forceinline__ int run() const {
    return left < static_cast<uint32_t>(tiles - t) ? static_cast<int>(left) : tiles - t;
  }
  __device__ __forceinline__ void skip(int n) {  // n <= run()
    left -= n;
    t += n;
    if (t == tiles && left) {
      t = 0;
      if (++h == H_kv) {
        h = 0;
        ++b;
        enter();
      }
    }
  }
};

template <int D>
__global__ void __maxnreg__(kMassMaxRegs)
attention_mass_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_q,
                      const __grid_constant__ MassParams p) {
  constexpr int HALVES = D / 64;
  constexpr int kPageBytes = SF_PAGE_SIZE * D * 2, kTileBytes = kMassTile * D * 2;
  constexpr uint32_t kKSbo = HALVES == 2 ? 2048u : 1024u;  // 8-key atoms of a K tile
  constexpr float kLog2e = 1.4426950408889634f;
  constexpr int FULL = 0, EMPTY = kMassMaxStages, SFULL = 2 * kMassMaxStages, SEMPTY = SFULL + 4, QCOPY = SEMPTY + 4,
                QFULL = QCOPY + 2, QEMPTY = QFULL + 2, FIN = QEMPTY + 2;
  extern __shared__ __align__(1024) uint8_t smem[];
  const MassLayout lay = mass_layout(D, p.stages, p.q_bufs, p.cols, p.B);
  const uint32_t ring = smem_addr(smem);
  auto bar = [&](int i) -> uint32_t { return ring + lay.bar_off + 8u * static_cast<uint32_t>(i); };
  int *s_misc = reinterpret_cast<int *>(smem + lay.misc_off);
  volatile int *s_abort = s_misc + 1;
  float *s_const = reinterpret_cast<float *>(smem + lay.c_off);
  int *s_prefix = reinterpret_cast<int *>(smem + lay.prefix_off), *s_len = s_prefix + p.B + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp_id();

  if (tid == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(bar(FULL + s), 1);
      mbar_init(bar(EMPTY + s), 1);
    }
    for (int s = 0; s < 4; ++s) {
      mbar_init(bar(SFULL + s), 1);
      mbar_init(bar(SEMPTY + s), 4);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar(QCOPY + s), 1);
      mbar_init(bar(QFULL + s), 1);
      mbar_init(bar(QEMPTY + s), 1 + 8);  // the MMAs, and the summing warps (which read the constants)
    }
    mbar_init(bar(FIN), 1);
    fence_mbar_init();
    prefetch_tensormap(&tmap_k);
    prefetch_tensormap(&tmap_q);
    s_misc[1] = 0;
  }
  // q rows that pad the last chunk are zeros
  for (int i = tid; i < p.q_bufs * HALVES * (p.cols - p.R) * 8; i += kMassThreads) {
    const int pad = (p.cols - p.R) * 8, part = i / pad, x = i - part * pad;
    reinterpret_cast<uint4 *>(smem + lay.q_off + (part / HALVES) * lay.q_bytes + (part % HALVES) * p.cols * 128 +
                              p.R * 128)[x] = make_uint4(0u, 0u, 0u, 0u);
  }
  fence_proxy_async_smem();
  grid_dependency_wait();
  grid_launch_dependents();
  if (warp == 0) {
    // lengths, and the tiles in front of every sequence
    int sum = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const int b = b0 + lane;
      int L = 0;
      if (b < p.B) {
        const int T = p.seq_lens[b];
        L = T - p.n_q;
        if (T == 0) L = 0;
        else if (L < 0 || T > p.max_pages * SF_PAGE_SIZE || L > p.width) {
          if (blockIdx.x == 0) set_status(p.status, SF_DEVICE_BAD_SEQLEN);
          L = max(0, min(L, min(p.width, p.max_pages * SF_PAGE_SIZE - p.n_q)));
        }
        s_len[b] = L;
      }
      int incl = (L + kMassTile - 1) / kMassTile;
      const int mine = incl;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (b < p.B) s_prefix[b] = sum + incl - mine;
      sum += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) s_prefix[p.B] = sum;
  } else if (warp == kMassMmaWarp) {
    tmem_alloc(smem_addr(s_misc), kMassTmemCols);
    tmem_relinquish_alloc_permit();
    tc_fence_before_sync();
  }
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = static_cast<uint32_t>(s_misc[0]);
  const uint32_t Tot = static_cast<uint32_t>(p.H_kv) * static_cast<uint32_t>(s_prefix[p.B]);
  const uint32_t G = gridDim.x, share = Tot / G, rest = Tot % G, c = blockIdx.x;
  const uint32_t from = c * share + min(c, rest), to = from + share + (c < rest ? 1u : 0u);
  MassWalk w;
  w.prefix = s_prefix;
  w.lens = s_len;
  w.H_kv = p.H_kv;
  w.start(from, to, p.B);

  if (warp == kMassQueryWarp) {
    // a segment's rows of q and its constants
    bool ok = true;
    uint32_t seg = 0;
    const uint64_t policy = l2_policy_evict_last();
    for (; w.left && ok; w.skip(w.run()), ++seg) {
      const uint32_t buf = seg % p.q_bufs, round = seg / p.q_bufs;
      if (round > 0 && !(ok = __all_sync(0xffffffffu, mbar_wait_or_abort(bar(QEMPTY + buf), (round - 1) & 1u, s_abort)))) break;
      const uint32_t q = ring + lay.q_off + buf * lay.q_bytes;
      if (lane == 0) {
        mbar_arrive_expect_tx(bar(QCOPY + buf), static_cast<uint32_t>(p.R * D * 2));
        for (int hf = 0; hf < HALVES; ++hf)
          tma_load_4d(q + hf * p.cols * 128, &tmap_q, 64 * hf, 0, w.h, w.b * p.n_q, bar(QCOPY + buf), policy);
      }
      __syncwarp();
      float *s_c = s_const + buf * p.cols;
      bool none = false;  // rows that do not count
      constexpr int kBatch = 8;
      for (int r0 = lane; r0 < p.cols; r0 += 32 * kBatch) {
        float lse[kBatch], weight[kBatch];  // all loads in front of their use
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int r = r0 + 32 * u, i = r / p.group, j = r - i * p.group;
          lse[u] = weight[u] = 0.f;
          if (r >= p.R) continue;
          const size_t row = static_cast<size_t>(w.b) * p.n_q + i;
          lse[u] = p.lse[row * p.H_q + w.h * p.group + j];
          weight[u] = p.weights ? p.weights[row] : 1.f;
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int r = r0 + 32 * u;
          if (r >= p.cols) continue;
          float k = kMassNoRow;
          if (r < p.R) {
            if (weight[u] > 0.f && lse[u] != -INFINITY) k = (weight[u] == 1.f ? 0.f : log2f(weight[u])) - lse[u] * kLog2e;
            else none = true;
          }
          s_c[r] = k;
        }
      }
      if (!(ok = __all_sync(0xffffffffu, mbar_wait_or_abort(bar(QCOPY + buf), round & 1u, s_abort)))) break;
      for (int r = lane; none && r < p.R; r += 32) {
        if (s_c[r] != kMassNoRow) continue;
        for (int hf = 0; hf < HALVES; ++hf)
          for (int x = 0; x < 8; ++x)
            reinterpret_cast<uint4 *>(smem + lay.q_off + buf * lay.q_bytes + (hf * p.cols + r) * 128)[x] =
                make_uint4(0u, 0u, 0u, 0u);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(QFULL + buf));
    }
    if (*s_abort && lane == 0) {  // a copy in flight lands (bounded) before shared memory is left
      if (seg > 0) (void)mbar_wait_bounded(bar(QCOPY + (seg - 1) % p.q_bufs), ((seg - 1) / p.q_bufs) & 1u);
      if (w.left) (void)mbar_wait_bounded(bar(QCOPY + seg % p.q_bufs), (seg / p.q_bufs) & 1u);
    }
    __syncwarp();
  } else if (warp == kMassCopyWarp) {
    const uint64_t once = l2_policy_evict_first();
    uint32_t pos = 0;
    bool ok = true;
    for (; w.left && ok; w.skip(w.run())) {
      const int n = w.run();
      const int32_t *table = p.block_table + static_cast<size_t>(w.b) * p.max_pages;
      int ids = kBeyondEnd;
      for (int it = 0; it < n; ++it, ++pos) {
        if ((it & 3) == 0) {  // page ids of the next four tiles, one a lane
          const int lt = it + (lane >> 3), page = (w.t + lt) * kMassTilePages + (lane & 7);
          ids = lt < n && page * SF_PAGE_SIZE < w.L ? table[page] : kBeyondEnd;
        }
        const int phys = __shfl_sync(0xffffffffu, ids, ((it & 3) << 3) + (lane & 7));
        int row = p.oob_row;  // pages past the end or outside the pool load as zeros
        if (phys != kBeyondEnd) {
          if (phys < 0 || phys >= p.num_pages) {
            if (lane < kMassTilePages) set_status(p.status, SF_DEVICE_BAD_PAGE);
          } else {
            row = (phys * p.H_kv + w.h) * SF_PAGE_SIZE;
          }
        }
        int rows[kMassTilePages];
#pragma unroll
        for (int j = 0; j < kMassTilePages; ++j) rows[j] = __shfl_sync(0xffffffffu, row, j);
        const uint32_t slot = pos % p.stages, round = pos / p.stages;
        int go = 1;
        if (round > 0 && lane == 0) go = mbar_wait_or_abort(bar(EMPTY + slot), (round - 1) & 1u, s_abort);
        if (!(ok = __shfl_sync(0xffffffffu, go, 0) != 0)) break;
        const uint32_t dst = ring + slot * kTileBytes, full = bar(FULL + slot);
        if (elect_one()) {
          mbar_arrive_expect_tx(full, kTileBytes);
#pragma unroll
          for (int j = 0; j < kMassTilePages; ++j) {
            if constexpr (HALVES == 2) tma_load_4d(dst + j * kPageBytes, &tmap_k, 0, 0, 0, rows[j] / 8, full, once);
            else tma_load_2d(dst + j * kPageBytes, &tmap_k, 0, rows[j], full, once);
          }
        }
        __syncwarp();
      }
      if (!ok) break;
    }
    if (*s_abort && lane == 0) {
      for (uint32_t x = pos > static_cast<uint32_t>(p.stages) ? pos - p.stages : 0; x < pos; ++x)
        (void)mbar_wait_bounded(bar(FULL + x % p.stages), (x / p.stages) & 1u);
    }
    __syncwarp();
  } else if (warp == kMassMmaWarp) {
    const uint32_t base = __shfl_sync(0xffffffffu, tmem, 0);
    const uint32_t idesc = idesc_bf16_f32(kMassTile, p.chunk, 0, 0);
    auto wait = [&](uint32_t b, uint32_t parity) -> bool {
      return __all_sync(0xffffffffu, mbar_wait_or_abort(b, parity, s_abort));
    };
    uint32_t pos = 0, seg = 0;
    uint32_t jobs0 = 0, jobs1 = 0;  // chunks issued for each group
    bool ok = true;
    for (; w.left && ok; w.skip(w.run()), ++seg) {
      const int n = w.run();
      const uint32_t buf = seg % p.q_bufs;
      if (!(ok = wait(bar(QFULL + buf), (seg / p.q_bufs) & 1u))) break;
      const uint64_t q0 = smem_desc_sw128(ring + lay.q_off + buf * lay.q_bytes, 16, 1024);
      const uint32_t half = static_cast<uint32_t>(p.cols * 128) >> 4, step = static_cast<uint32_t>(p.chunk * 128) >> 4;
      for (int it = 0; it < n && ok; ++it, ++pos) {
        const uint32_t slot = pos % p.stages, group = pos & 1u;
        if (!(ok = wait(bar(FULL + slot), (pos / p.stages) & 1u))) break;
        const uint64_t k0 = smem_desc_sw128(ring + slot * kTileBytes, 16, kKSbo);
        for (int ch = 0; ch < p.chunks; ++ch) {
          const uint32_t job = group ? jobs1 : jobs0, s = group * 2u + (job & 1u);
          if (job >= 2 && !(ok = wait(bar(SEMPTY + s), ((job >> 1) - 1) & 1u))) break;
          tc_fence_after_sync();
          const uint64_t qc = q0 + static_cast<uint64_t>(ch * step);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              tc_mma_ss(base + s * kMassChunk, k0 + (((kk >> 2) * 1024 + (kk & 3) * 32) >> 4),
                        qc + static_cast<uint64_t>((kk >> 2) * half) + ((kk & 3) * 32 >> 4), idesc, kk > 0 ? 1u : 0u);
            tc_commit(bar(SFULL + s));
            if (ch + 1 == p.chunks) {
              tc_commit(bar(EMPTY + slot));
              if (it + 1 == n) tc_commit(bar(QEMPTY + buf));
            }
          }
          __syncwarp();
          if (group) ++jobs1; else ++jobs0;
        }
      }
    }
    // every MMA issued has completed once this arrives
    if (elect_one()) tc_commit(bar(FIN));
    __syncwarp();
    (void)mbar_wait_bounded(bar(FIN), 0);
  } else {
    const uint32_t group = warp >> 2;
    const int r = tid & 127;
    const uint32_t ts = tmem + group * 2u * kMassChunk + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    auto wait = [&](uint32_t b, uint32_t parity) -> bool {
      return __all_sync(0xffffffffu, mbar_wait_or_abort(b, parity, s_abort));
    };
    const unsigned long long scale2 = f32x2(p.scale_log2, p.scale_log2);
    uint32_t pos = 0, seg = 0, job = 0;
    bool ok = true;
    for (; w.left && ok; w.skip(w.run()), ++seg) {
      const int n = w.run();
      const uint32_t buf = seg % p.q_bufs;
      if (!(ok = wait(bar(QFULL + buf), (seg / p.q_bufs) & 1u))) break;
      const float *s_c = s_const + buf * p.cols;
      const size_t out0 = (static_cast<size_t>(w.b) * p.H_kv + w.h) * p.width;
      for (int it = 0; it < n && ok; ++it, ++pos) {
        if ((pos & 1u) != group) continue;
        const int key = (w.t + it) * kMassTile + r;
        float total = 0.f;
        if (p.mass && key < w.L) total = p.mass[out0 + key];
        unsigned long long sum0 = 0ull, sum1 = 0ull;
        for (int ch = 0; ch < p.chunks; ++ch, ++job) {
          const uint32_t s = group * 2u + (job & 1u);
          if (!(ok = wait(bar(SFULL + s), (job >> 1) & 1u))) break;
          tc_fence_after_sync();
          const float4 *c4 = reinterpret_cast<const float4 *>(s_c + ch * p.chunk);
          const uint32_t at = ts + (job & 1u) * kMassChunk;
          const unsigned long long before = f32x2_add(sum0, sum1);
          auto add = [&](const uint32_t (&v)[16], int first) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const float4 k = c4[(first + i) / 4];
              float x0, x1, x2, x3;
              f32x2_split(f32x2_fma(f32x2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), scale2, f32x2(k.x, k.y)), x0, x1);
              f32x2_split(f32x2_fma(f32x2(__uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])), scale2, f32x2(k.z, k.w)), x2, x3);
              sum0 = f32x2_add(sum0, f32x2(fast_exp2(x0), fast_exp2(x1)));
              sum1 = f32x2_add(sum1, f32x2(fast_exp2(x2), fast_exp2(x3)));
            }
          };
          // 16 columns on their way while 16 are summed
          uint32_t va[16], vb[16];
          tmem_ld_async_x16(at, va);
          tmem_ld_wait_x16(va);
          int first = 0;
          for (; first + 32 <= p.chunk; first += 32) {
            tmem_ld_async_x16(at + first + 16, vb);
            add(va, first);
            tmem_ld_wait_x16(vb);
            if (first + 32 < p.chunk) tmem_ld_async_x16(at + first + 32, va);
            add(vb, first + 16);
            if (first + 32 < p.chunk) tmem_ld_wait_x16(va);
          }
          if (first < p.chunk) add(va, first);
          float s0, s1;
          f32x2_split(f32x2_add(sum0, sum1), s0, s1);
          const bool again = key < w.L && isnan(s0 + s1);  // (no term is negative)
          if (__any_sync(0xffffffffu, again)) {  // an infinite key, or NaN
            float sum = 0.f;
#pragma unroll 1
            for (first = 0; first < p.chunk; first += 16) {
              tmem_ld_async_x16(at + first, va);
              tmem_ld_wait_x16(va);
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float k = s_c[ch * p.chunk + first + i];
                if (k != kMassNoRow) sum += fast_exp2(fmaf(__uint_as_float(va[i]), p.scale_log2, k));
              }
            }
            if (again) {
              sum0 = f32x2_add(before, f32x2(sum, 0.f));
              sum1 = 0ull;
            }
          }
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(SEMPTY + s));
        }
        if (!ok) break;
        float a, b;
        f32x2_split(f32x2_add(sum0, sum1), a, b);
        if (key < w.L) p.out[out0 + key] = total + (a + b);
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(QEMPTY + buf));
    }
    tc_fence_before_sync();
  }

  __syncthreads();
  if (*s_abort && tid == 0) set_status(p.status, SF_DEVICE_TIMEOUT);
  if (warp == kMassMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, kMassTmemCols);
  }
}

using MassKernel = void (*)(const CUtensorMap, const CUtensorMap, const MassParams);

static int mass_setup(int device) {
  static std::mutex mu;
  static bool done[64] = {};
  if (device < 0 || device >= 64) return fail(SF_ERR_UNSUPPORTED, "device ordinal %d", device);
  std::lock_guard<std::mutex> lock(mu);
  if (done[device]) return SF_OK;
  for (MassKernel fn : {static_cast<MassKernel>(attention_mass_kernel<128>), static_cast<MassKernel>(attention_mass_kernel<64>)}) {
    const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kMassSmemMax);
    if (e != cudaSuccess) return fail(SF_ERR_CUDA, "cudaFuncSetAttribute (attention mass): %s", cudaGetErrorString(e));
  }
  done[device] = true;
  return SF_OK;
}

// Chunks of equal width, the q buffers and the ring that shared memory has room for.
static int mass_plan(MassParams *p, int D, int *smem) {
  p->chunks = (p->R + kMassChunk - 1) / kMassChunk;
  p->chunk = ((p->R + p->chunks - 1) / p->chunks + 15) / 16 * 16;
  p->cols = p->chunk * p->chunks;
  // A second q buffer hides the change of segment, which is worth ring slots: 224 rows, 16
  // segments of 32768 keys 30.6 us with two buffers and three slots, 33.8 with one and five.
  for (p->q_bufs = 2; p->q_bufs >= 1; --p->q_bufs)
    for (p->stages = kMassMaxStages; p->stages >= (p->q_bufs == 2 ? 3 : 2); --p->stages) {
      *smem = mass_layout(D, p->stages, p->q_bufs, p->cols, p->B).total;
      if (*smem <= kMassSmemMax) return SF_OK;
    }
  return fail(SF_ERR_UNSUPPORTED, "%d rows per KV head", p->R);
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
  if ((long long)B * H_kv * ((long long)max_pages_per_seq / kMassTilePages + 1) >= (1LL << 31))
    return fail(SF_ERR_UNSUPPORTED, "%d sequences of up to %d pages with %d heads", B, max_pages_per_seq, H_kv);
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(lse, 4) || !aligned(block_table, 4) ||
      !aligned(seq_lens, 4) || !aligned(mass, 4) || !aligned(row_weights, 4) || !aligned(mass_out, 4))
    return fail(SF_ERR_INVALID_ARG, "q and k_cache must be 16-byte aligned, other arrays 4-byte aligned");
  if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale))
    return fail(SF_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0");
  if (!workspace || !aligned(workspace, 256))
    return fail(SF_ERR_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
  if (workspace_bytes < 256) return fail(SF_ERR_WORKSPACE, "workspace has %zu bytes, needs 256", workspace_bytes);
  DeviceInfo dev;
  int st = current_device(&dev);
  if (st != SF_OK || (st = mass_setup(dev.ordinal)) != SF_OK) return st;
  MassParams p;
  p.lse = lse;
  p.mass = mass;
  p.weights = row_weights;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.out = mass_out;
  p.status = static_cast<uint32_t *>(workspace);
  p.B = B;
  p.n_q = n_q;
  p.H_q = H_q;
  p.H_kv = H_kv;
  p.group = H_q / H_kv;
  p.R = n_q * p.group;
  p.num_pages = num_pages;
  p.max_pages = max_pages_per_seq;
  p.width = mass_width;
  p.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim)) * 1.4426950408889634f;
  int smem = 0;
  if ((st = mass_plan(&p, head_dim, &smem)) != SF_OK) return st;
  // K pages as [8-token group][half][8 tokens][128 B]; 64 columns of a segment's rows of q
  const uint64_t rows = (uint64_t)num_pages * H_kv * SF_PAGE_SIZE, group = p.group, e = 2ull * head_dim;
  p.oob_row = static_cast<int>(rows);
  CUtensorMap mk, mq;
  if (head_dim == 128) {
    const uint64_t kd[4] = {64, 8, 2, rows / 8}, ks[3] = {256, 128, 2048};
    const uint32_t kb[4] = {64, 8, 2, 2};
    st = encode_tensor_map_bf16(&mk, k_cache, 4, kd, ks, kb);
  } else {
    const uint64_t kd[2] = {64, rows}, ks[1] = {128};
    const uint32_t kb[2] = {64, SF_PAGE_SIZE};
    st = encode_tensor_map_bf16(&mk, k_cache, 2, kd, ks, kb);
  }
  if (st != SF_OK) return st;
  const uint64_t qd[4] = {(uint64_t)head_dim, group, (uint64_t)H_kv, (uint64_t)B * n_q}, qs[3] = {e, group * e, H_q * e};
  const uint32_t qb[4] = {64, (uint32_t)group, 1, (uint32_t)n_q};
  if ((st = encode_tensor_map_bf16(&mq, q, 4, qd, qs, qb)) != SF_OK) return st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(dev.sm_count);
  cfg.blockDim = dim3(kMassThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t err = head_dim == 128 ? cudaLaunchKernelEx(&cfg, attention_mass_kernel<128>, mk, mq, p)
                                          : cudaLaunchKernelEx(&cfg, attention_mass_kernel<64>, mk, mq, p);
  if (err != cudaSuccess) return fail(SF_ERR_CUDA, "attention mass launch: %s", cudaGetErrorString(err));
  return SF_OK;
}

}  // extern "C"
