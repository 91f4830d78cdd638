// add_rms_norm.cu -- residual addition and root-mean-square norm of the rows
// between a decoder layer's projections, with bf16 or 8-bit output.
//
//     h = x + residual,  y = h * weight / sqrt(mean(h^2) + eps)
//
// Bound by HBM for many rows (x and the residual are read once, the new residual
// and the output written once) and by latency for few.  A row lives in the
// registers of one CTA: every thread holds 8 * kChunks of its h, as fp32, between
// the one reduction and the output.  For 8-bit output the reduction takes the
// maximum of |h * weight| along with the sum of squares (y is that times one
// positive factor), so that the scales need no pass of their own; a group of 128
// columns is 16 neighbouring threads.  CTAs stay for several rows, with the next
// row's loads in flight during the reduction of the present one.  Rows that start off
// 16-byte boundaries, but all tensors' alike (d odd, say), are cut at those
// boundaries instead of at the row's start, so that only a row's first and last chunk
// go element by element.  With a grid of a multiple of 8 CTAs, a CTA's rows all lie
// alike, and it keeps its weights in registers as it does for aligned rows.
//
// Slower: tensors whose rows do not lie alike go one element at a time (kNormSingle;
// 16384 x 3584 to bf16 183 us, 74 alike; to e4m3 with groups 311, 69), and rows of more
// chunks than registers hold with the next row load one row at a time, and the weights
// again for each (8192 x 8192 from fp32 139 us, 2 % above the copy rate; 4096 x 16384 from
// bf16 97, 22 % above).
#include <algorithm>
#include <cmath>
#include <mutex>

#include <cuda_fp8.h>

#include "sf_device.cuh"
#include "sf_host.h"

namespace sf {

constexpr int kNormMaxThreads = 1024;
constexpr int kNormMaxRows = 0x7fff0000;  // a row and a step of the grid fit an int
constexpr int kNormGroup = 128;       // columns per scale
constexpr float kE4m3Max = 448.f;     // largest finite e4m3 value
constexpr float kLeastScale = 1.17549435e-38f;  // 2^-126

struct NormParams {
  const void *x, *residual, *weight;
  void *residual_out, *out;
  float *scales;
  long long x_stride, residual_stride, residual_out_stride, out_stride;
  int T, d, groups;
  int weight_wide;
  int shift;  // kNormShifted: elements from x's last 16-byte boundary (of 8 elements) to x
  int margin;  // kNormShifted: rows that hold 7 elements
  float eps;
  float per_d;  // 1 / d
};

// How a thread's elements lie in a row: 8 neighbours, with every row on a 16-byte
// boundary; 8 neighbours between boundaries that are the same in all tensors; or a
// block's width apart, one element at a time.
constexpr int kNormVec = 0, kNormShifted = 1, kNormSingle = 2;
// 8 elements as they lie in memory
template <bool kWide>
struct NormChunk {
  uint4 v[kWide ? 2 : 1];
};

__device__ __forceinline__ float norm_elem(const NormChunk<false> &c, int i) {
  const uint32_t w = i < 2 ? c.v[0].x : i < 4 ? c.v[0].y : i < 6 ? c.v[0].z : c.v[0].w;
  return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
}
__device__ __forceinline__ float norm_elem(const NormChunk<true> &c, int i) {
  const uint4 &q = c.v[i >> 2];
  const int k = i & 3;
  return __uint_as_float(k == 0 ? q.x : k == 1 ? q.y : k == 2 ? q.z : q.w);
}

// Column of element (k, i) of a thread; `o`: elements from a 16-byte boundary to
// the row's start.
template <int kMode>
__device__ __forceinline__ int norm_column(int k, int i, int nt, int o) {
  if constexpr (kMode == kNormSingle) return (k * 8 + i) * nt + static_cast<int>(threadIdx.x);
  else return (k * nt + static_cast<int>(threadIdx.x)) * 8 + i - (kMode == kNormShifted ? o : 0);
}

// A row's first and last chunk between boundaries hold elements of the neighbouring
// rows, or of the space between, which are read and dropped.  `first`, `last`: rows
// before or behind which the tensor may have fewer than the 7 elements of a chunk.
template <bool kWide, int kMode>
__device__ __forceinline__ void norm_load(const void *base, long long row, bool first, bool last, int k, int nt, int d, int o,
                                          NormChunk<kWide> &c) {
  const int col = norm_column<kMode>(k, 0, nt, o);
  if constexpr (kMode != kNormSingle) {
    c.v[0] = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (kWide) c.v[1] = make_uint4(0u, 0u, 0u, 0u);
    if (col >= d) return;
    const bool whole = kMode == kNormVec || ((col >= 0 || !first) && (col + 8 <= d || !last));
    if (whole) {
      const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const char *>(base) + (row + col) * (kWide ? 4 : 2));
      c.v[0] = src[0];
      if constexpr (kWide) c.v[1] = src[1];
      return;
    }
  }
  if constexpr (kMode != kNormVec) {
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = norm_column<kMode>(k, i, nt, o);
      e[i] = 0u;
      if (at >= 0 && at < d)
        e[i] = kWide ? static_cast<const uint32_t *>(base)[row + at]
                     : static_cast<uint32_t>(static_cast<const uint16_t *>(base)[row + at]);
    }
    if constexpr (kWide) {
      c.v[0] = make_uint4(e[0], e[1], e[2], e[3]);
      c.v[1] = make_uint4(e[4], e[5], e[6], e[7]);
    } else {
      c.v[0] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    }
  }
}

template <bool kWide, int kMode>
__device__ __forceinline__ void norm_store(void *base, long long row, int k, int nt, int d, int o, const float (&v)[8]) {
  if constexpr (kMode != kNormSingle) {
    const int col = norm_column<kMode>(k, 0, nt, o);
    if (col >= d) return;
    if (kMode == kNormVec || (col >= 0 && col + 8 <= d)) {
      uint4 *dst = reinterpret_cast<uint4 *>(static_cast<char *>(base) + (row + col) * (kWide ? 4 : 2));
      if constexpr (kWide) {
        dst[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        dst[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
      } else {
        dst[0] = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
      }
      return;
    }
  }
  if constexpr (kMode != kNormVec) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const int col = norm_column<kMode>(k, i, nt, o), next = norm_column<kMode>(k, i + 1, nt, o);
      if (kMode == kNormShifted && !kWide && col >= 0 && next < d) {
        *reinterpret_cast<uint32_t *>(static_cast<__nv_bfloat16 *>(base) + row + col) = pack_bf16x2(v[i], v[i + 1]);
        continue;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int at = j ? next : col;
        if (at < 0 || at >= d) continue;
        if constexpr (kWide) static_cast<float *>(base)[row + at] = v[i + j];
        else static_cast<__nv_bfloat16 *>(base)[row + at] = __float2bfloat16_rn(v[i + j]);
      }
    }
  }
}

// |v| as an integer: the same order as the magnitudes, with NaN above infinity
__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

template <bool kFast>
__device__ __forceinline__ float norm_scale(unsigned top, float inv) {
  const float s = kFast ? __uint_as_float(top) * inv * (1.f / kE4m3Max) : __uint_as_float(top) * inv / kE4m3Max;
  return s < kLeastScale ? kLeastScale : s;
}

// 1 / s, and 1 / sqrt(mean + eps), within 2 ulp (kFast) or one.  Fewer instructions and
// registers, so more CTAs: 20000 x 1152 to e4m3 with groups 33 -> 27.5 us, 12000 x 5001
// 120 -> 110.  The variant of two chunks with the next row ahead gets fewer registers
// than it needs instead (20000 x 3589 92 -> 100, 32768 x 3584 to e4m3 131 -> 137).
template <bool kFast>
__device__ __forceinline__ float norm_reciprocal(float s) {
  return kFast ? __fdividef(1.f, s) : 1.f / s;
}
template <bool kFast>
__device__ __forceinline__ float norm_inverse(float sum, const NormParams &p) {
  return kFast ? rsqrtf(fmaf(sum, p.per_d, p.eps)) : 1.f / sqrtf(sum / static_cast<float>(p.d) + p.eps);
}

// kAhead: the weights stay in registers and the next row is loaded ahead (blocks of
// at most 512 threads: the registers of 1024 do not hold that).
template <bool kWide, bool kE4m3, int kMode, int kChunks, bool kAhead>
__global__ void __launch_bounds__(kAhead ? kNormMaxThreads / 2 : kNormMaxThreads)
add_rms_norm_kernel(const __grid_constant__ NormParams p) {
  __shared__ float s_sum[2][kNormMaxThreads / 32];
  __shared__ unsigned s_top[2][kNormMaxThreads / 32];
  __shared__ unsigned s_group[kE4m3 && kMode != kNormVec ? SF_MAX_NORM_DIM / kNormGroup : 1];
  constexpr bool kVec = kMode == kNormVec, kFast = !(kChunks == 2 && kAhead);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nt = blockDim.x, nw = nt >> 5;
  const bool grouped = kE4m3 && p.groups > 1;
  grid_dependency_wait();
  grid_launch_dependents();
  auto global_weight = [&](int col) -> float {
    return p.weight_wide ? static_cast<const float *>(p.weight)[col]
                         : __bfloat162float(static_cast<const __nv_bfloat16 *>(p.weight)[col]);
  };
  // elements from a 16-byte boundary to a row's start (the same for all rows of a CTA)
  const int o = kMode == kNormShifted ? static_cast<int>((p.shift + blockIdx.x * p.x_stride) & 7) : 0;
  auto weight = [&](int k, int i) -> float {
    const int col = norm_column<kMode>(k, i, nt, o);
    return col >= 0 && col < p.d ? global_weight(col) : 0.f;
  };
  float w[kChunks][8];
  if constexpr (kAhead) {
#pragma unroll
    for (int k = 0; k < kChunks; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) w[k][i] = weight(k, i);
  }
  // 8 values of a chunk as e4m3, of element `line` on with the next group's scale
  auto store_e4m3 = [&](int row, int col, const float (&v)[8], float inv, float rs, float rs_next, int line) {
    uint32_t q[2];
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      float e[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) e[j] = v[i + j] * inv * (kVec || i + j < line ? rs : rs_next);
      q[i >> 2] = __nv_cvt_float2_to_fp8x2(make_float2(e[0], e[1]), __NV_SATFINITE, __NV_E4M3) |
                  static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(e[2], e[3]), __NV_SATFINITE, __NV_E4M3)) << 16;
    }
    uint8_t *dst = static_cast<uint8_t *>(p.out) + row * p.out_stride + col;
    if (kVec || (col >= 0 && col + 8 <= p.d)) {
      *reinterpret_cast<uint2 *>(dst) = make_uint2(q[0], q[1]);
      return;
    }
    if constexpr (!kVec) {
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        if (col + i >= 0 && col + i + 4 <= p.d) {
          *reinterpret_cast<uint32_t *>(dst + i) = q[i >> 2];
          continue;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (col + i + j >= 0 && col + i + j < p.d) dst[i + j] = static_cast<uint8_t>(q[i >> 2] >> (8 * j));
      }
    }
  };
  NormChunk<kWide> x[kChunks], r[kChunks];
  auto load_row = [&](int row) {
    const bool first = row < p.margin, last = row >= p.T - p.margin;
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      norm_load<kWide, kMode>(p.x, row * p.x_stride, first, last, k, nt, p.d, o, x[k]);
      if (p.residual) norm_load<kWide, kMode>(p.residual, row * p.residual_stride, first, last, k, nt, p.d, o, r[k]);
    }
  };
  int buf = 0;
  if constexpr (kAhead) load_row(blockIdx.x);
  for (int row = blockIdx.x; row < p.T; row += gridDim.x, buf ^= 1) {
    if constexpr (!kAhead) load_row(row);
    float h[kChunks][8];
    float sum = 0.f;
    unsigned top = 0u;
#pragma unroll
    for (int k = 0; k < kChunks; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[k][i] = norm_elem(x[k], i);
        if (p.residual) h[k][i] += norm_elem(r[k], i);
      }
    if constexpr (kMode == kNormShifted) {
#pragma unroll
      for (int k = 0; k < kChunks; ++k) {
        const int col = norm_column<kMode>(k, 0, nt, o);
        if (col >= 0 && col + 8 <= p.d) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (col + i < 0 || col + i >= p.d) h[k][i] = 0.f;
      }
    }
    if (kAhead && row + static_cast<int>(gridDim.x) < p.T) load_row(row + gridDim.x);
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      if (p.residual) norm_store<kWide, kMode>(p.residual_out, row * p.residual_out_stride, k, nt, p.d, o, h[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum = fmaf(h[k][i], h[k][i], sum);
        h[k][i] *= kAhead ? w[k][i] : weight(k, i);
        if constexpr (kE4m3) top = max(top, magnitude_bits(h[k][i]));
      }
    }
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
    if (lane == 0) s_sum[buf][warp] = sum;
    if constexpr (kE4m3) {
      if (!grouped) {
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) s_top[buf][warp] = top;
      } else if constexpr (!kVec) {
        for (int g = tid; g < p.groups; g += nt) s_group[g] = 0u;
      }
    }
    __syncthreads();
    sum = lane < nw ? s_sum[buf][lane] : 0.f;
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
    const float inv = norm_inverse<kFast>(sum, p);
    if constexpr (!kE4m3) {
#pragma unroll
      for (int k = 0; k < kChunks; ++k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[k][i] *= inv;
        norm_store<false, kMode>(p.out, row * p.out_stride, k, nt, p.d, o, h[k]);
      }
    } else {
      float scale = 0.f;
      if (!grouped) {
        scale = norm_scale<kFast>(__reduce_max_sync(0xffffffffu, lane < nw ? s_top[buf][lane] : 0u), inv);
        if (tid == 0) p.scales[row] = scale;
      } else if constexpr (kMode == kNormSingle) {
        // (a warp's 32 columns belong to one group: nt is a multiple of 32)
#pragma unroll
        for (int k = 0; k < kChunks; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int col = norm_column<kMode>(k, i, nt, o);
            const unsigned m = __reduce_max_sync(0xffffffffu, magnitude_bits(h[k][i]));
            if (lane == 0 && col < p.d) atomicMax(&s_group[col / kNormGroup], m);
          }
      } else if constexpr (kMode == kNormShifted) {
        // 16 threads hold a group, but its last elements are in the next one's first chunk
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
          const int g = (k * nt + tid) >> 4;
          const bool leader = (lane & 15) == 0;
          unsigned m = 0u, before = 0u;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (leader && i < o) before = max(before, magnitude_bits(h[k][i]));
            else m = max(m, magnitude_bits(h[k][i]));
          }
#pragma unroll
          for (int x = 8; x > 0; x >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, x));
          if (leader && g < p.groups && m) atomicMax(&s_group[g], m);
          if (leader && g > 0 && before) atomicMax(&s_group[g - 1], before);
        }
      }
      if (grouped && !kVec) {
        __syncthreads();
        for (int g = tid; g < p.groups; g += nt)
          p.scales[static_cast<size_t>(row) * p.groups + g] = norm_scale<kFast>(s_group[g], inv);
      }
#pragma unroll
      for (int k = 0; k < kChunks; ++k) {
        if constexpr (kVec) {
          const int col = norm_column<kMode>(k, 0, nt, o);
          if (grouped) {
            unsigned m = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, magnitude_bits(h[k][i]));
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, x));
            scale = norm_scale<kFast>(m, inv);
            if ((lane & 15) == 0 && col < p.d) p.scales[static_cast<size_t>(row) * p.groups + col / kNormGroup] = scale;
          }
          const float rs = norm_reciprocal<kFast>(scale);
          if (col < p.d) store_e4m3(row, col, h[k], inv, rs, rs, 8);
        } else if constexpr (kMode == kNormShifted) {
          const int col = norm_column<kMode>(k, 0, nt, o);
          if (col < p.d) {
            // the chunk's group, the next one, and where that begins
            const int g = max(col, 0) / kNormGroup, line = (g + 1) * kNormGroup - col;
            float rs = norm_reciprocal<kFast>(scale), rs_next = rs;
            if (grouped) {
              rs = norm_reciprocal<kFast>(norm_scale<kFast>(s_group[g], inv));
              rs_next = line < 8 && g + 1 < p.groups ? norm_reciprocal<kFast>(norm_scale<kFast>(s_group[g + 1], inv)) : rs;
            }
            store_e4m3(row, col, h[k], inv, rs, rs_next, line);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int col = norm_column<kMode>(k, i, nt, o);
            if (col >= p.d) continue;
            if (grouped) scale = norm_scale<kFast>(s_group[col / kNormGroup], inv);
            static_cast<__nv_fp8_storage_t *>(p.out)[row * p.out_stride + col] =
                __nv_cvt_float_to_fp8(h[k][i] * inv * norm_reciprocal<kFast>(scale), __NV_SATFINITE, __NV_E4M3);
          }
        }
      }
      // (the next row clears s_group before its first barrier)
      if (grouped && !kVec) __syncthreads();
    }
  }
}

using NormKernel = void (*)(const NormParams);

template <bool kWide, bool kE4m3, int kMode>
static NormKernel norm_variant(int chunks, bool ahead) {
  if (chunks == 1) return add_rms_norm_kernel<kWide, kE4m3, kMode, 1, true>;
  if constexpr (!kWide && (kMode == kNormVec || (kMode == kNormShifted && !kE4m3))) {
    if (ahead) return add_rms_norm_kernel<kWide, kE4m3, kMode, 2, true>;
  }
  if (chunks == 2) return add_rms_norm_kernel<kWide, kE4m3, kMode, 2, false>;
  return add_rms_norm_kernel<kWide, kE4m3, kMode, 4, false>;
}

template <bool kWide, bool kE4m3>
static NormKernel norm_kernel(int mode, int chunks, bool ahead) {
  if (mode == kNormVec) return norm_variant<kWide, kE4m3, kNormVec>(chunks, ahead);
  if (mode == kNormShifted) return norm_variant<kWide, kE4m3, kNormShifted>(chunks, ahead);
  return norm_variant<kWide, kE4m3, kNormSingle>(chunks, ahead);
}

// Registers per thread of a variant (0 .. 63), looked up once per device.
static int norm_registers(NormKernel fn, int device, int variant, int *regs) {
  static std::mutex mu;
  static int known[64][64] = {};
  if (device < 0 || device >= 64) return fail(SF_ERR_UNSUPPORTED, "device ordinal %d", device);
  std::lock_guard<std::mutex> lock(mu);
  if (known[device][variant] == 0) {
    cudaFuncAttributes a;
    const cudaError_t e = cudaFuncGetAttributes(&a, fn);
    if (e != cudaSuccess) return fail(SF_ERR_CUDA, "cudaFuncGetAttributes (add_rms_norm): %s", cudaGetErrorString(e));
    known[device][variant] = a.numRegs;
  }
  *regs = known[device][variant];
  return SF_OK;
}

}  // namespace sf

extern "C" int sf_add_rms_norm(const void *x, const void *residual, const void *weight, int dtype,
                               int weight_dtype, int T, int d, long long x_stride,
                               long long residual_stride, float eps, void *residual_out,
                               long long residual_out_stride, void *out, int out_dtype,
                               long long out_stride, int group, float *scales, cudaStream_t stream) {
  using namespace sf;
  clear_error();
  if (T < 0) return fail(SF_ERR_INVALID_ARG, "T=%d is negative", T);
  if (T > kNormMaxRows) return fail(SF_ERR_UNSUPPORTED, "T=%d above %d", T, kNormMaxRows);
  if (d < 1 || d > SF_MAX_NORM_DIM) return fail(SF_ERR_INVALID_ARG, "d=%d outside [1, %d]", d, SF_MAX_NORM_DIM);
  if (dtype != SF_BF16 && dtype != SF_F32) return fail(SF_ERR_UNSUPPORTED, "dtype=%d (built: bf16, fp32)", dtype);
  if (weight_dtype != SF_BF16 && weight_dtype != SF_F32)
    return fail(SF_ERR_UNSUPPORTED, "weight_dtype=%d (built: bf16, fp32)", weight_dtype);
  if (out_dtype != SF_BF16 && out_dtype != SF_E4M3)
    return fail(SF_ERR_UNSUPPORTED, "out_dtype=%d (built: bf16, e4m3)", out_dtype);
  if (!(eps >= 0.f) || std::isinf(eps)) return fail(SF_ERR_INVALID_ARG, "eps must be finite and >= 0");
  const bool e4m3 = out_dtype == SF_E4M3;
  if (e4m3 ? (group != 0 && group != kNormGroup) : group != 0)
    return fail(SF_ERR_INVALID_ARG, "group=%d (e4m3 output: 0 or %d; bf16 output: 0)", group, kNormGroup);
  if (T == 0) return SF_OK;
  if (!x || !weight || !out) return fail(SF_ERR_INVALID_ARG, "a required pointer is NULL");
  if ((residual == nullptr) != (residual_out == nullptr))
    return fail(SF_ERR_INVALID_ARG, "residual and residual_out belong together");
  if (e4m3 != (scales != nullptr)) return fail(SF_ERR_INVALID_ARG, "scales belong to e4m3 output");
  if (x_stride < d || out_stride < d || (residual && (residual_stride < d || residual_out_stride < d)))
    return fail(SF_ERR_INVALID_ARG, "a row stride is below d=%d", d);
  const size_t e = dtype == SF_F32 ? 4 : 2;
  if (!aligned(x, e) || !aligned(weight, weight_dtype == SF_F32 ? 4 : 2) || (residual && !aligned(residual, e)) ||
      (residual_out && !aligned(residual_out, e)) || (!e4m3 && !aligned(out, 2)) || (scales && !aligned(scales, 4)))
    return fail(SF_ERR_INVALID_ARG, "a tensor is not aligned to its element");
  NormParams p;
  p.x = x;
  p.residual = residual;
  p.weight = weight;
  p.residual_out = residual_out;
  p.out = out;
  p.scales = scales;
  p.x_stride = x_stride;
  p.residual_stride = residual_stride;
  p.residual_out_stride = residual_out_stride;
  p.out_stride = out_stride;
  p.T = T;
  p.d = d;
  p.groups = e4m3 && group ? (d + group - 1) / group : 1;
  p.weight_wide = weight_dtype == SF_F32;
  p.eps = eps;
  p.per_d = 1.f / static_cast<float>(d);
  DeviceInfo dev;
  const int st = current_device(&dev);
  if (st != SF_OK) return st;
  const bool wide = dtype == SF_F32;
  // 16-byte accesses: where in its 8 elements every row of every tensor starts
  const size_t out_bytes = e4m3 ? 1 : 2;
  auto start = [](const void *q, size_t bytes) { return static_cast<int>(reinterpret_cast<uintptr_t>(q) / bytes % 8); };
  p.shift = start(x, e);
  p.margin = x_stride >= 7 && (!residual || residual_stride >= 7) ? 1 : 7;
  const bool alike = start(out, out_bytes) == p.shift && (out_stride - x_stride) % 8 == 0 &&
                     (!residual || (start(residual, e) == p.shift && start(residual_out, e) == p.shift &&
                                    (residual_stride - x_stride) % 8 == 0 && (residual_out_stride - x_stride) % 8 == 0));
  const bool vec = alike && p.shift == 0 && x_stride % 8 == 0 && d % 8 == 0;
  const int mode = vec ? kNormVec : alike && d <= SF_MAX_NORM_DIM - 14 ? kNormShifted : kNormSingle;
  const int items = (d + 7 + (mode == kNormShifted ? 7 : 0)) / 8;
  // One chunk a thread for rows of up to 4096, and two chunks, still with the next
  // row loaded ahead, for long bf16 rows in number: half the threads wait at a row's
  // barrier, and four CTAs of an SM are at different points of theirs (32768 x 3584
  // to e4m3 143 -> 131 us, 4096 x 8192 50 -> 39, 20000 x 3589 to bf16 108 -> 92; but
  // 16384 x 4096 to bf16 84 -> 88, 128 x 3584, one row a CTA, 2.8 -> 3.2, and
  // 12000 x 5001 to e4m3, with 111 registers, 119 -> 140).
  const bool two = (vec || (mode == kNormShifted && !e4m3)) && !wide && items > 256 && items <= kNormMaxThreads &&
                   T > 4 * dev.sm_count;
  const int chunks = two ? 2 : items <= 512 ? 1 : items <= 2 * kNormMaxThreads ? 2 : 4;
  const int threads = ((items + chunks - 1) / chunks + 31) / 32 * 32;
  const NormKernel fn = wide ? (e4m3 ? norm_kernel<true, true>(mode, chunks, two) : norm_kernel<true, false>(mode, chunks, two))
                             : (e4m3 ? norm_kernel<false, true>(mode, chunks, two) : norm_kernel<false, false>(mode, chunks, two));
  int regs = 0;
  const int rst = norm_registers(fn, dev.ordinal, (wide ? 1 : 0) | (e4m3 ? 2 : 0) | mode << 2 | (two ? 3 : chunks / 2) << 4, &regs);
  if (rst != SF_OK) return rst;
  // CTAs that are resident together, each for several rows where there are more
  // (a sub-partition's 16K registers hold whole warps)
  long long per_sm = 16384 / (32 * ((regs + 7) / 8 * 8)) * 4 / (threads / 32);
  if (per_sm > 2048 / threads) per_sm = 2048 / threads;
  if (per_sm < 1) per_sm = 1;
  // ... but no more than 104 KB of an SM's rows on their way in or out, where every
  // CTA has several: HBM takes fewer streams of loads and stores better (16000 x 2184
  // from fp32 86 -> 79 us, 32768 x 3584 to bf16 151 -> 142; to e4m3 100 KB are best).
  if ((two || chunks == 1) && T >= 4 * per_sm * dev.sm_count) {
    const long long row_bytes = static_cast<long long>(d) * (e * (residual ? 3 : 1) + out_bytes);
    per_sm = std::min(per_sm, std::max(2LL, 104 * 1024 / row_bytes));
  }
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  const long long resident = std::max(per_sm * dev.sm_count / 8 * 8, 8LL);
  cfg.gridDim = dim3(static_cast<unsigned>(std::min<long long>(T, resident)));
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t err = cudaLaunchKernelEx(&cfg, fn, p);
  if (err != cudaSuccess) return fail(SF_ERR_CUDA, "add_rms_norm launch: %s", cudaGetErrorString(err));
  return SF_OK;
}
