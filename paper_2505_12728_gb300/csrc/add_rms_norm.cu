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
// row's loads in flight during the reduction of the present one.
#include <cmath>
#include <mutex>

#include <cuda_fp8.h>

#include "sf_device.cuh"
#include "sf_host.h"

namespace sf {

constexpr int kNormMaxThreads = 1024;
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
  float eps;
};

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

// Where element (k, i) of a thread lies in its row: chunks of 8 neighbours, or,
// where 16-byte accesses are not possible, a block's width apart.
template <bool kVec>
__device__ __forceinline__ int norm_column(int k, int i, int nt) {
  return kVec ? (k * nt + static_cast<int>(threadIdx.x)) * 8 + i : (k * 8 + i) * nt + static_cast<int>(threadIdx.x);
}

template <bool kWide, bool kVec>
__device__ __forceinline__ void norm_load(const void *base, long long row, int k, int nt, int d, NormChunk<kWide> &c) {
  if constexpr (kVec) {
    const int col = norm_column<true>(k, 0, nt);
    if (col < d) {
      const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const char *>(base) + (row + col) * (kWide ? 4 : 2));
      c.v[0] = src[0];
      if constexpr (kWide) c.v[1] = src[1];
      return;
    }
    c.v[0] = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (kWide) c.v[1] = make_uint4(0u, 0u, 0u, 0u);
  } else {
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int col = norm_column<false>(k, i, nt);
      e[i] = 0u;
      if (col < d)
        e[i] = kWide ? static_cast<const uint32_t *>(base)[row + col]
                     : static_cast<uint32_t>(static_cast<const uint16_t *>(base)[row + col]);
    }
    if constexpr (kWide) {
      c.v[0] = make_uint4(e[0], e[1], e[2], e[3]);
      c.v[1] = make_uint4(e[4], e[5], e[6], e[7]);
    } else {
      c.v[0] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    }
  }
}

template <bool kWide, bool kVec>
__device__ __forceinline__ void norm_store(void *base, long long row, int k, int nt, int d, const float (&v)[8]) {
  if constexpr (kVec) {
    const int col = norm_column<true>(k, 0, nt);
    if (col >= d) return;
    uint4 *dst = reinterpret_cast<uint4 *>(static_cast<char *>(base) + (row + col) * (kWide ? 4 : 2));
    if constexpr (kWide) {
      dst[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      dst[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    } else {
      dst[0] = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int col = norm_column<false>(k, i, nt);
      if (col >= d) continue;
      if constexpr (kWide) static_cast<float *>(base)[row + col] = v[i];
      else static_cast<__nv_bfloat16 *>(base)[row + col] = __float2bfloat16_rn(v[i]);
    }
  }
}

// |v| as an integer: the same order as the magnitudes, with NaN above infinity
__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ float norm_scale(unsigned top, float inv) {
  const float s = __uint_as_float(top) * inv / kE4m3Max;
  return s < kLeastScale ? kLeastScale : s;
}

// kAhead: the weights stay in registers and the next row is loaded ahead (blocks of
// at most 512 threads: the registers of 1024 do not hold that).
template <bool kWide, bool kE4m3, bool kVec, int kChunks, bool kAhead>
__global__ void __launch_bounds__(kAhead ? kNormMaxThreads / 2 : kNormMaxThreads)
add_rms_norm_kernel(const __grid_constant__ NormParams p) {
  __shared__ float s_sum[2][kNormMaxThreads / 32];
  __shared__ unsigned s_top[2][kNormMaxThreads / 32];
  __shared__ unsigned s_group[kE4m3 && !kVec ? SF_MAX_NORM_DIM / kNormGroup : 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nt = blockDim.x, nw = nt >> 5;
  const bool grouped = kE4m3 && p.groups > 1;
  grid_dependency_wait();
  grid_launch_dependents();
  auto weight = [&](int k, int i) -> float {
    const int col = norm_column<kVec>(k, i, nt);
    if (col >= p.d) return 0.f;
    return p.weight_wide ? static_cast<const float *>(p.weight)[col]
                         : __bfloat162float(static_cast<const __nv_bfloat16 *>(p.weight)[col]);
  };
  float w[kChunks][8];
  if constexpr (kAhead) {
#pragma unroll
    for (int k = 0; k < kChunks; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) w[k][i] = weight(k, i);
  }
  NormChunk<kWide> x[kChunks], r[kChunks];
  auto load_row = [&](int row) {
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      norm_load<kWide, kVec>(p.x, row * p.x_stride, k, nt, p.d, x[k]);
      if (p.residual) norm_load<kWide, kVec>(p.residual, row * p.residual_stride, k, nt, p.d, r[k]);
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
    if (kAhead && row + static_cast<int>(gridDim.x) < p.T) load_row(row + gridDim.x);
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
      if (p.residual) norm_store<kWide, kVec>(p.residual_out, row * p.residual_out_stride, k, nt, p.d, h[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum = fmaf(h[k][i], h[k][i], sum);
        h[k][i] *= kAhead ? w[k][i] : weight(k, i);
        if constexpr (kE4m3) top = max(top, magnitude_bits(h[k][i]));
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
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
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float inv = 1.f / sqrtf(sum / static_cast<float>(p.d) + p.eps);
    if constexpr (!kE4m3) {
#pragma unroll
      for (int k = 0; k < kChunks; ++k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[k][i] *= inv;
        norm_store<false, kVec>(p.out, row * p.out_stride, k, nt, p.d, h[k]);
      }
    } else {
      float scale = 0.f;
      if (!grouped) {
        scale = norm_scale(__reduce_max_sync(0xffffffffu, lane < nw ? s_top[buf][lane] : 0u), inv);
        if (tid == 0) p.scales[row] = scale;
      } else if constexpr (!kVec) {
        // (a warp's 32 columns belong to one group: nt is a multiple of 32)
#pragma unroll
        for (int k = 0; k < kChunks; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int col = norm_column<false>(k, i, nt);
            const unsigned m = __reduce_max_sync(0xffffffffu, magnitude_bits(h[k][i]));
            if (lane == 0 && col < p.d) atomicMax(&s_group[col / kNormGroup], m);
          }
        __syncthreads();
        for (int g = tid; g < p.groups; g += nt)
          p.scales[static_cast<size_t>(row) * p.groups + g] = norm_scale(s_group[g], inv);
      }
#pragma unroll
      for (int k = 0; k < kChunks; ++k) {
        if constexpr (kVec) {
          const int col = norm_column<true>(k, 0, nt);
          if (grouped) {
            unsigned m = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, magnitude_bits(h[k][i]));
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
            scale = norm_scale(m, inv);
            if ((lane & 15) == 0 && col < p.d) p.scales[static_cast<size_t>(row) * p.groups + col / kNormGroup] = scale;
          }
          const float rs = 1.f / scale;
          if (col < p.d) {
            uint32_t q[2];
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
              const float a = h[k][i] * inv * rs, b = h[k][i + 1] * inv * rs, c = h[k][i + 2] * inv * rs,
                          e = h[k][i + 3] * inv * rs;
              q[i >> 2] = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3) |
                          static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(c, e), __NV_SATFINITE, __NV_E4M3)) << 16;
            }
            *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(p.out) + row * p.out_stride + col) = make_uint2(q[0], q[1]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int col = norm_column<false>(k, i, nt);
            if (col >= p.d) continue;
            if (grouped) scale = norm_scale(s_group[col / kNormGroup], inv);
            static_cast<__nv_fp8_storage_t *>(p.out)[row * p.out_stride + col] =
                __nv_cvt_float_to_fp8(h[k][i] * inv * (1.f / scale), __NV_SATFINITE, __NV_E4M3);
          }
        }
      }
      // (the next row clears s_group before its first barrier)
      if (grouped && !kVec) __syncthreads();
    }
  }
}

using NormKernel = void (*)(const NormParams);

template <bool kWide, bool kE4m3, bool kVec>
static NormKernel norm_kernel(int chunks, bool ahead) {
  if (chunks == 1) return add_rms_norm_kernel<kWide, kE4m3, kVec, 1, true>;
  if constexpr (kVec && !kWide) {
    if (ahead) return add_rms_norm_kernel<kWide, kE4m3, true, 2, true>;
  }
  if (chunks == 2) return add_rms_norm_kernel<kWide, kE4m3, kVec, 2, false>;
  return add_rms_norm_kernel<kWide, kE4m3, kVec, 4, false>;
}

// Registers per thread of a variant (0 .. 31), looked up once per device.
static int norm_registers(NormKernel fn, int device, int variant, int *regs) {
  static std::mutex mu;
  static int known[64][32] = {};
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
  DeviceInfo dev;
  const int st = current_device(&dev);
  if (st != SF_OK) return st;
  const bool wide = dtype == SF_F32;
  // 16-byte accesses need 8 neighbouring elements in every tensor
  const size_t out_bytes = e4m3 ? 1 : 2;
  const bool vec = d % 8 == 0 && x_stride % 8 == 0 && out_stride % 8 == 0 && aligned(x, 16) &&
                   aligned(out, 8 * out_bytes) &&
                   (!residual || (residual_stride % 8 == 0 && residual_out_stride % 8 == 0 && aligned(residual, 16) &&
                                  aligned(residual_out, 16)));
  const int items = (d + 7) / 8;
  // One chunk a thread for rows of up to 4096, and two chunks, still with the next
  // row loaded ahead, for long bf16 rows in number: half the threads wait at a row's
  // barrier, and four CTAs of an SM are at different points of theirs (32768 x 3584
  // to e4m3 143 -> 131 us, 4096 x 8192 50 -> 39, 2048 x 3584 to bf16 13.2 -> 11.6; but
  // 16384 x 4096 to bf16 84 -> 88,
  // and 128 x 3584, one row a CTA, 2.8 -> 3.2).
  const bool two = vec && !wide && items > 256 && items <= kNormMaxThreads && T > 4 * dev.sm_count;
  const int chunks = two ? 2 : items <= 512 ? 1 : items <= 2 * kNormMaxThreads ? 2 : 4;
  const int threads = ((items + chunks - 1) / chunks + 31) / 32 * 32;
  NormKernel fn;
  if (wide)
    fn = e4m3 ? (vec ? norm_kernel<true, true, true>(chunks, two) : norm_kernel<true, true, false>(chunks, two))
              : (vec ? norm_kernel<true, false, true>(chunks, two) : norm_kernel<true, false, false>(chunks, two));
  else
    fn = e4m3 ? (vec ? norm_kernel<false, true, true>(chunks, two) : norm_kernel<false, true, false>(chunks, two))
              : (vec ? norm_kernel<false, false, true>(chunks, two) : norm_kernel<false, false, false>(chunks, two));
  int regs = 0;
  const int rst = norm_registers(fn, dev.ordinal, (wide ? 1 : 0) | (e4m3 ? 2 : 0) | (vec ? 4 : 0) | (two ? 3 : chunks / 2) << 3, &regs);
  if (rst != SF_OK) return rst;
  // CTAs that are resident together, each for several rows where there are more
  long long per_sm = 65536 / (static_cast<long long>(threads) * ((regs + 7) / 8 * 8));
  if (per_sm > 2048 / threads) per_sm = 2048 / threads;
  if (per_sm < 1) per_sm = 1;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(T < per_sm * dev.sm_count ? T : per_sm * dev.sm_count));
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t err = cudaLaunchKernelEx(&cfg, fn, p);
  if (err != cudaSuccess) return fail(SF_ERR_CUDA, "add_rms_norm launch: %s", cudaGetErrorString(err));
  return SF_OK;
}
