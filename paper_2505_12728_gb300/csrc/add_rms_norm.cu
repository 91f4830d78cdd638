// add_rms_norm.cu -- residual addition and root-mean-square norm of the rows
// between a decoder layer's projections, with bf16 or 8-bit output.
//
//     h = x + residual,  y = h * weight / sqrt(mean(h^2) + eps)
//
// One CTA per row; h stays in shared memory as fp32 between the sum of squares
// and the scaling, so x and the residual are read once.
#include <cmath>

#include <cuda_fp8.h>

#include "sf_device.cuh"
#include "sf_host.h"

namespace sf {

constexpr int kNormThreads = 256;
constexpr int kNormGroup = 128;       // columns per scale
constexpr float kE4m3Max = 448.f;     // largest finite e4m3 value
constexpr float kLeastScale = 1.17549435e-38f;  // 2^-126

struct NormParams {
  const void *x, *residual, *weight;
  void *residual_out, *out;
  float *scales;
  long long x_stride, residual_stride, residual_out_stride, out_stride;
  int T, d, groups;
  int wide, weight_wide, e4m3;
  float eps;
};

__device__ __forceinline__ float load_elem(const void *p, size_t i, int wide) {
  return wide ? static_cast<const float *>(p)[i]
              : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

__device__ __forceinline__ void store_elem(void *p, size_t i, int wide, float v) {
  if (wide) static_cast<float *>(p)[i] = v;
  else static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
}

// |v| as an integer: the same order as the magnitudes, with NaN above infinity
__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__global__ void __launch_bounds__(kNormThreads) add_rms_norm_kernel(const __grid_constant__ NormParams p) {
  extern __shared__ float s_h[];  // [d]
  __shared__ float s_sum[kNormThreads / 32];
  __shared__ unsigned s_top[SF_MAX_NORM_DIM / kNormGroup];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  grid_dependency_wait();
  const size_t row = blockIdx.x;
  const size_t xo = row * p.x_stride, ro = row * p.residual_stride, so = row * p.residual_out_stride,
               oo = row * p.out_stride;
  float sum = 0.f;
  for (int c = tid; c < p.d; c += kNormThreads) {
    float h = load_elem(p.x, xo + c, p.wide);
    if (p.residual) {
      h += load_elem(p.residual, ro + c, p.wide);
      store_elem(p.residual_out, so + c, p.wide, h);
    }
    s_h[c] = h;
    sum += h * h;
  }
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[warp] = sum;
  for (int g = tid; g < p.groups; g += kNormThreads) s_top[g] = 0u;
  __syncthreads();
  sum = 0.f;
  for (int w = 0; w < kNormThreads / 32; ++w) sum += s_sum[w];
  const float inv = 1.f / sqrtf(sum / static_cast<float>(p.d) + p.eps);
  for (int c = tid; c < p.d; c += kNormThreads) {
    const float y = s_h[c] * inv * load_elem(p.weight, c, p.weight_wide);
    if (p.e4m3) {
      s_h[c] = y;
      atomicMax(&s_top[p.groups == 1 ? 0 : c / kNormGroup], magnitude_bits(y));
    } else {
      store_elem(p.out, oo + c, 0, y);
    }
  }
  if (!p.e4m3) return;
  __syncthreads();
  for (int c = tid; c < p.d; c += kNormThreads) {
    const int g = p.groups == 1 ? 0 : c / kNormGroup;
    const float top = __uint_as_float(s_top[g]) / kE4m3Max;
    const float scale = top < kLeastScale ? kLeastScale : top;
    static_cast<__nv_fp8_e4m3 *>(p.out)[oo + c] = __nv_fp8_e4m3(s_h[c] / scale);
    if (c == g * kNormGroup) p.scales[row * p.groups + g] = scale;
  }
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
  p.wide = dtype == SF_F32;
  p.weight_wide = weight_dtype == SF_F32;
  p.e4m3 = e4m3;
  p.eps = eps;
  const size_t smem = sizeof(float) * static_cast<size_t>(d);
  cudaError_t err = cudaFuncSetAttribute(add_rms_norm_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         SF_MAX_NORM_DIM * static_cast<int>(sizeof(float)));
  if (err == cudaSuccess) {
    add_rms_norm_kernel<<<T, kNormThreads, smem, stream>>>(p);
    err = cudaGetLastError();
  }
  if (err != cudaSuccess) return fail(SF_ERR_CUDA, "add_rms_norm launch: %s", cudaGetErrorString(err));
  return SF_OK;
}
