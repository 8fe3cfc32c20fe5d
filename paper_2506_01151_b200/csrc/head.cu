// The output head: values in 8-bit floating point with a scale for each block, and their product under the mask.
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/fmt.h"
#include "kernels.h"
#include "op_args.h"

using namespace fmt;

namespace {

constexpr uint32_t BLOCK = 128;  // columns (and, of weights, rows) that share a scale

__device__ __forceinline__ float to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float to_f32(float x) { return x; }

// The scale of a block from the bits of its largest |x|: bits of magnitudes are ordered as the magnitudes are, infinities and
// NaNs above them all.
__device__ __forceinline__ float block_scale(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  const float s = __fdiv_rn(__uint_as_float(amax_bits), 448.0f);
  return s == 0.0f ? 1.0f : s;
}

__device__ __forceinline__ uint8_t to_e4m3(float x, float scale) {  // a NaN becomes 0x7F; a scale that was rounded as a denormal saturates
  return (uint8_t)__nv_cvt_float_to_fp8(__fdiv_rn(x, scale), __NV_SATFINITE, __NV_E4M3);
}

// A thread block to a block of ROWS x 128 values.
template <typename T, uint32_t ROWS>
__global__ void __launch_bounds__(256) quantize_kernel(const T* x, uint32_t rows, uint32_t cols, size_t row_stride, uint8_t* q,
                                                       size_t q_stride, float* scales, size_t scale_stride) {
  before_me();
  __shared__ uint32_t most;
  const uint32_t r0 = blockIdx.x * ROWS, b = blockIdx.y, c0 = b * BLOCK;
  if (threadIdx.x == 0) most = 0u;
  __syncthreads();
  const uint32_t n = min(ROWS, rows - r0) * BLOCK;
  uint32_t amax = 0u;
  for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
    const uint32_t c = c0 + i % BLOCK;
    if (c < cols) amax = max(amax, __float_as_uint(to_f32(x[(size_t)(r0 + i / BLOCK) * row_stride + c])) & 0x7FFFFFFFu);
  }
  atomicMax(&most, amax);
  __syncthreads();
  const float scale = block_scale(most);
  if (threadIdx.x == 0) scales[ROWS == 1 ? (size_t)b * scale_stride + r0 : (size_t)blockIdx.x * scale_stride + b] = scale;
  for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
    const uint32_t c = c0 + i % BLOCK;
    if (c < cols) q[(size_t)(r0 + i / BLOCK) * q_stride + c] = to_e4m3(to_f32(x[(size_t)(r0 + i / BLOCK) * row_stride + c]), scale);
  }
}

__device__ __forceinline__ float e4m3(uint8_t v) { return __half2float(__nv_cvt_fp8_to_halfraw(v, __NV_E4M3)); }

template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ uint16_t from_f32<uint16_t>(float x) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0x7FFFu;
  return (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}

// A warp to a token and up to eight rows, its lanes along K.
constexpr uint32_t HEAD_ROWS = 8;
template <typename T>
__global__ void __launch_bounds__(256) head_kernel(const uint8_t* x, size_t x_stride, const float* xs, size_t xs_stride, const uint8_t* w,
                                                   size_t w_stride, const float* ws, size_t ws_stride, uint32_t rows, uint32_t V, uint32_t K,
                                                   const uint32_t* mask, size_t mask_stride, T* logits, size_t row_stride) {
  before_me();
  const uint32_t lane = threadIdx.x & 31u, v = blockIdx.x * 8u + threadIdx.x / 32u;
  if (v >= V) return;
  for (uint32_t r0 = blockIdx.y * HEAD_ROWS; r0 < rows; r0 += gridDim.y * HEAD_ROWS) {
    float acc[HEAD_ROWS] = {};
    uint32_t want = 0u;
    for (uint32_t r = 0; r < HEAD_ROWS && r0 + r < rows; ++r)
      if (!mask || (mask[(size_t)(r0 + r) * mask_stride + (v >> 5)] >> (v & 31u)) & 1u) want |= 1u << r;
    if (want)
      for (uint32_t b = 0; b * BLOCK < K; ++b) {
        float y[4];
        for (uint32_t i = 0; i < 4u; ++i) {
          const uint32_t k = b * BLOCK + lane + 32u * i;
          y[i] = k < K ? e4m3(w[(size_t)v * w_stride + k]) : 0.0f;
        }
        const float s = ws[(size_t)(v / BLOCK) * ws_stride + b];
#pragma unroll
        for (uint32_t r = 0; r < HEAD_ROWS; ++r) {
          if (r0 + r >= rows) break;
          float sum = 0.0f;
          for (uint32_t i = 0; i < 4u; ++i) {
            const uint32_t k = b * BLOCK + lane + 32u * i;
            if (k < K) sum = fmaf(y[i], e4m3(x[(size_t)(r0 + r) * x_stride + k]), sum);
          }
          acc[r] = fmaf(sum, s * xs[(size_t)b * xs_stride + r0 + r], acc[r]);
        }
      }
#pragma unroll
    for (uint32_t r = 0; r < HEAD_ROWS; ++r) {
      for (uint32_t o = 16u; o; o >>= 1) acc[r] += __shfl_xor_sync(0xFFFFFFFFu, acc[r], o);
      if (lane == r && r0 + r < rows)
        logits[(size_t)(r0 + r) * row_stride + v] = from_f32<T>((want >> r) & 1u ? acc[r] : -__int_as_float(0x7F800000));
    }
  }
}

}  // namespace

extern "C" fmt_status fmt_quantize_blocks(const void* x_dev, fmt_dtype dtype, uint32_t rows, uint32_t cols, size_t row_stride_elems,
                                          uint32_t block_rows, uint8_t* q_dev, size_t q_stride, float* scales_dev, size_t scale_stride,
                                          void* stream) {
  if (!x_dev || !q_dev || !scales_dev) return refuse("NULL argument");
  if (dtype != FMT_BF16 && dtype != FMT_FP32) return refuse("unknown dtype");
  if (block_rows != 1 && block_rows != BLOCK) return refuse("block_rows must be 1 or 128");
  if (cols == 0 || cols > (1u << 20) || rows > (1u << 24)) return refuse("rows or cols out of range");
  if (row_stride_elems < cols || q_stride < cols || scale_stride < (block_rows == 1 ? rows : (cols + BLOCK - 1) / BLOCK))
    return refuse("a stride is too small");
  if (misaligned(x_dev, dtype == FMT_BF16 ? 2 : 4) || misaligned(scales_dev, 4)) return refuse("a pointer is not aligned to its elements");
  if (rows == 0) return FMT_OK;
  if (fmt_status s = reachable({x_dev, q_dev, scales_dev})) return s;
  const dim3 grid((rows + block_rows - 1) / block_rows, (cols + BLOCK - 1) / BLOCK);
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == FMT_BF16) {
    auto* k = block_rows == 1 ? quantize_kernel<uint16_t, 1> : quantize_kernel<uint16_t, BLOCK>;
    return launch_result(launch_overlapped(k, grid, dim3(block_rows == 1 ? 128 : 256), 0, st, (const uint16_t*)x_dev, rows, cols, row_stride_elems, q_dev, q_stride,
                                           scales_dev, scale_stride));
  }
  auto* k = block_rows == 1 ? quantize_kernel<float, 1> : quantize_kernel<float, BLOCK>;
  return launch_result(launch_overlapped(k, grid, dim3(block_rows == 1 ? 128 : 256), 0, st, (const float*)x_dev, rows, cols, row_stride_elems, q_dev, q_stride, scales_dev,
                                         scale_stride));
}

extern "C" fmt_status fmt_head_logits(const uint8_t* hidden_dev, size_t hidden_stride, const float* hidden_scales_dev,
                                      size_t hidden_scale_stride, const uint8_t* weight_dev, size_t weight_stride,
                                      const float* weight_scales_dev, size_t weight_scale_stride, uint32_t rows, uint32_t V, uint32_t K,
                                      const uint32_t* mask_dev, size_t mask_stride_words, void* logits_dev, fmt_dtype dtype,
                                      size_t row_stride_elems, void* stream) {
  if (!hidden_dev || !hidden_scales_dev || !weight_dev || !weight_scales_dev || !logits_dev) return refuse("NULL argument");
  if (dtype != FMT_BF16 && dtype != FMT_FP32) return refuse("unknown dtype");
  if (V == 0 || V > (1u << 24) || K == 0 || K > (1u << 20) || rows > (1u << 24)) return refuse("rows, V or K out of range");
  if (hidden_stride < K || weight_stride < K || hidden_scale_stride < rows || weight_scale_stride < (K + BLOCK - 1) / BLOCK ||
      row_stride_elems < V || (mask_dev && mask_stride_words < (V + 31) / 32))
    return refuse("a stride is too small");
  if (hidden_stride % 16 || weight_stride % 16 || misaligned(hidden_dev, 16) || misaligned(weight_dev, 16))
    return refuse("hidden states and weights must be 16-byte aligned, their strides multiples of 16");
  if (misaligned(hidden_scales_dev, 4) || misaligned(weight_scales_dev, 4) || misaligned(mask_dev, 4) ||
      misaligned(logits_dev, dtype == FMT_BF16 ? 2 : 4))
    return refuse("a pointer is not aligned to its elements");
  if (rows == 0) return FMT_OK;
  if (fmt_status s = reachable({hidden_dev, hidden_scales_dev, weight_dev, weight_scales_dev, mask_dev, logits_dev})) return s;
  const dim3 grid((V + 7) / 8, std::min<uint32_t>((rows + HEAD_ROWS - 1) / HEAD_ROWS, 65535u));
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == FMT_BF16)
    return launch_result(launch_overlapped(head_kernel<uint16_t>, grid, dim3(256), 0, st, hidden_dev, hidden_stride, hidden_scales_dev, hidden_scale_stride,
                                           weight_dev, weight_stride, weight_scales_dev, weight_scale_stride, rows, V, K, mask_dev,
                                           mask_stride_words, (uint16_t*)logits_dev, row_stride_elems));
  return launch_result(launch_overlapped(head_kernel<float>, grid, dim3(256), 0, st, hidden_dev, hidden_stride, hidden_scales_dev, hidden_scale_stride,
                                         weight_dev, weight_stride, weight_scales_dev, weight_scale_stride, rows, V, K, mask_dev,
                                         mask_stride_words, (float*)logits_dev, row_stride_elems));
}
