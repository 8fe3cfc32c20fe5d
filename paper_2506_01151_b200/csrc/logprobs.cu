// Log probabilities, entropy and likeliest tokens of the rows' distributions under their masks, and the gradient.
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/fmt.h"
#include "kernels.h"
#include "op_args.h"

using namespace fmt;

namespace {

constexpr float INF = __builtin_huge_valf();
constexpr uint32_t THREADS = 256;

struct Rows {  // what the forward and the backward pass read
  uint32_t rows, V;
  const void* logits;
  size_t stride;
  const uint32_t* mask;
  size_t mask_stride;
  const float* temperature;
  const int32_t* tokens;
  uint32_t n_tokens;
};
struct Outputs {
  uint32_t n_top;
  float* logprobs;
  float* norm;
  float* entropy;
  int32_t* top_ids;
  float* top_logprobs;
  int32_t* status;
};
struct Gradients {
  const float* norm;
  const float* entropy;
  const float* by_logprob;
  const float* by_entropy;
  void* out;
  size_t stride;
};

__device__ __forceinline__ float to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) {  // to the nearest bf16, ties to even
  const uint32_t u = __float_as_uint(x);
  *p = (u & 0x7FFFFFFFu) > 0x7F800000u ? (uint16_t)0x7FFFu : (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}

// The logit where the mask allows the token, else -inf.
template <typename T>
__device__ __forceinline__ float allowed(const Rows& R, uint32_t row, uint32_t v) {
  if (R.mask && !((R.mask[(size_t)row * R.mask_stride + (v >> 5)] >> (v & 31u)) & 1u)) return -INF;
  return to_f32(static_cast<const T*>(R.logits)[(size_t)row * R.stride + v]);
}

// Logits in the order wanted as whole numbers: larger first, of equal ones (0 and -0 are equal) the lower id.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t v) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (0xFFFFFFFFu - v);
}

template <typename V, typename F>
__device__ __forceinline__ V block_reduce(V x, V* buf, F join) {
  __syncthreads();
  buf[threadIdx.x] = x;
  for (uint32_t n = THREADS / 2; n; n /= 2) {
    __syncthreads();
    if (threadIdx.x < n) buf[threadIdx.x] = join(buf[threadIdx.x], buf[threadIdx.x + n]);
  }
  __syncthreads();
  return buf[0];
}

template <typename T>
__global__ void __launch_bounds__(THREADS) logprobs_kernel(const Rows R, const Outputs O) {
  before_me();
  __shared__ float fbuf[THREADS];
  __shared__ uint64_t kbuf[THREADS];
  const uint32_t row = blockIdx.x, tid = threadIdx.x;
  const float temperature = R.temperature ? R.temperature[row] : 1.0f;
  float most = -INF, odd = 0.0f;
  for (uint32_t v = tid; v < R.V; v += THREADS) {
    const float x = allowed<T>(R, row, v);
    if (!(x < INF)) odd = 1.0f;
    most = fmaxf(most, x);
  }
  most = block_reduce(most, fbuf, [](float a, float b) { return fmaxf(a, b); });
  odd = block_reduce(odd, fbuf, [](float a, float b) { return fmaxf(a, b); });
  const bool bad = odd != 0.0f || !(temperature > 0.0f && temperature < INF);
  const float inv = __fdiv_rn(1.0f, temperature);
  float s = 0.0f, t = 0.0f;
  if (!bad && most > -INF)
    for (uint32_t v = tid; v < R.V; v += THREADS) {
      const float d = (allowed<T>(R, row, v) - most) * inv, p = expf(d);
      s += p;
      if (p > 0.0f) t = fmaf(p, d, t);
    }
  auto add = [](float a, float b) { return a + b; };
  s = block_reduce(s, fbuf, add);
  t = block_reduce(t, fbuf, add);
  const float nan = __int_as_float(0x7FC00000);
  const float ln = bad ? nan : logf(s);  // (-inf of nothing)
  auto logprob = [&](float x) { return bad ? nan : x == -INF ? -INF : (x - most) * inv - ln; };
  bool wrong = false;
  for (uint32_t k = tid; k < R.n_tokens; k += THREADS) {
    const int32_t v = R.tokens[(size_t)row * R.n_tokens + k];
    const bool out = v < -1 || v >= (int64_t)R.V;
    wrong |= out;
    if (O.logprobs) O.logprobs[(size_t)row * R.n_tokens + k] = v == -1 ? 0.0f : out ? nan : logprob(allowed<T>(R, row, (uint32_t)v));
  }
  const int any_wrong = __syncthreads_or(wrong);
  if (tid == 0) {
    if (O.norm) O.norm[2 * (size_t)row] = bad ? nan : most, O.norm[2 * (size_t)row + 1] = ln;
    if (O.entropy) O.entropy[row] = bad ? nan : s > 0.0f ? ln - t / s : 0.0f;
    if (O.status) O.status[row] = bad || any_wrong ? FMT_ERR_INVALID_ARG : FMT_OK;
  }
  uint64_t last = ~0ull;
  for (uint32_t k = 0; k < O.n_top; ++k) {
    uint64_t best = 0;
    if (!bad)
      for (uint32_t v = tid; v < R.V; v += THREADS) {
        const float x = allowed<T>(R, row, v);
        const uint64_t key = order_key(x, v);
        if (x > -INF && key < last && key > best) best = key;
      }
    last = block_reduce(best, kbuf, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
    const uint32_t v = 0xFFFFFFFFu - (uint32_t)last;
    if (tid == 0) {
      if (O.top_ids) O.top_ids[(size_t)row * O.n_top + k] = last ? (int32_t)v : -1;
      if (O.top_logprobs) O.top_logprobs[(size_t)row * O.n_top + k] = last ? logprob(allowed<T>(R, row, v)) : bad ? nan : -INF;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(THREADS) logprobs_backward_kernel(const Rows R, const Gradients D) {
  before_me();
  __shared__ int32_t tok[FMT_MAX_GIVEN_TOKENS];
  __shared__ float g[FMT_MAX_GIVEN_TOKENS];
  const uint32_t row = blockIdx.x, tid = threadIdx.x;
  const float inv = __fdiv_rn(1.0f, R.temperature ? R.temperature[row] : 1.0f);
  const float most = D.norm[2 * (size_t)row], ln = D.norm[2 * (size_t)row + 1];
  const float gh = D.by_entropy ? D.by_entropy[row] : 0.0f, h = D.by_entropy ? D.entropy[row] : 0.0f;
  if (tid < R.n_tokens) {
    const int32_t v = R.tokens[(size_t)row * R.n_tokens + tid];
    const bool ok = v >= 0 && v < (int64_t)R.V && (allowed<T>(R, row, (uint32_t)v) - most) * inv > -INF;
    tok[tid] = ok ? v : -1;
    g[tid] = ok && D.by_logprob ? D.by_logprob[(size_t)row * R.n_tokens + tid] : 0.0f;
  }
  __syncthreads();
  float total = 0.0f;
  for (uint32_t k = 0; k < R.n_tokens; ++k) total += g[k];
  for (uint32_t v = tid; v < R.V; v += THREADS) {
    const float x = allowed<T>(R, row, v);
    float d = 0.0f;
    if (x != -INF) {
      const float lp = (x - most) * inv - ln, p = expf(lp);
      d = -p * total;
      if (!(p == 0.0f)) d -= gh * p * (lp + h);
      for (uint32_t k = 0; k < R.n_tokens; ++k)
        if (tok[k] == (int32_t)v) d += g[k];
      d *= inv;
    }
    put(static_cast<T*>(D.out) + (size_t)row * D.stride + v, d);
  }
}

fmt_status check_rows(const Rows& R, fmt_dtype dtype) {
  if (!R.logits) return refuse("NULL argument");
  if (dtype != FMT_BF16 && dtype != FMT_FP32) return refuse("unknown dtype");
  if (R.V == 0 || R.V > (1u << 30)) return refuse("V out of range");
  if (R.rows > (1u << 24)) return refuse("rows out of range");
  if (R.stride < R.V || (R.mask && R.mask_stride < ((size_t)R.V + 31) / 32)) return refuse("a stride is too small");
  if (R.n_tokens > FMT_MAX_GIVEN_TOKENS) return refuse("more than FMT_MAX_GIVEN_TOKENS tokens a row");
  if (R.n_tokens && !R.tokens) return refuse("NULL tokens");
  if (misaligned(R.logits, dtype == FMT_BF16 ? 2 : 4) || misaligned(R.mask, 4) || misaligned(R.temperature, 4) || misaligned(R.tokens, 4))
    return refuse("a pointer is not aligned to its elements");
  return FMT_OK;
}

}  // namespace

extern "C" fmt_status fmt_token_logprobs(const void* logits_dev, fmt_dtype dtype, uint32_t rows, uint32_t V, size_t row_stride_elems,
                                         const uint32_t* mask_dev, size_t mask_stride_words, const float* temperature_dev,
                                         const int32_t* tokens_dev, uint32_t n_tokens, uint32_t n_top, float* logprobs_dev, float* norm_dev,
                                         float* entropy_dev, int32_t* top_ids_dev, float* top_logprobs_dev, int32_t* status_dev,
                                         void* stream) {
  const Rows R{rows, V, logits_dev, row_stride_elems, mask_dev, mask_stride_words, temperature_dev, tokens_dev, n_tokens};
  if (fmt_status s = check_rows(R, dtype)) return s;
  if (n_top > FMT_MAX_TOP) return refuse("more than FMT_MAX_TOP alternatives");
  for (const void* p : {(const void*)logprobs_dev, (const void*)norm_dev, (const void*)entropy_dev, (const void*)top_ids_dev, (const void*)top_logprobs_dev,
                        (const void*)status_dev})
    if (misaligned(p, 4)) return refuse("a pointer is not aligned to its elements");
  if (rows == 0) return FMT_OK;
  if (fmt_status s = reachable({logits_dev, mask_dev, temperature_dev, n_tokens ? tokens_dev : nullptr, logprobs_dev, norm_dev, entropy_dev,
                                top_ids_dev, top_logprobs_dev, status_dev}))
    return s;
  const Outputs O{top_ids_dev || top_logprobs_dev ? n_top : 0u, logprobs_dev, norm_dev, entropy_dev, top_ids_dev, top_logprobs_dev, status_dev};
  auto* k = dtype == FMT_BF16 ? logprobs_kernel<uint16_t> : logprobs_kernel<float>;
  return launch_result(launch_overlapped(k, dim3(rows), dim3(THREADS), 0, (cudaStream_t)stream, R, O));
}

extern "C" fmt_status fmt_token_logprobs_backward(const void* logits_dev, fmt_dtype dtype, uint32_t rows, uint32_t V, size_t row_stride_elems,
                                                  const uint32_t* mask_dev, size_t mask_stride_words, const float* temperature_dev,
                                                  const int32_t* tokens_dev, uint32_t n_tokens, const float* norm_dev,
                                                  const float* entropy_dev, const float* grad_logprobs_dev, const float* grad_entropy_dev,
                                                  void* grad_logits_dev, size_t grad_stride_elems, void* stream) {
  const Rows R{rows, V, logits_dev, row_stride_elems, mask_dev, mask_stride_words, temperature_dev, tokens_dev, n_tokens};
  if (fmt_status s = check_rows(R, dtype)) return s;
  if (!norm_dev || !grad_logits_dev) return refuse("NULL argument");
  if (grad_entropy_dev && !entropy_dev) return refuse("the entropy's gradient needs the entropy");
  if (grad_stride_elems < V) return refuse("a stride is too small");
  if (grad_logits_dev == logits_dev && grad_stride_elems != row_stride_elems) return refuse("a gradient in the logits' place needs their stride");
  if (misaligned(grad_logits_dev, dtype == FMT_BF16 ? 2 : 4)) return refuse("a pointer is not aligned to its elements");
  for (const float* p : {norm_dev, entropy_dev, grad_logprobs_dev, grad_entropy_dev})
    if (misaligned(p, 4)) return refuse("a pointer is not aligned to its elements");
  if (rows == 0) return FMT_OK;
  if (fmt_status s = reachable({logits_dev, mask_dev, temperature_dev, n_tokens ? tokens_dev : nullptr, norm_dev, entropy_dev, grad_logprobs_dev,
                                grad_entropy_dev, grad_logits_dev}))
    return s;
  const Gradients D{norm_dev, entropy_dev, grad_logprobs_dev, grad_entropy_dev, grad_logits_dev, grad_stride_elems};
  auto* k = dtype == FMT_BF16 ? logprobs_backward_kernel<uint16_t> : logprobs_backward_kernel<float>;
  return launch_result(launch_overlapped(k, dim3(rows), dim3(THREADS), 0, (cudaStream_t)stream, R, D));
}
