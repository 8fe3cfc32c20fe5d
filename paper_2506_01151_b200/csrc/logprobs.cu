// Log probabilities, entropy and likeliest tokens of the rows' distributions under their masks, and the gradient.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/fmt.h"
#include "kernels.h"
#include "op_args.h"

using namespace fmt;

namespace {

constexpr float INF = __builtin_huge_valf();
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
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = __bfloat16_as_ushort(__float2bfloat16_rn(x)); }

__device__ __forceinline__ float ex2(float x) {  // below 2^-126: 0, which sums that begin at 1 do not notice
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ------------------------------------------------------------------------------------------------ rows in units of 32 bytes
//
// A row may begin at any address: units are counted from its first 32-byte boundary on, and the few logits before it and behind the
// last whole unit ("edges") are taken one at a time.  A unit has as many logits as a number of the mask has bits (16 of bf16, 8
// of fp32), and begins `head` bits behind number i: its bits come from numbers i and i + 1.

struct Unit {
  uint32_t v[8];
};
// Loads that are left out leave what was there.
__device__ __forceinline__ void load_if(uint32_t not_zero, const void* p, Unit& u) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %9, 0;\n@p ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n}"
               : "+r"(u.v[0]), "+r"(u.v[1]), "+r"(u.v[2]), "+r"(u.v[3]), "+r"(u.v[4]), "+r"(u.v[5]), "+r"(u.v[6]), "+r"(u.v[7])
               : "l"(p), "r"(not_zero));
}
__device__ __forceinline__ uint32_t load_below(uint32_t i, uint32_t n, const uint16_t* p) {  // 0 unless i < n
  uint32_t x = 0u;
  asm volatile("{\n.reg .pred p;\nsetp.lt.u32 p, %2, %3;\n@p ld.global.u16 %0, [%1];\n}" : "+r"(x) : "l"(p), "r"(i), "r"(n));
  return x;
}
__device__ __forceinline__ uint32_t load_below(uint32_t i, uint32_t n, const uint8_t* p) {
  uint32_t x = 0u;
  asm volatile("{\n.reg .pred p;\nsetp.lt.u32 p, %2, %3;\n@p ld.global.u8 %0, [%1];\n}" : "+r"(x) : "l"(p), "r"(i), "r"(n));
  return x;
}
__device__ __forceinline__ void store_unit(void* p, const Unit& u) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(u.v[0]), "r"(u.v[1]), "r"(u.v[2]), "r"(u.v[3]), "r"(u.v[4]),
               "r"(u.v[5]), "r"(u.v[6]), "r"(u.v[7])
               : "memory");
}

template <size_t SIZE>
struct MaskNumber;
template <>
struct MaskNumber<2> {
  using type = uint16_t;
};
template <>
struct MaskNumber<4> {
  using type = uint8_t;
};

template <typename T>
struct Row {
  static constexpr uint32_t W = 32u / sizeof(T), ALL = (1u << W) - 1u;  // logits of a unit
  using Number = typename MaskNumber<sizeof(T)>::type;
  const T* x;
  const uint32_t* mask;  // or nullptr
  uint32_t V, head, units, edges;

  __device__ __forceinline__ Row(const Rows& R, uint32_t row)
      : x(static_cast<const T*>(R.logits) + (size_t)row * R.stride), mask(R.mask ? R.mask + (size_t)row * R.mask_stride : nullptr), V(R.V) {
    head = min(V, (uint32_t)((0u - (uint32_t)reinterpret_cast<uintptr_t>(x)) & 31u) / (uint32_t)sizeof(T));
    units = (V - head) / W;
    edges = V - units * W;
  }
  __device__ __forceinline__ uint32_t edge(uint32_t i) const { return i < head ? i : i + units * W; }
  __device__ __forceinline__ bool allows(uint32_t v) const { return !mask || (mask[v >> 5] >> (v & 31u)) & 1u; }
  __device__ __forceinline__ float at(uint32_t v) const { return allows(v) ? to_f32(x[v]) : -INF; }  // -inf: not allowed
  __device__ __forceinline__ uint32_t first(uint32_t unit) const { return head + unit * W; }
  template <bool ALIGNED = false>  // (head is 0)
  __device__ __forceinline__ uint32_t bits(uint32_t unit) const {  // none behind the last unit
    const Number* const at = reinterpret_cast<const Number*>(mask) + unit;
    uint32_t b = load_below(unit, units, at);
    if (!ALIGNED && head) b = (b | load_below(unit, units, at + 1) << W) >> head & ALL;  // (a unit ends before V: it is there)
    return b;
  }
  __device__ __forceinline__ void load(uint32_t unit, Unit& u, uint32_t not_zero = 1u) const { load_if(not_zero, x + first(unit), u); }
};

// What the mask forbids becomes -inf.  `of` holds, for every value that the bits of half a unit (bf16: 8, fp32: 4) may have, the bits
// of that half to keep.
template <typename T>
struct Keep {
  static constexpr uint32_t BITS = 16u / sizeof(T);
  uint4 of[1u << BITS];
};
template <typename T>
__device__ __forceinline__ uint4 keep_of(uint32_t bits) {
  auto word = [&](uint32_t i) {
    if (sizeof(T) == 4) return (bits >> i) & 1u ? 0xFFFFFFFFu : 0u;
    return ((bits >> (2u * i)) & 1u ? 0x0000FFFFu : 0u) | ((bits >> (2u * i + 1u)) & 1u ? 0xFFFF0000u : 0u);
  };
  return make_uint4(word(0), word(1), word(2), word(3));
}
template <typename T>
__device__ __forceinline__ void forbid(Unit& x, const uint4& low, const uint4& high) {
  constexpr uint32_t n = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
  const uint32_t k[8] = {low.x, low.y, low.z, low.w, high.x, high.y, high.z, high.w};
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) x.v[i] = (x.v[i] & k[i]) | (n & ~k[i]);
}
template <typename T>
__device__ __forceinline__ void forbid(Unit& x, const Keep<T>& keep, uint32_t bits) {
  forbid<T>(x, keep.of[bits & ((1u << Keep<T>::BITS) - 1u)], keep.of[bits >> Keep<T>::BITS]);
}
template <typename T>
__device__ __forceinline__ void forbid(Unit& x, uint32_t bits) {  // the same without a table
  forbid<T>(x, keep_of<T>(bits & ((1u << Keep<T>::BITS) - 1u)), keep_of<T>(bits >> Keep<T>::BITS));
}
__device__ __forceinline__ float value(const Unit& x, uint32_t i, uint16_t) {
  return __uint_as_float(i % 2 ? x.v[i / 2] & 0xFFFF0000u : x.v[i / 2] << 16);
}
__device__ __forceinline__ float value(const Unit& x, uint32_t i, float) { return __uint_as_float(x.v[i]); }
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {  // (of a NaN and a number: the number)
  uint32_t m;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
  return m;
}
template <uint32_t N>
__device__ __forceinline__ float largest(const Unit (&x)[N], uint16_t) {
  uint32_t m = 0xFF80FF80u;
#pragma unroll
  for (uint32_t u = 0; u < N; ++u)
#pragma unroll
    for (uint32_t i = 0; i < 8; i += 2) m = max_pair(m, max_pair(x[u].v[i], x[u].v[i + 1]));
  return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
}
template <uint32_t N>
__device__ __forceinline__ float largest(const Unit (&x)[N], float) {
  float m = -INF;
#pragma unroll
  for (uint32_t u = 0; u < N; ++u)
#pragma unroll
    for (uint32_t i = 0; i < 8; i += 2) m = fmaxf(m, fmaxf(__uint_as_float(x[u].v[i]), __uint_as_float(x[u].v[i + 1])));
  return m;
}

// Two values at a time.
__device__ __forceinline__ uint64_t two(float lo, float hi) {
  uint64_t p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
  return p;
}
__device__ __forceinline__ float lo(uint64_t p) { return __uint_as_float((uint32_t)p); }
__device__ __forceinline__ float hi(uint64_t p) { return __uint_as_float((uint32_t)(p >> 32)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// A unit's values in pairs, nothing below LOW (-inf becomes LOW; a NaN stays).  LOW lies so far below a row's largest logit that
// its probability is 0, and is finite, so that 0 times what is made of it is 0.  This holds for rows whose largest logit is between
// LOW / 10 and -LOW / 10 and whose temperature is between 2e-6 and 1e8 (`ordinary`): 0.9 x 2^40 x 1e-8 is 9,900 powers of two, and
// 1.1 x 2^40 x 1e6 a number.  In others every value is looked at.
constexpr float LOW = -0x1p40f;
__device__ __forceinline__ bool ordinary(float largest, float c) { return fabsf(largest) < LOW * -0.1f && c > 1e-8f && c < 1e6f; }
__device__ __forceinline__ uint64_t pair_of(const Unit& x, uint32_t i, uint16_t) {
  uint32_t w;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(w) : "r"(x.v[i]), "r"(0xD380D380u));
  return two(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ uint64_t pair_of(const Unit& x, uint32_t i, float) {
  float a = __uint_as_float(x.v[2 * i]), b = __uint_as_float(x.v[2 * i + 1]);
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(a), "f"(LOW));
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(b) : "f"(b), "f"(LOW));
  return two(a, b);
}

// A thread's units from, from + step, ..., N at a time: the next N are on their way, and the bits of those after them, while
// work(first, units) is at some.  What the mask forbids, and what is behind the row's last unit, is -inf.  SKIP: without work where
// nothing is allowed.
template <typename T, bool MASK, bool ALIGNED, bool SKIP, uint32_t N, class F>
__device__ __forceinline__ void row_turns_of(const Row<T>& row, uint32_t from, uint32_t step, const Keep<T>& keep, F work) {
  const uint32_t n = row.units, stride = N * step;
  auto ask_bits = [&](uint32_t i, uint32_t (&to)[N]) {
#pragma unroll
    for (uint32_t u = 0; u < N; ++u) to[u] = MASK ? row.template bits<ALIGNED>(i + u * step) : i + u * step < n ? Row<T>::ALL : 0u;
  };
  auto ask = [&](uint32_t i, const uint32_t (&bits)[N], Unit (&to)[N]) {
#pragma unroll
    for (uint32_t u = 0; u < N; ++u) row.load(i + u * step, to[u], bits[u]);
  };
  Unit xa[N] = {}, xb[N] = {};
  uint32_t ba[N], bb[N];
  auto turn = [&](uint32_t i, Unit (&x)[N], uint32_t (&bits)[N], Unit (&next)[N], const uint32_t (&ahead)[N]) {
    ask(i + stride, ahead, next);
    uint32_t any = 1u;
    if (MASK) {
      if (SKIP) any = 0u;
#pragma unroll
      for (uint32_t u = 0; u < N; ++u) {
        forbid(x[u], keep, bits[u]);
        if (SKIP) any |= bits[u];
      }
    } else if (i + (N - 1u) * step >= n) {
#pragma unroll
      for (uint32_t u = 1; u < N; ++u) forbid<T>(x[u], bits[u]);
    }
    ask_bits(i + 2u * stride, bits);
    if (any) work(i, x);
  };
  ask_bits(from, ba);
  ask(from, ba, xa);
  ask_bits(from + stride, bb);
  for (uint32_t i = from; i < n; i += 2u * stride) {
    turn(i, xa, ba, xb, bb);
    if (i + stride < n) turn(i + stride, xb, bb, xa, ba);
  }
}

template <typename T, bool MASK, bool SKIP, uint32_t N, class F>
__device__ __forceinline__ void row_turns(const Row<T>& row, uint32_t from, uint32_t step, const Keep<T>& keep, F work) {
  if (MASK && row.head == 0) row_turns_of<T, MASK, true, SKIP, N>(row, from, step, keep, work);
  else row_turns_of<T, MASK, false, SKIP, N>(row, from, step, keep, work);
}

// ------------------------------------------------------------------------------------------------ sums of a row
//
// One pass: s = sum of 2^d and t = sum of 2^d d with d = (x - m) log2(e) / T and m the largest logit so far, rescaled when m grows.
// (x - m is formed first: of two logits of the type's lowest value it is 0, where a product with either would overflow.)
// The entropy is ln s - (t / s) ln 2, two parts of one sign.  A NaN or +inf among the allowed logits makes s NaN, and nothing else does.

// (x - m) / T.  x - m may be beyond fp32 where that over T is not, and so may 1 / T be below its normal numbers: from T = 1 on a quarter of
// all three is taken, which is exact (of ordinary logits: the same bits).  Below 1, what is beyond fp32 stays so.  The pass takes c alone, but
// for m, where it grows (2,048 rows of 128,256 bf16: 99.1 us, and 98.5 when it took x - m there, both before its sums were apart).
constexpr float LOG2E = 1.44269504f;
struct Heat {
  float part, c, c_part;  // 1/4 or 1, log2(e) / T, and that over part
  __device__ __forceinline__ explicit Heat(float temperature) {
    part = temperature >= 1.0f ? 0.25f : 1.0f;
    c_part = inv(temperature) * LOG2E, c = part * c_part;
  }
  __device__ __forceinline__ float inv(float temperature) const { return __fdiv_rn(1.0f, part * temperature); }  // 1 / T over part
  __device__ __forceinline__ float apart(float x, float m) const { return __fsub_rn(part * x, part * m); }
  __device__ __forceinline__ float exponent(float x, float m) const { return apart(x, m) * c_part; }  // (x - m) log2(e) / T
};

struct Sums {
  float m = -INF, s = 0.0f, t = 0.0f;

  __device__ __forceinline__ void grow(float to, const Heat& heat) {  // a larger m
    if (!(to > m)) return;
    if (m > -INF) {
      const float d = heat.exponent(m, to), f = ex2(d);
      t = f > 0.0f ? (t + s * d) * f : s * 0.0f;  // (s * 0: what is NaN stays NaN)
      s *= f;
    }
    m = to;
  }
  __device__ __forceinline__ float base() const { return m > -INF ? m : 0.0f; }
  __device__ __forceinline__ void add(float x, float base, const Heat& heat) {
    const float d = heat.exponent(x, base), p = ex2(d);
    s += p;
    t = fmaf(p, fmaxf(d, -1024.0f), t);  // (d may be -inf; p is 0 below -1024)
  }
  // Units whose largest logits m has grown for, added up before they come to what is there: terms that are alike would all be rounded the
  // same way, by up to half a unit of the whole sum (2^18 and 2^20 equal logits to a block: ln S off by 7e-6 and 3e-5, and so by 1e-6 and 2e-6;
  // 2,048 rows of 128,256 bf16 99.3 us, and so 100.8).
  template <typename T, uint32_t N>
  __device__ __forceinline__ void add(const Unit (&x)[N], const Heat& heat) {
    const float b = base(), c = heat.c;
    if (ordinary(m, c)) {
      const uint64_t b2 = two(-b, -b), c2 = two(c, c);
      uint64_t s2 = 0, t2 = 0;
#pragma unroll
      for (uint32_t u = 0; u < N; ++u)
#pragma unroll
        for (uint32_t e = 0; e < 16u / sizeof(T); ++e) {
          const uint64_t d = mul2(add2(pair_of(x[u], e, T()), b2), c2), p = two(ex2(lo(d)), ex2(hi(d)));
          s2 = add2(s2, p);
          t2 = fma2(p, d, t2);
        }
      s += lo(s2) + hi(s2), t += lo(t2) + hi(t2);
    } else {
      const float s0 = s, t0 = t;
      s = t = 0.0f;
#pragma unroll
      for (uint32_t u = 0; u < N; ++u)
#pragma unroll
        for (uint32_t e = 0; e < 32u / sizeof(T); ++e) add(value(x[u], e, T()), b, heat);
      s += s0, t += t0;
    }
  }
  template <uint32_t LANES>
  __device__ __forceinline__ void join_lanes(const Heat& heat) {  // of a warp's first so many lanes, all of which get the result
    float most = m;
#pragma unroll
    for (uint32_t o = LANES / 2; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    grow(most, heat);
#pragma unroll
    for (uint32_t o = LANES / 2; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o), t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
  }
};

// Logits in the order wanted as whole numbers: larger first, of equal ones (0 and -0 are equal) the lower id.  0: none.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t v) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (0xFFFFFFFFu - v);
}
__device__ __forceinline__ uint32_t key_token(uint64_t k) { return 0xFFFFFFFFu - (uint32_t)k; }
__device__ __forceinline__ float key_logit(uint64_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ uint64_t max_key(uint64_t a, uint64_t b) { return a > b ? a : b; }

// ------------------------------------------------------------------------------------------------ the forward pass
//
// A cluster of 1 to 8 thread blocks to a row; block r takes units r * THREADS + thread, and so on in steps of the whole cluster.
//
// The likeliest tokens.  In the pass over the row each thread keeps the first units with its largest logit.  The threads make
// 128 groups; of the groups' largest keys (logit, lowest id) the n_top-th is a bound that n_top logits at least reach, and only
// the n_top groups whose own largest reaches it hold any: their units alone are read again (L2), and what reaches the bound is
// listed and put in order.  A row is passed once, and n_top 128ths of it twice (20: a sixth, 32: a quarter), whatever its order; where more
// reach the bound than the list holds, those groups' units are read a third time.

constexpr uint32_t THREADS = 256, WARPS = THREADS / 32, UNROLL = 2, BACK_UNROLL = 1, BACK_PER_SM = 4;
// Blocks to an SM: four have 64 registers a thread, which a masked pass outgrows (masked rows of 128,256 bf16, us with three and with four, without
// and with 20 alternatives: 48 rows 5.9 and 7.0, 12.4 and 14.1; 256 rows, where four run two blocks to a row at a time, 21.4 and 17.7, 30.2
// and 28.8; 2,048 rows 87.6 and 88.6, 129 and 147; 1,024 rows of fp32 75 and 71, 108 and 104.  Unmasked, 2,048 rows: 101 and 98.5).
constexpr uint32_t per_sm(bool masked) { return masked ? 3u : 4u; }
constexpr uint32_t GROUPS = 128, GROUP = THREADS / GROUPS;
constexpr uint32_t MAX_CLUSTER = 8;
constexpr uint32_t SORT = THREADS;                // listed logits that are put in order by counting
constexpr uint32_t LISTED = SORT + THREADS * 16u;  // what one round of re-reading may add

struct TopShared {
  alignas(16) uint64_t group[GROUPS];
  alignas(16) uint64_t list[LISTED + 8];
  uint64_t best[FMT_MAX_TOP];
  uint64_t join[MAX_CLUSTER * FMT_MAX_TOP];  // of the cluster's blocks, in the first one's memory
  uint64_t bound;
  uint32_t chosen[GROUPS];
  uint32_t n_listed, n_chosen;
};
struct JoinShared {
  Sums warps[WARPS];
  Sums blocks[MAX_CLUSTER];  // in the first one's memory
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t in_first_block(const void* p) {  // the same variable in the memory of the cluster's first block
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)));
  return a;
}
__device__ __forceinline__ void put_remote(uint32_t addr, float x) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(x) : "memory"); }
__device__ __forceinline__ void put_remote(uint32_t addr, uint64_t x) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(x) : "memory"); }

// The `want` largest of the listed keys, in order, into best; the rest of best is 0.  All threads of the block.
__device__ void best_of_list(TopShared& P, uint32_t want) {
  const uint32_t tid = threadIdx.x, n = P.n_listed;
  if (tid < want) P.best[tid] = 0;
  __syncthreads();
  if (n <= SORT) {
    if (tid < n) {
      const uint64_t mine = P.list[tid];
      uint32_t above = 0;
      for (uint32_t i = 0; i < n; i += 8) {  // (eight at a time: each is 30 cycles away)
        ulonglong2 k[4];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) k[u] = *reinterpret_cast<const ulonglong2*>(P.list + i + 2 * u);
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) above += (i + 2 * u < n && k[u].x > mine) + (i + 2 * u + 1 < n && k[u].y > mine);
      }
      if (above < want) P.best[above] = mine;
    }
    __syncthreads();
    return;
  }
  uint64_t last = ~0ull;
  for (uint32_t k = 0; k < want; ++k) {  // one at a time: n is above SORT, so there are enough
    uint64_t most = 0;
    for (uint32_t i = tid; i < n; i += THREADS) {
      const uint64_t key = P.list[i];
      if (key < last) most = max_key(most, key);
    }
    for (uint32_t o = 16; o; o >>= 1) most = max_key(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    if (tid % 32u == 0) P.group[tid / 32u] = most;
    __syncthreads();
    most = 0;
    for (uint32_t i = 0; i < WARPS; ++i) most = max_key(most, P.group[i]);
    last = most;
    if (tid == 0) P.best[k] = most;
    __syncthreads();
  }
}

template <typename T, bool MASK>
__device__ __forceinline__ void find_top(const Row<T>& row, const Keep<T>& keep, uint32_t from, uint32_t step, uint32_t edges, uint64_t mine, uint32_t want,
                                         TopShared& P) {
  const uint32_t tid = threadIdx.x;
  for (uint32_t o = 1; o < GROUP; o <<= 1) mine = max_key(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, o));
  if (tid % GROUP == 0) P.group[tid / GROUP] = mine;
  if (tid == 0) P.n_listed = 0, P.n_chosen = 0, P.bound = 1, P.best[0] = 0;
  __syncthreads();
  uint32_t above = 0;
  if (tid < GROUPS) {
    mine = P.group[tid];
#pragma unroll 8
    for (uint32_t i = 0; i < GROUPS; i += 2) {
      const ulonglong2 k = *reinterpret_cast<const ulonglong2*>(P.group + i);
      above += (k.x > mine) + (k.y > mine);
    }
    if (mine && above < want) {
      P.chosen[atomicAdd(&P.n_chosen, 1u)] = tid;
      if (above == want - 1) P.bound = mine;
      if (above == 0) P.best[0] = mine;
    }
  }
  __syncthreads();
  if (want == 1) return;  // the largest of all
  uint64_t bound = P.bound;
  const uint32_t rounds_of = (row.units + step - 1) / step;  // units of a thread, at most
  const uint32_t items = P.n_chosen * GROUP * rounds_of;
  const uint32_t each = GROUP * rounds_of;
  auto offer = [&](float x, uint32_t v) {
    const uint64_t key = order_key(x, v);
    if (x > -INF && key >= bound) {
      const uint32_t at = atomicAdd(&P.n_listed, 1u);
      if (at < LISTED) P.list[at] = key;
    }
  };
  auto unit_of = [&](uint32_t item) {
    const uint32_t rest = item % each;
    return item < items ? from - tid + P.chosen[item / each] * GROUP + rest % GROUP + rest / GROUP * step : 0xFFFFFFFFu;
  };
  auto reaches = [&](Unit& x, uint32_t bits) {
    if (MASK) forbid(x, keep, bits);
    const Unit one[1] = {x};
    return bits && (largest(one, T()) >= key_logit(bound) || bound == 1);
  };
  auto offer_unit = [&](uint32_t unit, const Unit& x) {
#pragma unroll
    for (uint32_t i = 0; i < Row<T>::W; ++i) offer(value(x, i, T()), row.first(unit) + i);
  };
  if (tid < edges) offer(row.at(row.edge(tid)), row.edge(tid));
  constexpr uint32_t AT_ONCE = 4;
  for (uint32_t base = 0; base < items; base += AT_ONCE * THREADS) {
    Unit x[AT_ONCE];
    uint32_t unit[AT_ONCE], bits[AT_ONCE];
#pragma unroll
    for (uint32_t u = 0; u < AT_ONCE; ++u) {
      unit[u] = unit_of(base + u * THREADS + tid);
      row.load(unit[u], x[u], unit[u] < row.units);
      bits[u] = MASK ? row.bits(unit[u]) : unit[u] < row.units ? Row<T>::ALL : 0u;
    }
    uint32_t hits = 0u;
#pragma unroll
    for (uint32_t u = 0; u < AT_ONCE; ++u) hits |= reaches(x[u], bits[u]) ? 1u << u : 0u;
#pragma unroll 1
    while (hits) {  // (few have one)
      const uint32_t u = __ffs(hits) - 1u;
      hits &= hits - 1u;
      Unit y = x[0];
      uint32_t at = unit[0];
#pragma unroll
      for (uint32_t k = 1; k < AT_ONCE; ++k)
        if (u == k) y = x[k], at = unit[k];
      offer_unit(at, y);
    }
  }
  __syncthreads();
  if (P.n_listed > LISTED) {  // many of the largest logits are in few groups: again, with the list cut down in time
    __syncthreads();
    if (tid == 0) P.n_listed = 0;
    __syncthreads();
    if (tid < edges) offer(row.at(row.edge(tid)), row.edge(tid));
    for (uint32_t base = 0; base < items; base += THREADS) {
      const uint32_t unit = unit_of(base + tid);
      if (unit < row.units) {
        Unit x;
        row.load(unit, x);
        if (reaches(x, MASK ? row.bits(unit) : Row<T>::ALL)) offer_unit(unit, x);
      }
      __syncthreads();
      if (P.n_listed > SORT) {
        best_of_list(P, want);
        if (tid < want) P.list[tid] = P.best[tid];
        if (tid == 0) P.n_listed = want, P.bound = P.best[want - 1];
        __syncthreads();
        bound = P.bound;
      }
      __syncthreads();
    }
  }
  best_of_list(P, want);
}

template <typename T, bool MASK, bool TOP>
__global__ void __launch_bounds__(THREADS, per_sm(MASK)) logprobs_kernel(const Rows R, const Outputs O, const uint32_t cluster) {
  __shared__ JoinShared J;
  __shared__ Keep<T> keep;  // (of masked rows)
  __shared__ __align__(16) uint8_t top_raw[TOP ? sizeof(TopShared) : 16];
  TopShared& P = *reinterpret_cast<TopShared*>(top_raw);
  const uint32_t tid = threadIdx.x;
  if (cluster > 1) cluster_arrive();
  if (MASK) {
    if (tid < sizeof(Keep<T>) / sizeof(uint4)) keep.of[tid] = keep_of<T>(tid);
    __syncthreads();
  }
  before_me();
  const uint32_t rank = cluster > 1 ? cluster_rank() : 0u, row_id = blockIdx.x / cluster;
  const Row<T> row(R, row_id);
  const Heat heat(R.temperature ? R.temperature[row_id] : 1.0f);
  int32_t token = -1;  // (asked for now, wanted at the end)
  float token_logit = 0.0f;
  if (rank == 0 && tid < R.n_tokens) {
    token = R.tokens[(size_t)row_id * R.n_tokens + tid];
    if (token >= 0 && token < (int64_t)R.V) token_logit = row.at((uint32_t)token);
  }

  Sums a;
  uint32_t where = 0xFFFFFFFFu;  // the first of the units among which the thread's largest logit is, or, behind all units, an edge
  const uint32_t edges = rank == 0 ? row.edges : 0u;
  if (tid < edges && row.edge(tid) < row.head) {
    const float x = row.at(row.edge(tid));
    if (x > a.m) where = row.units + tid;
    a.grow(x, heat), a.add(x, a.base(), heat);
  }

  const uint32_t from = rank * THREADS + tid, step = cluster * THREADS;
  row_turns<T, MASK, true, UNROLL>(row, from, step, keep, [&](uint32_t i, const Unit (&x)[UNROLL]) {
    const float most = largest(x, T());
    if (most > a.m) {
      if (TOP) where = i;
      a.grow(most, heat);
    }
    a.template add<T, UNROLL>(x, heat);
  });
  if (tid < edges && row.edge(tid) >= row.head) {
    const float x = row.at(row.edge(tid));
    if (x > a.m) where = row.units + tid;
    a.grow(x, heat), a.add(x, a.base(), heat);
  }

  if (TOP) {
    uint64_t mine = 0;
    if (where != 0xFFFFFFFFu) {
      if (where >= row.units) {
        mine = order_key(a.m, row.edge(where - row.units));
      } else {
        uint32_t at = 0xFFFFFFFFu;
#pragma unroll
        for (uint32_t u = UNROLL; u-- > 0;) {
          Unit x = {};
          row.load(where + u * step, x, where + u * step < row.units);
          if (MASK) forbid(x, keep, row.bits(where + u * step));
#pragma unroll
          for (uint32_t e = Row<T>::W; e-- > 0;)
            if (value(x, e, T()) == a.m && where + u * step < row.units) at = u * step * Row<T>::W + e;
        }
        mine = order_key(a.m, row.first(where) + at);
      }
    }
    find_top<T, MASK>(row, keep, from, step, edges, mine, O.n_top, P);
  }

  const float temperature = R.temperature ? *const_cast<const volatile float*>(R.temperature + row_id) : 1.0f;  // (not kept in the pass)
  a.join_lanes<32>(heat);
  if (tid % 32u == 0) J.warps[tid / 32u] = a;
  __syncthreads();
  if (tid < 32) {
    a = tid < WARPS ? J.warps[tid] : Sums();
    a.join_lanes<WARPS>(heat);
  }
  if (cluster > 1) {
    cluster_wait();  // the first block has begun: its memory may be written
    if (tid == 0) {
      const uint32_t at = in_first_block(&J.blocks[rank]);
      put_remote(at, a.m), put_remote(at + 4u, a.s), put_remote(at + 8u, a.t);
    }
    if (TOP && tid < O.n_top) put_remote(in_first_block(&P.join[rank * O.n_top + tid]), P.best[tid]);
    cluster_arrive();
    cluster_wait();
    if (rank) return;
    if (tid < 32) {
      a = tid < cluster ? J.blocks[tid] : Sums();
      a.join_lanes<MAX_CLUSTER>(heat);
    }
    if (TOP) {
      // the blocks' lists are in order: a key's place is its own in its list and, of every other one, how many are above
      const uint32_t n = cluster * O.n_top;
      if (tid < O.n_top) P.best[tid] = 0;
      __syncthreads();
      if (tid < n && P.join[tid]) {
        const uint64_t mine = P.join[tid];
        uint32_t above = 0, at[MAX_CLUSTER] = {};  // by halves, in all lists at once
#pragma unroll
        for (uint32_t half = FMT_MAX_TOP; half; half /= 2)
#pragma unroll
          for (uint32_t b = 0; b < MAX_CLUSTER; ++b) {
            const uint32_t to = at[b] + half;
            if (b < cluster && to <= O.n_top && P.join[b * O.n_top + to - 1] > mine) at[b] = to;
          }
#pragma unroll
        for (uint32_t b = 0; b < MAX_CLUSTER; ++b) above += at[b];
        if (above < O.n_top) P.best[above] = mine;
      }
    }
  }
  if (tid == 0) J.warps[0] = a;
  __syncthreads();
  a = J.warps[0];

  const float nan = __int_as_float(0x7FC00000);
  const bool bad = a.s != a.s || !(temperature >= 0x1p-126f && temperature < INF);  // (below, log2(e) / T overflows)
  const float ln = bad ? nan : logf(a.s);  // (-inf of nothing)
  const float inv = heat.inv(temperature);
  auto logprob = [&](float x) { return bad ? nan : x == -INF ? -INF : heat.apart(x, a.m) * inv - ln; };
  const bool wrong = token < -1 || token >= (int64_t)R.V;
  if (tid < R.n_tokens && O.logprobs) O.logprobs[(size_t)row_id * R.n_tokens + tid] = token == -1 ? 0.0f : wrong ? nan : logprob(token_logit);
  if (TOP && tid < O.n_top) {
    const uint64_t key = P.best[tid];
    const bool there = key && !bad;
    if (O.top_ids) O.top_ids[(size_t)row_id * O.n_top + tid] = there ? (int32_t)key_token(key) : -1;
    if (O.top_logprobs) O.top_logprobs[(size_t)row_id * O.n_top + tid] = there ? logprob(key_logit(key)) : bad ? nan : -INF;
  }
  if (tid < 32) {
    const bool any_wrong = __any_sync(0xFFFFFFFFu, wrong);
    if (tid == 0) {
      if (O.norm) O.norm[2 * (size_t)row_id] = bad ? nan : a.m, O.norm[2 * (size_t)row_id + 1] = ln;
      if (O.entropy) O.entropy[row_id] = bad ? nan : a.s > 0.0f ? ln - a.t / a.s * 0.693147181f : 0.0f;
      if (O.status) O.status[row_id] = bad || any_wrong ? FMT_ERR_INVALID_ARG : FMT_OK;
    }
  }
}

// ------------------------------------------------------------------------------------------------ the backward pass
//
// grad = (p (A + B lp2) + the g of the given tokens) / T with lp2 = log2 p, A = -(sum g + g_H H) and B = -g_H ln 2.  In ordinary rows 1 / T is
// part of A, B and g; in others, where that may be beyond fp32 (1 / T is up to 2^126, and so may the incoming gradients be), it comes last, and
// what p = 0 is multiplied with is not looked at.  A row's sizes decide, not a logit's, and the loop costs nothing for it (2,048 rows of 128,256
// bf16: 166 us, 168 before; 48 rows of 50,001 fp32 with three given tokens 7.3, 7.1 before).  A gradient at another address modulo 32 than
// the logits is written by single values (1,532 us), and each given token is compared with each unit (5: 175 us, 32: 321).
// The given tokens' own logits decide whether they count: all of a cluster's blocks have read them before the first writes,
// since the gradient may take the logits' place.

template <typename T, bool MASK>
__global__ void __launch_bounds__(THREADS, BACK_PER_SM) logprobs_backward_kernel(const Rows R, const Gradients D, const uint32_t cluster) {
  __shared__ int32_t tok[FMT_MAX_GIVEN_TOKENS];
  __shared__ float g[FMT_MAX_GIVEN_TOKENS];
  __shared__ Keep<T> keep;
  const uint32_t tid = threadIdx.x;
  if (MASK && tid < sizeof(Keep<T>) / sizeof(uint4)) keep.of[tid] = keep_of<T>(tid);  // (used behind a barrier)
  before_me();
  const uint32_t rank = cluster > 1 ? cluster_rank() : 0u, row_id = blockIdx.x / cluster;
  const Row<T> row(R, row_id);
  const float temperature = R.temperature ? R.temperature[row_id] : 1.0f;
  const Heat heat(temperature);
  const float inv_part = heat.inv(temperature), inv = heat.part * inv_part, c = heat.c;
  const float most = D.norm[2 * (size_t)row_id], ln = D.norm[2 * (size_t)row_id + 1], log2s = ln * LOG2E;
  const float gh = D.by_entropy ? D.by_entropy[row_id] : 0.0f, h = D.by_entropy ? D.entropy[row_id] : 0.0f;
  const uint32_t n_tokens = D.by_logprob ? R.n_tokens : 0u;
  if (tid < n_tokens) {
    const int32_t v = R.tokens[(size_t)row_id * R.n_tokens + tid];
    const bool ok = v >= 0 && v < (int64_t)R.V && heat.apart(row.at((uint32_t)v), most) * inv_part > -INF;
    tok[tid] = ok ? v : -1;
    g[tid] = ok ? D.by_logprob[(size_t)row_id * R.n_tokens + tid] : 0.0f;
  }
  __syncthreads();
  if (cluster > 1) cluster_arrive(), cluster_wait();
  float total = 0.0f, sizes = fabsf(gh * h);
  for (uint32_t k = 0; k < n_tokens; ++k) total += g[k], sizes += fabsf(g[k]);
  const float A = -(total + gh * h), B = gh * -0.693147181f;
  T* const out = static_cast<T*>(D.out) + (size_t)row_id * D.stride;
  const bool aligned = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.x)) & 31u) == 0;
  auto grad = [&](float x, uint32_t v) {
    if (x == -INF) return 0.0f;
    const float lp2 = fmaf(heat.apart(x, most), heat.c_part, -log2s), p = exp2f(lp2);
    float d = p == 0.0f ? 0.0f : p * fmaf(B, lp2, A);
    for (uint32_t k = 0; k < n_tokens; ++k)
      if (tok[k] == (int32_t)v) d += g[k];
    return heat.part * d * inv_part;
  };
  if (rank == 0 && tid < row.edges) {
    const uint32_t v = row.edge(tid);
    put(out + v, grad(row.at(v), v));
  }
  // p = q^2 with q = 2^(lp2 / 2): in range whenever p is, denormal or not.  What q = 0 is multiplied with is a number: lp2 / 2 is at most
  // 0.6 2^40 c (LOW is its least x), below 2^60, times at most 2^61.
  const bool is_ordinary = ordinary(most, c) && sizes * inv < 0x1p60f && fabsf(B) * inv < 0x1p60f;
  const uint64_t most2 = two(-most, -most), c2 = two(0.5f * c, 0.5f * c), log2s2 = two(-0.5f * log2s, -0.5f * log2s), A2 = two(A * inv, A * inv), B2 = two(2.0f * B * inv, 2.0f * B * inv);
  const uint32_t step = cluster * THREADS;
  row_turns<T, MASK, false, BACK_UNROLL>(row, rank * THREADS + tid, step, keep, [&](uint32_t first, const Unit (&x)[BACK_UNROLL]) {
#pragma unroll
    for (uint32_t u = 0; u < BACK_UNROLL; ++u) {
      const uint32_t i = first + u * step, v = row.first(i);
      if (i >= row.units) break;
      uint64_t y[Row<T>::W / 2];
      if (is_ordinary) {
#pragma unroll
        for (uint32_t e = 0; e < Row<T>::W / 2; ++e) {
          const uint64_t half = fma2(add2(pair_of(x[u], e, T()), most2), c2, log2s2), q = two(ex2(lo(half)), ex2(hi(half)));
          y[e] = mul2(mul2(q, q), fma2(B2, half, A2));
        }
        for (uint32_t k = 0; k < n_tokens; ++k)
          if ((uint32_t)tok[k] - v < Row<T>::W) {
            const float add = g[k] * inv;
#pragma unroll
            for (uint32_t e = 0; e < Row<T>::W / 2; ++e)
              y[e] = add2(y[e], two(tok[k] == (int32_t)(v + 2 * e) ? add : 0.0f, tok[k] == (int32_t)(v + 2 * e + 1) ? add : 0.0f));
          }
      } else {
#pragma unroll
        for (uint32_t e = 0; e < Row<T>::W / 2; ++e) y[e] = two(grad(value(x[u], 2 * e, T()), v + 2 * e), grad(value(x[u], 2 * e + 1, T()), v + 2 * e + 1));
      }
      if (aligned) {
        Unit w;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(lo(y[e]), hi(y[e]));
            w.v[e] = *reinterpret_cast<const uint32_t*>(&b);
          }
        } else {
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) w.v[e] = (uint32_t)(y[e / 2] >> (e % 2 * 32u));
        }
        store_unit(out + v, w);
      } else {
#pragma unroll
        for (uint32_t e = 0; e < Row<T>::W; ++e) put(out + v + e, e % 2 ? hi(y[e / 2]) : lo(y[e / 2]));
      }
    }
  });
}

// Blocks to a row: as many as run at a time (`resident` to an SM), while each has a unit for every thread at least.  A second wave of
// blocks costs more than halves of rows save: 256 masked rows of 128,256 bf16 with 20 alternatives take 33.6 us from memory with a block
// each and 43.1 with two, without alternatives 24.8 and 29.5; 222 rows, whose two blocks all run at a time, 32.1 and 28.9, 24.0 and 21.2.
// A block that looks for alternatives spends several microseconds on them however short its part is, so of those there are no more
// than two to an SM from the third block to a row on (rows of 50,001 with 5 alternatives, 48 of them: 8 blocks a row 14.3 us, 4 12.2,
// 2 12.1; 64 rows of 128,256 with 20: 18.4, 15.1, 17.0).
uint32_t cluster_size(uint32_t rows, uint32_t V, uint32_t width, uint32_t resident, bool top, uint32_t sms) {
  uint32_t c = 1;
  while (c < MAX_CLUSTER && (uint64_t)rows * c * 2u <= (uint64_t)(top && c > 1 ? 2u : resident) * sms && (uint64_t)c * 2u * THREADS * width <= V) c *= 2u;
  return c;
}

template <class... P, class... A>
cudaError_t launch_clusters(void (*kernel)(P...), uint32_t rows, uint32_t cluster, cudaStream_t st, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(rows * cluster), cfg.blockDim = dim3(THREADS), cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
  cfg.attrs = at, cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
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
  uint32_t sms;
  if (fmt_status s = count_sms(&sms)) return s;
  const uint32_t cluster = cluster_size(rows, V, dtype == FMT_BF16 ? 16 : 8, per_sm(mask_dev != nullptr), O.n_top != 0, sms);
  void (*k)(Rows, Outputs, uint32_t);
  if (dtype == FMT_BF16)
    k = mask_dev ? O.n_top ? logprobs_kernel<uint16_t, true, true> : logprobs_kernel<uint16_t, true, false>
                 : O.n_top ? logprobs_kernel<uint16_t, false, true> : logprobs_kernel<uint16_t, false, false>;
  else
    k = mask_dev ? O.n_top ? logprobs_kernel<float, true, true> : logprobs_kernel<float, true, false>
                 : O.n_top ? logprobs_kernel<float, false, true> : logprobs_kernel<float, false, false>;
  return launch_result(launch_clusters(k, rows, cluster, (cudaStream_t)stream, R, O, cluster));
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
  uint32_t sms;
  if (fmt_status s = count_sms(&sms)) return s;
  const uint32_t cluster = cluster_size(rows, V, dtype == FMT_BF16 ? 16 : 8, BACK_PER_SM, false, sms);
  auto* k = dtype == FMT_BF16 ? mask_dev ? logprobs_backward_kernel<uint16_t, true> : logprobs_backward_kernel<uint16_t, false>
                              : mask_dev ? logprobs_backward_kernel<float, true> : logprobs_backward_kernel<float, false>;
  return launch_result(launch_clusters(k, rows, cluster, (cudaStream_t)stream, R, D, cluster));
}
