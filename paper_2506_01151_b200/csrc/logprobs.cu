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

// ------------------------------------------------------------------------------------------------ rows in vectors of 16 bytes
//
// A row may begin at any address: vectors are counted from its first 16-byte boundary on, and the few logits before it and behind
// the last whole vector ("edges") are taken one at a time.  A vector's bits of the mask come from one or two of its words.

template <typename T>
struct Row {
  static constexpr uint32_t W = 16u / sizeof(T);  // logits of a vector
  const T* x;
  const uint32_t* mask;  // or nullptr
  uint32_t V, head, vectors, edges;

  __device__ __forceinline__ Row(const Rows& R, uint32_t row)
      : x(static_cast<const T*>(R.logits) + (size_t)row * R.stride), mask(R.mask ? R.mask + (size_t)row * R.mask_stride : nullptr), V(R.V) {
    head = min(V, (uint32_t)((0u - (uint32_t)reinterpret_cast<uintptr_t>(x)) & 15u) / (uint32_t)sizeof(T));
    vectors = (V - head) / W;
    edges = V - vectors * W;
  }
  __device__ __forceinline__ uint32_t edge(uint32_t i) const { return i < head ? i : i + vectors * W; }
  __device__ __forceinline__ bool allows(uint32_t v) const { return !mask || (mask[v >> 5] >> (v & 31u)) & 1u; }
  __device__ __forceinline__ float at(uint32_t v) const { return allows(v) ? to_f32(x[v]) : -INF; }  // -inf: not allowed
  __device__ __forceinline__ uint32_t first(uint32_t vector) const { return head + vector * W; }
  __device__ __forceinline__ uint32_t bits(uint32_t vector) const {
    const uint32_t v = first(vector), sh = v & 31u;
    if (head == 0) return reinterpret_cast<const uint8_t*>(mask)[v >> 3] >> (v & 7u) & ((1u << W) - 1u);  // in one byte
    const uint32_t lo = mask[v >> 5], hi = sh + W > 32u ? mask[(v >> 5) + 1u] : 0u;  // (the vector ends before V: the word is there)
    return __funnelshift_r(lo, hi, sh) & ((1u << W) - 1u);
  }
  __device__ __forceinline__ uint4 load(uint32_t vector) const { return *reinterpret_cast<const uint4*>(x + first(vector)); }
};

// What the mask forbids becomes -inf.
__device__ __forceinline__ uint32_t keep_pair(uint32_t x, uint32_t spread, uint32_t which) {  // bytes of `spread`: 0x80 or 0
  uint32_t k;
  asm("prmt.b32 %0, %1, 0, %2;" : "=r"(k) : "r"(spread), "r"(which));  // (selectors 8 and up repeat a byte's highest bit)
  return (x & k) | (0xFF80FF80u & ~k);
}
__device__ __forceinline__ void forbid(uint4& x, uint32_t bits, uint16_t) {
  const uint32_t lo = ((bits & 15u) * 0x00204081u & 0x01010101u) << 7, hi = ((bits >> 4) * 0x00204081u & 0x01010101u) << 7;
  x.x = keep_pair(x.x, lo, 0x9988u), x.y = keep_pair(x.y, lo, 0xBBAAu);
  x.z = keep_pair(x.z, hi, 0x9988u), x.w = keep_pair(x.w, hi, 0xBBAAu);
}
__device__ __forceinline__ void forbid(uint4& x, uint32_t bits, float) {
  x.x = bits & 1u ? x.x : 0xFF800000u, x.y = bits & 2u ? x.y : 0xFF800000u;
  x.z = bits & 4u ? x.z : 0xFF800000u, x.w = bits & 8u ? x.w : 0xFF800000u;
}
template <typename T>
__device__ __forceinline__ uint4 all_forbidden() {
  const uint32_t n = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
  return make_uint4(n, n, n, n);
}
__device__ __forceinline__ float value(const uint4& x, uint32_t i, uint16_t) {
  const uint32_t w = i / 2 == 0 ? x.x : i / 2 == 1 ? x.y : i / 2 == 2 ? x.z : x.w;
  return __uint_as_float(i % 2 ? w & 0xFFFF0000u : w << 16);
}
__device__ __forceinline__ float value(const uint4& x, uint32_t i, float) {
  return __uint_as_float(i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w);
}
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {  // (of a NaN and a number: the number)
  uint32_t m;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
  return m;
}
__device__ __forceinline__ float largest(const uint4& x, uint16_t) {
  const uint32_t m = max_pair(max_pair(x.x, x.y), max_pair(x.z, x.w));
  return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
}
__device__ __forceinline__ float largest(const uint4& x, float) {
  return fmaxf(fmaxf(__uint_as_float(x.x), __uint_as_float(x.y)), fmaxf(__uint_as_float(x.z), __uint_as_float(x.w)));
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

// A vector's values in pairs, nothing below LOW (-inf becomes LOW; a NaN stays).  LOW lies so far below a row's largest logit that
// its probability is 0, and is finite, so that 0 times what is made of it is 0.  This holds for rows whose largest logit is above
// LOW / 10 and whose temperature is between 2e-6 and 1e8 (`ordinary`): 0.9 x 2^40 x 1e-8 is 9,900 powers of two.  In others
// every value is looked at.
constexpr float LOW = -0x1p40f;
__device__ __forceinline__ bool ordinary(float largest, float c) { return largest > LOW * 0.1f && c > 1e-8f && c < 1e6f; }
__device__ __forceinline__ uint64_t pair_of(const uint4& x, uint32_t i, uint16_t) {
  uint32_t w = i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(w) : "r"(w), "r"(0xD380D380u));
  return two(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ uint64_t pair_of(const uint4& x, uint32_t i, float) {
  float a = __uint_as_float(i == 0 ? x.x : x.z), b = __uint_as_float(i == 0 ? x.y : x.w);
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(a), "f"(LOW));
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(b) : "f"(b), "f"(LOW));
  return two(a, b);
}

// ------------------------------------------------------------------------------------------------ sums of a row
//
// One pass: s = sum of 2^d and t = sum of 2^d d with d = (x - m) log2(e) / T and m the largest logit so far, rescaled when m grows.
// (x - m is formed first: of two logits of the type's lowest value it is 0, where a product with either would overflow.)
// The entropy is ln s - (t / s) ln 2, two parts of one sign.  A NaN or +inf among the allowed logits makes s NaN, and nothing else does.

struct Sums {
  float m = -INF, s = 0.0f, t = 0.0f;

  __device__ __forceinline__ void grow(float to, float c) {  // a larger m
    if (!(to > m)) return;
    if (m > -INF) {
      const float d = (m - to) * c, f = ex2(d);
      t = f > 0.0f ? (t + s * d) * f : s * 0.0f;  // (s * 0: what is NaN stays NaN)
      s *= f;
    }
    m = to;
  }
  __device__ __forceinline__ float base() const { return m > -INF ? m : 0.0f; }
  __device__ __forceinline__ void add(float x, float base, float c) {
    const float d = (x - base) * c, p = ex2(d);
    s += p;
    t = fmaf(p, fmaxf(d, -1024.0f), t);  // (d may be -inf; p is 0 below -1024)
  }
  // Vectors whose largest logits m has grown for.
  template <typename T, uint32_t N>
  __device__ __forceinline__ void add(const uint4 (&x)[N], float c) {
    const float b = base();
    if (ordinary(m, c)) {
      const uint64_t b2 = two(-b, -b), c2 = two(c, c);
      uint64_t s2 = two(s, 0.0f), t2 = two(t, 0.0f);
#pragma unroll
      for (uint32_t u = 0; u < N; ++u)
#pragma unroll
        for (uint32_t e = 0; e < 8u / sizeof(T); ++e) {
          const uint64_t d = mul2(add2(pair_of(x[u], e, T()), b2), c2), p = two(ex2(lo(d)), ex2(hi(d)));
          s2 = add2(s2, p);
          t2 = fma2(p, d, t2);
        }
      s = lo(s2) + hi(s2), t = lo(t2) + hi(t2);
    } else {
#pragma unroll
      for (uint32_t u = 0; u < N; ++u)
#pragma unroll
        for (uint32_t e = 0; e < 16u / sizeof(T); ++e) add(value(x[u], e, T()), b, c);
    }
  }
  __device__ __forceinline__ void join(Sums o, float c) {
    const float to = fmaxf(m, o.m);
    grow(to, c), o.grow(to, c);
    s += o.s, t += o.t;
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
// A cluster of 1 to 8 thread blocks to a row; block r takes vectors r * THREADS + thread, and so on in steps of the whole cluster.
//
// The likeliest tokens.  In the pass over the row each thread keeps the first vector with its largest logit.  The threads make
// 128 groups; of the groups' largest keys (logit, lowest id) the n_top-th is a bound that n_top logits at least reach, and only
// the n_top groups whose own largest reaches it hold any: their vectors alone are read again (L2), and what reaches the bound is
// listed and put in order.  A row of 128,256 logits is passed once, and a sixth of it twice for n_top = 20, whatever its order.

constexpr uint32_t THREADS = 512, WARPS = THREADS / 32, UNROLL = 4, BACK_UNROLL = 2;
constexpr uint32_t GROUPS = 128, GROUP = THREADS / GROUPS;
constexpr uint32_t MAX_CLUSTER = 8;
constexpr uint32_t SORT = 512;                    // listed logits that are put in order by counting
constexpr uint32_t LISTED = SORT + THREADS * 8u;  // what one round of re-reading may add

struct TopShared {
  uint64_t list[LISTED];
  uint64_t group[GROUPS];
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
      for (uint32_t i = 0; i < n; ++i) above += P.list[i] > mine;
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

template <typename T>
__device__ void find_top(const Row<T>& row, uint32_t from, uint32_t step, uint32_t edges, uint64_t mine, uint32_t want, TopShared& P) {
  const uint32_t tid = threadIdx.x;
  for (uint32_t o = 1; o < GROUP; o <<= 1) mine = max_key(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, o));
  if (tid % GROUP == 0) P.group[tid / GROUP] = mine;
  if (tid == 0) P.n_listed = 0, P.n_chosen = 0, P.bound = 1;
  __syncthreads();
  uint32_t above = 0;
  if (tid < GROUPS) {
    mine = P.group[tid];
    for (uint32_t i = 0; i < GROUPS; ++i) above += P.group[i] > mine;
    if (mine && above < want) {
      P.chosen[atomicAdd(&P.n_chosen, 1u)] = tid;
      if (above == want - 1) P.bound = mine;
    }
  }
  __syncthreads();
  uint64_t bound = P.bound;
  const uint32_t rounds_of = (row.vectors + step - 1) / step;  // vectors of a thread, at most
  const uint32_t items = P.n_chosen * GROUP * rounds_of;
  auto offer = [&](float x, uint32_t v) {
    const uint64_t key = order_key(x, v);
    if (x > -INF && key >= bound) P.list[atomicAdd(&P.n_listed, 1u)] = key;
  };
  if (tid < edges) offer(row.at(row.edge(tid)), row.edge(tid));
  for (uint32_t base = 0; base < items; base += THREADS) {
    if (base) {
      __syncthreads();
      if (P.n_listed > SORT) {  // only if many of the largest logits are in few groups
        best_of_list(P, want);
        if (tid < want) P.list[tid] = P.best[tid];
        if (tid == 0) P.n_listed = want, P.bound = P.best[want - 1];
        __syncthreads();
        bound = P.bound;
      }
      __syncthreads();
    }
    const uint32_t item = base + tid;
    if (item < items) {
      const uint32_t rest = item % (GROUP * rounds_of);
      const uint32_t vector = from - tid + P.chosen[item / (GROUP * rounds_of)] * GROUP + rest % GROUP + rest / GROUP * step;
      if (vector < row.vectors) {
        const uint32_t bits = row.mask ? row.bits(vector) : (1u << Row<T>::W) - 1u;
        if (bits) {
          uint4 x = row.load(vector);
          forbid(x, bits, T());
          if (largest(x, T()) >= key_logit(bound) || bound == 1)
            for (uint32_t i = 0; i < Row<T>::W; ++i) offer(value(x, i, T()), row.first(vector) + i);
        }
      }
    }
  }
  __syncthreads();
  best_of_list(P, want);
}

template <typename T, bool MASK, bool TOP>
__global__ void __launch_bounds__(THREADS, 2) logprobs_kernel(const Rows R, const Outputs O, const uint32_t cluster) {
  __shared__ JoinShared J;
  __shared__ __align__(8) uint8_t top_raw[TOP ? sizeof(TopShared) : 8];
  TopShared& P = *reinterpret_cast<TopShared*>(top_raw);
  if (cluster > 1) cluster_arrive();
  before_me();
  const uint32_t tid = threadIdx.x, rank = cluster > 1 ? cluster_rank() : 0u, row_id = blockIdx.x / cluster;
  const Row<T> row(R, row_id);
  const float temperature = R.temperature ? R.temperature[row_id] : 1.0f;
  const float inv = __fdiv_rn(1.0f, temperature), c = inv * 1.44269504f;  // log2(e)

  Sums a;
  uint32_t where = 0xFFFFFFFFu;  // the first vector with the thread's largest logit, or, behind all vectors, an edge
  const uint32_t edges = rank == 0 ? row.edges : 0u;
  if (tid < edges && row.edge(tid) < row.head) {
    const float x = row.at(row.edge(tid));
    if (x > a.m) where = row.vectors + tid;
    a.grow(x, c), a.add(x, a.base(), c);
  }
  const uint32_t from = rank * THREADS + tid, step = cluster * THREADS;
  // The next vectors are on their way, and the bits of those after them, while some are added up.
  uint4 x[UNROLL], next[UNROLL];
  uint32_t bits[UNROLL], ahead[UNROLL];
  auto ask_bits = [&](uint32_t i, uint32_t (&to)[UNROLL]) {
#pragma unroll
    for (uint32_t u = 0; u < UNROLL; ++u)
      to[u] = i + u * step >= row.vectors ? 0u : MASK ? row.bits(i + u * step) : (1u << Row<T>::W) - 1u;
  };
  auto ask = [&](uint32_t i, const uint32_t (&want)[UNROLL], uint4 (&to)[UNROLL]) {
#pragma unroll
    for (uint32_t u = 0; u < UNROLL; ++u) to[u] = want[u] ? row.load(i + u * step) : all_forbidden<T>();
  };
  ask_bits(from, bits);
  ask(from, bits, x);
  ask_bits(from + UNROLL * step, ahead);
  for (uint32_t i = from; i < row.vectors; i += UNROLL * step) {
    ask(i + UNROLL * step, ahead, next);
    float m = a.m;
#pragma unroll
    for (uint32_t u = 0; u < UNROLL; ++u) {
      if (MASK) forbid(x[u], bits[u], T());
      bits[u] = ahead[u];
      const float most = largest(x[u], T());
      if (most > m) {
        m = most;
        if (TOP) where = i + u * step;
      }
    }
    ask_bits(i + 2u * UNROLL * step, ahead);
    a.grow(m, c);
    a.template add<T, UNROLL>(x, c);
#pragma unroll
    for (uint32_t u = 0; u < UNROLL; ++u) x[u] = next[u];
  }
  if (tid < edges && row.edge(tid) >= row.head) {
    const float x = row.at(row.edge(tid));
    if (x > a.m) where = row.vectors + tid;
    a.grow(x, c), a.add(x, a.base(), c);
  }

  if (TOP) {
    uint64_t mine = 0;
    if (where != 0xFFFFFFFFu) {
      if (where >= row.vectors) {
        mine = order_key(a.m, row.edge(where - row.vectors));
      } else {
        uint4 x = row.load(where);
        forbid(x, MASK ? row.bits(where) : (1u << Row<T>::W) - 1u, T());
        uint32_t at = 0;
        for (uint32_t e = Row<T>::W; e-- > 0;)
          if (value(x, e, T()) == a.m) at = e;
        mine = order_key(a.m, row.first(where) + at);
      }
    }
    find_top(row, from, step, edges, mine, O.n_top, P);
  }

  for (uint32_t o = 16; o; o >>= 1) {
    Sums b;
    b.m = __shfl_xor_sync(0xFFFFFFFFu, a.m, o), b.s = __shfl_xor_sync(0xFFFFFFFFu, a.s, o), b.t = __shfl_xor_sync(0xFFFFFFFFu, a.t, o);
    a.join(b, c);
  }
  if (tid % 32u == 0) J.warps[tid / 32u] = a;
  __syncthreads();
  if (tid < 32) {
    a = tid < WARPS ? J.warps[tid] : Sums();
    for (uint32_t o = WARPS / 2; o; o >>= 1) {
      Sums b;
      b.m = __shfl_xor_sync(0xFFFFFFFFu, a.m, o), b.s = __shfl_xor_sync(0xFFFFFFFFu, a.s, o), b.t = __shfl_xor_sync(0xFFFFFFFFu, a.t, o);
      a.join(b, c);
    }
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
    if (tid == 0) {
      a = Sums();
      for (uint32_t i = 0; i < cluster; ++i) a.join(J.blocks[i], c);
    }
    if (TOP) {
      // the blocks' lists are in order: a key's place is its own in its list and, of every other one, how many are above
      const uint32_t n = cluster * O.n_top;
      if (tid < O.n_top) P.best[tid] = 0;
      __syncthreads();
      if (tid < n && P.join[tid]) {
        const uint64_t mine = P.join[tid];
        uint32_t above = 0;
        for (uint32_t b = 0; b < cluster; ++b) {
          const uint64_t* l = P.join + b * O.n_top;
          uint32_t lo = 0, hi = O.n_top;
          while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (l[mid] > mine) lo = mid + 1;
            else hi = mid;
          }
          above += lo;
        }
        if (above < O.n_top) P.best[above] = mine;
      }
    }
  }
  if (tid == 0) J.warps[0] = a;
  __syncthreads();
  a = J.warps[0];

  const float nan = __int_as_float(0x7FC00000);
  const bool bad = a.s != a.s || !(temperature > 0.0f && temperature < INF);
  const float ln = bad ? nan : logf(a.s);  // (-inf of nothing)
  auto logprob = [&](float x) { return bad ? nan : x == -INF ? -INF : (x - a.m) * inv - ln; };
  bool wrong = false;
  if (tid < R.n_tokens) {
    const int32_t v = R.tokens[(size_t)row_id * R.n_tokens + tid];
    wrong = v < -1 || v >= (int64_t)R.V;
    if (O.logprobs) O.logprobs[(size_t)row_id * R.n_tokens + tid] = v == -1 ? 0.0f : wrong ? nan : logprob(row.at((uint32_t)v));
  }
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
// grad = p (A + B lp2) with lp2 = log2 p, A = -(sum g + g_H H) / T and B = -g_H ln 2 / T, and the g of the given tokens on top.
// The given tokens' own logits decide whether they count: all of a cluster's blocks have read them before the first writes,
// since the gradient may take the logits' place.

template <typename T, bool MASK>
__global__ void __launch_bounds__(THREADS) logprobs_backward_kernel(const Rows R, const Gradients D, const uint32_t cluster) {
  before_me();
  __shared__ int32_t tok[FMT_MAX_GIVEN_TOKENS];
  __shared__ float g[FMT_MAX_GIVEN_TOKENS];
  const uint32_t tid = threadIdx.x, rank = cluster > 1 ? cluster_rank() : 0u, row_id = blockIdx.x / cluster;
  const Row<T> row(R, row_id);
  const float inv = __fdiv_rn(1.0f, R.temperature ? R.temperature[row_id] : 1.0f), c = inv * 1.44269504f;
  const float most = D.norm[2 * (size_t)row_id], ln = D.norm[2 * (size_t)row_id + 1], log2s = ln * 1.44269504f;
  const float gh = D.by_entropy ? D.by_entropy[row_id] : 0.0f, h = D.by_entropy ? D.entropy[row_id] : 0.0f;
  const uint32_t n_tokens = D.by_logprob ? R.n_tokens : 0u;
  if (tid < n_tokens) {
    const int32_t v = R.tokens[(size_t)row_id * R.n_tokens + tid];
    const bool ok = v >= 0 && v < (int64_t)R.V && (row.at((uint32_t)v) - most) * inv > -INF;
    tok[tid] = ok ? v : -1;
    g[tid] = ok ? D.by_logprob[(size_t)row_id * R.n_tokens + tid] : 0.0f;
  }
  __syncthreads();
  if (cluster > 1) cluster_arrive(), cluster_wait();
  float total = 0.0f;
  for (uint32_t k = 0; k < n_tokens; ++k) total += g[k];
  const float A = -(total + gh * h) * inv, B = gh * -0.693147181f * inv;
  T* const out = static_cast<T*>(D.out) + (size_t)row_id * D.stride;
  const bool aligned = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.x)) & 15u) == 0;
  auto grad = [&](float x) {
    const float lp2 = fmaf(x - most, c, -log2s), p = exp2f(lp2);
    return x == -INF ? 0.0f : p * fmaf(B, fmaxf(lp2, -1024.0f), A);
  };
  if (rank == 0 && tid < row.edges) {
    const uint32_t v = row.edge(tid);
    float sum = 0.0f;
    for (uint32_t k = 0; k < n_tokens; ++k)
      if (tok[k] == (int32_t)v) sum += g[k];
    put(out + v, grad(row.at(v)) + sum * inv);
  }
  // p = q^2 with q = 2^(lp2 / 2): in range whenever p is, denormal or not
  const bool is_ordinary = ordinary(most, c);
  const uint64_t most2 = two(-most, -most), c2 = two(0.5f * c, 0.5f * c), log2s2 = two(-0.5f * log2s, -0.5f * log2s), A2 = two(A, A), B2 = two(2.0f * B, 2.0f * B);
  const uint32_t step = cluster * THREADS;
  for (uint32_t base = rank * THREADS + tid; base < row.vectors; base += BACK_UNROLL * step) {
    uint32_t bits[BACK_UNROLL];
    uint4 x[BACK_UNROLL];
#pragma unroll
    for (uint32_t u = 0; u < BACK_UNROLL; ++u) {
      const uint32_t i = base + u * step;
      bits[u] = i >= row.vectors ? 0u : MASK ? row.bits(i) : (1u << Row<T>::W) - 1u;
    }
#pragma unroll
    for (uint32_t u = 0; u < BACK_UNROLL; ++u) x[u] = bits[u] ? row.load(base + u * step) : all_forbidden<T>();
#pragma unroll
    for (uint32_t u = 0; u < BACK_UNROLL; ++u) {
      const uint32_t i = base + u * step, v = row.first(i);
      if (i >= row.vectors) break;
      uint64_t y[Row<T>::W / 2];
#pragma unroll
      for (uint32_t e = 0; e < Row<T>::W / 2; ++e) y[e] = 0;
      if (bits[u]) {
        if (MASK) forbid(x[u], bits[u], T());
        if (is_ordinary) {
#pragma unroll
          for (uint32_t e = 0; e < Row<T>::W / 2; ++e) {
            const uint64_t half = fma2(add2(pair_of(x[u], e, T()), most2), c2, log2s2), q = two(ex2(lo(half)), ex2(hi(half)));
            y[e] = mul2(mul2(q, q), fma2(B2, half, A2));
          }
        } else {
#pragma unroll
          for (uint32_t e = 0; e < Row<T>::W / 2; ++e) y[e] = two(grad(value(x[u], 2 * e, T())), grad(value(x[u], 2 * e + 1, T())));
        }
        for (uint32_t k = 0; k < n_tokens; ++k)
          if ((uint32_t)tok[k] - v < Row<T>::W) {
            const float add = g[k] * inv;
#pragma unroll
            for (uint32_t e = 0; e < Row<T>::W / 2; ++e)
              y[e] = add2(y[e], two(tok[k] == (int32_t)(v + 2 * e) ? add : 0.0f, tok[k] == (int32_t)(v + 2 * e + 1) ? add : 0.0f));
          }
      }
      if (aligned) {
        uint4 w;
        if constexpr (sizeof(T) == 2) {
          auto both = [](uint64_t p) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(lo(p), hi(p));
            return *reinterpret_cast<const uint32_t*>(&b);
          };
          w = make_uint4(both(y[0]), both(y[1]), both(y[2]), both(y[3]));
        } else {
          w = make_uint4((uint32_t)y[0], (uint32_t)(y[0] >> 32), (uint32_t)y[1], (uint32_t)(y[1] >> 32));
        }
        *reinterpret_cast<uint4*>(out + v) = w;
      } else {
#pragma unroll
        for (uint32_t e = 0; e < Row<T>::W; ++e) put(out + v + e, e % 2 ? hi(y[e / 2]) : lo(y[e / 2]));
      }
    }
  }
}

// Blocks to a row: as many as fill the GPU (two to an SM), while each has a vector for every thread at least.
uint32_t cluster_size(uint32_t rows, uint32_t V, uint32_t width) {
  uint32_t c = 1;
  while (c < MAX_CLUSTER && rows * (c * 2u) <= 2u * 148u && (uint64_t)c * 2u * THREADS * width <= V) c *= 2u;
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
  const uint32_t cluster = cluster_size(rows, V, dtype == FMT_BF16 ? 8 : 4);
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
  const uint32_t cluster = cluster_size(rows, V, dtype == FMT_BF16 ? 8 : 4);
  auto* k = dtype == FMT_BF16 ? mask_dev ? logprobs_backward_kernel<uint16_t, true> : logprobs_backward_kernel<uint16_t, false>
                              : mask_dev ? logprobs_backward_kernel<float, true> : logprobs_backward_kernel<float, false>;
  return launch_result(launch_clusters(k, rows, cluster, (cudaStream_t)stream, R, D, cluster));
}
