// The output head: values in 8-bit floating point with a scale for each block, and their product under the mask.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
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

// ------------------------------------------------------------------------------------------------ the product
//
// D[token of the vocabulary][row] on the tensor cores, one block of 128 columns at a time: four tcgen05.mma of 32 columns each make
// the block's 128 x N sums in tensor memory, from where eight warps take them, multiply them with the block's two scales and add
// them up in registers.  (Scales of any value cannot ride along in the instruction, whose own are powers of two.)  The vocabulary
// is the M side: a decoding step has few rows and very many tokens, and M is 128 whatever N is.
//
// A thread block to an SM.  The vocabulary goes to the blocks in slabs of 32 tokens, a word of the mask and a quarter of a tile:
// slab s to block s mod C.  A block makes a list of its slabs that some row may use, and takes four at a time, wherever they lie;
// the others are written as -inf and their weights not read.  Work is even to a slab (128,256 tokens: 27 or 28 of 4,008 to each of 148).
//
// Warps: 0 copies tiles to shared memory (TMA, a ring of stages), 1 issues the products, 2 copies the scales (a ring of their own,
// as they are needed later than the tiles), 4 to 11 add up and write.

constexpr uint32_t SLAB = 32, TILE_SLABS = 4;
constexpr uint32_t HEAD_THREADS = 384, ADD_WARPS = 8;
constexpr uint32_t LIST = 512;        // slabs of a block that are looked at in one go
constexpr uint32_t SCALE_SLOTS = 8;
constexpr uint32_t SLAB_BYTES = SLAB * BLOCK;
constexpr uint32_t WAIT_POLLS = 1u << 20;  // of at most 2 us each

template <uint32_t N>
struct HeadShape {
  static constexpr uint32_t stages = N == 256 ? 4 : N == 128 ? 6 : N == 64 ? 8 : 10;
  static constexpr uint32_t bufs = N == 256 ? 2 : N == 128 ? 4 : 8;  // of tensor memory, N columns each
  static constexpr uint32_t stage_bytes = TILE_SLABS * SLAB_BYTES + N * BLOCK;
  static constexpr uint32_t slot_floats = N + TILE_SLABS;
  static constexpr uint32_t smem = 1024 + stages * stage_bytes + SCALE_SLOTS * slot_floats * 4;
};

struct HeadArgs {
  const float* xs;
  size_t xs_stride;
  const float* ws;
  size_t ws_stride;
  uint32_t rows, V, K;
  const uint32_t* mask;
  size_t mask_stride;
  void* logits;
  size_t row_stride;
};

struct HeadShared {
  uint64_t full[10], empty[10], sums_full[8], sums_empty[8], scales_full[SCALE_SLOTS], scales_empty[SCALE_SLOTS];
  uint32_t tmem, n_live, n_dead;
  volatile uint32_t gave_up;
  uint32_t bits[LIST / 32];
  uint16_t live[LIST], dead[LIST];
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_test(uint64_t* b, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(done) : "r"(smem_addr(b)), "r"(parity), "r"(2000u) : "memory");
  return done != 0u;
}
// Waits until the barrier's phase of this parity is over.  False: given up, here or by another warp of the block.
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, HeadShared& S) {
  if (bar_test(b, parity)) return true;
  for (uint32_t i = 0; i < WAIT_POLLS && !S.gave_up; ++i)
    if (bar_test(b, parity)) return true;
  S.gave_up = 1u;
  return false;
}
__device__ __forceinline__ void bar_drain(uint64_t* b, uint32_t parity) {  // the same after giving up, for what is in flight
  for (uint32_t i = 0; i < WAIT_POLLS && !bar_test(b, parity); ++i) {}
}

// A place in a ring and how often it has been round.
template <uint32_t SIZE>
struct Ring {
  uint32_t at = 0, round = 0;
  __device__ __forceinline__ void next() {
    if (++at == SIZE) at = 0, round ^= 1u;
  }
};

__device__ __forceinline__ void tma_load(const CUtensorMap* map, uint64_t* bar, uint32_t dst, uint32_t x, uint32_t y) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst), "l"(map),
               "r"(smem_addr(bar)), "r"(x), "r"(y)
               : "memory");
}
// Rows of 128 bytes, swizzled in groups of eight (1,024 bytes), version 1 of the descriptor.
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
               "r"((uint32_t)add)
               : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

template <uint32_t COLS>
__device__ __forceinline__ void tmem_read(uint32_t addr, float (&v)[COLS]);
#define R4(i) "=f"(v[i]), "=f"(v[i + 1]), "=f"(v[i + 2]), "=f"(v[i + 3])
template <>
__device__ __forceinline__ void tmem_read<8>(uint32_t addr, float (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : R4(0), R4(4) : "r"(addr));
}
template <>
__device__ __forceinline__ void tmem_read<16>(uint32_t addr, float (&v)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : R4(0), R4(4), R4(8), R4(12) : "r"(addr));
}
template <>
__device__ __forceinline__ void tmem_read<32>(uint32_t addr, float (&v)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
               "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : R4(0), R4(4), R4(8), R4(12), R4(16), R4(20), R4(24), R4(28) : "r"(addr));
}
#undef R4
// The values that a read of tensor memory gave may be used from here on.
template <uint32_t COLS>
__device__ __forceinline__ void tmem_read_done(float (&v)[COLS]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (uint32_t i = 0; i < COLS; ++i) asm volatile("" : "+f"(v[i]));
}

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = __bfloat16_as_ushort(__float2bfloat16_rn(x)); }

template <typename T, uint32_t N>
__global__ void __launch_bounds__(HEAD_THREADS, 1) head_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const HeadArgs A) {
  using Shape = HeadShape<N>;
  constexpr uint32_t COLS = N / 2;                   // of a tile, to each of the adding warps
  constexpr uint32_t CHUNK = COLS < 32 ? COLS : 32;  // read from tensor memory in one go
  constexpr uint32_t TMEM = Shape::bufs * N;
  extern __shared__ uint8_t raw[];
  __shared__ HeadShared S;
  const uint32_t tiles_at = (smem_addr(raw) + 1023u) & ~1023u;
  float* const scales = reinterpret_cast<float*>(raw + (tiles_at - smem_addr(raw)) + Shape::stages * Shape::stage_bytes);
  const uint32_t tid = threadIdx.x, warp = tid / 32u, lane = tid % 32u;
  const uint32_t n_slabs = (A.V + SLAB - 1) / SLAB, n_blocks = (A.K + BLOCK - 1) / BLOCK, row_tiles = (A.rows + N - 1) / N;

  if (tid == 0) {
    for (uint32_t i = 0; i < Shape::stages; ++i) bar_init(&S.full[i], 1), bar_init(&S.empty[i], 1);
    for (uint32_t i = 0; i < Shape::bufs; ++i) bar_init(&S.sums_full[i], 1), bar_init(&S.sums_empty[i], ADD_WARPS);
    for (uint32_t i = 0; i < SCALE_SLOTS; ++i) bar_init(&S.scales_full[i], 32), bar_init(&S.scales_empty[i], ADD_WARPS);
    S.gave_up = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&S.tmem)), "n"(TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  before_sync();
  __syncthreads();
  after_sync();
  before_me();

  Ring<Shape::stages> stage;
  Ring<Shape::bufs> buf;
  Ring<SCALE_SLOTS> slot;
  uint32_t issued = 0;  // tiles under way, or done (warps 0 and 1)
  bool failed = false;

  for (uint32_t first = blockIdx.x; first < n_slabs; first += LIST * gridDim.x) {
    // which of the block's slabs some row may use
    const uint32_t here = min(LIST, (n_slabs - first + gridDim.x - 1) / gridDim.x);
    if (tid < LIST / 32) S.bits[tid] = A.mask ? 0u : 0xFFFFFFFFu;
    __syncthreads();
    if (A.mask)
      for (uint32_t i = warp; i < here; i += HEAD_THREADS / 32) {
        const uint32_t* m = A.mask + first + (size_t)i * gridDim.x;
        uint32_t any = 0u;
        for (uint32_t r0 = 0; r0 < A.rows && !any; r0 += 256) {
#pragma unroll
          for (uint32_t u = 0; u < 8; ++u)
            if (r0 + u * 32u + lane < A.rows) any |= __ldg(m + (size_t)(r0 + u * 32u + lane) * A.mask_stride);
          any = __any_sync(0xFFFFFFFFu, any != 0u);
        }
        if (lane == 0 && any) atomicOr(&S.bits[i / 32], 1u << (i % 32));
      }
    __syncthreads();
    if (warp == 0) {
      uint32_t n_live = 0, n_dead = 0;
      for (uint32_t i = 0; i < here; i += 32) {
        const uint32_t word = S.bits[i / 32], in = here - i < 32u ? (1u << (here - i)) - 1u : 0xFFFFFFFFu;
        const uint32_t alive = word & in, gone = ~word & in, before = (1u << lane) - 1u;
        if ((alive >> lane) & 1u) S.live[n_live + __popc(alive & before)] = (uint16_t)(i + lane);
        if ((gone >> lane) & 1u) S.dead[n_dead + __popc(gone & before)] = (uint16_t)(i + lane);
        n_live += __popc(alive), n_dead += __popc(gone);
      }
      if (lane == 0) S.n_live = n_live, S.n_dead = n_dead;
    }
    __syncthreads();
    const uint32_t n_live = S.n_live;
    auto slab = [&](uint32_t i) { return first + (uint32_t)S.live[i] * gridDim.x; };

    if (warp == 0) {
      if (lane == 0)
        for (uint32_t g = 0; g < n_live && !failed; g += TILE_SLABS)
          for (uint32_t j = blockIdx.y; j < row_tiles && !failed; j += gridDim.y) {
            const uint32_t count = min(TILE_SLABS, n_live - g);
            uint32_t y[TILE_SLABS];
#pragma unroll
            for (uint32_t i = 0; i < TILE_SLABS; ++i) y[i] = slab(g + (i < count ? i : 0u)) * SLAB;
            for (uint32_t b = 0; b < n_blocks; ++b) {
              if (!bar_wait(&S.empty[stage.at], stage.round ^ 1u, S)) {
                failed = true;
                break;
              }
              const uint32_t at = tiles_at + stage.at * Shape::stage_bytes;
              uint64_t* bar = &S.full[stage.at];
              bar_expect(bar, count * SLAB_BYTES + N * BLOCK);
#pragma unroll
              for (uint32_t i = 0; i < TILE_SLABS; ++i)
                if (i < count) tma_load(&wmap, bar, at + i * SLAB_BYTES, b * BLOCK, y[i]);
              tma_load(&xmap, bar, at + TILE_SLABS * SLAB_BYTES, b * BLOCK, j * N);
              ++issued;
              stage.next();
            }
          }
    } else if (warp == 1) {
      if (lane == 0) {
        // e4m3 x e4m3 into fp32, both K-major, N columns, 128 lanes
        constexpr uint32_t idesc = 1u << 4 | (N >> 3) << 17 | (128u >> 4) << 24;
        const uint32_t tiles = ((n_live + TILE_SLABS - 1) / TILE_SLABS) * ((row_tiles + gridDim.y - 1 - blockIdx.y) / gridDim.y);
        for (uint32_t t = 0; t < tiles && !failed; ++t)
          for (uint32_t b = 0; b < n_blocks; ++b) {
            if (!bar_wait(&S.sums_empty[buf.at], buf.round ^ 1u, S) || !bar_wait(&S.full[stage.at], stage.round, S)) {
              failed = true;
              break;
            }
            after_sync();
            const uint32_t at = tiles_at + stage.at * Shape::stage_bytes;
            const uint64_t a = tile_desc(at), x = tile_desc(at + TILE_SLABS * SLAB_BYTES);
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) mma(S.tmem + buf.at * N, a + 2 * k, x + 2 * k, idesc, k != 0);
            mma_commit(&S.empty[stage.at]);
            mma_commit(&S.sums_full[buf.at]);
            ++issued;
            stage.next(), buf.next();
          }
      }
    } else if (warp == 2) {
      for (uint32_t g = 0; g < n_live && !failed; g += TILE_SLABS)
        for (uint32_t j = blockIdx.y; j < row_tiles && !failed; j += gridDim.y) {
          const uint32_t count = min(TILE_SLABS, n_live - g), r0 = j * N;
          const float* wp = A.ws + (size_t)(slab(g + (lane < count ? lane : 0u)) / TILE_SLABS) * A.ws_stride;
          for (uint32_t b = 0; b < n_blocks; ++b) {
            if (__any_sync(0xFFFFFFFFu, !bar_wait(&S.scales_empty[slot.at], slot.round ^ 1u, S))) {
              failed = true;
              break;
            }
            const uint32_t dst = smem_addr(scales + slot.at * Shape::slot_floats);
            const float* xp = A.xs + (size_t)b * A.xs_stride + r0;
#pragma unroll
            for (uint32_t i = 0; i < (N + 31u) / 32u; ++i) {
              const uint32_t c = i * 32u + lane;
              if (c < N && r0 + c < A.rows)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + c * 4u), "l"(xp + c) : "memory");
            }
            if (lane < count) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + (N + lane) * 4u), "l"(wp + b) : "memory");
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(&S.scales_full[slot.at])) : "memory");
            slot.next();
          }
        }
      asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp >= 4) {
      const uint32_t quarter = warp % 4u, half = (warp - 4u) / 4u;  // 32 lanes of tensor memory, half of the columns
      T* const logits = static_cast<T*>(A.logits);
      // the slabs that no row may use
      for (uint32_t i = warp - 4u; i < S.n_dead; i += ADD_WARPS) {
        const uint32_t v = (first + (uint32_t)S.dead[i] * gridDim.x) * SLAB + lane;
        if (v < A.V)
          for (uint32_t r = blockIdx.y; r < A.rows; r += gridDim.y) put(logits + (size_t)r * A.row_stride + v, -__int_as_float(0x7F800000));
      }
      for (uint32_t g = 0; g < n_live; g += TILE_SLABS)
        for (uint32_t j = blockIdx.y; j < row_tiles; j += gridDim.y) {
          const bool mine = quarter < n_live - g;
          const uint32_t s = slab(mine ? g + quarter : g), v = s * SLAB + lane;
          float sum[COLS];
#pragma unroll
          for (uint32_t c = 0; c < COLS; ++c) sum[c] = 0.0f;
          for (uint32_t b = 0; b < n_blocks; ++b) {
            if (failed || __any_sync(0xFFFFFFFFu, !bar_wait(&S.sums_full[buf.at], buf.round, S) || !bar_wait(&S.scales_full[slot.at], slot.round, S))) {
              failed = true;
              break;
            }
            after_sync();
            if (mine) {
              const float* sc = scales + slot.at * Shape::slot_floats;
              const float w = sc[N + quarter];
              const float* x = sc + half * COLS;
              const uint32_t from = S.tmem + (quarter * 32u << 16) + buf.at * N + half * COLS;
#pragma unroll
              for (uint32_t c0 = 0; c0 < COLS; c0 += CHUNK) {
                float d[CHUNK];
                tmem_read<CHUNK>(from + c0, d);
                tmem_read_done<CHUNK>(d);
#pragma unroll
                for (uint32_t c = 0; c < CHUNK; c += 4) {
                  const float4 f = *reinterpret_cast<const float4*>(x + c0 + c);
                  sum[c0 + c] = fmaf(d[c], f.x * w, sum[c0 + c]);
                  sum[c0 + c + 1] = fmaf(d[c + 1], f.y * w, sum[c0 + c + 1]);
                  sum[c0 + c + 2] = fmaf(d[c + 2], f.z * w, sum[c0 + c + 2]);
                  sum[c0 + c + 3] = fmaf(d[c + 3], f.w * w, sum[c0 + c + 3]);
                }
              }
            }
            before_sync();
            __syncwarp();
            if (lane == 0) bar_arrive(&S.sums_empty[buf.at]), bar_arrive(&S.scales_empty[slot.at]);
            buf.next(), slot.next();
          }
          if (!mine) continue;
          const uint32_t r0 = j * N + half * COLS;
#pragma unroll
          for (uint32_t c0 = 0; c0 < COLS; c0 += CHUNK) {
            if (r0 + c0 >= A.rows) break;
            uint32_t word = 0xFFFFFFFFu;  // lane c holds the mask's word of row c
            if (A.mask && lane < CHUNK && r0 + c0 + lane < A.rows) word = __ldg(A.mask + (size_t)(r0 + c0 + lane) * A.mask_stride + s);
#pragma unroll
            for (uint32_t c = 0; c < CHUNK; ++c) {
              const uint32_t m = __shfl_sync(0xFFFFFFFFu, word, c);
              const float y = !((m >> lane) & 1u) ? -__int_as_float(0x7F800000) : failed ? __int_as_float(0x7FC00000) : sum[c0 + c];
              if (r0 + c0 + c < A.rows && v < A.V) put(logits + (size_t)(r0 + c0 + c) * A.row_stride + v, y);
            }
          }
        }
    }
    __syncthreads();  // the lists are made anew
  }

  // nothing of this block's is in flight when it ends: every copy has landed and every product is through
  if (warp <= 1 && lane == 0) {
    uint64_t* const bars = warp == 0 ? S.full : S.empty;
    for (uint32_t i = 0; i < Shape::stages; ++i) {
      const uint32_t uses = issued / Shape::stages + (i < issued % Shape::stages ? 1u : 0u);
      if (uses) bar_drain(&bars[i], (uses - 1u) & 1u);
    }
  }
  before_sync();
  __syncthreads();
  after_sync();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(S.tmem), "n"(TMEM) : "memory");
}

using EncodeTiled = decltype(&cuTensorMapEncodeTiled);
EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult got;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &got) != cudaSuccess || got != cudaDriverEntryPointSuccess) p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

// Bytes in rows, copied in boxes of box_rows x 128 as tile_desc() describes them; what lies outside is zero.
bool byte_map(CUtensorMap* map, const uint8_t* p, uint32_t cols, uint32_t rows, size_t stride, uint32_t box_rows) {
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {stride};
  const cuuint32_t box[2] = {BLOCK, box_rows}, steps[2] = {1, 1};
  return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct HeadOperands {
  const uint8_t *hidden, *weight;
  size_t hidden_stride, weight_stride;
};

template <typename T, uint32_t N>
fmt_status launch_head(const HeadOperands& O, const HeadArgs& A, uint32_t sms, cudaStream_t st) {
  CUtensorMap wmap, xmap;
  if (!encode_tiled() || !byte_map(&wmap, O.weight, A.K, A.V, O.weight_stride, SLAB) || !byte_map(&xmap, O.hidden, A.K, A.rows, O.hidden_stride, N)) {
    set_last_error("the operands cannot be described to the copy engine");
    return FMT_ERR_CUDA;
  }
  auto* k = head_kernel<T, N>;
  if (cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, HeadShape<N>::smem)) return launch_result(e);
  // Rows that need several tiles: a block takes all of them for its slabs (the weights come from L2 after the first), unless
  // the slabs divide badly among the blocks; then the tiles of rows are dealt out, too.  A tile costs the same however few
  // of its four slabs are there.
  const uint32_t slabs = (A.V + SLAB - 1) / SLAB, row_tiles = (A.rows + N - 1) / N;
  uint32_t split = 1, least = 0xFFFFFFFFu;
  for (uint32_t y = 1; y <= row_tiles && y <= sms; ++y) {
    const uint32_t x = std::min(sms / y, slabs);
    const uint32_t cost = ((slabs + x - 1) / x + TILE_SLABS - 1) / TILE_SLABS * ((row_tiles + y - 1) / y);
    if (cost < least) least = cost, split = y;
  }
  return launch_result(launch_overlapped(k, dim3(std::min(sms / split, slabs), split), dim3(HEAD_THREADS), HeadShape<N>::smem, st, wmap, xmap, A));
}

template <typename T>
fmt_status head(const HeadOperands& O, const HeadArgs& A, uint32_t sms, cudaStream_t st) {
  if (A.rows <= 16) return launch_head<T, 16>(O, A, sms, st);
  if (A.rows <= 32) return launch_head<T, 32>(O, A, sms, st);
  if (A.rows <= 64) return launch_head<T, 64>(O, A, sms, st);
  if (A.rows <= 128) return launch_head<T, 128>(O, A, sms, st);
  return launch_head<T, 256>(O, A, sms, st);
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
  int dev = 0, sms = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return launch_result(e);
  if (cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) return launch_result(e);
  const HeadOperands O{hidden_dev, weight_dev, hidden_stride, weight_stride};
  const HeadArgs A{hidden_scales_dev, hidden_scale_stride, weight_scales_dev, weight_scale_stride, rows, V, K, mask_dev, mask_stride_words,
                   logits_dev, row_stride_elems};
  return dtype == FMT_BF16 ? head<uint16_t>(O, A, (uint32_t)sms, (cudaStream_t)stream) : head<float>(O, A, (uint32_t)sms, (cudaStream_t)stream);
}
