// The output head: values in 8-bit floating point with a scale for each block, and their product under the mask.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "../../include/fmt.h"
#include "kernels.h"
#include "op_args.h"

using namespace fmt;

namespace {

constexpr uint32_t BLOCK = 128;  // columns (and, of weights, rows) that share a scale

__device__ __forceinline__ float to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

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

// Four values of a row in one go where they are whole and aligned, else one by one; what is behind the row's end is 0.
__device__ __forceinline__ float4 load4(const uint16_t* x, uint32_t n, bool aligned) {
  if (aligned && n >= 4) {
    const uint2 u = *reinterpret_cast<const uint2*>(x);
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xFFFF0000u));
  }
  return make_float4(n > 0 ? to_f32(x[0]) : 0.0f, n > 1 ? to_f32(x[1]) : 0.0f, n > 2 ? to_f32(x[2]) : 0.0f, n > 3 ? to_f32(x[3]) : 0.0f);
}
__device__ __forceinline__ float4 load4(const float* x, uint32_t n, bool aligned) {
  if (aligned && n >= 4) return *reinterpret_cast<const float4*>(x);
  return make_float4(n > 0 ? x[0] : 0.0f, n > 1 ? x[1] : 0.0f, n > 2 ? x[2] : 0.0f, n > 3 ? x[3] : 0.0f);
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ void store4(uint8_t* q, uint32_t n, bool aligned, float4 x, float scale) {
  const uint32_t v = to_e4m3(x.x, scale) | (uint32_t)to_e4m3(x.y, scale) << 8 | (uint32_t)to_e4m3(x.z, scale) << 16 | (uint32_t)to_e4m3(x.w, scale) << 24;
  if (aligned && n >= 4) *reinterpret_cast<uint32_t*>(q) = v;
  else
    for (uint32_t i = 0; i < n && i < 4; ++i) q[i] = (uint8_t)(v >> (8u * i));
}

// Hidden states: a warp to 128 values of a row, four to a lane.  Weights: a thread block to 128 x 128, 16 rows to a warp, which keeps
// them in registers until the block's largest is known.  Either way a value is read once.  Us of bf16 and fp32, and those of the
// bytes: hidden states 64 x 4,096 1.8, 2,048 x 4,096 12.8 and 12.7 (3.8, 6.4), 8,192 x 8,192 98 and 97 (31, 51), which instructions bound
// (180 for four values, the quotients in IEEE single precision among them; 85 % of all issue slots); weights 128,256 x 4,096, once a
// model, 1,313 and 654 (241, 401), with a quarter of the warps, of which bf16 ones wait for their loads most of the time.
constexpr uint32_t QUANTIZE_WARPS = 8;
template <typename T, uint32_t ROWS>
__global__ void __launch_bounds__(QUANTIZE_WARPS * 32) quantize_kernel(const T* x, uint32_t rows, uint32_t cols, size_t row_stride, uint8_t* q,
                                                                       size_t q_stride, float* scales, size_t scale_stride) {
  before_me();
  constexpr uint32_t EACH = ROWS == 1 ? 1 : ROWS / QUANTIZE_WARPS;  // rows of a warp
  __shared__ uint32_t most[QUANTIZE_WARPS];
  const uint32_t warp = threadIdx.x / 32u, lane = threadIdx.x % 32u, blocks = (cols + BLOCK - 1) / BLOCK;
  const uint64_t unit = ROWS == 1 ? (uint64_t)blockIdx.x * QUANTIZE_WARPS + warp : blockIdx.x;
  const uint32_t b = (uint32_t)(unit % blocks), c = b * BLOCK + lane * 4u, left = c < cols ? cols - c : 0u;
  const uint64_t group = unit / blocks;  // of ROWS rows
  const uint64_t r0 = ROWS == 1 ? group : group * ROWS + warp * EACH;
  const bool x_aligned = ((reinterpret_cast<uintptr_t>(x) | row_stride * sizeof(T)) & (4u * sizeof(T) - 1u)) == 0;
  const bool q_aligned = ((reinterpret_cast<uintptr_t>(q) | q_stride) & 3u) == 0;
  float4 v[EACH];
  uint32_t amax = 0u;
#pragma unroll
  for (uint32_t i = 0; i < EACH; ++i) v[i] = load4(x + (r0 + i) * row_stride + c, r0 + i < rows ? left : 0u, x_aligned);
#pragma unroll
  for (uint32_t i = 0; i < EACH; ++i) amax = max(max(max(amax, magnitude(v[i].x)), max(magnitude(v[i].y), magnitude(v[i].z))), magnitude(v[i].w));
  amax = __reduce_max_sync(0xFFFFFFFFu, amax);
  if (ROWS > 1) {
    if (lane == 0) most[warp] = amax;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < QUANTIZE_WARPS; ++i) amax = max(amax, most[i]);
  }
  const float scale = block_scale(amax);
  if (r0 < rows && lane == 0 && (ROWS == 1 || warp == 0)) scales[ROWS == 1 ? (size_t)b * scale_stride + r0 : (size_t)group * scale_stride + b] = scale;
#pragma unroll
  for (uint32_t i = 0; i < EACH; ++i)
    if (r0 + i < rows) store4(q + (r0 + i) * q_stride + c, left, q_aligned, v[i], scale);
}

// ------------------------------------------------------------------------------------------------ the product
//
// On the tensor cores, one block of 128 columns at a time: four tcgen05.mma of 32 columns each make the block's sums in tensor
// memory, from where eight warps take them, multiply them with the block's two scales and add them up in registers.  (Scales of
// any value cannot ride along in the instruction, whose own are powers of two.)
//
// A thread block to an SM.  The vocabulary goes to the blocks in slabs of 32 tokens, a word of the mask: four at a time, one block
// after the other, and what is left then one by one, so that work is even to a slab (128,256 tokens: 27 or 28 of 4,008 to each of
// 148).  A block makes a list of its slabs that some row may use, and takes several at a time, wherever they lie; the others are
// written as -inf and their weights not read.  Four slabs that follow one another are copied in one go (64 rows x 128,256 x 4,096,
// weights from HBM: 95.1 us, and 97.4 with a copy for each slab; from 256 rows on no difference).
//
// Few rows (up to 64): the vocabulary is the M side, four slabs to the 128 lanes of tensor memory, and 16, 32 or 64 rows the N
// side: M is 128 whatever is there, and a decoding step has many tokens and few rows.  More rows: 128 rows are the M side and eight
// slabs the N side.  A lane is a row then, and one product of scales serves the 32 sums of a slab.  More than 128 rows: two blocks
// on neighbouring SMs work as a pair (cta_group::2) on 256 rows and eight slabs, each with its own 128 rows and half of the slabs in
// memory.  A block of columns is then 32 KB of shared memory written and read by each SM, where it was 48 KB, and shared memory
// (128 bytes a cycle) was what the products waited for.
//
// Warps: 0 copies weights and 3 hidden states to shared memory (TMA, a ring of stages), 1 issues the products, 2 copies the scales
// (a ring of their own, as they are needed later), 4 to 11 add up and write.

constexpr uint32_t SLAB = 32;
constexpr uint32_t HEAD_THREADS = 384, ADD_WARPS = 8;
constexpr uint32_t LIST = 512;        // slabs of a block, at most
constexpr uint32_t MOST_TOKENS = 1u << 20;
// Masks that every block looks at as a whole, and of what vocabularies (whose bits are 1 KB then).  Looking takes every block the time of all
// words: us of 32,000 and of 128,256 x 4,096 with a block's own slabs alone, and as a whole: 8 narrow rows 13.3 and 10.6, 14.2 and 13.2; 16
// rows 13.8 and 11.9, 15.8 and 16.7; 32 rows 20.4 and 17.5, 36.8 and 36.7; 64 rows 26 and 34, 50 and 70; where half of the rows may use all
// slabs, nothing is won: 8 rows 24.7 and 26.3, 83.3 and 87.1; 32 rows 25.8 and 30.6, 87 and 102.
constexpr uint32_t ALL_SLABS = 8192, ALL_WORDS = 32768;
constexpr uint32_t SCALE_SLOTS = 8;
constexpr uint32_t SLAB_BYTES = SLAB * BLOCK;
constexpr uint32_t WAIT_POLLS = 1u << 18;  // of 2,900 cycles, the time after which a wait for nothing comes back
std::atomic<uint32_t> wait_polls{WAIT_POLLS};
constexpr uint32_t WIDE_ROWS = 128;        // the M side's
constexpr uint32_t TURN = 16;              // words of a row that a warp turns round in shared memory on their way out

// FEW: rows (at most 64) are the N side.  WIDE: 128 rows are the M side.  PAIR: 256 rows are, 128 in each of two blocks.
enum HeadForm { FEW, WIDE, PAIR };

template <uint32_t ROWS, HeadForm FORM>
struct HeadShape {
  static constexpr uint32_t slabs = FORM == FEW ? 4 : 8;                        // of a tile
  static constexpr uint32_t slabs_here = FORM == PAIR ? 4 : slabs;              // of them in this block's memory
  static constexpr uint32_t columns = FORM == FEW ? ROWS : slabs * SLAB;        // of tensor memory
  static constexpr uint32_t depth = FORM != FEW ? 1 : ROWS == 16 ? 4 : 2;       // blocks of columns that make a stage: each round of waits costs some 400 cycles (8 narrow rows of 32,000 x 4,096: 13.2 us by twos, 12.1 by fours)
  static constexpr uint32_t stages = FORM == PAIR ? 6 : FORM == WIDE ? 4 : ROWS == 64 ? 4 : ROWS == 32 ? 5 : 3;
  static constexpr uint32_t bufs = FORM == FEW ? 4 : 2;                         // of tensor memory, depth x columns each
  static constexpr uint32_t block_bytes = slabs_here * SLAB_BYTES + ROWS * BLOCK;
  static constexpr uint32_t stage_bytes = depth * block_bytes;
  static constexpr uint32_t block_floats = ROWS + slabs;                        // scales
  static constexpr uint32_t slot_floats = depth * block_floats;
  static constexpr uint32_t own_floats = FORM == FEW ? 0 : 32 * (TURN + 1);     // of an adding warp
  static constexpr uint32_t smem = 1024 + stages * stage_bytes + (SCALE_SLOTS * slot_floats + ADD_WARPS * own_floats) * 4;
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
  uint32_t polls;  // of a wait, at most
};

struct HeadShared {
  uint64_t full[6], empty[6], sums_full[4], sums_empty[4], both_empty[4], through;
  uint32_t tmem, n_live, n_dead, polls, copied[4];  // (copied: stages, by the copying warps of this block and the other one)
  volatile uint32_t gave_up;
  uint32_t bits[ALL_SLABS / 32], upto[ALL_SLABS / 32];
  uint32_t live[LIST], dead[LIST];
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory");
}
__device__ __forceinline__ bool bar_test(uint64_t* b, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(done) : "r"(smem_addr(b)), "r"(parity) : "memory");
  return done != 0u;
}
// The same variable in the memory of the pair's first block (of a block by itself: its own).
template <HeadForm FORM>
__device__ __forceinline__ uint32_t at_first(const void* p) {
  uint32_t a = smem_addr(p);
  if (FORM == PAIR) asm("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(a));
  return a;
}
template <HeadForm FORM>
__device__ __forceinline__ void bar_arrive_at(uint32_t addr) {
  if (FORM == PAIR) asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
  else asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(addr) : "memory");
}
template <HeadForm FORM>
__device__ __forceinline__ void bar_expect_at(uint32_t addr, uint32_t bytes) {
  if (FORM == PAIR) asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(addr), "r"(bytes) : "memory");
  else asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(addr), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint32_t pair_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Waits until the barrier's phase of this parity is over.  False: given up, here or by another warp of the block.  Who has given up asks for
// no copy or product any more and arrives at no barrier of scales or sums: a phase that is over is so by whom it waits for, and nothing is
// overwritten that another warp, or the other block of a pair (which may not have given up), still reads.  What the block writes from
// then on is NaN.  (Looking at gave_up before each product instead takes 5 % in pairs: 2,048 rows 1,065 us, and so 1,013.)
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, HeadShared& S) {
  if (bar_test(b, parity)) return true;
  for (uint32_t i = 0; !S.gave_up && i < S.polls; ++i)
    if (bar_test(b, parity)) return true;
  S.gave_up = 1u;
  return false;
}
// The same for a whole warp, which goes on either way and looks at gave_up when it is through with a tile.
__device__ __forceinline__ bool bar_wait_on(uint64_t* b, uint32_t parity, HeadShared& S) {
  const bool there = bar_wait(b, parity, S);
  __syncwarp();
  return there;
}
__device__ __forceinline__ void bar_drain(uint64_t* b, uint32_t parity) {  // the same after giving up, for what is in flight
  for (uint32_t i = 0; i < WAIT_POLLS && !bar_test(b, parity); ++i) {}
}

// One thread of a warp that is all here.  (The compiler knows what this is: operands of copies and products that it sees in one
// thread alone go into uniform registers as they are; under `lane == 0` it makes loops around each of them.)
__device__ __forceinline__ bool elected() {
  uint32_t yes;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(yes));
  return yes != 0u;
}

// A place in a ring and how often it has been round.
template <uint32_t SIZE>
struct Ring {
  uint32_t at = 0, round = 0;
  __device__ __forceinline__ void next() {
    if (++at == SIZE) at = 0, round ^= 1u;
  }
};

template <HeadForm FORM>
__device__ __forceinline__ void tma_load(const CUtensorMap* map, uint32_t bar, uint32_t dst, uint32_t x, uint32_t y) {
  if (FORM == PAIR)  // (the barrier may be the other block's)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                 "l"(map), "r"(bar), "r"(x), "r"(y)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst), "l"(map), "r"(bar),
                 "r"(x), "r"(y)
                 : "memory");
}
// Rows of 128 bytes, swizzled in groups of eight (1,024 bytes), version 1 of the descriptor.
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
template <HeadForm FORM>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  if (FORM == PAIR)
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                 "r"((uint32_t)add)
                 : "memory");
  else
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                 "r"((uint32_t)add)
                 : "memory");
}
// The barrier (in both blocks of a pair) hears when the products issued so far are through.
template <HeadForm FORM>
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
  if (FORM == PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)), "h"((uint16_t)3)
                 : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

template <uint32_t COLS>
__device__ __forceinline__ void tmem_read(uint32_t addr, float (&v)[COLS]);
#define R4(i) "=f"(v[i]), "=f"(v[i + 1]), "=f"(v[i + 2]), "=f"(v[i + 3])
template <>
__device__ __forceinline__ void tmem_read<8>(uint32_t addr, float (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : R4(0), R4(4) : "r"(addr) : "memory");
}
template <>
__device__ __forceinline__ void tmem_read<16>(uint32_t addr, float (&v)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : R4(0), R4(4), R4(8), R4(12) : "r"(addr) : "memory");
}
template <>
__device__ __forceinline__ void tmem_read<32>(uint32_t addr, float (&v)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
               "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : R4(0), R4(4), R4(8), R4(12), R4(16), R4(20), R4(24), R4(28) : "r"(addr) : "memory");
}
#undef R4
// What has been read from tensor memory may be used from here on, by what stays behind it (add_products).
__device__ __forceinline__ void tmem_read_done() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Two products at a time.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
  return p;
}
__device__ __forceinline__ void add_products(uint64_t& sum, float lo, float hi, uint64_t scales) {
  asm volatile("{\n.reg .b64 x;\nmov.b64 x, {%1, %2};\nfma.rn.f32x2 %0, x, %3, %0;\n}" : "+l"(sum) : "f"(lo), "f"(hi), "l"(scales));
}
__device__ __forceinline__ float part(uint64_t p, uint32_t i) { return __uint_as_float((uint32_t)(p >> (32u * i))); }

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = __bfloat16_as_ushort(__float2bfloat16_rn(x)); }

__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
}

// A pair of bf16, -inf where the bytes of `bits` that `which` names do not have their highest bits.
__device__ __forceinline__ uint32_t keep_pair(uint32_t x, uint32_t bits, uint32_t which) {
  uint32_t k;
  asm("prmt.b32 %0, %1, 0, %2;" : "=r"(k) : "r"(bits), "r"(which));  // (selectors 8 and up repeat a byte's highest bit)
  return (x & k) | (0xFF80FF80u & ~k);
}

template <typename T, uint32_t ROWS, HeadForm FORM>
__global__ void __launch_bounds__(HEAD_THREADS, 1) head_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap wmap4,
                                                               const __grid_constant__ CUtensorMap xmap, const HeadArgs A) {
  using Shape = HeadShape<ROWS, FORM>;
  constexpr uint32_t SLABS = Shape::slabs, DEPTH = Shape::depth, BUF = DEPTH * Shape::columns, TMEM = Shape::bufs * BUF, BLOCKS = FORM == PAIR ? 2 : 1;
  constexpr bool LANE_IS_ROW = FORM != FEW;
  extern __shared__ uint8_t raw[];
  __shared__ HeadShared S;
  const uint32_t tiles_at = (smem_addr(raw) + 1023u) & ~1023u;  // (the same in both blocks of a pair)
  float* const scales = reinterpret_cast<float*>(raw + (tiles_at - smem_addr(raw)) + Shape::stages * Shape::stage_bytes);
  const uint32_t tid = threadIdx.x, warp = tid / 32u, lane = tid % 32u;
  const uint32_t rank = FORM == PAIR ? pair_rank() : 0u;
  const uint32_t n_slabs = (A.V + SLAB - 1) / SLAB, n_blocks = (A.K + BLOCK - 1) / BLOCK, row_tiles = (A.rows + BLOCKS * ROWS - 1) / (BLOCKS * ROWS);
  const uint32_t party = blockIdx.x / BLOCKS, parties = gridDim.x / BLOCKS;  // a party is a block or a pair: both blocks have the same slabs

  if (tid == 0) {
    for (uint32_t i = 0; i < Shape::stages; ++i) bar_init(&S.full[i], 2 * BLOCKS), bar_init(&S.empty[i], 1);
    for (uint32_t i = 0; i < Shape::bufs; ++i) bar_init(&S.sums_full[i], 2), bar_init(&S.sums_empty[i], ADD_WARPS), bar_init(&S.both_empty[i], 2 * ADD_WARPS);
    bar_init(&S.through, 1);
    S.polls = A.polls, S.gave_up = A.polls == 0u, S.copied[0] = S.copied[1] = S.copied[2] = S.copied[3] = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (FORM == PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&S.tmem)), "n"(TMEM) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&S.tmem)), "n"(TMEM) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  before_sync();
  __syncthreads();
  if (FORM == PAIR) pair_sync();  // the other block's barriers are there
  after_sync();
  before_me();

  Ring<Shape::stages> stage;
  Ring<Shape::bufs> buf;
  Ring<SCALE_SLOTS> slot;
  uint32_t copied = 0;  // stages, by this thread
  bool failed = false;

  // n things are dealt out four at a time, as long as there are four for every block (`fours` times), and then one by one
  auto share = [&](uint32_t n, uint32_t fours) { return 4u * fours + (n - 4u * fours * parties + parties - 1u - party) / parties; };
  auto place = [&](uint32_t i, uint32_t fours) {  // of the block's i-th
    return i < 4u * fours ? 4u * (i / 4u * parties + party) + i % 4u : i * parties + party;
  };
  const uint32_t fours = n_slabs / (4u * parties), n_mine = share(n_slabs, fours);
  auto slab_no = [&](uint32_t i) { return place(i, fours); };
  // Small masks are looked at as a whole by every block, and what is left of the vocabulary is dealt out anew: where a grammar leaves
  // few tokens, a block's own slabs have five or six of them, or none (8 rows of 32,000 x 4,096: 13.3 us, so 10.6).
  const bool whole = A.mask && n_slabs <= ALL_SLABS && (uint64_t)n_slabs * A.rows <= ALL_WORDS && n_slabs > parties;  // (a block has no more of those than of all)
  // The block's slabs that some row may use, and the others.
  if (whole) {
    // lanes are slabs, whose words lie side by side; four times 32 slabs and eight rows are asked for at a time
    constexpr uint32_t AT_ONCE = 4, WARPS = HEAD_THREADS / 32;
    for (uint32_t i = warp; i < (n_slabs + 31u) / 32u; i += AT_ONCE * WARPS) {
      uint32_t any[AT_ONCE] = {};
#pragma unroll 8
      for (uint32_t r = 0; r < A.rows; ++r)
#pragma unroll
        for (uint32_t u = 0; u < AT_ONCE; ++u) {
          const uint32_t no = (i + u * WARPS) * 32u + lane;
          if (no < n_slabs) any[u] |= A.mask[(size_t)r * A.mask_stride + no];
        }
#pragma unroll
      for (uint32_t u = 0; u < AT_ONCE; ++u) {
        const uint32_t word = __ballot_sync(0xFFFFFFFFu, any[u] != 0u);
        if (lane == 0 && i + u * WARPS < (n_slabs + 31u) / 32u) S.bits[i + u * WARPS] = word;
      }
    }
    __syncthreads();
    if (warp == 0) {  // the slabs that some row may use are dealt out among the blocks as all are otherwise
      uint32_t seen = 0;
      for (uint32_t i = 0; i < (n_slabs + 31u) / 32u; i += 32) {
        uint32_t upto = i + lane < (n_slabs + 31u) / 32u ? __popc(S.bits[i + lane]) : 0u;
#pragma unroll
        for (uint32_t o = 1; o < 32u; o <<= 1) {
          const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
          if (lane >= o) upto += x;
        }
        upto += seen;
        if (i + lane < ALL_SLABS / 32) S.upto[i + lane] = upto;  // how many there are up to the end of this word
        seen = __shfl_sync(0xFFFFFFFFu, upto, 31);
      }
      __syncwarp();
      const uint32_t by_four = seen / (4u * parties), n_live = share(seen, by_four);
      for (uint32_t k = lane; k < n_live; k += 32) {
        const uint32_t no = place(k, by_four);  // among those
        uint32_t lo = 0, hi = (n_slabs + 31u) / 32u - 1u;
        while (lo < hi) {
          const uint32_t mid = (lo + hi) / 2;
          if (S.upto[mid] > no) hi = mid;
          else lo = mid + 1;
        }
        S.live[k] = lo * 32u + __fns(S.bits[lo], 0, (int)(no - (lo ? S.upto[lo - 1] : 0u)) + 1);
      }
      uint32_t n_dead = 0;
      for (uint32_t k = lane; k < (n_mine + 31u) / 32u * 32u; k += 32) {
        const uint32_t no = k < n_mine ? slab_no(k) : 0u;
        const bool gone = k < n_mine && !((S.bits[no / 32u] >> (no % 32u)) & 1u);
        const uint32_t all = __ballot_sync(0xFFFFFFFFu, gone);
        if (gone) S.dead[n_dead + __popc(all & ((1u << lane) - 1u))] = no;
        n_dead += __popc(all);
      }
      if (lane == 0) S.n_live = n_live, S.n_dead = n_dead;
    }
  } else {
    if (tid < LIST / 32) S.bits[tid] = A.mask ? 0u : 0xFFFFFFFFu;
    __syncthreads();
    if (A.mask)
      for (uint32_t i = warp; i < n_mine; i += HEAD_THREADS / 32) {
        const uint32_t* m = A.mask + slab_no(i);
        uint32_t any = 0u;
        for (uint32_t r0 = 0; r0 < A.rows && !any; r0 += 256) {
#pragma unroll
          for (uint32_t u = 0; u < 8; ++u)
            if (r0 + u * 32u + lane < A.rows) any |= m[(size_t)(r0 + u * 32u + lane) * A.mask_stride];
          any = __any_sync(0xFFFFFFFFu, any != 0u);
        }
        if (lane == 0 && any) atomicOr(&S.bits[i / 32], 1u << (i % 32));
      }
    __syncthreads();
    if (warp == 0) {
      uint32_t n_live = 0, n_dead = 0;
      for (uint32_t i = 0; i < n_mine; i += 32) {
        const uint32_t word = S.bits[i / 32], in = n_mine - i < 32u ? (1u << (n_mine - i)) - 1u : 0xFFFFFFFFu;
        const uint32_t alive = word & in, gone = ~word & in, before = (1u << lane) - 1u, no = slab_no(i + lane);
        if ((alive >> lane) & 1u) S.live[n_live + __popc(alive & before)] = no;
        if ((gone >> lane) & 1u) S.dead[n_dead + __popc(gone & before)] = no;
        n_live += __popc(alive), n_dead += __popc(gone);
      }
      if (lane == 0) S.n_live = n_live, S.n_dead = n_dead;
    }
  }
  __syncthreads();
  const uint32_t n_live = S.n_live;

  if (warp < 4) {
    if (LANE_IS_ROW) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");  // 384 threads of 168 registers: 256 x 216 + 128 x 72 are no more
    if (warp == 0 && elected()) {
      for (uint32_t g = 0; g < n_live && !failed; g += SLABS)
        for (uint32_t j = blockIdx.y; j < row_tiles && !failed; j += gridDim.y) {
          // this block's slabs of the tile: all, or the first or second half of them
          const uint32_t there = min(SLABS, n_live - g), half = (there + 1u) / 2u, from = FORM == PAIR ? g + rank * half : g;
          const uint32_t count = FORM == PAIR ? (rank ? there - half : half) : there;
          uint32_t y[Shape::slabs_here], whole = 0u;  // the slabs' rows, and of four slabs, whether they follow one another
#pragma unroll
          for (uint32_t i = 0; i < Shape::slabs_here; ++i) {
            y[i] = i < count ? S.live[from + i] * SLAB : 0u;
            if (i % 4u == 3u && i < count && y[i] == y[i - i % 4u] + 3u * SLAB) whole |= 1u << i / 4u;
          }
          for (uint32_t b = 0; b < n_blocks; b += DEPTH) {
            if (!bar_wait(&S.empty[stage.at], stage.round ^ 1u, S)) {
              failed = true;
              break;
            }
            const uint32_t blocks = min(DEPTH, n_blocks - b), bar = at_first<FORM>(&S.full[stage.at]);
            uint32_t at = tiles_at + stage.at * Shape::stage_bytes;
            if (FORM != PAIR || count) bar_expect_at<FORM>(bar, blocks * count * SLAB_BYTES);
            else bar_arrive_at<FORM>(bar);
            for (uint32_t k = b; k < b + blocks; ++k, at += Shape::block_bytes) {
#pragma unroll
              for (uint32_t i = 0; i < Shape::slabs_here / 4; ++i) {
                if ((whole >> i) & 1u) {
                  tma_load<FORM>(&wmap4, bar, at + 4u * i * SLAB_BYTES, k * BLOCK, y[4u * i]);
                } else {
#pragma unroll
                  for (uint32_t q = 4u * i; q < 4u * i + 4u; ++q)
                    if (q < count) tma_load<FORM>(&wmap, bar, at + q * SLAB_BYTES, k * BLOCK, y[q]);
                }
              }
            }
            ++copied;
            stage.next();
          }
        }
    } else if (warp == 3 && elected()) {
      for (uint32_t g = 0; g < n_live && !failed; g += SLABS)
        for (uint32_t j = blockIdx.y; j < row_tiles && !failed; j += gridDim.y)
          for (uint32_t b = 0; b < n_blocks; b += DEPTH) {
            if (!bar_wait(&S.empty[stage.at], stage.round ^ 1u, S)) {
              failed = true;
              break;
            }
            const uint32_t blocks = min(DEPTH, n_blocks - b), bar = at_first<FORM>(&S.full[stage.at]);
            uint32_t at = tiles_at + stage.at * Shape::stage_bytes + Shape::slabs_here * SLAB_BYTES;
            bar_expect_at<FORM>(bar, blocks * ROWS * BLOCK);
            for (uint32_t k = b; k < b + blocks; ++k, at += Shape::block_bytes) tma_load<FORM>(&xmap, bar, at, k * BLOCK, (j * BLOCKS + rank) * ROWS);
            ++copied;
            stage.next();
          }
    } else if (warp == 1 && rank == 0 && elected()) {  // (a pair's products are issued by its first block, for both)
      for (uint32_t g = 0; g < n_live && !failed; g += SLABS)
        for (uint32_t j = blockIdx.y; j < row_tiles && !failed; j += gridDim.y) {
          // e4m3 x e4m3 into fp32, both K-major, 128 lanes (of each block)
          const uint32_t there = min(SLABS, n_live - g), columns = FORM == FEW ? ROWS : FORM == WIDE ? there * SLAB : (there + 1u) / 2u * 2u * SLAB;
          const uint32_t idesc = 1u << 4 | (columns >> 3) << 17 | (BLOCKS * 128u >> 4) << 24;
          for (uint32_t b = 0; b < n_blocks; b += DEPTH) {
            const uint32_t at = tiles_at + stage.at * Shape::stage_bytes, d = S.tmem + buf.at * BUF;
            const uint64_t w = tile_desc(at), x = tile_desc(at + Shape::slabs_here * SLAB_BYTES);
            // the copies are early, mostly; the sums' place is what it waits for
            if (!bar_wait(&S.full[stage.at], stage.round, S) || !bar_wait(FORM == PAIR ? &S.both_empty[buf.at] : &S.sums_empty[buf.at], buf.round ^ 1u, S)) {
              failed = true;
              break;
            }
            after_sync();
#pragma unroll
            for (uint32_t k = 0; k < DEPTH; ++k)
              if (k == 0 || b + k < n_blocks) {
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                  const uint32_t more = (k * Shape::block_bytes + 32u * i) >> 4;
                  mma<FORM>(d + k * Shape::columns, (LANE_IS_ROW ? x : w) + more, (LANE_IS_ROW ? w : x) + more, idesc, i != 0);
                }
              }
            mma_commit<FORM>(&S.empty[stage.at]);
            mma_commit<FORM>(&S.sums_full[buf.at]);
            stage.next(), buf.next();
          }
        }
    } else if (warp == 2) {
      // A stage's scales are asked for AHEAD stages early, and their being there is one of the two things that sums_full waits for.
      constexpr uint32_t AHEAD = SCALE_SLOTS - Shape::bufs;
      const uint32_t total = (n_live + SLABS - 1) / SLABS * ((row_tiles + gridDim.y - 1 - blockIdx.y) / gridDim.y) * ((n_blocks + DEPTH - 1) / DEPTH);
      uint32_t g = 0, j = blockIdx.y, b = 0;
      for (uint32_t t = 0; t < total + AHEAD; ++t) {
        if (t >= AHEAD && !bar_wait_on(&S.sums_empty[buf.at], buf.round ^ 1u, S)) failed = true;
        if (t < total) {
          const uint32_t count = min(SLABS, n_live - g), r0 = (j * BLOCKS + rank) * ROWS;
          for (uint32_t k = b; k < min(b + DEPTH, n_blocks); ++k) {
            const uint32_t dst = smem_addr(scales + slot.at * Shape::slot_floats + (k - b) * Shape::block_floats);
            const float* xp = A.xs + (size_t)k * A.xs_stride + r0;
#pragma unroll
            for (uint32_t i = 0; i < (ROWS + 31u) / 32u; ++i) {
              const uint32_t c = i * 32u + lane;
              if (c < ROWS && r0 + c < A.rows) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + c * 4u), "l"(xp + c) : "memory");
            }
            if (lane < count)
              asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + (ROWS + lane) * 4u),
                           "l"(A.ws + (size_t)(S.live[g + lane] * SLAB / BLOCK) * A.ws_stride + k) : "memory");
          }
          slot.next();
          b += DEPTH;
          if (b >= n_blocks) {
            b = 0, j += gridDim.y;
            if (j >= row_tiles) j = blockIdx.y, g += SLABS;
          }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (t >= AHEAD) {
          asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory");
          __syncwarp();
          if (lane == 0 && !failed) bar_arrive(&S.sums_full[buf.at]);
          buf.next();
        }
      }
    }
    __syncwarp();
    if (warp == 1 && rank == 0 && elected()) mma_commit<FORM>(&S.through);
    if ((warp == 0 || warp == 3) && copied)  // (the thread that was elected)
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at_first<FORM>(&S.copied[rank * 2u + (warp ? 1u : 0u)])), "r"(copied) : "memory");
    __syncwarp();
  } else {
    if (LANE_IS_ROW) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const uint32_t quarter = warp % 4u, half = (warp - 4u) / 4u;  // 32 lanes of tensor memory, half of the columns
    T* const logits = static_cast<T*>(A.logits);
    float* const own = scales + SCALE_SLOTS * Shape::slot_floats + (warp - 4u) * Shape::own_floats;
    const float minus_inf = -__int_as_float(0x7F800000), nan = __int_as_float(0x7FC00000);
    const uintptr_t begins = reinterpret_cast<uintptr_t>(logits) | A.row_stride * sizeof(T);  // rows begin at multiples of
    const bool by_units = (begins & 31u) == 0, by_words = (begins & 3u) == 0;                 // 32 or of four bytes
    // the slabs that no row may use
    for (uint32_t i = warp - 4u; i < S.n_dead; i += ADD_WARPS) {
      const uint32_t v = S.dead[i] * SLAB + lane;
      if (v < A.V)
        for (uint32_t r = blockIdx.y * BLOCKS + rank; r < A.rows; r += gridDim.y * BLOCKS) put(logits + (size_t)r * A.row_stride + v, minus_inf);
    }
    for (uint32_t g = 0; g < n_live; g += SLABS)
      for (uint32_t j = blockIdx.y; j < row_tiles; j += gridDim.y) {
        constexpr uint32_t COLS = Shape::columns / 2;      // of the tile, this warp's
        constexpr uint32_t CHUNK = COLS < 32 ? COLS : 32;  // read from tensor memory in one go
        constexpr uint32_t READS = DEPTH * COLS / CHUNK;   // of a stage; an even number
        constexpr uint32_t FACTORS = LANE_IS_ROW ? 4 : DEPTH * COLS / 2;
        const uint32_t count = n_live - g;                 // slabs that are there
        const uint32_t mine = LANE_IS_ROW ? (count > half * 4u ? min(4u, count - half * 4u) : 0u) : quarter < count ? 1u : 0u;
        // The masks' words are asked for now.  Where a lane is a row, a word for each of its slabs; else lane c holds row c's.
        constexpr uint32_t WORDS = LANE_IS_ROW ? 4 : 1;
        const uint32_t r0 = (j * BLOCKS + rank) * ROWS + (LANE_IS_ROW ? quarter * 32u : half * COLS);  // the first of the warp's rows
        uint32_t word[WORDS];
#pragma unroll
        for (uint32_t i = 0; i < WORDS; ++i) {
          word[i] = 0xFFFFFFFFu;
          if (A.mask && (LANE_IS_ROW ? i < mine : mine && lane < COLS) && r0 + lane < A.rows)
            word[i] = A.mask[(size_t)(r0 + lane) * A.mask_stride + S.live[g + (LANE_IS_ROW ? half * 4u + i : quarter)]];
        }
        uint64_t sum[COLS / 2];
#pragma unroll
        for (uint32_t c = 0; c < COLS / 2; ++c) sum[c] = 0;
        // Two pieces are on their way at a time; the first two of the next stage (if it is there) while the last two of this one are added.
        float d[2][CHUNK];
        const uint32_t lanes = S.tmem + (quarter * 32u << 16) + half * COLS;
        auto read = [&](uint32_t r) { tmem_read<CHUNK>(lanes + buf.at * BUF + r * CHUNK / COLS * Shape::columns + r * CHUNK % COLS, d[r % 2]); };
        auto stage_ready = [&] {
          if (!bar_wait_on(&S.sums_full[buf.at], buf.round, S)) failed = true;
          after_sync();
        };
        stage_ready();
        read(0), read(1);
        for (uint32_t b = 0; b < n_blocks; b += DEPTH) {
          uint64_t by[FACTORS];  // the products of two scales
          const float* sc = scales + slot.at * Shape::slot_floats;
          if (LANE_IS_ROW) {  // a row's scale times its slabs'
            const float x = sc[quarter * 32u + lane];
            const float4 w = *reinterpret_cast<const float4*>(sc + ROWS + half * 4u);
            by[0] = pair(x * w.x, x * w.x), by[1 % FACTORS] = pair(x * w.y, x * w.y);
            by[2 % FACTORS] = pair(x * w.z, x * w.z), by[3 % FACTORS] = pair(x * w.w, x * w.w);
          } else {  // the slab's scale times its rows'
#pragma unroll
            for (uint32_t k = 0; k < DEPTH; ++k) {
              const float w = sc[k * Shape::block_floats + ROWS + quarter];
#pragma unroll
              for (uint32_t c = 0; c < COLS; c += 4) {
                const float4 x = *reinterpret_cast<const float4*>(sc + k * Shape::block_floats + half * COLS + c);
                by[(k * COLS + c) / 2 % FACTORS] = pair(x.x * w, x.y * w), by[((k * COLS + c) / 2 + 1) % FACTORS] = pair(x.z * w, x.w * w);
              }
            }
          }
          constexpr uint32_t PER = COLS / CHUNK;  // reads of a block of columns
          auto add = [&](uint32_t r) {
            if (r < PER || b + r / PER < n_blocks) {
#pragma unroll
              for (uint32_t c = 0; c < CHUNK; c += 2)
                add_products(sum[(r % PER * CHUNK + c) / 2], d[r % 2][c], d[r % 2][c + 1], by[LANE_IS_ROW ? r : (r * CHUNK + c) / 2]);
            }
          };
          const bool more = b + DEPTH < n_blocks;
#pragma unroll
          for (uint32_t r = 0; r < READS; r += 2) {
            tmem_read_done();
            if (r + 2 == READS) {
              before_sync();
              __syncwarp();
              if (lane == 0 && !failed) {
                if (FORM == PAIR) bar_arrive_at<FORM>(at_first<FORM>(&S.both_empty[buf.at]));
                bar_arrive(&S.sums_empty[buf.at]);
              }
              buf.next(), slot.next();
            }
            add(r);
            if (r + 2 < READS) read(r + 2);
            else if (more) stage_ready(), read(0);
            add(r + 1);
            if (r + 2 < READS) read(r + 3);
            else if (more) read(1);
          }
        }
        if (S.gave_up) {
#pragma unroll
          for (uint32_t c = 0; c < COLS / 2; ++c) sum[c] = pair(nan, nan);
        }
        if (LANE_IS_ROW && by_units && S.live[g + min(count, SLABS) - 1u] * SLAB + SLAB <= A.V) {
          // a lane holds 32 tokens of a row for each slab, which are two (bf16) or four units of 32 bytes
          if (r0 + lane < A.rows) {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
              if (i >= mine) break;
              uint32_t* const to = reinterpret_cast<uint32_t*>(logits + (size_t)(r0 + lane) * A.row_stride + S.live[g + half * 4u + i] * SLAB);
              const uint32_t allowed = word[i % WORDS];
              uint32_t y[sizeof(T) * SLAB / 4];
#pragma unroll
              for (uint32_t c = 0; c < SLAB; c += 2) {
                const uint64_t two = sum[(i * SLAB + c) / 2 % (COLS / 2)];
                if (sizeof(T) == 2) y[c / 2] = two_bf16(part(two, 0), part(two, 1));
                else y[c % (sizeof(y) / 4)] = (uint32_t)two, y[(c + 1) % (sizeof(y) / 4)] = (uint32_t)(two >> 32);
              }
              if (allowed != 0xFFFFFFFFu) {
                if (sizeof(T) == 2) {
#pragma unroll
                  for (uint32_t c = 0; c < SLAB; c += 4) {
                    const uint32_t bits = ((allowed >> c & 15u) * 0x00204081u & 0x01010101u) << 7;  // each bit the highest of a byte
                    y[c / 2] = keep_pair(y[c / 2], bits, 0x9988u), y[c / 2 + 1] = keep_pair(y[c / 2 + 1], bits, 0xBBAAu);
                  }
                } else {
#pragma unroll
                  for (uint32_t c = 0; c < SLAB; ++c) y[c % (sizeof(y) / 4)] = (allowed >> c) & 1u ? y[c % (sizeof(y) / 4)] : 0xFF800000u;
                }
              }
#pragma unroll
              for (uint32_t q = 0; q < sizeof(y) / 4; q += 8)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + q), "r"(y[q]), "r"(y[q + 1]), "r"(y[q + 2]), "r"(y[q + 3]),
                             "r"(y[q + 4]), "r"(y[q + 5]), "r"(y[q + 6]), "r"(y[q + 7])
                             : "memory");
            }
          }
        } else if (LANE_IS_ROW) {
          const uint32_t rows_here = r0 < A.rows ? min(32u, A.rows - r0) : 0u;
          uint32_t* const words = reinterpret_cast<uint32_t*>(own);
          // One slab's code for all four, which has to be fetched for every tile: sums move down a slab's places each time.
#pragma unroll 1
          for (uint32_t i = 0; i < mine; ++i) {
            if (!rows_here) break;
            const uint32_t v0 = S.live[g + half * 4u + i] * SLAB;
            uint64_t now[SLAB / 2];
            const uint32_t allowed = word[0];
#pragma unroll
            for (uint32_t c = 0; c < SLAB / 2; ++c) now[c] = sum[c % (COLS / 2)];
#pragma unroll
            for (uint32_t c = SLAB / 2; c < COLS / 2; ++c) sum[(c - SLAB / 2) % (COLS / 2)] = sum[c];
#pragma unroll
            for (uint32_t k = 1; k < WORDS; ++k) word[k - 1] = word[k];
            auto masked = [&](uint32_t c) { return (allowed >> c) & 1u ? part(now[c / 2], c % 2) : minus_inf; };
            auto packed = [&](uint32_t c) {  // word c of the slab's row
              return sizeof(T) == 4 ? __float_as_uint(masked(c % SLAB)) : two_bf16(masked(2 * c % SLAB), masked((2 * c + 1) % SLAB));
            };
            // rows that begin elsewhere: turned round in shared memory, 16 words of a row at a time, so that a warp writes them side by side
            constexpr uint32_t TOKENS = TURN * 4 / sizeof(T);
#pragma unroll
            for (uint32_t t = 0; t < SLAB; t += TOKENS) {
#pragma unroll
              for (uint32_t c = 0; c < TURN; ++c) words[lane * (TURN + 1) + c] = packed(t * sizeof(T) / 4 + c);
              __syncwarp();
              if (by_words) {
                const uint32_t c = lane % TURN, v = v0 + t + c * (4 / sizeof(T));
                T* to = logits + (size_t)(r0 + lane / TURN) * A.row_stride + v;
                const bool all = v + 4 / sizeof(T) <= A.V, some = v < A.V;
#pragma unroll
                for (uint32_t r = 0; r < 32u; r += 32u / TURN, to += 2 * A.row_stride) {
                  const uint32_t y = words[(r + lane / TURN) * (TURN + 1) + c];
                  if (r + lane / TURN < rows_here) {
                    if (all) *reinterpret_cast<uint32_t*>(to) = y;
                    else if (some) *reinterpret_cast<uint16_t*>(to) = (uint16_t)y;
                  }
                }
              } else {  // bf16
                const uint32_t v = v0 + t + lane;
                T* to = logits + (size_t)r0 * A.row_stride + v;
#pragma unroll
                for (uint32_t r = 0; r < 32u; ++r, to += A.row_stride) {
                  const uint16_t y = reinterpret_cast<const uint16_t*>(words + r * (TURN + 1))[lane];
                  if (r < rows_here && v < A.V) *reinterpret_cast<uint16_t*>(to) = y;
                }
              }
              __syncwarp();
            }
          }
        } else if (mine && r0 < A.rows) {
          const uint32_t v = S.live[g + quarter] * SLAB + lane;
          T* to = logits + (size_t)r0 * A.row_stride + v;
#pragma unroll 1
          for (uint32_t c0 = 0; c0 < COLS && r0 + c0 < A.rows; c0 += 8) {
#pragma unroll
            for (uint32_t c = 0; c < 8; ++c, to += A.row_stride) {
              const uint32_t m = __shfl_sync(0xFFFFFFFFu, word[0], c0 + c);
              const float y = (m >> lane) & 1u ? part(sum[c / 2], c % 2) : minus_inf;
              if (r0 + c0 + c < A.rows && v < A.V) put(to, y);
            }
#pragma unroll
            for (uint32_t c = 4; c < COLS / 2; ++c) sum[c - 4] = sum[c];
          }
        }
      }
  }
  // Nothing is in flight when a block ends: every copy has landed (a stage that not all the copying threads came to fill is filled up
  // first), every product is through, and nobody writes to a block's barriers any more.
  before_sync();
  __syncthreads();
  if (FORM == PAIR) pair_sync();
  after_sync();
  if (warp == 0 && lane == 0 && rank == 0) {
    uint32_t most = 0u;
    for (uint32_t i = 0; i < 2u * BLOCKS; ++i) most = max(most, S.copied[i]);
    for (uint32_t i = 0; i < 2u * BLOCKS; ++i)
      for (uint32_t k = S.copied[i]; k < most; ++k) bar_arrive(&S.full[k % Shape::stages]);
    for (uint32_t k = most - min(most, Shape::stages); k < most; ++k) bar_drain(&S.full[k % Shape::stages], k / Shape::stages & 1u);
  }
  if (warp == 1 && lane == 0) bar_drain(&S.through, 0u);
  before_sync();
  __syncthreads();
  if (FORM == PAIR) pair_sync();
  after_sync();
  if (warp == 1) {
    if (FORM == PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(S.tmem), "n"(TMEM) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(S.tmem), "n"(TMEM) : "memory");
  }
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

template <typename T, uint32_t ROWS, HeadForm FORM>
fmt_status launch_head(const HeadOperands& O, const HeadArgs& A, uint32_t sms, cudaStream_t st) {
  using Shape = HeadShape<ROWS, FORM>;
  constexpr uint32_t BLOCKS = FORM == PAIR ? 2 : 1;
  CUtensorMap wmap, wmap4, xmap;
  if (!encode_tiled()) {
    set_last_error("the driver has no cuTensorMapEncodeTiled");
    return FMT_ERR_CUDA;
  }
  if (!byte_map(&wmap, O.weight, A.K, A.V, O.weight_stride, SLAB) || !byte_map(&wmap4, O.weight, A.K, A.V, O.weight_stride, 4 * SLAB) ||
      !byte_map(&xmap, O.hidden, A.K, A.rows, O.hidden_stride, ROWS)) {
    return refuse("the operands cannot be described to the copy engine (a stride of 2^40 bytes or more?)");
  }
  auto* k = head_kernel<T, ROWS, FORM>;
  // asked for every time: it belongs to the context, of which a process may have several, or another after a reset (no difference in 6.9 us a call)
  if (cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::smem)) return launch_result(e);
  // Rows that need several tiles: a party takes all of them for its slabs (the weights come from L2 after the first), unless
  // the slabs divide badly among the parties; then the tiles of rows are dealt out, too.
  const uint32_t slabs = (A.V + SLAB - 1) / SLAB, row_tiles = (A.rows + BLOCKS * ROWS - 1) / (BLOCKS * ROWS), most = std::max(1u, sms / BLOCKS);
  uint32_t split = 1, least = 0xFFFFFFFFu;
  for (uint32_t y = 1; y <= row_tiles && y <= most; ++y) {
    const uint32_t x = std::min(most / y, slabs), each = (slabs + x - 1) / x, turns = (row_tiles + y - 1) / y;
    if (each <= LIST && (uint64_t)each * turns < least) least = each * turns, split = y;
  }
  if (least == 0xFFFFFFFFu) return refuse("the vocabulary is too large for this device's number of SMs");
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(std::min(most / split, slabs) * BLOCKS, split), cfg.blockDim = dim3(HEAD_THREADS), cfg.dynamicSmemBytes = Shape::smem, cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = 2, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
  cfg.attrs = at, cfg.numAttrs = FORM == PAIR ? 2 : 1;
  return launch_result(cudaLaunchKernelEx(&cfg, k, wmap, wmap4, xmap, A));
}

// us, 128,256 x 4,096 / 32,000 x 4,096: 32 rows by tiles of 16 106 / 45.7, by one of 32 90.4 / 33.8; 16 rows 87.9 / 29.6 and 89.8 / 31.3.
// 64 rows by tiles of 32 118 / 42.2, by one of 64 91.0 / 29.5, with a lane to a row 109 / 33.6; 128 rows by tiles of 64 154 / 48.6, with a
// lane to a row 117 / 34.9, in pairs 148 / 44.1; 200 rows with a lane to a row 179 / 58.6, in pairs 157 / 49.1.  fp32 logits: 128 rows 120 / 37.2
// (bf16 110 / 33.9 then), 256 rows 170 / 58.0, 1,024 rows 591 / 166.
template <typename T>
fmt_status head(const HeadOperands& O, const HeadArgs& A, uint32_t sms, cudaStream_t st) {
  if (A.rows <= 16) return launch_head<T, 16, FEW>(O, A, sms, st);
  if (A.rows <= 32) return launch_head<T, 32, FEW>(O, A, sms, st);
  if (A.rows <= 64) return launch_head<T, 64, FEW>(O, A, sms, st);
  if (A.rows <= WIDE_ROWS) return launch_head<T, WIDE_ROWS, WIDE>(O, A, sms, st);
  return launch_head<T, WIDE_ROWS, PAIR>(O, A, sms, st);
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
  const uint64_t units = (uint64_t)((rows + block_rows - 1) / block_rows) * ((cols + BLOCK - 1) / BLOCK), per = block_rows == 1 ? QUANTIZE_WARPS : 1;
  if ((units + per - 1) / per > 0x7FFFFFFFu) return refuse("rows x cols out of range");
  const dim3 grid((uint32_t)((units + per - 1) / per));
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == FMT_BF16) {
    auto* k = block_rows == 1 ? quantize_kernel<uint16_t, 1> : quantize_kernel<uint16_t, BLOCK>;
    return launch_result(launch_overlapped(k, grid, dim3(QUANTIZE_WARPS * 32), 0, st, (const uint16_t*)x_dev, rows, cols, row_stride_elems, q_dev, q_stride,
                                           scales_dev, scale_stride));
  }
  auto* k = block_rows == 1 ? quantize_kernel<float, 1> : quantize_kernel<float, BLOCK>;
  return launch_result(launch_overlapped(k, grid, dim3(QUANTIZE_WARPS * 32), 0, st, (const float*)x_dev, rows, cols, row_stride_elems, q_dev, q_stride, scales_dev,
                                         scale_stride));
}

extern "C" fmt_status fmt_head_logits(const uint8_t* hidden_dev, size_t hidden_stride, const float* hidden_scales_dev,
                                      size_t hidden_scale_stride, const uint8_t* weight_dev, size_t weight_stride,
                                      const float* weight_scales_dev, size_t weight_scale_stride, uint32_t rows, uint32_t V, uint32_t K,
                                      const uint32_t* mask_dev, size_t mask_stride_words, void* logits_dev, fmt_dtype dtype,
                                      size_t row_stride_elems, void* stream) {
  if (!hidden_dev || !hidden_scales_dev || !weight_dev || !weight_scales_dev || !logits_dev) return refuse("NULL argument");
  if (dtype != FMT_BF16 && dtype != FMT_FP32) return refuse("unknown dtype");
  if (V == 0 || V > MOST_TOKENS || K == 0 || K > (1u << 20) || rows > (1u << 24)) return refuse("rows, V or K out of range");
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
  uint32_t sms;
  if (fmt_status s = count_sms(&sms)) return s;
  const HeadOperands O{hidden_dev, weight_dev, hidden_stride, weight_stride};
  const HeadArgs A{hidden_scales_dev, hidden_scale_stride, weight_scales_dev, weight_scale_stride, rows, V, K, mask_dev, mask_stride_words,
                   logits_dev, row_stride_elems, wait_polls.load(std::memory_order_relaxed)};
  return dtype == FMT_BF16 ? head<uint16_t>(O, A, sms, (cudaStream_t)stream) : head<float>(O, A, sms, (cudaStream_t)stream);
}

extern "C" fmt_status fmt_head_set_wait_limit(uint32_t polls) {
  wait_polls.store(std::min(polls, WAIT_POLLS), std::memory_order_relaxed);
  return FMT_OK;
}
