// Microscaled 4-bit operands: quantisation of bf16 rows, the way back, and the product of two such matrices (a point-wise layer)
// on the block-scaled tensor-core instruction.
#include <cuda.h>
#include <cuda_runtime.h>

#include "activation.cuh"
#include "launch.cuh"
#include "layout.cuh"
#include "mxfp4.cuh"
#include "sm100_ptx.cuh"

namespace ssconv {

namespace {

// ---------------------------------------------------------------------------------------
// Quantisation.  The scale's exponent comes from the exponent field E of the block's largest magnitude: floor(log2) = E - 127, so
// the code (bias 127) is E - 2, at least 0; E = 255 (an infinity or a NaN) gives 255.  Elements are multiplied by the inverse
// power of two (exact) and rounded once.  A thread block takes the 128 rows x 128 channels of a scale image, four lanes a block of
// 32, LANES a row and 32 rows at a time, and the image is written whole.  LANES is 16, or 12, 8 or 4 where rows have no more: us there /
// back with 16 lanes and so, 401408 x 96 22.6 / 20.4 and 17.1 / 17.1 (5.7 TB/s), 402714 x 64 with 8 of blocks of 512 threads 14.3 / 12.3
// and 12.3 / 11.0, 402714 x 8 19 / - and 6.2 / 5.7.  2.53 bytes per element; 25088 x 1536 in 18.5 us (5.2 TB/s).
// ---------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// The larger of two pairs of magnitudes, a NaN where there is one.
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// (Scaled as bf16 pairs: a product by a power of two is exact, but for those so small that they round to zero anyway.)
__device__ __forceinline__ uint32_t e2m1_x8(const uint4& v, uint32_t scale_x2) {
  const uint32_t w[4] = {mul_bf16x2(v.x, scale_x2), mul_bf16x2(v.y, scale_x2), mul_bf16x2(v.z, scale_x2), mul_bf16x2(v.w, scale_x2)};
  uint32_t out;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(out)
      : "f"(bf16_lo(w[0])), "f"(bf16_hi(w[0])), "f"(bf16_lo(w[1])), "f"(bf16_hi(w[1])), "f"(bf16_lo(w[2])), "f"(bf16_hi(w[2])), "f"(bf16_lo(w[3])),
        "f"(bf16_hi(w[3])));
  return out;
}

template <int LANES>
__global__ void __launch_bounds__(32 * LANES, 48 / LANES) quantize_mxfp4_kernel(const uint4* x, uint32_t* codes, uint4* scales, uint32_t rows, uint32_t chunks,
                                                             uint32_t blocks, uint32_t C8) {
  __shared__ __align__(16) uint32_t image[128];
  grid_launch_dependents();
  const uint32_t tile = blockIdx.x / chunks, chunk = blockIdx.x - tile * chunks;
  constexpr uint32_t kRows = 32, kTurns = 128 / kRows;  // rows at a time
  const uint32_t lane = threadIdx.x % LANES, r0 = threadIdx.x / LANES;
  const uint32_t piece = chunk * 16u + lane;  // of 8 channels
  const uint32_t there = rows - tile * 128u;  // rows from the tile's first on
  grid_dependency_wait();
  uint4 v[kTurns];
#pragma unroll
  for (int u = 0; u < (int)kTurns; ++u) {
    const uint32_t r = r0 + kRows * u;
    v[u] = make_uint4(0u, 0u, 0u, 0u);
    if (r < there && piece < C8) v[u] = x[(uint64_t)(tile * 128u + r) * C8 + piece];
  }
#pragma unroll
  for (int u = 0; u < (int)kTurns; ++u) {
    const uint32_t r = r0 + kRows * u;
    constexpr uint32_t kMagnitudes = 0x7FFF7FFFu;
    uint32_t m = max_bf16x2(max_bf16x2(v[u].x & kMagnitudes, v[u].y & kMagnitudes), max_bf16x2(v[u].z & kMagnitudes, v[u].w & kMagnitudes));
    m = max_bf16x2(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    m = max_bf16x2(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    const uint32_t e = max(m & 0xFFFFu, m >> 16) >> 7;
    const uint32_t code = e == 255u ? 255u : e < 2u ? 0u : e - 2u;
    const uint32_t inverse = ((254u - min(code, 252u)) << 7) * 0x10001u;
    if (r < there && (piece >> 2) < blocks) codes[(uint64_t)(tile * 128u + r) * (4u * blocks) + piece] = e2m1_x8(v[u], inverse);
    if (LANES == 12) {  // (a row's lanes may be in two warps)
      uint8_t* bytes = reinterpret_cast<uint8_t*>(image + (r & 31u) * 4u + (r >> 5));
      if ((lane & 3u) == 0) bytes[lane >> 2] = (uint8_t)code;
      if (lane == 1) bytes[3] = 0;
    } else {
      uint32_t word = code << (8u * (lane >> 2));
      if (LANES > 4) word |= __shfl_xor_sync(0xFFFFFFFFu, word, 4);
      if (LANES > 8) word |= __shfl_xor_sync(0xFFFFFFFFu, word, 8);
      if (lane == 0) image[(r & 31u) * 4u + (r >> 5)] = word;
    }
  }
  __syncthreads();
  if (threadIdx.x < 32) scales[(uint64_t)blockIdx.x * 32u + threadIdx.x] = reinterpret_cast<const uint4*>(image)[threadIdx.x];
}

// The bf16 values of four codes (the low 16 bits): their high and low bytes looked up by the three bits below the sign, the
// bytes put together, the signs above.  0, 1/2, 1, 3/2, 2, 3, 4, 6 are 0, 3F00, 3F80, 3FC0, 4000, 4040, 4080, 40C0.
__device__ __forceinline__ void e2m1_values_x4(uint32_t codes, uint32_t& low, uint32_t& high) {
  const uint32_t select = codes & 0x7777u;
  const uint32_t hi = __byte_perm(0x3F3F3F00u, 0x40404040u, select), lo = __byte_perm(0xC0800000u, 0xC0804000u, select);
  low = __byte_perm(lo, hi, 0x5140) | ((codes << 12) & 0x8000u) | ((codes << 24) & 0x80000000u);
  high = __byte_perm(lo, hi, 0x7362) | ((codes << 4) & 0x8000u) | ((codes << 16) & 0x80000000u);
}
template <int LANES>
__global__ void __launch_bounds__(32 * LANES) dequantize_mxfp4_kernel(const uint32_t* codes, const uint8_t* scales, uint4* x, uint32_t rows, uint32_t chunks,
                                                               uint32_t blocks, uint32_t C8) {
  grid_launch_dependents();
  const uint32_t tile = blockIdx.x / chunks, chunk = blockIdx.x - tile * chunks;
  constexpr uint32_t kRows = 32, kTurns = 128 / kRows;
  const uint32_t lane = threadIdx.x % LANES, r0 = threadIdx.x / LANES;
  const uint32_t piece = chunk * 16u + lane;
  const uint32_t there = rows - tile * 128u;
  grid_dependency_wait();
  if (piece >= C8) return;
  uint32_t c[kTurns], s[kTurns];
#pragma unroll
  for (int u = 0; u < (int)kTurns; ++u) {
    const uint32_t r = r0 + kRows * u;
    c[u] = s[u] = 0u;
    if (r < there) {
      c[u] = codes[(uint64_t)(tile * 128u + r) * (4u * blocks) + piece];
      s[u] = scales[(uint64_t)blockIdx.x * 512u + (r & 31u) * 16u + (r >> 5) * 4u + (lane >> 2)];
    }
  }
#pragma unroll
  for (int u = 0; u < (int)kTurns; ++u) {
    const uint32_t r = r0 + kRows * u;
    // the scale as bf16: 2^-127 is below the normal numbers, 255 is a NaN
    const uint32_t scale = (s[u] == 255u ? 0x7FC0u : s[u] == 0u ? 0x0040u : s[u] << 7) * 0x10001u;
    uint4 o;
    e2m1_values_x4(c[u] & 0xFFFFu, o.x, o.y);
    e2m1_values_x4(c[u] >> 16, o.z, o.w);
    if (r < there)
      x[(uint64_t)(tile * 128u + r) * C8 + piece] =
          make_uint4(mul_bf16x2(o.x, scale), mul_bf16x2(o.y, scale), mul_bf16x2(o.z, scale), mul_bf16x2(o.w, scale));
  }
}

// ---------------------------------------------------------------------------------------
// Product.  y[p, co] = act(bias[co] + sum_ci x_q[p, ci] w_q[co, ci]): tiles of 128 pixels (the accumulator's rows) x BN channels,
// K in stages of 256 channels (128 bytes of codes per row, the 128-byte swizzle; two scale images per 128 rows).  One thread block
// per SM walks over tiles, channels first, so that the blocks at work at a time share few rows of x; two accumulators, so that a
// tile's epilogue runs beside the next one's MMAs.  The epilogue's pieces (64 channels) go to kMxSets sets of four warps in turn;
// each warp stages and stores its 32 rows by itself.  Three more warps are the producer, the MMA issuer and the one that moves
// the scales into TMEM.
// ---------------------------------------------------------------------------------------
constexpr long long kMxWaitLimit = 4000000000LL;  // cycles: about 2 s
constexpr int kMxStoreBytes = 32 * 128;           // staged outputs of a warp: 32 pixels x 64 channels of bf16
constexpr int kMxSets = 3;
constexpr int kMxMostSmem = 227 * 1024;

template <int BN, bool PAIR>
struct MxTile {
  static constexpr int kProducer = 4 * kMxSets, kIssuer = kProducer + 1, kScaler = kProducer + 2, kThreads = 32 * (kScaler + 1);
  static constexpr int kStagedBytes = 4 * kMxSets * kMxStoreBytes;
  static constexpr int kScaleTiles = BN > 128 ? 2 : 1;  // images along the tile's channels
  static constexpr int kBytesA = 128 * 128, kBytesB = BN * 128 / (PAIR ? 2 : 1), kBytesScales = 1024 * (1 + kScaleTiles);
  static constexpr int kBytes = kBytesA + kBytesB + kBytesScales;
  static constexpr int kRoom = kMxMostSmem - 1024 - kStagedBytes - 256;
  static constexpr int kStages = kRoom / kBytes < 6 ? kRoom / kBytes : 6;
  static constexpr int kScaleColumns = 8 * (1 + kScaleTiles);  // of TMEM, per stage: two images of x, two (four) of w
  static constexpr int kTmem = 2 * BN + kStages * kScaleColumns <= 256 ? 256 : 512;
  static constexpr int kSmem = 1024 + kStages * kBytes + kStagedBytes + 256;
  static_assert(2 * BN + kStages * kScaleColumns <= 512 && kStages >= 3, "");
};

struct MxParams {
  const uint8_t *x_scales, *w_scales;  // (pairs read them through tensor maps)
  const float* bias;
  int32_t* dev_status;
  int m_tiles, n_tiles, w_tiles;  // w_tiles: scale images along C_out
  int rows, C_out, chunks, steps; // steps of 64 channels
  int x_rows, w_rows;             // of a tile's boxes: no more than there are (what lies past them is not stored)
  int tail_bytes;                 // of codes per row in the last stage's tiles: 32, 64 or 128
  uint32_t tail_desc;             // high half of their descriptors
};

// High halves of descriptors of K-major tiles with rows of 64 and of 32 bytes in the swizzles of those widths.
constexpr uint32_t kDescHiSw64 = (512u >> 4) | (1u << 14) | (4u << 29);
constexpr uint32_t kDescHiSw32 = (256u >> 4) | (1u << 14) | (6u << 29);

// The roles' warps go on in lock step, and one lane issues.  It is elected once: elected for each instruction, the same instructions
// kept the tensor cores and copies waiting (us before and after, 8192 x 4096 -> 4096 70.7 / 63.7, 16 x 4096 -> 4096 8.9 / 7.6, 25088 x
// 1536 -> 384 14.3 / 13.3).  The commits elect by themselves: with all 32 lanes asking it is always the same lane.
__device__ __forceinline__ uint32_t elected() {
  uint32_t lead;
  asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(lead));
  return lead;
}
// 32x128b.warpx4: 512 bytes (32 rows of 16, unswizzled) into 4 TMEM columns, the same 32 lanes in each of the four quarters.
__device__ __forceinline__ void tc_cp_32x128b_x4(uint32_t dst_tmem, uint32_t src_lo, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t.reg .b64 ds;\n\t"
      "setp.ne.b32 e, %3, 0;\n\t"
      "mov.b64 ds, {%1, %2};\n\t"
      "@e tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], ds;\n\t}"
      ::"r"(dst_tmem), "r"(src_lo), "r"(kDescHiNoSwizzle128), "r"(lead)
      : "memory");
}
// D[128 x N] (+)= A[128 x 64] B[N x 64]^T, e2m1 operands with one e8m0 scale per 32 elements of a row, taken from TMEM.
__device__ __forceinline__ void tc_mma_mxf4(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t desc_hi, uint32_t idesc, uint32_t sfa,
                                              uint32_t sfb, uint32_t accumulate, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 e, %8, 0;\n\t"
      "mov.b64 da, {%1, %7};\n\t"
      "mov.b64 db, {%2, %7};\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], da, db, %3, [%4], [%5], p;\n\t}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(desc_hi), "r"(lead)
      : "memory");
}
// The same two for a pair: both blocks' scales into their own TMEM; 256 rows of A, the blocks' halves of B one after the other.
__device__ __forceinline__ void tc2_cp_32x128b_x4(uint32_t dst_tmem, uint32_t src_lo, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t.reg .b64 ds;\n\t"
      "setp.ne.b32 e, %3, 0;\n\t"
      "mov.b64 ds, {%1, %2};\n\t"
      "@e tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], ds;\n\t}"
      ::"r"(dst_tmem), "r"(src_lo), "r"(kDescHiNoSwizzle128), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void tc2_mma_mxf4(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t desc_hi, uint32_t idesc, uint32_t sfa,
                                               uint32_t sfb, uint32_t accumulate, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 e, %8, 0;\n\t"
      "mov.b64 da, {%1, %7};\n\t"
      "mov.b64 db, {%2, %7};\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], da, db, %3, [%4], [%5], p;\n\t}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(desc_hi), "r"(lead)
      : "memory");
}
// Instruction descriptor of kind::mxf4: bits 4-5 and 29-30 which of a row's scales in its TMEM word (0 or 2: the first two or the
// last two) for B and A, bits 7-9 and 10-12 the formats (1 = e2m1), bits 17-22 N >> 3, bit 23 the scales' format (1 = e8m0),
// bits 27-28 M >> 7.
__host__ __device__ constexpr uint32_t make_idesc_mxf4(uint32_t M, uint32_t N, uint32_t which) {
  return (which << 4) | (1u << 7) | (1u << 10) | ((N >> 3) << 17) | (1u << 23) | ((M >> 7) << 27) | (which << 29);
}
// 16 columns of the warp's 32 lanes: register i of lane t holds column i of row t, after the wait below.
__device__ __forceinline__ void tc_ld_32x32b_x16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
// (The registers go through the wait, so that nothing that uses them is moved before it.)
__device__ __forceinline__ void tc_wait_ld_x16(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}

// A load whose completion is signalled on an mbarrier of either block of a pair, by one thread.
__device__ __forceinline__ void tma2_load_2d_a(uint32_t dst, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y)
      : "memory");
}

template <int BN, bool PAIR, int ACT>
__global__ void __launch_bounds__(MxTile<BN, PAIR>::kThreads, 1) mxfp4_kernel(const __grid_constant__ CUtensorMap tm_x,
                                                             const __grid_constant__ CUtensorMap tm_w,
                                                             const __grid_constant__ CUtensorMap tm_x_tail,
                                                             const __grid_constant__ CUtensorMap tm_w_tail,
                                                             const __grid_constant__ CUtensorMap tm_x_scales,
                                                             const __grid_constant__ CUtensorMap tm_w_scales,
                                                             const __grid_constant__ CUtensorMap tm_y, const MxParams p) {
  using T = MxTile<BN, PAIR>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* ring_a = smem;
  uint8_t* ring_b = ring_a + T::kStages * T::kBytesA;
  uint8_t* staged = ring_b + T::kStages * T::kBytesB;
  uint8_t* ring_s = staged + T::kStagedBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(ring_s + T::kStages * T::kBytesScales);
  uint64_t *full = bars, *empty = bars + T::kStages, *scaled = bars + 2 * T::kStages, *acc_full = bars + 3 * T::kStages, *acc_empty = acc_full + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5;

  grid_launch_dependents();
  if (threadIdx.x == 0) {
    for (int s = 0; s < T::kStages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
      mbar_init(scaled + s, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(acc_full + i, 1);
      mbar_init(acc_empty + i, 4 * kMxSets * (PAIR ? 2 : 1));
    }
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == T::kProducer) {
    prefetch_tensormap(&tm_x);
    prefetch_tensormap(&tm_w);
    prefetch_tensormap(&tm_x_tail);
    prefetch_tensormap(&tm_w_tail);
    prefetch_tensormap(&tm_y);
  }
  if (warp == T::kIssuer) {
    if (PAIR) {
      tmem_alloc2(tmem_slot, T::kTmem);
      tmem_relinquish2();
    } else {
      tmem_alloc(tmem_slot, T::kTmem);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) {  // (the other block's barriers are there too)
    cluster_arrive();
    cluster_wait();
  }
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // a pair: rank 0 leads; it issues the MMAs, and both blocks' copies arrive on its barriers
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const int first_tile = PAIR ? blockIdx.x >> 1 : blockIdx.x, tile_step = PAIR ? gridDim.x >> 1 : gridDim.x;
  grid_dependency_wait();

  const int tiles = p.m_tiles * p.n_tiles;
  const int stages = (p.steps + 3) >> 2;
  if (warp == T::kProducer) {
    // ---------------------------------------------------------------- producer
    const uint32_t a0 = smem_u32(ring_a), b0 = smem_u32(ring_b), s0 = smem_u32(ring_s), empty0 = smem_u32(empty);
    const uint32_t full0 = PAIR ? map_to_cta(smem_u32(full), 0) : smem_u32(full);
    uint32_t s = 0, phase = 0;
    bool ok = true;
    const uint32_t lead = elected();
    for (int t = first_tile; t < tiles && ok; t += tile_step) {
      const int mt = t / p.n_tiles, n = t - mt * p.n_tiles, m = PAIR ? 2 * mt + (int)rank : mt;
      const int first = n * BN >> 7;
      const int images = min((n * BN + BN - 1) >> 7, p.w_tiles - 1) - first + 1;
      const uint8_t* xs = p.x_scales + (int64_t)m * p.chunks * kMxImageBytes;
      const uint8_t* ws = p.w_scales + (int64_t)first * p.chunks * kMxImageBytes;
      for (int kb = 0; kb < stages; ++kb) {
        if (!mbar_wait_warp_a(empty0 + 8 * s, phase ^ 1u, abort_flag, kMxWaitLimit)) {
          ok = false;
          break;
        }
        const uint32_t bar = full0 + 8 * s, sc = s0 + s * T::kBytesScales;
        const bool tail = kb == stages - 1;
        const uint32_t codes = (tail ? p.tail_bytes : 128) * (p.x_rows + p.w_rows);
        if (lead) {
          if constexpr (PAIR) {
            // (two images per copy, whether there is a second one or not: what it brings instead is not used)
            if (rank == 0) mbar_expect_tx_a(smem_u32(full) + 8 * s, 2 * (codes + T::kBytesScales));
            tma2_load_2d_a(a0 + s * T::kBytesA, tail ? &tm_x_tail : &tm_x, bar, kb * 128, m * 128);
            tma2_load_2d_a(b0 + s * T::kBytesB, tail ? &tm_w_tail : &tm_w, bar, kb * 128, n * BN + (int)rank * (BN / 2));
            tma2_load_2d_a(sc, &tm_x_scales, bar, 0, m * p.chunks + 2 * kb);
#pragma unroll
            for (int i = 0; i < T::kScaleTiles; ++i) tma2_load_2d_a(sc + 1024 * (1 + i), &tm_w_scales, bar, 0, (first + i) * p.chunks + 2 * kb);
          } else {
            const uint32_t part = min(2, p.chunks - 2 * kb) * kMxImageBytes;
            mbar_expect_tx_a(bar, codes + part * (1 + images));
            tma_load_2d_a(a0 + s * T::kBytesA, tail ? &tm_x_tail : &tm_x, bar, kb * 128, m * 128);
            tma_load_2d_a(b0 + s * T::kBytesB, tail ? &tm_w_tail : &tm_w, bar, kb * 128, n * BN);
            bulk_load_a(sc, xs + kb * 2 * kMxImageBytes, part, bar);
#pragma unroll
            for (int i = 0; i < T::kScaleTiles; ++i)
              if (i < images) bulk_load_a(sc + 1024 * (1 + i), ws + ((int64_t)i * p.chunks + 2 * kb) * kMxImageBytes, part, bar);
          }
        }
        if (++s == T::kStages) {
          s = 0;
          phase ^= 1u;
        }
      }
    }
  } else if (warp == T::kIssuer) {
   if (rank == 0) {
    // ---------------------------------------------------------------- MMA issuer
    const uint32_t a0 = desc_lo(smem_u32(ring_a)), b0 = desc_lo(smem_u32(ring_b));
    const uint32_t scaled0 = smem_u32(scaled), empty0 = smem_u32(empty), acc_full0 = smem_u32(acc_full), acc_empty0 = smem_u32(acc_empty);
    uint32_t s = 0, phase = 0, buf = 0, acc_phase = 0, ready = 0;
    const uint32_t lead = elected();
    bool ok = true;
    for (int t = first_tile; t < tiles && ok; t += tile_step) {
      // tiles that start inside an image take its later columns
      const uint32_t shift = ((uint32_t)(t % p.n_tiles) * BN & 127u) >> 5;
      if (!mbar_wait_warp_a(acc_empty0 + 8 * buf, acc_phase ^ 1u, abort_flag, kMxWaitLimit)) break;
      tc_fence_after();
      const uint32_t d = tmem + buf * BN;
      for (int kb = 0; kb < stages; ++kb) {
        if (!__all_sync(0xFFFFFFFFu, ready) && !mbar_wait_warp_a(scaled0 + 8 * s, phase, abort_flag, kMxWaitLimit)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t next = s + 1 == T::kStages ? 0 : s + 1, next_phase = next == 0 ? phase ^ 1u : phase;
        ready = mbar_test_a(scaled0 + 8 * next, next_phase);  // (its latency passes beside the MMAs)
        const uint32_t sfa = tmem + 2 * BN + s * T::kScaleColumns, sfb = sfa + 8 + shift;
        const int steps = min(4, p.steps - 4 * kb);
        const uint32_t desc_hi = kb == stages - 1 ? p.tail_desc : kDescHiSw128;
        const uint32_t a_lo = a0 + s * (T::kBytesA >> 4), b_lo = b0 + s * (T::kBytesB >> 4);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k < steps) {
            const uint32_t idesc = make_idesc_mxf4(PAIR ? 256 : 128, BN, 2 * (k & 1));
            const uint32_t sa = sfa + 4 * (k >> 1), sb = sfb + 4 * T::kScaleTiles * (k >> 1);
            if (PAIR)
              tc2_mma_mxf4(d, a_lo + 2 * k, b_lo + 2 * k, desc_hi, idesc, sa, sb, (kb | k) != 0, lead);
            else
              tc_mma_mxf4(d, a_lo + 2 * k, b_lo + 2 * k, desc_hi, idesc, sa, sb, (kb | k) != 0, lead);
          }
        if (PAIR)
          tc2_commit_both_w(empty0 + 8 * s);
        else
          tc_commit_w(empty0 + 8 * s);
        s = next;
        phase = next_phase;
      }
      if (!ok) break;
      if (PAIR)
        tc2_commit_both_w(acc_full0 + 8 * buf);
      else
        tc_commit_w(acc_full0 + 8 * buf);
      buf ^= 1u;
      if (buf == 0) acc_phase ^= 1u;
    }
   }
  } else if (warp == T::kScaler) {
   if (rank == 0) {
    // ---------------------------------------------------------------- scales into TMEM
    // (by a warp of its own: waits and tcgen05 instructions cost an issuer time, and there are six of these beside four MMAs)
    const uint32_t s0 = desc_lo(smem_u32(ring_s)), full0 = smem_u32(full), scaled0 = smem_u32(scaled);
    uint32_t s = 0, phase = 0, ready = 0;
    const uint32_t lead = elected();
    bool ok = true;
    for (int t = first_tile; t < tiles && ok; t += tile_step) {
      for (int kb = 0; kb < stages; ++kb) {
        if (!__all_sync(0xFFFFFFFFu, ready) && !mbar_wait_warp_a(full0 + 8 * s, phase, abort_flag, kMxWaitLimit)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t next = s + 1 == T::kStages ? 0 : s + 1, next_phase = next == 0 ? phase ^ 1u : phase;
        ready = mbar_test_a(full0 + 8 * next, next_phase);
        const uint32_t sfa = tmem + 2 * BN + s * T::kScaleColumns, sfb = sfa + 8, src = s0 + s * (T::kBytesScales >> 4);
        const bool second = p.steps - 4 * kb > 2;
        const auto copy = [lead](uint32_t to, uint32_t from) {
          if (PAIR)
            tc2_cp_32x128b_x4(to, from, lead);
          else
            tc_cp_32x128b_x4(to, from, lead);
        };
        copy(sfa, src);
#pragma unroll
        for (int i = 0; i < T::kScaleTiles; ++i) copy(sfb + 4 * i, src + 64 * (1 + i));
        if (second) {
          copy(sfa + 4, src + 32);
#pragma unroll
          for (int i = 0; i < T::kScaleTiles; ++i) copy(sfb + 4 * T::kScaleTiles + 4 * i, src + 64 * (1 + i) + 32);
        }
        if (PAIR)
          tc2_commit_w(map_to_cta(scaled0 + 8 * s, 0));
        else
          tc_commit_w(scaled0 + 8 * s);
        s = next;
        phase = next_phase;
      }
    }
   }
  } else {
    // ---------------------------------------------------------------- epilogue
    const int set = warp >> 2, row = 32 * (warp & 3), lane = threadIdx.x & 31;
    uint8_t* out = staged + warp * kMxStoreBytes;
    uint32_t buf = 0, acc_phase = 0;
    static_assert(BN / 64 <= kMxSets, "");  // a set has one piece of a tile at most
    int turn = 0;  // the set that takes the next piece
    for (int t = first_tile; t < tiles; t += tile_step) {
      const int mt = t / p.n_tiles, n = t - mt * p.n_tiles, m = PAIR ? 2 * mt + (int)rank : mt;
      const int pieces = min(BN / 64, (p.C_out - n * BN + 63) >> 6), g = set - turn + (set < turn ? kMxSets : 0);
      turn += pieces;
      if (turn >= kMxSets) turn -= kMxSets;
      const int c0 = n * BN + 64 * g;
      // The piece's 64 biases, while its accumulator is on its way.  (Plain loads, see launch.cuh, which the instructions below would
      // keep in their order: 16 at a time where they are used, us instead of so: 1 x 2048 -> 1000 6.2 / 5.5, 16 x 4096 -> 4096 8.2 / 7.5,
      // 25088 x 384 -> 1536 28.7 / 26.7.)
      ulonglong2 bias[16];
#pragma unroll
      for (int q = 0; q < 16; ++q) bias[q] = make_ulonglong2(0ull, 0ull);
      if (p.bias != nullptr && g < pieces) {
#pragma unroll
        for (int q = 0; q < 16; ++q)  // (columns past the last channel are not stored)
          bias[q] = *reinterpret_cast<const ulonglong2*>(p.bias + min(c0 + 4 * q, p.C_out - 4));
      }
      if (!mbar_wait_warp(acc_full + buf, acc_phase, abort_flag, kMxWaitLimit)) break;
      tc_fence_after();
      const uint32_t acc = tmem + buf * BN + ((uint32_t)row << 16);
      if (g < pieces) {
        // a row's 64 outputs per lane; the next 16 columns are on their way
        uint32_t r[2][16];
        tc_ld_32x32b_x16(acc + 64 * g, r[0]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          tc_wait_ld_x16(r[i & 1]);
          if (i < 3) tc_ld_32x32b_x16(acc + 64 * g + 16 * (i + 1), r[(i + 1) & 1]);
          uint32_t w[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float lo, hi;
            unsigned long long v;
            asm("add.rn.f32x2 %0, %1, %2;"
                : "=l"(v)
                : "l"(f32x2(__uint_as_float(r[i & 1][2 * j]), __uint_as_float(r[i & 1][2 * j + 1]))),
                  "l"(j & 1 ? bias[4 * i + (j >> 1)].y : bias[4 * i + (j >> 1)].x));
            split2(v, lo, hi);
            w[j] = activate_pack<ACT>(lo, hi);
          }
          if (i == 0) {  // (not before: it took 401408 x 96 -> 384 from 97.3 us to 93.8, 12544 x 2048 -> 512 from 12.3 to 11.7)
            if (lane == 0) bulk_wait_group_read0();  // the warp's last piece has left its buffer
            __syncwarp();
          }
          *reinterpret_cast<uint4*>(out + lane * 128 + (((2 * i) ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
          *reinterpret_cast<uint4*>(out + lane * 128 + (((2 * i + 1) ^ (lane & 7)) << 4)) = make_uint4(w[4], w[5], w[6], w[7]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (!PAIR || m * 128 + row < p.rows) tma_store_2d(&tm_y, out, c0, m * 128 + row);
          bulk_commit_group();
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR)
          mbar_arrive_cluster(map_to_cta(smem_u32(acc_empty + buf), 0));
        else
          mbar_arrive(acc_empty + buf);
      }
      buf ^= 1u;
      if (buf == 0) acc_phase ^= 1u;
    }
    if (lane == 0) bulk_wait_group_read0();
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag != 0) {
    // give copies and MMAs still in flight time to land before shared memory and TMEM go away
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) __nanosleep(1000);
    if (threadIdx.x == 0 && p.dev_status != nullptr) atomicExch(p.dev_status, (int)SSCONV_ERR_TIMEOUT);
    __syncthreads();
  }
  if (PAIR) {  // (neither block leaves while the other may still arrive on its barriers or read its memory)
    cluster_arrive();
    cluster_wait();
  }
  if (warp == T::kIssuer) {
    tc_fence_after();
    if (PAIR)
      tmem_dealloc2(tmem, T::kTmem);
    else
      tmem_dealloc(tmem, T::kTmem);
  }
}

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encoder() {
  static std::atomic<EncodeFn> known{nullptr};  // (every thread finds the same function)
  EncodeFn f = known.load(std::memory_order_relaxed);
  if (f == nullptr) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess || !p)
      return nullptr;
    f = reinterpret_cast<EncodeFn>(p);
    known.store(f, std::memory_order_relaxed);
  }
  return f;
}
// A matrix of `rows` rows of `inner` elements, copied in boxes of `width` (32, 64 or 128) bytes x box_rows in the swizzle of that
// width.  (Lines of 128 bytes in L2: promoted to 256 bytes, rows of 48 bytes were fetched several times over, 401408 x 96 -> 384
// 112 us instead of 90; and boxes that reach past the rows' ends are slow: 128-byte ones on those rows 67.6 us for 192 channels,
// on rows of 128 bytes 40.7.)
bool encode_matrix(EncodeFn f, CUtensorMap* map, CUtensorMapDataType type, int element, const void* base, int64_t inner, int64_t rows, int width,
                   int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)inner * element};
  const cuuint32_t box[2] = {(cuuint32_t)(width / element), (cuuint32_t)box_rows}, ones[2] = {1, 1};
  const CUtensorMapSwizzle swizzle = width == 128  ? CU_TENSOR_MAP_SWIZZLE_128B
                                     : width == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                                                   : CU_TENSOR_MAP_SWIZZLE_32B;
  return f(map, type, 2, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
           CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Scale images, two per copy, unswizzled.
bool encode_images(EncodeFn f, CUtensorMap* map, const void* base, int64_t images) {
  const cuuint64_t dims[2] = {kMxImageBytes / 4, (cuuint64_t)images}, strides[1] = {kMxImageBytes};
  const cuuint32_t box[2] = {kMxImageBytes / 4, 2}, ones[2] = {1, 1};
  return f(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
           CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

using MxKernel = void (*)(CUtensorMap, CUtensorMap, CUtensorMap, CUtensorMap, CUtensorMap, CUtensorMap, CUtensorMap, MxParams);
template <int BN, bool PAIR>
MxKernel mx_kernel(int act, int* smem) {
  *smem = MxTile<BN, PAIR>::kSmem;
  return act == kActGelu ? mxfp4_kernel<BN, PAIR, kActGelu> : act == kActRelu ? mxfp4_kernel<BN, PAIR, kActRelu> : mxfp4_kernel<BN, PAIR, kActNone>;
}
constexpr int kMxThreads = MxTile<64, false>::kThreads;

cudaLaunchConfig_t mx_config(unsigned blocks, int smem, bool pair, cudaStream_t st, cudaLaunchAttribute (&attrs)[2]) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = blocks;
  cfg.blockDim = kMxThreads;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = 2;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = pair ? 2 : 1;
  return cfg;
}

// Checks a device and allows the kernels their shared memory on it, once; the pairs of blocks that it holds at a time.
int32_t mx_device(int dev, int* pairs) {
  static std::atomic<int> known[64];
  *pairs = known[dev].load(std::memory_order_acquire);
  if (*pairs > 0) return SSCONV_OK;
  int major = 0, smem = 0;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return SSCONV_ERR_CUDA;
  if (major != 10) return SSCONV_ERR_ARCH;
  for (const int act : {kActNone, kActRelu, kActGelu})
    for (const MxKernel kernel : {mx_kernel<64, false>(act, &smem), mx_kernel<128, false>(act, &smem), mx_kernel<192, false>(act, &smem),
                                  mx_kernel<192, true>(act, &smem)})
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMxMostSmem) != cudaSuccess) return SSCONV_ERR_CUDA;
  cudaLaunchAttribute attrs[2];
  const MxKernel kernel = mx_kernel<192, true>(kActNone, &smem);
  const cudaLaunchConfig_t cfg = mx_config(2u * device_sms(), smem, true, nullptr, attrs);
  if (cudaOccupancyMaxActiveClusters(pairs, kernel, &cfg) != cudaSuccess || *pairs <= 0) return SSCONV_ERR_CUDA;
  known[dev].store(*pairs, std::memory_order_release);
  return SSCONV_OK;
}

// The form that a product of this extent takes on a device with so many SMs, which holds so many pairs of blocks at a time.
struct MxChoice {
  int columns;
  bool pair;
};
MxChoice mx_choose(const MxGeometry& gx, int C_out, int act, int sms, int pairs) {
  // The width, by cycles (fitted to 401408 x 96 -> 384 and 8192 x 4096 -> 4096): a tile takes the longer of filling shared memory and
  // of its epilogue, and the first of the one and the last of the other are not hidden.  Shared memory fills at 50 bytes per cycle and
  // SM, 12 TB/s out of L2 in all, which is most of what long K takes (with three of four MMAs left out 8192 x 4096 -> 4096 took 62.5 us
  // at 192 columns and 58.1 on pairs, with all of them 69.8 and 63.6).  Pairs halve the weights' share of it, at a lower rate.  us at 192 /
  // 128 / 64 columns / 192 on pairs: 401408 x 96 -> 384 76.4 / 78.8 / 90.3 / 101, with GELU 90.7 / 99.6 / 112 / 123, 8192 x 4096 -> 4096 69.8 /
  // 76.0 / 125 / 63.6, 25088 x 1536 -> 384 13.6 / 13.0 / 18.7 / 14.3, 25088 x 384 -> 1536 with GELU 27.2 / 28.0 / 36.5 / 36.8, 1024 x 4096 ->
  // 4096 16.6 / 14.4 / 20.5 / 15.8, 512 x 1024 -> 1024 6.1 / 5.5 / 4.8 / 6.9.  (The rule takes the fastest but for 25088 x 1536 -> 384, whose 192
  // columns come out within the margin of 128 and are 0.6 us slower.)
  const int mx_stages = (gx.blocks + 7) / 8;
  MxChoice best = {0, false};
  double least = 0.0;
  const auto consider = [&](int w, bool two) {
    const int64_t rows_of_tiles = two ? (gx.row_tiles + 1) / 2 : gx.row_tiles, at_once = two ? pairs : sms;
    const int64_t turns = (rows_of_tiles * ((C_out + w - 1) / w) + at_once - 1) / at_once;
    const double fill = mx_stages * (two ? 790.0 : (128 + w + 8) * 128 / 50.0), epilogue = 800.0 + w * (act == kActGelu ? 19.0 : 14.0);
    const double cost = turns * (fill > epilogue ? fill : epilogue) + (fill > epilogue ? epilogue : fill);
    if (best.columns == 0 || cost < (two ? 0.95 : 0.9) * least) {
      best = {w, two};
      least = cost;
    }
  };
  consider(192, false);
  consider(128, false);
  consider(64, false);
  consider(192, true);
  return best;
}

}  // namespace

// Lanes of a row.
static int mx_lanes(const MxGeometry& g) { return g.blocks <= 4 ? 4 * g.blocks : 16; }

cudaError_t launch_quantize_mxfp4(const void* x, int64_t rows, int C, void* codes, void* scales, cudaStream_t st) {
  const MxGeometry g = mx_geometry(rows, C);
  count_launch();
  const int lanes = mx_lanes(g);
  const auto kernel = lanes == 4 ? quantize_mxfp4_kernel<4> : lanes == 8 ? quantize_mxfp4_kernel<8> : lanes == 12 ? quantize_mxfp4_kernel<12> : quantize_mxfp4_kernel<16>;
  return launch_dependent(kernel, (unsigned)(g.row_tiles * g.chunks), 32 * lanes, st, (const uint4*)x, (uint32_t*)codes, (uint4*)scales,
                          (uint32_t)rows, (uint32_t)g.chunks, (uint32_t)g.blocks, (uint32_t)(C / 8));
}

cudaError_t launch_dequantize_mxfp4(const void* codes, const void* scales, int64_t rows, int C, void* x, cudaStream_t st) {
  const MxGeometry g = mx_geometry(rows, C);
  count_launch();
  const int lanes = mx_lanes(g);
  const auto kernel = lanes == 4 ? dequantize_mxfp4_kernel<4> : lanes == 8 ? dequantize_mxfp4_kernel<8> : lanes == 12 ? dequantize_mxfp4_kernel<12> : dequantize_mxfp4_kernel<16>;
  return launch_dependent(kernel, (unsigned)(g.row_tiles * g.chunks), 32 * lanes, st, (const uint32_t*)codes, (const uint8_t*)scales,
                          (uint4*)x, (uint32_t)rows, (uint32_t)g.chunks, (uint32_t)g.blocks, (uint32_t)(C / 8));
}

int32_t plan_mxfp4(const ssconv_desc_t& d, int sms, int pairs, int32_t* columns, int32_t* pair, int32_t* ctas) {
  const MxGeometry gx = mx_geometry((int64_t)d.N * d.H * d.W, d.C_in);
  if (sms == 0) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SSCONV_ERR_CUDA;
    const int32_t known = mx_device(dev, &pairs);
    if (known != SSCONV_OK) return known;
    sms = device_sms();
  }
  const MxChoice c = mx_choose(gx, d.C_out, activation_of(d.flags), sms, pairs);
  const int64_t tiles = (c.pair ? (gx.row_tiles + 1) / 2 : gx.row_tiles) * ((d.C_out + c.columns - 1) / c.columns), at_once = c.pair ? pairs : sms;
  if (columns) *columns = c.columns;
  if (pair) *pair = c.pair;
  if (ctas) *ctas = (int32_t)((tiles < at_once ? tiles : at_once) * (c.pair ? 2 : 1));
  return SSCONV_OK;
}

int32_t launch_forward_mxfp4(const ssconv_desc_t& d, const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales,
                             const float* bias, void* y, int32_t* dev_status, cudaStream_t st) {
  const int64_t rows = (int64_t)d.N * d.H * d.W;
  const MxGeometry gx = mx_geometry(rows, d.C_in), gw = mx_geometry(d.C_out, d.C_in);
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SSCONV_ERR_CUDA;
  int pairs = 0;
  const int32_t known = mx_device(dev, &pairs);
  if (known != SSCONV_OK) return known;
  const int sms = device_sms();
  const int act = activation_of(d.flags);
  const MxChoice choice = mx_choose(gx, d.C_out, act, sms, pairs);
  const int bn = choice.columns;
  const bool pair = choice.pair;
  int smem = 0;
  const MxKernel kernel = pair        ? mx_kernel<192, true>(act, &smem)
                          : bn == 192 ? mx_kernel<192, false>(act, &smem)
                          : bn == 128 ? mx_kernel<128, false>(act, &smem)
                                      : mx_kernel<64, false>(act, &smem);
  const int64_t row_bytes = (int64_t)gx.blocks * 16;
  MxParams p = {};
  p.x_scales = static_cast<const uint8_t*>(x_scales);
  p.w_scales = static_cast<const uint8_t*>(w_scales);
  p.bias = (d.flags & SSCONV_FLAG_BIAS) ? bias : nullptr;
  p.dev_status = dev_status;
  p.rows = (int)rows;
  p.m_tiles = (int)(pair ? (gx.row_tiles + 1) / 2 : gx.row_tiles);
  p.n_tiles = (d.C_out + bn - 1) / bn;
  p.w_tiles = (int)gw.row_tiles;
  p.C_out = d.C_out;
  p.chunks = gx.chunks;
  p.steps = (gx.blocks + 1) / 2;
  const int tail = (int)((row_bytes - 1) % 128 + 1), stages = (p.steps + 3) / 4;
  p.x_rows = (int)(rows < 128 ? (rows + 7) / 8 * 8 : 128);
  p.w_rows = pair ? bn / 2 : d.C_out < bn ? d.C_out : bn;
  if (pair) p.x_rows = 128;
  p.tail_bytes = tail <= 32 ? 32 : tail <= 64 ? 64 : 128;
  p.tail_desc = tail <= 32 ? kDescHiSw32 : tail <= 64 ? kDescHiSw64 : kDescHiSw128;
  const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles;
  if (tiles > 0x7FFFFFFF - 4096) return SSCONV_ERR_UNSUPPORTED_SHAPE;
  const EncodeFn encode = encoder();
  if (encode == nullptr) return SSCONV_ERR_CUDA;
  CUtensorMap tm_x, tm_w, tm_x_tail, tm_w_tail, tm_x_scales, tm_w_scales, tm_y;
  const auto codes = [&](CUtensorMap* map, const void* base, int64_t n, int width, int box_rows) {
    return encode_matrix(encode, map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, base, row_bytes, n, width, box_rows);
  };
  if (!codes(&tm_x_tail, x_codes, rows, p.tail_bytes, p.x_rows) || !codes(&tm_w_tail, w_codes, d.C_out, p.tail_bytes, p.w_rows) ||
      !encode_matrix(encode, &tm_y, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, y, d.C_out, rows, 128, 32))
    return SSCONV_ERR_CUDA;
  tm_x = tm_x_tail;
  tm_w = tm_w_tail;
  if (stages > 1 && p.tail_bytes != 128 && (!codes(&tm_x, x_codes, rows, 128, p.x_rows) || !codes(&tm_w, w_codes, d.C_out, 128, p.w_rows)))
    return SSCONV_ERR_CUDA;
  tm_x_scales = tm_w_scales = tm_y;  // (not used without pairs)
  if (pair && (!encode_images(encode, &tm_x_scales, x_scales, gx.row_tiles * gx.chunks) || !encode_images(encode, &tm_w_scales, w_scales, gw.row_tiles * gw.chunks)))
    return SSCONV_ERR_CUDA;
  const int64_t at_once = pair ? pairs : sms;
  const unsigned blocks = (unsigned)((tiles < at_once ? tiles : at_once) * (pair ? 2 : 1));
  cudaLaunchAttribute attrs[2];
  const cudaLaunchConfig_t cfg = mx_config(blocks, smem, pair, st, attrs);
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, tm_x, tm_w, tm_x_tail, tm_w_tail, tm_x_scales, tm_w_scales, tm_y, p) == cudaSuccess ? SSCONV_OK
                                                                                                                            : SSCONV_ERR_CUDA;
}

}  // namespace ssconv
