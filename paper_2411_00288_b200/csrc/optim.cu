// The end of a training step over all tensors of a network: the global gradient norm, the gradients scaled down to it, and
// AdamW (Appendix, training details) on every tensor, in one or two launches each however many tensors there are.
//
// A call's tensors travel as a kernel argument: addresses, extents and, per tensor, the number of its first chunk.  A chunk is
// up to `chunk` consecutive elements of one tensor and is one block's work at a time; a block finds its chunk's tensor by bisection in
// the argument (constant memory, the same for all threads of a block).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "launch.cuh"
#include "layout.cuh"
#include "optim.cuh"
#include "sm100_ptx.cuh"
#include "ssconv.h"

namespace ssconv {

constexpr int kOptThreads = 256;

template <int MOST, int ARRAYS>
struct TensorTable {
  int tensors;
  uint32_t chunk;                        // elements
  uint32_t chunks;                       // of all tensors
  uint32_t first[MOST];                  // chunk that tensor i starts with
  int64_t n[MOST];                       // elements; in the top bit: bf16 gradients
  void* p[ARRAYS][MOST];
};
constexpr int64_t kBf16 = INT64_MIN;

// The tensor that chunk c belongs to: the last one that starts at or before it (tensors of no elements are not in the table).
template <class Table>
__device__ __forceinline__ int tensor_of(const Table& t, uint32_t c) {
  int lo = 0, hi = t.tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= c)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// 8 gradients of type f32 or bf16 from an aligned address.
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
  const uint4 a = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = bf16_lo(w[j]);
    v[2 * j + 1] = bf16_hi(w[j]);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  uint4 o;
  o.x = pack_bf16x2<false>(v[0], v[1]);
  o.y = pack_bf16x2<false>(v[2], v[3]);
  o.z = pack_bf16x2<false>(v[4], v[5]);
  o.w = pack_bf16x2<false>(v[6], v[7]);
  *reinterpret_cast<uint4*>(p) = o;
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// What the norm is folded from: the sum of squares, or the largest magnitude as its bits, which order as the magnitudes do and
// hold a NaN above all of them.
struct SumOfSquares {
  double total = 0.0;
  // The squares of a few numbers are added in 32 bits and go into a 64-bit sum; where 32 bits overflow or lose small squares
  // (also for zeros, infinities and NaN, which come out as they should) they are added in 64 bits again.
  template <int K>
  __device__ __forceinline__ void add(const float (&v)[K]) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < K; ++j) s = fmaf(v[j], v[j], s);
    if (s > 1e-25f && s < 1e38f) {
      total += (double)s;
    } else {
      double d = 0.0;
#pragma unroll
      for (int j = 0; j < K; ++j) d = fma((double)v[j], (double)v[j], d);
      total += d;
    }
  }
  __device__ __forceinline__ void add1(float v) { total = fma((double)v, (double)v, total); }
  __device__ __forceinline__ void join(double other) { total += other; }
  __device__ __forceinline__ double value() const { return total; }
  __device__ __forceinline__ double shuffled(int o) const { return __shfl_down_sync(0xFFFFFFFFu, total, o); }
  static __device__ __forceinline__ float norm(double v) { return (float)sqrt(v); }
};
struct LargestMagnitude {
  uint32_t bits = 0;
  template <int K>
  __device__ __forceinline__ void add(const float (&v)[K]) {
#pragma unroll
    for (int j = 0; j < K; ++j) add1(v[j]);
  }
  __device__ __forceinline__ void add1(float v) { bits = max(bits, __float_as_uint(v) & 0x7FFFFFFFu); }
  // (through a double, which holds a 32-bit count exactly: the scratch is the same for both kinds)
  __device__ __forceinline__ void join(double other) { bits = max(bits, (uint32_t)other); }
  __device__ __forceinline__ double value() const { return (double)bits; }
  __device__ __forceinline__ double shuffled(int o) const { return (double)__shfl_down_sync(0xFFFFFFFFu, bits, o); }
  static __device__ __forceinline__ float norm(double v) { return __uint_as_float((uint32_t)v); }
};

// The block's fold, in thread 0: lanes, then warps, always in the same order.
template <class Fold>
__device__ __forceinline__ double block_fold(Fold f) {
  __shared__ double part[32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) f.join(f.shuffled(o));
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  if ((threadIdx.x & 31) == 0) part[warp] = f.value();
  __syncthreads();
  Fold all;
  if (threadIdx.x == 0)
    for (int i = 0; i < warps; ++i) all.join(part[i]);
  return all.value();
}

template <int THREADS, class Fold, class T>
__device__ __forceinline__ void fold_chunk(Fold& f, const T* p, int n, int t) {
  if ((reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
    const int whole = n >> 3;
    // (two pieces of 8 at a time: four 16-byte loads in flight of fp32, two of bf16; four pieces where a warp has a chunk to itself)
    constexpr int kAtOnce = THREADS == 32 ? 4 : 2;
    int i = t;
    for (; i + (kAtOnce - 1) * THREADS < whole; i += kAtOnce * THREADS) {
      float v[kAtOnce][8];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) load8(p + 8 * (i + k * THREADS), v[k]);
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) f.add(v[k]);
    }
    for (; i < whole; i += THREADS) {
      float v[8];
      load8(p + 8 * i, v);
      f.add(v);
    }
    if (t < (n & 7)) f.add1(load1(p + 8 * whole + t));
  } else {
    for (int i = t; i < n; i += THREADS) f.add1(load1(p + i));
  }
}

// Where chunk c of its tensor i starts, and how many elements it has.
template <class Table>
__device__ __forceinline__ int64_t chunk_start(const Table& t, int i, uint32_t c) {
  return (int64_t)(c - t.first[i]) * t.chunk;
}
template <class Table>
__device__ __forceinline__ int chunk_length(const Table& t, int i, int64_t at) {
  const int64_t left = (t.n[i] & ~kBf16) - at;
  return left < (int64_t)t.chunk ? (int)left : (int)t.chunk;
}

// One partial result per block.  4 (2) bytes per gradient, DRAM-bound: 35,168,256 of fp32 in 52 tensors in 24.6 us with the sum of the
// parts (5.7 TB/s, 87 % of a copy's rate; reads alone).  WHOLE: the grid is one cluster of blocks whose warps take
// a chunk each, and whose first block adds up the others' results in their shared memory and writes the norm: one launch.
template <class Fold, bool WHOLE, int MOST>
__global__ void __launch_bounds__(WHOLE ? 1024 : kOptThreads) grad_norm_kernel(const __grid_constant__ TensorTable<MOST, 1> t, double* partial,
                                                                               float* norm) {
  __shared__ double whole;
  grid_launch_dependents();
  grid_dependency_wait();
  const int thread = WHOLE ? threadIdx.x & 31 : threadIdx.x;
  constexpr int kThreads = WHOLE ? 32 : kOptThreads;
  Fold f;
  for (uint32_t c = WHOLE ? (threadIdx.x >> 5) * gridDim.x + blockIdx.x : blockIdx.x; c < t.chunks; c += WHOLE ? 32 * gridDim.x : gridDim.x) {
    const int i = tensor_of(t, c);
    const int64_t at = chunk_start(t, i, c);
    const int len = chunk_length(t, i, at);
    if (t.n[i] < 0)
      fold_chunk<kThreads>(f, static_cast<const __nv_bfloat16*>(t.p[0][i]) + at, len, thread);
    else
      fold_chunk<kThreads>(f, static_cast<const float*>(t.p[0][i]) + at, len, thread);
  }
  const double v = block_fold(f);
  if (!WHOLE) {
    if (threadIdx.x == 0) partial[blockIdx.x] = v;
    return;
  }
  if (threadIdx.x == 0) whole = v;
  cluster_arrive();
  cluster_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    Fold all;
    for (uint32_t r = 0; r < gridDim.x; ++r) {
      double other;
      asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(other) : "r"(map_to_cta(smem_u32(&whole), r)) : "memory");
      all.join(other);
    }
    *norm = Fold::norm(all.value());
  }
  cluster_arrive();  // (no block leaves while its result may still be read)
  cluster_wait();
}

// The partial results together, in an order that depends on their number alone.
template <class Fold>
__global__ void __launch_bounds__(256) grad_norm_finish_kernel(const double* partial, int n, float* norm) {
  grid_launch_dependents();
  grid_dependency_wait();
  Fold f;
  for (int i = threadIdx.x; i < n; i += 256) f.join(partial[i]);
  const double v = block_fold(f);
  if (threadIdx.x == 0) *norm = Fold::norm(v);
}

// min(1, max_norm / (norm + 1e-6)); NaN where the norm is.
__device__ __forceinline__ float clip_factor(const float* norm, float max_norm) {
  const float q = max_norm / (*norm + 1e-6f);
  return q >= 1.0f ? 1.0f : q;
}

template <class T>
__device__ __forceinline__ void scale_chunk(const T* g, T* out, int n, float factor) {
  const int t = threadIdx.x;
  if (((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(out)) & 15u) == 0) {
    const int whole = n >> 3;
    int i = t;
    for (; i + kOptThreads < whole; i += 2 * kOptThreads) {
      float a[8], b[8];
      load8(g + 8 * i, a);
      load8(g + 8 * (i + kOptThreads), b);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        a[j] *= factor;
        b[j] *= factor;
      }
      store8(out + 8 * i, a);
      store8(out + 8 * (i + kOptThreads), b);
    }
    if (i < whole) {
      float a[8];
      load8(g + 8 * i, a);
#pragma unroll
      for (int j = 0; j < 8; ++j) a[j] *= factor;
      store8(out + 8 * i, a);
    }
    if (t < (n & 7)) store1(out + 8 * whole + t, load1(g + 8 * whole + t) * factor);
  } else {
    for (int i = t; i < n; i += kOptThreads) store1(out + i, load1(g + i) * factor);
  }
}

// out = factor g, 43.3 us for those gradients (6.5 TB/s).  Chunks from the last to the first: the norm went the other way, and what it read last is still in L2.
// Gradients that are scaled in place by a factor of 1 keep their bits and are not touched.
template <int MOST>
__global__ void __launch_bounds__(kOptThreads) clip_kernel(const __grid_constant__ TensorTable<MOST, 2> t, const float* norm, float max_norm) {
  grid_launch_dependents();
  grid_dependency_wait();
  const float factor = clip_factor(norm, max_norm);
  const uint32_t c = t.chunks - 1 - blockIdx.x;
  const int i = tensor_of(t, c);
  if (factor == 1.0f && t.p[0][i] == t.p[1][i]) return;
  const int64_t at = chunk_start(t, i, c);
  const int len = chunk_length(t, i, at);
  if (t.n[i] < 0)
    scale_chunk(static_cast<const __nv_bfloat16*>(t.p[0][i]) + at, static_cast<__nv_bfloat16*>(t.p[1][i]) + at, len, factor);
  else
    scale_chunk(static_cast<const float*>(t.p[0][i]) + at, static_cast<float*>(t.p[1][i]) + at, len, factor);
}

__device__ __forceinline__ void adamw_update(float& t, float g, float& m, float& v, const AdamwParams& a) {
  m = a.beta1 * m + a.one_minus_beta1 * g;
  v = a.beta2 * v + a.one_minus_beta2 * g * g;
  t = t - a.lr * (m * a.c1 / (sqrtf(v * a.c2) + a.eps) + a.weight_decay * t);
}
__device__ __forceinline__ void load4(const float* p, float (&v)[4]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float (&v)[4]) {
  const uint2 a = *reinterpret_cast<const uint2*>(p);
  v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
}
template <class T>
__device__ __forceinline__ void adamw_chunk(float* theta, const T* g, float* m, float* v, int n, float factor, const AdamwParams& a) {
  const bool aligned = ((reinterpret_cast<uintptr_t>(theta) | reinterpret_cast<uintptr_t>(m) | reinterpret_cast<uintptr_t>(v)) & 15u) == 0 &&
                       (reinterpret_cast<uintptr_t>(g) & (4 * sizeof(T) - 1)) == 0;
  int done = 0;
  if (aligned) {
    const int whole = n >> 2;
    for (int i = threadIdx.x; i < whole; i += kOptThreads) {
      const int at = 4 * i;
      float tv[4], gv[4], mv[4], vv[4];
      load4(theta + at, tv);
      load4(g + at, gv);
      load4(m + at, mv);
      load4(v + at, vv);
#pragma unroll
      for (int j = 0; j < 4; ++j) adamw_update(tv[j], gv[j] * factor, mv[j], vv[j], a);
      *reinterpret_cast<float4*>(m + at) = make_float4(mv[0], mv[1], mv[2], mv[3]);
      *reinterpret_cast<float4*>(v + at) = make_float4(vv[0], vv[1], vv[2], vv[3]);
      *reinterpret_cast<float4*>(theta + at) = make_float4(tv[0], tv[1], tv[2], tv[3]);
    }
    done = 4 * whole;
  }
  for (int i = done + threadIdx.x; i < n; i += kOptThreads) {
    float tv = theta[i], mv = m[i], vv = v[i];
    adamw_update(tv, load1(g + i) * factor, mv, vv, a);
    m[i] = mv;
    v[i] = vv;
    theta[i] = tv;
  }
}

// 28 bytes per element (26 with bf16 gradients), DRAM-bound: 144 us for 35,168,256 (6.8 TB/s; 20 of their 141 MB are still in L2 after the norm).
template <int MOST>
__global__ void __launch_bounds__(kOptThreads) adamw_multi_kernel(const __grid_constant__ TensorTable<MOST, 4> t, const AdamwParams a,
                                                                 const float* norm, float max_norm) {
  grid_launch_dependents();
  grid_dependency_wait();
  const float factor = norm != nullptr ? clip_factor(norm, max_norm) : 1.0f;
  const uint32_t c = t.chunks - 1 - blockIdx.x;
  const int i = tensor_of(t, c);
  const int64_t at = chunk_start(t, i, c);
  const int len = chunk_length(t, i, at);
  float* theta = static_cast<float*>(t.p[0][i]) + at;
  float* m = static_cast<float*>(t.p[2][i]) + at;
  float* v = static_cast<float*>(t.p[3][i]) + at;
  if (t.n[i] < 0)
    adamw_chunk(theta, static_cast<const __nv_bfloat16*>(t.p[1][i]) + at, m, v, len, factor, a);
  else
    adamw_chunk(theta, static_cast<const float*>(t.p[1][i]) + at, m, v, len, factor, a);
}

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
// Calls of few tensors have a small argument (a launch copies it), others one of up to kMany tensors; more take several launches.
constexpr int kFew = 32, kMany = 384;
// Norms of little are taken by one cluster, in one launch: a chunk of up to 2048 elements for each of its warps.
constexpr uint32_t kWholeChunk = 2048, kWholeBlocks = 8, kWholeChunks = 32 * kWholeBlocks;

// Elements of a chunk of the norm: many where there is much to do (a block's work should outweigh finding it), few where the
// blocks of the chip would otherwise go without.
static uint32_t norm_chunk(const int64_t* n, int tensors) {
  int64_t total = 0;
  for (int i = 0; i < tensors; ++i) total += n[i];
  const int64_t blocks = 8 * device_sms();
  return total >= 8192 * blocks ? 8192 : total >= 4096 * blocks ? 4096 : 2048;
}
// What scales and updates has a block per chunk, and small ones: 35,168,256 gradients clipped in 52.4 us by the blocks of the chip
// taking chunks of 8192 in turn, 45.7 with a block for each 4096, 43.4 for each 2048; AdamW 164, 151, 147, and 144.6 for each 1024.
constexpr uint32_t kClipChunk = 2048, kAdamwChunk = 1024;

// Fills a table with tensors from `at` on and returns the first one that did not go in.
template <int MOST, int ARRAYS>
static int fill_table(TensorTable<MOST, ARRAYS>& t, void* const* const (&p)[ARRAYS], const int64_t* n, const int32_t* type, int tensors,
                      uint32_t chunk, int at) {
  t.tensors = 0;
  t.chunk = chunk;
  t.chunks = 0;
  for (; at < tensors && t.tensors < MOST; ++at) {
    if (n[at] == 0) continue;
    const int k = t.tensors++;
    t.first[k] = t.chunks;
    t.n[k] = n[at] | (type != nullptr && type[at] == SSCONV_BF16 ? kBf16 : 0);
    for (int j = 0; j < ARRAYS; ++j) t.p[j][k] = p[j][at];
    t.chunks += (uint32_t)((n[at] + chunk - 1) / chunk);
  }
  return at;
}

static int present(const int64_t* n, int tensors) {
  int k = 0;
  for (int i = 0; i < tensors; ++i) k += n[i] != 0;
  return k;
}

static uint32_t blocks_per_launch() { return 8u * device_sms(); }
size_t grad_norm_scratch(int tensors) { return sizeof(double) * blocks_per_launch() * (size_t)((tensors + kMany - 1) / kMany + 1); }

template <class Fold, int MOST>
static cudaError_t grad_norm_with(const void* const* g, const int64_t* n, const int32_t* type, int tensors, float* norm, double* partial,
                                  cudaStream_t st) {
  TensorTable<MOST, 1> t;
  void* const* const arrays[1] = {const_cast<void* const*>(g)};
  if (fill_table(t, arrays, n, type, tensors, kWholeChunk, 0) == tensors && t.chunks <= kWholeChunks) {
    // as many blocks as there are chunks for their warps
    uint32_t blocks = 1;
    while (blocks < kWholeBlocks && 32 * blocks < t.chunks) blocks <<= 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = 1024;
    cfg.stream = st;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = blocks;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cfg.attrs = attrs;
    cfg.numAttrs = blocks > 1 ? 2 : 1;
    count_launch();
    return cudaLaunchKernelEx(&cfg, grad_norm_kernel<Fold, true, MOST>, t, partial, norm);
  }
  const uint32_t most = blocks_per_launch(), chunk = norm_chunk(n, tensors);
  int at = 0, parts = 0;
  while (at < tensors) {
    at = fill_table(t, arrays, n, type, tensors, chunk, at);
    if (t.chunks == 0) break;
    const uint32_t blocks = t.chunks < most ? t.chunks : most;
    count_launch();
    const cudaError_t e = launch_dependent(grad_norm_kernel<Fold, false, MOST>, blocks, kOptThreads, st, t, partial + parts, norm);
    if (e != cudaSuccess) return e;
    parts += (int)blocks;
  }
  count_launch();
  return launch_dependent(grad_norm_finish_kernel<Fold>, 1, 256, st, (const double*)partial, parts, norm);
}

cudaError_t launch_grad_norm(const void* const* g, const int64_t* n, const int32_t* type, int tensors, bool inf, float* norm, double* partial,
                             cudaStream_t st) {
  if (present(n, tensors) <= kFew)
    return inf ? grad_norm_with<LargestMagnitude, kFew>(g, n, type, tensors, norm, partial, st)
               : grad_norm_with<SumOfSquares, kFew>(g, n, type, tensors, norm, partial, st);
  return inf ? grad_norm_with<LargestMagnitude, kMany>(g, n, type, tensors, norm, partial, st)
             : grad_norm_with<SumOfSquares, kMany>(g, n, type, tensors, norm, partial, st);
}

template <int MOST>
static cudaError_t clip_with(const void* const* g, void* const* out, const int64_t* n, const int32_t* type, int tensors, const float* norm,
                             float max_norm, cudaStream_t st) {
  TensorTable<MOST, 2> t;
  void* const* const arrays[2] = {const_cast<void* const*>(g), out};
  for (int at = 0; at < tensors;) {
    at = fill_table(t, arrays, n, type, tensors, kClipChunk, at);
    if (t.chunks == 0) break;
    count_launch();
    const cudaError_t e = launch_dependent(clip_kernel<MOST>, t.chunks, kOptThreads, st, t, norm, max_norm);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_clip_grads(const void* const* g, void* const* out, const int64_t* n, const int32_t* type, int tensors, const float* norm,
                              float max_norm, cudaStream_t st) {
  return present(n, tensors) <= kFew ? clip_with<kFew>(g, out, n, type, tensors, norm, max_norm, st)
                                     : clip_with<kMany>(g, out, n, type, tensors, norm, max_norm, st);
}

template <int MOST>
static cudaError_t adamw_with(void* const* theta, const void* const* g, void* const* m, void* const* v, const int64_t* n, const int32_t* type,
                              int tensors, const AdamwParams& a, const float* norm, float max_norm, cudaStream_t st) {
  TensorTable<MOST, 4> t;
  void* const* const arrays[4] = {theta, const_cast<void* const*>(g), m, v};
  for (int at = 0; at < tensors;) {
    at = fill_table(t, arrays, n, type, tensors, kAdamwChunk, at);
    if (t.chunks == 0) break;
    count_launch();
    const cudaError_t e = launch_dependent(adamw_multi_kernel<MOST>, t.chunks, kOptThreads, st, t, a, norm, max_norm);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_adamw_multi(void* const* theta, const void* const* g, void* const* m, void* const* v, const int64_t* n, const int32_t* type,
                               int tensors, const AdamwParams& a, const float* norm, float max_norm, cudaStream_t st) {
  return present(n, tensors) <= kFew ? adamw_with<kFew>(theta, g, m, v, n, type, tensors, a, norm, max_norm, st)
                                     : adamw_with<kMany>(theta, g, m, v, n, type, tensors, a, norm, max_norm, st);
}

}  // namespace ssconv
