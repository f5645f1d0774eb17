// The end of a block and the beginning of the next one in one pass: the norm of the block's output, its gate (a ConvNeXt
// block's layer scale, or a row of gates per image), the scaled residual and the next block's norm,
//   p = post(b),   h = scale x + gate p,   y = pre(h),
// and the gradients of all of it.  Both directions move 2 bytes per element and tensor (four of them forward, six backward).  Without
// norms they run at a copy's rate (12017 x 1000 11.6 us); with them at the instructions and latencies of the sums along a row: 60 % of
// the issue slots are used and 25 to 45 % of an SM's warps are there.  401408 x 96, gate and second norm: forward 57 us (5.4 TB/s),
// gradients 86 us (5.4 TB/s); 12017 x 1000 with both norms and gates per image 19.6 us (4.9 TB/s) and 46 us (3.2 TB/s).
//
// A row is held in the registers of a team of threads, V pieces of 8 channels each: part of a warp for few channels, a whole
// block for many.  Sums along a row go through shuffles, and through shared memory where the team has several warps.  A thread's
// next rows are on their way into shared memory meanwhile, into slots that only this thread reads: no barriers, no registers.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>

#include "launch.cuh"
#include "layout.cuh"
#include "resnorm.cuh"
#include "sm100_ptx.cuh"

namespace ssconv {

namespace {

// Eight values are four pairs: most of the arithmetic works on two values at once.
using Pair = unsigned long long;
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ Pair both(float v) { return f32x2(v, v); }
__device__ __forceinline__ float sum_of(Pair v) {
  float lo, hi;
  split2(v, lo, hi);
  return lo + hi;
}
__device__ __forceinline__ void unpack8(const uint4& a, Pair (&v)[4]) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = f32x2(bf16_lo(w[j]), bf16_hi(w[j]));
}
__device__ __forceinline__ uint32_t pack2(Pair v) {
  float lo, hi;
  split2(v, lo, hi);
  return pack_bf16x2<false>(lo, hi);
}
__device__ __forceinline__ uint4 pack8(const Pair (&v)[4]) { return make_uint4(pack2(v[0]), pack2(v[1]), pack2(v[2]), pack2(v[3])); }
// 8 of a vector of parameters, `otherwise` where there is no vector; zeros for a piece past the row, whose values then stay zero.
__device__ __forceinline__ void params8(const float* p, int piece, bool live, float otherwise, Pair (&v)[4]) {
  if (p == nullptr || !live) {
    const float o = live ? otherwise : 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = both(o);
    return;
  }
  const ulonglong2 a = reinterpret_cast<const ulonglong2*>(p)[2 * piece], b = reinterpret_cast<const ulonglong2*>(p)[2 * piece + 1];
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}
// A vector of parameters as a thread uses it: its pieces stay in registers, or (not HELD) are loaded, from L1, for every row.
template <int V, bool HELD>
struct Params {
  const float* p = nullptr;
  float otherwise = 0.0f;
  Pair held[HELD ? V : 1][4];
  __device__ __forceinline__ void set(const float* from, float without, int sub, int run, const bool (&live)[V]) {
    p = from;
    otherwise = without;
    if (HELD) {
#pragma unroll
      for (int k = 0; k < V; ++k) params8(from, sub + k * run, live[k], without, held[k]);
    }
  }
  __device__ __forceinline__ void get(int k, int piece, bool live, Pair (&v)[4]) const {
    if (HELD) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = held[k][j];
    } else {
      params8(p, piece, live, otherwise, v);
    }
  }
};
__device__ __forceinline__ void store_pairs(float* p, int piece, const Pair (&v)[4]) {
  reinterpret_cast<ulonglong2*>(p)[2 * piece] = make_ulonglong2(v[0], v[1]);
  reinterpret_cast<ulonglong2*>(p)[2 * piece + 1] = make_ulonglong2(v[2], v[3]);
}

// A team: LANES threads of a warp (a power of two), or all of a block's (LANES = 32 then).
//
// Sums over a block go through 16 slots per value, one per warp, zeros where there is no warp.  Two sets of them are used in turn,
// so that one barrier per sum is enough: a thread writes into a set again only after the barrier of the sum in between, which
// every reader of that set passes after it has read.
template <int LANES, bool BLOCK>
struct TeamSum {
  float* scratch;  // [2][2][16]
  int warps;
  __device__ __forceinline__ void begin(float* smem) {
    scratch = smem;
    warps = blockDim.x >> 5;
    if (BLOCK) {
      if (threadIdx.x < 32) scratch[threadIdx.x] = scratch[32 + threadIdx.x] = 0.0f;
      __syncthreads();
    }
  }
  __device__ __forceinline__ static void lanes(float& a) {
#pragma unroll
    for (int o = LANES >> 1; o > 0; o >>= 1) a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
  }
  __device__ __forceinline__ static float four(const float4& v) { return (v.x + v.y) + (v.z + v.w); }
  __device__ __forceinline__ float all_warps(const float* s) const {
    const float4* v = reinterpret_cast<const float4*>(s);
    float t = four(v[0]);
    if (warps > 4) t += four(v[1]);
    if (warps > 8) t += four(v[2]) + four(v[3]);
    return t;
  }
  __device__ __forceinline__ float* take_set() {
    float* s = scratch;
    // (the two sets are 128 bytes apart, at a multiple of 256)
    scratch = reinterpret_cast<float*>(reinterpret_cast<uintptr_t>(scratch) ^ 128u);
    return s;
  }
  __device__ __forceinline__ void operator()(float& a) {
    lanes(a);
    if (BLOCK) {
      float* s = take_set();
      if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = a;
      __syncthreads();
      a = all_warps(s);
    }
  }
  __device__ __forceinline__ void operator()(float& a, float& b) {
    lanes(a);
    lanes(b);
    if (BLOCK) {
      float* s = take_set();
      if ((threadIdx.x & 31) == 0) {
        s[threadIdx.x >> 5] = a;
        s[16 + (threadIdx.x >> 5)] = b;
      }
      __syncthreads();
      a = all_warps(s);
      b = all_warps(s + 16);
    }
  }
};

// Mean (0 for RMS) and 1 / deviation of a row; two passes over the registers, so that a mean far from zero costs no digits.  (A
// block's warps could put sums about their own means together with one barrier instead of two: 3000 x 4096 78 us instead of 40.)
template <int LANES, int V, bool BLOCK, int R>
__device__ __forceinline__ void row_statistics(const Pair (&v)[R][V][4], const bool (&live)[V], bool layer, float inv_c, float eps,
                                               TeamSum<LANES, BLOCK>& sum, float (&mean)[R], float (&rstd)[R]) {
  const auto sums = [&](float(&a)[R]) {
    if constexpr (R == 1)
      sum(a[0]);
    else
      sum(a[0], a[1]);
  };
#pragma unroll
  for (int i = 0; i < R; ++i) mean[i] = 0.0f;
  if (layer) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      Pair s = v[i][0][0];
#pragma unroll
      for (int k = 0; k < V; ++k)
#pragma unroll
        for (int j = k == 0 ? 1 : 0; j < 4; ++j) s = add2(s, v[i][k][j]);  // (zeros in pieces past the row)
      mean[i] = sum_of(s);
    }
    sums(mean);
#pragma unroll
    for (int i = 0; i < R; ++i) mean[i] *= inv_c;
  }
  float t[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    Pair q = 0;
    const Pair less = both(-mean[i]);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      Pair r = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Pair d = add2(v[i][k][j], less);
        r = fma2(d, d, r);
      }
      q = add2(q, live[k] ? r : 0ull);
    }
    t[i] = sum_of(q);
  }
  sums(t);
#pragma unroll
  for (int i = 0; i < R; ++i) rstd[i] = rsqrtf(t[i] * inv_c + eps);
}

constexpr int kCrewThreads = 256;  // of a block whose teams are parts of warps

// A thread's slots of 16 bytes for rows that are on their way: DEPTH rows of SLOTS pieces.  The threads' slots of one piece follow
// each other: with all slots of a thread side by side the copies took 83 us where they now take 59 (401408 x 96 forward).
template <int SLOTS, int DEPTH, bool BLOCK>
struct RowRing {
  uint32_t at, first, last;  // this thread's slot 0 of the row that is read and then filled next; of the first and the last row
  __device__ __forceinline__ static uint32_t slot_bytes() { return 16u * (BLOCK ? blockDim.x : (uint32_t)kCrewThreads); }
  __device__ __forceinline__ RowRing(const void* smem) {
    at = first = smem_u32(smem) + 16 * threadIdx.x;
    last = first + (DEPTH - 1) * SLOTS * slot_bytes();
  }
  // (nothing is read where bytes = 0: the slot gets zeros)
  __device__ __forceinline__ void fetch(int slot, const void* src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at + slot * slot_bytes()), "l"(src), "r"(bytes) : "memory");
  }
  __device__ __forceinline__ void next_row() {
    asm volatile("cp.async.commit_group;" ::: "memory");
    at = at == last ? first : at + SLOTS * slot_bytes();
  }
  // Once the row that is DEPTH - 1 behind the last one fetched has arrived; that is the one next to be filled again.
  __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory"); }
  __device__ __forceinline__ uint4 read(int slot) const {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "r"(at + slot * slot_bytes())
                 : "memory");
    return v;
  }
};
constexpr int kForwardDepth = 3;
__host__ __device__ constexpr int backward_depth(int V) { return V == 1 ? 3 : 2; }
constexpr int forward_smem(int V, int threads, int R) { return kForwardDepth * 2 * V * R * 16 * threads; }
constexpr int backward_smem(int V, int threads) { return backward_depth(V) * (4 * V + 1) * 16 * threads; }
constexpr int kMostSlots = 160 * 1024;  // bytes of any block's slots

struct ForwardParams {
  ResnormTensors t;
  int rows, rows_per_gate, C8;
  int crew_rows;              // consecutive rows of a crew (a warp with its teams, or a block)
  int post_layer, pre_layer;
  float scale, eps;
};

template <int LANES, int V, bool BLOCK, bool POST, bool PRE, int R = 1>
__global__ void __launch_bounds__(BLOCK ? 512 : kCrewThreads) resnorm_kernel(const ForwardParams p) {
  extern __shared__ __align__(16) uint8_t slots[];
  __shared__ __align__(256) float scratch[64];
  grid_launch_dependents();
  const int run = BLOCK ? blockDim.x : LANES;  // pieces between a thread's pieces
  const int sub = BLOCK ? threadIdx.x : threadIdx.x & (LANES - 1);
  constexpr int kTeams = BLOCK ? 1 : 32 / LANES;
  const int team = BLOCK ? 0 : (threadIdx.x & 31) / LANES;
  const int C8 = p.C8;
  const float inv_c = 1.0f / (float)(8 * C8);
  TeamSum<LANES, BLOCK> sum;
  sum.begin(scratch);
  RowRing<2 * V * R, kForwardDepth, BLOCK> ring(slots);
  bool own[V];
#pragma unroll
  for (int k = 0; k < V; ++k) own[k] = sub + k * run < C8;

  // (a warp's teams go on together: its first row decides)
  const int crew = BLOCK ? blockIdx.x : blockIdx.x * (kCrewThreads / 32) + (threadIdx.x >> 5);
  const int64_t first = (int64_t)crew * p.crew_rows;
  const int last = (int)min((int64_t)p.rows, first + p.crew_rows);
  int row = (int)min((int64_t)p.rows, first) + team;
  // bytes from the tensors' starts: of this thread's piece in the row that is fetched next, and in the one that is worked on
  const int64_t stride = (int64_t)kTeams * C8 * 16;
  int64_t coming = ((int64_t)row * C8 + sub) * 16, here = coming;
  int coming_row = row;
  const auto fetch = [&] {
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const bool mine = coming_row + i < last && own[k];
        const int64_t at = mine ? coming + i * stride + k * 16 * run : 0;
        ring.fetch(2 * (i * V + k), static_cast<const uint8_t*>(p.t.x) + at, mine ? 16u : 0u);
        ring.fetch(2 * (i * V + k) + 1, static_cast<const uint8_t*>(p.t.b) + at, mine ? 16u : 0u);
      }
    coming += R * stride;
    coming_row += R * kTeams;
    ring.next_row();
  };
  grid_dependency_wait();
#pragma unroll
  for (int d = 0; d < kForwardDepth - 1; ++d) fetch();
  constexpr bool kHeld = V == 1 || !BLOCK;
  Params<V, kHeld> gates, post_gamma, post_beta, pre_gamma, pre_beta;
  gates.set(p.rows_per_gate == 0 ? p.t.gate : nullptr, 1.0f, sub, run, own);
  if (POST) post_gamma.set(p.t.post_gamma, 1.0f, sub, run, own);
  if (POST) post_beta.set(p.t.post_beta, 0.0f, sub, run, own);
  if (PRE) pre_gamma.set(p.t.pre_gamma, 1.0f, sub, run, own);
  if (PRE) pre_beta.set(p.t.pre_beta, 0.0f, sub, run, own);
  int gates_end = p.rows_per_gate > 0 ? 0 : p.rows;  // the first row with other gates
  const Pair scale = both(p.scale);
  for (; row - team < last; row += R * kTeams, here += R * stride) {
    fetch();
    ring.wait();
    Pair bv[R][V][4], hv[R][V][4];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        unpack8(ring.read(2 * (i * V + k)), hv[i][k]);
        unpack8(ring.read(2 * (i * V + k) + 1), bv[i][k]);
      }
    float post_mean[R] = {}, post_rstd[R] = {}, pre_mean[R] = {}, pre_rstd[R] = {};
    if (POST) row_statistics<LANES, V, BLOCK, R>(bv, own, p.post_layer, inv_c, p.eps, sum, post_mean, post_rstd);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const bool there = row + i < last;
      if (there && row + i >= gates_end) {
        const int image = (row + i) / p.rows_per_gate;
        gates_end = (int)min((int64_t)p.rows, (int64_t)(image + 1) * p.rows_per_gate);
        gates.set(p.t.gate != nullptr ? p.t.gate + (int64_t)image * (8 * C8) : p.t.gate, 1.0f, sub, run, own);
      }
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int piece = sub + k * run;
        Pair g[4];
        gates.get(k, piece, own[k], g);
        if (POST) {
          Pair a[4], c[4];
          post_gamma.get(k, piece, own[k], a);
          post_beta.get(k, piece, own[k], c);
#pragma unroll
          for (int j = 0; j < 4; ++j) bv[i][k][j] = fma2(mul2(add2(bv[i][k][j], both(-post_mean[i])), both(post_rstd[i])), a[j], c[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) hv[i][k][j] = fma2(g[j], bv[i][k][j], mul2(scale, hv[i][k][j]));
        if (there && own[k] && p.t.h != nullptr)
          *reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.t.h) + here + i * stride + k * 16 * run) = pack8(hv[i][k]);
      }
    }
    if (PRE) {
      row_statistics<LANES, V, BLOCK, R>(hv, own, p.pre_layer, inv_c, p.eps, sum, pre_mean, pre_rstd);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int piece = sub + k * run;
        Pair a[4], c[4];
        pre_gamma.get(k, piece, own[k], a);
        pre_beta.get(k, piece, own[k], c);
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
          for (int j = 0; j < 4; ++j) hv[i][k][j] = fma2(mul2(add2(hv[i][k][j], both(-pre_mean[i])), both(pre_rstd[i])), a[j], c[j]);
          if (row + i < last && own[k]) *reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.t.y) + here + i * stride + k * 16 * run) = pack8(hv[i][k]);
        }
      }
    }
    if (sub == 0 && p.t.stats != nullptr) {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (row + i < last) reinterpret_cast<float4*>(p.t.stats)[row + i] = make_float4(post_mean[i], post_rstd[i], pre_mean[i], pre_rstd[i]);
    }
  }
}

// ---------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------
// With D = dL/dh in all (dh plus what comes back through the second norm) and the normalised rows bhat, hhat:
//   D = dh + r_h (g - mean(g) - hhat mean(g hhat)),  g = pre_gamma dy   (mean(g) for layer norms only),
//   dx = scale D,  dgate = sum D p,  dp = gate D,  db = r_b (q - mean(q) - bhat mean(q bhat)),  q = post_gamma dp,
//   dpre_gamma = sum dy hhat,  dpre_beta = sum dy,  dpost_gamma = sum dp bhat,  dpost_beta = sum dp.
// p, bhat and hhat are computed again from x and b, in 32 bits (h as it is stored has been rounded, and reading it instead of
// x would move the same bytes).
//
// The rows are cut into units of consecutive rows with the same row of gates; a crew (a warp with its teams, or a block) takes
// units in turn.  The sums over rows stay in registers; those of a row of gates are written at the end of each of its units,
// the others at the end of the block, and a second kernel adds up what the units and blocks have left, in a fixed order.
enum { kGate, kPostGamma, kPostBeta, kPreGamma, kPreBeta, kSums };

struct BackwardParams {
  ResnormTensors t;
  ResnormGradients g;
  int rows, gate_rows;        // gate_rows: rows with the same gates (all of them for shared or no gates)
  int units, unit_rows, units_per_gate;
  int C8;
  int post_layer, pre_layer, image_gates;
  float scale;
  float* block_sums;          // [blocks][kSums][C]
  float* unit_sums;           // [units][C]
};

// A place among a crew's rows: a unit, the first of the teams' rows in it, and the unit's end.
struct Place {
  int unit, image, row, end;
};
__device__ __forceinline__ Place start_of(const BackwardParams& p, int unit) {
  const int image = unit / p.units_per_gate;
  const int64_t first = (int64_t)image * p.gate_rows + (int64_t)(unit - image * p.units_per_gate) * p.unit_rows;
  const int64_t end = min((int64_t)p.rows, min((int64_t)(image + 1) * p.gate_rows, first + p.unit_rows));
  return {unit, image, (int)min((int64_t)p.rows, first), (int)end};
}

template <int LANES, int V, bool BLOCK, bool POST, bool PRE>
__global__ void __launch_bounds__(BLOCK ? 512 : kCrewThreads) resnorm_backward_kernel(const BackwardParams p) {
  extern __shared__ __align__(16) uint8_t slots[];
  float* rows_of_warps = reinterpret_cast<float*>(slots);  // [warps][C], of warp crews, in the end
  __shared__ __align__(256) float scratch[64];
  grid_launch_dependents();
  const int run = BLOCK ? blockDim.x : LANES;
  const int sub = BLOCK ? threadIdx.x : threadIdx.x & (LANES - 1);
  constexpr int kTeams = BLOCK ? 1 : 32 / LANES;
  const int team = BLOCK ? 0 : (threadIdx.x & 31) / LANES;
  constexpr int kCrewsPerBlock = BLOCK ? 1 : kCrewThreads / 32;
  const int crews = gridDim.x * kCrewsPerBlock;
  const int C8 = p.C8, C = 8 * C8;
  const float inv_c = 1.0f / (float)C;
  TeamSum<LANES, BLOCK> sum;
  sum.begin(scratch);
  constexpr int kDepth = backward_depth(V), kStats = 4 * V;  // slots: b, x, dy, dh of each piece, and the row's statistics
  RowRing<4 * V + 1, kDepth, BLOCK> ring(slots);
  bool own[V];
#pragma unroll
  for (int k = 0; k < V; ++k) own[k] = sub + k * run < C8;
  Pair acc[kSums][V][4];
#pragma unroll
  for (int a = 0; a < kSums; ++a)
#pragma unroll
    for (int k = 0; k < V; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[a][k][j] = 0;
  const bool with_dh = p.g.dh != nullptr;

  const auto go_on = [&](Place& at) {
    at.row += kTeams;
    if (at.row >= at.end) at = start_of(p, at.unit + crews);
  };
  const auto fetch = [&](Place& at) {
    const int row = at.row + team;
    const bool there = row < at.end && at.unit < p.units;
    if (POST || PRE) ring.fetch(kStats, p.t.stats + 4 * (int64_t)(there ? row : 0), there ? 16u : 0u);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const bool mine = there && own[k];
      const int64_t i = mine ? ((int64_t)row * C8 + sub + k * run) * 16 : 0;
      const uint32_t bytes = mine ? 16u : 0u;
      ring.fetch(4 * k, static_cast<const uint8_t*>(p.t.b) + i, bytes);
      if (PRE) {
        ring.fetch(4 * k + 1, static_cast<const uint8_t*>(p.t.x) + i, bytes);
        ring.fetch(4 * k + 2, static_cast<const uint8_t*>(p.g.dy) + i, bytes);
      }
      if (with_dh) ring.fetch(4 * k + 3, static_cast<const uint8_t*>(p.g.dh) + i, bytes);
    }
    ring.next_row();
    if (at.unit < p.units) go_on(at);
  };

  grid_dependency_wait();
  Place at = start_of(p, blockIdx.x * kCrewsPerBlock + (BLOCK ? 0 : threadIdx.x >> 5)), coming = at;
#pragma unroll
  for (int d = 0; d < kDepth - 1; ++d) fetch(coming);
  constexpr bool kHeld = V == 1 || !BLOCK;
  Params<V, kHeld> gates, post_gamma, post_beta, pre_gamma;
  const auto set_gates = [&] { gates.set(p.t.gate != nullptr && p.image_gates ? p.t.gate + (int64_t)at.image * C : p.t.gate, 1.0f, sub, run, own); };
  if (at.unit < p.units) set_gates();
  if (POST) post_gamma.set(p.t.post_gamma, 1.0f, sub, run, own);
  if (POST) post_beta.set(p.t.post_beta, 0.0f, sub, run, own);
  if (PRE) pre_gamma.set(p.t.pre_gamma, 1.0f, sub, run, own);
  const Pair scale = both(p.scale);
  while (at.unit < p.units) {
    fetch(coming);
    Place next = at;
    go_on(next);
    ring.wait();
    float4 stats = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (POST || PRE) {
      const uint4 v = ring.read(kStats);
      stats = make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
    }
    const bool there = at.row + team < at.end;
    const int64_t here = ((int64_t)(at.row + team) * C8 + sub) * 16;

    // (pieces past the row and rows past the unit are zeros with parameters or gradients of zero: nothing of them is left in a sum)
    Pair d[V][4], hat[V][4], pv[V][4];  // pv: bhat with a first norm, else b itself
    Pair s1 = 0, s2 = 0;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int piece = sub + k * run;
      unpack8(ring.read(4 * k), pv[k]);
      unpack8(with_dh ? ring.read(4 * k + 3) : make_uint4(0u, 0u, 0u, 0u), d[k]);
      if (POST) {
#pragma unroll
        for (int j = 0; j < 4; ++j) pv[k][j] = mul2(add2(pv[k][j], both(-stats.x)), both(stats.y));
      }
      if (PRE) {
        Pair gv[4], a[4], c[4], g[4];
        unpack8(ring.read(4 * k + 1), hat[k]);
        unpack8(ring.read(4 * k + 2), gv);
        gates.get(k, piece, own[k], g);
        if (POST) {
          post_gamma.get(k, piece, own[k], a);
          post_beta.get(k, piece, own[k], c);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const Pair pj = POST ? fma2(pv[k][j], a[j], c[j]) : pv[k][j];
          const Pair h = fma2(g[j], pj, mul2(scale, hat[k][j]));
          hat[k][j] = mul2(add2(h, both(-stats.z)), both(stats.w));
          acc[kPreGamma][k][j] = fma2(gv[j], hat[k][j], acc[kPreGamma][k][j]);
          acc[kPreBeta][k][j] = add2(acc[kPreBeta][k][j], gv[j]);
        }
        pre_gamma.get(k, piece, own[k], a);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const Pair q = mul2(gv[j], a[j]);
          s1 = add2(s1, q);
          s2 = fma2(q, hat[k][j], s2);
          // dh plus what the norm hands back, but for the means
          d[k][j] = fma2(q, both(stats.w), d[k][j]);
        }
      }
    }
    Pair from_mean = 0, from_hat = 0;
    if (PRE) {
      float m = sum_of(s1), q = sum_of(s2);
      sum(m, q);
      from_mean = both(p.pre_layer ? -stats.w * (m * inv_c) : 0.0f);
      from_hat = both(-stats.w * (q * inv_c));
    }
    Pair t1 = 0, t2 = 0;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int piece = sub + k * run;
      const bool mine = there && own[k];
      Pair a[4], c[4], g[4];
      if (PRE) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          d[k][j] = add2(fma2(hat[k][j], from_hat, from_mean), d[k][j]);
        }
      }
      if (mine && p.g.dx != nullptr) {
        Pair o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = mul2(scale, d[k][j]);
        *reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.g.dx) + here + k * 16 * run) = pack8(o);
      }
      gates.get(k, piece, own[k], g);
      if (POST) {
        post_gamma.get(k, piece, own[k], a);
        post_beta.get(k, piece, own[k], c);
      }
      if (mine)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Pair pj = POST ? fma2(pv[k][j], a[j], c[j]) : pv[k][j];
        acc[kGate][k][j] = fma2(d[k][j], pj, acc[kGate][k][j]);
        d[k][j] = mul2(d[k][j], g[j]);  // dp from here on
        if (POST) {
          acc[kPostGamma][k][j] = fma2(d[k][j], pv[k][j], acc[kPostGamma][k][j]);
          acc[kPostBeta][k][j] = add2(acc[kPostBeta][k][j], d[k][j]);
          d[k][j] = mul2(d[k][j], a[j]);
          t1 = add2(t1, d[k][j]);
          t2 = fma2(d[k][j], pv[k][j], t2);
        }
      }
    }
    if (POST) {
      float m = sum_of(t1), q = sum_of(t2);
      sum(m, q);
      from_mean = both(p.post_layer ? -stats.y * (m * inv_c) : 0.0f);
      from_hat = both(-stats.y * (q * inv_c));
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (POST) {
#pragma unroll
        for (int j = 0; j < 4; ++j) d[k][j] = fma2(d[k][j], both(stats.y), fma2(pv[k][j], from_hat, from_mean));
      }
      if (there && own[k] && p.g.db != nullptr) *reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.g.db) + here + k * 16 * run) = pack8(d[k]);
    }

    if (next.unit != at.unit && p.image_gates && p.g.dgate != nullptr) {
      float* to = p.units_per_gate == 1 ? p.g.dgate + (int64_t)at.image * C : p.unit_sums + (int64_t)at.unit * C;
#pragma unroll
      for (int k = 0; k < V; ++k) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int o = 16; o >= LANES; o >>= 1) acc[kGate][k][j] = add2(acc[kGate][k][j], __shfl_xor_sync(0xFFFFFFFFu, acc[kGate][k][j], o));
        if (own[k] && team == 0) store_pairs(to, sub + k * run, acc[kGate][k]);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[kGate][k][j] = 0;
      }
    }
    const bool other = next.image != at.image;
    at = next;
    if (other && at.unit < p.units) set_gates();
  }

  // What is left in the registers, summed over the block's warps and teams (in the slots' memory: every copy into it is over).
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (!BLOCK) __syncthreads();
  float* mine = p.block_sums + (int64_t)blockIdx.x * kSums * C;
#pragma unroll
  for (int a = 0; a < kSums; ++a) {
    const float* wanted = a == kGate ? (p.image_gates ? nullptr : p.g.dgate) : a == kPostGamma ? p.g.dpost_gamma : a == kPostBeta ? p.g.dpost_beta
                          : a == kPreGamma ? p.g.dpre_gamma : p.g.dpre_beta;
    if (wanted == nullptr) continue;
    if ((a == kPostGamma || a == kPostBeta) && !POST) continue;
    if ((a == kPreGamma || a == kPreBeta) && !PRE) continue;
    float* out = BLOCK ? mine + a * C : rows_of_warps + (threadIdx.x >> 5) * C;
#pragma unroll
    for (int k = 0; k < V; ++k) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int o = 16; o >= LANES; o >>= 1) acc[a][k][j] = add2(acc[a][k][j], __shfl_xor_sync(0xFFFFFFFFu, acc[a][k][j], o));
      if (own[k] && team == 0) store_pairs(out, sub + k * run, acc[a][k]);
    }
    if (!BLOCK) {
      __syncthreads();
      for (int c = threadIdx.x; c < C; c += blockDim.x) {
        float s = 0.0f;
        for (int w = 0; w < (int)(blockDim.x >> 5); ++w) s += rows_of_warps[w * C + c];
        mine[a * C + c] = s;
      }
      __syncthreads();
    }
  }
}

struct FinishParams {
  const float* block_sums;
  const float* unit_sums;
  float* out[kSums];          // the sums that are wanted ...
  int kind[kSums];            // ... and where they are among a block's
  int wanted, blocks, C;
  int images, units_per_gate; // of gates per image whose units were several (0 images: none)
  int block_shift, image_shift;  // base-2 logarithms of R
  float* dgate;
};
// 4 columns per thread and 1024 / R threads side by side; the R threads of the same columns share the rows, so that none adds up
// hundreds of them by itself.  (R = 1 for the images, us of the gradients: 4 images of 100352 x 96 121, 99 so; R = 32: 61 images of
// 197 x 1000 71, 47 so.)  First the sums over blocks, then those of the images' units.
__global__ void __launch_bounds__(1024) resnorm_finish_kernel(const FinishParams p) {
  __shared__ float4 part[1024];
  grid_launch_dependents();
  grid_dependency_wait();
  const int C4 = p.C / 4, groups = (C4 + (1024 >> p.block_shift) - 1) >> (10 - p.block_shift), job = blockIdx.x - groups * p.wanted;
  const bool images = job >= 0;
  const int shift = images ? p.image_shift : p.block_shift;  // R = 1 << shift
  const int side = 1024 >> shift, r = threadIdx.x >> (10 - shift);
  const float4* in;
  float4* out;
  int64_t pitch;
  int count;
  bool any;
  if (images) {
    const int64_t i = (int64_t)job * side + (threadIdx.x & (side - 1)), image = i / C4;
    any = i < (int64_t)p.images * C4;
    count = p.units_per_gate;
    in = reinterpret_cast<const float4*>(p.unit_sums) + image * count * C4 + (i - image * C4);
    out = reinterpret_cast<float4*>(p.dgate) + i;
    pitch = C4;
  } else {
    const int which = blockIdx.x / groups, i = (blockIdx.x - which * groups) * side + (threadIdx.x & (side - 1));
    any = i < C4;
    count = p.blocks;
    in = reinterpret_cast<const float4*>(p.block_sums) + (int64_t)p.kind[which] * C4 + i;
    out = reinterpret_cast<float4*>(p.out[which]) + i;
    pitch = (int64_t)kSums * C4;
  }
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const auto add = [&](const float4& v) {
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  };
  if (!any) count = 0;
  for (int u = r; u < count; u += 8 << shift) {  // eight loads under way
    float4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = u + (k << shift) < count ? in[(u + (k << shift)) * pitch] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < 8; ++k) add(v[k]);
  }
  if (shift != 0) {
    for (int o = 16; o >= side; o >>= 1)  // the same columns in a warp
      add(make_float4(__shfl_xor_sync(0xFFFFFFFFu, s.x, o), __shfl_xor_sync(0xFFFFFFFFu, s.y, o), __shfl_xor_sync(0xFFFFFFFFu, s.z, o),
                      __shfl_xor_sync(0xFFFFFFFFu, s.w, o)));
    part[threadIdx.x] = s;
    __syncthreads();
    if (r != 0) return;
    const int next = side < 32 ? 32 : side;
#pragma unroll 8
    for (int k = threadIdx.x + next; k < 1024; k += next) add(part[k]);
  }
  if (any) *out = s;
}

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
struct Team {
  bool block;
  int V, lanes, threads;  // threads of a block
};
int power_of_two_from(int n) {
  int p = 1;
  while (p < n) p <<= 1;
  return p;
}
// Rows of up to 768 channels are part of a warp, with up to `most` pieces per lane: as few lane-pieces as hold a row, and of equal
// ones the fewer lanes, because what is done once per row costs every lane the same.  Parameters and sums of a lane's channels
// stay in its registers.  Longer rows are a block's, one piece per thread (two beyond 4096 channels), and so are those of more than
// 256 channels where there are few rows, for their latency (49 x 768: 2.1 us instead of 4.1).
// us, forward: 401408 x 96 on 16 lanes of one piece 62, on 4 of three 57; 25088 x 384 on a block of 64 threads 23.9, on 16 lanes of
// three 15.8.
Team team_for(int C8, int most, int64_t rows) {
  const bool few = rows <= 4 * (int64_t)device_sms();
  if (C8 <= 32 * (few ? 1 : most)) {
    Team best = {false, 1, 1 << 20, kCrewThreads};
    for (int V = few ? 1 : most; V >= 1; --V) {
      const int lanes = power_of_two_from((C8 + V - 1) / V);
      // (several pieces only where a row's lanes still load 64 bytes side by side: 400000 x 16 on one lane of two 15.8, on two 8.9)
      if (lanes <= 32 && (V == 1 || lanes >= 4) && lanes * V < best.lanes * best.V) best = {false, V, lanes, kCrewThreads};
    }
    return best;
  }
  const int V = C8 <= 512 ? 1 : 2;
  const int threads = (((C8 + V - 1) / V) + 31) / 32 * 32;
  return {true, V, threads, threads};
}

// Allows a kernel its dynamic shared memory, once per device, and says how many of its blocks an SM then holds.
struct Resident {
  std::atomic<uint64_t> key{0};  // the kernel's address and the threads of its blocks
  std::atomic<int> blocks[64];
};
int resident_blocks(const void* kernel, int threads, int smem) {
  static Resident known[512];
  int dev = 0, blocks = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  const uint64_t key = (uint64_t)reinterpret_cast<uintptr_t>(kernel) ^ ((uint64_t)threads << 50);
  Resident* r = nullptr;
  for (Resident& k : known) {
    uint64_t at = k.key.load(std::memory_order_relaxed);
    if (at == 0 && k.key.compare_exchange_strong(at, key)) at = key;
    if (at == key) {
      r = &k;
      break;
    }
  }
  if (r != nullptr) blocks = r->blocks[dev].load(std::memory_order_relaxed);
  if (blocks == 0) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSlots) != cudaSuccess) return 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, kernel, threads, smem) != cudaSuccess || blocks <= 0) return 0;
    if (r != nullptr) r->blocks[dev].store(blocks, std::memory_order_relaxed);
  }
  return blocks;
}

static_assert(forward_smem(1, 512, 2) <= kMostSlots && forward_smem(2, 512, 1) <= kMostSlots && forward_smem(3, 256, 1) <= kMostSlots && backward_smem(1, 512) <= kMostSlots && backward_smem(2, 512) <= kMostSlots, "");

// The kernel of a team.
#define SSCONV_LANES_KERNEL(kernel, V)                        \
  switch (t.lanes) {                                          \
    case 1: return kernel<1, V, false, POST, PRE>;            \
    case 2: return kernel<2, V, false, POST, PRE>;            \
    case 4: return kernel<4, V, false, POST, PRE>;            \
    case 8: return kernel<8, V, false, POST, PRE>;            \
    case 16: return kernel<16, V, false, POST, PRE>;          \
    default: return kernel<32, V, false, POST, PRE>;          \
  }
template <bool POST, bool PRE>
void (*forward_kernel(const Team& t, int R))(ForwardParams) {
  if (t.block && R == 2) return resnorm_kernel<32, 1, true, POST, PRE, 2>;
  if (t.block) return t.V == 1 ? resnorm_kernel<32, 1, true, POST, PRE> : resnorm_kernel<32, 2, true, POST, PRE>;
  if (t.V == 1) SSCONV_LANES_KERNEL(resnorm_kernel, 1)
  if (t.V == 2) SSCONV_LANES_KERNEL(resnorm_kernel, 2)
  SSCONV_LANES_KERNEL(resnorm_kernel, 3)
}
template <bool POST, bool PRE>
void (*backward_kernel(const Team& t))(BackwardParams) {
  if (t.block) return t.V == 1 ? resnorm_backward_kernel<32, 1, true, POST, PRE> : resnorm_backward_kernel<32, 2, true, POST, PRE>;
  if (t.V == 1) SSCONV_LANES_KERNEL(resnorm_backward_kernel, 1)
  SSCONV_LANES_KERNEL(resnorm_backward_kernel, 2)
}
#undef SSCONV_LANES_KERNEL

// How the backward pass is cut: units, and blocks (the scratch is sized by them).
struct Cut {
  Team team;
  int units, unit_rows, units_per_gate, gate_rows, blocks, images;
  bool image_gates;
};
constexpr int kBackwardWarps = 16;       // per SM, of crews at work at once; half as many where a lane has two pieces' sums in registers
constexpr int kRowsPerTeam = 4;          // of a unit, at least: its sums are written once

Cut cut_backward(const ssconv_resnorm_t& d) {
  Cut c;
  // Two pieces with two norms or more than 256 channels, us of the gradients alone, one piece / two (/ three): 120170 x 96 with two norms
  // 52 / 38 (/ 58), 25088 x 384 with one 42 / 34 (/ 50); but 401408 x 96 with one 86 / 91.
  const bool both_norms = d.post != SSCONV_NORM_NONE && d.pre != SSCONV_NORM_NONE;
  c.team = team_for(d.C / 8, both_norms || d.C > 256 ? 2 : 1, d.rows);
  c.image_gates = d.rows_per_gate > 0;
  const int64_t rows = d.rows;
  c.gate_rows = (int)(c.image_gates && d.rows_per_gate < rows ? d.rows_per_gate : rows);
  c.images = (int)((rows + c.gate_rows - 1) / c.gate_rows);
  const int crew_warps = c.team.block ? c.team.threads / 32 : 1;
  const int teams = c.team.block ? 1 : 32 / c.team.lanes;
  const int crews_per_block = c.team.block ? 1 : c.team.threads / 32;
  const int warps = c.team.V > 1 && !c.team.block ? kBackwardWarps / 2 : kBackwardWarps;
  const int64_t most = (int64_t)device_sms() * (warps / crew_warps > 0 ? warps / crew_warps : 1);
  // Units per row of gates: as many as keep the crew with the most rows short, fewer where it makes no difference.
  const int64_t worth = (c.gate_rows + teams * kRowsPerTeam - 1) / (teams * kRowsPerTeam);
  const int64_t all = most / c.images < 1 ? 1 : most / c.images;
  int64_t least = -1;
  for (int64_t k = 1; k <= 9; ++k) {
    int64_t units = k == 9 ? all : k;
    if (units > worth) units = worth;
    const int64_t unit_rows = (c.gate_rows + units - 1) / units;
    units = (c.gate_rows + unit_rows - 1) / unit_rows;
    const int64_t turns = (c.images * units + most - 1) / most;
    const int64_t cost = turns * ((unit_rows + teams - 1) / teams + 1);
    if (least < 0 || cost < least) {
      least = cost;
      c.unit_rows = (int)unit_rows;
      c.units_per_gate = (int)units;
    }
  }
  c.units = c.images * c.units_per_gate;
  const int64_t crews = c.units < most ? c.units : most;
  c.blocks = (int)((crews + crews_per_block - 1) / crews_per_block);
  return c;
}

}  // namespace

cudaError_t launch_resnorm(const ssconv_resnorm_t& d, const ResnormTensors& t, cudaStream_t st) {
  const int C8 = d.C / 8;
  const Team team = team_for(C8, 3, d.rows);
  const bool post = d.post != SSCONV_NORM_NONE, pre = d.pre != SSCONV_NORM_NONE && t.y != nullptr;
  const auto kernel_of = [&](int rows) {
    return post ? (pre ? forward_kernel<true, true>(team, rows) : forward_kernel<true, false>(team, rows))
                : (pre ? forward_kernel<false, true>(team, rows) : forward_kernel<false, false>(team, rows));
  };
  const auto resident = [&](int rows) {
    return resident_blocks((const void*)kernel_of(rows), team.threads, forward_smem(team.V, team.threads, rows));
  };
  // Blocks take two rows at a time, whose sums share barriers, where as many blocks with two rows as with one fit an SM.  us with
  // one / two, both norms: 9000 x 4096 97 / 83, 3500 x 3584 39 / 33, 6000 x 2048 31 / 28; where fewer fit: 5000 x 2504 33 / 38.
  const int R = team.block && team.V == 1 && d.rows > 8 * (int64_t)device_sms() && resident(2) >= resident(1) ? 2 : 1;
  const auto kernel = kernel_of(R);
  const int smem = forward_smem(team.V, team.threads, R);
  const int teams = team.block ? 1 : 32 / team.lanes, crews_per_block = team.block ? 1 : team.threads / 32;
  const int64_t most = (int64_t)device_sms() * resident(R) * crews_per_block;
  if (most == 0) return cudaErrorUnknown;
  const int64_t turns = (d.rows + most * teams * R - 1) / (most * teams * R);
  ForwardParams p = {};
  p.t = t;
  p.rows = (int)d.rows;
  p.rows_per_gate = (int)(d.rows_per_gate < d.rows ? d.rows_per_gate : d.rows);
  p.C8 = C8;
  p.crew_rows = (int)(turns * teams * R);
  p.post_layer = d.post == SSCONV_NORM_LAYER;
  p.pre_layer = d.pre == SSCONV_NORM_LAYER;
  p.scale = d.scale;
  p.eps = d.eps;
  const int64_t crews = (d.rows + p.crew_rows - 1) / p.crew_rows;
  count_launch();
  return launch_dependent_smem(kernel, (unsigned)((crews + crews_per_block - 1) / crews_per_block), team.threads, smem, st, p);
}

size_t resnorm_scratch(const ssconv_resnorm_t& d) {
  if (d.rows == 0) return 0;
  const Cut c = cut_backward(d);
  size_t floats = (size_t)c.blocks * kSums * d.C;
  if (c.image_gates && c.units_per_gate > 1) floats += (size_t)c.units * d.C;
  return floats * sizeof(float);
}

cudaError_t launch_resnorm_backward(const ssconv_resnorm_t& d, const ResnormTensors& t, const ResnormGradients& g, float* ws, cudaStream_t st) {
  float* const sums[kSums] = {g.dgate, g.dpost_gamma, g.dpost_beta, g.dpre_gamma, g.dpre_beta};
  const Cut c = cut_backward(d);
  BackwardParams p;
  p.t = t;
  p.g = g;
  p.rows = (int)d.rows;
  p.gate_rows = c.gate_rows;
  p.units = c.units;
  p.unit_rows = c.unit_rows;
  p.units_per_gate = c.units_per_gate;
  p.C8 = d.C / 8;
  p.post_layer = d.post == SSCONV_NORM_LAYER;
  p.pre_layer = d.pre == SSCONV_NORM_LAYER;
  p.image_gates = c.image_gates;
  p.scale = d.scale;
  p.block_sums = ws;
  p.unit_sums = ws + (size_t)c.blocks * kSums * d.C;
  const bool post = d.post != SSCONV_NORM_NONE, pre = d.pre != SSCONV_NORM_NONE;
  const auto kernel = post ? (pre ? backward_kernel<true, true>(c.team) : backward_kernel<true, false>(c.team))
                           : (pre ? backward_kernel<false, true>(c.team) : backward_kernel<false, false>(c.team));
  const int smem = backward_smem(c.team.V, c.team.threads);  // (more than a row of sums per warp)
  if (resident_blocks((const void*)kernel, c.team.threads, smem) == 0) return cudaErrorUnknown;
  count_launch();
  cudaError_t e = launch_dependent_smem(kernel, (unsigned)c.blocks, c.team.threads, smem, st, p);
  if (e != cudaSuccess) return e;

  FinishParams f = {};
  f.block_sums = p.block_sums;
  f.unit_sums = p.unit_sums;
  for (int i = 0; i < kSums; ++i)
    if (sums[i] != nullptr && !(i == kGate && c.image_gates)) {
      f.out[f.wanted] = sums[i];
      f.kind[f.wanted++] = i;
    }
  f.blocks = c.blocks;
  f.C = d.C;
  f.units_per_gate = c.units_per_gate;
  f.images = c.image_gates && c.units_per_gate > 1 && g.dgate != nullptr ? c.images : 0;
  f.dgate = g.dgate;
  const int64_t C4 = d.C / 4;
  const auto jobs = [](int64_t columns, int shift) { return (columns + (1024 >> shift) - 1) >> (10 - shift); };
  // the images' units: up to eight rows per thread; the blocks' sums: as many threads as make for two blocks per SM
  while (f.image_shift < 5 && (8 << f.image_shift) < c.units_per_gate) ++f.image_shift;
  f.block_shift = 5;
  while (f.block_shift < 7 && jobs(C4, f.block_shift + 1) * f.wanted <= 2 * device_sms()) ++f.block_shift;
  const int64_t blocks = jobs(C4, f.block_shift) * f.wanted + jobs(f.images * C4, f.image_shift);
  if (blocks == 0) return cudaSuccess;
  count_launch();
  return launch_dependent(resnorm_finish_kernel, (unsigned)blocks, 1024, st, f);
}

}  // namespace ssconv
