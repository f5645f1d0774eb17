// The end of a block and the beginning of the next one in one pass: the norm of the block's output, its gate (a ConvNeXt
// block's layer scale, or a row of gates per image), the scaled residual and the next block's norm,
//   p = post(b),   h = scale x + gate p,   y = pre(h),
// and the gradients of all of it.  Both directions move 2 bytes per element and tensor and do some tens of flops per element:
// DRAM-bound, or short.
//
// A row is held in the registers of a team of threads, V pieces of 8 channels each: part of a warp for few channels, a whole
// block for many.  Sums along a row go through shuffles, and through shared memory where the team has several warps.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>

#include "launch.cuh"
#include "layout.cuh"
#include "resnorm.cuh"
#include "sm100_ptx.cuh"

namespace ssconv {

namespace {

__device__ __forceinline__ void unpack8(const uint4& a, float (&v)[8]) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = bf16_lo(w[j]);
    v[2 * j + 1] = bf16_hi(w[j]);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(pack_bf16x2<false>(v[0], v[1]), pack_bf16x2<false>(v[2], v[3]), pack_bf16x2<false>(v[4], v[5]),
                    pack_bf16x2<false>(v[6], v[7]));
}
// 8 of a vector of parameters, `otherwise` where there is none.
__device__ __forceinline__ void params8(const float* p, int piece, bool live, float otherwise, float (&v)[8]) {
  if (p == nullptr || !live) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = otherwise;
    return;
  }
  const float4 a = reinterpret_cast<const float4*>(p)[2 * piece], b = reinterpret_cast<const float4*>(p)[2 * piece + 1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// Sums over a team's threads, known to all of them afterwards.  Teams of several warps are whole blocks; their sums alternate
// between two halves of the scratch, so that one barrier per sum is enough: a thread writes into a half again only after the
// barrier of the sum in between, which every reader of that half passes after it has read.
template <bool BLOCK>
struct TeamSum {
  float* scratch;  // [2][2][16]
  int lanes;       // of a team within a warp
  int half = 0;
  __device__ __forceinline__ void operator()(float& a, float& b) {
    if (BLOCK) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
      }
      float* s = scratch + 32 * half;
      half ^= 1;
      const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
      if ((threadIdx.x & 31) == 0) {
        s[warp] = a;
        s[16 + warp] = b;
      }
      __syncthreads();
      a = b = 0.0f;
      for (int i = 0; i < warps; ++i) {
        a += s[i];
        b += s[16 + i];
      }
    } else {
      for (int o = lanes >> 1; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
      }
    }
  }
  __device__ __forceinline__ void operator()(float& a) {
    float unused = 0.0f;
    if (BLOCK) {
      (*this)(a, unused);
    } else {
      for (int o = lanes >> 1; o > 0; o >>= 1) a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
    }
  }
};

// Mean (0 for RMS) and 1 / deviation of a row; two passes over the registers, so that a mean far from zero costs no digits.
template <int V, bool BLOCK>
__device__ __forceinline__ void row_statistics(const float (&v)[V][8], const bool (&live)[V], bool layer, float inv_c, float eps,
                                               TeamSum<BLOCK>& sum, float& mean, float& rstd) {
  mean = 0.0f;
  if (layer) {
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < V; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[k][j];  // (zeros in pieces past the row)
    sum(s);
    mean = s * inv_c;
  }
  float q = 0.0f;
#pragma unroll
  for (int k = 0; k < V; ++k)
    if (live[k]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = v[k][j] - mean;
        q = fmaf(d, d, q);
      }
    }
  sum(q);
  rstd = rsqrtf(q * inv_c + eps);
}

struct ForwardParams {
  ResnormTensors t;
  int rows, rows_per_gate, C8, lanes;
  int post_layer, pre_layer;
  float scale, eps;
};

template <int V, bool BLOCK, bool POST, bool PRE>
__global__ void __launch_bounds__(BLOCK ? 512 : 256) resnorm_kernel(const ForwardParams p) {
  __shared__ float scratch[64];
  grid_launch_dependents();
  const int lanes = BLOCK ? blockDim.x : p.lanes;
  const int sub = BLOCK ? threadIdx.x : threadIdx.x & (lanes - 1);
  const int per_block = BLOCK ? 1 : blockDim.x / lanes;
  const int step = gridDim.x * per_block;
  const float inv_c = 1.0f / (float)(8 * p.C8);
  TeamSum<BLOCK> sum{scratch, lanes};
  const uint4* x = static_cast<const uint4*>(p.t.x);
  const uint4* b = static_cast<const uint4*>(p.t.b);
  uint4* h = static_cast<uint4*>(p.t.h);
  uint4* y = static_cast<uint4*>(p.t.y);
  bool own[V];
#pragma unroll
  for (int k = 0; k < V; ++k) own[k] = sub + k * lanes < p.C8;
  grid_dependency_wait();
  // (a warp's teams go on together: its first row decides)
  int row = BLOCK ? blockIdx.x : blockIdx.x * per_block + threadIdx.x / lanes;
  const int ahead = BLOCK ? 0 : (threadIdx.x & 31) / lanes;
  uint4 xn[V], bn[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    xn[k] = bn[k] = make_uint4(0u, 0u, 0u, 0u);
    if (row < p.rows && own[k]) {
      xn[k] = x[(int64_t)row * p.C8 + sub + k * lanes];
      bn[k] = b[(int64_t)row * p.C8 + sub + k * lanes];
    }
  }
  for (; row - ahead < p.rows; row += step) {
    const bool there = row < p.rows;
    float bv[V][8], hv[V][8];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      unpack8(bn[k], bv[k]);
      unpack8(xn[k], hv[k]);
    }
    const int64_t next = (int64_t)row + step;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      xn[k] = bn[k] = make_uint4(0u, 0u, 0u, 0u);
      if (next < p.rows && own[k]) {
        xn[k] = x[next * p.C8 + sub + k * lanes];
        bn[k] = b[next * p.C8 + sub + k * lanes];
      }
    }
    float4 stats = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (POST) row_statistics(bv, own, p.post_layer, inv_c, p.eps, sum, stats.x, stats.y);
    const float* gate = p.t.gate;
    if (gate != nullptr && p.rows_per_gate > 0 && there) gate += (int64_t)(row / p.rows_per_gate) * (8 * p.C8);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int piece = sub + k * lanes;
      float g[8];
      params8(gate, piece, own[k], 1.0f, g);
      if (POST) {
        float a[8], c[8];
        params8(p.t.post_gamma, piece, own[k], 1.0f, a);
        params8(p.t.post_beta, piece, own[k], 0.0f, c);
#pragma unroll
        for (int j = 0; j < 8; ++j) bv[k][j] = fmaf((bv[k][j] - stats.x) * stats.y, a[j], c[j]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) hv[k][j] = own[k] ? fmaf(g[j], bv[k][j], p.scale * hv[k][j]) : 0.0f;
      if (there && own[k] && h != nullptr) h[(int64_t)row * p.C8 + piece] = pack8(hv[k]);
    }
    if (PRE) {
      row_statistics(hv, own, p.pre_layer, inv_c, p.eps, sum, stats.z, stats.w);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int piece = sub + k * lanes;
        float a[8], c[8];
        params8(p.t.pre_gamma, piece, own[k], 1.0f, a);
        params8(p.t.pre_beta, piece, own[k], 0.0f, c);
#pragma unroll
        for (int j = 0; j < 8; ++j) hv[k][j] = fmaf((hv[k][j] - stats.z) * stats.w, a[j], c[j]);
        if (there && own[k]) y[(int64_t)row * p.C8 + piece] = pack8(hv[k]);
      }
    }
    if (p.t.stats != nullptr && there && sub == 0) reinterpret_cast<float4*>(p.t.stats)[row] = stats;
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
  int C8, lanes;
  int post_layer, pre_layer, image_gates;
  float scale;
  float* block_sums;          // [blocks][kSums][C]
  float* unit_sums;           // [units][C]
};

template <int V, bool BLOCK, bool POST, bool PRE>
__global__ void __launch_bounds__(BLOCK ? 512 : 256) resnorm_backward_kernel(const BackwardParams p) {
  extern __shared__ float rows_of_warps[];  // [warps][C], of warp crews
  __shared__ float scratch[64];
  grid_launch_dependents();
  const int lanes = BLOCK ? blockDim.x : p.lanes;
  const int sub = BLOCK ? threadIdx.x : threadIdx.x & (lanes - 1);
  const int teams = BLOCK ? 1 : 32 / lanes, team = BLOCK ? 0 : (threadIdx.x & 31) / lanes;
  const int crews_per_block = BLOCK ? 1 : blockDim.x >> 5;
  const int crew = blockIdx.x * crews_per_block + (BLOCK ? 0 : threadIdx.x >> 5);
  const int crews = gridDim.x * crews_per_block;
  const int C = 8 * p.C8;
  const float inv_c = 1.0f / (float)C;
  TeamSum<BLOCK> sum{scratch, lanes};
  const uint4* x = static_cast<const uint4*>(p.t.x);
  const uint4* b = static_cast<const uint4*>(p.t.b);
  const uint4* dh = static_cast<const uint4*>(p.g.dh);
  const uint4* dy = static_cast<const uint4*>(p.g.dy);
  uint4* dx = static_cast<uint4*>(p.g.dx);
  uint4* db = static_cast<uint4*>(p.g.db);
  bool own[V];
#pragma unroll
  for (int k = 0; k < V; ++k) own[k] = sub + k * lanes < p.C8;
  float acc[kSums][V][8];
#pragma unroll
  for (int a = 0; a < kSums; ++a)
#pragma unroll
    for (int k = 0; k < V; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[a][k][j] = 0.0f;
  grid_dependency_wait();

  for (int u = crew; u < p.units; u += crews) {
    const int image = u / p.units_per_gate;
    const int64_t image_end = min((int64_t)p.rows, (int64_t)(image + 1) * p.gate_rows);
    const int64_t first = (int64_t)image * p.gate_rows + (int64_t)(u - image * p.units_per_gate) * p.unit_rows;
    const int64_t end = min(image_end, first + p.unit_rows);
    const float* gate = p.t.gate;
    if (gate != nullptr && p.image_gates) gate += (int64_t)image * C;
    for (int64_t r0 = first; r0 < end; r0 += teams) {
      const int64_t row = r0 + team;
      const bool there = row < end;
      float4 stats = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if ((POST || PRE) && there) stats = reinterpret_cast<const float4*>(p.t.stats)[row];
      uint4 xr[V], br[V], hr[V], yr[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        xr[k] = br[k] = hr[k] = yr[k] = make_uint4(0u, 0u, 0u, 0u);
        if (there && own[k]) {
          const int64_t at = row * p.C8 + sub + k * lanes;
          br[k] = b[at];
          if (PRE) {
            xr[k] = x[at];
            yr[k] = dy[at];
          }
          if (dh != nullptr) hr[k] = dh[at];
        }
      }
      float d[V][8], hat[V][8], pv[V][8];  // pv: bhat with a first norm, else b itself
      float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int piece = sub + k * lanes;
        unpack8(br[k], pv[k]);
        unpack8(hr[k], d[k]);
        if (POST) {
#pragma unroll
          for (int j = 0; j < 8; ++j) pv[k][j] = (pv[k][j] - stats.x) * stats.y;
        }
        if (PRE) {
          float gv[8], a[8], c[8], g[8];
          unpack8(xr[k], hat[k]);
          unpack8(yr[k], gv);
          params8(gate, piece, own[k], 1.0f, g);
          params8(p.t.post_gamma, piece, POST && own[k], 1.0f, a);
          params8(p.t.post_beta, piece, POST && own[k], 0.0f, c);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float pj = POST ? fmaf(pv[k][j], a[j], c[j]) : pv[k][j];
            hat[k][j] = (fmaf(g[j], pj, p.scale * hat[k][j]) - stats.z) * stats.w;
            acc[kPreGamma][k][j] = fmaf(gv[j], hat[k][j], acc[kPreGamma][k][j]);
            acc[kPreBeta][k][j] += gv[j];
          }
          params8(p.t.pre_gamma, piece, own[k], 1.0f, a);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float q = gv[j] * a[j];
            s1 += q;
            s2 = fmaf(q, hat[k][j], s2);
          }
        }
      }
      if (PRE) {
        sum(s1, s2);
        s1 = p.pre_layer ? s1 * inv_c : 0.0f;
        s2 *= inv_c;
      }
      float t1 = 0.0f, t2 = 0.0f;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int piece = sub + k * lanes;
        float a[8], c[8], g[8];
        if (PRE) {
          float gv[8];
          unpack8(yr[k], gv);
          params8(p.t.pre_gamma, piece, own[k], 1.0f, a);
#pragma unroll
          for (int j = 0; j < 8; ++j) d[k][j] += stats.w * (gv[j] * a[j] - s1 - hat[k][j] * s2);
        }
        if (there && own[k] && dx != nullptr) {
          float o[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = p.scale * d[k][j];
          dx[row * p.C8 + piece] = pack8(o);
        }
        params8(gate, piece, own[k], 1.0f, g);
        params8(p.t.post_gamma, piece, POST && own[k], 1.0f, a);
        params8(p.t.post_beta, piece, POST && own[k], 0.0f, c);
        if (there && own[k]) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float pj = POST ? fmaf(pv[k][j], a[j], c[j]) : pv[k][j];
            acc[kGate][k][j] = fmaf(d[k][j], pj, acc[kGate][k][j]);
            d[k][j] *= g[j];  // dp from here on
            if (POST) {
              acc[kPostGamma][k][j] = fmaf(d[k][j], pv[k][j], acc[kPostGamma][k][j]);
              acc[kPostBeta][k][j] += d[k][j];
              d[k][j] *= a[j];
              t1 += d[k][j];
              t2 = fmaf(d[k][j], pv[k][j], t2);
            }
          }
        }
      }
      if (POST) {
        sum(t1, t2);
        t1 = p.post_layer ? t1 * inv_c : 0.0f;
        t2 *= inv_c;
      }
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (POST) {
#pragma unroll
          for (int j = 0; j < 8; ++j) d[k][j] = stats.y * (d[k][j] - t1 - pv[k][j] * t2);
        }
        if (there && own[k] && db != nullptr) db[row * p.C8 + sub + k * lanes] = pack8(d[k]);
      }
    }
    if (p.image_gates && p.g.dgate != nullptr) {
      float* out = p.units_per_gate == 1 ? p.g.dgate + (int64_t)image * C : p.unit_sums + (int64_t)u * C;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (!BLOCK)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            for (int o = 16; o >= lanes; o >>= 1) acc[kGate][k][j] += __shfl_xor_sync(0xFFFFFFFFu, acc[kGate][k][j], o);
        if (own[k] && team == 0) {
          float4* w = reinterpret_cast<float4*>(out) + 2 * (sub + k * lanes);
          w[0] = make_float4(acc[kGate][k][0], acc[kGate][k][1], acc[kGate][k][2], acc[kGate][k][3]);
          w[1] = make_float4(acc[kGate][k][4], acc[kGate][k][5], acc[kGate][k][6], acc[kGate][k][7]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[kGate][k][j] = 0.0f;
      }
    }
  }

  // What is left in the registers, summed over the block's warps and teams.
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
      if (!BLOCK)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          for (int o = 16; o >= lanes; o >>= 1) acc[a][k][j] += __shfl_xor_sync(0xFFFFFFFFu, acc[a][k][j], o);
      if (own[k] && team == 0) {
        float4* w = reinterpret_cast<float4*>(out) + 2 * (sub + k * lanes);
        w[0] = make_float4(acc[a][k][0], acc[a][k][1], acc[a][k][2], acc[a][k][3]);
        w[1] = make_float4(acc[a][k][4], acc[a][k][5], acc[a][k][6], acc[a][k][7]);
      }
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
  float* out[kSums];          // (nullptr: not wanted)
  int blocks, C;
  int images, units_per_gate; // of gates per image whose units were several (0 images: none)
  float* dgate;
};
// 32 columns x 32 rows of threads: column sums of one kind over the blocks, or of one image's units.
__global__ void __launch_bounds__(1024) resnorm_finish_kernel(const FinishParams p) {
  __shared__ float part[32][33];
  grid_launch_dependents();
  grid_dependency_wait();
  const int groups = (p.C + 31) / 32;
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int col = (blockIdx.x % groups) * 32 + tx;
  const int job = blockIdx.x / groups;
  const float* in;
  float* out;
  int n;
  int64_t pitch;
  if (job < kSums) {
    in = p.block_sums + (int64_t)job * p.C;
    out = p.out[job];
    n = p.blocks;
    pitch = (int64_t)kSums * p.C;
  } else {
    const int image = job - kSums;
    in = p.unit_sums + (int64_t)image * p.units_per_gate * p.C;
    out = p.dgate + (int64_t)image * p.C;
    n = p.units_per_gate;
    pitch = p.C;
  }
  if (out == nullptr) return;
  float s = 0.0f;
  if (col < p.C) {
#pragma unroll 4
    for (int r = ty; r < n; r += 32) s += in[r * pitch + col];
  }
  part[ty][tx] = s;
  __syncthreads();
  s = part[tx][ty];  // column ty of the group, row tx of the partial sums
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_down_sync(0xFFFFFFFFu, s, o);
  const int c = (blockIdx.x % groups) * 32 + ty;
  if (tx == 0 && c < p.C) out[c] = s;
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
// Up to `warp_pieces` pieces per lane a row is part of a warp, else a block's.
Team team_for(int C8, int warp_pieces) {
  if (C8 <= 32) return {false, 1, power_of_two_from(C8), 256};
  if (C8 <= 32 * warp_pieces) return {false, (C8 + 31) / 32, 32, 256};
  const int V = C8 <= 512 ? 1 : 2;
  const int threads = (((C8 + V - 1) / V) + 31) / 32 * 32;
  return {true, V, threads, threads};
}

template <bool POST, bool PRE>
void (*forward_kernel(const Team& t))(ForwardParams) {
  if (t.block) return t.V == 1 ? resnorm_kernel<1, true, POST, PRE> : resnorm_kernel<2, true, POST, PRE>;
  return t.V == 1   ? resnorm_kernel<1, false, POST, PRE>
         : t.V == 2 ? resnorm_kernel<2, false, POST, PRE>
         : t.V == 3 ? resnorm_kernel<3, false, POST, PRE>
                    : resnorm_kernel<4, false, POST, PRE>;
}
template <bool POST, bool PRE>
void (*backward_kernel(const Team& t))(BackwardParams) {
  if (t.block) return t.V == 1 ? resnorm_backward_kernel<1, true, POST, PRE> : resnorm_backward_kernel<2, true, POST, PRE>;
  return t.V == 1 ? resnorm_backward_kernel<1, false, POST, PRE> : resnorm_backward_kernel<2, false, POST, PRE>;
}

// How the backward pass is cut: units, and blocks (the scratch is sized by them).
struct Cut {
  Team team;
  int units, unit_rows, units_per_gate, gate_rows, blocks, images;
  bool image_gates;
};
constexpr int kBackwardWarps = 16;       // per SM, of crews at work at once
constexpr int kRowsPerTeam = 4;          // of a unit, at least: its sums are written once

Cut cut_backward(const ssconv_resnorm_t& d) {
  Cut c;
  c.team = team_for(d.C / 8, 2);
  c.image_gates = d.rows_per_gate > 0;
  const int64_t rows = d.rows;
  c.gate_rows = (int)(c.image_gates && d.rows_per_gate < rows ? d.rows_per_gate : rows);
  c.images = (int)((rows + c.gate_rows - 1) / c.gate_rows);
  const int crew_warps = c.team.block ? c.team.threads / 32 : 1;
  const int teams = c.team.block ? 1 : 32 / c.team.lanes;
  const int crews_per_block = c.team.block ? 1 : c.team.threads / 32;
  const int64_t most = (int64_t)device_sms() * (kBackwardWarps / crew_warps > 0 ? kBackwardWarps / crew_warps : 1);
  int64_t per_gate = (most + c.images - 1) / c.images;
  const int64_t worth = (c.gate_rows + teams * kRowsPerTeam - 1) / (teams * kRowsPerTeam);
  if (per_gate > worth) per_gate = worth;
  c.unit_rows = (int)((c.gate_rows + per_gate - 1) / per_gate);
  c.units_per_gate = (c.gate_rows + c.unit_rows - 1) / c.unit_rows;
  c.units = c.images * c.units_per_gate;
  const int64_t crews = c.units < most ? c.units : most;
  c.blocks = (int)((crews + crews_per_block - 1) / crews_per_block);
  return c;
}

}  // namespace

cudaError_t launch_resnorm(const ssconv_resnorm_t& d, const ResnormTensors& t, cudaStream_t st) {
  const int C8 = d.C / 8;
  const Team team = team_for(C8, 4);
  ForwardParams p = {t, (int)d.rows, d.rows_per_gate < d.rows ? (int)d.rows_per_gate : (int)d.rows, C8, team.lanes,
                     d.post == SSCONV_NORM_LAYER, d.pre == SSCONV_NORM_LAYER, d.scale, d.eps};
  const bool post = d.post != SSCONV_NORM_NONE, pre = d.pre != SSCONV_NORM_NONE && t.y != nullptr;
  const auto kernel = post ? (pre ? forward_kernel<true, true>(team) : forward_kernel<true, false>(team))
                           : (pre ? forward_kernel<false, true>(team) : forward_kernel<false, false>(team));
  const int per_block = team.block ? 1 : team.threads / team.lanes;
  const int64_t blocks = (d.rows + per_block - 1) / per_block;
  const int64_t most = (int64_t)device_sms() * (team.block ? 1024 / team.threads : 4);
  count_launch();
  return launch_dependent(kernel, (unsigned)(blocks < most ? blocks : most), team.threads, st, p);
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
  p.lanes = c.team.lanes;
  p.post_layer = d.post == SSCONV_NORM_LAYER;
  p.pre_layer = d.pre == SSCONV_NORM_LAYER;
  p.image_gates = c.image_gates;
  p.scale = d.scale;
  p.block_sums = ws;
  p.unit_sums = ws + (size_t)c.blocks * kSums * d.C;
  const bool post = d.post != SSCONV_NORM_NONE, pre = d.pre != SSCONV_NORM_NONE;
  const auto kernel = post ? (pre ? backward_kernel<true, true>(c.team) : backward_kernel<true, false>(c.team))
                           : (pre ? backward_kernel<false, true>(c.team) : backward_kernel<false, false>(c.team));
  const size_t smem = c.team.block ? 0 : (size_t)(c.team.threads / 32) * d.C * sizeof(float);
  count_launch();
  cudaError_t e = launch_dependent_smem(kernel, (unsigned)c.blocks, c.team.threads, smem, st, p);
  if (e != cudaSuccess) return e;

  FinishParams f = {};
  f.block_sums = p.block_sums;
  f.unit_sums = p.unit_sums;
  bool any = false;
  for (int i = 0; i < kSums; ++i) {
    f.out[i] = i == kGate && c.image_gates ? nullptr : sums[i];
    any = any || f.out[i] != nullptr;
  }
  f.blocks = c.blocks;
  f.C = d.C;
  f.units_per_gate = c.units_per_gate;
  f.images = c.image_gates && c.units_per_gate > 1 && g.dgate != nullptr ? c.images : 0;
  f.dgate = g.dgate;
  if (!any && f.images == 0) return cudaSuccess;
  count_launch();
  return launch_dependent(resnorm_finish_kernel, (unsigned)((d.C + 31) / 32 * (kSums + f.images)), 1024, st, f);
}

}  // namespace ssconv
