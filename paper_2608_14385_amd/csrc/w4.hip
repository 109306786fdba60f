// Products with 4-bit weights and group scales, for one matrix or for the
// experts' matrices over rows sorted by expert.
//
//   y[m, r] = sum over groups G of scale[r, G] * sum over c in G of (q[r, c] - 8) x[m, c]
//
// A code becomes a bf16 number with two integer instructions for a pair: put
// into mantissa bits 3 to 6 of 16.0 it reads 16 + q, exactly.  The matrix cores
// take these, and a second product with -24 everywhere, shared by all weight
// rows, starts each group's sum at -24 * sum(x): together sum((q - 8) x) in
// fp32, without rounding a weight.  |16 + q| and 24 are a few times |q - 8|,
// which costs the sum about three of fp32's 24 bits.
#include "ops.h"

namespace deamoe {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// Eight codes (columns c .. c + 7, low bits first) as 16 + q, in the order
// 0 4 1 5 2 6 3 7 ...
__device__ inline bf16x8 codes_to_bf16(uint32_t w) {
  const u32x4 r = {((w << 3) & 0x00780078u) | 0x41804180u, ((w >> 1) & 0x00780078u) | 0x41804180u,
                   ((w >> 5) & 0x00780078u) | 0x41804180u, ((w >> 9) & 0x00780078u) | 0x41804180u};
  return __builtin_bit_cast(bf16x8, r);
}

// ... and eight columns of x in the same order.
__device__ inline bf16x8 order_columns(u32x4 v) {
  const u32x4 r = {__builtin_amdgcn_perm(v[2], v[0], 0x05040100u),
                   __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
                   __builtin_amdgcn_perm(v[3], v[1], 0x05040100u),
                   __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
  return __builtin_bit_cast(bf16x8, r);
}

__device__ inline bf16x8 minus_24() {
  const u32x4 r = {0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u};
  return __builtin_bit_cast(bf16x8, r);
}

__device__ inline float scale_at(const void *p, size_t i, int bf16) {
  return bf16 ? bf16_to_f32(static_cast<const uint16_t *>(p)[i]) : static_cast<const float *>(p)[i];
}

// Rows [lo, hi) of matrix e, with every offset kept within [0, M].
__device__ inline void expert_rows(const W4Args &a, int e, int &lo, int &hi) {
  lo = min(max(a.offset[e], 0), a.M);
  hi = min(max(a.offset[e + 1], lo), a.M);
}

// The matrix e and the token rows [m0, m1) of tile `tile`, the tiles of `rows`
// rows counted over the matrices in order.  False past the last.  Every wave
// finds its tile by itself, with no barrier: a lane counts the tiles of a run
// of matrices.
__device__ inline bool find_tile(const W4Args &a, int64_t tile, int rows, int &e, int &m0,
                                 int &m1) {
  if (!a.offset) {
    e = 0;
    if (tile * rows >= a.M) return false;
    m0 = (int)tile * rows;
    m1 = min(m0 + rows, a.M);
    return true;
  }
  const int lane = lane_id(), per = (a.n + kWave - 1) / kWave, e0 = min(lane * per, a.n);
  const int e1 = min(e0 + per, a.n);
  int mine = 0;
  for (int i = e0; i < e1; ++i) {
    int lo, hi;
    expert_rows(a, i, lo, hi);
    mine += (hi - lo + rows - 1) / rows;
  }
  int inc = mine;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int o = __shfl_up(inc, d);
    inc += lane >= d ? o : 0;
  }
  const uint64_t past = __ballot(inc > tile);
  if (!past) return false;
  const int from = __ffsll((unsigned long long)past) - 1;   // the lane whose run holds the tile
  int at = __builtin_amdgcn_readlane(inc - mine, from);
  const int f0 = min(from * per, a.n), f1 = min(f0 + per, a.n);
  for (int i = f0; i < f1; ++i) {
    int lo, hi;
    expert_rows(a, i, lo, hi);
    const int t = (hi - lo + rows - 1) / rows;
    if (tile < at + t) {
      e = i;
      m0 = lo + ((int)tile - at) * rows;
      m1 = min(m0 + rows, hi);
      return true;
    }
    at += t;
  }
  return false;   // not reached
}

__device__ inline float silu(float v) { return v / (1.0f + __expf(-v)); }

typedef __bf16 bf16;

// Code dwords of 128 columns as loaded (dword m of lane group g: columns
// 32 g + 8 m ...) -> dword m of lane group g: columns 32 m + 8 g ..., so that
// one matrix product covers 32 columns that share a scale.
__device__ inline void columns_together(u32x4 &v) {
  auto s0 = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
  auto s1 = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
  auto t0 = __builtin_amdgcn_permlane16_swap(s0[0], s1[0], false, false);
  auto t1 = __builtin_amdgcn_permlane16_swap(s0[1], s1[1], false, false);
  v = u32x4{t0[0], t0[1], t1[0], t1[1]};
}

}  // namespace

// Few token rows: the weights are streamed, each byte once per 16 * NTT rows.
// A wave takes NR 16-row tiles of each matrix and every KS-th step of SC
// columns; the loads of a step are requested together, a step ahead of its
// products, straight into registers in operand order (16 rows of whole cache
// lines).  Waves that share tiles add their sums over LDS at the end.
template <int MATS, int NR, int NTT, int G32>
__global__ __launch_bounds__(kThreads) void w4_stream_kernel(W4Args a, int64_t items, int ks) {
  constexpr int SC = NTT > 2 ? 128 : 256, CH = SC / 128;   // columns of a step, 128 at a time
  constexpr int NT = MATS * NR, SG = SC / 32 / G32;        // weight tiles, scales of a row
  __shared__ f32x4 s_red[kWaves][NT][NTT][kWave];
  const int lane = lane_id(), j = lane & 15, g = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int parts = kWaves / ks, kp = wv % ks;   // row parts of the workgroup, this wave's K part
  const int rows = parts * NR * kTile, rt = (a.R + rows - 1) / rows;
  const int steps = (a.K + SC - 1) / SC, groups = a.K / (32 * G32);
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    int e, m0, m1;
    if (!find_tile(a, item / rt, kTile * NTT, e, m0, m1)) return;
    const int r0 = (int)(item % rt) * rows + (wv / ks) * NR * kTile;
    const char *wp[NT];
    size_t sp[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const size_t r = (size_t)e * a.R + min(r0 + (n % NR) * kTile + j, a.R - 1);
      wp[n] = static_cast<const char *>(a.w[n / NR]) + r * (a.K / 2) + g * 16;
      sp[n] = r * groups;
    }
    const char *xp[NTT];
#pragma unroll
    for (int t = 0; t < NTT; ++t)
      xp[t] = static_cast<const char *>(a.x) +
              ((size_t)min(m0 + t * kTile + j, m1 - 1) * a.K + g * 8) * 2;
    u32x4 W[2][NT][CH], X[2][NTT][CH * 4];
    float S[2][NT][SG];
    auto request = [&](int q, int s) {
      const int k0 = s * SC;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int k = k0 + c * 128;   // past the end: any codes, their x is 0
          W[q][n][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(
              wp[n] + (k + g * 32 < a.K ? k / 2 : -g * 16)));
        }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < SG; ++i) {
          const int q0 = s * SG + i;
          S[q][n][i] = q0 < groups ? scale_at(a.scale[n / NR], sp[n] + q0, a.scale_bf16) : 0.f;
        }
#pragma unroll
      for (int t = 0; t < NTT; ++t)
#pragma unroll
        for (int b = 0; b < CH * 4; ++b) {
          const int k = k0 + b * 32;
          X[q][t][b] = u32x4{0, 0, 0, 0};
          if (k < a.K) X[q][t][b] = *reinterpret_cast<const u32x4 *>(xp[t] + (size_t)k * 2);
        }
    };
    f32x4 acc[NT][NTT] = {};
    auto multiply = [&](int q) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        bf16x8 xb[NTT][4];
#pragma unroll
        for (int t = 0; t < NTT; ++t)
#pragma unroll
          for (int m = 0; m < 4; ++m) xb[t][m] = order_columns(X[q][t][c * 4 + m]);
        f32x4 start[NTT][4 / G32];   // -24 sum(x) of every group
#pragma unroll
        for (int t = 0; t < NTT; ++t)
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            start[t][m / G32] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                xb[t][m], minus_24(), m % G32 ? start[t][m / G32] : zero, 0, 0, 0);
          }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          columns_together(W[q][n][c]);
          bf16x8 wb[4];
#pragma unroll
          for (int m = 0; m < 4; ++m) wb[m] = codes_to_bf16(W[q][n][c][m]);
#pragma unroll
          for (int t = 0; t < NTT; ++t)
#pragma unroll
            for (int i = 0; i < 4 / G32; ++i) {
              f32x4 p = start[t][i];
#pragma unroll
              for (int m = 0; m < G32; ++m)
                p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xb[t][i * G32 + m], wb[i * G32 + m], p,
                                                            0, 0, 0);
              acc[n][t] += S[q][n][c * (4 / G32) + i] * p;
            }
        }
      }
    };
    if (kp < steps) request(0, kp);
    for (int s = kp; s < steps; s += 2 * ks) {
      if (s + ks < steps) request(1, s + ks);
      multiply(0);
      if (s + ks >= steps) break;
      if (s + 2 * ks < steps) request(0, s + 2 * ks);
      multiply(1);
    }
    if (ks > 1) {
      __syncthreads();   // the previous item's sums have been read
      if (kp)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int t = 0; t < NTT; ++t) s_red[wv][n][t][lane] = acc[n][t];
      __syncthreads();
      if (kp) continue;
      for (int i = 1; i < ks; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int t = 0; t < NTT; ++t) acc[n][t] += s_red[wv + i][n][t][lane];
    }
    // lane (j, g) holds weight row j of its tile for tokens 4 g .. 4 g + 3
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = r0 + n * kTile + j;
#pragma unroll
      for (int t = 0; t < NTT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int m = m0 + t * kTile + g * 4 + i;
          const float v = MATS == 2 ? silu(acc[n][t][i]) * acc[NT - NR + n][t][i] : acc[n][t][i];
          if (r < a.R && m < m1)
            reinterpret_cast<bf16 *>(a.y)[(size_t)m * a.R + r] = (bf16)v;
        }
    }
  }
}

namespace {

template <int MATS, int NR, int NTT>
hipError_t stream_grouped(const W4Args &a, int ks, hipStream_t s) {
  const int tr = kTile * NTT, rows = kWaves / ks * NR * kTile;
  const int64_t tiles = a.offset ? a.M / tr + (a.n < a.M ? a.n : a.M) : (a.M + tr - 1) / tr;
  const int64_t items = tiles * ((a.R + rows - 1) / rows);   // the most there can be
  const dim3 grid((unsigned)(items < (1 << 20) ? items : 1 << 20)), block(kThreads);
  if (a.group == 32)
    hipLaunchKernelGGL((w4_stream_kernel<MATS, NR, NTT, 1>), grid, block, 0, s, a, items, ks);
  else if (a.group == 64)
    hipLaunchKernelGGL((w4_stream_kernel<MATS, NR, NTT, 2>), grid, block, 0, s, a, items, ks);
  else
    hipLaunchKernelGGL((w4_stream_kernel<MATS, NR, NTT, 4>), grid, block, 0, s, a, items, ks);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_w4(const W4Args &a, int mats, hipStream_t s) {
  const int per = a.offset ? (a.M + a.n - 1) / a.n : a.M;   // rows of a matrix on average
  if (mats == 2) return per <= 16 ? stream_grouped<2, 1, 1>(a, 4, s) : stream_grouped<2, 1, 2>(a, 4, s);
  return per <= 16 ? stream_grouped<1, 1, 1>(a, 4, s) : stream_grouped<1, 1, 4>(a, 4, s);
}

}  // namespace deamoe
