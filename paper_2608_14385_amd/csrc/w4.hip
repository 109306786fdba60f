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

// The matrix and the token rows of row tile `tile`, the tiles of `rows` rows
// counted over the matrices in order.  False past the last.
__device__ inline bool find_tile(const W4Args &a, int tile, int rows, int &e, int &m0, int &m1) {
  if (!a.offset) {
    e = 0;
    m0 = tile * rows;
    m1 = min(m0 + rows, a.M);
    return m0 < a.M;
  }
  __shared__ int s_sum[kWaves], s_found[3];
  __syncthreads();   // an earlier tile's s_found has been read
  const int tid = threadIdx.x, lane = tid % kWave, wv = tid / kWave;
  if (tid == 0) s_found[0] = -1;
  int base = 0;
  for (int e0 = 0; e0 < a.n && base <= tile; e0 += kThreads) {
    int lo = 0, hi = 0;
    if (e0 + tid < a.n) expert_rows(a, e0 + tid, lo, hi);
    const int mine = (hi - lo + rows - 1) / rows;
    int inc = mine;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int o = __shfl_up(inc, d);
      inc += lane >= d ? o : 0;
    }
    __syncthreads();
    if (lane == kWave - 1) s_sum[wv] = inc;
    __syncthreads();
    int at = base + inc - mine;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      at += i < wv ? s_sum[i] : 0;
      base += s_sum[i];
    }
    if (at <= tile && tile < at + mine) {
      s_found[0] = e0 + tid;
      s_found[1] = lo + (tile - at) * rows;
      s_found[2] = hi;
    }
  }
  __syncthreads();
  e = s_found[0];
  m0 = s_found[1];
  m1 = min(m0 + rows, s_found[2]);
  return e >= 0;
}

__device__ inline float silu(float v) { return v / (1.0f + __expf(-v)); }

// One wave: 16 token rows by 16 weight rows, over all columns.
template <int MATS>
__device__ inline void tile_product(const W4Args &a, int e, int m0, int m1, int r0) {
  const int lane = lane_id(), j = lane & 15, g = lane >> 4;
  const int r = min(r0 + j, a.R - 1), groups = a.K / a.group;
  const char *x = static_cast<const char *>(a.x) + ((size_t)min(m0 + j, m1 - 1) * a.K + g * 8) * 2;
  const size_t wrow = (size_t)e * a.R + r;
  f32x4 acc[MATS] = {};
  for (int q = 0; q < groups; ++q) {
    f32x4 part[MATS];
    f32x4 c0 = {0.f, 0.f, 0.f, 0.f};
    for (int k = q * a.group; k < (q + 1) * a.group; k += 32)
      c0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          order_columns(*reinterpret_cast<const u32x4 *>(x + k * 2)), minus_24(), c0, 0, 0, 0);
    for (int n = 0; n < MATS; ++n) {
      part[n] = c0;
      for (int k = q * a.group; k < (q + 1) * a.group; k += 32) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(
            static_cast<const char *>(a.w[n]) + (wrow * a.K + k) / 2 + g * 4);
        part[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            order_columns(*reinterpret_cast<const u32x4 *>(x + k * 2)), codes_to_bf16(w), part[n],
            0, 0, 0);
      }
      acc[n] += scale_at(a.scale[n], wrow * groups + q, a.scale_bf16) * part[n];
    }
  }
  // lane (j, g) holds weight row r0 + j of tokens m0 + 4 g .. + 3
  if (r0 + j >= a.R) return;
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + g * 4 + i;
    if (m >= m1) break;
    const float v = MATS == 2 ? silu(acc[0][i]) * acc[MATS - 1][i] : acc[0][i];
    static_cast<uint16_t *>(a.y)[(size_t)m * a.R + r0 + j] = f32_to_bf16(v);
  }
}

}  // namespace

template <int MATS>
__global__ __launch_bounds__(kThreads) void w4_kernel(W4Args a, int64_t items) {
  const int rt = (a.R + kTile * kWaves - 1) / (kTile * kWaves);
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    int e, m0, m1;
    if (!find_tile(a, (int)(item / rt), kTile, e, m0, m1)) return;
    const int r0 = ((int)(item % rt) * kWaves + threadIdx.x / kWave) * kTile;
    if (r0 < a.R) tile_product<MATS>(a, e, m0, m1, r0);
  }
}

hipError_t launch_w4(const W4Args &a, int mats, hipStream_t s) {
  const int64_t tiles = a.M / kTile + (a.offset ? (a.n < a.M ? a.n : a.M) : 1);   // the most there can be
  const int64_t items = tiles * ((a.R + kTile * kWaves - 1) / (kTile * kWaves));
  const dim3 grid((unsigned)(items < (1 << 20) ? items : 1 << 20));
  if (mats == 2) hipLaunchKernelGGL(w4_kernel<2>, grid, dim3(kThreads), 0, s, a, items);
  else hipLaunchKernelGGL(w4_kernel<1>, grid, dim3(kThreads), 0, s, a, items);
  return hipGetLastError();
}

}  // namespace deamoe
