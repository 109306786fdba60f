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
#include "gemm_tile.h"
#include "ops.h"

namespace deamoe {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// The two constants stand in vector registers: an and-or takes them in one
// instruction there, as literals it would be two.
struct Magic {
  uint32_t mask = 0x00780078u, one = 0x41804180u;
  __device__ Magic() { asm("" : "+v"(mask), "+v"(one)); }
};

// Eight codes (columns c .. c + 7, low bits first) as 16 + q, in the order
// 0 4 1 5 2 6 3 7 ...
__device__ inline bf16x8 codes_to_bf16(uint32_t w, const Magic &k) {
  const u32x4 r = {((w << 3) & k.mask) | k.one, ((w >> 1) & k.mask) | k.one,
                   ((w >> 5) & k.mask) | k.one, ((w >> 9) & k.mask) | k.one};
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

// The matrix e and the token rows [m0, m1) of tile `tile`, the tiles of `rows`
// rows counted over the matrices in order.  False past the last.  Every wave
// finds its tile by itself, with no barrier: a lane counts the tiles of a run
// of matrices.  Offsets outside [0, M] count as the nearer end.
__device__ inline bool find_tile(const W4Args &a, int64_t tile, int rows, int &e, int &m0,
                                 int &m1) {
  if (!a.offset) {
    e = 0;
    if (tile * rows >= a.M) return false;
    m0 = (int)tile * rows;
    m1 = min(m0 + rows, a.M);
    return true;
  }
  const int lane = lane_id(), per = (a.n + kWave - 1) / kWave, e0 = lane * per;
  constexpr int U = 4;   // offsets read at once
  int mine = 0;
  for (int i = 0; i < per; i += U) {
    int o[U + 1];
#pragma unroll
    for (int u = 0; u <= U; ++u) o[u] = min(max(a.offset[min(e0 + min(i + u, per), a.n)], 0), a.M);
#pragma unroll
    for (int u = 0; u < U; ++u) mine += (max(o[u + 1] - o[u], 0) + rows - 1) / rows;
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
  // the lanes look at the matrices of that run, 64 at most (DEAMOE_MAX_EXPERTS / 64 are fewer)
  const int base = __builtin_amdgcn_readlane(inc - mine, from), f = from * per + lane;
  const int lo = min(max(a.offset[min(f, a.n)], 0), a.M);
  const int hi = max(min(max(a.offset[min(f + 1, a.n)], 0), a.M), lo);
  const int here = lane < per && f < a.n ? (hi - lo + rows - 1) / rows : 0;
  inc = here;
#pragma unroll
  for (int d = 1; d < DEAMOE_MAX_EXPERTS / kWave; d *= 2) {
    const int o = __shfl_up(inc, d);
    inc += lane >= d ? o : 0;
  }
  const int at = __ffsll((unsigned long long)__ballot(base + inc > tile)) - 1;
  e = from * per + at;
  m0 = __builtin_amdgcn_readlane(lo, at) +
       ((int)tile - base - __builtin_amdgcn_readlane(inc - here, at)) * rows;
  m1 = min(m0 + rows, __builtin_amdgcn_readlane(hi, at));
  return true;
}

// A pointer every lane holds alike, in scalar registers.
template <class P>
__device__ inline P *uniform_ptr(P *p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<P *>((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 |
                               (uint32_t)uniform((int)v));
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

// Codes of 256 columns of 16 rows as loaded: a of rows 0 to 7 and b of rows 8 to
// 15, lane (j, g) holding row j % 8 and columns 128 (j / 8) + 32 g ..., so that
// each load touches 8 whole cache lines.  Afterwards lane (j, g) holds row j,
// a of the first 128 columns and b of the second: halves of 8 lanes change
// places.
__device__ inline void rows_together(u32x4 &a, u32x4 &b) {
  constexpr int kRotate8 = 0x128, kAllRows = 0xf, kUpper = 0xc, kLower = 0x3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int x = a[i], y = b[i];
    a[i] = __builtin_amdgcn_update_dpp(x, y, kRotate8, kAllRows, kUpper, false);
    b[i] = __builtin_amdgcn_update_dpp(y, x, kRotate8, kAllRows, kLower, false);
  }
}

}  // namespace

// Few token rows: the weights are streamed, each byte once per 16 * NTT rows.
// A wave takes NR 16-row tiles of each matrix and every ks-th step of 128 * CH
// columns.  The loads of a step are requested D steps ahead, straight into
// registers, each load 8 whole cache lines (halves of 16 lines streamed at 4.8
// TB/s, these at 5.6, by loads alone on 490 MB).  The token rows
// stand in LDS, a panel of columns at a time, already in the codes' order: read
// from memory by every wave they would take several times the weights'
// bandwidth, and since loads retire in order, waiting for them would wait for
// weights.  The scales of a panel's columns stand beside them, for each wave
// its tiles': read by the lanes that need them, they would touch as many cache
// lines as the weights.  Waves that share tiles add their sums over LDS at the
// end.
constexpr int kPanelWords = 16 * (1024 + 8) / 2;   // of a token tile, 4 bytes each
constexpr int kPanelScales = 32;                   // of a weight row, at most
constexpr int kNonTemporal = 2;                    // cache policy of a buffer load
template <int MATS, int NR, int NTT, int G32, bool SBF, int D, int CH>
__global__ __launch_bounds__(kThreads, 2) void w4_stream_kernel(W4Args a, int64_t items, int ks) {
  constexpr int SC = 128 * CH, NT = MATS * NR, GS = 32 * G32;
  constexpr int TR = NTT * kTile, WORDS = kPanelWords * NTT;
  __shared__ __align__(16) uint32_t s_x[WORDS];
  __shared__ float s_scale[kWaves][NT][kTile][kPanelScales + 1];
  static_assert(kWaves * NT * NTT * 4 * kWave <= WORDS, "the sums of the waves");
  static_assert(CH % 2 == 0, "steps of whole cache lines");
  static_assert(D * CH * 128 <= 1024, "a panel holds a round of the ring at 16 * NTT rows");
  const int lane = lane_id(), j = lane & 15, g = lane >> 4, tid = threadIdx.x;
  const int wv = uniform(tid / kWave);
  const int kp = wv % ks, rows = kWaves / ks * NR * kTile, rt = (a.R + rows - 1) / rows;
  const int steps = (a.K + SC - 1) / SC, groups = a.K / GS;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    int e, m0, m1;
    if (!uniform(find_tile(a, item / rt, TR, e, m0, m1))) return;
    e = uniform(e), m0 = uniform(m0);
    const int ntok = uniform(m1) - m0;
    const int r0 = uniform((int)(item % rt) * rows + (wv / ks) * NR * kTile);
    // The codes are read through buffer descriptors of the matrix's rows from r0
    // on: a scalar offset moves with the step, each lane's offset stays, and
    // rows past the last read as zeros (they are never stored).  A step that
    // ends past the row's end reads the next row there, times an x of 0; a
    // request past the last step goes to an empty buffer, which reads nothing,
    // so that every iteration issues the same loads.
    const uint32_t wrow = a.K / 2;
    char *wb[MATS];
    const void *sb[MATS];
    const int left = max(a.R - r0, 1);   // a wave past the last row repeats it
    const size_t first = (size_t)e * a.R + min(r0, a.R - 1);
#pragma unroll
    for (int n = 0; n < MATS; ++n) {
      wb[n] = const_cast<char *>(uniform_ptr(static_cast<const char *>(a.w[n]) + first * wrow));
      sb[n] = uniform_ptr(static_cast<const char *>(a.scale[n]) + first * groups * (SBF ? 2 : 4));
    }
    uint32_t wo[NR][2];   // rows_together's order
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        wo[n][i] = (n * kTile + i * 8 + (j & 7)) * wrow + ((j >> 3) * 4 + g) * 16;
    u32x4 W[D][NT][CH];
    auto request = [&](int q, int s) {
      const int at = s < steps ? s * (SC / 2) : 0, bytes = s < steps ? (int)(left * wrow) : 0;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const auto buf = __builtin_amdgcn_make_buffer_rsrc(wb[n / NR], 0, bytes, 0x00027000);
#pragma unroll
        for (int c = 0; c < CH; ++c)
          W[q][n][c] =
              __builtin_amdgcn_raw_buffer_load_b128(buf, wo[n % NR][c & 1] + c / 2 * 128, at, kNonTemporal);
      }
    };
#pragma unroll
    for (int d = 0; d < D; ++d) request(d, kp + d * ks);

    // panels: whole rounds of all ring places of all K parts
    const int round = D * ks * SC, prow = min(ntok, TR);
    const int pcol = min(min(WORDS * 2 / prow - 8, a.K + round - 1), kPanelScales * GS) / round * round;
    const int ldx = pcol + 8;
    uint32_t xo[NTT];
#pragma unroll
    for (int t = 0; t < NTT; ++t) xo[t] = (min(t * kTile + j, prow - 1) * ldx + g * 8) * 2;
    f32x4 acc[NT][NTT] = {};
    const Magic magic;
    const char *lds = reinterpret_cast<const char *>(s_x);
    auto multiply = [&](int q, int k) {   // k: first column of the step in the panel
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        bf16x8 xv[NTT][4];
#pragma unroll
        for (int t = 0; t < NTT; ++t)
#pragma unroll
          for (int m = 0; m < 4; ++m)
            xv[t][m] = __builtin_bit_cast(
                bf16x8, *reinterpret_cast<const u32x4 *>(lds + xo[t] + k * 2 + c * 256 + m * 64));
        f32x4 start[NTT][4 / G32];   // -24 sum(x) of every group
#pragma unroll
        for (int t = 0; t < NTT; ++t)
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            start[t][m / G32] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                xv[t][m], minus_24(), m % G32 ? start[t][m / G32] : zero, 0, 0, 0);
          }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (c % 2 == 0) rows_together(W[q][n][c], W[q][n][c + 1]);
          columns_together(W[q][n][c]);
          bf16x8 w8[4];
#pragma unroll
          for (int m = 0; m < 4; ++m) w8[m] = codes_to_bf16(W[q][n][c][m], magic);
#pragma unroll
          for (int t = 0; t < NTT; ++t)
#pragma unroll
            for (int i = 0; i < 4 / G32; ++i) {
              f32x4 p = start[t][i];
#pragma unroll
              for (int m = 0; m < G32; ++m)
                p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv[t][i * G32 + m], w8[i * G32 + m], p,
                                                            0, 0, 0);
              acc[n][t] += s_scale[wv][n][j][k / GS + c * (4 / G32) + i] * p;
            }
        }
      }
    };
    for (int p0 = 0; p0 < a.K; p0 += pcol) {
      __syncthreads();   // the last panel, or the last item's sums, have been read
      const int q0 = p0 / GS, nq = min(groups - q0, pcol / GS);
      float sv[NT][kTile * kPanelScales / kWave];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < kTile * kPanelScales / kWave; ++i) {   // two rows at a time
          const int r = (n % NR) * kTile + i * 2 + lane / kPanelScales, q = lane % kPanelScales;
          // past the end the sums are 0, and their scale is
          const bool ok = q < nq && r < left;
          const uint32_t at = ok ? r * groups + q0 + q : 0;
          float v;
          if constexpr (SBF) v = bf16_to_f32(glob(static_cast<const uint16_t *>(sb[n / NR]))[at]);
          else v = glob(static_cast<const float *>(sb[n / NR]))[at];
          sv[n][i] = ok ? v : 0.f;
        }
      constexpr int U = 4;   // 16-byte chunks of x in flight
      const int chunks = pcol / 8, total = prow * chunks;
      for (int i0 = tid; i0 < total; i0 += U * kThreads) {
        u32x4 v[U];
        int at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + u * kThreads, r = i / chunks, k = (i - r * chunks) * 8;
          const bool ok = i < total && p0 + k < a.K;
          at[u] = i < total ? (r * ldx + k) * 2 : -1;
          v[u] = *gptr(static_cast<const char *>(a.x) + (ok ? ((size_t)(m0 + r) * a.K + p0 + k) * 2 : 0));
          if (!ok) v[u] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (at[u] >= 0)
            *reinterpret_cast<bf16x8 *>(reinterpret_cast<char *>(s_x) + at[u]) = order_columns(v[u]);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < kTile * kPanelScales / kWave; ++i)
          s_scale[wv][n][i * 2 + lane / kPanelScales][lane % kPanelScales] = sv[n][i];
      __syncthreads();
      const int end = min(p0 + pcol, a.K);
      auto steps_of_panel = [&] {
        for (int s = p0 / SC + kp;; s += D * ks)
#pragma unroll
          for (int d = 0; d < D; ++d) {
            const int at = s + d * ks;
            if (at * SC >= end) return;
            multiply(d, at * SC - p0);
            request(d, at + D * ks);
          }
      };
      steps_of_panel();
    }
    if (ks > 1) {
      f32x4(*red)[NT][NTT][kWave] = reinterpret_cast<f32x4(*)[NT][NTT][kWave]>(s_x);
      __syncthreads();   // the token rows have been read
      if (kp)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int t = 0; t < NTT; ++t) red[wv][n][t][lane] = acc[n][t];
      __syncthreads();
      if (kp) continue;
      for (int i = 1; i < ks; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int t = 0; t < NTT; ++t) acc[n][t] += red[wv + i][n][t][lane];
    }
    // lane (j, g) holds weight row j of its tile for tokens 4 g .. 4 g + 3
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = r0 + n * kTile + j;
#pragma unroll
      for (int t = 0; t < NTT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int m = t * kTile + g * 4 + i;
          const float v = MATS == 2 ? silu(acc[n][t][i]) * acc[NT - NR + n][t][i] : acc[n][t][i];
          if (r < a.R && m < ntok)
            reinterpret_cast<bf16 *>(a.y)[(size_t)(m0 + m) * a.R + r] = (bf16)v;
        }
    }
  }
}

namespace {

// K parts of a workgroup, at most `want`: a panel holds a round of the ring.
int k_parts(const W4Args &a, int ntt, int step, int want) {
  const int rows = a.M < kTile * ntt ? a.M : kTile * ntt;
  int ks = want;
  while (ks > 1 && (ks * step > kPanelScales * a.group || ks * step > kPanelWords * ntt * 2 / rows - 8))
    ks /= 2;
  return ks;
}

template <int MATS, int NR, int NTT, int D, int CH>
hipError_t stream_grouped(const W4Args &a, int want, hipStream_t s) {
  const int ks = k_parts(a, NTT, D * CH * 128, want);
  const int tr = kTile * NTT, rows = kWaves / ks * NR * kTile;
  const int64_t tiles = a.offset ? a.M / tr + (a.n < a.M ? a.n : a.M) : (a.M + tr - 1) / tr;
  const int64_t items = tiles * ((a.R + rows - 1) / rows);   // the most there can be
  const dim3 grid((unsigned)(items < (1 << 20) ? items : 1 << 20)), block(kThreads);
#define W4_STREAM(G, B)                                                                         \
  hipLaunchKernelGGL((w4_stream_kernel<MATS, NR, NTT, G, B, D, CH>), grid, block, 0, s, a, items, ks)
  if (a.scale_bf16) {
    if (a.group == 32) W4_STREAM(1, true);
    else if (a.group == 64) W4_STREAM(2, true);
    else W4_STREAM(4, true);
  } else {
    if (a.group == 32) W4_STREAM(1, false);
    else if (a.group == 64) W4_STREAM(2, false);
    else W4_STREAM(4, false);
  }
#undef W4_STREAM
  return hipGetLastError();
}

}  // namespace

hipError_t launch_w4(const W4Args &a, int mats, hipStream_t s) {
  const int per = a.offset ? (a.M + a.n - 1) / a.n : a.M;   // rows of a matrix on average
  const int ks = a.offset ? 1 : 4;
  if (mats == 2)
    return per <= 16 ? stream_grouped<2, 1, 1, 2, 2>(a, ks, s) : stream_grouped<2, 1, 2, 2, 2>(a, ks, s);
  return per <= 16 ? stream_grouped<1, 1, 1, 2, 2>(a, ks, s) : stream_grouped<1, 1, 4, 2, 2>(a, ks, s);
}

}  // namespace deamoe
