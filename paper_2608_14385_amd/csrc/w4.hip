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

// The row tiles of all matrices, `rows` rows each, counted over the matrices in
// order.  Every wave counts and finds tiles by itself, with no barrier: a lane
// counts the tiles of a run of matrices.  Offsets outside [0, M] count as the
// nearer end.
struct Tiles {
  int rows, per, mine, inc;   // matrices of a lane's run, its tiles, those up to its end
  int total;

  __device__ Tiles(const W4Args &a, int rows_) : rows(rows_) {
    if (!a.offset) {
      total = (a.M + rows - 1) / rows;
      return;
    }
    const int lane = lane_id(), e0 = lane * (per = (a.n + kWave - 1) / kWave);
    constexpr int U = 4;   // offsets read at once
    mine = 0;
    for (int i = 0; i < per; i += U) {
      int o[U + 1];
#pragma unroll
      for (int u = 0; u <= U; ++u) o[u] = clamped(a, e0 + min(i + u, per));
#pragma unroll
      for (int u = 0; u < U; ++u) mine += (max(o[u + 1] - o[u], 0) + rows - 1) / rows;
    }
    inc = mine;
    scan<kWave>(inc);
    total = __builtin_amdgcn_readlane(inc, kWave - 1);
  }

  // Matrix and token rows [m0, m1) of a tile below `total`.
  __device__ void find(const W4Args &a, int tile, int &e, int &m0, int &m1) const {
    if (!a.offset) {
      e = 0;
      m0 = tile * rows;
      m1 = min(m0 + rows, a.M);
      return;
    }
    const int lane = lane_id();
    const int from = first(inc > tile);   // the lane whose run holds the tile
    // the lanes look at the matrices of that run: DEAMOE_MAX_EXPERTS / 64 at most
    const int base = __builtin_amdgcn_readlane(inc - mine, from), f = from * per + lane;
    const int lo = clamped(a, f), hi = max(clamped(a, f + 1), lo);
    const int here = lane < per && f < a.n ? (hi - lo + rows - 1) / rows : 0;
    int upto = here;
    scan<DEAMOE_MAX_EXPERTS / kWave>(upto);
    const int at = first(base + upto > tile);
    e = from * per + at;
    m0 = __builtin_amdgcn_readlane(lo, at) +
         (tile - base - __builtin_amdgcn_readlane(upto - here, at)) * rows;
    m1 = min(m0 + rows, __builtin_amdgcn_readlane(hi, at));
  }

 private:
  __device__ static int clamped(const W4Args &a, int e) {
    return min(max(a.offset[min(e, a.n)], 0), a.M);
  }
  __device__ static int first(bool v) { return __ffsll((unsigned long long)__ballot(v)) - 1; }
  template <int LANES>
  __device__ static void scan(int &v) {   // inclusive, over the first LANES lanes
    const int lane = lane_id();
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) {
      const int o = __shfl_up(v, d);
      v += lane >= d ? o : 0;
    }
  }
};

// f(pointer) with the scales' type: one branch around a batch of loads, which
// are all in flight before the first is waited for.
template <class F>
__device__ inline void with_scales(const void *p, int bf16, F f) {
  if (bf16) f(glob(static_cast<const uint16_t *>(p)), 16);
  else f(glob(static_cast<const uint32_t *>(p)), 0);
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

template <int CTRL>
__device__ inline float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}

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

// -24 times the sum of the eight columns of x held by each lane and by its
// neighbours in runs of LANES (4, 8 or 16), in fp32.
template <int LANES>
__device__ inline float minus_24_sum(u32x4 v) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 c = {(__bf16)-24.f, (__bf16)-24.f};
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t pair = v[i];   // a bit cast of the element itself would take element 0
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), c, s, false);
  }
  // lane i adds lane i ^ 1, i ^ 2, then a lane of the other quad, of the other half row
  s += dpp<0xb1>(s);
  s += dpp<0x4e>(s);
  if constexpr (LANES > 4) s += dpp<0x141>(s);
  if constexpr (LANES > 8) s += dpp<0x140>(s);
  return s;
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

// Few token rows: the weights are streamed, each byte once per 16 * NTT rows
// (KEEP, dense products of more than 16 rows: through the caches, for another 16
// to come; experts' products never, though the few experts of more than 16 rows
// then read their codes again).  A wave takes NR 16-row tiles of each matrix and
// every ks-th step of 256 columns.  The loads of a step are requested two steps
// ahead, straight into registers, each load 8 whole cache lines (halves of 16 lines streamed at 4.8
// TB/s, these at 5.6, by loads alone on 490 MB).  The token rows
// stand in LDS, a panel of columns at a time, already in the codes' order: read
// from memory by every wave they would take several times the weights'
// bandwidth, and since loads retire in order, waiting for them would wait for
// weights.  The scales of a panel's columns stand beside them, for each wave
// its tiles': read by the lanes that need them, they would touch as many cache
// lines as the weights.  Waves that share tiles add their sums over LDS at the
// end.  Every panel costs a round trip to the caches, so that WIDE panels take
// all of a CU's LDS where a CU has one workgroup.
// About 75 of 128 experts of 2 x 1536 x 4096 for 16 tokens, 490 MB, take 90 to 93 us:
// 5.3 to 5.5 TB/s, bound by HBM, which reads 1.02 times the touched weights.  About
// 75 experts of 4096 x 1536, 246 MB, take 73 us, 3.4 TB/s: a workgroup finds its item
// in two dependent round trips, for six steps of work.  7168 x 7168 for one row takes
// 11 us, of which the weights' 27 MB need 5.5.  Dense products of 8 rows and more
// are far from their weights' time: every 16 token rows read and unpack all codes
// again, and every workgroup all of K (4096 x 4096: 9.8 us at 8 rows, 17 at 64, 22 at
// 128, 31 at 256).
constexpr int kPanelWords = 16 * (1024 + 8) / 2;   // of a token tile, 4 bytes each
constexpr int kPanelScales = 32;                   // of a weight row, at most
constexpr int kWidePanel = 4;                      // token tiles' words in a wide panel
// wide: 16 token rows of 4096 columns and the scales, 149 of 160 KB
constexpr int panel_words(int ntt, bool wide) { return kPanelWords * (wide ? kWidePanel : ntt); }
constexpr int panel_scales(int tiles, bool wide) { return wide ? 64 / tiles : kPanelScales; }
constexpr int kNonTemporal = 2;                    // cache policy of a buffer load
constexpr int kRingColumns = 512;                  // two steps of 256: a round of the ring
template <int MATS, int NR, int NTT, int G32, bool KEEP, bool WIDE>
__global__ __launch_bounds__(kThreads, 2) void w4_stream_kernel(W4Args a, int ks) {
  constexpr int D = 2, CH = 2, SC = 128 * CH, NT = MATS * NR, GS = 32 * G32;
  constexpr int TR = NTT * kTile, WORDS = panel_words(NTT, WIDE), SCALES = panel_scales(NT, WIDE);
  __shared__ __align__(16) uint32_t s_x[WORDS];
  __shared__ float s_scale[kWaves][NT][kTile][SCALES + 1];
  static_assert(kWaves * NT * NTT * 4 * kWave <= WORDS, "the sums of the waves");
  static_assert(CH % 2 == 0, "steps of whole cache lines");
  static_assert(D * SC == kRingColumns && kRingColumns <= 1024, "a panel holds a round of the ring");
  const int lane = lane_id(), j = lane & 15, g = lane >> 4, tid = threadIdx.x;
  const int wv = uniform(tid / kWave);
  const int kp = wv % ks, rows = kWaves / ks * NR * kTile, rt = (a.R + rows - 1) / rows;
  const int steps = (a.K + SC - 1) / SC, groups = a.K / GS;
  const Tiles tiles(a, TR);
  const int64_t items = (int64_t)uniform(tiles.total) * rt;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    int e, m0, m1;
    tiles.find(a, (int)(item / rt), e, m0, m1);
    e = uniform(e), m0 = uniform(m0);
    const int ntok = uniform(m1) - m0;
    const int r0 = uniform((int)(item % rt) * rows + (wv / ks) * NR * kTile);
    // The codes are read through buffer descriptors of the matrix's rows from r0
    // on: base and size move with the step, each lane's offset stays, and rows
    // past the last read as zeros (they are never stored).  A step that ends past
    // the row's end reads the next row there, or past the last row zeros, times
    // an x of 0; a request past the last step goes to an empty buffer, which reads
    // nothing, so that every iteration issues the same loads.
    const uint32_t wrow = a.K / 2;
    char *wb[MATS];
    const void *sb[MATS];
    const int left = max(a.R - r0, 1);   // a wave past the last row repeats it
    const size_t first = (size_t)e * a.R + min(r0, a.R - 1);
#pragma unroll
    for (int n = 0; n < MATS; ++n) {
      wb[n] = const_cast<char *>(uniform_ptr(static_cast<const char *>(a.w[n]) + first * wrow));
      sb[n] = uniform_ptr(static_cast<const char *>(a.scale[n]) + first * groups * (a.scale_bf16 ? 2 : 4));
    }
    uint32_t wo[NR][2];   // rows_together's order
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        wo[n][i] = (n * kTile + i * 8 + (j & 7)) * wrow + ((j >> 3) * 4 + g) * 16;
    u32x4 W[D][NT][CH];
    auto request = [&](int q, int s) {
      const int at = s < steps ? s * (SC / 2) : 0, bytes = s < steps ? (int)(left * wrow - at) : 0;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const auto buf = __builtin_amdgcn_make_buffer_rsrc(wb[n / NR] + at, 0, bytes, 0x00027000);
#pragma unroll
        for (int c = 0; c < CH; ++c)
          W[q][n][c] =
              __builtin_amdgcn_raw_buffer_load_b128(buf, wo[n % NR][c & 1] + c / 2 * 128, 0, KEEP ? 0 : kNonTemporal);
      }
    };
#pragma unroll
    for (int d = 0; d < D; ++d) request(d, kp + d * ks);

    // panels: whole rounds of all ring places of all K parts
    const int round = D * ks * SC, prow = min(ntok, TR);
    const int pcol = min(min(WORDS * 2 / prow - 8, a.K + round - 1), SCALES * GS) / round * round;
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
      // this wave's scales; past the end the sums are 0, and
      // their scale is
      constexpr int N = kTile * SCALES / kWave;
      const int sr = lane / SCALES, sq = lane % SCALES;
      uint32_t sv[NT][N];
#pragma unroll
      for (int n = 0; n < NT; ++n)
        with_scales(sb[n / NR], a.scale_bf16, [&](auto *from, int) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int r = (n % NR) * kTile + i * (kWave / SCALES) + sr;
            sv[n][i] = from[sq < nq && r < left ? r * groups + q0 + sq : 0];
          }
        });
      constexpr int U = NTT == 1 && !WIDE ? 8 : 16;   // 16-byte chunks of x in flight
      const int chunks = pcol / 8, total = prow * chunks;
      // i / chunks = i * inverse / 2^32: both are below 2^15, so that the
      // inverse's excess times i stays below 2^32
      const uint32_t inverse = 0xffffffffu / chunks + 1;
      for (int i0 = 0; i0 < total; i0 += U * kThreads) {
        u32x4 v[U];
        uint32_t at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (i0 + u * kThreads >= total) break;
          const uint32_t i = min(i0 + u * kThreads + tid, total - 1), r = __umulhi(i, inverse);
          const uint32_t k = (i - r * chunks) * 8;
          const bool ok = p0 + k < (uint32_t)a.K;
          at[u] = (r * ldx + k) * 2 + !ok;   // odd: zeros, once all loads are on their way
          v[u] = *gptr(static_cast<const char *>(a.x) + ((size_t)(m0 + r) * a.K + (ok ? p0 + k : 0)) * 2);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (i0 + u * kThreads >= total) break;
          const u32x4 x = at[u] & 1 ? u32x4{0, 0, 0, 0} : v[u];
          *reinterpret_cast<bf16x8 *>(reinterpret_cast<char *>(s_x) + (at[u] & ~1u)) = order_columns(x);
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < N; ++i)
          s_scale[wv][n][i * (kWave / SCALES) + sr][sq] =
              sq < nq && (n % NR) * kTile + i * (kWave / SCALES) + sr < left
                  ? __uint_as_float(sv[n][i] << (a.scale_bf16 ? 16 : 0)) : 0.f;
      __syncthreads();
      const int end = min(p0 + pcol, a.K);
      auto steps_of_panel = [&] {
#pragma unroll 1
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

// Many token rows: a workgroup multiplies 64 of them with 256 weight rows (with
// two matrices 128 of each), every wave 64 rows of its own, so that no code is
// unpacked twice.  The -24 sums are made once, by the threads that bring the
// token rows to LDS.  A wave multiplies two of its four weight tiles at a time:
// the sums of all four beside acc and the next step's operands would not fit
// 256 registers, and reading the token rows from LDS twice costs less.
// Both operands of the next step are requested before a step's products; the
// token rows go through registers, where they take the codes' order, into the
// other half of the LDS buffer.
// 8192 rows through 2048 x 8192 run at 810 to 840 TFLOP/s; 12288 rows through 64
// experts of 2 x 1280 x 2048, whose tiles are a seventh empty and whose sums are
// short, in 210 us, 610 TFLOP/s.  There the matrix cores are busy for 29 % of the
// time, HBM reads 1.4 TB/s and four of five requests hit L2, so that none of them
// is the bound: a step's 32 KB per workgroup arrive at 19 bytes per ns on a CU with
// one step on its way, and by instruction count unpacking takes half as many issue
// cycles as the products.  Weights requested two steps at a time spilled registers,
// 215 -> 224 us.
constexpr int kTileTok = 64, kTileStep = 128, kTileStride = kTileStep + 8;
constexpr int kTileThreads = 256, kTileWaves = kTileThreads / kWave, kTileWeights = 4;
template <int MATS, int G32>
__global__ __launch_bounds__(kTileThreads, 2) void w4_tile_kernel(W4Args a) {
  constexpr int NT = kTileWeights, NP = 2, NR = NT / MATS, NTT = kTileTok / kTile, GS = 32 * G32;
  constexpr int XC = (kTileTok * kTileStep / 8 + kTileThreads - 1) / kTileThreads;   // 16-byte chunks of x per thread
  __shared__ __align__(16) uint16_t s_x[2][kTileTok][kTileStride];
  __shared__ __align__(16) float s_start[2][4 / G32][kTileTok];
  __shared__ float s_scale[kTileWaves][NT][kTile][kPanelScales + 1];
  const int lane = lane_id(), j = lane & 15, g = lane >> 4, tid = threadIdx.x;
  const int wv = uniform(tid / kWave);
  const int rows = kTileWaves * NR * kTile, rt = (a.R + rows - 1) / rows;
  const int steps = (a.K + kTileStep - 1) / kTileStep, groups = a.K / GS;
  const Tiles tiles(a, kTileTok);
  // Consecutive workgroups run on the 8 XCDs in turn: each XCD gets a run of
  // neighbouring items, which share weights and token rows in its L2.
  const int64_t items = (int64_t)uniform(tiles.total) * rt, run = (items + 7) / 8;
  for (int64_t i = blockIdx.x / 8; i < run; i += gridDim.x / 8) {
    const int64_t item = blockIdx.x % 8 * run + i;
    if (item >= items) return;
    int e, m0, m1;
    tiles.find(a, (int)(item / rt), e, m0, m1);
    e = uniform(e), m0 = uniform(m0);
    const int ntok = uniform(m1) - m0;
    const int r0 = uniform((int)(item % rt) * rows + wv * NR * kTile);
    const int left = max(a.R - r0, 1);   // a wave past the last row repeats it
    const size_t first = (size_t)e * a.R + min(r0, a.R - 1);
    const uint32_t wrow = a.K / 2;
    char *wb[MATS];
    const void *sb[MATS];
#pragma unroll
    for (int n = 0; n < MATS; ++n) {
      wb[n] = const_cast<char *>(uniform_ptr(static_cast<const char *>(a.w[n]) + first * wrow));
      sb[n] = uniform_ptr(static_cast<const char *>(a.scale[n]) + first * groups * (a.scale_bf16 ? 2 : 4));
    }
    uint32_t wo[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) wo[n] = (n * kTile + j) * wrow + g * 16;
    char *xb = const_cast<char *>(
        uniform_ptr(static_cast<const char *>(a.x) + (size_t)m0 * a.K * 2));
    uint32_t xo[XC];   // token row tid / 16 + 16 i
#pragma unroll
    for (int i = 0; i < XC; ++i)
      xo[i] = (uint32_t)min(tid / 16 + i * (kTileThreads / 16), ntok - 1) * a.K * 2;
    u32x4 W[2][NT], X[XC];
    auto request_w = [&](int q, int s) {
      const int at = s < steps ? s * (kTileStep / 2) : 0, bytes = s < steps ? (int)(left * wrow - at) : 0;
#pragma unroll
      for (int n = 0; n < NT; ++n)
        W[q][n] = __builtin_amdgcn_raw_buffer_load_b128(
            __builtin_amdgcn_make_buffer_rsrc(wb[n / NR] + at, 0, bytes, 0x00027000), wo[n % NR], 0, 0);
    };
    auto request_x = [&](int s) {   // chunk tid % 16 of the step; past the row's end its first
      const uint32_t col = s * kTileStep + tid % 16 * 8, at = col < (uint32_t)a.K ? col * 2 : 0u;
#pragma unroll
      for (int i = 0; i < XC; ++i) X[i] = *gptr(xb + (xo[i] + at));
    };
    auto put_x = [&](int q, int s) {
      const bool ok = s * kTileStep + tid % 16 * 8 < a.K;
#pragma unroll
      for (int i = 0; i < XC; ++i) {
        const u32x4 v = ok ? X[i] : u32x4{0, 0, 0, 0};
        const int row = tid / 16 + i * (kTileThreads / 16);
        if (row >= kTileTok) break;   // whole waves
        *reinterpret_cast<bf16x8 *>(&s_x[q][row][tid % 16 * 8]) = order_columns(v);
        const float sum = minus_24_sum<G32 * 4>(v);
        if (tid % (G32 * 4) == 0) s_start[q][tid % 16 / (G32 * 4)][row] = sum;
      }
    };
    auto put_scales = [&](int q0) {   // this wave's, of kPanelScales groups
      constexpr int N = kTile * kPanelScales / kWave;
      const int sr = lane / kPanelScales, sq = lane % kPanelScales;
#pragma unroll 1
      for (int n = 0; n < NT; ++n)
        with_scales(n < NR ? sb[0] : sb[MATS - 1], a.scale_bf16, [&](auto *from, int shift) {
          uint32_t v[N];
#pragma unroll
          for (int i = 0; i < N; ++i) {   // two rows at a time
            const int r = n % NR * kTile + i * 2 + sr;
            v[i] = from[q0 + sq < groups && r < left ? r * groups + q0 + sq : 0];
          }
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const bool ok = q0 + sq < groups && n % NR * kTile + i * 2 + sr < left;
            s_scale[wv][n][i * 2 + sr][sq] = ok ? __uint_as_float(v[i] << shift) : 0.f;
          }
        });
    };
    float acc[NT][NTT][4] = {};
    const Magic magic;
    auto multiply = [&](int q, int s) {
      const int q0 = s * (4 / G32) % kPanelScales;
#pragma unroll
      for (int n = 0; n < NT; ++n) columns_together(W[q][n]);
#pragma unroll
      for (int i = 0; i < 4 / G32; ++i)
#pragma unroll
        for (int n0 = 0; n0 < NT; n0 += NP) {
          f32x4 p[NP][NTT];
#pragma unroll
          for (int t = 0; t < NTT; ++t) {   // lane group g: tokens 4 g .. 4 g + 3 of the tile
            p[0][t] = *reinterpret_cast<const f32x4 *>(&s_start[q][i][t * kTile + g * 4]);
#pragma unroll
            for (int n = 1; n < NP; ++n) p[n][t] = p[0][t];
          }
#pragma unroll
          for (int m = i * G32; m < (i + 1) * G32; ++m) {
            bf16x8 xv[NTT];
#pragma unroll
            for (int t = 0; t < NTT; ++t)
              xv[t] = *reinterpret_cast<const bf16x8 *>(&s_x[q][t * kTile + j][m * 32 + g * 8]);
#pragma unroll
            for (int n = 0; n < NP; ++n) {
              const bf16x8 w = codes_to_bf16(W[q][n0 + n][m], magic);
#pragma unroll
              for (int t = 0; t < NTT; ++t)
                p[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv[t], w, p[n][t], 0, 0, 0);
            }
          }
#pragma unroll
          for (int n = 0; n < NP; ++n) {
            const float sc = s_scale[wv][n0 + n][j][q0 + i];
#pragma unroll
            for (int t = 0; t < NTT; ++t)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                float &v = acc[n0 + n][t][r];
                v = __builtin_fmaf(sc, p[n][t][r], v);
                // here and now: left to the end of the step, all groups' sums
                // would have to be kept
                asm volatile("" : "+v"(v));
              }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
    };
    __syncthreads();   // the last item's token rows have been read
    request_w(0, 0);
    request_x(0);
    put_scales(0);
    put_x(0, 0);
    __syncthreads();
    auto all_steps = [&] {
#pragma unroll 1
      for (int s = 0;; s += 2)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          if (s + q >= steps) return;
          request_x(s + q + 1);
          request_w(q ^ 1, s + q + 1);
          __builtin_amdgcn_sched_barrier(0);   // not among the products
          multiply(q, s + q);
          if ((s + q + 1) * (4 / G32) % kPanelScales == 0) put_scales((s + q + 1) * (4 / G32));
          put_x(q ^ 1, s + q + 1);
          __syncthreads();
        }
    };
    all_steps();
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

// Row tiles of the matrices at most: with offsets, every matrix may end inside
// one.
int64_t row_tiles(const W4Args &a, int rows) {
  return a.offset ? a.M / rows + (a.n < a.M ? a.n : a.M) : (a.M + rows - 1) / rows;
}

dim3 grid_of(int64_t items) { return dim3((unsigned)(items < (1 << 20) ? items : 1 << 20)); }

// K parts of the streaming kernel's workgroups, which there are `groups` of with
// one part: as many as keep all workgroups on the CUs at once (stream_resident
// each), and as a panel holds a round of the ring for.  us, one | two | four parts: 4096 x 7168, one row, 64 workgroups of one
// part, 20.5 | 13.5 | 9.7; 16384 x 7168, 256 of them, 22.0 | 16.9 | 21.8; 28672 x
// 7168, 448 of them, 26.8 | 31.3 | 33.1; 8 rows of 8 experts of 2 x 2048 x 7168,
// 256 of them, 31.8 | 27.7 | 34.9.  Groups of 32, two matrices, of which a CU holds
// two workgroups: 257 of them, 16448 x 2048 of one row, 18.8 | 22.8; 384, 24576 x
// 4096 of 16 rows, 38.3 | 51.4; 320, one row of 10 experts of 2048 x 4096, 34.7 | 43.0.
struct Parts {
  int ks, columns;   // K parts, columns of a panel
};
Parts k_parts(const W4Args &a, int ntt, int64_t groups, int most, int words, int scales) {
  const int rows = a.M < kTile * ntt ? a.M : kTile * ntt, in_x = words * 2 / rows - 8;
  const int columns = in_x < scales * a.group ? in_x : scales * a.group;
  int ks = 1;
  while (ks < kWaves && groups * ks * 2 <= most && ks * 2 * kRingColumns <= columns) ks *= 2;
  return {ks, columns / (ks * kRingColumns) * (ks * kRingColumns)};
}

template <int MATS, int NR, int NTT, bool KEEP, bool WIDE>
hipError_t stream_panels(const W4Args &a, int64_t tiles, int ks, hipStream_t s) {
  const int rows = kWaves / ks * NR * kTile;
  const dim3 grid = grid_of(tiles * ((a.R + rows - 1) / rows));
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a, ks); };
  if (a.group == 32) launch(w4_stream_kernel<MATS, NR, NTT, 1, KEEP, WIDE>);
  else if (a.group == 64) launch(w4_stream_kernel<MATS, NR, NTT, 2, KEEP, WIDE>);
  else launch(w4_stream_kernel<MATS, NR, NTT, 4, KEEP, WIDE>);
  return hipGetLastError();
}

template <int MATS, int NR, int NTT, bool KEEP>
hipError_t stream(const W4Args &a, hipStream_t s) {
  constexpr int kCus = 256;
  const int64_t tiles = row_tiles(a, kTile * NTT);
  const int64_t groups = tiles * ((a.R + kWaves * NR * kTile - 1) / (kWaves * NR * kTile));
  const int most = kCus * stream_resident(MATS, NR, NTT, a.group, false);
  const Parts p = k_parts(a, NTT, groups, most, panel_words(NTT, false), kPanelScales);
  if constexpr (NR == 1 && NTT == 1) {
    // With no more workgroups than CUs, panels that fill a CU's LDS, where they
    // allow more parts or are four times as wide; us, narrow | wide: 4096 x 7168,
    // 16 rows, 22.9 | 18.2, two matrices of 4096 x 4096 19.7 | 12.8; with as many
    // parts of panels twice as wide, 7168 x 7168 in groups of 32, 22.7 | 25.9.
    const Parts w = k_parts(a, NTT, groups, kCus, panel_words(NTT, true), panel_scales(MATS, true));
    if (groups * w.ks <= kCus && p.columns < a.K &&
        (w.ks > p.ks || (w.ks == p.ks && w.columns >= 4 * p.columns)))
      return stream_panels<MATS, NR, NTT, KEEP, true>(a, tiles, w.ks, s);
  }
  return stream_panels<MATS, NR, NTT, KEEP, false>(a, tiles, p.ks, s);
}

template <int MATS>
hipError_t tile(const W4Args &a, hipStream_t s) {
  const int rows = kTileWaves * kTileWeights / MATS * kTile;
  const int64_t items = row_tiles(a, kTileTok) * ((a.R + rows - 1) / rows);
  const dim3 grid = grid_of((items + 7) / 8 * 8);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kTileThreads), 0, s, a); };
  if (a.group == 32) launch(w4_tile_kernel<MATS, 1>);
  else if (a.group == 64) launch(w4_tile_kernel<MATS, 2>);
  else launch(w4_tile_kernel<MATS, 4>);
  return hipGetLastError();
}

template <int MATS>
hipError_t run(const W4Args &a, hipStream_t s) {
  const int blocks = (a.R + 255) / 256 * MATS;
  if (a.offset) {
    // The mean rows of a matrix decide, us, streamed | tiled: 64 experts of 2 x
    // 1280 x 2048, 57 | 78 at 12 rows, 77 | 79 at 19, 96 | 83 at 24; 128 of 2 x 1536 x
    // 4096, 304 | 309 at 20, 353 | 309 at 24; 256 of 2 x 512 x 2048, 121 | 127 at 20,
    // 141 | 129 at 24.  One matrix: 64 of 2048 x 1280, 36 | 37 at 7, 49 | 49 at 15, 59 |
    // 49 at 19; 128 of 4096 x 1536, 161 | 170 at 14, 201 | 172 at 20; 16 of 7168 x 2048,
    // 52 | 52 at 14.
    const int64_t mean = a.M / a.n;
    if (mean > (MATS == 2 ? 20 : 14)) return tile<MATS>(a, s);
    // Many workgroups, of one matrix: four weight tiles per wave (about 75 experts of
    // 4096 x 1536: 81 -> 75 us; but 48 of 2048 x 1280 34 -> 41).
    if (MATS == 1 && row_tiles(a, kTile) * ((a.R + 63) / 64) >= 5120) return stream<1, 4, 1, false>(a, s);
    return stream<MATS, 1, 1, false>(a, s);
  }
  // The tiled kernel from more than one workgroup on every second CU on, us, streamed |
  // tiled: 4096 x 4096, 59 | 60 at 448 rows (112 workgroups), 74 | 61 at 640 (160);
  // 7168 x 7168, 82 | 99 at 192 (84), 126 | 100 at 320 (140), 166 | 102 at 512 (224);
  // two matrices of 4096 x 4096, 43 | 59 at 192 (96), 79 | 60 at 384 (192).
  if ((int64_t)((a.M + 63) / 64) * blocks > 128) return tile<MATS>(a, s);
  if (a.M <= kTile) return stream<MATS, 1, 1, false>(a, s);
  // two token tiles per pass over the weights, us, one | two: 4096 x 4096, 22.8 |
  // 25.8 at 128 rows, 38.9 | 34.4 at 256; two matrices 53 | 64 at 200
  if (MATS == 1 && a.M > 160) return stream<1, 1, 2, true>(a, s);
  return stream<MATS, 1, 1, true>(a, s);
}

}  // namespace

hipError_t launch_w4(const W4Args &a, int mats, hipStream_t s) {
  return mats == 2 ? run<2>(a, s) : run<1>(a, s);
}

}  // namespace deamoe
