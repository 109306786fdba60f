// RMSNorm before and after a block, with the block's gate and residual scale,
// and their gradients.
//
//   v^ = v r,  r = 1 / sqrt(mean(v^2) + eps)
//   u = x^ w                                          (before a block)
//   z = a x + g (y^ w),  u = z^ w'                    (after it, and the next)
// Gradients, with <m> the mean over a row:
//   norm(v, q)  = r (q - v^ <q v^>)       q: gradient of v^
//   d  = dz + norm(z, du w'),  dw' = sum_t du z^
//   dx = a d,  dg = d y^ w,  dw = sum_t d g y^,  dy = norm(y, d g w)
#include <type_traits>

#include "ops.h"

namespace deamoe {

namespace {

template <int CTRL>
__device__ inline float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}

// The sum over a row of 16 lanes, on all of them: lane i adds lane i ^ 1, i ^ 2,
// then a lane of the other quad, of the other half.  In registers: a shuffle
// through LDS per step took a quarter of a row's time.
__device__ inline float sum16(float v) {
  v += dpp<0xb1>(v);    // quad_perm [1, 0, 3, 2]
  v += dpp<0x4e>(v);    // quad_perm [2, 3, 0, 1]
  v += dpp<0x141>(v);   // row_half_mirror
  v += dpp<0x140>(v);   // row_mirror
  return v;
}
__device__ inline float lane_value(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// Sums of N values over the workgroup, the same on every thread.  Two
// reductions in a row use different halves of `s`, so that one barrier each is
// enough.
constexpr int kMaxWaves = 16, kMaxSums = 3;
constexpr int kRowWaves = 4;   // rows at a time in the gradients of rows of one wave
struct Reduce {
  float (*s)[kMaxSums][kMaxWaves];
  int flip = 0;
  template <int N>
  __device__ void sum(float (&v)[N]) {
    const int waves = blockDim.x / kWave, lane = threadIdx.x % kWave;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = sum16(v[i]);
      v[i] = (lane_value(v[i], 0) + lane_value(v[i], 16)) + (lane_value(v[i], 32) + lane_value(v[i], 48));
    }
    if (waves == 1) return;
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) s[flip][i][threadIdx.x / kWave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = sum16(lane % 16 < waves ? s[flip][i][lane % 16] : 0.f);
    flip ^= 1;
  }
};

// The chunks of one row that a thread works on: chunk i starts at column
// (i * threads + thread) * V.  N > 0: N chunks, held in registers; N == 0: rows
// too wide for that are read again at every use.
template <bool F32, int N>
struct Row {
  static constexpr int V = kVec<F32>;
  const char *p;
  int h;
  Chunk<F32> held[N > 0 ? N : 1];
  __device__ Row(const void *base, size_t t, int h_) : p(row_at<F32>(base, t, h_)), h(h_) {
    if constexpr (N > 0)
#pragma unroll
      for (int i = 0; i < N; ++i)
        held[i] = load_chunk<F32>(p, (i * (int)blockDim.x + (int)threadIdx.x) * V, h);
  }
  __device__ Chunk<F32> get(int i, int c) const {
    if constexpr (N > 0) return held[i];
    return load_chunk<F32>(p, c, h);
  }
};

// f(i, c) for every chunk of the thread; N > 0: also for those past the row's
// end, whose loads give zeros and whose stores do nothing.
template <bool F32, int N, class F>
__device__ inline void chunks(int h, F f) {
  constexpr int V = kVec<F32>;
  if constexpr (N > 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) f(i, (i * (int)blockDim.x + (int)threadIdx.x) * V);
  } else {
    for (int c = threadIdx.x * V; c < h; c += blockDim.x * V) f(0, c);
  }
}

__device__ inline float rms_factor(float sum, int h, float eps) {
  return 1.0f / sqrtf(sum / (float)h + eps);
}

// u = x^ w of one row.  One read and one write: 2051 rows of 2048 in fp32, 34 MB,
// take 7.4 us (4.5 TB/s out of the last-level cache and a launch).
template <bool F32, int N>
__device__ inline void norm_row(const Row<F32, N> &x, const Row<F32, N> &w, char *u, int h,
                                float eps, Reduce &red) {
  constexpr int V = kVec<F32>;
  float ss[1] = {0.f};
  chunks<F32, N>(h, [&](int i, int c) {
    const Chunk<F32> v = x.get(i, c);
#pragma unroll
    for (int e = 0; e < V; ++e) ss[0] = __builtin_fmaf(v.at(e), v.at(e), ss[0]);
  });
  red.sum(ss);
  const float r = rms_factor(ss[0], h, eps);
  chunks<F32, N>(h, [&](int i, int c) {
    const Chunk<F32> v = x.get(i, c), g = w.get(i, c);
    float o[V];
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = v.at(e) * r * g.at(e);
    store_chunk<F32>(u, c, h, pack_chunk<F32>(o));
  });
}

}  // namespace

template <bool F32, int N, int MAXG>
__global__ __launch_bounds__(MAXG) void prenorm_kernel(PrenormArgs a) {
  __shared__ float s_red[2][kMaxSums][kMaxWaves];
  Reduce red{s_red};
  for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
    const Row<F32, N> x(a.x, t, a.h), w(a.w, 0, a.h);
    norm_row<F32, N>(x, w, row_at<F32>(a.u, t, a.h), a.h, a.eps, red);
  }
}

template <bool F32, int N, int MAXG>
__global__ __launch_bounds__(MAXG) void postnorm_kernel(PostnormArgs a) {
  constexpr int V = kVec<F32>;
  __shared__ float s_red[2][kMaxSums][kMaxWaves];
  Reduce red{s_red};
  for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
    // all of the row's loads before the first sum is waited for
    const Row<F32, N> y(a.y, t, a.h), x(a.x, t, a.h), w(a.w, 0, a.h);
    const Row<F32, N> gate(a.gate_mode ? a.gate : a.w, a.gate_mode == DEAMOE_GATE_FULL ? t : 0, a.h);
    const Row<F32, N> w_next(a.u ? a.w_next : a.w, 0, a.h);
    float ss[1] = {0.f};
    chunks<F32, N>(a.h, [&](int i, int c) {
      const Chunk<F32> v = y.get(i, c);
#pragma unroll
      for (int e = 0; e < V; ++e) ss[0] = __builtin_fmaf(v.at(e), v.at(e), ss[0]);
    });
    red.sum(ss);
    const float r = rms_factor(ss[0], a.h, a.eps);
    char *zp = row_at<F32>(a.z, t, a.h);
    Row<F32, N> z = x;
    z.p = zp;
    chunks<F32, N>(a.h, [&](int i, int c) {
      const Chunk<F32> yv = y.get(i, c), xv = x.get(i, c), wv = w.get(i, c);
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = yv.at(e) * r * wv.at(e);
      if (a.gate_mode != DEAMOE_GATE_NONE) {
        const Chunk<F32> g = gate.get(i, c);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] *= g.at(e);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = __builtin_fmaf(a.res_scale, xv.at(e), o[e]);
      z.held[i] = pack_chunk<F32>(o);   // past the row's end: zeros, as loaded
      store_chunk<F32>(zp, c, a.h, z.held[i]);
    });
    if (a.u) norm_row<F32, N>(z, w_next, row_at<F32>(a.u, t, a.h), a.h, a.eps, red);
  }
}

// Gradients.  MODE: the norm before a block alone, the one after it alone, or
// the one after it with the next one before.  A workgroup walks over rows t,
// t + grid, ... and keeps its sums over them for its columns: in registers, or
// for wide rows in its part of the workspace.  Rows that one wave holds are taken
// four at a time, a wave each (blockDim.y), whose sums are joined in LDS.  8192 rows
// of 4096 in bf16 with both norms and a shared gate, 403 MB, take 89 us: 4.5 TB/s, of
// a copy's 4.9.
//   Two chunks in each of 1024 threads (fp32 rows of 4097 to 8192 columns, bf16 of
// 8193 to 16384) leave 128 registers, and four of those six forms keep a part of
// the row, its successor or the sums in scratch: fp32 with both norms 61 registers,
// bf16 30 (pre), 70 (post) and 174 (both).  2048 rows with both norms: fp32 of 5120
// 113 us, of 7168 128 (floors 51 and 71; 471 MB read for 235, 187 written for 117);
// bf16 of 9216 302 us, of 12288 312, of 16384 335 (floors 46, 61 and 82; 1130 MB read
// for 201 and 604 written for 101 at 12288).  The two forms that do not spill are
// within 1.4 of their floors.
enum NormMode : int { NORM_PRE = 0, NORM_POST = 1, NORM_BOTH = 2 };

template <bool F32, int N, int MODE>
struct BackwardRows {   // what one row reads
  Row<F32, MODE != NORM_POST ? N : 0> z, du;
  Row<F32, MODE != NORM_PRE ? N : 0> y;
  Row<F32, N> dz;
  __device__ BackwardRows(const NormBackwardArgs &a, int t)
      : z(a.z, t, a.h), du(a.du, t, a.h), y(a.y, t, a.h), dz(a.dz ? a.dz : a.du, t, a.h) {}
};

template <bool F32, int N, int MAXG, int MODE>
__global__ __launch_bounds__(MAXG) void norm_backward_kernel(NormBackwardArgs a) {
  constexpr int V = kVec<F32>, NH = N > 0 ? N : 1;
  constexpr bool POST = MODE != NORM_PRE, NEXT = MODE != NORM_POST;
  __shared__ float s_red[2][kMaxSums][kMaxWaves];
  Reduce red{s_red};
  const int h = a.h;
  float *part = a.part + (size_t)blockIdx.x * 3 * h;   // dw, dw_next, dgate
  constexpr bool ROWS = N == 1 && MAXG == 256;   // several rows at a time; the row stays a scalar
  const int y = ROWS ? __builtin_amdgcn_readfirstlane(threadIdx.y) : 0, ny = ROWS ? blockDim.y : 1;
  const int t0 = blockIdx.x * ny + y, step = gridDim.x * ny;
  float sum[3][NH][V] = {};
  auto add = [&](int which, int i, int c, bool first, const float (&v)[V]) {
    if constexpr (N > 0) {
#pragma unroll
      for (int e = 0; e < V; ++e) sum[which][i][e] += v[e];
    } else {
      for (int e = 0; e < V; ++e)
        if (c + e < h) {
          float *p = part + (size_t)which * h + c + e;
          *p = first ? v[e] : *p + v[e];
        }
    }
  };
  const Row<F32, POST ? N : 0> w(a.w, 0, h);
  const Row<F32, NEXT ? N : 0> w_next(a.w_next, 0, h);
  BackwardRows<F32, N, MODE> next(a, min(t0, a.T - 1));
  for (int t = t0; t < a.T; t += step) {
    const bool first = t == t0;
    const BackwardRows<F32, N, MODE> r = next;
    const Row<F32, POST ? N : 0> gate(a.gate_mode == DEAMOE_GATE_NONE ? a.w : a.gate,
                                      a.gate_mode == DEAMOE_GATE_FULL ? t : 0, h);
    // the next row is on its way while this one waits for its sums
    if (t + step < a.T) next = BackwardRows<F32, N, MODE>(a, t + step);
    float s1[3] = {0.f, 0.f, 0.f};   // z^2, du w' z, y^2
    chunks<F32, N>(h, [&](int i, int c) {
      if constexpr (NEXT) {
        const Chunk<F32> zv = r.z.get(i, c), g = r.du.get(i, c), wv = w_next.get(i, c);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          s1[0] = __builtin_fmaf(zv.at(e), zv.at(e), s1[0]);
          s1[1] = __builtin_fmaf(g.at(e) * wv.at(e), zv.at(e), s1[1]);
        }
      }
      if constexpr (POST) {
        const Chunk<F32> yv = r.y.get(i, c);
#pragma unroll
        for (int e = 0; e < V; ++e) s1[2] = __builtin_fmaf(yv.at(e), yv.at(e), s1[2]);
      }
    });
    red.sum(s1);
    const float rz = rms_factor(s1[0], h, a.eps), mz = s1[1] * rz / (float)h;
    const float ry = rms_factor(s1[2], h, a.eps);
    // d of one chunk: the gradient that reaches z
    auto reach = [&](int i, int c, float (&d)[V]) {
      const Chunk<F32> v = r.dz.get(i, c);
#pragma unroll
      for (int e = 0; e < V; ++e) d[e] = a.dz ? v.at(e) : 0.f;
      if constexpr (NEXT) {
        const Chunk<F32> zv = r.z.get(i, c), g = r.du.get(i, c), wv = w_next.get(i, c);
#pragma unroll
        for (int e = 0; e < V; ++e) d[e] += rz * (g.at(e) * wv.at(e) - zv.at(e) * rz * mz);
      }
    };
    float dh[NH][V];   // d of every held chunk
    float s2[1] = {0.f};
    chunks<F32, N>(h, [&](int i, int c) {
      reach(i, c, dh[i]);
      if constexpr (POST) {
        const Chunk<F32> yv = r.y.get(i, c), wv = w.get(i, c);
        float dn[V];
#pragma unroll
        for (int e = 0; e < V; ++e) dn[e] = dh[i][e];
        if (a.gate_mode != DEAMOE_GATE_NONE) {
          const Chunk<F32> g = gate.get(i, c);
#pragma unroll
          for (int e = 0; e < V; ++e) dn[e] *= g.at(e);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) s2[0] = __builtin_fmaf(dn[e] * wv.at(e), yv.at(e) * ry, s2[0]);
      }
    });
    if constexpr (POST) red.sum(s2);
    const float my = s2[0] / (float)h;
    chunks<F32, N>(h, [&](int i, int c) {
      float d[V], o[V], g[V];
      if constexpr (N > 0) {
#pragma unroll
        for (int e = 0; e < V; ++e) d[e] = dh[i][e];
      } else {
        reach(i, c, d);
      }
      if constexpr (NEXT) {
        const Chunk<F32> zv = r.z.get(i, c), gv = r.du.get(i, c);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = gv.at(e) * (zv.at(e) * rz);
        add(1, i, c, first, o);
      }
      if constexpr (POST) {
        const Chunk<F32> yv = r.y.get(i, c), wv = w.get(i, c);
        float dn[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dn[e] = d[e];
          g[e] = d[e] * (yv.at(e) * ry * wv.at(e));
        }
        if (a.gate_mode != DEAMOE_GATE_NONE) {
          const Chunk<F32> gv = gate.get(i, c);
#pragma unroll
          for (int e = 0; e < V; ++e) dn[e] *= gv.at(e);
          if (a.gate_mode == DEAMOE_GATE_FULL)
            store_chunk<F32>(row_at<F32>(a.dgate, t, h), c, h, pack_chunk<F32>(g));
          else
            add(2, i, c, first, g);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = dn[e] * (yv.at(e) * ry);
        add(0, i, c, first, o);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = ry * (dn[e] * wv.at(e) - yv.at(e) * ry * my);
        store_chunk<F32>(row_at<F32>(a.dy, t, h), c, h, pack_chunk<F32>(o));
      }
#pragma unroll
      for (int e = 0; e < V; ++e) d[e] *= a.res_scale;
      store_chunk<F32>(row_at<F32>(a.dx, t, h), c, h, pack_chunk<F32>(d));
    });
  }
  if constexpr (ROWS)
    if (ny > 1) {
      __shared__ float s_sum[kRowWaves - 1][3][V][kWave];
      if (y)
#pragma unroll
        for (int which = 0; which < 3; ++which)
#pragma unroll
          for (int e = 0; e < V; ++e) s_sum[y - 1][which][e][threadIdx.x] = sum[which][0][e];
      __syncthreads();
      if (y) return;
      for (int o = 0; o < kRowWaves - 1; ++o)
#pragma unroll
        for (int which = 0; which < 3; ++which)
#pragma unroll
          for (int e = 0; e < V; ++e) sum[which][0][e] += s_sum[o][which][e][threadIdx.x];
    }
  if constexpr (N > 0)
    chunks<F32, N>(h, [&](int i, int c) {
#pragma unroll
      for (int which = 0; which < 3; ++which) {
        if ((which == 0 && !POST) || (which == 1 && !NEXT) ||
            (which == 2 && (!POST || a.gate_mode != DEAMOE_GATE_SHARED)))
          continue;
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (c + e < h) part[(size_t)which * h + c + e] = sum[which][i][e];
      }
    });
}

// out[c] = sum over the workgroups' parts.  A workgroup takes COLS columns; its
// 1024 / COLS runs of lanes take a part in turn, 8 loads in flight, and are
// joined in order.
struct ColumnSumArgs {
  const float *part[3];     // stride of the parts: 3 * h
  float *out[3];
  int32_t h, blocks;
};
template <int COLS>
__global__ __launch_bounds__(1024) void column_sum_kernel(ColumnSumArgs a) {
  constexpr int W = 1024 / COLS, U = 8;
  __shared__ float s_sum[W][COLS];
  const int lane = threadIdx.x % COLS, at = threadIdx.x / COLS;
  const int c = blockIdx.x * COLS + lane;
  const float *p = a.part[blockIdx.y] + min(c, a.h - 1);
  float v = 0.f;
  for (int b0 = at; b0 < a.blocks; b0 += W * U) {
    float t[U];
#pragma unroll
    for (int u = 0; u < U; ++u) t[u] = p[(size_t)min(b0 + u * W, a.blocks - 1) * 3 * a.h];
#pragma unroll
    for (int u = 0; u < U; ++u) v += b0 + u * W < a.blocks ? t[u] : 0.f;
  }
  s_sum[at][lane] = v;
  __syncthreads();
  if (at == 0 && c < a.h) {
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) total += s_sum[i][lane];
    a.out[blockIdx.y][c] = total;
  }
}

namespace {

// Threads and held chunks of 16 bytes per thread for a row: as few threads as
// hold it with two chunks each while that leaves several rows per CU; from 4097
// bf16 columns on one chunk each, in 1024 threads (the gradient of 2048 rows of
// 7168: 71 us with 512 threads of two chunks, 50 with these); rows wider than
// 2048 chunks are not held (the same of 2048 rows of 16400: 344 us, held ones of
// 16384 335; in fp32 of 8200 and 8192 columns 197 and 134).
struct Shape {
  int threads, held;
};
Shape shape_of(int h, int act_f32) {
  const int chunks = (h + (act_f32 ? 3 : 7)) / (act_f32 ? 4 : 8);
  if (chunks <= 64) return {64, 1};
  if (chunks <= 128) return {128, 1};
  if (chunks <= 256) return {256, 1};
  if (chunks <= 512) return {256, 2};
  if (chunks <= 1024) return {1024, 1};
  if (chunks <= 2048) return {1024, 2};
  return {1024, 0};
}
constexpr int kRowGrid = 1 << 16;   // workgroups at most; further rows are walked to

template <bool F32, int N, int MAXG>
hipError_t backward_shaped(const NormBackwardArgs &a, dim3 threads, int blocks, hipStream_t s) {
  if (!a.y)
    hipLaunchKernelGGL((norm_backward_kernel<F32, N, MAXG, NORM_PRE>), dim3(blocks), threads, 0,
                       s, a);
  else if (a.du)
    hipLaunchKernelGGL((norm_backward_kernel<F32, N, MAXG, NORM_BOTH>), dim3(blocks),
                       threads, 0, s, a);
  else
    hipLaunchKernelGGL((norm_backward_kernel<F32, N, MAXG, NORM_POST>), dim3(blocks),
                       threads, 0, s, a);
  return hipGetLastError();
}

// f(type, held, threads at most) with the row's shape as constants
template <class F>
hipError_t with_shape(Shape sh, bool f32, F f) {
  using std::integral_constant;
  auto typed = [&](auto F32) {
    if (sh.held == 0) return f(F32, integral_constant<int, 0>{}, integral_constant<int, 1024>{});
    if (sh.threads == 1024 && sh.held == 2)
      return f(F32, integral_constant<int, 2>{}, integral_constant<int, 1024>{});
    if (sh.threads == 1024) return f(F32, integral_constant<int, 1>{}, integral_constant<int, 1024>{});
    // bounded as for 512 threads: 256 registers, two waves per SIMD
    if (sh.held == 2) return f(F32, integral_constant<int, 2>{}, integral_constant<int, 512>{});
    return f(F32, integral_constant<int, 1>{}, integral_constant<int, 256>{});
  };
  return f32 ? typed(integral_constant<bool, true>{}) : typed(integral_constant<bool, false>{});
}

}  // namespace

// As many workgroups as run at once (eight waves on each of the 256 CUs, sixteen
// of rows of one wave; one workgroup at least; 1024 at most, whose parts are
// summed afterwards), and of those as many as share the rows evenly.  Four rows
// at a time: pre-norm and gradient of 16384 rows of 256 in 24.7 us, one at a time
// 40.5.
int norm_backward_blocks(int T, int h, int act_f32) {
  const int threads = shape_of(h, act_f32).threads;
  const int most = threads >= 512 ? 256 : threads >= 128 ? 131072 / threads : 1024;
  const int at_once = threads == kWave ? kRowWaves : 1, groups = (T + at_once - 1) / at_once;
  if (groups <= most) return groups;
  const int rows = (groups + most - 1) / most;
  return (groups + rows - 1) / rows;
}

hipError_t launch_prenorm(const PrenormArgs &a, hipStream_t s) {
  const Shape sh = shape_of(a.h, a.act_f32);
  return with_shape(sh, a.act_f32, [&](auto F32, auto N, auto G) {
    hipLaunchKernelGGL((prenorm_kernel<F32.value, N.value, G.value>),
                       dim3(a.T < kRowGrid ? a.T : kRowGrid), dim3(sh.threads), 0, s, a);
    return hipGetLastError();
  });
}

hipError_t launch_postnorm(const PostnormArgs &a, hipStream_t s) {
  const Shape sh = shape_of(a.h, a.act_f32);
  return with_shape(sh, a.act_f32, [&](auto F32, auto N, auto G) {
    hipLaunchKernelGGL((postnorm_kernel<F32.value, N.value, G.value>),
                       dim3(a.T < kRowGrid ? a.T : kRowGrid), dim3(sh.threads), 0, s, a);
    return hipGetLastError();
  });
}

hipError_t launch_norm_backward(const NormBackwardArgs &a, hipStream_t s) {
  const Shape sh = shape_of(a.h, a.act_f32);
  const int blocks = norm_backward_blocks(a.T, a.h, a.act_f32);
  const hipError_t e = with_shape(sh, a.act_f32, [&](auto F32, auto N, auto G) {
    return backward_shaped<F32.value, N.value, G.value>(
        a, dim3(sh.threads, sh.threads == kWave ? kRowWaves : 1), blocks, s);
  });
  if (e != hipSuccess) return e;
  ColumnSumArgs c;
  int n = 0;
  auto sum_of = [&](int which, void *out) {
    c.part[n] = a.part + (size_t)which * a.h;
    c.out[n++] = static_cast<float *>(out);
  };
  if (a.y) sum_of(0, a.dw);
  if (a.dw_next) sum_of(1, a.dw_next);
  if (a.gate_mode == DEAMOE_GATE_SHARED) sum_of(2, a.dgate);
  c.h = a.h;
  c.blocks = blocks;
  // Few columns: half a wave of them each, for twice the workgroups.  us of the
  // whole gradient, 64 | 32 columns: 8192 rows of 1024, 30 | 28; 64 of 7168, 16.5 |
  // 17.1.
  if (a.h <= 2048) hipLaunchKernelGGL(column_sum_kernel<32>, dim3((a.h + 31) / 32, n), dim3(1024), 0, s, c);
  else hipLaunchKernelGGL(column_sum_kernel<64>, dim3((a.h + 63) / 64, n), dim3(1024), 0, s, c);
  return hipGetLastError();
}

}  // namespace deamoe
