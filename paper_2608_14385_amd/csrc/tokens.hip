// Tokens sorted by expert, and back with their routing weights.
//
// The sort is a stable counting sort of the pairs p = t * k + s by their group:
//   row_p = #{q : key_q < key_p} + #{q < p : key_q = key_p}
// Counts are sums of integers and ranks follow the pair order, so the lists do
// not depend on the order in which workgroups run.
#include <type_traits>

#include "ops.h"

namespace deamoe {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// Group of an id; dropped pairs get n.
__device__ inline int key_of(int id, int n) { return (uint32_t)id < (uint32_t)n ? id : n; }

// Exclusive prefix of v over the workgroup's threads, and the workgroup's sum.
__device__ inline int block_exclusive(int v, int *s_wave, int &sum) {
  const int lane = threadIdx.x % kWave, wv = threadIdx.x / kWave;
  int inc = v;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int o = __shfl_up(inc, d);
    inc += lane >= d ? o : 0;
  }
  __syncthreads();   // the last use of s_wave
  if (lane == kWave - 1) s_wave[wv] = inc;
  __syncthreads();
  int base = 0;
  sum = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    base += i < wv ? s_wave[i] : 0;
    sum += s_wave[i];
  }
  return base + inc - v;
}

// counts[0 .. n) in LDS become their exclusive prefix; returns the sum.
__device__ inline int scan_counts(int *counts, int n, int *s_wave) {
  const int per = (n + kThreads - 1) / kThreads, lo = threadIdx.x * per;
  int v = 0, sum;
  for (int i = lo; i < min(lo + per, n); ++i) v += counts[i];
  int at = block_exclusive(v, s_wave, sum);
  for (int i = lo; i < min(lo + per, n); ++i) {
    const int c = counts[i];
    counts[i] = at;
    at += c;
  }
  __syncthreads();
  return sum;
}

// Chunks of x of one token stored to its rows.
template <bool F32, bool STREAM = false>
__device__ inline void scatter_row(const DispatchArgs &a, const int *rows, int c,
                                   const Chunk<F32> &v) {
  for (int s = 0; s < a.k; ++s) {
    const int r = rows[s];
    if (r >= 0) store_chunk<F32, STREAM>(row_at<F32>(a.xs, r, a.h), c, a.h, v);
  }
}

}  // namespace

// Sort and gather of at most kSortSmallPairs pairs in one launch.  Workgroup
// (t, y) counts the rows before each of its token's pairs itself, by comparing
// all pairs with them, and stores part y of the token's row; the
// last workgroup writes the offsets and the unused tail of `pair`.  10 pairs and
// rows of 1024 take 3.8 us, bound by a launch and three round trips to memory,
// where a sort in steps would take as many launches.
template <bool F32>
__global__ __launch_bounds__(kThreads) void dispatch_small_kernel(DispatchArgs a) {
  __shared__ int s_count[DEAMOE_MAX_EXPERTS];
  __shared__ int s_wave[kWaves];
  __shared__ int s_part[DEAMOE_MAX_TOPK][kWaves];
  __shared__ int s_row[DEAMOE_MAX_TOPK];
  const int P = a.T * a.k, tid = threadIdx.x;
  if ((int)blockIdx.x == a.T) {
    if (blockIdx.y) return;
    for (int e = tid; e < a.n; e += kThreads) s_count[e] = 0;
    __syncthreads();
    for (int p = tid; p < P; p += kThreads) {
      const int e = key_of(a.ids[p], a.n);
      if (e < a.n) atomicAdd(&s_count[e], 1);
    }
    __syncthreads();
    const int used = scan_counts(s_count, a.n, s_wave);
    for (int e = tid; e < a.n; e += kThreads) a.offset[e] = s_count[e];
    if (tid == 0) a.offset[a.n] = used;
    for (int p = used + tid; p < P; p += kThreads) a.pair[p] = -1;
    return;
  }
  const int t = blockIdx.x, c = (blockIdx.y * kThreads + tid) * kVec<F32>;
  Chunk<F32> v;
  if (a.xs && c < a.h) v = load_chunk<F32>(row_at<F32>(a.x, t, a.h), c, a.h);
  // (group, pair) as one number: groups and pairs take 12 bits and 13 bits
  const int lane = tid % kWave, wv = tid / kWave;
  for (int s0 = 0; s0 < a.k; s0 += 8) {
    int mine[8], count[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = t * a.k + min(s0 + i, a.k - 1);
      mine[i] = key_of(a.ids[p], a.n) << 13 | p;
      count[i] = 0;
    }
    for (int q0 = wv * kWave; q0 < P; q0 += kThreads) {
      const int q = q0 + lane;
      const int other = q < P ? key_of(a.ids[q], a.n) << 13 | q : 0x7fffffff;
#pragma unroll
      for (int i = 0; i < 8; ++i) count[i] += __popcll(__ballot(other < mine[i]));
    }
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (s0 + i < a.k) s_part[s0 + i][wv] = count[i];
  }
  __syncthreads();
  if (tid < a.k) {
    int r = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) r += s_part[tid][i];
    const int p = t * a.k + tid;
    const bool held = (uint32_t)a.ids[p] < (uint32_t)a.n;
    s_row[tid] = held ? r : -1;
    if (blockIdx.y == 0) {
      a.row[p] = held ? r : -1;
      if (held) a.pair[r] = p;
    }
  }
  __syncthreads();
  if (a.xs && c < a.h) scatter_row<F32>(a, s_row, c, v);
}

// Large sorts: counts per (group, chunk of pairs) ...  65536 pairs of 128 groups
// take 4.8 + 4.5 + 4.8 us in the three kernels, bound by their launches and
// round trips: 0.3 MB is read.
template <int CHUNK>
__global__ __launch_bounds__(kThreads) void sort_count_kernel(DispatchArgs a, int chunks) {
  __shared__ int s_count[DEAMOE_MAX_EXPERTS];
  const int P = a.T * a.k;
  for (int e = threadIdx.x; e < a.n; e += kThreads) s_count[e] = 0;
  __syncthreads();
  const int lo = blockIdx.x * CHUNK, hi = min(lo + CHUNK, P);
  for (int p = lo + threadIdx.x; p < hi; p += kThreads) {
    const int e = key_of(a.ids[p], a.n);
    if (e < a.n) atomicAdd(&s_count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.n; e += kThreads)
    a.hist[(size_t)e * chunks + blockIdx.x] = s_count[e];
}

// ... become, per group, the exclusive prefix over the chunks and the total ...
__global__ __launch_bounds__(kThreads) void sort_scan_kernel(DispatchArgs a, int chunks) {
  __shared__ int s_wave[kWaves];
  int32_t *h = a.hist + (size_t)blockIdx.x * chunks;
  int base = 0;
  for (int c0 = 0; c0 < chunks; c0 += kThreads) {
    const int c = c0 + threadIdx.x;
    const int v = c < chunks ? h[c] : 0;
    int sum;
    const int at = base + block_exclusive(v, s_wave, sum);
    if (c < chunks) h[c] = at;
    base += sum;
  }
  if (threadIdx.x == 0) a.total[blockIdx.x] = base;
}

// ... from which every chunk ranks its pairs.  Each wave takes a quarter of the
// chunk, 64 pairs at a time: the lanes of one group find each other by one
// ballot per bit of the group number.
template <int CHUNK>
__global__ __launch_bounds__(kThreads) void sort_rank_kernel(DispatchArgs a, int chunks) {
  __shared__ int s_offset[DEAMOE_MAX_EXPERTS];
  __shared__ int s_next[kWaves][DEAMOE_MAX_EXPERTS];   // next row of a group, per wave
  __shared__ int s_wave[kWaves];
  const int n = a.n, P = a.T * a.k, tid = threadIdx.x;
  const int lane = tid % kWave, wv = tid / kWave;
  for (int e = tid; e < n; e += kThreads) {
    s_offset[e] = a.total[e];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s_next[w][e] = 0;
  }
  __syncthreads();
  const int used = scan_counts(s_offset, n, s_wave);
  if (blockIdx.x == 0) {
    for (int e = tid; e < n; e += kThreads) a.offset[e] = s_offset[e];
    if (tid == 0) a.offset[n] = used;
  }
  constexpr int kPart = CHUNK / kWaves, kRounds = kPart / kWave;
  const int lo = blockIdx.x * CHUNK + wv * kPart;
  int key[kRounds];
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int p = lo + i * kWave + lane;
    key[i] = p < P ? key_of(a.ids[p], n) : n;
    if (key[i] < n) atomicAdd(&s_next[wv][key[i]], 1);
    if (p < P && p >= used) a.pair[p] = -1;
  }
  __syncthreads();
  for (int e = tid; e < n; e += kThreads) {
    int at = s_offset[e] + a.hist[(size_t)e * chunks + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int c = s_next[w][e];
      s_next[w][e] = at;
      at += c;
    }
  }
  __syncthreads();
  const int bits = 32 - __clz(n - 1);   // n == 1: 0
  volatile int *next = s_next[wv];
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int p = lo + i * kWave + lane;
    const bool held = key[i] < n;
    uint64_t same = __ballot(held);
    for (int b = 0; b < bits; ++b) {
      const bool one = key[i] >> b & 1;
      const uint64_t m = __ballot(one);
      same &= one ? m : ~m;
    }
    if (held) {
      const int before = __popcll(same & ((1ull << lane) - 1ull));
      const int r = next[key[i]] + before;
      a.row[p] = r;
      a.pair[r] = p;
      if (before == 0) next[key[i]] = r + __popcll(same);
    } else if (p < P) {
      a.row[p] = -1;
    }
  }
}

// Every token's row read once and stored to its k rows.  8192 tokens of 4096 bf16
// columns to 8 groups each, a few dropped, move 571 MB in 102 us: 5.6 TB/s, bound
// by HBM's stores.
template <bool F32, bool STREAM>
__global__ __launch_bounds__(kThreads) void gather_rows_kernel(DispatchArgs a) {
  const int t = blockIdx.x, c = (blockIdx.y * kThreads + threadIdx.x) * kVec<F32>;
  if (c >= a.h) return;
  scatter_row<F32, STREAM>(a, a.row + (size_t)t * a.k, c,
                   load_chunk<F32>(row_at<F32>(a.x, t, a.h), c, a.h));
}

namespace {

template <bool F32>
hipError_t dispatch_typed(const DispatchArgs &a, hipStream_t s) {
  const int per = kThreads * kVec<F32>, parts = a.xs ? (a.h + per - 1) / per : 1;
  const int64_t P = (int64_t)a.T * a.k;
  if (P <= kSortSmallPairs) {
    hipLaunchKernelGGL(dispatch_small_kernel<F32>, dim3(a.T + 1, parts), dim3(kThreads), 0, s, a);
    return hipGetLastError();
  }
  const int chunk = sort_chunk(P), chunks = (int)((P + chunk - 1) / chunk);
  auto sort = [&](auto C) {
    constexpr int CHUNK = decltype(C)::value;
    hipLaunchKernelGGL(sort_count_kernel<CHUNK>, dim3(chunks), dim3(kThreads), 0, s, a, chunks);
    hipLaunchKernelGGL(sort_scan_kernel, dim3(a.n), dim3(kThreads), 0, s, a, chunks);
    hipLaunchKernelGGL(sort_rank_kernel<CHUNK>, dim3(chunks), dim3(kThreads), 0, s, a, chunks);
  };
  if (chunk == kSortChunk) sort(std::integral_constant<int, kSortChunk>{});
  else sort(std::integral_constant<int, kSortChunkLarge>{});
  if (a.xs && P * a.h * (F32 ? 4 : 2) > kStreamBytes)
    hipLaunchKernelGGL((gather_rows_kernel<F32, true>), dim3(a.T, parts), dim3(kThreads), 0, s, a);
  else if (a.xs)
    hipLaunchKernelGGL((gather_rows_kernel<F32, false>), dim3(a.T, parts), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dispatch(const DispatchArgs &a, hipStream_t s) {
  return a.act_f32 ? dispatch_typed<true>(a, s) : dispatch_typed<false>(a, s);
}

__global__ __launch_bounds__(kThreads) void zero_kernel(uint32_t *p, size_t words) {
  const size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < words) p[i] = 0;
}

hipError_t launch_zero(void *p, size_t bytes, hipStream_t s) {
  const size_t words = bytes / 4;
  hipLaunchKernelGGL(zero_kernel, dim3((unsigned)((words + kThreads - 1) / kThreads)),
                     dim3(kThreads), 0, s, static_cast<uint32_t *>(p), words);
  return hipGetLastError();
}

// y[t] = sum over the token's held pairs, in slot order, of w * ys[row].  The
// loads of a batch of slots are all issued before the batch is summed.  The same
// 571 MB the other way take 102 us, bound by HBM; 61 tokens of 7168, 8 MB, take
// 3.8 us.
template <bool F32>
__global__ __launch_bounds__(kThreads) void collect_kernel(CollectArgs a) {
  constexpr int U = 8, V = kVec<F32>;
  const int t = blockIdx.x, c = (blockIdx.y * blockDim.x + threadIdx.x) * V;
  if (c >= a.h) return;
  const int32_t *row = a.row + (size_t)t * a.k;
  const float *w = a.w ? a.w + (size_t)t * a.k : nullptr;
  const int rows = a.T * a.k;
  float acc[V] = {};
  for (int s0 = 0; s0 < a.k; s0 += U) {
    Chunk<F32> v[U];
    float f[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = s0 + u < a.k ? row[s0 + u] : -1;
      v[u].raw = u32x4{0, 0, 0, 0};
      f[u] = 0.f;
      if ((uint32_t)r < (uint32_t)rows) {
        v[u] = load_chunk<F32, true>(row_at<F32>(a.ys, r, a.h), c, a.h);
        f[u] = w ? w[s0 + u] : 1.f;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] = __builtin_fmaf(f[u], v[u].at(i), acc[i]);
  }
  store_chunk<F32>(row_at<F32>(a.y, t, a.h), c, a.h, pack_chunk<F32>(acc));
}

hipError_t launch_collect(const CollectArgs &a, hipStream_t s) {
  const int per = kThreads * (a.act_f32 ? 4 : 8);
  const dim3 grid(a.T, (a.h + per - 1) / per);
  if (a.act_f32) hipLaunchKernelGGL(collect_kernel<true>, grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(collect_kernel<false>, grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

// dys[row] = w * dy[t] and dw = <dy[t], ys[row]>: one workgroup per token, a
// batch of slots at a time; each thread's products of a slot are summed over
// its columns, then over the wave, then over the waves.  The same sizes read 571
// MB and write 504 in 211 us: 5.1 TB/s, bound by HBM.
template <bool F32, bool STREAM>
__global__ __launch_bounds__(kThreads) void collect_backward_kernel(CollectBackwardArgs a) {
  constexpr int U = 4, V = kVec<F32>;
  __shared__ float s_dot[DEAMOE_MAX_TOPK][kWaves];
  const int t = blockIdx.x, tid = threadIdx.x;
  const int32_t *row = a.row + (size_t)t * a.k;
  const float *w = a.dys ? a.w + (size_t)t * a.k : nullptr;
  const int rows = a.T * a.k;
  for (int s0 = 0; s0 < a.k; s0 += U) {
    int r[U];
    float f[U], dot[U] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u] = s0 + u < a.k ? row[s0 + u] : -1;
      if ((uint32_t)r[u] >= (uint32_t)rows) r[u] = -1;
      f[u] = r[u] >= 0 && w ? w[s0 + u] : 0.f;
    }
    for (int c = tid * V; c < a.h; c += kThreads * V) {
      const Chunk<F32> d = load_chunk<F32>(row_at<F32>(a.dy, t, a.h), c, a.h);
      Chunk<F32> v[U];
      if (a.dw)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          v[u].raw = u32x4{0, 0, 0, 0};
          if (r[u] >= 0) v[u] = load_chunk<F32, true>(row_at<F32>(a.ys, r[u], a.h), c, a.h);
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (r[u] < 0) continue;
        if (a.dw)
#pragma unroll
          for (int i = 0; i < V; ++i) dot[u] = __builtin_fmaf(d.at(i), v[u].at(i), dot[u]);
        if (a.dys) {
          float g[V];
#pragma unroll
          for (int i = 0; i < V; ++i) g[i] = f[u] * d.at(i);
          store_chunk<F32, STREAM>(row_at<F32>(a.dys, r[u], a.h), c, a.h, pack_chunk<F32>(g));
        }
      }
    }
    if (a.dw)
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int o = kWave / 2; o; o /= 2) dot[u] += __shfl_xor(dot[u], o);
        if (tid % kWave == 0 && s0 + u < a.k) s_dot[s0 + u][tid / kWave] = dot[u];
      }
  }
  if (!a.dw) return;
  __syncthreads();
  if (tid < a.k) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) v += s_dot[tid][i];
    a.dw[(size_t)t * a.k + tid] = v;
  }
}

hipError_t launch_collect_backward(const CollectBackwardArgs &a, hipStream_t s) {
  const bool stream = (int64_t)a.T * a.k * a.h * (a.act_f32 ? 4 : 2) > kStreamBytes;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.T), dim3(kThreads), 0, s, a); };
  if (a.act_f32) launch(stream ? collect_backward_kernel<true, true> : collect_backward_kernel<true, false>);
  else launch(stream ? collect_backward_kernel<false, true> : collect_backward_kernel<false, false>);
  return hipGetLastError();
}

}  // namespace deamoe
