// Argument blocks and launchers of the operators beside the decode layer:
// sorted tokens (tokens.hip), 4-bit products (w4.hip), norms (norm.hip).
#pragma once

#include "internal.h"

namespace deamoe {

// 16-byte chunks of a row: kVec<f32> elements each.  Rows need only element
// alignment (an odd width starts every second bf16 row at 2 bytes): gfx950
// takes 16-byte global accesses at any address, so there is one access path,
// and only the chunk that holds the end of the row goes element by element.
template <bool F32>
inline constexpr int kVec = F32 ? 4 : 8;

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// STREAM: an access that keeps its lines out of the caches' way.  Loads of rows
// that are read once (8192 x 8 rows of 4096, 539 MB, collected in 101 us, not
// 119; 1024 x 8 in 13 us, not 19), and stores of more than the 256 MB of the
// last-level cache can keep for the next kernel (the same 539 MB dispatched in
// 94 us, not 113; of 67 MB no faster).
constexpr int64_t kStreamBytes = 256 << 20;

template <bool F32>
struct Chunk {
  u32x4 raw;
  __device__ float at(int i) const {
    if constexpr (F32) return __uint_as_float(raw[i]);
    return __uint_as_float(i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
  }
};

// Elements [c, c + kVec) of the row at p (h elements); zeros past the end.
template <bool F32, bool STREAM = false>
__device__ inline Chunk<F32> load_chunk(const void *p, int c, int h) {
  constexpr int V = kVec<F32>;
  Chunk<F32> r;
  const char *q = static_cast<const char *>(p) + (size_t)c * (F32 ? 4 : 2);
  if (c + V <= h) {
    const auto *v = reinterpret_cast<const u32x4_any *>(q);
    r.raw = STREAM ? __builtin_nontemporal_load(v) : *v;
  } else {
    r.raw = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (c + i < h) {
        if constexpr (F32) r.raw[i] = reinterpret_cast<const uint32_t *>(q)[i];
        else r.raw[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(q)[i] << (16 * (i & 1));
      }
  }
  return r;
}

template <bool F32, bool STREAM = false>
__device__ inline void store_chunk(void *p, int c, int h, const Chunk<F32> &r) {
  constexpr int V = kVec<F32>;
  char *q = static_cast<char *>(p) + (size_t)c * (F32 ? 4 : 2);
  if (c + V <= h) {
    auto *v = reinterpret_cast<u32x4_any *>(q);
    if constexpr (STREAM) __builtin_nontemporal_store((u32x4_any)r.raw, v);
    else *v = r.raw;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (c + i < h) {
        if constexpr (F32) reinterpret_cast<uint32_t *>(q)[i] = r.raw[i];
        else reinterpret_cast<uint16_t *>(q)[i] = (uint16_t)(r.raw[i / 2] >> (16 * (i & 1)));
      }
  }
}

// fp32 values rounded to the row's type (nearest even).
template <bool F32>
__device__ inline Chunk<F32> pack_chunk(const float (&v)[kVec<F32>]) {
  Chunk<F32> r;
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.raw[i] = __float_as_uint(v[i]);
  } else {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r.raw[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]});
  }
  return r;
}

// Row r of an [., h] matrix of the activation type.
template <bool F32>
__device__ inline const char *row_at(const void *p, size_t r, int h) {
  return static_cast<const char *>(p) + r * (size_t)h * (F32 ? 4 : 2);
}
template <bool F32>
__device__ inline char *row_at(void *p, size_t r, int h) {
  return static_cast<char *>(p) + r * (size_t)h * (F32 ? 4 : 2);
}

// ---- tokens.hip
struct DispatchArgs {
  int32_t T, k, n, h, act_f32;
  const int32_t *ids;
  const void *x;
  int32_t *offset, *pair, *row;
  void *xs;                 // NULL: lists only
  int32_t *hist, *total;    // workspace of a large sort
};
constexpr int kSortSmallPairs = 4096;   // up to here one launch sorts and gathers
// Pairs that one workgroup of a large sort counts and ranks: few, so that many
// workgroups share the work, until their counts per group would outgrow the
// caches.
constexpr int kSortChunk = 512, kSortChunkLarge = 4096;
inline int sort_chunk(int64_t pairs) { return pairs <= 1 << 18 ? kSortChunk : kSortChunkLarge; }
hipError_t launch_dispatch(const DispatchArgs &a, hipStream_t s);
hipError_t launch_zero(void *p, size_t bytes, hipStream_t s);   // multiples of 4 bytes

struct CollectArgs {
  int32_t T, k, h, act_f32;
  const int32_t *row;
  const float *w;           // NULL: ones
  const void *ys;
  void *y;
};
hipError_t launch_collect(const CollectArgs &a, hipStream_t s);

struct CollectBackwardArgs {
  int32_t T, k, h, act_f32;
  const int32_t *row;
  const float *w;
  const void *ys, *dy;
  void *dys;
  float *dw;
};
hipError_t launch_collect_backward(const CollectBackwardArgs &a, hipStream_t s);

// ---- w4.hip
struct W4Args {
  int32_t M, R, K, n, group, scale_bf16;
  const void *x;
  const int32_t *offset;
  const void *w[2], *scale[2];   // gate and up, or one matrix
  void *y;
};
// Workgroups of the streaming kernel that a CU holds at once.  A workgroup is a
// wave on each of the four SIMDs: three fit up to 168 registers and 53 KB of LDS.
// Two matrices in groups of 32 take 169, four weight tiles (nr) per wave about 256,
// two token tiles (ntt) 209 to 233 and 73 KB; a wide panel takes the LDS for itself.
constexpr int stream_resident(int mats, int nr, int ntt, int group, bool wide) {
  return wide ? 1 : nr > 1 || ntt > 1 || (mats == 2 && group == 32) ? 2 : 3;
}
hipError_t launch_w4(const W4Args &a, int mats, hipStream_t s);

// ---- norm.hip
struct PrenormArgs {
  int32_t T, h, act_f32;
  float eps;
  const void *x, *w;
  void *u;
};
struct PostnormArgs {
  int32_t T, h, act_f32, gate_mode;
  float eps, res_scale;
  const void *x, *y, *w, *gate, *w_next;
  void *z, *u;
};
// The gradients of both: prenorm's x, w, du, dres and dx, dw stand in z,
// w_next, du, dz and dx, dw_next, and y is NULL.
struct NormBackwardArgs {
  int32_t T, h, act_f32, gate_mode;
  float eps, res_scale;
  const void *y, *w, *gate, *z, *w_next, *dz, *du;
  void *dx, *dy, *dgate;
  float *dw, *dw_next;
  float *part;              // workspace: [blocks, 3, h]
};
int norm_backward_blocks(int T, int h, int act_f32);
hipError_t launch_prenorm(const PrenormArgs &a, hipStream_t s);
hipError_t launch_postnorm(const PostnormArgs &a, hipStream_t s);
hipError_t launch_norm_backward(const NormBackwardArgs &a, hipStream_t s);

}  // namespace deamoe
