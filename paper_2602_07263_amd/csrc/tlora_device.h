// Device helpers that several kernel files share: vector types, 16-byte accesses, conversions, sums.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tlora_kernels.h"

namespace tlora {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u32x4 ldg16(const void* p) { return *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 v = {(__bf16)lo, (__bf16)hi};   // round-to-nearest-even
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float bf16_float(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }

// Eight consecutive elements from i on (16-byte aligned), bf16 (BF) or fp32.
template <bool BF>
__device__ __forceinline__ void load8(const void* p, int64_t i, float (&v)[8]) {
  if (BF) {
    const u32x4 r = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __builtin_bit_cast(float, r[e] << 16);
      v[2 * e + 1] = __builtin_bit_cast(float, r[e] & 0xffff0000u);
    }
  } else {
    const f32x4* f = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i);
    const f32x4 a = f[0], b = f[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e];  v[4 + e] = b[e]; }
  }
}
template <bool BF>
__device__ __forceinline__ void store8(void* p, int64_t i, const float (&v)[8]) {
  if (BF) {
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + i) =
        u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  } else {
    f32x4* f = reinterpret_cast<f32x4*>(static_cast<float*>(p) + i);
    f[0] = f32x4{v[0], v[1], v[2], v[3]};
    f[1] = f32x4{v[4], v[5], v[6], v[7]};
  }
}
// sum over the 256 threads of a workgroup (every thread gets the total)
__device__ __forceinline__ float block_sum(float x, float* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  const float t = red[0] + red[1] + red[2] + red[3];
  __syncthreads();
  return t;
}

// op over lanes l, l ^ 16, l ^ 32, l ^ 48, in registers (row swaps of the lane's value with itself).
template <class Op>
__device__ __forceinline__ float across_16_32(float x, const Op& op) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  x = op(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
  const auto h = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  return op(__builtin_bit_cast(float, (uint32_t)h[0]), __builtin_bit_cast(float, (uint32_t)h[1]));
}
// Sum over the wave, in registers, in a fixed order; every lane gets it.  (The backward of the norms, 31744 x 4096 bf16, took 446 us
// while its sums were exchanges through LDS, one after the other, and 405 with these.)
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float row_sum(float x) {      // of the lane's 16
  x += dpp<0xB1>(x);       // lanes l ^ 1
  x += dpp<0x4E>(x);       // l ^ 2
  x += dpp<0x141>(x);      // the other four of eight
  x += dpp<0x140>(x);      // the other eight of sixteen
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
  x = row_sum(x);
  return across_16_32(x, [](float a, float b) { return a + b; });
}

// Tile L of the walk: groups of 4 row tiles, so that workgroups that run together share activation and weight panels.
__device__ __forceinline__ void gemm_tile_of(int L, int tiles_m, int tiles_n, int& tm, int& tn) {
  constexpr int GM = 4;
  const int per_group = GM * tiles_n;
  const int grp = L / per_group, first_m = grp * GM;
  const int gsize = min(GM, tiles_m - first_m);
  const int Lg = L - grp * per_group;
  // (the divisions run on the vector ALU; everything derived from the tile id is wave-uniform and belongs in
  // scalar registers)
  tm = __builtin_amdgcn_readfirstlane(first_m + Lg % gsize);
  tn = __builtin_amdgcn_readfirstlane(Lg / gsize);
}

enum { kHeadNone = 0, kHeadLogits = 1, kHeadGrad = 2 };
struct HeadShape {
  int rows, tiles_m;
  GemmSplit split;
};
// Rows of the piece that are there, and how a product's tiles are cut along K: whole rounds of 256 tiles (the chip's CUs) as they are,
// the rest into as many shares as fill one round or two, whichever ends first: a round of shares takes their K-steps and, for what it
// writes and the reduction reads again, as long as 32 steps (256 tiles of 256 rows, twice 64 MB).
__device__ __forceinline__ HeadShape head_shape(const HeadParams& h, int tiles_n, int steps) {
  HeadShape s;
  s.rows = __builtin_amdgcn_readfirstlane(min(max(*h.live - h.first, 0), h.max_rows));
  s.tiles_m = (s.rows + kGemmBM - 1) / kGemmBM;
  const int tiles = s.tiles_m * tiles_n, rest = tiles & 255;
  s.split.n_direct = tiles;
  if (rest) {
    const int extra = 32 * min(s.rows, kGemmBM) / kGemmBM, most = min(kHeadMaxSplits, max(steps / kHeadShare, 1));
    const int s1 = min(256 / rest, most), s2 = min(512 / rest, most);
    const int cost1 = s1 > 1 ? (steps + s1 - 1) / s1 + extra : steps, cost2 = 2 * ((steps + s2 - 1) / s2 + extra);
    s.split.splits = __builtin_amdgcn_readfirstlane(cost2 < cost1 && rest * s2 > 256 ? s2 : s1 > 1 && cost1 < steps ? s1 : 1);
    if (s.split.splits > 1) s.split.n_direct = tiles - rest;
  }
  return s;
}

}  // namespace tlora
