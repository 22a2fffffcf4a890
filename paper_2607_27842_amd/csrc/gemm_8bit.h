// What the products of 8-bit operands share: loads of 4 and 8 values in the output's type, and the order of
// tiles.
#pragma once
#include "dev_common.h"

namespace ff {

template <int DT>
__device__ __forceinline__ f32x4_t load4(const void* p, size_t i) {
  if (DT == DT_F32) return *reinterpret_cast<const f32x4_t*>(reinterpret_cast<const float*>(p) + i);
  const u32x2_t w = *reinterpret_cast<const u32x2_t*>(reinterpret_cast<const uint16_t*>(p) + i);
  return f32x4_t{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
}

// 8 values as they are stored, to be added later
template <int DT> struct Raw8;
template <> struct Raw8<DT_BF16> {
  typedef u32x4_t type;
  __device__ __forceinline__ static type load(const void* p, size_t i) { return *reinterpret_cast<const u32x4_t*>(reinterpret_cast<const uint16_t*>(p) + i); }
  __device__ __forceinline__ static float at(const type& w, int e) { return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16); }
  __device__ __forceinline__ static void add(type w, float* v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += at(w, e);
  }
};
template <> struct Raw8<DT_F32> {
  struct type { f32x4_t x[2]; };
  __device__ __forceinline__ static type load(const void* p, size_t i) {
    const f32x4_t* q = reinterpret_cast<const f32x4_t*>(reinterpret_cast<const float*>(p) + i);
    return type{{q[0], q[1]}};
  }
  __device__ __forceinline__ static float at(const type& w, int e) { return w.x[e / 4][e % 4]; }
  __device__ __forceinline__ static void add(const type& w, float* v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += at(w, e);
  }
};

// Workgroup -> tile: workgroups go round-robin over the 8 XCDs, so every XCD gets a contiguous range
// of tiles, in groups of 8 tile rows, whose operand rows its L2 then shares.
__device__ __forceinline__ void tile_at(int wg, int n, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int full = n / 8 * 8;
  const int id = wg < full ? (wg % 8) * (full / 8) + wg / 8 : wg;
  const int per = 8 * tiles_n, first = id / per * 8, size = min(tiles_m - first, 8), in = id % per;
  tm = __builtin_amdgcn_readfirstlane(first + in % size);
  tn = __builtin_amdgcn_readfirstlane(in / size);
}

}  // namespace ff
