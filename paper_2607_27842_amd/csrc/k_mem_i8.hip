// The feature history in 8-bit integers (Eq. 2): a slot holds a sample's values in blocks of 128, each
// with its scale, written as a refresh forms them and read back by the draft and the verify pass.  The blocks of a
// sample start at its first value, so that no block reaches over two samples.
#include "i8_common.h"

namespace ff {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 16;   // values a lane: 16 bytes of a slot; 8 lanes hold a block
constexpr int kMaxGroups = 2048;

// 8 values of a tensor's sample, zeros past its end (the sample's size is a multiple of 8)
template <int DT>
__device__ __forceinline__ void load_in(const void* p, size_t base, size_t i, size_t n, float* v) {
#pragma unroll
  for (int h = 0; h < kPer; h += 8) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[h + e] = 0.f;
    if (i + h < n) load8<DT>(p, base + i + h, v + h);
  }
}
template <int DT>
__device__ __forceinline__ void store_in(void* p, size_t base, size_t i, size_t n, const float* v) {
#pragma unroll
  for (int h = 0; h < kPer; h += 8)
    if (i + h < n) store8<DT>(p, base + i + h, v + h);
}

// Delta = h - u (or h) in fp32, then its blocks.  Values past the sample's end are written as zeros.
template <int DT, bool RES>
__global__ __launch_bounds__(kThreads) void k_cache_update_i8(uint8_t* __restrict__ slot, float* __restrict__ scales,
                                                              const void* __restrict__ u, const void* __restrict__ h, size_t n,
                                                              size_t blocks) {
  const size_t base = (size_t)blockIdx.y * n, q0 = (size_t)blockIdx.y * blocks * kI8Block;
  for (size_t c = (size_t)blockIdx.x * kThreads + threadIdx.x; c < blocks * 8; c += (size_t)gridDim.x * kThreads) {
    const size_t i = c * kPer;
    float v[kPer];
    load_in<DT>(h, base, i, n, v);
    if (RES) {
      float x[kPer];
      load_in<DT>(u, base, i, n, x);
#pragma unroll
      for (int e = 0; e < kPer; ++e) v[e] -= x[e];
    }
    const I8Scale k(top8(top_bits<kPer>(v)));
    u32x4_t w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = i8_pack4(v + 4 * e, k);
    *reinterpret_cast<u32x4_t*>(slot + q0 + i) = w;
    if ((c & 7) == 0) scales[(size_t)blockIdx.y * blocks + c / 8] = k.s;
  }
}

// 16 values of the draft h_d = u + sum_m c_m s_m q_m: fp32 sums in the order of the terms, one rounding
template <int DT, bool RES>
__device__ __forceinline__ void draft_chunk_i8(const TermsI8& t, const void* u, size_t base, size_t n, size_t c, size_t q0, size_t s0, float* out) {
  const size_t i = c * kPer;
  float f[kPer];
  load_in<DT>(RES ? u : nullptr, base, i, RES ? n : 0, out);
#pragma unroll
  for (int e = 0; e < kPer; ++e) f[e] = 0.f;
#pragma unroll
  for (int m = 0; m < kMaxTerms; ++m) {
    if (m >= t.n) continue;
    const u32x4_t w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(t.slot[m] + q0 + i));
    const float s = t.scales[m][s0 + c / 8];
    float q[kPer];
#pragma unroll
    for (int e = 0; e < 4; ++e) i8_unpack4(w[e], q + 4 * e);
#pragma unroll
    for (int e = 0; e < kPer; ++e) f[e] = fmaf(t.c[m], s * q[e], f[e]);
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e) out[e] = St<DT>::rnd(RES ? out[e] + f[e] : f[e]);
}

template <int DT, bool RES>
__global__ __launch_bounds__(kThreads) void k_draft_i8(TermsI8 t, const void* u, void* hd, size_t n, size_t blocks) {
  const size_t base = (size_t)blockIdx.y * n, s0 = (size_t)blockIdx.y * blocks, q0 = s0 * kI8Block;
  for (size_t c = (size_t)blockIdx.x * kThreads + threadIdx.x; c < blocks * 8; c += (size_t)gridDim.x * kThreads) {
    float o[kPer];
    draft_chunk_i8<DT, RES>(t, u, base, n, c, q0, s0, o);
    store_in<DT>(hd, base, c * kPer, n, o);
  }
}

// Verify and replace (Eq. 3-5) on that draft: what k_verify does, with the same two-stage sums
template <int DT, bool RES>
__global__ __launch_bounds__(kThreads) void k_verify_i8(TermsI8 t, const void* u, const void* __restrict__ hf, void* hout, Forward fw,
                                                        size_t n, size_t blocks, float* __restrict__ partials) {
  __shared__ float red[2][kThreads / 64];
  const size_t base = (size_t)blockIdx.y * n, s0 = (size_t)blockIdx.y * blocks, q0 = s0 * kI8Block;
  float num = 0.f, den = 0.f;
  for (size_t c = (size_t)blockIdx.x * kThreads + threadIdx.x; c < blocks * 8; c += (size_t)gridDim.x * kThreads) {
    const size_t i = c * kPer;
    float d[kPer], f[kPer];
    draft_chunk_i8<DT, RES>(t, u, base, n, c, q0, s0, d);
    load_in<DT>(hf, base, i, n, f);
#pragma unroll
    for (int h = 0; h < kPer; h += 8) {
      if (i + h >= n) continue;
#pragma unroll
      for (int e = h; e < h + 8; ++e) {
        num += fabsf(d[e] - f[e]);
        den += fabsf(f[e]);
      }
      if (fw.kind >= FWD_TOKENS) {   // 8 values lie in one row (C % 8 == 0)
        const int row = (int)((i + h) / fw.C), ch = (int)((i + h) % fw.C);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool exact = fw.kind == FWD_TOKENS ? row % fw.stride == 0 : (ch + e) % fw.stride == 0;
          d[h + e] = exact ? f[h + e] : d[h + e];
        }
      }
    }
    store_in<DT>(hout, base, i, n, fw.kind == FWD_EXACT ? f : d);
  }
  num = wave_sum(num);
  den = wave_sum(den);
  if ((threadIdx.x & 63) == 0) { red[0][threadIdx.x >> 6] = num; red[1][threadIdx.x >> 6] = den; }
  __syncthreads();
  if (threadIdx.x == 0) {
    float* p = partials + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2;
    p[0] = (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]);
    p[1] = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  }
}

int groups_for(size_t blocks) {
  const size_t g = (blocks * 8 + kThreads - 1) / kThreads;
  return (int)(g > kMaxGroups ? kMaxGroups : g);
}

}  // namespace

#define FF_BY_TYPE(kernel, res, ...)                                                     \
  do {                                                                                   \
    if (dtype == DT_BF16) {                                                              \
      if (res) FF_LAUNCH((kernel<DT_BF16, true>), grid, kThreads, 0, s, __VA_ARGS__);    \
      else FF_LAUNCH((kernel<DT_BF16, false>), grid, kThreads, 0, s, __VA_ARGS__);       \
    } else {                                                                             \
      if (res) FF_LAUNCH((kernel<DT_F32, true>), grid, kThreads, 0, s, __VA_ARGS__);     \
      else FF_LAUNCH((kernel<DT_F32, false>), grid, kThreads, 0, s, __VA_ARGS__);        \
    }                                                                                    \
  } while (0)

hipError_t cache_update_i8(int dtype, uint8_t* slot, float* scales, const void* u, const void* h, int B, size_t n, hipStream_t s) {
  const size_t blocks = i8_blocks(n);
  const dim3 grid(groups_for(blocks), B);
  FF_BY_TYPE(k_cache_update_i8, u != nullptr, slot, scales, u, h, n, blocks);
  return hipGetLastError();
}

hipError_t draft_i8(int dtype, const TermsI8& t, const void* u, void* hd, int B, size_t n, hipStream_t s) {
  const size_t blocks = i8_blocks(n);
  const dim3 grid(groups_for(blocks), B);
  FF_BY_TYPE(k_draft_i8, u != nullptr, t, u, hd, n, blocks);
  return hipGetLastError();
}

hipError_t verify_i8(int dtype, const TermsI8& t, const void* u, const void* hf, void* hout, const Forward& fw, int B, size_t n,
                     float eps, float* rel, float* partials, hipStream_t s) {
  const size_t blocks = i8_blocks(n);
  const dim3 grid(groups_for(blocks), B);
  FF_BY_TYPE(k_verify_i8, u != nullptr, t, u, hf, hout, fw, n, blocks, partials);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !rel) return e;
  return verify_finish(partials, B, grid.x, eps, rel, s);
}
#undef FF_BY_TYPE

}  // namespace ff
