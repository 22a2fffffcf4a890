// The feature history in 8-bit integers (Eq. 2): a slot holds a sample's values in blocks of 128, each
// with its scale, written as a refresh forms them and read back by the draft and the verify pass.  The blocks of a
// sample start at its first value, so that no block reaches over two samples.
#include "i8_common.h"

namespace ff {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;   // values a lane; 16 lanes hold a block
constexpr int kMaxGroups = kMaxVerifyBlocks;   // a sample; the verify pass keeps two sums of each

// Delta = h - u (or h) in fp32, then its blocks.  Values past the sample's end are written as zeros.  A sample's size is a
// multiple of 8.
template <int DT, bool RES>
__global__ __launch_bounds__(kThreads) void k_cache_update_i8(uint8_t* __restrict__ slot, float* __restrict__ scales,
                                                              const void* __restrict__ u, const void* __restrict__ h, size_t n,
                                                              size_t blocks) {
  const size_t base = (size_t)blockIdx.y * n, q0 = (size_t)blockIdx.y * blocks * kI8Block;
  for (size_t c = (size_t)blockIdx.x * kThreads + threadIdx.x; c < blocks * (kI8Block / kPer); c += (size_t)gridDim.x * kThreads) {
    const size_t i = c * kPer;
    float v[kPer], x[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) v[e] = x[e] = 0.f;
    if (i < n) {
      load8<DT>(h, base + i, v);
      if (RES) load8<DT>(u, base + i, x);
    }
    if (RES) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) v[e] -= x[e];
    }
    const I8Scale k(top16(top_bits<kPer>(v)));
    *reinterpret_cast<u32x2_t*>(slot + q0 + i) = i8_pack8(v, k);
    if ((c & 15) == 0) scales[(size_t)blockIdx.y * blocks + c / 16] = k.s;
  }
}

// 8 values of the draft h_d = u + sum_m c_m s_m q_m: fp32 sums in the order of the NT terms, one rounding.  All terms'
// bytes and scales are requested before the first is used.  16 values a lane, or a number of terms that the
// kernel finds out, are slower (8 x 256 x 1152 bf16, 3 terms: 4.6 us; 5.2; 6.1).
template <int DT, bool RES, int NT>
__device__ __forceinline__ void draft_chunk_i8(const TermsI8& t, const void* u, size_t at, size_t i, size_t q0, size_t s0, float* out) {
  u32x2_t w[NT];
  float s[NT], f[kPer], x[kPer];
#pragma unroll
  for (int m = 0; m < NT; ++m) {
    w[m] = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(t.slot[m] + q0 + i));
    s[m] = t.scales[m][s0 + i / kI8Block];
  }
  if (RES) load8<DT>(u, at, x);
#pragma unroll
  for (int e = 0; e < kPer; ++e) f[e] = 0.f;
#pragma unroll
  for (int m = 0; m < NT; ++m) {
    float q[kPer];
    i8_unpack4(w[m][0], q);
    i8_unpack4(w[m][1], q + 4);
#pragma unroll
    for (int e = 0; e < kPer; ++e) f[e] = fmaf(t.c[m], s[m] * q[e], f[e]);
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e) out[e] = St<DT>::rnd(RES ? x[e] + f[e] : f[e]);
}

template <int DT, bool RES, int NT>
__global__ __launch_bounds__(kThreads) void k_draft_i8(TermsI8 t, const void* u, void* hd, size_t n, size_t blocks) {
  const size_t base = (size_t)blockIdx.y * n, s0 = (size_t)blockIdx.y * blocks, q0 = s0 * kI8Block;
  for (size_t i = ((size_t)blockIdx.x * kThreads + threadIdx.x) * kPer; i < n; i += (size_t)gridDim.x * kThreads * kPer) {
    float o[kPer];
    draft_chunk_i8<DT, RES, NT>(t, u, base + i, i, q0, s0, o);
    store8<DT>(hd, base + i, o);
  }
}

// Verify and replace (Eq. 3-5) on that draft: what k_verify does, with the same two-stage sums; a workgroup that has a
// sample to itself finishes it.
template <int DT, bool RES, int NT>
__global__ __launch_bounds__(kThreads) void k_verify_i8(TermsI8 t, const void* u, const void* __restrict__ hf, void* hout, Forward fw,
                                                        size_t n, size_t blocks, float* __restrict__ partials, float eps,
                                                        float* __restrict__ rel) {
  __shared__ float red[2][kThreads / 64];
  const size_t base = (size_t)blockIdx.y * n, s0 = (size_t)blockIdx.y * blocks, q0 = s0 * kI8Block;
  float num = 0.f, den = 0.f;
  for (size_t i = ((size_t)blockIdx.x * kThreads + threadIdx.x) * kPer; i < n; i += (size_t)gridDim.x * kThreads * kPer) {
    float d[kPer], f[kPer];
    load8<DT>(hf, base + i, f);
    draft_chunk_i8<DT, RES, NT>(t, u, base + i, i, q0, s0, d);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      num += fabsf(d[e] - f[e]);
      den += fabsf(f[e]);
    }
    if (fw.kind >= FWD_TOKENS) {   // 8 values lie in one row (C % 8 == 0)
      const int row = (int)(i / fw.C), ch = (int)(i % fw.C);
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const bool exact = fw.kind == FWD_TOKENS ? row % fw.stride == 0 : (ch + e) % fw.stride == 0;
        d[e] = exact ? f[e] : d[e];
      }
    }
    store8<DT>(hout, base + i, fw.kind == FWD_EXACT ? f : d);
  }
  num = wave_sum(num);
  den = wave_sum(den);
  if ((threadIdx.x & 63) == 0) { red[0][threadIdx.x >> 6] = num; red[1][threadIdx.x >> 6] = den; }
  __syncthreads();
  if (threadIdx.x == 0) {
    num = (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]);
    den = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    float* p = partials + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2;
    if (gridDim.x > 1) {
      p[0] = num;
      p[1] = den;
    } else if (rel) {
      rel[blockIdx.y] = num / (den + eps);
    }
  }
}

int groups_for(size_t n) {
  const size_t g = (n + (size_t)kThreads * kPer - 1) / ((size_t)kThreads * kPer);
  return (int)(g > kMaxGroups ? kMaxGroups : g);
}

}  // namespace

#define FF_BY_TYPE(kernel, res, more, ...)                                                            \
  do {                                                                                                \
    if (dtype == DT_BF16) {                                                                           \
      if (res) FF_LAUNCH((kernel<DT_BF16, true more>), grid, kThreads, 0, s, __VA_ARGS__);            \
      else FF_LAUNCH((kernel<DT_BF16, false more>), grid, kThreads, 0, s, __VA_ARGS__);               \
    } else {                                                                                          \
      if (res) FF_LAUNCH((kernel<DT_F32, true more>), grid, kThreads, 0, s, __VA_ARGS__);             \
      else FF_LAUNCH((kernel<DT_F32, false more>), grid, kThreads, 0, s, __VA_ARGS__);                \
    }                                                                                                 \
  } while (0)
#define FF_COMMA(n) , n
#define FF_BY_TERMS(kernel, res, ...)                                        \
  do {                                                                       \
    switch (t.n) {                                                           \
      case 1: FF_BY_TYPE(kernel, res, FF_COMMA(1), __VA_ARGS__); break;      \
      case 2: FF_BY_TYPE(kernel, res, FF_COMMA(2), __VA_ARGS__); break;      \
      case 3: FF_BY_TYPE(kernel, res, FF_COMMA(3), __VA_ARGS__); break;      \
      case 4: FF_BY_TYPE(kernel, res, FF_COMMA(4), __VA_ARGS__); break;      \
      default: return hipErrorInvalidValue;                                  \
    }                                                                        \
  } while (0)

hipError_t cache_update_i8(int dtype, uint8_t* slot, float* scales, const void* u, const void* h, int B, size_t n, hipStream_t s) {
  const size_t blocks = i8_blocks(n);
  const dim3 grid(groups_for(blocks * kI8Block), B);
  FF_BY_TYPE(k_cache_update_i8, u != nullptr, , slot, scales, u, h, n, blocks);
  return hipGetLastError();
}

hipError_t draft_i8(int dtype, const TermsI8& t, const void* u, void* hd, int B, size_t n, hipStream_t s) {
  const size_t blocks = i8_blocks(n);
  const dim3 grid(groups_for(n), B);
  FF_BY_TERMS(k_draft_i8, u != nullptr, t, u, hd, n, blocks);
  return hipGetLastError();
}

hipError_t verify_i8(int dtype, const TermsI8& t, const void* u, const void* hf, void* hout, const Forward& fw, int B, size_t n,
                     float eps, float* rel, float* partials, hipStream_t s) {
  const size_t blocks = i8_blocks(n);
  // four turns of one workgroup take less than a second launch
  const dim3 grid(n <= 4 * kThreads * kPer ? 1 : groups_for(n), B);
  FF_BY_TERMS(k_verify_i8, u != nullptr, t, u, hf, hout, fw, n, blocks, partials, eps, rel);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !rel || grid.x == 1) return e;
  return verify_finish(partials, B, grid.x, eps, rel, s);
}
#undef FF_BY_TERMS
#undef FF_COMMA
#undef FF_BY_TYPE

}  // namespace ff
