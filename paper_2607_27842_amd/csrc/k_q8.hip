// 8-bit operands: e4m3 values with an fp32 scale per block of 128 columns of a row, or per square
// of 128 x 128, and the root-mean-square norm that writes them.
//   s = max(largest |v| of the block, 2^-100) / 448,   q = e4m3(v * (1 / s))
// The floor keeps 1 / s finite, so that a block of zeros gives zeros.  448 is the format's largest
// value: |v| * (1 / s) <= 448 (1 + 2^-22), which rounds to 448.
#include "dev_common.h"

namespace ff {

namespace {

constexpr float kQFloor = 0x1p-100f;

__device__ __forceinline__ float abs_max8(const float* v) {
  float m = fabsf(v[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) m = fmaxf(m, fabsf(v[e]));
  return m;
}
__device__ __forceinline__ float q_scale(float top) { return fmaxf(top, kQFloor) / 448.0f; }
// 8 values times inv as e4m3, rounded to nearest even
__device__ __forceinline__ u32x2_t q_pack8(const float* v, float inv) {
  u32x2_t w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * inv, v[4 * h + 1] * inv, 0, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * inv, v[4 * h + 3] * inv, p, true);
    w[h] = (uint32_t)p;
  }
  return w;
}

// ---------------------------------------------------------------- quantisation
// A workgroup takes 16 rows x 4 blocks: a wavefront 4 rows, one after the other in registers, with 16
// lanes on each block (1 KB of bf16 in a piece; 16 lanes on one row of four read 256-byte pieces
// and took 2 % longer).  Bound by memory: 4608 x 8192 bf16 25 to 27 us, 4.4 TB/s of the 5.0 that a large
// copy reaches; one row 2.3 us, a launch.
constexpr int kQBlocks = 4;
template <int DT>
__global__ __launch_bounds__(256) void k_quant_rows(QuantArgs a) {
  const int nb = (a.C + kQBlock - 1) / kQBlock, nbw = (nb + kQBlocks - 1) / kQBlocks;
  const int row0 = (blockIdx.x / nbw) * 16 + (threadIdx.x >> 6) * 4, lane = threadIdx.x & 63;
  const int c = (blockIdx.x % nbw) * kQBlocks * kQBlock + lane * 8, b = c / kQBlock;
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    if (row0 + i < a.rows && c < a.C) load8<DT>(a.x, (size_t)(row0 + i) * a.x_row + c, v[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float s = q_scale(max16(abs_max8(v[i])));
    if (row0 + i >= a.rows || c >= a.C) continue;
    *reinterpret_cast<u32x2_t*>(a.q + (size_t)(row0 + i) * a.q_row + c) = q_pack8(v[i], 1.0f / s);
    if ((lane & 15) == 0) a.qs[(size_t)b * a.qs_ld + row0 + i] = s;
  }
}

// One workgroup per square of 128 x 128, held in registers between the square's largest value and the
// rounding.  Bound by memory: 8200 x 2960 fp32 26 us, 4.7 TB/s.
template <int DT>
__global__ __launch_bounds__(256) void k_quant_squares(QuantArgs a) {
  __shared__ float top[16];
  const int nb = (a.C + kQBlock - 1) / kQBlock;
  const int ra = blockIdx.x / nb, b = blockIdx.x % nb;
  const int r0 = ra * kQBlock + (threadIdx.x >> 4), c = b * kQBlock + (threadIdx.x & 15) * 8;
  float v[8][8], m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    if (r0 + 16 * i < a.rows && c < a.C) load8<DT>(a.x, (size_t)(r0 + 16 * i) * a.x_row + c, v[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, abs_max8(v[i]));
  m = max16(m);
  if ((threadIdx.x & 15) == 0) top[threadIdx.x >> 4] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, top[i]);
  const float s = q_scale(m), inv = 1.0f / s;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (r0 + 16 * i < a.rows && c < a.C) *reinterpret_cast<u32x2_t*>(a.q + (size_t)(r0 + 16 * i) * a.q_row + c) = q_pack8(v[i], inv);
  if (threadIdx.x == 0) a.qs[(size_t)ra * a.qs_ld + b] = s;
}

// ---------------------------------------------------------------- norm
// W wavefronts hold a row, U units of 8 columns a lane: lane l of the row's 64 W takes units l + 64 W i,
// so that 16 neighbouring lanes hold a block of 128.  The row stays in registers between the sum of squares
// and the rounding.  The compiler widens residual and gain where it loads them, so each unit's loads are
// waited for before the next unit's go out; with many rows a CU's other wavefronts cover that.  Bound by
// memory: 14566 x 2048 bf16 with residual and sum 46 us, 4.5 TB/s; one row 2.1 us, a launch.
template <int DT, int W, int U>
__global__ __launch_bounds__(256) void k_rms_norm_q8(RmsArgs a) {
  __shared__ float part[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x * (4 / W) + (W == 1 ? wave : 0);
  const int l = W == 1 ? lane : (int)threadIdx.x;
  if (W == 1 && row >= a.rows) return;
  float t[U][8], r[U][8], g[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (l + 64 * W * i) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) { t[i][e] = 0.f; g[i][e] = 1.f; }
    if (c < a.C) {
      load8<DT>(a.x, (size_t)row * a.x_row + c, t[i]);
      if (a.resid) load8<DT>(a.resid, (size_t)row * a.resid_row + c, r[i]);
      if (a.gain) load8<DT>(a.gain, c, g[i]);
    }
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (l + 64 * W * i) * 8;
    if (a.resid && c < a.C) {
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][e] = St<DT>::rnd(t[i][e] + r[i][e]);
      if (a.sum) store8<DT>(a.sum, (size_t)row * a.sum_row + c, t[i]);
    }
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(t[i][e], t[i][e], s);
    ss += s;
  }
  ss = row_sum(ss);
  if (W > 1) {
    if (lane == 0) part[wave] = ss;
    __syncthreads();
    ss = (part[0] + part[1]) + (part[2] + part[3]);
  }
  const float inv = 1.0f / sqrtf(ss / (float)a.C + a.eps);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (l + 64 * W * i) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) t[i][e] = t[i][e] * inv * g[i][e];
    if (a.y && c < a.C) store8<DT>(a.y, (size_t)row * a.y_row + c, t[i]);
    if (!a.q) continue;
    const float s = q_scale(max16(abs_max8(t[i])));   // lanes past C hold zeros
    if (c < a.C) {
      *reinterpret_cast<u32x2_t*>(a.q + (size_t)row * a.q_row + c) = q_pack8(t[i], 1.0f / s);
      if ((l & 15) == 0) a.qs[(size_t)(c / kQBlock) * a.qs_ld + row] = s;
    }
  }
}

// A wavefront a row from 1024 rows on, four below (bf16; C = 512, 2048 rows: one 3.1 us, four 3.9; C = 2048, 512
// rows: one 4.9, four 3.2).  The best border depends on C: at C = 512 one is ahead from 64 rows (2.5 for 2.6),
// at C = 2048 four up to 4096 at least (1024 rows: 4.5 for 6.1; 4096: 12.1 for 13.0).
template <int DT>
void launch_rms(const RmsArgs& a, hipStream_t s) {
  const int units = a.C / 8;
  if (units <= 256 && a.rows >= 1024) {
    const int wg = (a.rows + 3) / 4;
    if (units <= 64) FF_LAUNCH((k_rms_norm_q8<DT, 1, 1>), wg, 256, 0, s, a);
    else if (units <= 128) FF_LAUNCH((k_rms_norm_q8<DT, 1, 2>), wg, 256, 0, s, a);
    else FF_LAUNCH((k_rms_norm_q8<DT, 1, 4>), wg, 256, 0, s, a);
  } else {
    if (units <= 256) FF_LAUNCH((k_rms_norm_q8<DT, 4, 1>), a.rows, 256, 0, s, a);
    else if (units <= 512) FF_LAUNCH((k_rms_norm_q8<DT, 4, 2>), a.rows, 256, 0, s, a);
    else if (units <= 1024) FF_LAUNCH((k_rms_norm_q8<DT, 4, 4>), a.rows, 256, 0, s, a);
    else FF_LAUNCH((k_rms_norm_q8<DT, 4, 8>), a.rows, 256, 0, s, a);
  }
}

}  // namespace

hipError_t quant_rows(int dtype, const QuantArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const int nb = (a.C + kQBlock - 1) / kQBlock;
  const long wg = (long)((a.rows + 15) / 16) * ((nb + kQBlocks - 1) / kQBlocks);
  if (wg > 0x7fffffffL) return hipErrorInvalidValue;
  if (dtype == DT_BF16) FF_LAUNCH(k_quant_rows<DT_BF16>, (unsigned)wg, 256, 0, s, a);
  else FF_LAUNCH(k_quant_rows<DT_F32>, (unsigned)wg, 256, 0, s, a);
  return hipGetLastError();
}

hipError_t quant_squares(int dtype, const QuantArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const long wg = (long)((a.rows + kQBlock - 1) / kQBlock) * ((a.C + kQBlock - 1) / kQBlock);
  if (wg > 0x7fffffffL) return hipErrorInvalidValue;
  if (dtype == DT_BF16) FF_LAUNCH(k_quant_squares<DT_BF16>, (unsigned)wg, 256, 0, s, a);
  else FF_LAUNCH(k_quant_squares<DT_F32>, (unsigned)wg, 256, 0, s, a);
  return hipGetLastError();
}

hipError_t rms_norm_q8(int dtype, const RmsArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  if (dtype == DT_BF16) launch_rms<DT_BF16>(a, s);
  else launch_rms<DT_F32>(a, s);
  return hipGetLastError();
}

}  // namespace ff
