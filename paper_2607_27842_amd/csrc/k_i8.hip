// Rows in 8-bit integers with a scale a row, and what stands between two branches of a block: the norm
// behind one branch, gate and scaled residual, the norm and modulation in front of the next.
#include "i8_common.h"

namespace ff {

namespace {

// ---------------------------------------------------------------- quantisation
// W wavefronts hold a row, U units of 8 columns a lane, in registers between the row's largest value and
// the rounding.
template <int DT, int W, int U>
__global__ __launch_bounds__(256) void k_quant_i8(QuantI8Args a) {
  __shared__ uint32_t part[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x * (4 / W) + (W == 1 ? wave : 0), l = W == 1 ? lane : (int)threadIdx.x;
  if (W == 1 && row >= a.rows) return;
  float v[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (l + 64 * W * i) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    if (c < a.C) load8<DT>(a.x, (size_t)row * a.x_row + c, v[i]);
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < U; ++i) top = top_bits<8>(v[i], top);
  top = top64(top);
  if (W > 1) {
    if (lane == 0) part[wave] = top;
    __syncthreads();
    top = max(max(part[0], part[1]), max(part[2], part[3]));
  }
  const I8Scale k(top);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (l + 64 * W * i) * 8;
    if (c < a.C) *reinterpret_cast<u32x2_t*>(a.q + (size_t)row * a.q_row + c) = i8_pack8(v[i], k);
  }
  if (l == 0) a.s[row] = k.s;
}

// Rows too long for the registers are read twice.
template <int DT>
__global__ __launch_bounds__(256) void k_quant_i8_long(QuantI8Args a) {
  __shared__ uint32_t part[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = blockIdx.x;
  float v[8];
  uint32_t top = 0;
  for (int c = threadIdx.x * 8; c < a.C; c += 2048) {
    load8<DT>(a.x, (size_t)row * a.x_row + c, v);
    top = top_bits<8>(v, top);
  }
  top = top64(top);
  if (lane == 0) part[wave] = top;
  __syncthreads();
  const I8Scale k(max(max(part[0], part[1]), max(part[2], part[3])));
  for (int c = threadIdx.x * 8; c < a.C; c += 2048) {
    load8<DT>(a.x, (size_t)row * a.x_row + c, v);
    *reinterpret_cast<u32x2_t*>(a.q + (size_t)row * a.q_row + c) = i8_pack8(v, k);
  }
  if (threadIdx.x == 0) a.s[row] = k.s;
}

template <int DT>
void launch_quant(const QuantI8Args& a, hipStream_t s) {
  const int units = a.C / 8;
  if (units <= 256 && a.rows >= 1024) {
    const int wg = (a.rows + 3) / 4;
    if (units <= 64) FF_LAUNCH((k_quant_i8<DT, 1, 1>), wg, 256, 0, s, a);
    else if (units <= 128) FF_LAUNCH((k_quant_i8<DT, 1, 2>), wg, 256, 0, s, a);
    else FF_LAUNCH((k_quant_i8<DT, 1, 4>), wg, 256, 0, s, a);
  } else {
    if (units <= 256) FF_LAUNCH((k_quant_i8<DT, 4, 1>), a.rows, 256, 0, s, a);
    else if (units <= 512) FF_LAUNCH((k_quant_i8<DT, 4, 2>), a.rows, 256, 0, s, a);
    else if (units <= 1024) FF_LAUNCH((k_quant_i8<DT, 4, 4>), a.rows, 256, 0, s, a);
    else if (units <= 2048) FF_LAUNCH((k_quant_i8<DT, 4, 8>), a.rows, 256, 0, s, a);
    else FF_LAUNCH(k_quant_i8_long<DT>, a.rows, 256, 0, s, a);
  }
}

// ---------------------------------------------------------------- between branches
// tanh by its series below 1/4 (the first term left out is below 2^-24 of the result) and as 1 - 2 / (e^2g + 1)
// above, where the subtraction keeps the digits; hardware exponential and reciprocal, about 2^-22.
__device__ __forceinline__ float tanh_f(float g) {
  const float g2 = g * g;
  const float near = g * fmaf(g2, fmaf(g2, fmaf(g2, fmaf(g2, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
  const float far = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(fabsf(g) * 2.885390081777927f) + 1.0f);
  return g2 < 0.0625f ? near : copysignf(far, g);
}

// A sum over the row's wavefronts; `at`: this reduction's place in LDS, none is used twice in a row's walk
template <int W>
__device__ __forceinline__ float over_row(float v, float* at, int wave) {
  v = row_sum(v);
  if (W == 1) return v;
  if ((threadIdx.x & 63) == 0) at[wave] = v;
  __syncthreads();
  return (at[0] + at[1]) + (at[2] + at[3]);
}

// v <- v normed.  Columns past the row hold zeros before and after.
template <int W, int U>
__device__ __forceinline__ void norm_row(float (&v)[U][8], const BranchArgs& a, int kind, int l, float* at, int wave) {
  if (kind == NORM_NONE) return;
  if (kind == NORM_LAYER) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += v[i][e];
    const float mean = over_row<W>(sum, at, wave) / (float)a.C;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = (l + 64 * W * i) * 8 < a.C ? v[i][e] - mean : 0.f;
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(v[i][e], v[i][e], ss);
  const float inv = 1.0f / sqrtf(over_row<W>(ss, at + 4, wave) / (float)a.C + a.eps);
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] *= inv;
}

template <int DT, int W, int U>
__global__ __launch_bounds__(256) void k_branch_norm(BranchArgs a) {
  __shared__ float part[20];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x * (4 / W) + (W == 1 ? wave : 0), l = W == 1 ? lane : (int)threadIdx.x;
  if (W == 1 && row >= a.rows) return;
  const size_t smp = row / a.mod_rows;
  float t[U][8], z[U][8], g[8], f[8];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (l + 64 * W * i) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) t[i][e] = z[i][e] = 0.f;
    if (c < a.C) {
      load8<DT>(a.x, (size_t)row * a.x_row + c, t[i]);
      if (a.branch) load8<DT>(a.branch, (size_t)row * a.branch_row + c, z[i]);
    }
  }
  if (a.branch) norm_row<W, U>(z, a, a.post, l, part, wave);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (l + 64 * W * i) * 8;
    if (c >= a.C) continue;
    if (a.post_gain) {
      load8<DT>(a.post_gain, c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[i][e] *= g[e];
    }
    if (a.gate) {
      load8<DT_F32>(a.gate, smp * a.gate_ld + c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[i][e] *= a.gate_tanh ? tanh_f(g[e]) : g[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) t[i][e] = St<DT>::rnd(fmaf(t[i][e], a.resid_scale, z[i][e]));
    if (a.sum) store8<DT>(a.sum, (size_t)row * a.sum_row + c, t[i]);
  }
  if (!a.y && !a.q) return;
  norm_row<W, U>(t, a, a.pre, l, part + 8, wave);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (l + 64 * W * i) * 8;
    if (c >= a.C) continue;
    if (a.pre_gain) {
      load8<DT>(a.pre_gain, c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][e] *= g[e];
    }
    if (a.scale) {
      load8<DT_F32>(a.scale, smp * a.mod_ld + c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][e] *= 1.0f + g[e];
    }
    if (a.shift) {
      load8<DT_F32>(a.shift, smp * a.mod_ld + c, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][e] += f[e];
    }
    if (a.y) store8<DT>(a.y, (size_t)row * a.y_row + c, t[i]);
    top = top_bits<8>(t[i], top);
  }
  if (!a.q) return;
  top = top64(top);
  if (W > 1) {
    if (lane == 0) part[16 + wave] = __uint_as_float(top);
    __syncthreads();
    top = max(max(__float_as_uint(part[16]), __float_as_uint(part[17])), max(__float_as_uint(part[18]), __float_as_uint(part[19])));
  }
  const I8Scale k(top);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (l + 64 * W * i) * 8;
    if (c < a.C) *reinterpret_cast<u32x2_t*>(a.q + (size_t)row * a.q_row + c) = i8_pack8(t[i], k);
  }
  if (l == 0) a.q_s[row] = k.s;
}

template <int DT>
void launch_branch(const BranchArgs& a, hipStream_t s) {
  const int units = a.C / 8;
  if (units <= 128) {
    const int wg = (a.rows + 3) / 4;
    if (units <= 64) FF_LAUNCH((k_branch_norm<DT, 1, 1>), wg, 256, 0, s, a);
    else FF_LAUNCH((k_branch_norm<DT, 1, 2>), wg, 256, 0, s, a);
  } else {
    if (units <= 256) FF_LAUNCH((k_branch_norm<DT, 4, 1>), a.rows, 256, 0, s, a);
    else if (units <= 512) FF_LAUNCH((k_branch_norm<DT, 4, 2>), a.rows, 256, 0, s, a);
    else if (units <= 1024) FF_LAUNCH((k_branch_norm<DT, 4, 4>), a.rows, 256, 0, s, a);
    else FF_LAUNCH((k_branch_norm<DT, 4, 8>), a.rows, 256, 0, s, a);
  }
}

}  // namespace

hipError_t quant_i8(int dtype, const QuantI8Args& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  if (dtype == DT_BF16) launch_quant<DT_BF16>(a, s);
  else launch_quant<DT_F32>(a, s);
  return hipGetLastError();
}

hipError_t branch_norm(int dtype, const BranchArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  if (dtype == DT_BF16) launch_branch<DT_BF16>(a, s);
  else launch_branch<DT_F32>(a, s);
  return hipGetLastError();
}

}  // namespace ff
