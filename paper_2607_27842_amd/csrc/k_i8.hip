// Rows in 8-bit integers with a scale a row, and what stands between two branches of a block: the norm
// behind one branch, gate and scaled residual, the norm and modulation in front of the next.
#include "i8_common.h"

namespace ff {

namespace {

// A row's values as they are stored: 8 columns a unit
template <int DT> struct Piece;
template <> struct Piece<DT_BF16> {
  u32x4_t w;
  __device__ __forceinline__ void load(const void* p, size_t i) { w = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(p) + i); }
  __device__ __forceinline__ float at(int e) const { return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16); }
};
template <> struct Piece<DT_F32> {
  f32x4_t w[2];
  __device__ __forceinline__ void load(const void* p, size_t i) {
    const f32x4_t* q = reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p) + i);
    w[0] = q[0];
    w[1] = q[1];
  }
  __device__ __forceinline__ float at(int e) const { return w[e / 4][e % 4]; }
};

// The largest of a row's wavefronts' values
template <int W>
__device__ __forceinline__ uint32_t top_row(uint32_t top, float* at, int wave) {
  top = top64(top);
  if (W == 1) return top;
  if ((threadIdx.x & 63) == 0) at[wave] = __uint_as_float(top);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < W; ++i) top = max(top, __float_as_uint(at[i]));
  return top;
}

// ---------------------------------------------------------------- quantisation
// W wavefronts hold a row, U units of 8 columns a lane, in registers between the row's largest value and
// the rounding; a workgroup (or, W = 1, a wavefront) walks every step-th row, the next one's values requested ahead.
template <int DT, int W, int U>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_quant_i8(QuantI8Args a, int step) {
  __shared__ float part[2][W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l = W == 1 ? lane : (int)threadIdx.x;
  int row = (W == 1 ? blockIdx.x * 4 + wave : blockIdx.x), turn = 0;
  if (row >= a.rows) return;   // all of a row's wavefronts
  Piece<DT> p[U];
  auto request = [&](int r) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if ((l + 64 * W * i) * 8 < a.C) p[i].load(a.x, (size_t)r * a.x_row + (l + 64 * W * i) * 8);
  };
  request(row);
  for (;; row += step) {
    float v[U][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = (l + 64 * W * i) * 8 < a.C ? p[i].at(e) : 0.f;
      top = top_bits<8>(v[i], top);
    }
    if (row + step < a.rows) request(row + step);
    const I8Scale k(top_row<W>(top, part[turn++ & 1], wave));
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int c = (l + 64 * W * i) * 8;
      if (c < a.C) *reinterpret_cast<u32x2_t*>(a.q + (size_t)row * a.q_row + c) = i8_pack8(v[i], k);
    }
    if (l == 0) a.s[row] = k.s;
    if (row + step >= a.rows) break;
  }
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

// As many walks as the card holds at once, each of W of about 6144 wavefronts (k_branch_norm, 14566 x 2048: 2048 walks
// instead of 1536, 54.7 us for 50.4, as some start late; twice as many 50.7, 8192 53.2).
int walks_for(int rows, int W) { return rows < 6144 / W ? rows : 6144 / W; }

template <int DT, int W, int U>
void launch_quant_walks(const QuantI8Args& a, hipStream_t s) {
  const int walks = walks_for(a.rows, W);
  if (W == 1) FF_LAUNCH((k_quant_i8<DT, W, U>), (walks + 3) / 4, 256, 0, s, a, (walks + 3) / 4 * 4);
  else FF_LAUNCH((k_quant_i8<DT, W, U>), walks, 64 * W, 0, s, a, walks);
}

// A row in registers: one unit a lane up to 2048 columns, two above, with as few wavefronts as that takes (8000 x 3000
// bf16 13.4 us, with one unit 14.2, with four 13.8; 4000 x 8192 17.8, 19.8, 18.4; 14566 x 1024 9.2, with two 9.4, with four 10.6).
template <int DT>
void launch_quant(const QuantI8Args& a, hipStream_t s) {
  const int units = a.C / 8;
  if (units <= 64) launch_quant_walks<DT, 1, 1>(a, s);
  else if (units <= 128) launch_quant_walks<DT, 2, 1>(a, s);
  else if (units <= 256) launch_quant_walks<DT, 4, 1>(a, s);
  else if (units <= 512) launch_quant_walks<DT, 4, 2>(a, s);
  else if (units <= 1024) launch_quant_walks<DT, 8, 2>(a, s);
  else if (units <= 2048) launch_quant_walks<DT, 16, 2>(a, s);
  else FF_LAUNCH(k_quant_i8_long<DT>, a.rows, 256, 0, s, a);
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
  if (W == 2) return at[0] + at[1];
  float sum = (at[0] + at[1]) + (at[2] + at[3]);
#pragma unroll
  for (int i = 4; i < W; i += 4) sum += (at[i] + at[i + 1]) + (at[i + 2] + at[i + 3]);
  return sum;
}

template <int U>
__device__ __forceinline__ float squares_of(const float (&v)[U][8]) {
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(v[i][e], v[i][e], ss);
  return ss;
}
template <int U>
__device__ __forceinline__ void times(float (&v)[U][8], float by) {
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] *= by;
}

// v <- v normed.  Columns past the row hold zeros before and after.  Nothing on the way leaves fp32: the mean is formed from
// 2^-14 of the values (C <= 2^14), and half of v - mean takes its place; a sum of squares that overflows is formed again
// from the row times 2^-80, in a branch that all of the row's lanes take together, as they hold the same sum.  Powers of
// two change no rounding, but that values below 2^-46 of a row whose root mean square is above 2^57 lose digits, results below
// 2^-103.  14566 x 2048 bf16 takes the same time with and without that branch; another one behind the mean, 3000 x 6000
// bf16, both LayerNorm, 59.8 us for 55.6.
constexpr int kNormSums = 3;   // reductions at most
template <int W, int U>
__device__ __forceinline__ void norm_row(float (&v)[U][8], const BranchArgs& a, int kind, int l, float* at, int wave) {
  if (kind == NORM_NONE) return;
  float eps = a.eps;
  if (kind == NORM_LAYER) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(v[i][e], 0x1p-14f, sum);
    const float half = over_row<W>(sum, at, wave) / (float)a.C * 0x1p13f;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = (l + 64 * W * i) * 8 < a.C ? fmaf(v[i][e], 0.5f, -half) : 0.f;
    eps = fmaxf(eps * 0.25f, 0x1p-149f);   // the least of all would be gone, and a row of zeros NaN
  }
  float ss = over_row<W>(squares_of<U>(v), at + W, wave);
  if (__builtin_expect(!(ss < __builtin_inff()), 0)) {
    times<U>(v, 0x1p-80f);
    eps = eps * 0x1p-80f * 0x1p-80f;
    ss = over_row<W>(squares_of<U>(v), at + 2 * W, wave);
  }
  times<U>(v, 1.0f / sqrtf(ss / (float)a.C + eps));
}

// What a row's columns are multiplied by and moved by, the same for all rows of a sample
template <int U>
struct Vectors { float a[U][8], p[U][8], s[U][8]; };   // gate post_gain, pre_gain (1 + scale), shift
template <int DT, int W, int U>
__device__ __forceinline__ void load_vectors(const BranchArgs& k, size_t smp, int l, Vectors<U>& v) {
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (l + 64 * W * i) * 8;
    float g[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { v.a[i][e] = v.p[i][e] = 1.f; v.s[i][e] = 0.f; }
    if (c >= k.C) continue;
    if (k.post_gain) load8<DT>(k.post_gain, c, v.a[i]);
    if (k.gate) {
      load8<DT_F32>(k.gate, smp * k.gate_ld + c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) v.a[i][e] *= k.gate_tanh ? tanh_f(g[e]) : g[e];
    }
    if (k.pre_gain) load8<DT>(k.pre_gain, c, v.p[i]);
    if (k.scale) {
      load8<DT_F32>(k.scale, smp * k.mod_ld + c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) v.p[i][e] *= 1.0f + g[e];
    }
    if (k.shift) load8<DT_F32>(k.shift, smp * k.mod_ld + c, v.s[i]);
  }
}

// W wavefronts hold a row, U units of 8 columns a lane; a workgroup (or, W = 1, a wavefront) walks every step-th row.
// The next row's values are requested before this row's sums meet, and the sample's vectors stay in registers
// from row to row: read again for each row they are twice a bf16 row's own bytes, from L2.  Bound by memory: 14566 x 2048
// bf16, both norms, gate, scale and shift, 47.9 to 50.4 us from run to run, 4.74 to 4.98 TB/s of the 5.0 that a large
// copy reaches; a row a workgroup 60.3 for 50.4, walks of neighbouring rows 54.1.  One row 3.6 us, a launch.
template <int DT, int W, int U>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_branch_norm(BranchArgs a, int step) {
  __shared__ float part[2][(2 * kNormSums + 1) * W];   // a row's reductions have a place each, and rows in turn two sets
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l = W == 1 ? lane : (int)threadIdx.x;
  int row = (W == 1 ? blockIdx.x * 4 + wave : blockIdx.x);
  int turn = 0;
  if (row >= a.rows) return;   // all of a row's wavefronts
  Piece<DT> px[U], pz[U];
  auto request = [&](int r) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int c = (l + 64 * W * i) * 8;
      if (c >= a.C) continue;
      px[i].load(a.x, (size_t)r * a.x_row + c);
      if (a.branch) pz[i].load(a.branch, (size_t)r * a.branch_row + c);
    }
  };
  // The widest rows need the registers: their lanes keep what the second norm meets in LDS, each for itself (2000 x 16384 fp32
  // 117.7 us; with all vectors in registers, some of which spill, 152.8; read again for each row 137).
  constexpr bool kPark = W * U > 16;
  __shared__ f32x4_t parked[kPark ? 4 * U : 1][kPark ? 64 * W : 1];
  auto park = [&](Vectors<U>& v, bool back) __attribute__((always_inline)) {
    if (!kPark) return;
#pragma unroll
    for (int i = 0; i < 4 * U; ++i) {
      float* const at = (i & 2 ? v.s : v.p)[i / 4] + (i & 1) * 4;
      f32x4_t& to = parked[i][l];
      if (back) for (int e = 0; e < 4; ++e) at[e] = to[e];
      else to = f32x4_t{at[0], at[1], at[2], at[3]};
    }
  };
  request(row);
  Vectors<U> v;
  int smp = row / a.mod_rows, next = min((smp + 1) * (int64_t)a.mod_rows, (int64_t)a.rows);   // the next sample's first row
  load_vectors<DT, W, U>(a, smp, l, v);
  park(v, false);
  for (;; row += step) {
    float* const at = part[turn++ & 1];
    float t[U][8], z[U][8];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const bool in = (l + 64 * W * i) * 8 < a.C;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        t[i][e] = in ? px[i].at(e) : 0.f;
        z[i][e] = in && a.branch ? pz[i].at(e) : 0.f;
      }
    }
    if (row >= next) {
      smp = row / a.mod_rows;
      next = min((smp + 1) * (int64_t)a.mod_rows, (int64_t)a.rows);
      load_vectors<DT, W, U>(a, smp, l, v);
      park(v, false);
    }
    if (row + step < a.rows) request(row + step);
    if (a.branch) norm_row<W, U>(z, a, a.post, l, at, wave);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int c = (l + 64 * W * i) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) t[i][e] = St<DT>::rnd(fmaf(t[i][e], a.resid_scale, z[i][e] * v.a[i][e]));
      if (a.sum && c < a.C) store8<DT>(a.sum, (size_t)row * a.sum_row + c, t[i]);
    }
    if (a.y || a.q) {
      norm_row<W, U>(t, a, a.pre, l, at + kNormSums * W, wave);
      park(v, true);
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int c = (l + 64 * W * i) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) t[i][e] = fmaf(t[i][e], v.p[i][e], v.s[i][e]);
        if (a.y && c < a.C) store8<DT>(a.y, (size_t)row * a.y_row + c, t[i]);
        top = top_bits<8>(t[i], top);   // columns past C hold zeros
      }
      if (a.q) {
        const I8Scale k(top_row<W>(top, at + 2 * kNormSums * W, wave));
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int c = (l + 64 * W * i) * 8;
          if (c < a.C) *reinterpret_cast<u32x2_t*>(a.q + (size_t)row * a.q_row + c) = i8_pack8(t[i], k);
        }
        if (l == 0) a.q_s[row] = k.s;
      }
    }
    if (row + step >= a.rows) break;
  }
}

template <int DT, int W, int U>
void launch_walks(const BranchArgs& a, hipStream_t s) {
  const int walks = walks_for(a.rows, W);
  if (W == 1) FF_LAUNCH((k_branch_norm<DT, W, U>), (walks + 3) / 4, 256, 0, s, a, (walks + 3) / 4 * 4);
  else FF_LAUNCH((k_branch_norm<DT, W, U>), walks, 64 * W, 0, s, a, walks);
}

// One unit a lane where the row allows it (20000 x 1024: one wavefront with two 40.3 us, two with one 35.7; 4608 x 2048:
// two wavefronts with two 18.9, four with one 16.2)
template <int DT>
void launch_branch(const BranchArgs& a, hipStream_t s) {
  const int units = a.C / 8;
  if (units <= 64) launch_walks<DT, 1, 1>(a, s);
  else if (units <= 128) launch_walks<DT, 2, 1>(a, s);
  else if (units <= 256) launch_walks<DT, 4, 1>(a, s);
  else if (units <= 512) launch_walks<DT, 8, 1>(a, s);
  else if (units <= 1024) launch_walks<DT, 16, 1>(a, s);
  else launch_walks<DT, 16, 2>(a, s);
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
