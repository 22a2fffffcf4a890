// Products of 8-bit integers with a scale for each row of either operand:
//   out = act(a_s[m] w_s[n] sum_k a[m, k] w[n, k] + bias) gate[m / gate_rows] + resid
// Sums of products are whole numbers in 32 bits (K <= 131056), the same in any order; a result is rounded to
// fp32 where the sum leaves them, once for each scale, and to the output's type at the end.  One
// v_mfma_i32_16x16x64_i8 covers 16 rows, 16 columns and 64 k.  The A operand holds weight rows (output
// columns n), the B operand activation rows m: lane l then holds output row l % 16 and columns
// 4 (l / 16) + 0..3.  Lane l of an operand takes row l % 16 and 16 bytes of the 64 k.
#include "gemm_8bit.h"
#include "i8_common.h"
#include <math.h>

namespace ff {

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4_t mfma_i8(u32x4_t a, u32x4_t b, i32x4_t c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, a), __builtin_bit_cast(i32x4_t, b), c, 0, 0, 0);
}

// ---------------------------------------------------------------- epilogue
// Results of V columns from their sums, written out so that every kernel rounds alike: a row's results depend neither on
// the other rows nor on the kernel that the call's sizes choose.  Absent parts: bias and resid 0, gate 1.
// sum sa may be beyond fp32 (sums are below 2^31) though sw brings it back.  FAR: where sa is from 2^96 on, the line is formed at
// 2^-32 of its size, which changes no rounding of results from 2^-94 on.
__device__ __forceinline__ bool is_far(float sa) { return fabsf(sa) >= 0x1p96f; }
template <bool FAR, int V>
__device__ __forceinline__ void results(const GemmI8Args& a, const int (&sum)[V], float sa, const float (&sw)[V], const float (&bias)[V],
                                        const float (&gate)[V], const float (&resid)[V], float (&v)[V]) {
  if (FAR && __builtin_expect(is_far(sa), 0)) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = fmaf((float)sum[e] * 0x1p-32f * sa, sw[e], bias[e] * 0x1p-32f) * 0x1p32f;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = fmaf((float)sum[e] * sa, sw[e], bias[e]);
  }
  if (a.gelu) {   // a branch around all of them: as a choice for each, GELU is computed where nothing asks for it
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = gelu_tanh_f(v[e]);
  }
  if (a.gate || a.resid) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = fmaf(v[e], gate[e], resid[e]);
  }
}
template <int V>
__device__ __forceinline__ void load_gate(const GemmI8Args& a, int r, int c, float (&g)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) g[e] = 1.f;
  if (a.gate) {
    const size_t at = (size_t)((uint32_t)(r + a.row0) / (uint32_t)a.gate_rows) * a.gate_ld + c;
#pragma unroll
    for (int e = 0; e < V; e += 4) St<DT_F32>::load(a.gate, at + e, g + e);
  }
}

// Word of a row's 4 columns col .. col + 3 in a wave's LDS region: rows of WN words, their 16-byte chunks in an order of the
// row's own (WN = 64), or four words more a row; 16 rows' same chunk then lies in 16 different sets of banks.
template <int WN>
__device__ __forceinline__ int sum_at(int row, int col) {
  if constexpr (WN == 64) return row * WN + (((col >> 2) ^ (row & 15)) << 2);
  else return row * (WN + 4) + col;
}
template <int WN> constexpr int sum_words(int rows) { return rows * (WN == 64 ? WN : WN + 4); }

// Those of the rows r0 .. r0 + rows - 1 whose scale is as large as FAR's (values from 10^31 on), columns c0 .. c0 + WN - 1, formed
// again from the operands, a column a lane.  As slow as that is, the epilogue's loop needs no registers for them.
template <int DT, int WN>
__device__ __forceinline__ void far_rows(const GemmI8Args& a, int r0, int rows, int c0) {
  const int lane = threadIdx.x & 63, c = c0 + lane % WN;
  if (c >= a.N) return;
  const uint8_t* const pw = a.w + (size_t)c * a.w_row;
#pragma unroll 1
  for (int r = r0 + lane / WN; r < min(r0 + rows, a.M); r += 64 / WN) {
    const float sa = a.a_s[r];
    if (!is_far(sa)) continue;
    const uint8_t* const pa = static_cast<const uint8_t*>(a.a) + (size_t)r * a.a_row;
    int sum = 0;
#pragma unroll 1
    for (int k = 0; k < a.K; k += 16) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t*>(pa + k), w = *reinterpret_cast<const u32x4_t*>(pw + k);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_sdot4((int)w[e], (int)x[e], sum, false);
    }
    const float bias = a.bias ? St<DT>::ld1(a.bias, c) : 0.f, resid = a.resid ? St<DT>::ld1(a.resid, (size_t)r * a.resid_row + c) : 0.f;
    const float gate = a.gate ? a.gate[(size_t)((uint32_t)(r + a.row0) / (uint32_t)a.gate_rows) * a.gate_ld + c] : 1.f;
    float v[1];
    results<true>(a, {sum}, sa, {a.w_s[c]}, {bias}, {gate}, {resid}, v);
    St<DT>::st1(a.out, (size_t)r * a.out_row + c, v[0]);
  }
}

// Rows r0 .. r0 + RB NB - 1, columns c0 .. c0 + WN - 1 of a wavefront: put(i) lays RB rows of sums at a time into
// the wave's own LDS region, and they come back as 8-column pieces, so that
// every load and store of bias, gate, residual and output is 16 bytes wide and covers whole row segments (in
// the MFMA layout each store would put 8 bytes into each of 16 rows).  N % 8 == 0: a piece is in range as
// a whole.  The caller has retired all waves' reads of what the region overlays.
template <int DT, int WN, int RB, int NB, class F>
__device__ __forceinline__ void epilogue(const GemmI8Args& a, int r0, int c0, int* lds, F&& put) {
  constexpr int CPR = WN / 8, RPP = 64 / CPR, NPASS = RB / RPP;
  static_assert(64 % CPR == 0 && NPASS >= 1 && 64 % RPP == 0, "whole rows a pass, passes within 64 rows");
  const int lane = threadIdx.x & 63;
  const int pc = lane % CPR * 8, pr = lane / CPR, c = c0 + pc;
  const int cl = c < a.N ? c : 0;   // loads past the matrix read its first column or last row
  float bias[8], sw[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = 0.f;
  if (a.bias) load8<DT>(a.bias, cl, bias);
  load8<DT_F32>(a.w_s, cl, sw);
  // All rows' scales are read first, one a lane: a load between the stores would be waited for behind the stores before
  // it.  The residual's pieces are requested a block ahead.
  constexpr int NS = (RB * NB + 63) / 64;
  float sa[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) sa[i] = a.a_s[min(r0 + 64 * i + lane, a.M - 1)];
  typedef typename Raw8<DT>::type raw_t;
  raw_t res[2][NPASS];
  auto request = [&](int i) __attribute__((always_inline)) {
    if (a.resid) {
#pragma unroll
      for (int p = 0; p < NPASS; ++p)
        res[i & 1][p] = Raw8<DT>::load(a.resid, (size_t)min(r0 + i * RB + p * RPP + pr, a.M - 1) * a.resid_row + cl);
    }
  };
  request(0);
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    // lanes read what other lanes wrote: to the compiler, too, the region changes here
    asm volatile("" ::: "memory");
    put(i);
    asm volatile("" ::: "memory");
    if (i + 1 < NB) request(i + 1);
#pragma unroll
    for (int p = 0; p < NPASS; ++p) {
      const int r = r0 + i * RB + p * RPP + pr;
      const i32x4_t x0 = *reinterpret_cast<const i32x4_t*>(lds + sum_at<WN>(p * RPP + pr, pc));
      const i32x4_t x1 = *reinterpret_cast<const i32x4_t*>(lds + sum_at<WN>(p * RPP + pr, pc + 4));
      const int ri = i * RB + p * RPP;   // + pr, below 64 more than the multiple of 64 that it lies behind
      const float sr = __shfl(sa[ri / 64], ri % 64 + pr, 64);
      float v[8], gate[8], resid[8];
      load_gate(a, min(r, a.M - 1), cl, gate);
#pragma unroll
      for (int e = 0; e < 8; ++e) resid[e] = a.resid ? Raw8<DT>::at(res[i & 1][p], e) : 0.f;
      const int sum[8] = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
      results<false>(a, sum, sr, sw, bias, gate, resid, v);
      if (r < a.M && c < a.N && !is_far(sr)) store8<DT>(a.out, (size_t)r * a.out_row + c, v);
    }
  }
  // Scales as large as FAR's.  A branch for each row above, in place of the mask, takes 215 us for 211 (14336 x 8192 x 2048).
  bool far = false;
#pragma unroll
  for (int i = 0; i < NS; ++i) far |= is_far(sa[i]);
  if (__builtin_expect(__any(far), 0)) far_rows<DT, WN>(a, r0, RB * NB, c0);
}

// ---------------------------------------------------------------- one and two rows
// A wavefront takes R rows of W, 1024 bytes of one at a time, and multiplies them with the MR rows of A from LDS by
// four-byte dot products; the lanes' sums meet by DPP.  Rows of A in a float type are put in 8 bits by every
// workgroup for itself while its first pieces of W are on their way, which saves the launch that would do it once.
// Bound by a launch, the latency of two dependent steps and W's bytes.  N = 8192, K = 2048 (16.8 MB), us, one row: 4.9,
// bf16 rows 5.4; k_gemm_i8_dir 5.5, with a launch before it 7.5.  Two rows 5.3 (5.6), bf16 6.7 (7.7); four rows 6.4
// (5.7), bf16 9.1 (7.7), so two at most.  N = 2048, K = 8192, one row 5.0 (7.2).
__device__ __forceinline__ int lanes_sum(int v) {
  v += __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, false);    // quad_perm [1, 0, 3, 2]
  v += __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, false);    // quad_perm [2, 3, 0, 1]
  v += __builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, false);   // row_half_mirror
  v += __builtin_amdgcn_mov_dpp(v, 0x140, 0xf, 0xf, false);   // row_mirror
  const auto r16 = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
  v = (int)(r16[0] + r16[1]);
  const auto r32 = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  return (int)(r32[0] + r32[1]);
}
constexpr int kVecRows = 2, kVecBytes = 65536;   // rows, and bytes of A that a workgroup holds

template <int DA, int DT, int MR, int R>
__global__ __launch_bounds__(256) void k_gemm_i8_vec(GemmI8Args a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t rows[];   // [MR][Kp]: zeros past K
  __shared__ uint32_t tops[MR][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = (blockIdx.x * 4 + wave) * R, steps = (a.K + 1023) / 1024, Kp = steps * 1024;
  constexpr int G = 8 / R;   // steps at once: 8 loads in flight
  u32x4_t w[G][R];
  auto request = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int r = 0; r < R; ++r) {   // past K or N: the first row's start, which meets zeros or is not stored
        const int k = (s0 + g) * 1024 + lane * 16;
        if (s0 + g < steps) w[g][r] = *reinterpret_cast<const u32x4_t*>(a.w + (size_t)(n0 + r < a.N ? n0 + r : 0) * a.w_row + (k < a.K ? k : 0));
      }
  };
  request(0);
  // what the last step needs, requested now
  const int om = lane / R, on = n0 + lane % R;   // the output that this lane finishes
  const bool mine = om < a.M && om < MR && on < a.N;
  float sa = 0.f, sw = 0.f, bias = 0.f, gate = 1.f, resid = 0.f;
  if (mine) {
    sw = a.w_s[on];
    if (DA == DT_I8) sa = a.a_s[om];
    if (a.bias) bias = St<DT>::ld1(a.bias, on);
    if (a.gate) gate = a.gate[(size_t)(om / a.gate_rows) * a.gate_ld + on];
    if (a.resid) resid = St<DT>::ld1(a.resid, (size_t)om * a.resid_row + on);
  }
  if constexpr (DA == DT_I8) {
    for (int i = threadIdx.x * 16; i < MR * Kp; i += 4096) {
      const int m = i / Kp, k = i - m * Kp;
      u32x4_t x = {0, 0, 0, 0};
      if (m < a.M && k < a.K) x = *reinterpret_cast<const u32x4_t*>(static_cast<const uint8_t*>(a.a) + (size_t)m * a.a_row + k);
      *reinterpret_cast<u32x4_t*>(rows + i) = x;
    }
  } else {
    uint32_t top[MR];
#pragma unroll
    for (int m = 0; m < MR; ++m) {
      top[m] = 0;
      for (int k = threadIdx.x * 8; m < a.M && k < a.K; k += 2048) {
        float v[8];
        load8<DA>(a.a, (size_t)m * a.a_row + k, v);
        top[m] = top_bits<8>(v, top[m]);
      }
      top[m] = top64(top[m]);
      if (lane == 0) tops[m][wave] = top[m];
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MR; ++m) {
      const I8Scale q(max(max(tops[m][0], tops[m][1]), max(tops[m][2], tops[m][3])));
      if (om == m) sa = q.s;
      for (int k = threadIdx.x * 8; k < Kp; k += 2048) {
        u32x2_t x = {0, 0};
        if (m < a.M && k < a.K) {
          float v[8];
          load8<DA>(a.a, (size_t)m * a.a_row + k, v);   // from the caches
          x = i8_pack8(v, q);
        }
        *reinterpret_cast<u32x2_t*>(rows + m * Kp + k) = x;
      }
    }
  }
  __syncthreads();
  int acc[MR][R];
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int r = 0; r < R; ++r) acc[m][r] = 0;
  for (int s0 = 0; s0 < steps; s0 += G) {
    if (s0) request(s0);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (s0 + g >= steps) break;
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(rows + m * Kp + (s0 + g) * 1024 + lane * 16);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[m][r] = __builtin_amdgcn_sdot4((int)w[g][r][e], (int)x[e], acc[m][r], false);
      }
    }
  }
  int sum = 0;
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int s = lanes_sum(acc[m][r]);
      if (lane == m * R + r) sum = s;
    }
  if (!mine) return;
  float v[1];
  results<true>(a, {sum}, sa, {sw}, {bias}, {gate}, {resid}, v);
  St<DT>::st1(a.out, (size_t)om * a.out_row + on, v[0]);
}

// 4 consecutive columns c.. of output row r (N % 8 == 0: in range as a whole), sa the row's scale
template <int DT>
__device__ __forceinline__ void finish4(const GemmI8Args& a, int r, int c, float sa, i32x4_t acc) {
  const f32x4_t none = {0.f, 0.f, 0.f, 0.f}, s4 = load4<DT_F32>(a.w_s, c), b4 = a.bias ? load4<DT>(a.bias, c) : none;
  const f32x4_t r4 = a.resid ? load4<DT>(a.resid, (size_t)r * a.resid_row + c) : none;
  float gate[4], v[4];
  load_gate(a, r, c, gate);
  results<true>(a, {acc[0], acc[1], acc[2], acc[3]}, sa, {s4[0], s4[1], s4[2], s4[3]}, {b4[0], b4[1], b4[2], b4[3]}, gate,
             {r4[0], r4[1], r4[2], r4[3]}, v);
  const size_t o = (size_t)r * a.out_row + c;
  if (DT == DT_BF16) *reinterpret_cast<u32x2_t*>(reinterpret_cast<uint16_t*>(a.out) + o) = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(a.out) + o) = f32x4_t{v[0], v[1], v[2], v[3]};
}

// Few rows: 16 x 16 tile, operands straight from memory, the NW waves of a workgroup on interleaved blocks of 128 k;
// their sums meet in LDS.  Bound by the latency of the loads: M = 16, N = 8192, K = 2048 6.4 us; groups of four blocks
// whatever is left, the rest clamped to the row's start, took 9.9.  16 waves were no faster (7.4; N = 2048,
// K = 8192 9.8 for 9.7).
template <int DT, int NW>
__global__ __launch_bounds__(NW * 64) void k_gemm_i8_dir(GemmI8Args a) {
  __shared__ i32x4_t red[NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int tn = (a.N + 15) / 16, m0 = (blockIdx.x / tn) * 16, n0 = (blockIdx.x % tn) * 16;
  const int m = m0 + l16 < a.M ? m0 + l16 : m0, n = n0 + l16 < a.N ? n0 + l16 : n0;   // past the matrix: never stored
  const uint8_t* pa = static_cast<const uint8_t*>(a.a) + (size_t)m * a.a_row;
  const uint8_t* pw = a.w + (size_t)n * a.w_row;
  i32x4_t acc = {0, 0, 0, 0};
  const int nk = (a.K + kQBlock - 1) / kQBlock;
  // U of the wave's blocks at once: their loads are all on their way before the first product
  auto blocks = [&](int b0, auto Uc) __attribute__((always_inline)) {
    constexpr int U = decltype(Uc)::value;
    u32x4_t x[U][2], w[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {   // chunks past K read the row's start, which is in bounds, and count for nothing
        const int k = (b0 + NW * u) * kQBlock + g * 16 + h * 64, kk = k < a.K ? k : 0;
        w[u][h] = *reinterpret_cast<const u32x4_t*>(pw + kk);
        x[u][h] = *reinterpret_cast<const u32x4_t*>(pa + kk);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool on = (b0 + NW * u) * kQBlock + g * 16 + h * 64 < a.K;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[u][h][e] = on ? w[u][h][e] : 0u;
        acc = mfma_i8(w[u][h], x[u][h], acc);
      }
  };
  int b0 = wave;
  for (; b0 + 3 * NW < nk; b0 += 4 * NW) blocks(b0, Int<4>{});
  for (; b0 + NW < nk; b0 += 2 * NW) blocks(b0, Int<2>{});
  if (b0 < nk) blocks(b0, Int<1>{});
  red[wave][lane] = acc;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int i = 1; i < NW; ++i) acc += red[i][lane];
  const int r = m0 + l16, c = n0 + 4 * g;
  if (r < a.M && c < a.N) finish4<DT>(a, r, c, a.a_s[r], acc);
}

// The same for up to 16 rows in a float type: every workgroup puts them in 8 bits for itself, into LDS, while its first
// pieces of W are on their way.  M = 4, N = 512, K = 512 2.6 us for 4.2 with a launch before; N = 2048, K = 2048 4.4 for 5.6.
constexpr int kOwnRows = 16;
size_t own_lds(int M, int K) { return (size_t)M * ((K + 127) / 128 * 128 + 16); }
template <int DA, int DT>
__global__ __launch_bounds__(512) void k_gemm_i8_own(GemmI8Args a) {
  constexpr int NW = 8, U = 4;
  extern __shared__ __attribute__((aligned(16))) uint8_t rows[];   // [M][pitch]: zeros past K
  __shared__ i32x4_t red[NW][64];
  __shared__ float scales[kOwnRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4, n0 = blockIdx.x * 16;
  const int Kp = (a.K + 127) / 128 * 128, pitch = Kp + 16, nk = Kp / kQBlock;
  const int m = l16 < a.M ? l16 : 0, n = n0 + l16 < a.N ? n0 + l16 : n0;   // past the matrix: never stored
  const uint8_t* pw = a.w + (size_t)n * a.w_row;
  u32x4_t w[U][2];
  auto request = [&](int b0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {   // chunks past K read the row's start, which is in bounds, and meet zeros
        const int k = (b0 + NW * u) * kQBlock + g * 16 + h * 64;
        if (b0 + NW * u < nk) w[u][h] = *reinterpret_cast<const u32x4_t*>(pw + (k < a.K ? k : 0));
      }
  };
  request(wave);
  for (int r = wave; r < a.M; r += NW) {
    uint32_t top = 0;
    for (int k = lane * 8; k < a.K; k += 512) {
      float v[8];
      load8<DA>(a.a, (size_t)r * a.a_row + k, v);
      top = top_bits<8>(v, top);
    }
    const I8Scale q(top64(top));
    if (lane == 0) scales[r] = q.s;
    for (int k = lane * 8; k < Kp; k += 512) {
      u32x2_t x = {0, 0};
      if (k < a.K) {
        float v[8];
        load8<DA>(a.a, (size_t)r * a.a_row + k, v);   // from the caches
        x = i8_pack8(v, q);
      }
      *reinterpret_cast<u32x2_t*>(rows + r * pitch + k) = x;
    }
  }
  __syncthreads();
  i32x4_t acc = {0, 0, 0, 0};
  for (int b0 = wave; b0 < nk; b0 += NW * U) {
    if (b0 != wave) request(b0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (b0 + NW * u >= nk) break;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        acc = mfma_i8(w[u][h], *reinterpret_cast<const u32x4_t*>(rows + m * pitch + (b0 + NW * u) * kQBlock + g * 16 + h * 64), acc);
    }
  }
  red[wave][lane] = acc;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int i = 1; i < NW; ++i) acc += red[i][lane];
  const int c = n0 + 4 * g;
  if (l16 < a.M && c < a.N) finish4<DT>(a, l16, c, scales[l16], acc);
}

// ---------------------------------------------------------------- large grids: two wave groups in turn
// 256 x 256 tile, a stage of 128 k, 8 waves in two groups of four, one wave of each group per SIMD; a stage has
// four phases, one per 32 rows of a wave's 128 x 64 block.  A phase is a memory part (fragment reads,
// DMA) and 16 MFMAs, with a barrier after each; the second group runs half a phase behind, so that on every SIMD one
// wave's MFMAs (256 cycles) cover the other's reads and DMA.
//
// Operands: 64-row pieces of 8 KB, each filled by one DMA instruction per wave, in two buffers per operand.  Phase
// p of stage k issues, in this order:
//   0: A3 of stage k+1   1: A0, B0, B1 of k+2   2: A1, B2 of k+2   3: A2, B3 of k+2
// and reads: phase 0 all B and A0 of stage k, phases 1-3 A1-A3.  So a piece's slot is refilled no earlier than
// one phase after its last read.
// K % 128 != 0: the last stage's chunks past K are out of the resource's range and load zeros.
// What bounds it: with random operands the card's power limit (the same cycles on zeros, at a higher clock, take 0.7 of the
// time at K = 8192), then the epilogue, which one workgroup a CU leaves uncovered.  So what an
// MFMA moves counts: 16 x 16 x 64 pass 8 KB of operands and sums through the registers where 32 x 32 x 32 pass 10 for the
// same products, and two in a row on the same sums less again.  M = 14336, N = 8192, K = 2048 (7 rounds of 256 tiles)
// 215 us, 2.24 POP/s (32 x 32 x 32 236, 16 x 16 x 64 with the sums in turn 218), 8192 x 8192 x 8192 394, 2.79 POP/s (437,
// 400); M = 14566 with bias and GELU 249 (274, 255).  A workgroup that walks over tiles and requests the next one's first
// stages before its epilogue took 240 us for 230 then: its stores hold the waits for the next tile's operands.
constexpr int kPPIssue[4][3] = {{3, -1, -1}, {0, 4, 5}, {1, 6, -1}, {2, 7, -1}};   // A0-A3, B0-B3
// How many of a wave's DMAs may be outstanding at the end of phase p of a stage with `left` stages
// after it (2: two or more), so that what phase p + 1 reads has landed.
constexpr int pp_vm(int p, int left) {
  int n = 0, need = -1;
  for (int j = -2; j <= 0; ++j)
    for (int q = 0; q < (j == 0 ? p + 1 : 4); ++q)
      for (int i = 0; i < 3; ++i) {
        const int pc = kPPIssue[q][i], st = pc == 3 ? j + 1 : j + 2;
        if (pc < 0 || st > left) continue;
        ++n;
        const bool next = (p == 0 && pc == 1 && st == 0) || (p == 1 && pc == 2 && st == 0) ||
                          (p == 2 && pc == 3 && st == 0) || (p == 3 && (pc == 0 || pc >= 4) && st == 1);
        if (next) need = n;
      }
  return need < 0 ? 63 : n - need;
}

template <int DT>
__global__ __launch_bounds__(512) void k_gemm_i8_pp(GemmI8Args a) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass needs the launch stub only
  constexpr int BM = 256, BN = 256, TN = 4, WN = 16 * TN, RB = kQBlock;   // RB: bytes of an LDS row
  constexpr int PC = 64 * RB, BUFA = 4 * PC, BUFB = TN * PC, OFFB = 2 * BUFA;
  constexpr int kMain = OFFB + 2 * BUFB, kEpi = 8 * sum_words<WN>(32) * 4;
  __shared__ __attribute__((aligned(1024))) char lds[kMain > kEpi ? kMain : kEpi];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int tm, tn;
  tile_at(blockIdx.x, gridDim.x, (a.M + BM - 1) / BM, (a.N + BN - 1) / BN, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int mw = wave >> 2, nw = wave & 3;
  const int nk = (a.K + kQBlock - 1) / kQBlock;   // >= 3 (host check)
  // Piece Aq holds rows 32 q .. 32 q + 31 of both wave rows, piece Bu columns 16 u .. 16 u + 15 of all
  // four wave columns.  Rows past the matrix read the tile's first row (never stored).
  auto rsrc = [](const void* p) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffff00u, 0x00020000);
  };
  __amdgpu_buffer_rsrc_t ra = rsrc(static_cast<const uint8_t*>(a.a) + (size_t)m0 * a.a_row), rw = rsrc(a.w + (size_t)n0 * a.w_row);
  const int R = wave * 8 + (lane >> 3);
  const uint32_t ch = ((lane & 7) ^ ((R >> 1) & 7)) * 16;
  uint32_t voa[4], vob[TN];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int r = (R >> 5) * 128 + q * 32 + (R & 31);
    voa[q] = (m0 + r < a.M ? (uint32_t)r * (uint32_t)a.a_row : 0u) + ch;
  }
#pragma unroll
  for (int u = 0; u < TN; ++u) {
    const int r = (R >> 4) * WN + u * 16 + (R & 15);
    vob[u] = (n0 + r < a.N ? (uint32_t)r * (uint32_t)a.w_row : 0u) + ch;
  }
  const bool cut = (int)ch >= a.K - (nk - 1) * kQBlock;   // this lane's chunk of the last stage lies past K
#define FF_DMA(rs, vo, dst, kb) __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, FF_AS3(lds + (dst) + wave * 1024), 16, vo, kb, 0, 0)
  i32x4_t acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
  const uint32_t lds0 = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) const void*)lds);
  const int fr = lane & 15, fh = lane >> 4;
  uint32_t rda[2], rdb[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const uint32_t c = ((4 * s + fh) ^ (fr >> 1)) * 16;
    rda[s] = lds0 + (mw * 32 + fr) * RB + c;
    rdb[s] = lds0 + OFFB + (nw * 16 + fr) * RB + c;
  }
  u32x4_t fa[2][2], fb[4][2];
  int kb = 0, ca = 0, cb = 0;   // this stage's byte offset along K, and its buffers
#define FF_RDA(off)                                                                               \
  do {                                                                                            \
    _Pragma("unroll") for (int s = 0; s < 2; ++s) {                                               \
      fa[0][s] = __builtin_bit_cast(u32x4_t, lds_rd128_at<(off)>(rda[s]));                        \
      fa[1][s] = __builtin_bit_cast(u32x4_t, lds_rd128_at<(off) + 16 * RB>(rda[s]));              \
    }                                                                                             \
  } while (0)
#define FF_MEM_END() asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory")
#define FF_MMA(q)                                                                                   \
  do {                                                                                              \
    _Pragma("unroll") for (int s = 0; s < 2; ++s) {                                                 \
      FF_TIE(fa[0][s]);                                                                             \
      FF_TIE(fa[1][s]);                                                                             \
    }                                                                                               \
    __builtin_amdgcn_sched_barrier(0);                                                              \
    __builtin_amdgcn_s_setprio(1);                                                                  \
    _Pragma("unroll") for (int t = 0; t < 2; ++t)                                                   \
      _Pragma("unroll") for (int u = 0; u < 4; ++u)                                                 \
        _Pragma("unroll") for (int s = 0; s < 2; ++s) {                                                \
          acc[2 * (q) + t][u] = mfma_i8(fb[u][s], fa[t][s], acc[2 * (q) + t][u]);                   \
          __builtin_amdgcn_sched_barrier(0);                                                        \
        }                                                                                           \
    __builtin_amdgcn_s_setprio(0);                                                                  \
    __builtin_amdgcn_sched_barrier(0);                                                              \
    asm volatile("s_barrier" ::: "memory");                                                         \
  } while (0)
  auto stage = [&](auto LEFTc) __attribute__((always_inline)) {
    constexpr int LEFT = decltype(LEFTc)::value;
    constexpr bool k1 = LEFT >= 1, k2 = LEFT >= 2;
    const int oa = BUFA - ca, ob = BUFB - cb;
    // phase 0
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int s = 0; s < 2; ++s) fb[u][s] = __builtin_bit_cast(u32x4_t, lds_rd128_off(rdb[s], u * PC));
    FF_RDA(0);
    if (k1) FF_DMA(ra, voa[3], 3 * PC + oa, kb + RB);
    wait_vm<pp_vm(0, LEFT)>();
    FF_MEM_END();
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int s = 0; s < 2; ++s) FF_TIE(fb[u][s]);
    FF_MMA(0);
    // phase 1
    FF_RDA(1 * PC);
    if (k2) {
      FF_DMA(ra, voa[0], ca, kb + 2 * RB);
      FF_DMA(rw, vob[0], OFFB + cb, kb + 2 * RB);
      FF_DMA(rw, vob[1], OFFB + PC + cb, kb + 2 * RB);
    }
    wait_vm<pp_vm(1, LEFT)>();
    FF_MEM_END();
    FF_MMA(1);
    // phase 2
    FF_RDA(2 * PC);
    if (k2) {
      FF_DMA(ra, voa[1], PC + ca, kb + 2 * RB);
      FF_DMA(rw, vob[2], OFFB + 2 * PC + cb, kb + 2 * RB);
    }
    wait_vm<pp_vm(2, LEFT)>();
    FF_MEM_END();
    FF_MMA(2);
    // phase 3
    FF_RDA(3 * PC);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      rda[s] += oa - ca;
      rdb[s] += ob - cb;
    }
    if (k2) {
      FF_DMA(ra, voa[2], 2 * PC + ca, kb + 2 * RB);
      FF_DMA(rw, vob[3], OFFB + 3 * PC + cb, kb + 2 * RB);
    }
    wait_vm<pp_vm(3, LEFT)>();
    FF_MEM_END();
    FF_MMA(3);
    kb += RB;
    ca = oa;
    cb = ob;
  };
  // prologue: what the stages -2 and -1 would have issued, in that order
#pragma unroll
  for (int j = -2; j < 0; ++j)
#pragma unroll
    for (int q = 0; q < 12; ++q) {
      const int pc = kPPIssue[q / 3][q % 3], s = pc == 3 ? j + 1 : j + 2;
      if (pc < 0 || s < 0) continue;
      if (pc < 4) FF_DMA(ra, voa[pc & 3], s * BUFA + pc * PC, s * RB);
      else FF_DMA(rw, vob[pc & 3], OFFB + s * BUFB + (pc - 4) * PC, s * RB);
    }
  wait_vm<3 + TN>();   // stage 0 has landed, and stage 1 but for A3 is on its way
  asm volatile("s_barrier" ::: "memory");
  if (wave >= 4) asm volatile("s_barrier" ::: "memory");   // the second group runs half a phase behind
  int left = nk - 2;   // >= 1
  do {
    if (left == 1) {   // the pieces issued from here on are the last stage's, but for A3 of the last but one
#pragma unroll
      for (int q = 0; q < 3; ++q) voa[q] = cut ? 0x80000000u : voa[q];
#pragma unroll
      for (int u = 0; u < TN; ++u) vob[u] = cut ? 0x80000000u : vob[u];
    }
    stage(Int<2>{});
  } while (--left);
  voa[3] = cut ? 0x80000000u : voa[3];
  stage(Int<1>{});
  stage(Int<0>{});
  if (wave < 4) asm volatile("s_barrier" ::: "memory");
#undef FF_MEM_END
#undef FF_DMA
#undef FF_RDA
#undef FF_MMA
  // every wave's LDS reads and DMA ended before the last barrier
  int* const own = reinterpret_cast<int*>(lds) + wave * sum_words<WN>(32);
  epilogue<DT, WN, 32, 4>(a, m0 + mw * 128, n0 + nw * WN, own, [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u) *reinterpret_cast<i32x4_t*>(own + sum_at<WN>(16 * t + fr, 16 * u + 4 * fh)) = acc[2 * i + t][u];
  });
#endif
}

// ---------------------------------------------------------------- smaller grids
// BM x BN tile, 8 waves in two groups of four; a group takes every second block of K for the whole tile
// (2 x 2 waves), so that a fragment read feeds up to four MFMAs, and has its own ring of NS blocks.
// Per block a wave has a memory slot (its fragments) and a matrix slot (the MFMAs, and behind each a DMA of the block
// NS ahead into the ring slot just read), each ended by a barrier; the second group runs one slot
// behind, one wave of each group per SIMD.  The two groups' sums meet in LDS: each finishes half of the rows.
// What bounds it: the operands' way into LDS, at 70 to 95 GB/s a CU in every tile, observed, without a cause found (64 x 64:
// 0.17 us a block of K with one workgroup on a CU, 0.36 a pair of blocks with two; 64 x 128: 0.27; 128 x 128: 0.38, 0.5
// with all CUs busy).  Neither a third block in the ring (M = 256, N = 6144, K = 2048 8.6 us for 8.4) nor half the LDS reads
// help: waves that take halves of a block's k for the whole column half, and join their sums at the end, took 9.2 us for 8.7
// there, 15.1 for 14.0 at M = 512, N = 8192.  Requesting what the epilogue needs before the first DMA: 13.9 for 13.5.
template <int DT, int BM, int BN, int NS>
__global__ __launch_bounds__(512) void k_gemm_i8_two(GemmI8Args a, int splits) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass needs the launch stub only
  constexpr int TM = BM / 32, TN = BN / 32, WN = BN / 2, RB = kQBlock;
  constexpr int STB = (BM + BN) * RB;   // bytes of a block
  constexpr int NA = BM / 32, NW = BN / 32, PER = NA + NW;   // DMA instructions of a wave and block
  constexpr int kMain = 2 * NS * STB;
  constexpr int HT = TM / 2, kXch = 8 * HT * TN * 1024, RE = HT > 1 ? 32 : 16, kEpi = kXch + 8 * sum_words<WN>(RE) * 4;
  static_assert(TM % 2 == 0 && PER <= 2 * TM * TN, "halves of the rows; a DMA behind an MFMA");
  __shared__ __attribute__((aligned(1024))) char lds[kMain > kEpi ? kMain : kEpi];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = wave >> 2, w = wave & 3, wr = w >> 1, wc = w & 1;
  int tm, tn;
  const int tiles = gridDim.x / splits, split = (int)blockIdx.x / tiles;
  tile_at((int)blockIdx.x - split * tiles, tiles, (a.M + BM - 1) / BM, (a.N + BN - 1) / BN, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  // this workgroup's blocks of K: [kb0, kb0 + nb)
  const int nk = (a.K + kQBlock - 1) / kQBlock, kb0 = (int)((long)nk * split / splits), nb = (int)((long)nk * (split + 1) / splits) - kb0;
  const int mine = (nb - grp + 1) / 2, turns = (nb + 1) / 2;
  auto rsrc = [](const void* p) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffff00u, 0x00020000);
  };
  __amdgpu_buffer_rsrc_t ra = rsrc(static_cast<const uint8_t*>(a.a) + (size_t)m0 * a.a_row), rw = rsrc(a.w + (size_t)n0 * a.w_row);
  // rows past the matrix read the tile's first row (never stored); chunks of the last block past K are
  // out of the resource's range and load zeros
  uint32_t voa[NA], vow[NW];
  unsigned cut = 0;
#pragma unroll
  for (int j = 0; j < NA + NW; ++j) {
    const int R = (w * (j < NA ? NA : NW) + (j < NA ? j : j - NA)) * 8 + (lane >> 3);
    const uint32_t ch = ((lane & 7) ^ ((R >> 1) & 7)) * 16;
    if (j < NA) voa[j < NA ? j : 0] = (m0 + R < a.M ? (uint32_t)R * (uint32_t)a.a_row : 0u) + ch;
    else vow[j < NA ? 0 : j - NA] = (n0 + R < a.N ? (uint32_t)R * (uint32_t)a.w_row : 0u) + ch;
    if ((int)ch >= a.K - (nk - 1) * kQBlock) cut |= 1u << j;
  }
  char* const ring = lds + grp * NS * STB;
  auto issue1 = [&](int i, int slot, int j) __attribute__((always_inline)) {   // DMA j of the group's block i
    const int kt = kb0 + 2 * i + grp, kb = kt * RB;
    const unsigned c = kt == nk - 1 ? cut : 0u;
    char* const dst = ring + slot * STB;
    if (j < NA)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, FF_AS3(dst + (w * NA + j) * 1024), 16, voa[j < NA ? j : 0] | (c >> j & 1u) << 31, kb, 0, 0);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, FF_AS3(dst + BM * RB + (w * NW + j - NA) * 1024), 16,
                                               vow[j < NA ? 0 : j - NA] | (c >> j & 1u) << 31, kb, 0, 0);
  };
  i32x4_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
  const int fr = lane & 15, fh = lane >> 4;
  const uint32_t lds0 = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) const void*)lds);
  uint32_t rda[2], rdw[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const uint32_t c = ((4 * s + fh) ^ (fr >> 1)) * 16, o = lds0 + grp * NS * STB;
    rda[s] = o + (wr * (BM / 2) + fr) * RB + c;
    rdw[s] = o + (BM + wc * WN + fr) * RB + c;
  }
  u32x4_t fa[2 * TM], fw[2 * TN];
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (i < mine) {
#pragma unroll
      for (int j = 0; j < PER; ++j) issue1(i, i, j);
    }
  // the first block has landed (a wait for all of them: 8.7 us for 8.4 at M = 256, N = 6144, K = 2048)
  if (mine >= NS) wait_vm<(NS - 1) * PER>();
  else wait_vm<0>();
  asm volatile("s_barrier" ::: "memory");
  if (grp) asm volatile("s_barrier" ::: "memory");   // the second group runs one slot behind
  int slot = 0;
  auto turn = [&](int i, auto Mc) __attribute__((always_inline)) {
    constexpr bool more = decltype(Mc)::value != 0;   // a block NS ahead is left
    // memory slot
    const uint32_t so = slot * STB;
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int s = 0; s < 2; ++s) fw[2 * t + s] = __builtin_bit_cast(u32x4_t, lds_rd128_off(rdw[s] + so, t * 16 * RB));
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
      for (int s = 0; s < 2; ++s) fa[2 * t + s] = __builtin_bit_cast(u32x4_t, lds_rd128_off(rda[s] + so, t * 16 * RB));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int t = 0; t < 2 * TN; ++t) FF_TIE(fw[t]);
#pragma unroll
    for (int t = 0; t < 2 * TM; ++t) FF_TIE(fa[t]);
    asm volatile("s_barrier" ::: "memory");
    // matrix slot
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int t = 0; t < TM; ++t) {
          acc[t][j] = mfma_i8(fw[2 * j + s], fa[2 * t + s], acc[t][j]);
          const int at = (s * TN + j) * TM + t;
          if (more && at < PER) {
            __builtin_amdgcn_sched_barrier(0);
            issue1(i + NS, slot, at);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    // the next block has landed; the ones after it may be on their way
    wait_vm<more ? (NS - 1) * PER : 0>();
    slot = slot == NS - 1 ? 0 : slot + 1;
    asm volatile("s_barrier" ::: "memory");
  };
  int i = 0;
  for (; i < mine - NS; ++i) turn(i, Int<1>{});
  for (; i < mine; ++i) turn(i, Int<0>{});
  if (mine < turns) {   // the second group, one block short
    asm volatile("s_barrier" ::: "memory");
    asm volatile("s_barrier" ::: "memory");
  }
  if (!grp) asm volatile("s_barrier" ::: "memory");
  // every wave's LDS reads and DMA ended before the last barrier; each group finishes half of the rows
  i32x4_t* const xch = reinterpret_cast<i32x4_t*>(lds) + lane;
  i32x4_t fin[HT][TN];
  auto half = [&](auto Gc) __attribute__((always_inline)) {
    constexpr int G = decltype(Gc)::value;
#pragma unroll
    for (int t = 0; t < HT; ++t)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        xch[((wave * HT + t) * TN + j) * 64] = acc[(1 - G) * HT + t][j];
        fin[t][j] = acc[G * HT + t][j];
      }
  };
  if (grp) half(Int<1>{});
  else half(Int<0>{});
  __syncthreads();
#pragma unroll
  for (int t = 0; t < HT; ++t)
#pragma unroll
    for (int j = 0; j < TN; ++j) fin[t][j] += xch[(((wave ^ 4) * HT + t) * TN + j) * 64];
  const int r0 = m0 + wr * (BM / 2) + grp * HT * 16, c0 = n0 + wc * WN;
  if (splits > 1) {   // bare sums for k_gemm_i8_join, each lane's four columns of its rows
    int* const part = a.part + (size_t)split * a.M * a.N;
#pragma unroll
    for (int t = 0; t < HT; ++t)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int r = r0 + 16 * t + fr, c = c0 + 16 * j + 4 * fh;
        if (r < a.M && c < a.N) *reinterpret_cast<i32x4_t*>(part + (size_t)r * a.N + c) = fin[t][j];
      }
    return;
  }
  int* const own = reinterpret_cast<int*>(lds + kXch) + wave * sum_words<WN>(RE);
  epilogue<DT, WN, RE, HT * 16 / RE>(a, r0, c0, own, [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < RE / 16; ++t)
#pragma unroll
      for (int j = 0; j < TN; ++j) *reinterpret_cast<i32x4_t*>(own + sum_at<WN>(16 * t + fr, 16 * j + 4 * fh)) = fin[i * (RE / 16) + t][j];
  });
#endif
}

// Joins the splits of K: 8 columns of a row a thread
template <int DT>
__global__ __launch_bounds__(256) void k_gemm_i8_join(GemmI8Args a, int splits) {
  const int per = a.N / 8;
  const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (size_t)a.M * per) return;
  const int r = (int)(id / per), c = (int)(id % per) * 8;
  i32x4_t s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  for (int i = 0; i < splits; ++i) {
    const i32x4_t* p = reinterpret_cast<const i32x4_t*>(a.part + (size_t)i * a.M * a.N + id * 8);
    s[0] += p[0];
    s[1] += p[1];
  }
  float v[8], sw[8], bias[8], resid[8], gate[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = resid[e] = 0.f;
  load8<DT_F32>(a.w_s, c, sw);
  if (a.bias) load8<DT>(a.bias, c, bias);
  if (a.resid) load8<DT>(a.resid, (size_t)r * a.resid_row + c, resid);
  load_gate(a, r, c, gate);
  results<true>(a, {s[0][0], s[0][1], s[0][2], s[0][3], s[1][0], s[1][1], s[1][2], s[1][3]}, a.a_s[r], sw, bias, gate, resid, v);
  store8<DT>(a.out, (size_t)r * a.out_row + c, v);
}

// ---------------------------------------------------------------- choice
long tiles(long M, long N, long t) { return ((M + t - 1) / t) * ((N + t - 1) / t); }

// rows that the call puts in 8 bits itself, and their scales behind them
size_t rows_bytes(int a_dtype, int M, int K) { return a_dtype == DT_I8 ? 0 : ((size_t)M * K + 255) / 256 * 256 + ((size_t)M * 4 + 255) / 256 * 256; }

// The kernel of a shape by estimated time (us): fits to 60 shapes of 1 to 14566 rows, N and K of 256 to 8192, 8-bit rows,
// bf16 out, nothing behind the product.  nk: blocks of K; t: tiles.  Examples, measured with each kernel:
//   M 16 N 8192 K 2048: 16 x 16 6.1 us, 64 x 64 6.6; M 64 N 2048: 5.6, 5.7; M 128 N 2048: 9.0, 5.7
//   M 64 N 2048 K 8192: 64 x 64 14.1 us, with 2 / 4 / 8 splits of K 12.4 / 10.9 / 12.5; 16 x 16 16.6
//   M 256 N 6144 K 2048: 64 x 128 8.4 us, 64 x 64 9.4, 128 x 128 11.4; M 1024 N 2048 K 8192: 21.4, 26.4, 28.1
//   M 512 N 8192 K 2048: 128 x 128 13.5 us, 64 x 128 16.7, 64 x 64 17.5, 256 x 256 26.0
//   M 4608 N 6144 K 2048: 256 x 256 55.8 us, 128 x 128 80.4, 64 x 64 95.4
// Of 19 shapes of 16 to 14566 rows the choice is the fastest for 17; 256 x 256 tiles are taken where 128 x 128 ones are for M 2048
// N 3456 K 1152 (20.1 us for 17.9) and M 700 N 8192 K 1024 (18.6 for 16.5).  fp32 outputs with bias, gate and residual, whose
// epilogue the estimates do not know: the fastest for 16; 64 x 64 tiles would be for these two (27.1 us for 24.6, 25.1
// for 20.0) and M 333 N 4096 K 1024 (8.4 for 8.0).
double us_dir(double t, double nk) { return 2.2 + fmax(t * nk * 0.45e-3, 0.115 * nk); }
double us_64(double t, double nk) {
  if (t <= 256) return 3.2 + (0.17 + 0.06 * t / 256) * nk;
  if (t <= 512) return 4.0 + (0.30 + 0.04 * (t - 256) / 256) * nk;   // two workgroups on some CUs
  return 2.7 + ceil(t / 256) / 2 * (0.36 * nk + 1.3);
}
double us_join(int splits, double outputs) { return 1.2 + splits * (0.55 + 0.5e-6 * outputs); }
double us_64x128(double t, double nk) {
  return t <= 256 ? 3.5 + t / 256 + (0.235 + 0.05 * t / 256) * nk : 2.7 + ceil(t / 256) * (0.285 * nk + 2.4);
}
double us_128(double t, double nk) { return t <= 256 ? 5.2 + (0.37 + 0.10 * t / 256) * nk : 2.7 + ceil(t / 256) * (0.5 * nk + 2.2); }
// rounds of all 256 CUs run at the power limit, a last one with fewer at a higher clock
double us_256(double t, double nk) {
  const double full = floor(t / 256), last = t / 256 - full, f = last * last;
  return 4.0 + full * (1.43 * nk + 6.8) + (last > 0 ? (0.90 + 0.53 * f) * nk + 1.0 + 5.8 * f : 0.0);
}

struct Timed { I8Plan plan; double us; };
Timed best_of(int M, int N, int K, bool cut) {
  const int nk = (K + kQBlock - 1) / kQBlock;
  const double t64 = (double)tiles(M, N, 64), t256 = (double)tiles(M, N, 256);
  Timed b{{I8_TILE128, 1, M}, us_128((double)tiles(M, N, 128), nk)};
  auto take = [&](int k, int splits, int head, double us) {
    if (us < b.us) b = Timed{{k, splits, head}, us};
  };
  if (M <= 256) take(I8_DIR, 1, M, us_dir((double)tiles(M, N, 16), nk));
  for (int s = 1; s <= 8; s *= 2) {
    if (s > 1 && nk / s < 8) break;
    take(I8_TILE64, s, M, us_64(t64 * s, (double)nk / s) + (s > 1 ? us_join(s, (double)M * N) : 0.0));
  }
  take(I8_TILE64x128, 1, M, us_64x128((double)((M + 63) / 64) * ((N + 127) / 128), nk));
  if (nk < 3) return b;
  take(I8_TILE256, 1, M, us_256(t256, nk));
  // Rows behind whole rounds of 256 x 256 tiles in a launch of their own, with the tile that suits them (M = 14566,
  // N = 8192, K = 2048, whose eighth round has 32 tiles: 240 us for 257 with 32 x 32 x 32 MFMAs)
  const int per = (N + 255) / 256;
  const int head = (int)(floor(t256 / 256) * 256) / per * 256;
  if (cut && head > 0 && head < M) take(I8_TILE256, 1, head, us_256((double)tiles(head, N, 256), nk) + best_of(M - head, N, K, false).us - 0.5);
  return b;
}

}  // namespace

I8Plan gemm_i8_plan(int out_dtype, int M, int N, int K) {
  (void)out_dtype;   // both types by the fits to bf16's times
  if (M <= kVecRows && (size_t)M * ((K + 1023) / 1024 * 1024) <= kVecBytes) return I8Plan{I8_VEC, 1, M};
  return best_of(M, N, K, true).plan;
}

namespace {

// The plan of the rows behind a plan's head
I8Plan tail_plan(const I8Plan& p, int M, int N, int K) { return best_of(M - p.head, N, K, false).plan; }
size_t part_bytes(const I8Plan& p, int M, int N) { return p.splits > 1 ? (size_t)p.splits * M * N * 4 : 0; }

// Whether a call of few rows in a float type puts them in 8 bits in the product's own launch: while a wavefront's rows are
// short (M = 16, N = 2048, K = 2048 6.3 us for 6.1 with a launch before, 4 rows of K = 8192 14.5 for 10.4), and what the
// workgroups read of them together is little (M = 8, N = 8192, K = 2048 8.0 us for 8.2, 16 rows 10.6 for 8.7)
bool own_rows(int a_dtype, int M, int N, int K) {
  return a_dtype != DT_I8 && M <= kOwnRows && (M + 7) / 8 * K <= 4608 && (int64_t)M * K * ((N + 15) / 16) <= 1 << 23;
}

template <int DA, int DT>
void launch_own(const GemmI8Args& a, hipStream_t s) {
  FF_LAUNCH((k_gemm_i8_own<DA, DT>), (unsigned)((a.N + 15) / 16), 512, own_lds(a.M, a.K), s, a);
}

template <int DA, int DT>
void launch_vec(const GemmI8Args& a, hipStream_t s) {
  const size_t lds = (size_t)a.M * ((a.K + 1023) / 1024 * 1024);
  const unsigned wg = (unsigned)((a.N + 7) / 8);
  if (a.M == 1) FF_LAUNCH((k_gemm_i8_vec<DA, DT, 1, 2>), wg, 256, lds, s, a);
  else FF_LAUNCH((k_gemm_i8_vec<DA, DT, 2, 2>), wg, 256, lds, s, a);
}

template <int DT>
hipError_t launch_i8(const GemmI8Args& a, const I8Plan& p, hipStream_t s) {
  switch (p.kernel) {
    case I8_DIR: FF_LAUNCH((k_gemm_i8_dir<DT, 8>), (unsigned)tiles(a.M, a.N, 16), 512, 0, s, a); break;
    case I8_TILE64: FF_LAUNCH((k_gemm_i8_two<DT, 64, 64, 2>), (unsigned)(tiles(a.M, a.N, 64) * p.splits), 512, 0, s, a, p.splits); break;
    case I8_TILE64x128: FF_LAUNCH((k_gemm_i8_two<DT, 64, 128, 2>), (unsigned)((a.M + 63) / 64) * (unsigned)((a.N + 127) / 128), 512, 0, s, a, 1); break;
    case I8_TILE128: FF_LAUNCH((k_gemm_i8_two<DT, 128, 128, 2>), (unsigned)tiles(a.M, a.N, 128), 512, 0, s, a, 1); break;
    case I8_TILE256: FF_LAUNCH((k_gemm_i8_pp<DT>), (unsigned)tiles(a.M, a.N, 256), 512, 0, s, a); break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const size_t wg = ((size_t)a.M * (a.N / 8) + 255) / 256;
  FF_LAUNCH(k_gemm_i8_join<DT>, (unsigned)wg, 256, 0, s, a, p.splits);
  return hipGetLastError();
}

}  // namespace

size_t gemm_i8_workspace(int a_dtype, int out_dtype, int M, int N, int K) {
  if (M <= 0) return 0;
  const I8Plan p = gemm_i8_plan(out_dtype, M, N, K);
  if (p.kernel == I8_VEC || own_rows(a_dtype, M, N, K)) return 0;
  return rows_bytes(a_dtype, M, K) + (p.head < M ? part_bytes(tail_plan(p, M, N, K), M - p.head, N) : part_bytes(p, M, N));
}

hipError_t gemm_i8(int a_dtype, int out_dtype, const GemmI8Args& a0, hipStream_t s) {
  if (a0.M <= 0) return hipSuccess;
  const I8Plan p = gemm_i8_plan(out_dtype, a0.M, a0.N, a0.K);
  const bool bf16 = out_dtype == DT_BF16;
  GemmI8Args a = a0;
  if (p.kernel == I8_VEC) {
    if (a_dtype == DT_I8) bf16 ? launch_vec<DT_I8, DT_BF16>(a, s) : launch_vec<DT_I8, DT_F32>(a, s);
    else if (a_dtype == DT_BF16) bf16 ? launch_vec<DT_BF16, DT_BF16>(a, s) : launch_vec<DT_BF16, DT_F32>(a, s);
    else bf16 ? launch_vec<DT_F32, DT_BF16>(a, s) : launch_vec<DT_F32, DT_F32>(a, s);
    return hipGetLastError();
  }
  if (own_rows(a_dtype, a.M, a.N, a.K)) {
    if (a_dtype == DT_BF16) bf16 ? launch_own<DT_BF16, DT_BF16>(a, s) : launch_own<DT_BF16, DT_F32>(a, s);
    else bf16 ? launch_own<DT_F32, DT_BF16>(a, s) : launch_own<DT_F32, DT_F32>(a, s);
    return hipGetLastError();
  }
  if (a_dtype != DT_I8) {
    uint8_t* const q = reinterpret_cast<uint8_t*>(a0.part);
    float* const qs = reinterpret_cast<float*>(q + ((size_t)a.M * a.K + 255) / 256 * 256);
    const hipError_t e = quant_i8(a_dtype, QuantI8Args{a0.a, a0.a_row, q, a.K, qs, a.M, a.K}, s);
    if (e != hipSuccess) return e;
    a.a = q;
    a.a_row = a.K;
    a.a_s = qs;
    a.part = reinterpret_cast<int*>(q + rows_bytes(a_dtype, a.M, a.K));
  }
  if (p.head < a.M) {
    GemmI8Args h = a;
    h.M = p.head;
    const hipError_t e = bf16 ? launch_i8<DT_BF16>(h, p, s) : launch_i8<DT_F32>(h, p, s);
    if (e != hipSuccess) return e;
    const size_t es = dsize(out_dtype), at = (size_t)p.head;
    const I8Plan tail = tail_plan(p, a.M, a.N, a.K);
    a.a = static_cast<const uint8_t*>(a.a) + at * a.a_row;
    a.a_s += at;
    a.out = static_cast<char*>(a.out) + at * a.out_row * es;
    if (a.resid) a.resid = static_cast<const char*>(a.resid) + at * a.resid_row * es;
    a.row0 = p.head;
    a.M -= p.head;
    return bf16 ? launch_i8<DT_BF16>(a, tail, s) : launch_i8<DT_F32>(a, tail, s);
  }
  return bf16 ? launch_i8<DT_BF16>(a, p, s) : launch_i8<DT_F32>(a, p, s);
}

}  // namespace ff
