// Products of 8-bit operands with a scale for each block of 128 along K:
//   out = act(sum_b a_s[b, m] w_s[n / 128, b] (sum_{k in b} a[m, k] w[n, k]) + bias) + resid
// One v_mfma_f32_16x16x128_f8f6f4 covers a block of 16 rows, 16 columns and 128 k.  Its sum starts
// at zero and is added to the fp32 accumulators times a_s w_s.  The A operand holds weight rows
// (output columns n), the B operand activation rows m: lane l then holds output row l % 16 and
// columns 4 (l / 16) + 0..3.  Lane l of an operand takes row l % 16 and two 16-byte chunks of the
// block, chunks l / 16 and 4 + l / 16; which k stands where within the block does not matter as
// long as both operands agree.
#include "dev_common.h"
#include <math.h>

namespace ff {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4_t mfma_q8(i32x8_t a, i32x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);   // e4m3, no block scales
}
__device__ __forceinline__ i32x8_t join(u32x4_t lo, u32x4_t hi) {
  return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// fp32 outputs take exact products: e4m3 values widened to bf16 (exactly) on the bf16 MFMAs, whose
// sums keep 24 bits (7.6e-8 of the result off on operands of widely spread exponents).  The 8-bit
// MFMAs align a block's products to fewer bits (5.5e-5 off on the same operands, 1.5e-5 on normal
// ones; a block's sum by at most 2^-11 of its largest |a| times its largest |w|, as measured): far below a bf16 output's rounding of 2^-9, far above fp32's.
__device__ __forceinline__ bf16x8_t widen(uint32_t lo, uint32_t hi) {
  const bf16x2_t p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true)};
  return bf16x8_t{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}
// one block's product of 16 weight rows (w0, w1) and 16 activation rows (x0, x1)
template <int DT>
__device__ __forceinline__ f32x4_t product(u32x4_t w0, u32x4_t w1, u32x4_t x0, u32x4_t x1) {
  f32x4_t p = {0.f, 0.f, 0.f, 0.f};
  if (DT == DT_BF16) return mfma_q8(join(w0, w1), join(x0, x1), p);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w0[2 * h], w0[2 * h + 1]), widen(x0[2 * h], x0[2 * h + 1]), p, 0, 0, 0);
    p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w1[2 * h], w1[2 * h + 1]), widen(x1[2 * h], x1[2 * h + 1]), p, 0, 0, 0);
  }
  return p;
}

// 4 consecutive columns c.. of output row r (N % 8 == 0: in range as a whole): what is added to the
// product, and the rest of the epilogue
struct Add4 { f32x4_t bias, resid; };
template <int DT>
__device__ __forceinline__ f32x4_t load4(const void* p, size_t i) {
  if (DT == DT_F32) return *reinterpret_cast<const f32x4_t*>(reinterpret_cast<const float*>(p) + i);
  const u32x2_t w = *reinterpret_cast<const u32x2_t*>(reinterpret_cast<const uint16_t*>(p) + i);
  return f32x4_t{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
}
template <int DT>
__device__ __forceinline__ Add4 request4(const GemmQ8Args& a, int r, int c) {
  Add4 x{{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  if (a.bias) x.bias = load4<DT>(a.bias, c);
  if (a.resid) x.resid = load4<DT>(a.resid, (size_t)r * a.resid_row + c);
  return x;
}
template <int DT>
__device__ __forceinline__ void finish4(const GemmQ8Args& a, const Add4& x, int r, int c, f32x4_t v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] += x.bias[e];
    if (a.gelu) v[e] = gelu_tanh_f(v[e]);
    v[e] += x.resid[e];
  }
  const size_t o = (size_t)r * a.out_row + c;
  if (DT == DT_BF16) *reinterpret_cast<u32x2_t*>(reinterpret_cast<uint16_t*>(a.out) + o) = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(a.out) + o) = v;
}

// Few rows: 16 x 16 tile, operands straight from memory, the NW waves of a workgroup on interleaved
// blocks of K; their sums meet in LDS in wave order.  Bound by the latency of the loads: M = 1, N = 8192,
// K = 2048 6.2 us (16.8 MB of weights).  The compiler puts a block's loads behind the test that ends the
// walk, so a wave has one block (four 16-byte loads) in flight, not the four that the loop requests, and
// with bf16 outputs the first wave waits for bias and residual, which it widens at once.
// Two or four 16-row tiles a workgroup, to read the weights once for them, were slower (M = 64, N =
// 2048, K = 2048: 6.0 us against 7.1 with four): the rows come from the caches.
template <int DT, int NW>
__global__ __launch_bounds__(NW * 64) void k_gemm_q8_dir(GemmQ8Args a) {
  constexpr int U = 4;
  __shared__ f32x4_t red[NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int tn = (a.N + 15) / 16, m0 = (blockIdx.x / tn) * 16, n0 = (blockIdx.x % tn) * 16;
  const int m = m0 + l16 < a.M ? m0 + l16 : m0, n = n0 + l16 < a.N ? n0 + l16 : n0;   // past the matrix: never stored
  const uint8_t* pa = a.a + (size_t)m * a.a_row;
  const uint8_t* pw = a.w + (size_t)n * a.w_row;
  const float* sa = a.a_s + m;
  const float* sw = a.w_s + (size_t)(n0 / kQBlock) * a.ws_ld;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  // the first wave finishes the tile: what it adds is read before the operands
  const bool in = m0 + l16 < a.M && n0 + 4 * g < a.N;
  Add4 extra{acc, acc};
  if (wave == 0) extra = request4<DT>(a, in ? m0 + l16 : m0, in ? n0 + 4 * g : n0);
  const int nk = (a.K + kQBlock - 1) / kQBlock;
  for (int b0 = wave; b0 < nk; b0 += NW * U) {
    u32x4_t x[U][2], w[U][2];
    float s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // blocks and chunks past K read the row's start, which is in bounds, and count for nothing
      const int b = b0 + NW * u < nk ? b0 + NW * u : 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = b * kQBlock + g * 16 + h * 64, kk = k < a.K ? k : 0;
        w[u][h] = *reinterpret_cast<const u32x4_t*>(pw + kk);
        x[u][h] = *reinterpret_cast<const u32x4_t*>(pa + kk);
      }
      s[u] = sa[(size_t)b * a.as_ld] * sw[b];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (b0 + NW * u >= nk) break;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool on = (b0 + NW * u) * kQBlock + g * 16 + h * 64 < a.K;
#pragma unroll
        for (int e = 0; e < 4; ++e) {   // both operands, so that 0 * 0 is added
          w[u][h][e] = on ? w[u][h][e] : 0u;
          x[u][h][e] = on ? x[u][h][e] : 0u;
        }
      }
      const f32x4_t p = product<DT>(w[u][0], w[u][1], x[u][0], x[u][1]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(p[e], s[u], acc[e]);
    }
  }
  red[wave][lane] = acc;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int i = 1; i < NW; ++i) {
    const f32x4_t p = red[i][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += p[e];
  }
  if (in) finish4<DT>(a, extra, m0 + l16, n0 + 4 * g, acc);
}

// 8 values as they are stored, to be added later
template <int DT> struct Raw8;
template <> struct Raw8<DT_BF16> {
  typedef u32x4_t type;
  __device__ __forceinline__ static type load(const void* p, size_t i) { return *reinterpret_cast<const u32x4_t*>(reinterpret_cast<const uint16_t*>(p) + i); }
  __device__ __forceinline__ static void add(type w, float* v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
};
template <> struct Raw8<DT_F32> {
  struct type { f32x4_t x[2]; };
  __device__ __forceinline__ static type load(const void* p, size_t i) {
    const f32x4_t* q = reinterpret_cast<const f32x4_t*>(reinterpret_cast<const float*>(p) + i);
    return type{{q[0], q[1]}};
  }
  __device__ __forceinline__ static void add(const type& w, float* v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += w.x[e / 4][e % 4];
  }
};

// Epilogue of a wavefront's 16 TM x 16 TN block at (r0, c0), acc in the MFMA layout (lane l: row l % 16
// of each 16, columns 4 (l / 16) + 0..3): 32 rows at a time go through the wave's own LDS region as
// fp32 rows and come back as 8-column pieces, so that every load and store of bias, residual and
// output is 16 bytes wide and covers whole row segments (in the MFMA layout each store would put 8
// bytes into each of 16 rows).  N % 8 == 0: a piece is in range as a whole.  The caller has retired
// all waves' reads of what the region overlays.
template <int DT, int TM, int TN>
__device__ __forceinline__ void epilogue(const GemmQ8Args& a, int r0, int c0, const f32x4_t (&acc)[TM][TN], float* lds) {
  constexpr int WN = 16 * TN, LDW = WN + 4, CPR = WN / 8, RPP = 64 / CPR, RB = TM > 1 ? 32 : 16, NPASS = RB / RPP;
  static_assert(64 % CPR == 0 && NPASS >= 1, "whole rows a pass");
  const int lane = threadIdx.x & 63, fr = lane & 15, fh = lane >> 4;
  const int pc = lane % CPR * 8, pr = lane / CPR, c = c0 + pc;
  const int cl = c < a.N ? c : 0;   // loads past the matrix read its first column or last row
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = 0.f;
  if (a.bias) load8<DT>(a.bias, cl, bias);
  constexpr int NB = TM * 16 / RB;
  // the residual's pieces are requested a block ahead
  typedef typename Raw8<DT>::type raw_t;
  raw_t res[2][NPASS];
  auto request = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < NPASS; ++p)
      res[i & 1][p] = Raw8<DT>::load(a.resid, (size_t)min(r0 + i * RB + p * RPP + pr, a.M - 1) * a.resid_row + cl);
  };
  if (a.resid) request(0);
#pragma unroll
  for (int i = 0; i < NB; ++i) {
#pragma unroll
    for (int t = 0; t < RB / 16; ++t)
#pragma unroll
      for (int u = 0; u < TN; ++u)
        *reinterpret_cast<f32x4_t*>(lds + (16 * t + fr) * LDW + 16 * u + 4 * fh) = acc[i * (RB / 16) + t][u];
    if (a.resid && i + 1 < NB) request(i + 1);
#pragma unroll
    for (int p = 0; p < NPASS; ++p) {
      const int r = r0 + i * RB + p * RPP + pr;
      const f32x4_t x0 = *reinterpret_cast<const f32x4_t*>(lds + (p * RPP + pr) * LDW + pc);
      const f32x4_t x1 = *reinterpret_cast<const f32x4_t*>(lds + (p * RPP + pr) * LDW + pc + 4);
      float v[8] = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += bias[e];
      if (a.gelu) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = gelu_tanh_f(v[e]);
      }
      if (a.resid) Raw8<DT>::add(res[i & 1][p], v);
      if (r < a.M && c < a.N) store8<DT>(a.out, (size_t)r * a.out_row + c, v);
    }
  }
}

// Workgroup -> tile: workgroups go round-robin over the 8 XCDs, so every XCD gets a contiguous range
// of tiles, in groups of 8 tile rows, whose operand rows its L2 then shares.
__device__ __forceinline__ void tile_at(int wg, int n, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int full = n / 8 * 8;
  const int id = wg < full ? (wg % 8) * (full / 8) + wg / 8 : wg;
  const int per = 8 * tiles_n, first = id / per * 8, size = min(tiles_m - first, 8), in = id % per;
  tm = __builtin_amdgcn_readfirstlane(first + in % size);
  tn = __builtin_amdgcn_readfirstlane(in / size);
}

// ---------------------------------------------------------------- large grids: two wave groups in turn
// 256 x 256 tile, a stage of one 128-wide block of K, 8 waves in two groups of four, one wave of
// each group per SIMD; a stage has four phases, one per 32 rows of a wave's 128 x 64 block.  A
// phase is a memory part (fragment reads, DMA) and 8 MFMAs among the fused multiply-adds that scale
// their sums into the accumulators, with a barrier after each; the second group runs half a phase
// behind, so that on every SIMD one wave's MFMAs (256 cycles) cover the other's reads and DMA.
//
// Operands: 64-row pieces of 8 KB, each filled by one DMA instruction per wave, in two buffers per
// operand, and the 256 rows' scales of a stage (1 KB, one 4-byte DMA a lane; waves w and w + 4 write
// the same values) in a ring of four.  Phase p of stage k issues, in this order:
//   0: A3 of stage k+1, the scales of k+2   1: A0, B0, B1 of k+2   2: A1, B2 of k+2   3: A2, B3 of k+2
// and reads: phase 0 all B and A0 of stage k, phases 1-3 A1-A3, each phase its rows' scales.  So a
// piece's slot is refilled no earlier than one phase after its last read.
// The weight's scale of a stage is a scalar per wave (its columns lie in one block of 128).
// K % 128 != 0: the last stage's chunks past K are out of the resource's range and load zeros.
// What bounds it: with random operands the card's power limit in the main loop, then the epilogue, which
// one workgroup a CU leaves uncovered, and the last round of tiles.  M = 14566, N = 8192, K = 2048 (7.1 rounds
// of 256 tiles, so 8): 248 to 271 us on different cards (1.8 to 2.0 PFLOP/s; a library's product with one
// scale a tensor takes 241), on the first of them 273 with bias and GELU, 279 with bias and residual, and 233
// for M = 14336, 7 rounds.
constexpr int kPPIssue[4][3] = {{3, 8, -1}, {0, 4, 5}, {1, 6, -1}, {2, 7, -1}};   // A0-A3, B0-B3, scales
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

__global__ __launch_bounds__(512) void k_gemm_q8_pp(GemmQ8Args a) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass needs the launch stub only
  constexpr int BM = 256, BN = 256, TN = 4, WN = 16 * TN, RB = kQBlock;   // RB: bytes of an LDS row
  constexpr int PC = 64 * RB, BUFA = 4 * PC, BUFB = TN * PC, OFFB = 2 * BUFA, OFFS = OFFB + 2 * BUFB;
  constexpr int kMain = OFFS + 4 * 1024, kEpi = 8 * 32 * (WN + 4) * 4;
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
  __amdgpu_buffer_rsrc_t ra = rsrc(a.a + (size_t)m0 * a.a_row), rw = rsrc(a.w + (size_t)n0 * a.w_row), rs = rsrc(a.a_s + m0);
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
  const uint32_t vos = (uint32_t)min((wave & 3) * 64 + lane, a.M - 1 - m0) * 4u;
  const uint32_t sstep = (uint32_t)a.as_ld * 4u;
  const bool cut = (int)ch >= a.K - (nk - 1) * kQBlock;   // this lane's chunk of the last stage lies past K
#define FF_DMA(rs, vo, dst, kb) __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, FF_AS3(lds + (dst) + wave * 1024), 16, vo, kb, 0, 0)
#define FF_DMAS(st) __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, FF_AS3(lds + OFFS + ((st) & 3) * 1024 + (wave & 3) * 256), 4, vos, (st) * sstep, 0, 0)
  f32x4_t acc[8][TN], part[3];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 3; ++i) part[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int fr = lane & 15, fh = lane >> 4;
  const uint32_t lds0 = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) const void*)lds);
  uint32_t rda[2], rdb[2];   // fragment addresses of the two 16-byte chunks, current buffers
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const uint32_t c = ((4 * s + fh) ^ (fr >> 1)) * 16;
    rda[s] = lds0 + (mw * 32 + fr) * RB + c;
    rdb[s] = lds0 + OFFB + (nw * 16 + fr) * RB + c;
  }
  const uint32_t rds = lds0 + OFFS + (mw * 128 + fr) * 4;
  const float* wsc = a.w_s + (size_t)min((n0 + nw * WN) / kQBlock, (a.N - 1) / kQBlock) * a.ws_ld;
  float vsw = wsc[min(lane, nk - 1)];   // the weight's scales of 64 stages, one a lane
  u32x4_t fa[4], fb[2 * TN];
  float sw = 0.f;
  int kb = 0, st = 0, ca = 0, cb = 0;   // this stage's byte offset along K and number, and its buffers
#define FF_RDA(off)                                                                               \
  do {                                                                                            \
    fa[0] = __builtin_bit_cast(u32x4_t, lds_rd128_at<(off)>(rda[0]));                             \
    fa[1] = __builtin_bit_cast(u32x4_t, lds_rd128_at<(off)>(rda[1]));                             \
    fa[2] = __builtin_bit_cast(u32x4_t, lds_rd128_at<(off) + 16 * RB>(rda[0]));                   \
    fa[3] = __builtin_bit_cast(u32x4_t, lds_rd128_at<(off) + 16 * RB>(rda[1]));                   \
  } while (0)
#define FF_RDS(q)                                                                                                          \
  do {                                                                                                                     \
    const uint32_t ad = rds + (st & 3) * 1024;                                                                             \
    asm volatile("ds_read2_b32 %0, %1 offset0:%2 offset1:%3" : "=v"(sv) : "v"(ad), "n"((q) * 32), "n"((q) * 32 + 16) : "memory"); \
  } while (0)
  f32x2_t sv = {0.f, 0.f};   // the scales of the phase's rows
  float sp[2] = {0.f, 0.f};  // ... times the weight's
#define FF_MEM_END() asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory")
  // The products of phase q's rows, from zero, and their scaled addition two products behind, between
  // the MFMAs; the last two open the next memory part.  Beside additions that stand as a whole in the
  // memory part this takes 27 registers less and 11% fewer cycles at M = 14566, N = 8192, K = 2048
  // (598 k for 670 k), of which the time keeps little, 271 us for 272: the clock gives way under the
  // load (1.90 GHz for 2.09 with every CU at work).  At 4608 x 2048 x 2048 it is 31.9 us for 33.8.
#define FF_ADD1(q, i)                                                                               \
  do {                                                                                              \
    _Pragma("unroll") for (int e = 0; e < 4; ++e)                                                   \
      acc[2 * (q) + (i) / TN][(i) % TN][e] = fmaf(part[(i) % 3][e], sp[(i) / TN], acc[2 * (q) + (i) / TN][(i) % TN][e]); \
    FF_TIE(acc[2 * (q) + (i) / TN][(i) % TN]);   /* here, not later: part's registers are free again */ \
  } while (0)
#define FF_MMA(q)                                                                                   \
  do {                                                                                              \
    _Pragma("unroll") for (int i = 0; i < 4; ++i) FF_TIE(fa[i]);                                    \
    FF_TIE(sv);                                                                                     \
    sp[0] = sv[0] * sw;                                                                             \
    sp[1] = sv[1] * sw;                                                                             \
    __builtin_amdgcn_sched_barrier(0);                                                              \
    __builtin_amdgcn_s_setprio(1);                                                                  \
    _Pragma("unroll") for (int i = 0; i < 2 * TN; ++i) {                                            \
      const int t = i / TN, u = i % TN;                                                             \
      part[i % 3] = mfma_q8(join(fb[2 * u], fb[2 * u + 1]), join(fa[2 * t], fa[2 * t + 1]), f32x4_t{0.f, 0.f, 0.f, 0.f}); \
      __builtin_amdgcn_sched_barrier(0);                                                            \
      if (i >= 2) FF_ADD1(q, i - 2);                                                                \
      __builtin_amdgcn_sched_barrier(0);                                                            \
    }                                                                                               \
    __builtin_amdgcn_s_setprio(0);                                                                  \
    __builtin_amdgcn_sched_barrier(0);                                                              \
    asm volatile("s_barrier" ::: "memory");                                                         \
  } while (0)
#define FF_ADD(q)                                                                                   \
  do {                                                                                              \
    FF_ADD1(q, 2 * TN - 2);                                                                         \
    FF_ADD1(q, 2 * TN - 1);                                                                         \
  } while (0)
  auto stage = [&](auto LEFTc) __attribute__((always_inline)) {
    constexpr int LEFT = decltype(LEFTc)::value;
    constexpr bool k1 = LEFT >= 1, k2 = LEFT >= 2;
    const int oa = BUFA - ca, ob = BUFB - cb;
    // phase 0
#pragma unroll
    for (int u = 0; u < TN; ++u) {
      fb[2 * u] = __builtin_bit_cast(u32x4_t, lds_rd128_off(rdb[0], u * PC));
      fb[2 * u + 1] = __builtin_bit_cast(u32x4_t, lds_rd128_off(rdb[1], u * PC));
    }
    FF_RDA(0);
    FF_RDS(0);
    FF_ADD(3);
    if (k1) FF_DMA(ra, voa[3], 3 * PC + oa, kb + RB);
    if (k2) FF_DMAS(st + 2);
    sw = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsw), st & 63));
    wait_vm<pp_vm(0, LEFT)>();
    FF_MEM_END();
#pragma unroll
    for (int i = 0; i < 2 * TN; ++i) FF_TIE(fb[i]);
    FF_MMA(0);
    // phase 1
    FF_RDA(1 * PC);
    FF_RDS(1);
    FF_ADD(0);
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
    FF_RDS(2);
    FF_ADD(1);
    if (k2) {
      FF_DMA(ra, voa[1], PC + ca, kb + 2 * RB);
      FF_DMA(rw, vob[2], OFFB + 2 * PC + cb, kb + 2 * RB);
    }
    wait_vm<pp_vm(2, LEFT)>();
    FF_MEM_END();
    FF_MMA(2);
    // phase 3
    FF_RDA(3 * PC);
    FF_RDS(3);
    FF_ADD(2);
    rda[0] += oa - ca; rda[1] += oa - ca;
    rdb[0] += ob - cb; rdb[1] += ob - cb;
    if (k2) {
      FF_DMA(ra, voa[2], 2 * PC + ca, kb + 2 * RB);
      FF_DMA(rw, vob[3], OFFB + 3 * PC + cb, kb + 2 * RB);
    }
    wait_vm<pp_vm(3, LEFT)>();
    FF_MEM_END();
    FF_MMA(3);
    kb += RB;
    ++st;
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
      if (pc == 8) FF_DMAS(s);
      else if (pc < 4) FF_DMA(ra, voa[pc & 3], s * BUFA + pc * PC, s * RB);
      else FF_DMA(rw, vob[pc & 3], OFFB + s * BUFB + (pc - 4) * PC, s * RB);
    }
  wait_vm<4 + TN>();   // stage 0 has landed, and stage 1 but for A3 is on its way
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
    if ((st & 63) == 0) vsw = wsc[min(st + lane, nk - 1)];
  } while (--left);
  voa[3] = cut ? 0x80000000u : voa[3];
  stage(Int<1>{});
  if ((st & 63) == 0) vsw = wsc[min(st + lane, nk - 1)];
  stage(Int<0>{});
  FF_ADD(3);
  if (wave < 4) asm volatile("s_barrier" ::: "memory");
#undef FF_ADD
#undef FF_ADD1
#undef FF_MEM_END
#undef FF_DMA
#undef FF_DMAS
#undef FF_RDA
#undef FF_RDS
#undef FF_MMA
  // every wave's LDS reads and DMA ended before the last barrier
  epilogue<DT_BF16, 8, TN>(a, m0 + mw * 128, n0 + nw * WN, acc, reinterpret_cast<float*>(lds) + wave * 32 * (WN + 4));
#endif
}

// ---------------------------------------------------------------- smaller grids, fp32 outputs
// BM x BN tile, 8 waves in two groups of four; a group takes every second block of K for the whole tile
// (2 x 2 waves), so that a fragment read feeds up to four MFMAs, and has its own ring of NS blocks.
// Per block a wave has a memory slot (its fragments and scales, and the scaled addition of the former
// block's sums) and a matrix slot (the DMA of the block NS ahead into the ring slot just read, then
// the MFMAs), each ended by a barrier; the second group runs one slot behind, one wave of each group
// per SIMD.  The two groups' sums meet in LDS: each finishes half of the rows.
// What bounds it: a slot's LDS reads, its waits and barrier (64 x 64: 0.21 us a block of K, with two
// workgroups on a CU 0.25; 128 x 128 0.36 alone), and with all CUs what the caches deliver (128 x 128
// 0.71 us a block).  Waiting for the scalar load of the weight's scale in each slot, and issuing the DMA
// ahead of the MFMAs instead of behind each, cost 10 to 15 %.  64 x 64 with rings of two blocks and two
// workgroups a CU: 16.3 us against 21.5 with rings of four (M = 1003, N = 1480, K = 2960).
//
template <int DT, int BM, int BN, int NS>
__global__ __launch_bounds__(512) void k_gemm_q8_two(GemmQ8Args a, int splits) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass needs the launch stub only
  constexpr int TM = BM / 32, TN = BN / 32, WN = BN / 2, RB = kQBlock;
  constexpr int STB = (BM + BN) * RB, SCB = BM * 4;   // bytes of a block, of its rows' scales
  constexpr int NA = BM / 32, NW = BN / 32, PER = NA + NW + 1;   // DMA instructions of a wave and block
  constexpr int OFFS = 2 * NS * STB, kMain = OFFS + 2 * NS * SCB;
  constexpr int HT = TM / 2, kXch = 8 * HT * TN * 1024, RE = HT > 1 ? 32 : 16, kEpi = kXch + 8 * RE * (WN + 4) * 4;
  static_assert(TM % 2 == 0 && BN <= kQBlock, "halves of the rows; one weight scale a tile and block");
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
  __amdgpu_buffer_rsrc_t ra = rsrc(a.a + (size_t)m0 * a.a_row), rw = rsrc(a.w + (size_t)n0 * a.w_row), rs = rsrc(a.a_s + m0);
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
  const uint32_t vos = (uint32_t)min((w * 64 + lane) % BM, a.M - 1 - m0) * 4u, sstep = (uint32_t)a.as_ld * 4u;
  constexpr int SW = BM / 64;   // waves whose scales differ; the others repeat them
  char* const ring = lds + grp * NS * STB;
  char* const sring = lds + OFFS + grp * NS * SCB;
  auto issue1 = [&](int i, int slot, int j) __attribute__((always_inline)) {   // DMA j of the group's block i
    const int kt = kb0 + 2 * i + grp, kb = kt * RB;
    const unsigned c = kt == nk - 1 ? cut : 0u;
    char* const dst = ring + slot * STB;
    if (j < NA)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, FF_AS3(dst + (w * NA + j) * 1024), 16, voa[j < NA ? j : 0] | (c >> j & 1u) << 31, kb, 0, 0);
    else if (j < NA + NW)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, FF_AS3(dst + BM * RB + (w * NW + j - NA) * 1024), 16,
                                               vow[j < NA || j >= NA + NW ? 0 : j - NA] | (c >> j & 1u) << 31, kb, 0, 0);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, FF_AS3(sring + slot * SCB + (w % SW) * 256), 4, vos, kt * sstep, 0, 0);
  };
  f32x4_t acc[TM][TN], part[TM][TN];
  const f32x4_t z4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = part[i][j] = z4;
  const int fr = lane & 15, fh = lane >> 4;
  const uint32_t lds0 = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) const void*)lds);
  uint32_t rda[2], rdw[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const uint32_t c = ((4 * s + fh) ^ (fr >> 1)) * 16, o = lds0 + grp * NS * STB;
    rda[s] = o + (wr * (BM / 2) + fr) * RB + c;
    rdw[s] = o + (BM + wc * WN + fr) * RB + c;
  }
  const uint32_t rds = lds0 + OFFS + grp * NS * SCB + (wr * (BM / 2) + fr) * 4;
  // the weight's scales of the group's next 64 blocks, one a lane (a scalar load per block took up to a
  // cache miss each 8 turns)
  const float* wsc = a.w_s + (size_t)(n0 / kQBlock) * a.ws_ld;
  float vsw = wsc[min(kb0 + grp + 2 * lane, nk - 1)];
  u32x4_t fa[2 * TM], fw[2 * TN];
  f32x2_t sv[HT];
#pragma unroll
  for (int t = 0; t < HT; ++t) sv[t] = f32x2_t{0.f, 0.f};
  float sw = 0.f;
  // the scales of the former block's sums, formed before sv's registers are read into again
  float sp[TM];
  auto scale = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      sp[i] = sv[i / 2][i % 2] * sw;
      FF_TIE(sp[i]);
    }
  };
  auto add = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int j = 0; j < TN; ++j) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(part[i][j][e], sp[i], acc[i][j][e]);
        FF_TIE(acc[i][j]);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (i < mine) {
#pragma unroll
      for (int j = 0; j < PER; ++j) issue1(i, i, j);
    }
  wait_vm<0>();
  asm volatile("s_barrier" ::: "memory");
  if (grp) asm volatile("s_barrier" ::: "memory");   // the second group runs one slot behind
  int slot = 0;
  auto turn = [&](int i, auto Mc) __attribute__((always_inline)) {
    constexpr bool more = decltype(Mc)::value != 0;   // a block NS ahead is left
    // memory slot
    scale();
    const uint32_t so = slot * STB;
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int s = 0; s < 2; ++s) fw[2 * t + s] = __builtin_bit_cast(u32x4_t, lds_rd128_off(rdw[s] + so, t * 16 * RB));
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
      for (int s = 0; s < 2; ++s) fa[2 * t + s] = __builtin_bit_cast(u32x4_t, lds_rd128_off(rda[s] + so, t * 16 * RB));
#pragma unroll
    for (int t = 0; t < HT; ++t)
      asm volatile("ds_read2_b32 %0, %1 offset0:%2 offset1:%3" : "=v"(sv[t]) : "v"(rds + slot * SCB), "i"(32 * t), "i"(32 * t + 16) : "memory");
    add();
    sw = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vsw), i & 63));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int t = 0; t < 2 * TN; ++t) FF_TIE(fw[t]);
#pragma unroll
    for (int t = 0; t < 2 * TM; ++t) FF_TIE(fa[t]);
#pragma unroll
    for (int t = 0; t < HT; ++t) FF_TIE(sv[t]);
    asm volatile("s_barrier" ::: "memory");
    // matrix slot: a DMA behind each MFMA
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
    if constexpr (DT == DT_BF16) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int t = 0; t < TM; ++t) {
          part[t][j] = mfma_q8(join(fw[2 * j], fw[2 * j + 1]), join(fa[2 * t], fa[2 * t + 1]), z4);
          if (more && j * TM + t < PER) {
            __builtin_amdgcn_sched_barrier(0);
            issue1(i + NS, slot, j * TM + t);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        bf16x8_t xa[TM], xw[TN];
#pragma unroll
        for (int t = 0; t < TM; ++t) xa[t] = widen(fa[2 * t + s / 2][s % 2 * 2], fa[2 * t + s / 2][s % 2 * 2 + 1]);
#pragma unroll
        for (int t = 0; t < TN; ++t) xw[t] = widen(fw[2 * t + s / 2][s % 2 * 2], fw[2 * t + s / 2][s % 2 * 2 + 1]);
#pragma unroll
        for (int t = 0; t < TM; ++t)
#pragma unroll
          for (int j = 0; j < TN; ++j) part[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xw[j], xa[t], s == 0 ? z4 : part[t][j], 0, 0, 0);
        if (more) {
#pragma unroll
          for (int j = s; j < (PER < TM * TN ? PER : TM * TN); j += 4) issue1(i + NS, slot, j);
        }
      }
    }
    if (more) {
#pragma unroll
      for (int j = TM * TN; j < PER; ++j) issue1(i + NS, slot, j);
    }
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    // the next block has landed; the ones after it may be on their way
    wait_vm<more ? (NS - 1) * PER : 0>();
    slot = slot == NS - 1 ? 0 : slot + 1;
    asm volatile("s_barrier" ::: "memory");
  };
  int i = 0;
  auto scales = [&]() __attribute__((always_inline)) {
    if (i && (i & 63) == 0) vsw = wsc[min(kb0 + grp + 2 * (i + lane), nk - 1)];
  };
  for (; i < mine - NS; ++i) { scales(); turn(i, Int<1>{}); }
  for (; i < mine; ++i) { scales(); turn(i, Int<0>{}); }
  if (mine < turns) {   // the second group, one block short
    asm volatile("s_barrier" ::: "memory");
    asm volatile("s_barrier" ::: "memory");
  }
  scale();
  add();
  if (!grp) asm volatile("s_barrier" ::: "memory");
  // every wave's LDS reads and DMA ended before the last barrier; each group finishes half of the rows
  f32x4_t* const xch = reinterpret_cast<f32x4_t*>(lds) + lane;
  f32x4_t fin[HT][TN];
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
    for (int j = 0; j < TN; ++j) {
      const f32x4_t p = xch[(((wave ^ 4) * HT + t) * TN + j) * 64];
#pragma unroll
      for (int e = 0; e < 4; ++e) fin[t][j][e] += p[e];
    }
  float* const stage = reinterpret_cast<float*>(lds + kXch) + wave * RE * (WN + 4);
  const int r0 = m0 + wr * (BM / 2) + grp * HT * 16, c0 = n0 + wc * WN;
  if (splits > 1) {   // bare sums for k_gemm_q8_join
    GemmQ8Args p = a;
    p.bias = p.resid = nullptr;
    p.gelu = 0;
    p.out = a.part + (size_t)split * a.M * a.N;
    p.out_row = a.N;
    epilogue<DT_F32, HT, TN>(p, r0, c0, fin, stage);
  } else {
    epilogue<DT, HT, TN>(a, r0, c0, fin, stage);
  }
#endif
}

// Joins the splits of K: 8 columns of a row a thread, the splits' sums in order
template <int DT>
__global__ __launch_bounds__(256) void k_gemm_q8_join(GemmQ8Args a, int splits) {
  const int per = a.N / 8;
  const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (size_t)a.M * per) return;
  const int r = (int)(id / per), c = (int)(id % per) * 8;
  float v[8], x[8];
  load8<DT_F32>(a.part, id * 8, v);
  for (int i = 1; i < splits; ++i) {
    load8<DT_F32>(a.part, (size_t)i * a.M * a.N + id * 8, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += x[e];
  }
  if (a.bias) {
    load8<DT>(a.bias, c, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += x[e];
  }
  if (a.gelu) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = gelu_tanh_f(v[e]);
  }
  if (a.resid) {
    load8<DT>(a.resid, (size_t)r * a.resid_row + c, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += x[e];
  }
  store8<DT>(a.out, (size_t)r * a.out_row + c, v);
}

// ---------------------------------------------------------------- choice
long tiles(long M, long N, long t) { return ((M + t - 1) / t) * ((N + t - 1) / t); }

}  // namespace

// The kernel of a shape by estimated time (us), fitted to 25 shapes of 1 to 4608 rows, N and K of 1152 to
// 8192.  A tile of 64 x 64 takes 0.21 us per block of K while each CU has one, 0.5 with two on every CU;
// 128 x 128 0.42 alone, 0.71 with all CUs (what the caches deliver); 256 x 256 1.95; fp32 outputs 1.4 to
// 2 times that.  Splits of K add the join: a launch, and writing and reading the partial sums.
//   N 8192 K 2048, M = 16: k_gemm_q8_dir 7.1 us against 8.0 with 64 x 64 tiles; M = 64: 17.8 against 8.1
//   M 128 N 2048 K 8192: 64 x 64 tiles 17.7 us, with 2 / 4 / 8 splits 14.2 / 12.4 / 14.7
//   M 512 N 8192 K 2048: 128 x 128 14.9 us, 64 x 64 20.9, 256 x 256 31.9
//   M 14566 N 8192 K 2048: 256 x 256 248 us, 128 x 128 315, 64 x 64 435 (fp32: 128 x 128 518, 64 x 64 649)
Q8Plan gemm_q8_plan(int dt, int M, int N, int K) {
  const int nk = (K + kQBlock - 1) / kQBlock;
  // us per block of K: few tiles, what 256 tiles add, and a round of all CUs (512 tiles of 64 x 64)
  const double c64[2][3] = {{0.21, 0.08, 0.50}, {0.30, 0.12, 0.71}}, c128[2][3] = {{0.42, 0.30, 0.71}, {0.73, 0.40, 1.13}};
  const double *c6 = c64[dt == DT_F32], *c12 = c128[dt == DT_F32];
  Q8Plan best{Q8_TILE128, 1};
  double least = 1e30;
  auto take = [&](int k, int splits, double us) {
    if (us < least) { least = us; best = Q8Plan{k, splits}; }
  };
  if (M <= 256) {
    const double t = (double)tiles(M, N, 16), chain = 0.4 * ((nk + 15) / 16);
    take(Q8_DIR, 1, 2.5 + (t * nk * 0.45e-3 > chain ? t * nk * 0.45e-3 : chain));
  }
  for (int s = 1; s <= 8; s *= 2) {
    if (s > 1 && nk / s < 8) break;
    const double t = (double)tiles(M, N, 64) * s, nb = (double)nk / s;
    const double main = t <= 256 ? (c6[0] + c6[1] * t / 256) * nb : ceil(t / 512) * c6[2] * nb;
    take(Q8_TILE64, s, 3.5 + main + (s > 1 ? 1.8 + s * (0.35 + 2.3e-6 * M * N) : 0.0));
  }
  const double t128 = (double)tiles(M, N, 128), t256 = (double)tiles(M, N, 256);
  take(Q8_TILE128, 1, 3.5 + (t128 <= 256 ? c12[0] + c12[1] * t128 / 256 : ceil(t128 / 256) * c12[2]) * nk);
  if (dt == DT_BF16 && nk >= 3) take(Q8_TILE256, 1, 4.0 + ceil(t256 / 256) * 1.95 * nk);
  return best;
}

namespace {

template <int DT>
hipError_t launch_q8(const GemmQ8Args& a, hipStream_t s) {
  const Q8Plan p = gemm_q8_plan(DT, a.M, a.N, a.K);
  switch (p.kernel) {
    case Q8_DIR: {
      // 16 waves where 8 would take their blocks in two rounds on a part of the CUs (one row, K = 8192: N = 2048
      // 7.8 us for 8.4; N = 8192, where all CUs are at work, 15.7 for 15.6)
      const long t = tiles(a.M, a.N, 16);
      if (a.K > 32 * kQBlock && t <= 256) FF_LAUNCH((k_gemm_q8_dir<DT, 16>), (unsigned)t, 1024, 0, s, a);
      else FF_LAUNCH((k_gemm_q8_dir<DT, 8>), (unsigned)t, 512, 0, s, a);
      break;
    }
    case Q8_TILE64: FF_LAUNCH((k_gemm_q8_two<DT, 64, 64, 2>), (unsigned)(tiles(a.M, a.N, 64) * p.splits), 512, 0, s, a, p.splits); break;
    case Q8_TILE128: FF_LAUNCH((k_gemm_q8_two<DT, 128, 128, 2>), (unsigned)tiles(a.M, a.N, 128), 512, 0, s, a, 1); break;
    case Q8_TILE256:
      if constexpr (DT == DT_BF16) FF_LAUNCH(k_gemm_q8_pp, (unsigned)tiles(a.M, a.N, 256), 512, 0, s, a);
      break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const size_t wg = ((size_t)a.M * (a.N / 8) + 255) / 256;
  FF_LAUNCH(k_gemm_q8_join<DT>, (unsigned)wg, 256, 0, s, a, p.splits);
  return hipGetLastError();
}

}  // namespace

size_t gemm_q8_workspace(int out_dtype, int M, int N, int K) {
  if (M <= 0) return 0;
  const int n = gemm_q8_plan(out_dtype, M, N, K).splits;
  return n > 1 ? (size_t)n * M * N * 4 : 0;
}

hipError_t gemm_q8(int out_dtype, const GemmQ8Args& a, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  if (tiles(a.M, a.N, 16) > 0x7fffffffL) return hipErrorInvalidValue;
  return out_dtype == DT_BF16 ? launch_q8<DT_BF16>(a, s) : launch_q8<DT_F32>(a, s);
}

}  // namespace ff
