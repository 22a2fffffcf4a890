// Products of 8-bit operands with a scale for each block of 128 along K:
//   out = act(sum_b a_s[b, m] w_s[n / 128, b] (sum_{k in b} a[m, k] w[n, k]) + bias) + resid
// One v_mfma_f32_16x16x128_f8f6f4 covers a block of 16 rows, 16 columns and 128 k.  Its sum starts
// at zero and is added to the fp32 accumulators times a_s w_s.  The A operand holds weight rows
// (output columns n), the B operand activation rows m: lane l then holds output row l % 16 and
// columns 4 (l / 16) + 0..3.  Lane l of an operand takes row l % 16 and two 16-byte chunks of the
// block, chunks l / 16 and 4 + l / 16; which k stands where within the block does not matter as
// long as both operands agree.
#include "dev_common.h"

namespace ff {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4_t mfma_q8(i32x8_t a, i32x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);   // e4m3, no block scales
}
__device__ __forceinline__ i32x8_t join(u32x4_t lo, u32x4_t hi) {
  return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// 4 consecutive columns c.. of output row r (N % 8 == 0: in range as a whole)
template <int DT>
__device__ __forceinline__ void finish4(const GemmQ8Args& a, int r, int c, f32x4_t v) {
  if (a.bias) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += St<DT>::ld1(a.bias, c + e);
  }
  if (a.gelu) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = gelu_tanh_f(v[e]);
  }
  if (a.resid) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += St<DT>::ld1(a.resid, (size_t)r * a.resid_row + c + e);
  }
  const size_t o = (size_t)r * a.out_row + c;
  if (DT == DT_BF16) *reinterpret_cast<u32x2_t*>(reinterpret_cast<uint16_t*>(a.out) + o) = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(a.out) + o) = v;
}

// 16 x 16 tile, operands straight from memory, the 8 waves of a workgroup on interleaved blocks of K;
// their sums meet in LDS in wave order.
template <int DT>
__global__ __launch_bounds__(512) void k_gemm_q8_dir(GemmQ8Args a) {
  __shared__ f32x4_t red[8][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int tn = (a.N + 15) / 16, m0 = (blockIdx.x / tn) * 16, n0 = (blockIdx.x % tn) * 16;
  const int m = m0 + l16 < a.M ? m0 + l16 : m0, n = n0 + l16 < a.N ? n0 + l16 : n0;   // past the matrix: never stored
  const uint8_t* pa = a.a + (size_t)m * a.a_row;
  const uint8_t* pw = a.w + (size_t)n * a.w_row;
  const float* sw = a.w_s + (size_t)(n0 / kQBlock) * a.ws_ld;
  const f32x4_t z = {0.f, 0.f, 0.f, 0.f};
  const u32x4_t zu = {0u, 0u, 0u, 0u};
  f32x4_t acc = z;
  const int nk = (a.K + kQBlock - 1) / kQBlock;
  for (int b = wave; b < nk; b += 8) {
    const int k0 = b * kQBlock + g * 16, k1 = k0 + 64;
    const u32x4_t x0 = k0 < a.K ? *reinterpret_cast<const u32x4_t*>(pa + k0) : zu, x1 = k1 < a.K ? *reinterpret_cast<const u32x4_t*>(pa + k1) : zu;
    const u32x4_t w0 = k0 < a.K ? *reinterpret_cast<const u32x4_t*>(pw + k0) : zu, w1 = k1 < a.K ? *reinterpret_cast<const u32x4_t*>(pw + k1) : zu;
    const float s = a.a_s[(size_t)b * a.as_ld + m] * sw[b];
    const f32x4_t p = mfma_q8(join(w0, w1), join(x0, x1), z);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = fmaf(p[e], s, acc[e]);
  }
  red[wave][lane] = acc;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    const f32x4_t p = red[i][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += p[e];
  }
  if (m0 + l16 < a.M && n0 + 4 * g < a.N) finish4<DT>(a, m0 + l16, n0 + 4 * g, acc);
}

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
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = 0.f;
  if (a.bias && c < a.N) load8<DT>(a.bias, c, bias);
#pragma unroll
  for (int i = 0; i < TM * 16 / RB; ++i) {
#pragma unroll
    for (int t = 0; t < RB / 16; ++t)
#pragma unroll
      for (int u = 0; u < TN; ++u)
        *reinterpret_cast<f32x4_t*>(lds + (16 * t + fr) * LDW + 16 * u + 4 * fh) = acc[i * (RB / 16) + t][u];
    float res[NPASS][8];
    if (a.resid) {   // requested before the first use
#pragma unroll
      for (int p = 0; p < NPASS; ++p) {
        const int r = r0 + i * RB + p * RPP + pr;
        if (r < a.M && c < a.N) load8<DT>(a.resid, (size_t)r * a.resid_row + c, res[p]);
      }
    }
#pragma unroll
    for (int p = 0; p < NPASS; ++p) {
      const int r = r0 + i * RB + p * RPP + pr;
      const f32x4_t x0 = *reinterpret_cast<const f32x4_t*>(lds + (p * RPP + pr) * LDW + pc);
      const f32x4_t x1 = *reinterpret_cast<const f32x4_t*>(lds + (p * RPP + pr) * LDW + pc + 4);
      float v[8] = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
      if (r >= a.M || c >= a.N) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += bias[e];
      if (a.gelu) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = gelu_tanh_f(v[e]);
      }
      if (a.resid) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += res[p][e];
      }
      store8<DT>(a.out, (size_t)r * a.out_row + c, v);
    }
  }
}

// Workgroup -> tile: workgroups go round-robin over the 8 XCDs, so every XCD gets a contiguous range
// of tiles, in groups of 8 tile rows, whose operand rows its L2 then shares.
__device__ __forceinline__ void tile_at(int tiles_m, int tiles_n, int& tm, int& tn) {
  const int n = gridDim.x, full = n / 8 * 8;
  const int id = (int)blockIdx.x < full ? (blockIdx.x % 8) * (full / 8) + blockIdx.x / 8 : blockIdx.x;
  const int per = 8 * tiles_n, first = id / per * 8, size = min(tiles_m - first, 8), in = id % per;
  tm = __builtin_amdgcn_readfirstlane(first + in % size);
  tn = __builtin_amdgcn_readfirstlane(in / size);
}

// ---------------------------------------------------------------- large grids: two wave groups in turn
// 256 x 64 TN tile, a stage of one 128-wide block of K, 8 waves in two groups of four, one wave of
// each group per SIMD; a stage has four phases, one per 32 rows of a wave's 128 x 16 TN block.  A
// phase is a memory part (fragment reads, DMA, and the fused multiply-adds that scale the former
// phase's sums into the accumulators) and 2 TN MFMAs, with a barrier after each; the second group
// runs half a phase behind, so that on every SIMD one wave's MFMAs (64 TN cycles) cover the other's
// reads, DMA and 8 TN + 2 vector instructions.
//
// Operands: 64-row pieces of 8 KB, each filled by one DMA instruction per wave, in two buffers per
// operand, and the 256 rows' scales of a stage (1 KB, one 4-byte DMA a lane; waves w and w + 4 write
// the same values) in a ring of four.  Phase p of stage k issues, in this order:
//   0: A3 of stage k+1, the scales of k+2   1: A0, B0, B1 of k+2   2: A1, B2 of k+2   3: A2, B3 of k+2
// and reads: phase 0 all B and A0 of stage k, phases 1-3 A1-A3, each phase its rows' scales.  So a
// piece's slot is refilled no earlier than one phase after its last read.
// The weight's scale of a stage is a scalar per wave (its columns lie in one block of 128).
// K % 128 != 0: the last stage's chunks past K are out of the resource's range and load zeros.
constexpr int kPPIssue[4][3] = {{3, 8, -1}, {0, 4, 5}, {1, 6, -1}, {2, 7, -1}};   // A0-A3, B0-B3, scales
// How many of a wave's DMAs may be outstanding at the end of phase p of a stage with `left` stages
// after it (2: two or more), so that what phase p + 1 reads has landed.
constexpr int pp_vm(int TN, int p, int left) {
  int n = 0, need = -1;
  for (int j = -2; j <= 0; ++j)
    for (int q = 0; q < (j == 0 ? p + 1 : 4); ++q)
      for (int i = 0; i < 3; ++i) {
        const int pc = kPPIssue[q][i], st = pc == 3 ? j + 1 : j + 2;
        if (pc < 0 || (pc < 8 && pc >= 4 + TN) || st > left) continue;
        ++n;
        const bool next = (p == 0 && pc == 1 && st == 0) || (p == 1 && pc == 2 && st == 0) ||
                          (p == 2 && pc == 3 && st == 0) || (p == 3 && (pc == 0 || pc >= 4) && st == 1);
        if (next) need = n;
      }
  return need < 0 ? 63 : n - need;
}

template <int TN>
__global__ __launch_bounds__(512) void k_gemm_q8_pp(GemmQ8Args a) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass needs the launch stub only
  constexpr int BM = 256, BN = 64 * TN, WN = 16 * TN, RB = kQBlock;   // RB: bytes of an LDS row
  constexpr int PC = 64 * RB, BUFA = 4 * PC, BUFB = TN * PC, OFFB = 2 * BUFA, OFFS = OFFB + 2 * BUFB;
  constexpr int kMain = OFFS + 4 * 1024, kEpi = 8 * 32 * (WN + 4) * 4;
  __shared__ __attribute__((aligned(1024))) char lds[kMain > kEpi ? kMain : kEpi];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int tm, tn;
  tile_at((a.M + BM - 1) / BM, (a.N + BN - 1) / BN, tm, tn);
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
  f32x4_t acc[8][TN], part[2][TN];
#pragma unroll
  for (int j = 0; j < TN; ++j) {
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    part[0][j] = part[1][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
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
  // scalar loads: a vector load would wait for the DMA before it
  typedef const __attribute__((address_space(4))) float* scalar_ptr;
  const scalar_ptr wsc = (scalar_ptr)(a.w_s + (size_t)min((n0 + nw * WN) / kQBlock, (a.N - 1) / kQBlock) * a.ws_ld);
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
    asm volatile("ds_read2_b32 %0, %1 offset0:%2 offset1:%3" : "=v"(sv[(q) & 1]) : "v"(ad), "n"((q) * 32), "n"((q) * 32 + 16) : "memory"); \
  } while (0)
  f32x2_t sv[2];
  sv[0] = sv[1] = f32x2_t{0.f, 0.f};
#define FF_MEM_END() asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory")
  // the products of phase q's rows, from zero
#define FF_MMA(q)                                                                                   \
  do {                                                                                              \
    _Pragma("unroll") for (int i = 0; i < 4; ++i) FF_TIE(fa[i]);                                    \
    FF_TIE(sv[(q) & 1]);                                                                            \
    __builtin_amdgcn_sched_barrier(0);                                                              \
    __builtin_amdgcn_s_setprio(1);                                                                  \
    _Pragma("unroll") for (int t = 0; t < 2; ++t)                                                   \
      _Pragma("unroll") for (int u = 0; u < TN; ++u)                                                \
        part[t][u] = mfma_q8(join(fb[2 * u], fb[2 * u + 1]), join(fa[2 * t], fa[2 * t + 1]), f32x4_t{0.f, 0.f, 0.f, 0.f}); \
    __builtin_amdgcn_s_setprio(0);                                                                  \
    __builtin_amdgcn_sched_barrier(0);                                                              \
    asm volatile("s_barrier" ::: "memory");                                                         \
  } while (0)
  // ... and their way into the accumulators, in the next phase's memory part
#define FF_ADD(q)                                                                                   \
  do {                                                                                              \
    _Pragma("unroll") for (int t = 0; t < 2; ++t) {                                                 \
      const float s = sv[(q) & 1][t] * sw;                                                          \
      _Pragma("unroll") for (int u = 0; u < TN; ++u)                                                \
        _Pragma("unroll") for (int e = 0; e < 4; ++e) acc[2 * (q) + t][u][e] = fmaf(part[t][u][e], s, acc[2 * (q) + t][u][e]); \
    }                                                                                               \
    _Pragma("unroll") for (int t = 0; t < 2; ++t)   /* here, not later: part's registers are free again */ \
      _Pragma("unroll") for (int u = 0; u < TN; ++u) FF_TIE(acc[2 * (q) + t][u]);                   \
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
    if (k1) FF_DMA(ra, voa[3], 3 * PC + oa, kb + RB);
    if (k2) FF_DMAS(st + 2);
    FF_ADD(3);
    sw = wsc[st];
    wait_vm<pp_vm(TN, 0, LEFT)>();
    FF_MEM_END();
#pragma unroll
    for (int i = 0; i < 2 * TN; ++i) FF_TIE(fb[i]);
    FF_MMA(0);
    // phase 1
    FF_RDA(1 * PC);
    FF_RDS(1);
    if (k2) {
      FF_DMA(ra, voa[0], ca, kb + 2 * RB);
      FF_DMA(rw, vob[0], OFFB + cb, kb + 2 * RB);
      FF_DMA(rw, vob[1], OFFB + PC + cb, kb + 2 * RB);
    }
    FF_ADD(0);
    wait_vm<pp_vm(TN, 1, LEFT)>();
    FF_MEM_END();
    FF_MMA(1);
    // phase 2
    FF_RDA(2 * PC);
    FF_RDS(2);
    if (k2) {
      FF_DMA(ra, voa[1], PC + ca, kb + 2 * RB);
      if (TN > 2) FF_DMA(rw, vob[TN > 2 ? 2 : 0], OFFB + 2 * PC + cb, kb + 2 * RB);
    }
    FF_ADD(1);
    wait_vm<pp_vm(TN, 2, LEFT)>();
    FF_MEM_END();
    FF_MMA(2);
    // phase 3
    FF_RDA(3 * PC);
    FF_RDS(3);
    rda[0] += oa - ca; rda[1] += oa - ca;
    rdb[0] += ob - cb; rdb[1] += ob - cb;
    if (k2) {
      FF_DMA(ra, voa[2], 2 * PC + ca, kb + 2 * RB);
      if (TN > 3) FF_DMA(rw, vob[TN > 3 ? 3 : 0], OFFB + 3 * PC + cb, kb + 2 * RB);
    }
    FF_ADD(2);
    wait_vm<pp_vm(TN, 3, LEFT)>();
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
      if (pc < 0 || (pc < 8 && pc >= 4 + TN) || s < 0) continue;
      if (pc == 8) FF_DMAS(s);
      else if (pc < 4) FF_DMA(ra, voa[pc & 3], s * BUFA + pc * PC, s * RB);
      else FF_DMA(rw, vob[pc - 4 < TN ? pc - 4 : 0], OFFB + s * BUFB + (pc - 4) * PC, s * RB);
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
  } while (--left);
  voa[3] = cut ? 0x80000000u : voa[3];
  stage(Int<1>{});
  stage(Int<0>{});
  FF_ADD(3);
  if (wave < 4) asm volatile("s_barrier" ::: "memory");
#undef FF_ADD
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

}  // namespace

size_t gemm_q8_workspace(int, int, int) { return 0; }

hipError_t gemm_q8(int out_dtype, const GemmQ8Args& a, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  if (out_dtype == DT_BF16 && a.K > 256 && a.M >= 512) {
    const long wg = (long)((a.M + 255) / 256) * ((a.N + 255) / 256);
    FF_LAUNCH(k_gemm_q8_pp<4>, (unsigned)wg, 512, 0, s, a);
    return hipGetLastError();
  }
  const long wg = (long)((a.M + 15) / 16) * ((a.N + 15) / 16);
  if (wg > 0x7fffffffL) return hipErrorInvalidValue;
  if (out_dtype == DT_BF16) FF_LAUNCH(k_gemm_q8_dir<DT_BF16>, (unsigned)wg, 512, 0, s, a);
  else FF_LAUNCH(k_gemm_q8_dir<DT_F32>, (unsigned)wg, 512, 0, s, a);
  return hipGetLastError();
}

}  // namespace ff
