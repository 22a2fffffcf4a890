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

}  // namespace

size_t gemm_q8_workspace(int, int, int) { return 0; }

hipError_t gemm_q8(int out_dtype, const GemmQ8Args& a, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  const long wg = (long)((a.M + 15) / 16) * ((a.N + 15) / 16);
  if (wg > 0x7fffffffL) return hipErrorInvalidValue;
  if (out_dtype == DT_BF16) FF_LAUNCH(k_gemm_q8_dir<DT_BF16>, (unsigned)wg, 512, 0, s, a);
  else FF_LAUNCH(k_gemm_q8_dir<DT_F32>, (unsigned)wg, 512, 0, s, a);
  return hipGetLastError();
}

}  // namespace ff
