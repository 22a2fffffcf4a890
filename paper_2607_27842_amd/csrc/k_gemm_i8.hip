// Products of 8-bit integers with a scale for each row of either operand:
//   out = act(a_s[m] w_s[n] sum_k a[m, k] w[n, k] + bias) gate[m / gate_rows] + resid
// Sums of products are whole numbers in 32 bits (K <= 131056), the same in any order; a result is rounded to
// fp32 where the sum leaves them, once for each scale, and to the output's type at the end.  One
// v_mfma_i32_16x16x64_i8 covers 16 rows, 16 columns and 64 k.  The A operand holds weight rows (output
// columns n), the B operand activation rows m: lane l then holds output row l % 16 and columns
// 4 (l / 16) + 0..3.  Lane l of an operand takes row l % 16 and 16 bytes of the 64 k.
#include "gemm_8bit.h"
#include "i8_common.h"

namespace ff {

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4_t mfma_i8(u32x4_t a, u32x4_t b, i32x4_t c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, a), __builtin_bit_cast(i32x4_t, b), c, 0, 0, 0);
}

// Few rows: 16 x 16 tile, operands straight from memory, the NW waves of a workgroup on interleaved blocks of 128 k;
// their sums meet in LDS.
template <int DT, int NW>
__global__ __launch_bounds__(NW * 64) void k_gemm_i8_dir(GemmI8Args a) {
  constexpr int U = 4;
  __shared__ i32x4_t red[NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int tn = (a.N + 15) / 16, m0 = (blockIdx.x / tn) * 16, n0 = (blockIdx.x % tn) * 16;
  const int m = m0 + l16 < a.M ? m0 + l16 : m0, n = n0 + l16 < a.N ? n0 + l16 : n0;   // past the matrix: never stored
  const uint8_t* pa = static_cast<const uint8_t*>(a.a) + (size_t)m * a.a_row;
  const uint8_t* pw = a.w + (size_t)n * a.w_row;
  i32x4_t acc = {0, 0, 0, 0};
  const int nk = (a.K + kQBlock - 1) / kQBlock;
  for (int b0 = wave; b0 < nk; b0 += NW * U) {
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
  }
  red[wave][lane] = acc;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int i = 1; i < NW; ++i) acc += red[i][lane];
  const int r = m0 + l16, c = n0 + 4 * g;
  if (r >= a.M || c >= a.N) return;   // N % 8 == 0: 4 columns are in range as a whole
  const float sa = a.a_s[r];
  const f32x4_t sw = load4<DT_F32>(a.w_s, c);
  f32x4_t v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (float)acc[e] * sa * sw[e];
  if (a.bias) v += load4<DT>(a.bias, c);
  if (a.gelu) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = gelu_tanh_f(v[e]);
  }
  if (a.gate) v *= load4<DT_F32>(a.gate, (size_t)(r / a.gate_rows) * a.gate_ld + c);
  if (a.resid) v += load4<DT>(a.resid, (size_t)r * a.resid_row + c);
  const size_t o = (size_t)r * a.out_row + c;
  if (DT == DT_BF16) *reinterpret_cast<u32x2_t*>(reinterpret_cast<uint16_t*>(a.out) + o) = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(a.out) + o) = v;
}

long tiles(long M, long N, long t) { return ((M + t - 1) / t) * ((N + t - 1) / t); }

// rows that the call puts in 8 bits itself, and their scales behind them
size_t rows_bytes(int a_dtype, int M, int K) { return a_dtype == DT_I8 ? 0 : ((size_t)M * K + 255) / 256 * 256 + ((size_t)M * 4 + 255) / 256 * 256; }

}  // namespace

I8Plan gemm_i8_plan(int, int, int, int, int) { return I8Plan{I8_DIR, 1}; }

size_t gemm_i8_workspace(int a_dtype, int out_dtype, int M, int N, int K) {
  if (M <= 0) return 0;
  const int n = gemm_i8_plan(a_dtype, out_dtype, M, N, K).splits;
  return rows_bytes(a_dtype, M, K) + (n > 1 ? (size_t)n * M * N * 4 : 0);
}

hipError_t gemm_i8(int a_dtype, int out_dtype, const GemmI8Args& a0, hipStream_t s) {
  if (a0.M <= 0) return hipSuccess;
  const long t = tiles(a0.M, a0.N, 16);
  if (t > 0x7fffffffL) return hipErrorInvalidValue;
  GemmI8Args a = a0;
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
  if (out_dtype == DT_BF16) FF_LAUNCH((k_gemm_i8_dir<DT_BF16, 8>), (unsigned)t, 512, 0, s, a);
  else FF_LAUNCH((k_gemm_i8_dir<DT_F32, 8>), (unsigned)t, 512, 0, s, a);
  return hipGetLastError();
}

}  // namespace ff
