// Attention of each query over its spans of keys, with shared key / value heads, capped and biased
// scores (include/featfix.h, ff_attention).
//
// The G query heads of a key head and the queries are one axis of rows (row r: query r / G, head
// r % G), so that heads sharing keys share their loads.  As in the blocks' attention, scores are
// formed transposed, S^T = K Q^T: every lane holds scores of ONE row, and the probabilities are
// already in the register layout of the B operand of O^T = V^T P^T.
#include "dev_common.h"

namespace ff {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFltMax = 3.402823466e38f;
constexpr int kKeys = 32;        // keys per wavefront and step of the direct kernels
constexpr int kMaxSplit = 64;

// What a lane keeps of its row.  Rows past the last repeat it (never stored).
struct Row {
  int lo0, n0, lo1, n1;   // the spans' first keys and lengths
  int pos;                // where the query stands among the keys
  const float* bias;      // its head's slope, or the middle of its table
  __device__ __forceinline__ bool sees(int k) const { return (unsigned)(k - lo0) < (unsigned)n0 || (unsigned)(k - lo1) < (unsigned)n1; }
};
__device__ __forceinline__ Row row_of(const AttnSpanArgs& a, int b, int hk, int r, int i) {
  Row w{0, a.n_k, 0, 0, i, nullptr};
  if (a.n_spans) {
    const int32_t* s = a.spans + (size_t)b * a.span_batch + (size_t)i * a.n_spans * 2;
    w.lo0 = min(max(s[0], 0), a.n_k);
    w.n0 = max(min(max(s[1], 0), a.n_k) - w.lo0, 0);
    if (a.n_spans > 1) {
      w.lo1 = min(max(s[2], 0), a.n_k);
      w.n1 = max(min(max(s[3], 0), a.n_k) - w.lo1, 0);
    }
  }
  if (a.bias_kind != BIAS_NONE) {
    if (a.pos) w.pos += min(max(a.pos[b], -(1 << 30)), 1 << 30);   // j - p_i stays an int32
    const int h = hk * a.G + r % a.G;
    w.bias = a.bias + (a.bias_kind == BIAS_TABLE ? (size_t)h * (2 * a.reach + 1) + a.reach : (size_t)h);
  }
  return w;
}

// Ranges of keys of a wavefront's rows, for whole blocks of keys: hull (some row may see them) and
// core (every row sees them), per span.
struct Ranges {
  int h0, e0, h1, e1;       // hulls
  int c0, d0, c1, d1;       // cores
  __device__ __forceinline__ bool some(int k, int n) const { return (k < e0 && k + n > h0) || (k < e1 && k + n > h1); }
  __device__ __forceinline__ bool all(int k, int n) const { return (k >= c0 && k + n <= d0) || (k >= c1 && k + n <= d1); }
};
template <int CTL>
__device__ __forceinline__ int dpp_movi(int x) { return __builtin_amdgcn_mov_dpp(x, CTL, 0xf, 0xf, false); }
__device__ __forceinline__ int min16(int v) {
  v = min(v, dpp_movi<0xB1>(v));
  v = min(v, dpp_movi<0x4E>(v));
  v = min(v, dpp_movi<0x141>(v));
  return __builtin_amdgcn_readfirstlane(min(v, dpp_movi<0x140>(v)));
}
template <int QT>
__device__ __forceinline__ Ranges ranges_of(const Row (&w)[QT]) {
  int h0 = 0x7fffffff, e0 = 0, h1 = 0x7fffffff, e1 = 0, c0 = 0, d0 = 0x7fffffff, c1 = 0, d1 = 0x7fffffff;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    if (w[t].n0) { h0 = min(h0, w[t].lo0); e0 = max(e0, w[t].lo0 + w[t].n0); }
    if (w[t].n1) { h1 = min(h1, w[t].lo1); e1 = max(e1, w[t].lo1 + w[t].n1); }
    c0 = max(c0, w[t].lo0); d0 = min(d0, w[t].lo0 + w[t].n0);
    c1 = max(c1, w[t].lo1); d1 = min(d1, w[t].lo1 + w[t].n1);
  }
  return Ranges{min16(h0), -min16(-e0), min16(h1), -min16(-e1), -min16(-c0), min16(d0), -min16(-c1), min16(d1)};
}

// The score of key k from the product x = q . k: natural units in fp32, log2 units in bf16 (where its
// exponential is the hardware's exp2 and tanh is formed from exp2 and rcp, a few 1e-7 of the cap
// off, far below a bf16 probability's rounding).  A finite score stays finite: the type's lowest
// value in a table is a score like any other.
template <bool F32>
__device__ __forceinline__ float score(const AttnSpanArgs& a, const Row& w, float x, int k) {
  float t = x * a.scale;
  if (a.cap > 0.f) {
    const float y = t / a.cap;
    t = a.cap * (F32 ? tanhf(y) : 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(2.f * kLog2e * y)));
  }
  if (a.bias_kind == BIAS_SLOPE) t -= w.bias[0] * fabsf((float)(k - w.pos));
  else if (a.bias_kind == BIAS_TABLE) t += w.bias[min(max(k - w.pos, -a.reach), a.reach)];
  if (F32) return t;
  const float u = t * kLog2e;
  return fabsf(t) <= kFltMax ? fminf(fmaxf(u, -kFltMax), kFltMax) : u;
}
template <bool F32>
__device__ __forceinline__ float exp_of(float t) { return F32 ? expf(t) : __builtin_amdgcn_exp2f(t); }

// exponents of one bf16 pair / one fp32 value that are all ones: an infinity or a NaN
__device__ __forceinline__ bool odd_bf16x2(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ uint32_t clean_bf16x2(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}
__device__ __forceinline__ bool odd_f32(float x) { return !(fabsf(x) <= kFltMax); }

// O^T of the merge and of a split's partial result: lane l holds row l % 16, dims 16 e + 4 (l / 16) + 0..3
template <int DT>
__device__ __forceinline__ void store_o4(void* out, size_t o, f32x4_t v) {
  if (DT == DT_BF16) *reinterpret_cast<u32x2_t*>(reinterpret_cast<uint16_t*>(out) + o) = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(out) + o) = v;
}

// Workspace of a split: per tile of 16 rows and split, 16 rows x 16 NE sums and 16 x (max, sum)
__host__ __device__ inline int part_floats(int ne) { return 16 * (16 * ne + 2); }

// Workgroup -> (split, 16-row tile, key head, sample)
struct Place { int split, tile, hk, b; };
__device__ __forceinline__ Place place_of(const AttnSpanArgs& a, int nsplit, int rows) {
  const int nt = (a.n_q * a.G + rows - 1) / rows;
  int id = blockIdx.x;
  Place p;
  p.split = id % nsplit; id /= nsplit;
  p.tile = id % nt; id /= nt;
  p.hk = id % a.H_kv;
  p.b = id / a.H_kv;
  return p;
}

// 16 rows a workgroup; its 4 waves take every fourth step of 32 keys, K straight from memory in
// operand layout, V (bf16) through the wave's own LDS rows for the transposed reads.  The next
// step's loads are in flight while this one's scores and products are formed.
template <int DT, int NE>
__global__ __launch_bounds__(256) void k_attn_dir(AttnSpanArgs a, int nsplit) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass needs the launch stub only
  constexpr bool F32 = DT == DT_F32;
  constexpr int NC = (NE + 1) / 2;              // bf16: k steps of 32 dims
  constexpr int CPR = NE * 2, NV = kKeys * CPR / 64;   // bf16: 16-byte chunks per V row, per lane
  constexpr int PV = NE * 32 + 16;              // bf16: bytes of a staged V row
  constexpr int kStage = F32 ? 0 : 4 * kKeys * PV, kMerge = 3 * (NE * 4 + 2) * 64 * 4;
  __shared__ __attribute__((aligned(1024))) char smem[kStage > kMerge ? kStage : kMerge];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const Place P = place_of(a, nsplit, 16);
  const int R = a.n_q * a.G, d = a.d;
  const int r = min(P.tile * 16 + l16, R - 1), qi = r / a.G;
  Row w[1] = {row_of(a, P.b, P.hk, r, qi)};
  const Ranges rg = ranges_of<1>(w);
  // this split's part of the rows' keys
  int first = min(rg.h0, rg.h1), end = max(rg.e0, rg.e1);
  if (first < end) {
    first &= ~(4 * kKeys - 1);
    const int chunk = ((end - first + nsplit - 1) / nsplit + 4 * kKeys - 1) & ~(4 * kKeys - 1);
    // split * chunk stays below n_k + 64 * 128 < 2^31
    first += P.split * chunk;
    end = min(end, first + chunk);
  } else {
    first = end = 0;
  }
  const size_t es = F32 ? 4 : 2;
  const char* qp = (const char*)a.q + ((size_t)P.b * a.qb + (size_t)qi * a.qr + (size_t)(P.hk * a.G + r % a.G) * a.qh) * es;
  const char* kp = (const char*)a.k + ((size_t)P.b * a.kb + (size_t)P.hk * a.kh) * es;
  const char* vp = (const char*)a.v + ((size_t)P.b * a.vb + (size_t)P.hk * a.vh) * es;
  const f32x4_t z4 = {0.f, 0.f, 0.f, 0.f};
  const u32x4_t zu = {0u, 0u, 0u, 0u};
  constexpr int NQ = F32 ? NE : NC, DQ = F32 ? 16 : 32, EQ = F32 ? 4 : 8;   // operand chunks, dims of each, dims a lane holds
  u32x4_t qf[NQ], kf[2][NQ], vf[F32 ? 1 : NV];
  float vv[F32 ? 8 : 1][F32 ? NE : 1];
#pragma unroll
  for (int c = 0; c < NQ; ++c) {
    const int e = DQ * c + EQ * g;
    qf[c] = e < d ? *reinterpret_cast<const u32x4_t*>(qp + e * es) : zu;
  }
  auto load = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < NQ; ++c) {
        const int k = k0 + 16 * i + l16, e = DQ * c + EQ * g;
        kf[i][c] = k < end && e < d ? *reinterpret_cast<const u32x4_t*>(kp + ((size_t)k * a.kr + e) * es) : zu;
      }
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int c = 0; c < NE; ++c) {
          const int k = k0 + 16 * (j / 4) + 4 * g + j % 4, e = 16 * c + l16;
          vv[j][c] = k < end && e < d ? *reinterpret_cast<const float*>(vp + ((size_t)k * a.vr + e) * 4) : 0.f;
        }
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int idx = j * 64 + lane, k = k0 + idx / CPR, e = idx % CPR * 8;
        vf[j] = k < end && e < d ? *reinterpret_cast<const u32x4_t*>(vp + ((size_t)k * a.vr + e) * 2) : zu;
      }
    }
  };
  f32x4_t o[NE];
#pragma unroll
  for (int e = 0; e < NE; ++e) o[e] = z4;
  float m = -INFINITY, l = 0.f;
  char* const stg = smem + wave * kKeys * PV;
  const uint32_t stg0 = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) const void*)stg);
  const uint32_t va = stg0 + (4 * g + (l16 >> 2)) * PV + (l16 & 3) * 8;
  auto next = [&](int k) __attribute__((always_inline)) {   // the next step whose keys some row sees
    while (k < end && !rg.some(k, kKeys)) k += 4 * kKeys;
    return k;
  };
  int k0 = next(first + wave * kKeys);
  if (k0 < end) load(k0);
  while (k0 < end) {
    const bool part = !rg.all(k0, kKeys);
    // rows that some queries see and others do not: an infinity or a NaN among them must not meet a
    // probability of zero.  Their products are formed without it, and it is added afterwards to
    // the rows that see its key.
    bool odd = false;
    if (part) {
      if constexpr (F32) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int c = 0; c < NE; ++c) odd = odd || odd_f32(vv[j][c]);
      } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) odd = odd || odd_bf16x2(vf[j][e]);
      }
      odd = __any(odd);
      if (odd) {
        if constexpr (F32) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int c = 0; c < NE; ++c) vv[j][c] = odd_f32(vv[j][c]) ? 0.f : vv[j][c];
        } else {
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[j][e] = clean_bf16x2(vf[j][e]);
        }
      }
    }
    if constexpr (!F32) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int idx = j * 64 + lane;
        *reinterpret_cast<u32x4_t*>(stg + idx / CPR * PV + idx % CPR * 16) = vf[j];
      }
    }
    f32x4_t sc[2] = {z4, z4};
#pragma unroll
    for (int c = 0; c < NQ; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (F32) {
          const f32x4_t kx = __builtin_bit_cast(f32x4_t, kf[i][c]), qx = __builtin_bit_cast(f32x4_t, qf[c]);
#pragma unroll
          for (int j = 0; j < 4; ++j) sc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[j], qx[j], sc[i], 0, 0, 0);
        } else {
          sc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[i][c]), __builtin_bit_cast(bf16x8_t, qf[c]), sc[i], 0, 0, 0);
        }
      }
    float p[8], x = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int k = k0 + 16 * (j / 4) + 4 * g + j % 4;
      p[j] = score<F32>(a, w[0], sc[j / 4][j % 4], k);
      if (part && !w[0].sees(k)) p[j] = -INFINITY;
      x = fmaxf(x, p[j]);
    }
    x = fmaxf(x, __shfl_xor(x, 16, 64));
    x = fmaxf(x, __shfl_xor(x, 32, 64));
    const float mn = fmaxf(m, x), mo = mn == -INFINITY ? 0.f : mn;
    const float al = exp_of<F32>(m - mo);   // exp(-inf) = 0
    m = mn;
    l *= al;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      p[j] = exp_of<F32>(p[j] - mo);
      l += p[j];
    }
#pragma unroll
    for (int e = 0; e < NE; ++e) o[e] *= al;
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int c = 0; c < NE; ++c) o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[j][c], p[j], o[c], 0, 0, 0);
      if (__builtin_expect(odd, 0)) {
        for (int k = k0; k < min(k0 + kKeys, end); ++k)
#pragma unroll
          for (int c = 0; c < NE; ++c) {
            if (16 * c + 4 * g >= d) continue;
            const f32x4_t y = *reinterpret_cast<const f32x4_t*>(vp + ((size_t)k * a.vr + 16 * c + 4 * g) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (odd_f32(y[e]) && w[0].sees(k)) o[c][e] += y[e];
          }
      }
      k0 = next(k0 + 4 * kKeys);
      if (k0 < end) load(k0);
    } else {
      const int kk = k0;
      k0 = next(k0 + 4 * kKeys);
      if (k0 < end) load(k0);
      const u32x4_t pw = {pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
      u32x2_t vt[NE][2];
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        vt[e][0] = lds_rd64_tr(va, e * 32);
        vt[e][1] = lds_rd64_tr(va, e * 32 + 16 * PV);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        FF_TIE(vt[e][0]);
        FF_TIE(vt[e][1]);
        const u32x4_t vw = {vt[e][0][0], vt[e][0][1], vt[e][1][0], vt[e][1][1]};
        o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vw), __builtin_bit_cast(bf16x8_t, pw), o[e], 0, 0, 0);
      }
      if (__builtin_expect(odd, 0)) {
        for (int k = kk; k < min(kk + kKeys, end); ++k)
#pragma unroll
          for (int c = 0; c < NE; ++c) {
            if (16 * c + 4 * g >= d) continue;
            const u32x2_t y = *reinterpret_cast<const u32x2_t*>(vp + ((size_t)k * a.vr + 16 * c + 4 * g) * 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float f = __uint_as_float(e & 1 ? y[e / 2] & 0xffff0000u : y[e / 2] << 16);
              if (odd_f32(f) && w[0].sees(k)) o[c][e] += f;
            }
          }
      }
    }
  }
  // the waves' (m, l, O) merge in wave order; l is per lane, m common to a row's four lanes
  float (*xch)[NE * 4 + 2][64] = reinterpret_cast<float (*)[NE * 4 + 2][64]>(smem);
  __syncthreads();   // every wave is done with its staged rows
  if (wave > 0) {
#pragma unroll
    for (int c = 0; c < NE; ++c)
#pragma unroll
      for (int v = 0; v < 4; ++v) xch[wave - 1][c * 4 + v][lane] = o[c][v];
    xch[wave - 1][NE * 4][lane] = m;
    xch[wave - 1][NE * 4 + 1][lane] = l;
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int v = 0; v < 3; ++v) {
    const float m2 = xch[v][NE * 4][lane], l2 = xch[v][NE * 4 + 1][lane];
    const float mn = fmaxf(m, m2), mo = mn == -INFINITY ? 0.f : mn;
    const float a1 = exp_of<F32>(m - mo), a2 = exp_of<F32>(m2 - mo);
    m = mn;
    l = l * a1 + l2 * a2;
#pragma unroll
    for (int c = 0; c < NE; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[c][e] = o[c][e] * a1 + xch[v][c * 4 + e][lane] * a2;
  }
  float s = l + __shfl_xor(l, 16, 64);
  s += __shfl_xor(s, 32, 64);
  if (nsplit > 1) {
    float* pt = a.part + (size_t)blockIdx.x * part_floats(NE);
#pragma unroll
    for (int c = 0; c < NE; ++c) *reinterpret_cast<f32x4_t*>(pt + l16 * 16 * NE + 16 * c + 4 * g) = o[c];
    if (g == 0) {
      pt[256 * NE + 2 * l16] = m;
      pt[256 * NE + 2 * l16 + 1] = s;
    }
    return;
  }
  if (P.tile * 16 + l16 >= R) return;
  const float inv = s == 0.f ? 0.f : 1.f / s;   // no key seen: zeros
  const size_t oo = (size_t)P.b * a.ob + (size_t)qi * a.orow + (size_t)(P.hk * a.G + r % a.G) * a.oh;
#pragma unroll
  for (int c = 0; c < NE; ++c)
    if (16 * c + 4 * g < d) store_o4<DT>(a.out, oo + 16 * c + 4 * g, o[c] * inv);
#endif
}

// Joins the splits of a row, a wavefront each: out = sum_s O_s e^(m_s - m) / sum_s l_s e^(m_s - m)
template <int DT>
__global__ __launch_bounds__(256) void k_attn_join(AttnSpanArgs a, int nsplit, int ne) {
  const int lane = threadIdx.x & 63;
  const int R = a.n_q * a.G, nt = (R + 15) / 16;
  const long row = (long)blockIdx.x * 4 + (threadIdx.x >> 6);   // (b, hk, r)
  if (row >= (long)a.B * a.H_kv * R) return;
  const int r = (int)(row % R), bh = (int)(row / R), hk = bh % a.H_kv, b = bh / a.H_kv;
  const float* pt = a.part + ((size_t)bh * nt + r / 16) * nsplit * part_floats(ne);
  const float* ml = pt + 256 * ne + 2 * (r % 16);
  // lane s < nsplit (at most 64) holds split s's statistics
  float ms = -INFINITY, ls = 0.f;
  if (lane < nsplit) {
    ms = ml[(size_t)lane * part_floats(ne)];
    ls = ml[(size_t)lane * part_floats(ne) + 1];
  }
  float m = ms;   // a NaN statistic makes its weight, and so the row, NaN
  m = wave_max(m);
  const float f = exp_of<DT == DT_F32>(ms - (m == -INFINITY ? 0.f : m));
  const float l = wave_sum(ls * f);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const size_t oo = (size_t)b * a.ob + (size_t)(r / a.G) * a.orow + (size_t)(hk * a.G + r % a.G) * a.oh;
  for (int e = lane; e < a.d; e += 64) {
    float x = 0.f;
    for (int s = 0; s < nsplit; ++s) x += pt[(size_t)s * part_floats(ne) + (size_t)(r % 16) * 16 * ne + e] * __shfl(f, s, 64);
    St<DT>::st1(a.out, oo + e, x * inv);
  }
}

int splits(long tiles, int n_k) {
  // four workgroups a CU, each with 256 keys or more
  const long by_grid = 1024 / (tiles > 0 ? tiles : 1), by_keys = n_k / 256;
  const long n = by_grid < by_keys ? by_grid : by_keys;
  return (int)(n < 1 ? 1 : n > kMaxSplit ? kMaxSplit : n);
}
int pieces(int d) { return d <= 32 ? 2 : d <= 48 ? 3 : d <= 64 ? 4 : d <= 80 ? 5 : d <= 96 ? 6 : 8; }
long tiles16(int B, int H_kv, int G, int n_q) { return (long)B * H_kv * (((long)n_q * G + 15) / 16); }

}  // namespace

size_t attention_span_workspace(int, int B, int H_kv, int G, int d, int n_q, int n_k) {
  const long t = tiles16(B, H_kv, G, n_q);
  const int n = splits(t, n_k);
  return n > 1 ? (size_t)t * n * part_floats(pieces(d)) * 4 : 0;
}

hipError_t attention_span(int dtype, const AttnSpanArgs& a, hipStream_t s) {
  if (a.n_q <= 0) return hipSuccess;
  const long t = tiles16(a.B, a.H_kv, a.G, a.n_q);
  const int n = splits(t, a.n_k), ne = pieces(a.d);
  if (t * n > 0x7fffffffL) return hipErrorInvalidValue;
#define FF_DIR(DT, NE) FF_LAUNCH((k_attn_dir<DT, NE>), (unsigned)(t * n), 256, 0, s, a, n)
#define FF_DIR_D(DT)                   \
  do {                                 \
    switch (ne) {                      \
      case 2: FF_DIR(DT, 2); break;    \
      case 3: FF_DIR(DT, 3); break;    \
      case 4: FF_DIR(DT, 4); break;    \
      case 5: FF_DIR(DT, 5); break;    \
      case 6: FF_DIR(DT, 6); break;    \
      default: FF_DIR(DT, 8); break;   \
    }                                  \
  } while (0)
  if (dtype == DT_BF16) FF_DIR_D(DT_BF16);
  else FF_DIR_D(DT_F32);
#undef FF_DIR_D
#undef FF_DIR
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || n == 1) return e;
  const long rows = (long)a.B * a.H_kv * a.n_q * a.G;
  if (dtype == DT_BF16) FF_LAUNCH(k_attn_join<DT_BF16>, (unsigned)((rows + 3) / 4), 256, 0, s, a, n, ne);
  else FF_LAUNCH(k_attn_join<DT_F32>, (unsigned)((rows + 3) / 4), 256, 0, s, a, n, ne);
  return hipGetLastError();
}

}  // namespace ff
