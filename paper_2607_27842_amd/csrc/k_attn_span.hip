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

typedef int i32x4_t __attribute__((ext_vector_type(4)));
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFltMax = 3.402823466e38f;
constexpr int kKeys = 32;        // keys per wavefront and step of the direct kernels
constexpr int kMaxSplit = 64;
// Largest cap for which bf16 forms cap tanh(t / cap) as cap - 2 cap / (1 + 2^(2 t log2(e) / cap)): near
// zero that is off by up to 1.3e-7 of the cap, 3e-5 at 256 (0.09 at 1e6, where a probability's rounding is
// 2^-8).  Above it, tanhf, as in fp32.
constexpr float kFastCap = 256.f;

// r / G and r % G of a row r < 2^30: mul = ceil(2^(31 + shift) / G) with 2^shift >= G is exact
__device__ __forceinline__ int query_of(const AttnSpanArgs& a, int r) { return (int)(((uint64_t)(uint32_t)r * a.gmul) >> (31 + a.gshift)); }

// What a lane keeps of its row.  Rows past the last repeat it (never stored).
struct Row {
  int lo0, n0, lo1, n1;   // the spans' first keys and lengths
  int pos;                // where the query stands among the keys
  const float* bias;      // its head's slope, or the middle of its table
  __device__ __forceinline__ bool none() const { return n0 == 0 && n1 == 0; }
  __device__ __forceinline__ bool sees(int k) const { return (unsigned)(k - lo0) < (unsigned)n0 || (unsigned)(k - lo1) < (unsigned)n1; }
};
// h: its head within the key head's
__device__ __forceinline__ Row row_of(const AttnSpanArgs& a, int b, int hk, int h, int i) {
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
    h += hk * a.G;
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
    if (w[t].none()) continue;   // gets zeros whatever is formed for it: its wavefront needs no mask
    c0 = max(c0, w[t].lo0); d0 = min(d0, w[t].lo0 + w[t].n0);
    c1 = max(c1, w[t].lo1); d1 = min(d1, w[t].lo1 + w[t].n1);
  }
  Ranges r{min16(h0), -min16(-e0), min16(h1), -min16(-e1), -min16(-c0), min16(d0), -min16(-c1), min16(d1)};
  r.d0 = min(r.d0, r.e0);   // (no rows at all: an empty core)
  r.d1 = min(r.d1, r.e1);
  return r;
}

// The scores of 8 keys from the products p = q . k, key j at k0 + 16 (j / 4) + j % 4: natural units in fp32,
// log2 units in bf16 (where the exponential is the hardware's exp2, and up to kFastCap tanh is formed from
// exp2 and rcp, far below a bf16 probability's rounding).  ANY: caps above kFastCap too.  A finite score stays
// finite: the type's lowest value in a table is a score like any other.  slope, tab: the head's slope or
// the keys' entries of its table.
template <bool F32, bool ANY>
__device__ __forceinline__ void scores(const AttnSpanArgs& a, const Row& w, float (&p)[8], int k0, float slope, const float (&tab)[8]) {
  if (ANY && a.cap > (F32 ? 0.f : kFastCap)) {
    const float c1 = a.scale / a.cap, c2 = a.cap;
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = c2 * tanhf(c1 * p[j]);
  } else if (a.cap > 0.f) {
    const float c1 = 2.f * kLog2e * a.scale / a.cap, c2 = a.cap;
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = fmaf(-2.f * c2, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(c1 * p[j])), c2);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] *= a.scale;
  }
  if (a.bias_kind == BIAS_SLOPE) {
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] -= slope * fabsf((float)(k0 + 16 * (j / 4) + j % 4 - w.pos));
  } else if (a.bias_kind == BIAS_TABLE) {
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] += tab[j];
  }
  if (!F32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float u = p[j] * kLog2e;
      p[j] = fabsf(p[j]) <= kFltMax ? fminf(fmaxf(u, -kFltMax), kFltMax) : u;
    }
  }
}
// e^t in fp32 (t <= 0: the rounding of t log2(e) is off by no more of t than the score's own, 2^-24), 2^t in bf16
template <bool F32>
__device__ __forceinline__ float exp_of(float t) { return __builtin_amdgcn_exp2f(F32 ? t * kLog2e : t); }

// Largest exponents of bf16 pairs / magnitude of fp32 values so far: all ones tell an infinity or a NaN
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
struct Top {
  u16x2_t b = {0, 0};
  uint32_t f = 0u;
  __device__ __forceinline__ void bf16x2(uint32_t w) { b = __builtin_elementwise_max(b, __builtin_bit_cast(u16x2_t, w & 0x7f807f80u)); }
  __device__ __forceinline__ void f32(float x) { f = max(f, __float_as_uint(x) & 0x7fffffffu); }
  __device__ __forceinline__ bool odd() const { return b[0] == 0x7f80u || b[1] == 0x7f80u || f >= 0x7f800000u; }
};
__device__ __forceinline__ uint32_t clean_bf16x2(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}
__device__ __forceinline__ bool odd_f32(float x) { return !(fabsf(x) <= kFltMax); }

// Chunks of 16 dims that stand together: in fp32 a lane loads 4, 2 or 1 neighbouring dims of a V row (as few
// and wide loads as NE allows), so that chunks c0 .. c0 + W - 1 hold every W-th of 16 W dims each.
template <bool F32, int NE>
__host__ __device__ constexpr int chunks_with(int c) { return !F32 ? 1 : c < (NE & ~3) ? 4 : c < (NE & ~1) ? 2 : 1; }
template <bool F32, int NE>
__host__ __device__ constexpr int chunk_first(int c) { return !F32 ? c : c < (NE & ~3) ? c & ~3 : c < (NE & ~1) ? NE & ~3 : c; }
// the dim of o[c][v] in lane l, g = l / 16
template <bool F32, int NE>
__device__ __forceinline__ int dim_of(int c, int v, int g) {
  const int c0 = chunk_first<F32, NE>(c), W = chunks_with<F32, NE>(c);
  return 16 * c0 + W * (4 * g + v) + c - c0;
}
// ... and the first of the four dims that piece c of in_order(o) holds
template <bool F32, int NE>
__device__ __forceinline__ int dims_at(int c, int g) {
  const int c0 = chunk_first<F32, NE>(c), W = chunks_with<F32, NE>(c);
  return 16 * c0 + 4 * (W * g + c - c0);
}
template <bool F32, int NE>
__device__ __forceinline__ f32x4_t in_order(const f32x4_t (&o)[NE], int c) {
  const int c0 = chunk_first<F32, NE>(c), W = chunks_with<F32, NE>(c);
  f32x4_t y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = o[c0 + (4 * (c - c0) + e) % W][(4 * (c - c0) + e) / W];
  return y;
}
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
  if (nsplit == 1) {
    // The last rows of all heads first, which see the most keys under a causal mask, so that short walks
    // close the grid (fp32, heads of 64: B = 2, 12 heads, 777 causal tokens 33.8 us, head after head 39.4;
    // 12 heads, 1500 tokens 51.4, 63.8)
    const int heads = a.B * a.H_kv;
    p.split = 0;
    p.tile = nt - 1 - id / heads;
    id %= heads;
  } else {
    p.split = id % nsplit; id /= nsplit;
    p.tile = id % nt; id /= nt;
  }
  p.hk = id % a.H_kv;
  p.b = id / a.H_kv;
  return p;
}

// One wavefront's 16 rows over the keys of [first, end) (first a multiple of 32) in steps of 32, `stride` keys
// from one step to the next: K straight from memory in operand layout, V (bf16) through the wave's
// own LDS rows (stg) for the transposed reads.  The next step's loads are in flight while this
// one's scores and products are formed.  Rows of V that some queries see and others do not may hold
// an infinity or a NaN, which must not meet a probability of zero: the product is formed without
// it, and it is added afterwards to the rows that see its key.
// Result: m (the same in a row's four lanes), l (to be added over them), o.  ANY: of any cap (scores).
template <int DT, int NE, bool ANY>
__device__ __forceinline__ void attend16(const AttnSpanArgs& a, const Row& w, const Ranges& rg, const char* qp, const char* kp,
                                         const char* vp, int first, int end, int stride, char* stg, f32x4_t (&o)[NE], float& m, float& l) {
  constexpr bool F32 = DT == DT_F32;
  constexpr int NC = (NE + 1) / 2;              // bf16: k steps of 32 dims
  constexpr int CPR = NE * 2, NV = kKeys * CPR / 64;   // bf16: 16-byte chunks per V row, per lane
  constexpr int PV = NE * 32 + 16;              // bf16: bytes of a staged V row
  constexpr size_t es = F32 ? 4 : 2;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, d = a.d;
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
  // A step's loads go through resources that end with its last key's last element: keys past it load
  // as zeros (or, with a stride below d, as elements of the last keys), and so do dims past d.
  constexpr uint32_t kOut = 0x80000000u;
  const uint32_t kl = (uint32_t)a.kr * (uint32_t)es, vl = (uint32_t)a.vr * (uint32_t)es;
  constexpr int NT = NQ > 2 ? 2 : NQ;           // the last chunks, where d may end
  constexpr bool kStep = !F32 && CPR == 16;     // chunks j lie 4 j rows further
  uint32_t ko[2], kt[2][NT], vo[F32 || kStep ? 1 : NV];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    ko[i] = (16 * i + l16) * kl + EQ * g * (uint32_t)es;
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      const int e = DQ * (NQ - NT + c);
      kt[i][c] = e + EQ * g < d ? ko[i] + e * (uint32_t)es : kOut;
    }
  }
  if constexpr (F32) {
    vo[0] = 4 * g * vl;
  } else {
#pragma unroll
    for (int j = 0; j < (kStep ? 1 : NV); ++j) {
      const int idx = j * 64 + lane, e = idx % CPR * 8;
      vo[j] = e < d ? (idx / CPR) * vl + e * 2u : kOut;
    }
  }
  constexpr bool kEarly = !F32 || NE <= 6;   // (fp32, d = 128: both steps' K and V do not fit the registers)
  auto load_k = [&](int k0) __attribute__((always_inline)) {
    const uint32_t last = min(end - k0, kKeys) - 1;
    __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(kp) + (size_t)k0 * kl, 0, last * kl + d * (int)es, 0x00020000);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < NQ; ++c)
        kf[i][c] = __builtin_amdgcn_raw_buffer_load_b128(rk, c < NQ - NT ? ko[i] + c * DQ * (int)es : kt[i][c < NQ - NT ? 0 : c - (NQ - NT)], 0, 0);
  };
  auto load_v = [&](int k0) __attribute__((always_inline)) {
    const uint32_t last = min(end - k0, kKeys) - 1;
    __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vp) + (size_t)k0 * vl, 0, last * vl + d * (int)es, 0x00020000);
    if constexpr (F32) {
      uint32_t at = vo[0];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j) at += j == 4 ? 13 * vl : vl;
        FF_TIE(at);   // formed here, one from the other: kept over the loop they would spill
#pragma unroll
        for (int c = 0; c < NE; c += chunks_with<F32, NE>(c)) {   // dims past d (d % 8 == 0): what lies there, or zeros; never stored
          const int W = chunks_with<F32, NE>(c);
          if (W == 4) {
            const u32x4_t y = __builtin_amdgcn_raw_buffer_load_b128(rv, at + c * 64 + l16 * 16, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) vv[j][c + e < NE ? c + e : 0] = __uint_as_float(y[e]);
          } else if (W == 2) {
            const u32x2_t y = __builtin_amdgcn_raw_buffer_load_b64(rv, at + c * 64 + l16 * 8, 0, 0);
            vv[j][c] = __uint_as_float(y[0]);
            vv[j][c + 1 < NE ? c + 1 : 0] = __uint_as_float(y[1]);
          } else {
            vv[j][c] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rv, at + c * 64 + l16 * 4, 0, 0));
          }
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) vf[j] = __builtin_amdgcn_raw_buffer_load_b128(rv, kStep ? vo[0] + j * 4 * vl : vo[kStep ? 0 : j], 0, 0);
    }
  };
  const float slope = a.bias_kind == BIAS_SLOPE ? w.bias[0] : 0.f;
#pragma unroll
  for (int e = 0; e < NE; ++e) o[e] = z4;
  m = -INFINITY;
  l = 0.f;
  const uint32_t stg0 = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) const void*)stg);
  const uint32_t va = stg0 + (4 * g + (l16 >> 2)) * PV + (l16 & 3) * 8;
  auto next = [&](int k) __attribute__((always_inline)) {   // the next step whose keys some row sees
    while (k < end && !rg.some(k, kKeys)) k += stride;
    return k;
  };
  int k0 = next(first);
  if (k0 < end) {
    load_k(k0);
    load_v(k0);
  }
  while (k0 < end) {
    float tab[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.bias_kind == BIAS_TABLE) {   // before the next step's loads, which would have to land first
#pragma unroll
      for (int j = 0; j < 8; ++j) tab[j] = w.bias[min(max(k0 + 4 * g + 16 * (j / 4) + j % 4 - w.pos, -a.reach), a.reach)];
    }
    const bool part = !rg.all(k0, kKeys);
    bool odd = false;
    auto look = [&]() __attribute__((always_inline)) {
      Top top;
      if constexpr (F32) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int c = 0; c < NE; ++c) top.f32(vv[j][c]);
      } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) top.bf16x2(vf[j][e]);
      }
      odd = __any(top.odd());
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
    };
    if constexpr (!F32) {
      if (part) look();
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
    const int kk = k0;
    k0 = next(k0 + stride);
    if (k0 < end) {   // K is in the scores; V in LDS, or (fp32) still needed
      if constexpr (kEarly) load_k(k0);
      if constexpr (!F32) load_v(k0);
    }
    float p[8], x = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = sc[j / 4][j % 4];
    scores<F32, ANY>(a, w, p, kk + 4 * g, slope, tab);
    if (part) {
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = w.sees(kk + 16 * (j / 4) + 4 * g + j % 4) ? p[j] : -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x = fmaxf(x, p[j]);
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
      if (part) look();
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int c = 0; c < NE; ++c) o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[j][c], p[j], o[c], 0, 0, 0);
      if (__builtin_expect(odd, 0)) {
        for (int k = kk; k < min(kk + kKeys, end); ++k) {
          const float* row = reinterpret_cast<const float*>(vp) + (size_t)k * a.vr;
          const bool sees = w.sees(k);
          int gd = g;
          FF_TIE(gd);   // nothing of this is formed ahead of the loop over the steps
#pragma unroll
          for (int c = 0; c < NE; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float y = row[min(dim_of<F32, NE>(c, e, gd), d - 1)];   // (dims past d are never stored)
              if (odd_f32(y) && sees) o[c][e] += y;
            }
        }
      }
      if (k0 < end) {
        if constexpr (!kEarly) load_k(k0);
        load_v(k0);
      }
    } else {
      const u32x4_t pw = {pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
      // in two halves, for the registers
      constexpr int NH = (NE + 1) / 2;
#pragma unroll
      for (int h = 0; h < NE; h += NH) {
        u32x2_t vt[NH][2];
#pragma unroll
        for (int e = 0; e < NH; ++e)
          if (h + e < NE) {
            vt[e][0] = lds_rd64_tr(va, (h + e) * 32);
            vt[e][1] = lds_rd64_tr(va, (h + e) * 32 + 16 * PV);
          }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int e = 0; e < NH; ++e)
          if (h + e < NE) {
            FF_TIE(vt[e][0]);
            FF_TIE(vt[e][1]);
            const u32x4_t vw = {vt[e][0][0], vt[e][0][1], vt[e][1][0], vt[e][1][1]};
            o[h + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vw), __builtin_bit_cast(bf16x8_t, pw), o[h + e], 0, 0, 0);
          }
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
              if (odd_f32(f) && w.sees(k)) o[c][e] += f;
            }
          }
      }
    }
  }
  if (w.none()) {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < NE; ++e) o[e] = z4;
  }
}

// 16 rows a workgroup, whose 4 waves take every fourth step of 32 keys; with few rows the keys of a row
// are split over workgroups too, in equal parts of the rows' own keys.
// What bounds it: memory on long caches (B = 8 ragged up to 32768 keys, 16 heads on 4 of 128: 67 us and
// 5 for the join, 4.5 TB/s), latency on short ones (33 tokens 6 us); in fp32 the fp32 MFMA rate and the
// softmax's vector instructions, which do not run beside them (1500 tokens, 12 heads of 64: 85 to 92 us, 75
// to 82 TFLOP/s; 32 rows a wavefront, with half the loads but two wavefronts a SIMD instead of three, 110).
template <int DT, int NE>
__global__ __launch_bounds__(256, 2) void k_attn_dir(AttnSpanArgs a, int nsplit) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass needs the launch stub only
  constexpr bool F32 = DT == DT_F32;
  constexpr int PV = NE * 32 + 16;              // bf16: bytes of a staged V row
  constexpr int kStage = F32 ? 0 : 4 * kKeys * PV, kMerge = 3 * (NE * 4 + 2) * 64 * 4;
  __shared__ __attribute__((aligned(1024))) char smem[kStage > kMerge ? kStage : kMerge];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const Place P = place_of(a, nsplit, 16);
  const int R = a.n_q * a.G, d = a.d;
  const int r = min(P.tile * 16 + l16, R - 1), qi = query_of(a, r), qh = r - qi * a.G;
  Row w[1] = {row_of(a, P.b, P.hk, qh, qi)};
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
  const char* qp = (const char*)a.q + ((size_t)P.b * a.qb + (size_t)qi * a.qr + (size_t)(P.hk * a.G + qh) * a.qh) * es;
  const char* kp = (const char*)a.k + ((size_t)P.b * a.kb + (size_t)P.hk * a.kh) * es;
  const char* vp = (const char*)a.v + ((size_t)P.b * a.vb + (size_t)P.hk * a.vh) * es;
  f32x4_t o[NE];
  float m, l;
  attend16<DT, NE, true>(a, w[0], rg, qp, kp, vp, first + wave * kKeys, end, 4 * kKeys, smem + wave * kKeys * PV, o, m, l);
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
    for (int c = 0; c < NE; ++c) *reinterpret_cast<f32x4_t*>(pt + l16 * 16 * NE + dims_at<F32, NE>(c, g)) = in_order<F32, NE>(o, c);
    if (g == 0) {
      pt[256 * NE + 2 * l16] = m;
      pt[256 * NE + 2 * l16 + 1] = s;
    }
    return;
  }
  if (P.tile * 16 + l16 >= R) return;
  // No key seen, or none with a weight: zeros, also where 0 * V has met an infinity or a NaN
  const bool none = s == 0.f;
  const float inv = 1.f / s;
  const size_t oo = (size_t)P.b * a.ob + (size_t)qi * a.orow + (size_t)(P.hk * a.G + qh) * a.oh;
#pragma unroll
  for (int c = 0; c < NE; ++c)
    if (dims_at<F32, NE>(c, g) < d) store_o4<DT>(a.out, oo + dims_at<F32, NE>(c, g), none ? f32x4_t{0.f, 0.f, 0.f, 0.f} : in_order<F32, NE>(o, c) * inv);
#endif
}

// Joins the splits of a row, a workgroup each: out = sum_s O_s e^(m_s - m) / sum_s l_s e^(m_s - m).
// 8 groups of 32 lanes take every eighth split, 4 dims a lane, so that a lane's loads (at most 8) are in
// flight together (one wavefront walking up to 64 splits took 35 us of a call's 50).
template <int DT>
__global__ __launch_bounds__(256) void k_attn_join(AttnSpanArgs a, int nsplit, int ne) {
  __shared__ float f[kMaxSplit], linv;
  __shared__ f32x4_t part[8][32];
  const int tid = threadIdx.x, lane = tid & 63, q = tid & 31, grp = tid >> 5;
  const int R = a.n_q * a.G, nt = (R + 15) / 16, pf = part_floats(ne);
  const int r = blockIdx.x % R, bh = blockIdx.x / R, hk = bh % a.H_kv, b = bh / a.H_kv;
  const float* pt = a.part + ((size_t)bh * nt + r / 16) * nsplit * pf;
  const float* row = pt + (r % 16) * 16 * ne + 4 * q;
  f32x4_t x[kMaxSplit / 8];
  const bool in = 4 * q < a.d;
#pragma unroll
  for (int i = 0; i < kMaxSplit / 8; ++i) {
    const int s = 8 * i + grp;
    x[i] = in && s < nsplit ? *reinterpret_cast<const f32x4_t*>(row + (size_t)s * pf) : f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  if (tid < 64) {   // lane s holds split s's statistics; a NaN sum makes the row NaN
    float ms = -INFINITY, ls = 0.f;
    if (lane < nsplit) {
      ms = pt[(size_t)lane * pf + 256 * ne + 2 * (r % 16)];
      ls = pt[(size_t)lane * pf + 256 * ne + 2 * (r % 16) + 1];
    }
    const float m = wave_max(ms), w = exp_of<DT == DT_F32>(ms - (m == -INFINITY ? 0.f : m)), l = wave_sum(ls * w);
    f[lane] = w;
    if (lane == 0) linv = l == 0.f ? 0.f : 1.f / l;   // 0: no split has a weight, zeros below whatever the sums are
  }
  __syncthreads();
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kMaxSplit / 8; ++i)
    if (8 * i + grp < nsplit) o += x[i] * f[8 * i + grp];
  part[grp][q] = o;
  __syncthreads();
  if (tid >= 32 || !in) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) o += part[i][q];
  const int qi = query_of(a, r);
  store_o4<DT>(a.out, (size_t)b * a.ob + (size_t)qi * a.orow + (size_t)(hk * a.G + r - qi * a.G) * a.oh + 4 * q,
               linv == 0.f ? f32x4_t{0.f, 0.f, 0.f, 0.f} : o * linv);
}

// ---------------------------------------------------------------- bf16, many rows: two wave groups in turn
// 8 waves of 16 QT rows in two groups of four (one wave of each per SIMD), 64-key tiles of K and V in
// rings of four, as in the blocks' own attention (k_attn_pp, where the slots, the layouts and what
// bounds them stand).  Per tile a wave has a softmax slot (the tile's probabilities, and the DMA of
// the tiles three and two ahead) and an MFMA slot (the next tile's scores, then this tile's P V),
// each ended by a barrier; the second group runs one slot behind.
// A workgroup walks the tiles that its rows' spans meet.  Per tile a wave knows whether all its rows
// see all keys (no mask), some (each score is tested against its row's spans), or none (zero
// probabilities at once).
// MOD: capped or biased scores, formed in log2 units before the softmax; caps above kFastCap have instances
// of their own (with both in one, tanhf's constants took up to 6 registers of the others' loop, and
// spilled 2 where there are 128).
// What bounds it: as k_attn_pp, in its time (N = 14566, H = 16, d = 128 1424 us).  With 256 of those rows
// padded text: 1390 to 1440 us, 1.16 to 1.2 PFLOP/s; 24 heads of 128, 8192 causal tokens 367 us, 1.12.  Short spans
// are bound by what a workgroup does once, 8 us, and by the softmax of its partly seen tiles (packed prompts of
// 4096 tokens with about 600 each, 16 heads on 8: 44 us, 180 TFLOP/s; capped 45 to 48).
// (two workgroups share a CU where a K or V row takes 128 bytes of LDS: at most 128 VGPRs)
enum Mod { kModNone, kMod, kModWide };
template <int RWB, int NC, int NE, int QT, Mod MOD>
__global__ __launch_bounds__(512, RWB == 128 ? 4 : 2) void k_attn_span_pp(AttnSpanArgs a) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass needs the launch stub only
  constexpr int KB = 64, NB = 4;                 // keys per tile, ring depth
  constexpr int TB = KB * RWB;                   // bytes of a K (or V) tile
  constexpr int DPW = RWB / 128;                 // DMA instructions per wave, tile and operand
  constexpr int CPR = RWB / 16;                  // 16-byte chunks per LDS row
  static_assert(NC * 64 <= RWB && NE * 32 <= RWB, "head dim tiles fit the LDS row");
  constexpr int LDO = NE * 16 + 8;               // staged output row pitch (elements)
  // after the walk each wavefront has a region of its own, for V rows (attend16) and for its output
  constexpr int kOwn = kKeys * (NE * 32 + 16) > 16 * QT * LDO * 2 ? kKeys * (NE * 32 + 16) : 16 * QT * LDO * 2;
  constexpr int kMain = 2 * NB * TB, kOut = 8 * kOwn;
  constexpr float kPLim = 256.0f;                // as in k_attn_pp: what raises a row's running maximum
  constexpr int kRows = kMain > kOut ? kMain : kOut;   // behind it, the rows' spans (read where a tile needs a mask)
  __shared__ __attribute__((aligned(1024))) char smem[kRows + 128 * QT * 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int R = a.n_q * a.G, d = a.d;
  int qb, hk, b;
  {
    const int nqb = (R + 128 * QT - 1) / (128 * QT), n = gridDim.x, id = blockIdx.x, heads = a.H_kv * a.B;
    // An XCD gets neighbouring places of one head after the other, the last rows first.  With spans its heads
    // go four at a time, the last rows of all four first (they see the most keys under a causal mask: 24
    // heads of 128, 8192 causal tokens 367 us for 416; 24 of 64, 2048 tokens 34 for 44); heads that do not
    // divide among the XCDs go all at once if they are few (20 of 128, 8000 tokens 314 us for 391).  All at
    // once, 33 to 60 heads would gain on causal masks too (33 of 128, 8000 tokens 520 us for 600), but 100
    // would lose (8000 tokens 1632 us for 1522 to 1577), and so would heads whose rows all see as much (33 of
    // 128, 14566 tokens, 256 of them padded: 3224 us for 2890 to 3000).
    int qr, bh;   // place from the last rows on, head of all samples
    if (a.n_spans && heads % 8 == 0) {
      const int i = id / 8, hx = heads / 8, first = i / (4 * nqb) * 4, m = min(4, hx - first), k = i - first * nqb;
      bh = id % 8 * hx + first + k % m;
      qr = k / m;
    } else if (a.n_spans && heads <= 32) {
      bh = id % heads;
      qr = id / heads;
    } else {
      const int full = n / 8 * 8;
      const int t = id < full ? (id % 8) * (full / 8) + id / 8 : id;
      bh = t / nqb;
      qr = t - bh * nqb;
    }
    qb = __builtin_amdgcn_readfirstlane(nqb - 1 - qr);
    hk = __builtin_amdgcn_readfirstlane(bh % a.H_kv);
    b = __builtin_amdgcn_readfirstlane(bh / a.H_kv);
  }
  const int q0 = qb * 128 * QT + wave * 16 * QT;
  Row rows[QT];
  bf16x8_t qf[QT][NC];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = min(q0 + 16 * t + l16, R - 1), i = query_of(a, r), h = r - i * a.G;
    rows[t] = row_of(a, b, hk, h, i);
    const uint16_t* qp = (const uint16_t*)a.q + (size_t)b * a.qb + (size_t)i * a.qr + (size_t)(hk * a.G + h) * a.qh;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int e = 32 * c + 8 * g;
      u32x4_t v = {0u, 0u, 0u, 0u};
      if (e < d) v = *reinterpret_cast<const u32x4_t*>(qp + e);
      qf[t][c] = __builtin_bit_cast(bf16x8_t, v);
    }
  }
  Ranges rg{0, a.n_k, 0x7fffffff, 0, 0, a.n_k, 0, 0};
  if (a.n_spans) rg = ranges_of<QT>(rows);
  int pos[QT];
  const float* bias[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    pos[t] = rows[t].pos;
    bias[t] = rows[t].bias;
    if (g == 0) *reinterpret_cast<i32x4_t*>(smem + kRows + (wave * 16 * QT + 16 * t + l16) * 16) = i32x4_t{rows[t].lo0, rows[t].n0, rows[t].lo1, rows[t].n1};
  }
  // the workgroup's tiles: those of the first hull, then those of the second beyond it, ascending
  int t0 = 0, n0 = (a.n_k + KB - 1) / KB, t1 = 0, nt = n0;
  if (a.n_spans) {
    // (LDS waits only: the queries' loads stay in flight)
    int* const x = reinterpret_cast<int*>(smem);
    if (lane == 0) *reinterpret_cast<i32x4_t*>(x + wave * 4) = i32x4_t{rg.h0, rg.e0, rg.h1, rg.e1};
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    int h0 = 0x7fffffff, e0 = 0, h1 = 0x7fffffff, e1 = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const i32x4_t y = *reinterpret_cast<const i32x4_t*>(x + w * 4);
      h0 = min(h0, y[0]); e0 = max(e0, y[1]); h1 = min(h1, y[2]); e1 = max(e1, y[3]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    int a0 = h0 / KB, b0 = (e0 + KB - 1) / KB, a1 = h1 / KB, b1 = (e1 + KB - 1) / KB;
    if (e0 <= 0) a0 = b0 = 0;
    if (e1 <= 0) a1 = b1 = 0;
    if (b0 == a0) { a0 = a1; b0 = b1; a1 = b1 = 0; }                        // one range, if any, comes first
    if (b1 > a1 && a1 < a0) { const int p = a0, q = b0; a0 = a1; b0 = b1; a1 = p; b1 = q; }
    if (b1 > a1 && a1 <= b0) { b0 = max(b0, b1); a1 = b1 = 0; }             // meeting ranges are one
    t0 = __builtin_amdgcn_readfirstlane(a0);
    n0 = __builtin_amdgcn_readfirstlane(b0 - a0);
    t1 = __builtin_amdgcn_readfirstlane(a1);
    nt = __builtin_amdgcn_readfirstlane(b0 - a0 + b1 - a1);
  }
  const char* const kp = (const char*)a.k + ((size_t)b * a.kb + (size_t)hk * a.kh) * 2;
  const char* const vp = (const char*)a.v + ((size_t)b * a.vb + (size_t)hk * a.vh) * 2;
  // the rows of an LDS tile are rotated by f(row) among their 16-byte chunks, so that both the
  // K reads (16 rows, one chunk) and the transposed V reads (8 rows, one chunk pair) of a
  // pass spread over all banks
  auto swz = [](int row) {
    const int hi = (row >> 3) & 1;
    return (CPR == 16 ? ((row & 7) ^ (hi << 2)) : (((row >> 1) & 3) ^ (hi << 1))) << 1 | hi;
  };
  uint32_t vok[DPW], vov[DPW];   // this lane's byte offsets within a tile; past d: out of range (zeros)
#pragma unroll
  for (int j = 0; j < DPW; ++j) {
    const int idx = (wave * DPW + j) * 64 + lane, row = idx / CPR, e = ((idx % CPR) ^ swz(row)) * 8;
    vok[j] = e < d ? (uint32_t)row * (uint32_t)a.kr * 2u + (uint32_t)e * 2u : 0x80000000u;
    vov[j] = e < d ? (uint32_t)row * (uint32_t)a.vr * 2u + (uint32_t)e * 2u : 0x80000000u;
  }
  // The walk over K's and V's tiles: the next tile's address, its keys up to the last, its number and
  // its ring slot, advanced tile by tile; what happens once or at the end is branched to (formed
  // anew for each tile, with selects, this took 100 scalar instructions of the softmax slot).
  struct Walk { const char* p; int left, j, stop, slot; };   // stop: the tile number at which a range ends
  const uint32_t kl = (uint32_t)a.kr * 2u, vl = (uint32_t)a.vr * 2u, fullk = (KB - 1) * kl + d * 2, fullv = (KB - 1) * vl + d * 2;
  Walk wk{kp + (size_t)t0 * KB * kl, a.n_k - t0 * KB, 0, n0, 0}, wv{vp + (size_t)t0 * KB * vl, a.n_k - t0 * KB, 0, n0, 0};
  // DMA of the walk's next tile.  The tile's resource ends with the last key's last element, so that
  // keys past it, and tiles past the walk, load as zeros (or, with a stride below d, as elements of
  // the last keys: their probabilities are zero)
  auto load = [&](Walk& w, const char* base, uint32_t ld, uint32_t full, const uint32_t (&vo)[DPW], int off) __attribute__((always_inline)) {
    uint32_t num = full;
    if (__builtin_expect(w.left < KB, 0)) {
      asm volatile("");
      num = w.left > 0 ? (uint32_t)(w.left - 1) * ld + d * 2 : 0u;
    }
    __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(w.p), 0, num, 0x00020000);
#pragma unroll
    for (int i = 0; i < DPW; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, FF_AS3(smem + off + w.slot + (wave * DPW + i) * 1024), 16, vo[i], 0, 0, 0);
    ++w.j;
    w.left -= KB;
    w.p += (size_t)KB * ld;
    if (__builtin_expect(w.j == w.stop, 0)) {   // on to the second range, or at the end
      asm volatile("");
      w.left = w.j < nt ? a.n_k - t1 * KB : 0;
      w.p = base + (size_t)t1 * KB * ld;
      w.stop = nt;
    }
    w.slot = (w.slot + TB) & (NB * TB - 1);
  };
  auto load_k = [&]() __attribute__((always_inline)) { load(wk, kp, kl, fullk, vok, 0); };
  auto load_v = [&]() __attribute__((always_inline)) { load(wv, vp, vl, fullv, vov, NB * TB); };
  // fragment addresses within a tile (k step c and output tile e enter by xor)
  const uint32_t lds0 = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) const void*)smem);
  const uint32_t ka = lds0 + l16 * RWB + ((g ^ swz(l16)) * 16);
  const int vr = 4 * g + (l16 >> 2);
  const uint32_t va = lds0 + NB * TB + vr * RWB + ((((l16 & 3) >> 1) ^ swz(vr)) * 16) + (l16 & 1) * 8;
  f32x4_t o[NE][QT], sc[4][QT];
#pragma unroll
  for (int e = 0; e < NE; ++e)
#pragma unroll
    for (int t = 0; t < QT; ++t) o[e][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m[QT], l[QT], lim[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) { m[t] = -INFINITY; l[t] = 0.f; lim[t] = -1.f; }
  const float sl2 = MOD ? 1.f : a.scale * kLog2e;
  bf16x8_t pb[2][QT];
  int ks = 0, vs = 0;            // ring slots being read
  // The MFMA slot of a tile is a chain of units of two A fragments and 2 QT MFMAs: first
  // the 2 NC units of the next tile's scores (K fragments), then the NE units of this tile's
  // PV product (V^T fragments, each two transposed reads).  A unit's reads are issued UD
  // units ahead.
  constexpr int UK = 2 * NC, UV = NE, UD = 3;
  bf16x8_t kf[UD + 1][2];
  u32x2_t vf[UD + 1][2][2] = {};
  uint32_t ka_ = ka, va_ = va;
  auto rd = [&](auto Uc) __attribute__((always_inline)) {
    constexpr int U = decltype(Uc)::value;
    if constexpr (U < UK) {
      constexpr int c = U / 2, i0 = U % 2 * 2;
      const uint32_t ad = ka_ ^ (c * 64);
      kf[U % (UD + 1)][0] = lds_rd128_at<i0 * 16 * RWB>(ad);
      kf[U % (UD + 1)][1] = lds_rd128_at<(i0 + 1) * 16 * RWB>(ad);
    } else if constexpr (U < UK + UV) {
      constexpr int f = 2 * (U - UK);
      const uint32_t a0 = va_ ^ (f % NE * 32), a1 = va_ ^ ((f + 1) % NE * 32);
      vf[U % (UD + 1)][0][0] = lds_rd64_tr(a0, f / NE * 32 * RWB);
      vf[U % (UD + 1)][0][1] = lds_rd64_tr(a0, f / NE * 32 * RWB + 16 * RWB);
      vf[U % (UD + 1)][1][0] = lds_rd64_tr(a1, (f + 1) / NE * 32 * RWB);
      vf[U % (UD + 1)][1][1] = lds_rd64_tr(a1, (f + 1) / NE * 32 * RWB + 16 * RWB);
    }
  };
  auto unit = [&](auto Uc) __attribute__((always_inline)) {
    constexpr int U = decltype(Uc)::value;
    rd(Int<U + UD>{});
    constexpr int later = (U + 1 < UK + UV ? (U + 1 < UK ? 2 : 4) : 0) + (U + 2 < UK + UV ? (U + 2 < UK ? 2 : 4) : 0) +
                          (U + 3 < UK + UV ? (U + 3 < UK ? 2 : 4) : 0);
    asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(later) : "memory");
    constexpr int buf = U % (UD + 1);
    if constexpr (U < UK) {
      FF_TIE(kf[buf][0]); FF_TIE(kf[buf][1]);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          constexpr int c = U / 2, i0 = U % 2 * 2;
          sc[i0 + i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[buf][i], qf[t][c], c == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sc[i0 + i][t], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) { FF_TIE(vf[buf][i][0]); FF_TIE(vf[buf][i][1]); }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        constexpr int f0 = 2 * (U - UK);
        const int s = (f0 + i) / NE, e = (f0 + i) % NE;
        const u32x4_t w = {vf[buf][i][0][0], vf[buf][i][0][1], vf[buf][i][1][0], vf[buf][i][1][1]};
#pragma unroll
        for (int t = 0; t < QT; ++t)
          o[e][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), pb[s][t], o[e][t], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // the V reads that run ahead of a chain of scores alone are used nowhere, but hold their
  // registers until they are in
  auto drain = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < (UD + 1) * 4; ++i) FF_TIE(vf[i / 4][i / 2 % 2][i % 2]);
  };
#define FF_BAR() asm volatile("s_barrier" ::: "memory")
  auto spans_at = [&](int t) __attribute__((always_inline)) {
    i32x4_t w;
    asm volatile("ds_read_b128 %0, %1 offset:%2\n\ts_waitcnt lgkmcnt(0)" : "=v"(w) : "v"(lds0 + kRows + (wave * 16 * QT + l16) * 16), "i"(t * 256) : "memory");
    return w;
  };
  // a row's bias beyond the table's reach, on either side (log2 units)
  float below[MOD ? QT : 1], above[MOD ? QT : 1];
  if constexpr (MOD) {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      below[t] = a.bias_kind == BIAS_TABLE ? bias[t][-a.reach] : a.bias_kind == BIAS_SLOPE ? bias[t][0] : 0.f;
      above[t] = a.bias_kind == BIAS_TABLE ? bias[t][a.reach] : 0.f;
    }
  }
  // sc -> scores in log2 units
  auto modify = [&](int k0) __attribute__((always_inline)) {
    if constexpr (MOD == kModWide) {
      const float c1 = a.scale / a.cap, c2 = a.cap;
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int v = 0; v < 4; ++v) sc[i][t][v] = c2 * tanhf(c1 * sc[i][t][v]);
    } else if (a.cap > 0.f) {
      const float c1 = 2.f * kLog2e * a.scale / a.cap, c2 = a.cap;
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            sc[i][t][v] = fmaf(-2.f * c2, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(c1 * sc[i][t][v])), c2);
    } else {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[i][t] *= a.scale;
    }
    if (a.bias_kind == BIAS_SLOPE) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const float at = (float)(k0 + 4 * g - pos[t]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int v = 0; v < 4; ++v) sc[i][t][v] = fmaf(-below[t], fabsf(at + (float)(16 * i + v)), sc[i][t][v]);
      }
    } else if (a.bias_kind == BIAS_TABLE) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const int at = k0 - pos[t];   // the tile's first distance
        const bool lo = __all(at + KB - 1 <= -a.reach), hi = __all(at >= a.reach);
        if (lo || hi) {
          const float c = lo ? below[t] : above[t];
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[i][t] += c;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) sc[i][t][v] += bias[t][min(max(at + 16 * i + 4 * g + v, -a.reach), a.reach)];
        }
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) {   // a finite score stays finite
          const float x = sc[i][t][v], y = x * kLog2e;
          sc[i][t][v] = fabsf(x) <= kFltMax ? fminf(fmaxf(y, -kFltMax), kFltMax) : y;
        }
  };
  // sc -> probabilities pb (complete when it returns: nothing of it moves past the barrier)
  auto softmax = [&](int k0, bool all, bool some) __attribute__((always_inline)) {
    if (!all && !some) {
#pragma unroll
      for (int t = 0; t < QT; ++t) pb[0][t] = pb[1][t] = __builtin_bit_cast(bf16x8_t, u32x4_t{0u, 0u, 0u, 0u});
    } else {
      if constexpr (MOD) modify(k0);
      if (!all) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          const i32x4_t w = spans_at(t);
          const int at = k0 + 4 * g - w[0], at1 = k0 + 4 * g - w[2];
          if (a.n_spans > 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int v = 0; v < 4; ++v)
                sc[i][t][v] = (unsigned)(at + 16 * i + v) < (unsigned)w[1] || (unsigned)(at1 + 16 * i + v) < (unsigned)w[3] ? sc[i][t][v] : -INFINITY;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int v = 0; v < 4; ++v) sc[i][t][v] = (unsigned)(at + 16 * i + v) < (unsigned)w[1] ? sc[i][t][v] : -INFINITY;
          }
        }
      }
      // probabilities against the running maxima m (log2 units), raised only where a lane's 16
      // probabilities of a row add up to more than kPLim or are not all numbers
      float p[QT][16], ps[QT];
      bool up = false;
      auto probs = [&](int t) __attribute__((always_inline)) {
        const float mo = m[t] == -INFINITY ? 0.f : m[t];
#pragma unroll
        for (int i = 0; i < 16; ++i) p[t][i] = __builtin_amdgcn_exp2f(MOD ? sc[i / 4][t][i % 4] - mo : fmaf(sc[i / 4][t][i % 4], sl2, -mo));
        float s4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s4[i] = (p[t][4 * i] + p[t][4 * i + 1]) + (p[t][4 * i + 2] + p[t][4 * i + 3]);
        ps[t] = (s4[0] + s4[1]) + (s4[2] + s4[3]);
      };
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        probs(t);
        up = up || !(ps[t] <= lim[t]);
      }
      if (__any(up)) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          float x = -INFINITY;
#pragma unroll
          for (int i = 0; i < 16; ++i) x = fmaxf(x, sc[i / 4][t][i % 4]);
          x = fmaxf(x, __shfl_xor(x, 16, 64));         // the four lanes of a row together
          x = fmaxf(x, __shfl_xor(x, 32, 64)) * sl2;   // scale > 0: max commutes with it
          const float mn = fmaxf(m[t], ceilf(x));      // whole: the rescale is by a power of two, exact
          const float al = mn == m[t] ? 1.f : __builtin_amdgcn_exp2f(m[t] - mn);   // exp2(-inf) = 0
          m[t] = mn;
          lim[t] = mn == -INFINITY ? -1.f : kPLim;     // -1: the next tile comes here too
          l[t] *= al;
#pragma unroll
          for (int e = 0; e < NE; ++e) o[e][t] *= al;
          probs(t);
        }
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        l[t] += ps[t];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const float* q = &p[t][8 * s];
          const u32x4_t w = {pack_bf16x2(q[0], q[1]), pack_bf16x2(q[2], q[3]), pack_bf16x2(q[4], q[5]), pack_bf16x2(q[6], q[7])};
          pb[s][t] = __builtin_bit_cast(bf16x8_t, w);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) { FF_TIE(pb[0][t]); FF_TIE(pb[1][t]); FF_TIE(l[t]); }
    __builtin_amdgcn_sched_barrier(0);
  };
  // tiles that start in [c, c + core) lie in a core as a whole
  const unsigned core0 = max(rg.d0 - rg.c0 - KB + 1, 0), core1 = max(rg.d1 - rg.c1 - KB + 1, 0);
  bool mixed = false;   // some tile held keys that a row does not see
  if (nt > 0) {
    load_k();
    load_k(); load_v();
    load_k(); load_v();
    wait_vm<2 * DPW>();
    FF_BAR();
    static_for<0, UD>(rd);
    static_for<0, UK>(unit);   // the first tile's scores
    drain();
    ks = TB;
    if (wave >= 4) FF_BAR();   // the second group runs one slot behind
    int k0 = t0 * KB, run = 0;
    for (int j = 0; j < nt; ++j) {
      load_k();
      load_v();
      __builtin_amdgcn_sched_barrier(0);
      bool all = true, some = false;
      if (__builtin_expect(k0 >= run, 0)) {   // outside the core that the walk was last in
        asm volatile("");
        const bool in0 = (unsigned)(k0 - rg.c0) < core0, in1 = (unsigned)(k0 - rg.c1) < core1;
        all = in0 || in1;
        run = in0 ? rg.c0 + (int)core0 : in1 ? rg.c1 + (int)core1 : 0;
        if (!all) {
          some = rg.some(k0, KB);
          mixed = true;
        }
      }
      softmax(k0, all, some);
      ka_ = ka + ks;
      va_ = va + vs;
      static_for<0, UD>(rd);
      wait_vm<2 * DPW>();
      FF_BAR();
      __builtin_amdgcn_s_setprio(1);
      static_for<0, UK + UV>(unit);
      __builtin_amdgcn_s_setprio(0);
      FF_BAR();
      ks = (ks + TB) & (NB * TB - 1);
      vs = (vs + TB) & (NB * TB - 1);
      k0 += KB;
      if (__builtin_expect(j + 1 == n0, 0)) {
        asm volatile("");
        k0 = t1 * KB;
      }
    }
    wait_vm<0>();
    if (wave < 4) FF_BAR();
    FF_BAR();   // the DMA of every wave has ended, before the staging below
  }
#undef FF_BAR
  // An infinity or a NaN in a row of V that a query does not see has met its probability of zero: such
  // results are not numbers, and the wavefront's rows are formed again without it (attend16).
  // Results that are not numbers by right come here too.
  if (mixed) {
    Top top;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const i32x4_t w = spans_at(t);
      if (w[1] == 0 && w[3] == 0) continue;
#pragma unroll
      for (int e = 0; e < NE; ++e)
#pragma unroll
        for (int v = 0; v < 4; ++v) top.f32(o[e][t][v]);
    }
    if (__builtin_expect(__any(top.odd()), 0)) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const int r = min(q0 + 16 * t + l16, R - 1), i = query_of(a, r), h = r - i * a.G;
        const Row w[1] = {row_of(a, b, hk, h, i)};
        const Ranges rt = ranges_of<1>(w);
        const char* qp = (const char*)((const uint16_t*)a.q + (size_t)b * a.qb + (size_t)i * a.qr + (size_t)(hk * a.G + h) * a.qh);
        const int end = max(rt.e0, rt.e1);
        f32x4_t x[NE];
        attend16<DT_BF16, NE, MOD == kModWide>(a, w[0], rt, qp, kp, vp, end > 0 ? min(rt.h0, rt.h1) & ~(kKeys - 1) : 0, end, kKeys,
                              smem + wave * kOwn, x, m[t], l[t]);
#pragma unroll
        for (int e = 0; e < NE; ++e) o[e][t] = x[e];
      }
    }
  }
  // o[e][t][v] = O[row q0 + 16 t + l16][16 e + 4 g + v], staged through the wave's own LDS
  // region and stored as 16-byte row pieces
  uint16_t* stg = reinterpret_cast<uint16_t*>(smem + wave * kOwn);
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float s = l[t] + __shfl_xor(l[t], 16, 64);
    s += __shfl_xor(s, 32, 64);
    const i32x4_t w = spans_at(t);
    const bool none = s == 0.f || (w[1] == 0 && w[3] == 0);   // no key seen: zeros, whatever has been formed
    const float inv = 1.0f / s;
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      const u32x2_t y = {pack_bf16x2(o[e][t][0] * inv, o[e][t][1] * inv), pack_bf16x2(o[e][t][2] * inv, o[e][t][3] * inv)};
      *reinterpret_cast<u32x2_t*>(stg + (16 * t + l16) * LDO + 16 * e + 4 * g) = none ? u32x2_t{0u, 0u} : y;
    }
  }
  uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + (size_t)b * a.ob;
  const int ppr = d / 8;
  for (int idx = lane; idx < 16 * QT * ppr; idx += 64) {
    const int row = idx / ppr, pc = idx - row * ppr, r = q0 + row, i = query_of(a, r);
    if (r < R)
      *reinterpret_cast<u32x4_t*>(out + (size_t)i * a.orow + (size_t)(hk * a.G + r - i * a.G) * a.oh + pc * 8) =
          *reinterpret_cast<const u32x4_t*>(stg + row * LDO + pc * 8);
  }
#endif
}

int splits(long tiles, int n_k) {
  // four workgroups a CU, each with 256 keys or more
  const long by_grid = 1024 / (tiles > 0 ? tiles : 1), by_keys = n_k / 256;
  const long n = by_grid < by_keys ? by_grid : by_keys;
  return (int)(n < 1 ? 1 : n > kMaxSplit ? kMaxSplit : n);
}
int pieces(int d) { return d <= 32 ? 2 : d <= 48 ? 3 : d <= 64 ? 4 : d <= 80 ? 5 : d <= 96 ? 6 : 8; }
template <Mod MOD>
hipError_t launch_pp_mod(const AttnSpanArgs& a, bool two, hipStream_t s) {
  const long nwg = ((long)a.n_q * a.G + (two ? 255 : 127)) / (two ? 256 : 128) * a.H_kv * a.B;
  if (nwg > 0x7fffffffL) return hipErrorInvalidValue;
#define FF_ATTN(RWB, NC, NE)                                                                                       \
  do {                                                                                                             \
    if constexpr (RWB > 128 && MOD == kModNone)                                                                    \
      if (two) { FF_LAUNCH((k_attn_span_pp<RWB, NC, NE, 2, MOD>), (unsigned)nwg, 512, 0, s, a); break; }           \
    FF_LAUNCH((k_attn_span_pp<RWB, NC, NE, 1, MOD>), (unsigned)nwg, 512, 0, s, a);                                 \
  } while (0)
  if (a.d <= 48) FF_ATTN(128, 2, 3);
  else if (a.d <= 64) FF_ATTN(128, 2, 4);
  else if (a.d <= 80) FF_ATTN(256, 3, 5);
  else if (a.d <= 96) FF_ATTN(256, 3, 6);
  else FF_ATTN(256, 4, 8);
#undef FF_ATTN
  return hipGetLastError();
}
bool modified(const AttnSpanArgs& a) { return a.cap > 0.f || a.bias_kind != BIAS_NONE; }
hipError_t launch_pp(const AttnSpanArgs& a, bool two, hipStream_t s) {
  if (a.cap > kFastCap) return launch_pp_mod<kModWide>(a, two, s);
  return modified(a) ? launch_pp_mod<kMod>(a, two, s) : launch_pp_mod<kModNone>(a, two, s);
}
long tiles16(int B, int H_kv, int G, int n_q) { return (long)B * H_kv * (((long)n_q * G + 15) / 16); }

}  // namespace

// The splits of the direct kernel's keys, or k_attn_span_pp, by estimated time (us; all keys seen),
// fitted to 1 to 16 heads of 64 and 128, 16 to 1000 tokens, B 1 to 8.  The direct kernel: 1.9 for each 128
// keys of a workgroup or 6.5e-3 for each of all workgroups' together; k_attn_span_pp: 1.1 (0.8 for d <= 64)
// for each 64 keys and round of workgroups.
//   B = 1, 16 heads of 128: 33 tokens 5.9 against 8.2 us, 256 tokens 9.0 against 10.3, 640 26 against 16
//   B = 4, 16 heads of 128: 64 tokens 6.1 against 7.6, 128 tokens 10.8 against 8.8, 1000 163 against 44
// k_attn_span_pp takes 16 rows a wave for d <= 64 (two workgroups then share a CU); above, 16 or 32, as
// k_attn_pp (32 with capped or biased scores does not fit the registers).
SpanPlan attention_span_plan(int dtype, int B, int H_kv, int G, int d, int n_q, int n_k, int mod) {
  const long t = tiles16(B, H_kv, G, n_q);
  const int n = splits(t, n_k);
  if (dtype == DT_F32) return SpanPlan{16, n};
  const double turns = (double)((n_k + 127) / 128), chain = 1.9 * turns / n, work = 6.5e-3 * t * turns;
  const double dir = 5.0 + (chain > work ? chain : work) + (n > 1 ? 5.0 : 0.0);
  const long hb = (long)B * H_kv, R = (long)n_q * G, w1 = (R + 127) / 128 * hb, w2 = (R + 255) / 256 * hb;
  const long at_once = d <= 64 ? 512 : 256;
  const double pp = 6.3 + (d <= 64 ? 0.8 : 1.1) * ((n_k + 63) / 64) * ((w1 + at_once - 1) / at_once);
  if (dir <= pp) return SpanPlan{16, n};
  return SpanPlan{!mod && d > 64 && (double)((w2 + 255) / 256) <= 0.63 * ((w1 + 255) / 256) ? 32 : 16, 0};
}

size_t attention_span_workspace(int dtype, int B, int H_kv, int G, int d, int n_q, int n_k) {
  if (n_q <= 0) return 0;
  const int n = attention_span_plan(dtype, B, H_kv, G, d, n_q, n_k, 0).splits;   // (the same for any scores)
  return n > 1 ? (size_t)tiles16(B, H_kv, G, n_q) * n * part_floats(pieces(d)) * 4 : 0;
}

hipError_t attention_span(int dtype, const AttnSpanArgs& args, hipStream_t s) {
  if (args.n_q <= 0) return hipSuccess;
  AttnSpanArgs a = args;
  while ((1L << a.gshift) < a.G) ++a.gshift;
  a.gmul = (uint32_t)(((1ull << (31 + a.gshift)) + a.G - 1) / a.G);
  const long t = tiles16(a.B, a.H_kv, a.G, a.n_q);
  const SpanPlan p = attention_span_plan(dtype, a.B, a.H_kv, a.G, a.d, a.n_q, a.n_k, modified(a));
  const int n = p.splits, ne = pieces(a.d);
  if (n == 0) return launch_pp(a, p.rows == 32, s);
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
  if (dtype == DT_BF16) FF_LAUNCH(k_attn_join<DT_BF16>, (unsigned)rows, 256, 0, s, a, n, ne);
  else FF_LAUNCH(k_attn_join<DT_F32>, (unsigned)rows, 256, 0, s, a, n, ne);
  return hipGetLastError();
}

}  // namespace ff
