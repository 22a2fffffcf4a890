// Host side of the operators on 8-bit operands and of attention over spans: argument checks and
// dispatch behind include/featfix.h.  Everything is checked before anything is launched.
#include <math.h>

#include "featfix.h"
#include "host.h"
#include "kernels.h"

using namespace ff;

namespace {

typedef __int128 wide;
constexpr int64_t kMaxPitch = (int64_t)1 << 40;   // products with row counts stay inside 128 bits
// Rows of a call: a launch has fewer than 2^32 threads, and up to 256 of them work on a row
constexpr int kMaxRows = 1 << 23;
constexpr float kLeastScale = 0x1p-60f;

bool dtype_ok(int dt) { return dt == FF_F32 || dt == FF_BF16; }

// A strided buffer's bytes, first to last, and where its rows take `width` bytes every `pitch` (0: no such rows)
struct Extent {
  const char* p;
  wide n, pitch, width;
  bool meets(const Extent& o) const {
    if (!p || !o.p || n <= 0 || o.n <= 0) return false;
    const wide at = (wide)(uintptr_t)p, ot = (wide)(uintptr_t)o.p;
    if (at >= ot + o.n || ot >= at + n) return false;
    if (pitch <= 0 || pitch != o.pitch) return true;
    // columns of one wider buffer
    const wide off = ((ot - at) % pitch + pitch) % pitch;
    return off < width || off + o.width > pitch;
  }
};
Extent rows_of(const void* p, int64_t rows, int64_t cols, int64_t pitch, int es) {
  return {(const char*)p, rows > 0 && cols > 0 ? ((wide)(rows - 1) * pitch + cols) * es : 0, (wide)pitch * es, (wide)cols * es};
}
// a pitch of `cols` columns that keeps every row on a multiple of `unit` elements
bool pitch_ok(int64_t pitch, int64_t cols, int unit) { return pitch >= cols && pitch <= kMaxPitch && pitch % unit == 0; }

#define CHECK(cond, code, ...) \
  do {                         \
    if (!(cond)) return fail(code, __VA_ARGS__); \
  } while (0)

ff_status check_quant(const ff_quant_desc* d) {
  CHECK(d, FF_E_NULL, "quant descriptor is NULL");
  CHECK(dtype_ok(d->dtype), FF_E_DTYPE, "unknown dtype %d", d->dtype);
  CHECK(d->block_rows == 1 || d->block_rows == kQBlock, FF_E_RANGE, "block_rows=%d must be 1 or %d", d->block_rows, kQBlock);
  CHECK(d->rows >= 0 && d->rows <= kMaxRows, FF_E_SHAPE, "rows=%d outside [0, 2^23]", d->rows);
  CHECK(d->C >= 8 && d->C % 8 == 0 && (int64_t)d->C * d->rows <= (int64_t)1 << 35 && d->C <= 1 << 24, FF_E_SHAPE,
        "C=%d must be a multiple of 8 in [8, 2^24] with rows * C <= 2^35", d->C);
  CHECK(pitch_ok(d->x_row, d->C, 8) && pitch_ok(d->q_row, d->C, 8), FF_E_SHAPE, "x_row and q_row must be multiples of 8 and >= C");
  const int64_t least = d->block_rows == 1 ? d->rows : (d->C + kQBlock - 1) / kQBlock;
  CHECK(d->qs_ld >= least && d->qs_ld <= kMaxPitch, FF_E_SHAPE, "qs_ld=%lld must be >= %lld", (long long)d->qs_ld, (long long)least);
  return FF_OK;
}

ff_status check_norm(const ff_norm_desc* d, bool resid, bool sum, bool y, bool q) {
  CHECK(d, FF_E_NULL, "norm descriptor is NULL");
  CHECK(dtype_ok(d->dtype), FF_E_DTYPE, "unknown dtype %d", d->dtype);
  CHECK(d->eps > 0.f && isfinite(d->eps), FF_E_RANGE, "eps must be > 0");
  CHECK(d->rows >= 0 && d->rows <= kMaxRows, FF_E_SHAPE, "rows=%d outside [0, 2^23]", d->rows);
  CHECK(d->C >= 8 && d->C % 8 == 0 && d->C <= kNormMaxC, FF_E_SHAPE, "C=%d must be a multiple of 8 in [8, %d]", d->C, kNormMaxC);
  CHECK(pitch_ok(d->x_row, d->C, 8), FF_E_SHAPE, "x_row must be a multiple of 8 and >= C");
  CHECK(!resid || pitch_ok(d->resid_row, d->C, 8), FF_E_SHAPE, "resid_row must be a multiple of 8 and >= C");
  CHECK(!sum || pitch_ok(d->sum_row, d->C, 8), FF_E_SHAPE, "sum_row must be a multiple of 8 and >= C");
  CHECK(!y || pitch_ok(d->y_row, d->C, 8), FF_E_SHAPE, "y_row must be a multiple of 8 and >= C");
  CHECK(!q || pitch_ok(d->q_row, d->C, 8), FF_E_SHAPE, "q_row must be a multiple of 8 and >= C");
  CHECK(!q || (d->qs_ld >= d->rows && d->qs_ld <= kMaxPitch), FF_E_SHAPE, "qs_ld must be >= rows");
  return FF_OK;
}

ff_status check_gemm(const ff_gemm_q8_desc* d, bool resid) {
  CHECK(d, FF_E_NULL, "gemm descriptor is NULL");
  CHECK(dtype_ok(d->out_dtype), FF_E_DTYPE, "unknown dtype %d", d->out_dtype);
  CHECK(d->gelu == 0 || d->gelu == 1, FF_E_RANGE, "gelu must be 0 or 1");
  CHECK(d->M >= 0 && d->M <= kMaxRows, FF_E_SHAPE, "M=%d outside [0, 2^23]", d->M);
  CHECK(d->N >= 8 && d->N % 8 == 0 && d->N <= 1 << 20 && (int64_t)d->M * d->N <= (int64_t)1 << 34, FF_E_SHAPE,
        "N=%d must be a multiple of 8 in [8, 2^20] with M * N <= 2^34", d->N);
  CHECK(d->K >= 16 && d->K % 16 == 0 && d->K <= 1 << 24, FF_E_SHAPE, "K=%d must be a multiple of 16 in [16, 2^24]", d->K);
  CHECK(pitch_ok(d->a_row, d->K, 16) && pitch_ok(d->w_row, d->K, 16), FF_E_SHAPE, "a_row and w_row must be multiples of 16 and >= K");
  CHECK(pitch_ok(d->out_row, d->N, 8) && (!resid || pitch_ok(d->resid_row, d->N, 8)), FF_E_SHAPE,
        "out_row and resid_row must be multiples of 8 and >= N");
  const int64_t nb = (d->K + kQBlock - 1) / kQBlock, na = (d->N + kQBlock - 1) / kQBlock;
  CHECK(d->as_ld >= d->M && d->ws_ld >= nb, FF_E_SHAPE, "as_ld must be >= M and ws_ld >= ceil(K / %d)", kQBlock);
  const int64_t lim = 0x7fffff00ll;   // byte offsets inside a tile's buffers are 32 bits wide
  CHECK(d->as_ld <= kMaxPitch && d->ws_ld <= kMaxPitch && (wide)256 * d->a_row < lim && (wide)256 * d->w_row < lim &&
        (wide)nb * d->as_ld * 4 < lim && (wide)na * d->ws_ld * 4 < lim, FF_E_SHAPE,
        "256 operand rows and the scales of an operand must lie within 2^31 bytes");
  return FF_OK;
}

// out's elements lie apart: by ascending stride, each axis steps over what the ones before it span
bool apart(int64_t s0, int64_t n0, int64_t s1, int64_t n1, int64_t s2, int64_t n2, int64_t inner) {
  int64_t s[3] = {s0, s1, s2}, n[3] = {n0, n1, n2};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (s[j] > s[j + 1]) {
        const int64_t x = s[j], y = n[j];
        s[j] = s[j + 1]; n[j] = n[j + 1];
        s[j + 1] = x; n[j + 1] = y;
      }
  wide span = inner;
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (s[i] < span) return false;
    span += (wide)s[i] * (n[i] - 1);
  }
  return true;
}

ff_status check_attn(const ff_attn_desc* d) {
  CHECK(d, FF_E_NULL, "attention descriptor is NULL");
  CHECK(dtype_ok(d->dtype), FF_E_DTYPE, "unknown dtype %d", d->dtype);
  CHECK(d->B >= 1 && d->H >= 1 && d->H_kv >= 1 && d->H % d->H_kv == 0, FF_E_SHAPE, "need B >= 1 and H a multiple of H_kv (B=%d H=%d H_kv=%d)",
        d->B, d->H, d->H_kv);
  CHECK(d->d >= 8 && d->d <= 128 && d->d % 8 == 0, FF_E_SHAPE, "d=%d must be a multiple of 8 in [8, 128]", d->d);
  CHECK(d->n_q >= 0 && d->n_k >= 0 && d->n_k < 1 << 30 && (wide)d->n_q * d->H * d->B < 1 << 30, FF_E_SHAPE,
        "n_q * H * B and n_k must be in [0, 2^30)");
  CHECK((wide)d->B * d->H_kv * (((int64_t)d->n_q * (d->H / d->H_kv) + 15) / 16) < kMaxRows, FF_E_SHAPE,
        "B * H_kv * ceil(n_q * H / H_kv / 16) must be below 2^23");
  const int64_t st[12] = {d->q_batch, d->q_row, d->q_head, d->k_batch, d->k_row, d->k_head,
                          d->v_batch, d->v_row, d->v_head, d->o_batch, d->o_row, d->o_head};
  for (int64_t x : st) CHECK(x >= 0 && x % 8 == 0 && x <= kMaxPitch, FF_E_SHAPE, "strides must be non-negative multiples of 8");
  const int es = (int)dsize(d->dtype);
  CHECK((wide)d->k_row * es * 64 < 0x7fffff00ll && (wide)d->v_row * es * 64 < 0x7fffff00ll, FF_E_SHAPE,
        "64 key or value rows must lie within 2^31 bytes");
  CHECK(apart(d->o_batch, d->B, d->o_row, d->n_q, d->o_head, d->H, d->d), FF_E_SHAPE, "out's rows overlap each other");
  // scale / cap has to be a normal number: an infinite one would make a score of zero NaN
  CHECK(d->scale >= kLeastScale && d->scale <= 1.f / kLeastScale, FF_E_RANGE, "scale must be in [2^-60, 2^60]");
  CHECK(d->cap == 0.f || (d->cap >= kLeastScale && d->cap <= 1.f / kLeastScale), FF_E_RANGE, "cap must be 0 or in [2^-60, 2^60]");
  CHECK(d->bias_kind >= FF_BIAS_NONE && d->bias_kind <= FF_BIAS_TABLE, FF_E_RANGE, "bias_kind=%d unknown", d->bias_kind);
  CHECK(d->bias_kind != FF_BIAS_TABLE || (d->bias_reach >= 0 && d->bias_reach <= 1 << 20), FF_E_RANGE, "bias_reach=%d outside [0, 2^20]", d->bias_reach);
  CHECK(d->n_spans >= 0 && d->n_spans <= 2, FF_E_RANGE, "n_spans=%d must be 0, 1 or 2", d->n_spans);
  CHECK(d->n_spans == 0 || (d->span_batch >= 0 && d->span_batch <= kMaxPitch), FF_E_SHAPE, "span_batch must be >= 0");
  return FF_OK;
}

Extent attn_extent(const void* p, int64_t B, int64_t sb, int64_t n, int64_t sr, int64_t H, int64_t sh, int64_t d, int es) {
  const wide width = (wide)(H - 1) * sh + d;
  const bool rows = sr >= width && (B == 1 || sb % sr == 0);   // a row's heads stand together, samples whole rows apart
  return {(const char*)p, B > 0 && n > 0 && H > 0 ? ((wide)(B - 1) * sb + (wide)(n - 1) * sr + width) * es : 0,
          rows ? (wide)sr * es : 0, width * es};
}

}  // namespace

extern "C" {

ff_status ff_quant_q8(const ff_quant_desc* d, const void* x, void* q, float* qs, ff_stream_t stream) {
  const ff_status e = check_quant(d);
  if (e) return e;
  if (d->rows == 0) return ok();
  CHECK(x && q && qs, FF_E_NULL, "x, q or qs is NULL");
  CHECK(aligned16(x) && aligned16(q) && aligned16(qs), FF_E_SHAPE, "pointers must be 16-byte aligned");
  const bool sq = d->block_rows != 1;
  const int64_t nb = (d->C + kQBlock - 1) / kQBlock;
  const Extent ex = rows_of(x, d->rows, d->C, d->x_row, (int)dsize(d->dtype)), eq = rows_of(q, d->rows, d->C, d->q_row, 1);
  const Extent es = sq ? rows_of(qs, ((int64_t)d->rows + kQBlock - 1) / kQBlock, nb, d->qs_ld, 4) : rows_of(qs, nb, d->rows, d->qs_ld, 4);
  CHECK(!ex.meets(eq) && !ex.meets(es) && !eq.meets(es), FF_E_SHAPE, "x, q and qs must not overlap");
  const QuantArgs a{x, d->x_row, (uint8_t*)q, d->q_row, qs, d->qs_ld, d->rows, d->C};
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  HIP_TRY(sq ? quant_squares(d->dtype, a, st) : quant_rows(d->dtype, a, st), "8-bit quantisation");
  return ok();
}

ff_status ff_rms_norm_q8(const ff_norm_desc* d, const void* x, const void* resid, const void* gain, void* sum, void* y,
                         void* q, float* qs, ff_stream_t stream) {
  const ff_status e = check_norm(d, resid != nullptr, sum != nullptr, y != nullptr, q != nullptr);
  if (e) return e;
  if (d->rows == 0) return ok();
  CHECK(x, FF_E_NULL, "x is NULL");
  CHECK(y || q, FF_E_NULL, "y and q are both NULL");
  CHECK((q == nullptr) == (qs == nullptr), FF_E_NULL, "q and qs go together");
  CHECK(!sum || resid, FF_E_NULL, "sum needs resid");
  const void* ps[] = {x, resid, gain, sum, y, q, qs};
  for (const void* p : ps) CHECK(!p || aligned16(p), FF_E_SHAPE, "pointers must be 16-byte aligned");
  const int es = (int)dsize(d->dtype);
  const Extent in[3] = {rows_of(x, d->rows, d->C, d->x_row, es), rows_of(resid, d->rows, d->C, d->resid_row, es),
                        rows_of(gain, 1, d->C, d->C, es)};
  const Extent out[4] = {rows_of(sum, d->rows, d->C, d->sum_row, es), rows_of(y, d->rows, d->C, d->y_row, es),
                         rows_of(q, d->rows, d->C, d->q_row, 1),
                         rows_of(qs, (d->C + kQBlock - 1) / kQBlock, d->rows, d->qs_ld, 4)};
  for (int o = 0; o < 4; ++o) {
    for (int i = 0; i < 3; ++i) {
      // the sum may take the place of either addend: a row's loads precede its stores
      if (o == 0 && ((i == 0 && sum == x && d->sum_row == d->x_row) || (i == 1 && sum == resid && d->sum_row == d->resid_row))) continue;
      CHECK(!out[o].meets(in[i]), FF_E_SHAPE, "an output overlaps an input");
    }
    for (int p = 0; p < o; ++p) CHECK(!out[o].meets(out[p]), FF_E_SHAPE, "two outputs overlap");
  }
  const RmsArgs a{x, d->x_row, resid, d->resid_row, gain, sum, d->sum_row, y, d->y_row, (uint8_t*)q, d->q_row, qs, d->qs_ld,
                  d->rows, d->C, d->eps};
  HIP_TRY(rms_norm_q8(d->dtype, a, reinterpret_cast<hipStream_t>(stream)), "rms norm");
  return ok();
}

size_t ff_gemm_q8_workspace_bytes(const ff_gemm_q8_desc* d) {
  return check_gemm(d, false) ? 0 : gemm_q8_workspace(d->out_dtype, d->M, d->N, d->K);
}

ff_status ff_gemm_q8(const ff_gemm_q8_desc* d, const void* a, const float* a_s, const void* w, const float* w_s,
                     const void* bias, const void* resid, void* out, void* ws, size_t ws_bytes, ff_stream_t stream) {
  const ff_status e = check_gemm(d, resid != nullptr);
  if (e) return e;
  if (d->M == 0) return ok();
  CHECK(a && a_s && w && w_s && out, FF_E_NULL, "a, a_s, w, w_s or out is NULL");
  const size_t need = gemm_q8_workspace(d->out_dtype, d->M, d->N, d->K);
  CHECK(!need || ws, FF_E_NULL, "ws is NULL");
  CHECK(ws_bytes >= need, FF_E_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, need);
  const void* ps[] = {a, a_s, w, w_s, bias, resid, out, need ? ws : nullptr};
  for (const void* p : ps) CHECK(!p || aligned16(p), FF_E_SHAPE, "pointers must be 16-byte aligned");
  const int es = (int)dsize(d->out_dtype);
  const int64_t nb = (d->K + kQBlock - 1) / kQBlock;
  const Extent in[6] = {rows_of(a, d->M, d->K, d->a_row, 1), rows_of(a_s, nb, d->M, d->as_ld, 4),
                        rows_of(w, d->N, d->K, d->w_row, 1),
                        rows_of(w_s, (d->N + kQBlock - 1) / kQBlock, nb, d->ws_ld, 4),
                        rows_of(bias, 1, d->N, d->N, es), rows_of(resid, d->M, d->N, d->resid_row, es)};
  const Extent eo = rows_of(out, d->M, d->N, d->out_row, es), ew{(const char*)ws, (wide)need, 0, 0};
  for (int i = 0; i < 6; ++i) {
    CHECK(!ew.meets(in[i]), FF_E_SHAPE, "the workspace overlaps an input");
    if (i == 5 && out == resid && d->out_row == d->resid_row) continue;   // each element is read by the lane that writes it
    CHECK(!eo.meets(in[i]), FF_E_SHAPE, "out overlaps an input");
  }
  CHECK(!eo.meets(ew), FF_E_SHAPE, "out overlaps the workspace");
  const GemmQ8Args g{(const uint8_t*)a, d->a_row, a_s, d->as_ld, (const uint8_t*)w, d->w_row, w_s, d->ws_ld, bias, resid,
                     d->resid_row, out, d->out_row, d->M, d->N, d->K, d->gelu, need ? (float*)ws : nullptr};
  HIP_TRY(gemm_q8(d->out_dtype, g, reinterpret_cast<hipStream_t>(stream)), "8-bit gemm");
  return ok();
}

size_t ff_attention_workspace_bytes(const ff_attn_desc* d) {
  return check_attn(d) ? 0 : attention_span_workspace(d->dtype, d->B, d->H_kv, d->H / d->H_kv, d->d, d->n_q, d->n_k);
}

ff_status ff_attention(const ff_attn_desc* d, const void* q, const void* k, const void* v, const float* bias,
                       const int32_t* pos, const int32_t* spans, void* out, void* ws, size_t ws_bytes, ff_stream_t stream) {
  const ff_status e = check_attn(d);
  if (e) return e;
  if (d->n_q == 0) return ok();
  CHECK(q && out && ((k && v) || d->n_k == 0), FF_E_NULL, "q, k, v or out is NULL");
  CHECK((d->bias_kind == FF_BIAS_NONE) == (bias == nullptr), FF_E_NULL, "bias and bias_kind disagree");
  CHECK((d->n_spans == 0) == (spans == nullptr), FF_E_NULL, "spans and n_spans disagree");
  const size_t need = attention_span_workspace(d->dtype, d->B, d->H_kv, d->H / d->H_kv, d->d, d->n_q, d->n_k);
  CHECK(!need || ws, FF_E_NULL, "ws is NULL");
  CHECK(ws_bytes >= need, FF_E_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, need);
  const void* ps[] = {q, k, v, bias, pos, spans, out, need ? ws : nullptr};
  for (const void* p : ps) CHECK(!p || aligned16(p), FF_E_SHAPE, "pointers must be 16-byte aligned");
  const int es = (int)dsize(d->dtype);
  const int64_t table = d->bias_kind == FF_BIAS_TABLE ? (int64_t)d->H * (2 * (int64_t)d->bias_reach + 1) : d->bias_kind == FF_BIAS_SLOPE ? d->H : 0;
  const Extent in[6] = {attn_extent(q, d->B, d->q_batch, d->n_q, d->q_row, d->H, d->q_head, d->d, es),
                        attn_extent(k, d->B, d->k_batch, d->n_k, d->k_row, d->H_kv, d->k_head, d->d, es),
                        attn_extent(v, d->B, d->v_batch, d->n_k, d->v_row, d->H_kv, d->v_head, d->d, es),
                        {(const char*)bias, (wide)table * 4, 0, 0}, {(const char*)pos, (wide)d->B * 4, 0, 0},
                        rows_of(spans, d->n_spans ? d->B : 0, (int64_t)d->n_q * d->n_spans * 2, d->span_batch, 4)};
  const Extent eo = attn_extent(out, d->B, d->o_batch, d->n_q, d->o_row, d->H, d->o_head, d->d, es), ew{(const char*)ws, (wide)need, 0, 0};
  for (const Extent& x : in) {
    CHECK(!eo.meets(x), FF_E_SHAPE, "out overlaps an input");
    CHECK(!ew.meets(x), FF_E_SHAPE, "the workspace overlaps an input");
  }
  CHECK(!eo.meets(ew), FF_E_SHAPE, "out overlaps the workspace");
  const AttnSpanArgs a{q, k, v, out, d->q_batch, d->q_row, d->q_head, d->k_batch, d->k_row, d->k_head, d->v_batch, d->v_row,
                       d->v_head, d->o_batch, d->o_row, d->o_head, d->B, d->H_kv, d->H / d->H_kv, d->d, d->n_q, d->n_k,
                       d->scale, d->cap, d->bias_kind, d->bias_reach, bias, pos, spans, d->n_spans, d->span_batch, 0, 0,
                       need ? (float*)ws : nullptr};
  HIP_TRY(attention_span(d->dtype, a, reinterpret_cast<hipStream_t>(stream)), "attention over spans");
  return ok();
}

}  // extern "C"
