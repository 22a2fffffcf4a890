"""Plain 64-bit forms of the operators on 8-bit operands and of attention over spans, with the
tolerances of their tests (derived beside each), and helpers around the calls."""
import math

import torch

from paper_2607_27842_amd import abi

E4M3 = torch.float8_e4m3fn
TINY = 2.0 ** -100
U = 2.0 ** -24                                   # half a step of fp32
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
CODE = {torch.float32: abi.FF_F32, torch.bfloat16: abi.FF_BF16}


def ptr(t):
    return t.data_ptr() if t is not None else None


def stream():
    return torch.cuda.current_stream().cuda_stream


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(shape, g, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, dtype=torch.float64) * std).to(dtype)


def close(got, ref, tol, what=""):
    """|got - ref| <= tol elementwise (tensors in 64 bits), NaN and infinities in the same places."""
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, (got.shape, ref.shape)
    odd = ~torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what + ": NaN elsewhere"
    assert torch.equal(got[odd & ~torch.isnan(ref)], ref[odd & ~torch.isnan(ref)]), what
    d = (got - ref).abs()
    bad = (d > tol) & ~odd
    assert not bad.any(), "%s: %d of %d off, worst %g at tolerance %g" % (
        what, int(bad.sum()), bad.numel(), float((d / tol)[bad].max()), float(tol.expand_as(d)[bad].max() if torch.is_tensor(tol) else tol))


# ------------------------------------------------------------------ 8-bit format

def quantise(x, block_rows):
    """(e4m3 values, scales [row blocks, column blocks]) of an fp32 matrix: the format's formula in IEEE
    fp32, which the kernels compute with the same roundings, so that both agree bit for bit."""
    x = x.float()
    r, C = x.shape
    nb, nr = -(-C // 128), -(-r // block_rows)
    p = torch.nn.functional.pad(x.abs().nan_to_num(nan=0.0, posinf=math.inf), (0, nb * 128 - C, 0, nr * block_rows - r))
    s = p.view(nr, block_rows, nb, 128).amax((1, 3)).clamp_min(TINY) / torch.tensor(448.0)
    inv = (torch.tensor(1.0) / s).repeat_interleave(block_rows, 0)[:r].repeat_interleave(128, 1)[:, :C]
    return (x * inv).to(E4M3), s


def spread(s, block_rows, rows, C):
    return s.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :C]


# ------------------------------------------------------------------ product

def gemm_ref(a, a_s, w, w_s, bias, gelu, resid, dtype):
    """a [M, K] e4m3, a_s [blocks, M], w [N, K], w_s [row blocks, blocks]; CPU.  Returns the result and its
    tolerance.  fp32 outputs: exact products, then at most one rounding (2^-23, a truncation) of the
    running sum for each of a block's 128 additions, one for each block and four behind it, each at
    most 2^-23 of the sum of magnitudes S.  bf16 outputs: the 8-bit MFMAs align the products of a
    block to fewer bits; measured on random codes, a block's sum is off by at most 2^-11 of its
    largest product, taken here as 2^-10; and the rounding of the result, 2^-8 of it.  GELU and the
    residual's addition: their slopes are at most 1.13 and 1; GELU's own arithmetic 2^-20 of |x|."""
    M, K = a.shape
    N = w.shape[0]
    A, W = a.double(), w.double()
    y = torch.zeros(M, N, dtype=torch.float64)
    S, top = torch.zeros_like(y), torch.zeros_like(y)
    for j in range(-(-K // 128)):
        at = slice(128 * j, 128 * j + 128)
        sc = a_s[j].double()[:, None] * w_s[:, j].double().repeat_interleave(128)[:N]
        y += (A[:, at] @ W[:, at].t()) * sc
        S += (A[:, at].abs() @ W[:, at].abs().t()) * sc.abs()
        top += A[:, at].abs().amax(1)[:, None] * W[:, at].abs().amax(1)[None] * sc.abs()
    tol = (128 + -(-K // 128) + 4) * 2.0 ** -23 * S
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -10 * top
    if bias is not None:
        y = y + bias.double()
        tol = tol + U * y.abs()
    if gelu:
        tol = 1.13 * tol + 2.0 ** -20 * y.abs()
        y = y * 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    if resid is not None:
        y = y + resid.double()
    return y, tol + (HALF[dtype] + U) * (y.abs() + tol)


def gemm_call(a, a_s, w, w_s, bias=None, gelu=False, resid=None, dtype=torch.bfloat16, out=None, N=None, st=None, ws=None):
    """Tensors on the GPU; out may be a strided view."""
    M, K = a.shape
    N = w.shape[0]
    out = torch.empty(M, N, dtype=dtype, device="cuda") if out is None else out
    d = abi.ff_gemm_q8_desc(M=M, N=N, K=K, out_dtype=CODE[dtype], gelu=int(gelu), a_row=a.stride(0), w_row=w.stride(0),
                            out_row=out.stride(0), resid_row=resid.stride(0) if resid is not None else 0,
                            as_ld=a_s.stride(0), ws_ld=w_s.stride(0))
    n = abi.ff_gemm_q8_workspace_bytes(d)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda") if ws is None else ws
    abi.ff_gemm_q8(d, ptr(a), ptr(a_s), ptr(w), ptr(w_s), ptr(bias), ptr(resid), ptr(out), ptr(ws), n, stream() if st is None else st)
    return out


# ------------------------------------------------------------------ attention

def attention_ref(q, k, v, scale, cap=0.0, bias_kind=abi.FF_BIAS_NONE, bias=None, reach=0, pos=None, spans=None):
    """q [B, nq, H, d], k and v [B, nk, Hkv, d] on the CPU; spans [B, nq, s, 2].  Returns the result and its
    tolerance.  A score's error: the dot product's (d + 2) roundings of fp32 at the sum of magnitudes,
    three more at the score's own size (scale, bias, log2 units), tanh's 2^-19 of the cap; e^t moves
    by twice that, its own error is 2^-20; each probability's rounding is 2^-8 in bf16; the row sums'
    roundings are at most nk 2^-24 (numerator and denominator); all relative to sum p |v|."""
    dt = q.dtype
    B, nq, H, d = q.shape
    nk, G = k.shape[1], H // k.shape[2]
    out = torch.zeros(B, nq, H, d, dtype=torch.float64)
    tol = torch.zeros(B, nq, H, d, dtype=torch.float64)
    j = torch.arange(nk)
    for b in range(B):
        seen = torch.ones(nq, nk, dtype=torch.bool)
        if spans is not None:
            seen.zero_()
            for sp in spans[b if spans.shape[0] > 1 else 0].long().unbind(1):
                seen |= (j >= sp[:, :1]) & (j < sp[:, 1:])
        dist = j[None] - (torch.arange(nq) + (int(pos[b]) if pos is not None else 0))[:, None]
        for h in range(H):
            Q, Kk, V = q[b, :, h].double(), k[b, :, h // G].double(), v[b, :, h // G].double()
            t = (Q @ Kk.t()) * scale
            dt_ = (Q.abs() @ Kk.abs().t()) * scale * (d + 2) * U
            if cap:
                t = cap * torch.tanh(t / cap)
                dt_ = dt_ + cap * 2.0 ** -19
            if bias_kind == abi.FF_BIAS_SLOPE:
                t = t - bias[h].double() * dist.abs()
                dt_ = dt_ + (bias[h].double() * dist.abs()).abs() * 2 * U
            elif bias_kind == abi.FF_BIAS_TABLE:
                t = t + bias[h].double()[dist.clamp(-reach, reach) + reach]
            # scores are fp32: where a table's entry swallows the product, it does so in fp32
            t = torch.where(t.abs() > 1e30, t.float().double(), t)
            t = t.masked_fill(~seen, -math.inf)
            m = t.amax(1, keepdim=True)
            m0 = torch.where(torch.isinf(m) & (m < 0), 0.0, m)
            p = torch.exp(t - m0)
            l = p.sum(1, keepdim=True)
            p = torch.where(l == 0, 0.0, p / l)
            Vs = torch.where(seen.any(0)[:, None], V, 0.0)
            # a key that a query does not see has no effect on it, whatever its row holds
            o = torch.where(torch.isfinite(Vs), Vs, 0.0)
            o = p @ o
            for kk in torch.nonzero(~torch.isfinite(Vs).all(1))[:, 0].tolist():
                bad = ~torch.isfinite(Vs[kk])
                o += torch.where(seen[:, kk][:, None] & bad[None], Vs[kk][None], 0.0)
            out[b, :, h] = o
            fin = torch.where(torch.isfinite(Vs), Vs, 0.0).abs()
            near = seen & torch.isfinite(t) & (t.abs() < 1e30)
            e = torch.where(near, dt_ + 3 * U * t.abs(), 0.0).amax(1, keepdim=True)
            rel = 2.2 * e + 2.0 ** -20 + nk * U + (2.0 ** -8 if dt == torch.bfloat16 else 0.0)
            x = rel * (torch.nan_to_num(p) @ fin)
            tol[b, :, h] = x + (HALF[dt] + U) * (torch.nan_to_num(o, posinf=0.0, neginf=0.0).abs() + x) + 1e-30
    return out, tol


def attn_desc(q, k, v, out, scale, cap=0.0, bias_kind=abi.FF_BIAS_NONE, reach=0, spans=None, **over):
    st = {}
    for n, t in (("q", q), ("k", k), ("v", v), ("o", out)):
        for i, w in enumerate(("batch", "row", "head")):
            st["%s_%s" % (n, w)] = t.stride(i)
    return abi.ff_attn_desc(**{**dict(
        dtype=CODE[q.dtype], B=q.shape[0], H=q.shape[2], H_kv=k.shape[2], d=q.shape[3], n_q=q.shape[1], n_k=k.shape[1], **st,
        scale=scale, cap=cap, bias_kind=bias_kind, bias_reach=reach, n_spans=spans.shape[2] if spans is not None else 0,
        span_batch=spans.stride(0) if spans is not None and spans.shape[0] > 1 else 0), **over})


def attention_call(q, k, v, scale, cap=0.0, bias_kind=abi.FF_BIAS_NONE, bias=None, reach=0, pos=None, spans=None, out=None,
                   st=None, ws=None):
    """Tensors on the GPU, any strides."""
    out = torch.empty(q.shape, dtype=q.dtype, device="cuda") if out is None else out
    d = attn_desc(q, k, v, out, scale, cap, bias_kind, reach, spans)
    n = abi.ff_attention_workspace_bytes(d)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda") if ws is None else ws
    abi.ff_attention(d, ptr(q), ptr(k), ptr(v), ptr(bias), ptr(pos), ptr(spans), ptr(out), ptr(ws), n, stream() if st is None else st)
    return out
