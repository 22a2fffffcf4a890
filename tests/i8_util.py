"""Plain 64-bit forms of the operators on 8-bit integers, with the tolerances of their tests (derived beside each),
and helpers around the calls."""
import math

import torch

import op_util as O
from paper_2607_27842_amd import abi

BF, F32 = torch.bfloat16, torch.float32
U, HALF, CODE = O.U, O.HALF, O.CODE
TINY = 2.0 ** -100
STEP = torch.tensor(1.0 / 127.0)                 # fp32
KINDS = {"none": abi.FF_NORM_NONE, "rms": abi.FF_NORM_RMS, "layer": abi.FF_NORM_LAYER}


def quantise(x):
    """(whole values, scales) along the last axis: the format's formula in IEEE fp32, which the kernels compute
    with the same roundings, so that both agree bit for bit."""
    x = x.float()
    odd = ~torch.isfinite(x).all(-1)
    s = torch.where(odd, 0.0, x.abs().nan_to_num(nan=0.0, posinf=0.0).amax(-1)).clamp_min(TINY) * STEP
    q = torch.round(x * (torch.tensor(1.0) / s)[..., None])
    return torch.where(odd[..., None], 0.0, q).to(torch.int8), torch.where(odd, math.nan, s)


# ------------------------------------------------------------------ product

def gelu(y):
    return y * 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))


def gemm_ref(a, a_s, w, w_s, bias=None, act=False, gate=None, gate_rows=1, resid=None, dtype=BF):
    """CPU tensors; the result and its tolerance.  The sum of products is exact; its conversion and the two scales round
    three times, bias, gate and residual once each (U of what they give); GELU's slope is at most 1.13 and its own
    arithmetic 2^-20 of |x|; the output's rounding is half a step."""
    y = (a.double() @ w.double().t()) * a_s.double()[:, None] * w_s.double()
    tol = 3.1 * U * y.abs()
    if bias is not None:
        y = y + bias.double()
        tol = tol + U * y.abs()
    if act:
        tol = 1.13 * tol + 2.0 ** -20 * y.abs()
        y = gelu(y)
    if gate is not None:
        g = gate.double()[torch.arange(a.shape[0]) // gate_rows]
        y = y * g
        tol = tol * g.abs() + U * y.abs()
    if resid is not None:
        y = y + resid.double()
        tol = tol + U * y.abs()
    return y, tol + (HALF[dtype] + U) * (y.abs() + tol) + 1e-44


def gemm_desc(a, w, out, gelu=0, gate=None, gate_rows=1, resid=None):
    return abi.ff_gemm_i8_desc(M=a.shape[0], N=w.shape[0], K=a.shape[1], a_dtype=abi.FF_I8 if a.dtype == torch.int8 else CODE[a.dtype],
                               out_dtype=CODE[out.dtype], gelu=int(gelu), gate_rows=gate_rows, a_row=a.stride(0), w_row=w.stride(0),
                               out_row=out.stride(0), resid_row=resid.stride(0) if resid is not None else 0,
                               gate_ld=gate.stride(0) if gate is not None else 0)


def gemm_call(a, a_s, w, w_s, bias=None, act=False, gate=None, gate_rows=1, resid=None, dtype=BF, out=None, st=None, ws=None):
    """Tensors on the GPU; a int8 with a_s, or in a float type with None."""
    out = torch.empty(a.shape[0], w.shape[0], dtype=dtype, device="cuda") if out is None else out
    d = gemm_desc(a, w, out, act, gate, gate_rows, resid)
    n = abi.ff_gemm_i8_workspace_bytes(d)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda") if ws is None else ws
    assert ws.numel() >= n
    abi.ff_gemm_i8(d, O.ptr(a), O.ptr(a_s), O.ptr(w), O.ptr(w_s), O.ptr(bias), O.ptr(gate), O.ptr(resid), O.ptr(out), O.ptr(ws), n,
                   O.stream() if st is None else st)
    return out


def quant_call(x, q=None, s=None, st=None):
    q = torch.empty(x.shape, dtype=torch.int8, device="cuda") if q is None else q
    s = torch.empty(x.shape[0], device="cuda") if s is None else s
    d = abi.ff_quant_i8_desc(rows=x.shape[0], C=x.shape[1], dtype=CODE[x.dtype], x_row=x.stride(0), q_row=q.stride(0))
    abi.ff_quant_i8(d, O.ptr(x), O.ptr(q), O.ptr(s), O.stream() if st is None else st)
    return q, s


# ------------------------------------------------------------------ between branches

def norm_ref(v, kind, eps):
    """v normed, and its error: sums over a row carry at most 22 roundings of a lane's and the wavefronts' additions,
    taken as 26 (52 halved by the root for the mean of squares), and up to six more follow; a mean is off by 26 U of
    the mean magnitude."""
    if kind == "none":
        return v, torch.zeros_like(v)
    mean = v.mean(1, keepdim=True) if kind == "layer" else 0.0
    off = 26 * U * v.abs().mean(1, keepdim=True) if kind == "layer" else 0.0
    c = v - mean
    inv = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    # the mean's error moves every value, and by their sum of squares the root
    return c * inv, 2.0 ** -19 * (c * inv).abs() + (off + U * v.abs()) * inv * (1 + (c * inv).abs())


def branch_t_ref(x, branch, post, post_gain, gate, tanh, rs, eps):
    """t before its rounding (CPU, [rows, C], gate per row), and its error; tanh of the hardware exponential and
    reciprocal: 2^-20."""
    z, e = torch.zeros_like(x, dtype=torch.float64), 0.0
    if branch is not None:
        z, e = norm_ref(branch.double(), post, eps)
        if post_gain is not None:
            z, e = z * post_gain.double(), e * post_gain.double().abs()
        if gate is not None:
            g = torch.tanh(gate.double()) if tanh else gate.double()
            z, e = z * g, e * g.abs() + (2.0 ** -20 if tanh else 0.0) * (z * g).abs()
    t = rs * x.double() + z
    return t, e + 4 * U * (z.abs() + (rs * x.double()).abs())


def branch_v_ref(t, pre, pre_gain, scale, shift, eps):
    v, e = norm_ref(t.double(), pre, eps)
    if pre_gain is not None:
        v, e = v * pre_gain.double(), e * pre_gain.double().abs()
    if scale is not None:
        m = 1 + scale.double()
        v, e = v * m, e * m.abs() + U * (v * m).abs() + U * v.abs()
    e = e + 3 * U * v.abs()
    if shift is not None:
        v = v + shift.double()
        e = e + U * v.abs()
    return v, e


def branch_call(x, branch=None, post="none", post_gain=None, gate=None, tanh=False, pre="none", pre_gain=None, scale=None, shift=None,
                mod_rows=1, rs=1.0, eps=1e-6, sum=None, y=None, q=None, q_s=None, st=None):
    p = lambda t: t.stride(0) if t is not None else 0  # noqa: E731
    v = lambda t: t.stride(0) if t is not None and t.shape[0] > 1 else 0  # noqa: E731
    d = abi.ff_branch_norm_desc(rows=x.shape[0], C=x.shape[1], dtype=CODE[x.dtype], post=KINDS[post], pre=KINDS[pre], gate_tanh=int(tanh),
                                mod_rows=mod_rows, eps=eps, resid_scale=rs, x_row=p(x), branch_row=p(branch), sum_row=p(sum), y_row=p(y),
                                q_row=p(q), gate_ld=v(gate), mod_ld=max(v(scale), v(shift)))
    abi.ff_branch_norm_i8(d, *(O.ptr(t) for t in (x, branch, post_gain, gate, pre_gain, scale, shift, sum, y, q, q_s)),
                          O.stream() if st is None else st)


def close_q(q, s, v, e):
    """8-bit rows against v: a scale is off by as much as the largest value and three roundings, a value by half a
    step and e (and the few roundings of the product with 1 / s)."""
    top = v.abs().amax(1)
    worst = (e.amax(1) if torch.is_tensor(e) else e) + 4 * U * top
    ref = top.clamp_min(TINY) / 127
    O.close(s, ref, worst / 127 + 2 * U * ref, "scales")
    S = s.cpu().double()[:, None]
    O.close(q.cpu().double() * S, v, 0.5 * S * (1 + 2.0 ** -14) + e, "q")


# ------------------------------------------------------------------ history

def model(B, N, C, dtype, layers=1):
    """A model of `layers` blocks on a stream [B, N, C]."""
    import ctypes
    return abi.ff_model_desc(n_layers=layers, kinds=(ctypes.c_int32 * layers)(*[abi.FF_DIT] * layers), C=C, H=C // 8, d=8, mlp_hidden=64,
                             n_img=N, n_txt=0, B=B, lat_c=8, lat_f=1, lat_h=1, lat_w=N, pt=1, ph=1, pw=1, dtype=CODE[dtype], ln_eps=1e-6)


def blocks(x):
    """[B, blocks, 128] of a [B, N, C] tensor, padded with zeros."""
    B, n = x.shape[0], x[0].numel()
    nb = -(-n // 128)
    return torch.nn.functional.pad(x.reshape(B, n), (0, nb * 128 - n)).view(B, nb, 128)


def slot_bytes(B, N, C):
    nb = -(-N * C // 128)
    return -(-B * nb * 132 // 128) * 128


def slot_views(cache, i, B, N, C):
    nb, size = -(-N * C // 128), slot_bytes(B, N, C)
    at = cache[i * size:(i + 1) * size]
    q = at[:B * nb * 128].view(torch.int8).view(B, nb, 128)
    return q, at[B * nb * 128:B * nb * 132].view(F32).view(B, nb)
