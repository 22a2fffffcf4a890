"""Quantisation to 8-bit integers, products on them and the step between two branches, against their plain
64-bit forms."""
import math

import pytest
import torch

import i8_util as I
import op_util as O
from gpu_util import need_gpu, say
from paper_2607_27842_amd import abi
from test_gpu_operators_q8 import guarded, untouched

pytestmark = pytest.mark.gpu
BF, F32, I8 = torch.bfloat16, torch.float32, torch.int8
TYPES = pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])


def rows_like(rows, C, g, dtype=F32):
    return (O.randn((rows, C), g) * torch.exp(0.5 * O.randn((1, C), g))).to(dtype)


# ------------------------------------------------------------------ quantisation

@TYPES
@pytest.mark.parametrize("rows,C,pad", [(1, 8, 0), (1, 2048, 0), (3, 136, 24), (17, 1480, 8), (2, 4096, 0), (5, 8200, 16), (2, 16384, 0),
                                        (2, 16400, 40), (1, 131056, 0), (1025, 264, 8), (1500, 1032, 0), (1030, 2048, 0),
                                        (6500, 72, 0), (3200, 600, 8), (1700, 1480, 0), (1600, 2056, 0), (800, 4104, 8), (390, 8200, 0)])
def test_quant_bit_for_bit(dtype, rows, C, pad):
    """Same formula, same IEEE roundings: values and scales are equal."""
    need_gpu()
    g = O.gen(rows * 7 + C)
    x = rows_like(rows, C, g)
    x[:, :8] *= torch.tensor([0.0, 1e-38, 1e30, 2.0 ** -140, -448.0, 1.0, 1.0, 1.0])
    x[rows // 2] = 0.0
    x[rows // 3, C - 1] = 2.0 ** -110
    x = x.to(dtype)
    q, s = I.quantise(x)
    dx, _ = guarded(rows, C, C + pad, dtype)
    dx.copy_(x)
    dq = torch.full((rows * (C + pad) + 64,), 0x55, dtype=I8, device="cuda")
    ds = torch.full((rows + 4,), 77.0, device="cuda")
    I.quant_call(dx, dq[:rows * (C + pad)].view(rows, C + pad)[:, :C], ds[:rows])
    assert torch.equal(ds[:rows].cpu(), s) and (ds[rows:] == 77.0).all()
    b = dq[:rows * (C + pad)].view(rows, C + pad)
    assert torch.equal(b[:, :C].cpu(), q) and (b[:, C:] == 0x55).all() and (dq[rows * (C + pad):] == 0x55).all()


@TYPES
def test_quant_ties_go_to_even(dtype):
    """Halves between integers under a scale of one (to a rounding)."""
    need_gpu()
    x = torch.arange(-63, 64).float().add(0.5).repeat(2)[:248].view(1, 248)
    x = torch.cat([x, torch.tensor([[127.0] + [0.0] * 7])], 1).to(dtype)
    q, s = I.quantise(x)
    dq, ds = I.quant_call(x.cuda())
    assert torch.equal(dq.cpu(), q) and torch.equal(ds.cpu(), s)


def test_quant_nan_and_infinity():
    """They make a row's scale NaN and its integers zeros; other rows are as ever."""
    need_gpu()
    for C in (264, 2048, 20000):
        x = O.randn((6, C), O.gen(1))
        x[1, C - 1], x[2, 5], x[4, C // 2] = math.nan, math.inf, -math.inf
        q, s = I.quantise(x)
        dq, ds = I.quant_call(x.cuda())
        assert torch.equal(dq.cpu(), q)
        assert torch.equal(torch.isnan(ds).cpu(), torch.isnan(s)) and torch.isnan(s).sum() == 3
        assert torch.equal(ds.cpu().nan_to_num(0.0), s.nan_to_num(0.0))


# ------------------------------------------------------------------ products

def operands(M, N, K, g, pads=(0, 0), full=False):
    """8-bit operands on the CPU and the GPU, rows at a longer pitch with large values between them."""
    if full:   # any byte, -128 among them
        a, w = (torch.randint(-128, 128, s, generator=g).to(I8) for s in ((M, K), (N, K)))
        a_s, w_s = torch.exp(O.randn((M,), g)), torch.exp(O.randn((N,), g))
    else:
        a, a_s = I.quantise(rows_like(M, K, g))
        w, w_s = I.quantise(O.randn((N, K), g, std=1 / math.sqrt(K)) * torch.exp(O.randn((N, 1), g)))
    da = torch.full((M, K + pads[0]), 127, dtype=I8, device="cuda")
    dw = torch.full((N, K + pads[1]), 127, dtype=I8, device="cuda")
    da[:, :K] = a.cuda()
    dw[:, :K] = w.cuda()
    return (a, a_s, w, w_s), (da[:, :K], a_s.cuda(), dw[:, :K], w_s.cuda())


# every kernel and split, odd rows, N and K off every tile, K shorter than a block, one, two and three blocks
SHAPES = [(1, 8, 16), (1, 2048, 8192), (1, 520, 4112), (2, 24, 144), (16, 136, 272), (17, 72, 128), (33, 1160, 1152), (63, 264, 400),
          (64, 2048, 2064), (100, 1480, 4608), (130, 2056, 8192), (200, 1160, 2960), (257, 6152, 400), (300, 72, 48),
          (520, 2056, 1168), (1003, 1480, 2960), (1100, 2048, 256), (5000, 2600, 400), (4700, 2312, 2064), (9, 40, 131056), (300, 72, 65552)]


@TYPES
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_against_64_bits(dtype, M, N, K):
    need_gpu()
    g = O.gen(M + N + K)
    h, d = operands(M, N, K, g, (16, 48), full=True)
    out, base = guarded(M, N, N + 8, dtype)
    I.gemm_call(*d, dtype=dtype, out=out)
    ref, tol = I.gemm_ref(*h, dtype=dtype)
    O.close(out, ref, tol, "gemm")
    untouched(base, M, N, N + 8)


@TYPES
@pytest.mark.parametrize("M,K", [(1, 131056), (300, 131056), (2200, 2064)])
def test_gemm_sums_at_the_limit(dtype, M, K):
    """Products of the largest magnitude, all of one sign: 131056 * 128 * 128 is the largest sum there is."""
    need_gpu()
    N = 72 if M < 1000 else 2056
    a, w = torch.full((M, K), -128, dtype=I8), torch.full((N, K), -128, dtype=I8)
    w[1] = 127
    one = torch.ones(M), torch.ones(N)
    got = I.gemm_call(a.cuda(), one[0].cuda(), w.cuda(), one[1].cuda(), dtype=dtype).cpu().double()
    want = torch.full((M, N), K * 16384.0, dtype=torch.float64)
    want[:, 1] = K * -128.0 * 127
    assert ((got - want).abs() <= O.HALF[dtype] * want.abs()).all()


@TYPES
@pytest.mark.parametrize("bias,act,gate,resid", [(1, 0, 0, 0), (0, 1, 0, 0), (1, 1, 0, 0), (0, 0, 3, 0), (1, 0, 7, 1), (1, 1, 1, 1), (0, 0, 0, 1)])
@pytest.mark.parametrize("M,N,K", [(5, 200, 272), (130, 2056, 8192), (600, 520, 528), (4500, 2568, 400)])
def test_gemm_epilogues(dtype, bias, act, gate, resid, M, N, K):
    """gate: how many vectors, at a longer pitch."""
    need_gpu()
    g = O.gen(M)
    h, d = operands(M, N, K, g)
    b = O.randn((N,), g, dtype) if bias else None
    r = O.randn((M, N), g, dtype) if resid else None
    per = -(-M // gate) if gate else 1
    v = O.randn((-(-M // per), N + 24), g)[:, :N] if gate else None
    dr = r.cuda() if resid else None
    dv = torch.full((v.shape[0], N + 24), math.nan, device="cuda")[:, :N].copy_(v) if gate else None
    got = I.gemm_call(*d, b.cuda() if bias else None, act, dv, per, dr, dtype, dr if resid else None)   # the residual in place
    ref, tol = I.gemm_ref(*h, b, act, v, per, r, dtype)
    O.close(got, ref, tol, "gemm")


def test_gemm_one_gate_for_all_rows():
    need_gpu()
    g = O.gen(8)
    for M, N, K in ((5, 200, 272), (600, 520, 528)):
        h, d = operands(M, N, K, g)
        v = O.randn((1, N), g)
        out = torch.empty(M, N, device="cuda")
        desc = I.gemm_desc(d[0], d[2], out, gate=v, gate_rows=2)
        desc.gate_ld = 0
        n = abi.ff_gemm_i8_workspace_bytes(desc)
        ws, dv = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"), v.cuda()
        abi.ff_gemm_i8(desc, *(O.ptr(t) for t in (*d, None, dv, None, out, ws)), n, O.stream())
        ref, tol = I.gemm_ref(*h, gate=v, gate_rows=M, dtype=F32)
        O.close(out, ref, tol, "gate")


@TYPES
@pytest.mark.parametrize("of", [BF, F32], ids=["rows_bf16", "rows_fp32"])
@pytest.mark.parametrize("M,N,K", [(1, 8, 16), (1, 8200, 2048), (1, 520, 16384), (2, 264, 8192), (4, 200, 272), (16, 520, 1040), (17, 264, 2064),
                                   (130, 2056, 8192), (600, 520, 528), (1100, 1160, 2064), (4500, 2568, 400)])
def test_gemm_of_rows_in_a_float_type(dtype, of, M, N, K):
    """The same bits as quantising the rows and multiplying them."""
    need_gpu()
    g = O.gen(M + 2 * K)
    x = torch.full((M, K + 8), math.inf, dtype=of, device="cuda")[:, :K].copy_(rows_like(M, K, g, of))
    w, w_s = I.quantise(O.randn((N, K), g, std=1 / math.sqrt(K)))
    b, r = O.randn((N,), g, dtype).cuda(), O.randn((M, N), g, dtype).cuda()
    dw, ds = w.cuda(), w_s.cuda()
    got = I.gemm_call(x, None, dw, ds, b, True, None, 1, r, dtype)
    q, s = I.quant_call(x)
    want = I.gemm_call(q, s, dw, ds, b, True, None, 1, r, dtype)
    assert torch.equal(got, want)
    ref, tol = I.gemm_ref(*I.quantise(x.cpu()), w, w_s, b.cpu(), True, None, 1, r.cpu(), dtype)
    O.close(got, ref, tol, "linear")


@pytest.mark.parametrize("of", [I8, BF, F32], ids=["i8", "bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(1, 520, 272), (5, 520, 2064), (130, 1160, 8192), (700, 520, 272), (4500, 2568, 400)])
def test_gemm_rows_are_apart(of, M, N, K):
    """A NaN reaches its row of A (by the row's scale, or in the row), one in a weight's scale its column; an all-zero row
    gives zeros."""
    need_gpu()
    g = O.gen(M + 1)
    h, d = operands(M, N, K, g)
    d[3][N - 1] = math.nan
    want = torch.zeros(M, N, dtype=torch.bool)
    want[M // 2] = True
    want[:, N - 1] = True
    if of == I8:
        d[1][M // 2] = math.nan
        d[0][0] = 0
        got = I.gemm_call(*d)
    else:
        x = (h[0].float() * h[1][:, None]).to(of).cuda()
        x[0] = 0.0
        x[M // 2, K - 1] = math.nan
        got = I.gemm_call(x, None, d[2], d[3])
    assert torch.equal(torch.isnan(got).cpu(), want)
    if M > 1:
        assert (got[0, :N - 1] == 0).all()


@pytest.mark.parametrize("M,N,K", [(5, 200, 272), (130, 1096, 528), (4500, 2568, 400)])
def test_gemm_into_other_columns(M, N, K):
    """The output beside its residual in one buffer, whose other columns stay."""
    need_gpu()
    g = O.gen(M + 1)
    h, d = operands(M, N, K, g)
    r = O.randn((M, 2 * N + 8), g, BF)
    buf = r.cuda()
    I.gemm_call(*d, resid=buf[:, :N], out=buf[:, N:2 * N])
    ref, tol = I.gemm_ref(*h, resid=r[:, :N])
    O.close(buf[:, N:2 * N], ref, tol, "gemm")
    assert torch.equal(buf[:, :N].cpu(), r[:, :N]) and torch.equal(buf[:, 2 * N:].cpu(), r[:, 2 * N:])


def test_gemm_same_bits_again_and_on_another_stream():
    need_gpu()
    for M, N, K, dt in ((3, 520, 4096, BF), (130, 2056, 8192, F32), (700, 1160, 1168, BF), (4500, 2568, 400, BF)):
        _, d = operands(M, N, K, O.gen(9))
        a = I.gemm_call(*d, dtype=dt)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b = I.gemm_call(*d, dtype=dt)
            c = I.gemm_call(*d, dtype=dt)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(a, b) and torch.equal(b, c)


def test_gemm_offsets_past_32_bits():
    """Output rows and operand tiles more than 2^32 bytes apart."""
    need_gpu()
    g = O.gen(4)
    M, N, K, pitch = 600, 136, 256, (8 << 20) - 4096    # 600 rows of 8 MB: 4.7 GiB
    h, _ = operands(M, N, K, g)
    da = torch.empty(M * pitch, dtype=I8, device="cuda").view(M, pitch)
    da[:, :K] = h[0].cuda()
    out = torch.empty(M * (pitch // 2), dtype=BF, device="cuda").view(M, pitch // 2)
    I.gemm_call(da[:, :K], h[1].cuda(), h[2].cuda(), h[3].cuda(), out=out[:, :N])
    ref, tol = I.gemm_ref(*h)
    O.close(out[:, :N].contiguous(), ref, tol, "far rows")
    x = da.view(torch.bfloat16)[:, :K]   # rows in a float type, as far apart
    y = rows_like(M, K, g, BF)
    x.copy_(y)
    got = I.gemm_call(x, None, h[2].cuda(), h[3].cuda())
    ref, tol = I.gemm_ref(*I.quantise(y), h[2], h[3])
    O.close(got, ref, tol, "far rows, bf16")


# ------------------------------------------------------------------ between branches

WIDTHS = [(1, 8, 1), (1, 2048, 1), (5, 136, 2), (7, 520, 3), (3, 1032, 3), (6, 1480, 4), (9, 4096, 3), (2, 8200, 1), (3, 16384, 2),
          (1025, 256, 1000), (1500, 1032, 7), (1027, 2048, 400),
          # more rows than there are walks, samples that end between a walk's rows
          (6500, 264, 1250), (3200, 600, 999), (1700, 2048, 400), (800, 2056, 100), (700, 4104, 9), (400, 8200, 1)]


@TYPES
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), ("none", "layer"), ("rms", "none")])
@pytest.mark.parametrize("rows,C,per", WIDTHS)
def test_branch_against_64_bits(dtype, post, pre, rows, C, per):
    """Every part, samples of `per` rows, every buffer at a pitch of its own."""
    need_gpu()
    g = O.gen(rows + C)
    x, z = rows_like(rows, C, g, dtype), (0.3 + rows_like(rows, C, g)).to(dtype)
    gains = [(1 + 0.1 * O.randn((C,), g)).to(dtype) for _ in range(2)]
    B = -(-rows // per)
    mod = O.randn((B, 3 * C + 8), g, std=0.4)
    gate, scale, shift = mod[:, :C], mod[:, C:2 * C], mod[:, 2 * C:3 * C]
    dm = mod.cuda()
    dx, _ = guarded(rows, C, C + 8, dtype)
    dz, _ = guarded(rows, C, C + 16, dtype)
    t, tb = guarded(rows, C, C + 24, dtype)
    y, yb = guarded(rows, C, C + 32, dtype)
    dx.copy_(x)
    dz.copy_(z)
    q = torch.full((rows, C + 40), 0x55, dtype=I8, device="cuda")
    s = torch.full((rows + 4,), 77.0, device="cuda")
    tanh, rs = post == "rms", 0.875 if pre == "layer" else 1.0
    I.branch_call(dx, dz, post, gains[0].cuda() if post != "none" else None, dm[:, :C], tanh, pre, gains[1].cuda() if pre == "rms" else None,
                  dm[:, C:2 * C], dm[:, 2 * C:3 * C], per, rs, sum=t, y=y, q=q[:, :C], q_s=s[:rows])
    at = torch.arange(rows) // per
    ref, e = I.branch_t_ref(x, z, post, gains[0] if post != "none" else None, gate[at], tanh, rs, 1e-6)
    O.close(t, ref, e + (O.HALF[dtype] + O.U) * (ref.abs() + e) + 1e-44, "t")
    ref, e = I.branch_v_ref(t.cpu(), pre, gains[1] if pre == "rms" else None, scale[at], shift[at], 1e-6)
    O.close(y, ref, e + (O.HALF[dtype] + O.U) * (ref.abs() + e) + 1e-44, "y")
    I.close_q(q[:, :C].contiguous(), s[:rows], ref, e)
    untouched(tb, rows, C, C + 24)
    untouched(yb, rows, C, C + 32)
    assert (q[:, C:] == 0x55).all() and (s[rows:] == 77.0).all()


@TYPES
@pytest.mark.parametrize("rows,C", [(9, 264), (70, 2048), (1100, 1480)])
def test_branch_parts(dtype, rows, C):
    """Each part left out: the bits of the others stay, and what is left is the formula's."""
    need_gpu()
    g = O.gen(3)
    x, z, gain = (O.randn(s, g, dtype) for s in ((rows, C), (rows, C), (C,)))
    dx, dz, dg = x.cuda(), z.cuda(), gain.cuda()
    v = O.randn((1, C), g)
    dv = v.cuda()
    new = lambda t=dtype: torch.empty(rows, C, dtype=t, device="cuda")  # noqa: E731
    t, y, q, s = new(), new(), new(I8), torch.empty(rows, device="cuda")
    full = dict(branch=dz, post="rms", post_gain=dg, gate=dv, pre="layer", scale=dv, shift=dv, mod_rows=rows)
    I.branch_call(dx, **full, sum=t, y=y, q=q, q_s=s)
    for keep in ("sum", "y", "q"):                          # one output alone
        o = dict(sum=new() if keep == "sum" else None, y=new() if keep == "y" else None, q=new(I8) if keep == "q" else None,
                 q_s=torch.empty_like(s) if keep == "q" else None)
        I.branch_call(dx, **full, **o)
        assert torch.equal(o[keep], dict(sum=t, y=y, q=q)[keep])
        assert keep != "q" or torch.equal(o["q_s"], s)
    for into in ("x", "branch"):                            # the sum in either one's place
        a, b = dx.clone(), dz.clone()
        at, y2 = a if into == "x" else b, new()
        I.branch_call(a, **{**full, "branch": b}, sum=at, y=y2)
        assert torch.equal(at, t) and torch.equal(y2, y)
    for pre in ("none", "rms", "layer"):                    # no branch: a norm with modulation
        I.branch_call(dx, None, pre=pre, pre_gain=dg, scale=dv, shift=None, mod_rows=rows, sum=t, y=y)
        assert torch.equal(t, dx)
        ref, e = I.branch_v_ref(x, pre, gain, v, None, 1e-6)
        O.close(y, ref, e + (O.HALF[dtype] + O.U) * (ref.abs() + e) + 1e-44, pre)
        I.branch_call(dx, None, pre=pre, shift=dv, mod_rows=rows, y=y)
        ref, e = I.branch_v_ref(x, pre, None, None, v, 1e-6)
        O.close(y, ref, e + (O.HALF[dtype] + O.U) * (ref.abs() + e) + 1e-44, pre)
    I.branch_call(dx, dz, sum=t, rs=-2.0)                   # neither norm, no gate
    ref, e = I.branch_t_ref(x, z, "none", None, None, False, -2.0, 1e-6)
    O.close(t, ref, e + (O.HALF[dtype] + O.U) * (ref.abs() + e) + 1e-44, "sum")


def test_branch_gates():
    """tanh where it is near its argument, near one, and at its ends; a NaN gate stays in its column."""
    need_gpu()
    C = 64
    v = torch.tensor([0.0, 1e-30, -1e-6, 1e-3, 0.0624, 0.249, 0.25, -0.2501, 0.5, -1.0, 2.0, 5.0, 9.0, -30.0, 1e30, math.inf, -math.inf] +
                     [0.01 * i for i in range(C - 17)]).view(1, C)
    one = torch.ones(1, C)
    t = torch.empty(1, C, device="cuda")
    I.branch_call(torch.zeros(1, C, device="cuda"), one.cuda(), gate=v.cuda(), tanh=True, sum=t)
    ref = torch.tanh(v.double())
    O.close(t, ref, 2.0 ** -20 * ref.abs(), "tanh")
    v[0, 3] = math.nan
    I.branch_call(torch.zeros(1, C, device="cuda"), one.cuda(), gate=v.cuda(), tanh=True, sum=t)
    assert torch.isnan(t).cpu().nonzero().tolist() == [[0, 3]]


@TYPES
def test_branch_rows_are_apart_and_zeros(dtype):
    """A NaN or an infinity spoils its own row; rows of zeros give zeros (and the shift)."""
    need_gpu()
    for rows, C in ((6, 264), (6, 2048), (1030, 1480)):
        x, z = (O.randn((rows, C), O.gen(i), dtype).cuda() for i in (1, 2))
        x[1, 3], z[4, C - 1] = math.nan, math.inf
        x[2], z[2] = 0.0, 0.0
        t, y = torch.empty_like(x), torch.empty_like(x)
        q, s = torch.empty(rows, C, dtype=I8, device="cuda"), torch.empty(rows, device="cuda")
        I.branch_call(x, z, "rms", pre="layer", sum=t, y=y, q=q, q_s=s)
        ok = [i for i in range(rows) if i not in (1, 4)]
        assert torch.isfinite(y[ok].float()).all() and torch.isfinite(s[ok]).all()
        assert torch.isnan(s[[1, 4]]).all() and torch.isnan(y[[1, 4]].float()).all() and (q[[1, 4]] == 0).all()
        assert (t[2] == 0).all() and (y[2] == 0).all() and (q[2] == 0).all()


def test_branch_offsets_past_32_bits():
    need_gpu()
    rows, C, pitch = 1100, 64, 4 << 20    # 1100 rows of 8 MB apart
    g = O.gen(5)
    x, z = (O.randn((rows, C), g, BF) for _ in range(2))
    buf = torch.empty(rows * pitch, dtype=BF, device="cuda").view(rows, pitch)
    cut = [buf[:, i * C:(i + 1) * C] for i in range(4)]
    cut[0].copy_(x)
    cut[1].copy_(z)
    I.branch_call(cut[0], cut[1], "rms", pre="rms", sum=cut[2], y=cut[3])
    ref, e = I.branch_t_ref(x, z, "rms", None, None, False, 1.0, 1e-6)
    O.close(cut[2].contiguous(), ref, e + (O.HALF[BF] + O.U) * (ref.abs() + e), "t")
    ref, e = I.branch_v_ref(cut[2].cpu(), "rms", None, None, None, 1e-6)
    O.close(cut[3].contiguous(), ref, e + (O.HALF[BF] + O.U) * (ref.abs() + e), "y")


def test_empty_calls_leave_outputs():
    need_gpu()
    out = torch.full((4, 64), 77.0, device="cuda")
    d = abi.ff_gemm_i8_desc(M=0, N=64, K=128, a_dtype=abi.FF_I8, out_dtype=abi.FF_F32, gelu=0, gate_rows=0, a_row=128, w_row=128, out_row=64,
                            resid_row=64, gate_ld=0)
    assert abi.ff_gemm_i8(d, None, None, None, None, None, None, None, O.ptr(out), None, 0, O.stream()) == 0
    I.branch_call(out[:0], sum=out[:0])
    torch.cuda.synchronize()
    assert (out == 77.0).all()
