"""Quantisation, root-mean-square norm and products on 8-bit operands against their plain 64-bit forms."""
import math

import pytest
import torch

import op_util as O
from gpu_util import need_gpu, say
from paper_2607_27842_amd import abi

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
GUARD = 77.0


def guarded(rows, cols, pitch, dtype):
    """A [rows, cols] view at `pitch` in a buffer of guard values, and the buffer."""
    need_gpu()
    base = torch.full((rows * pitch + 64,), GUARD, dtype=F32, device="cuda").to(dtype)
    return base[: rows * pitch].view(rows, pitch)[:, :cols], base


def untouched(base, rows, cols, pitch):
    b = base.cpu().float()
    assert (b[rows * pitch:] == GUARD).all(), "written behind the last row"
    assert (b[: rows * pitch].view(rows, pitch)[:, cols:] == GUARD).all(), "written between rows"


def q_desc(x, q, qs, block_rows):
    return abi.ff_quant_desc(rows=x.shape[0], C=x.shape[1], dtype=O.CODE[x.dtype], block_rows=block_rows, x_row=x.stride(0),
                             q_row=q.stride(0), qs_ld=qs.stride(0))


SPECIAL = (0.0, 1e-38, 3e38, 2.0 ** -140, -448.0)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,C,pad", [(1, 8, 0), (1, 1024, 0), (3, 136, 24), (17, 1480, 8), (129, 640, 0), (300, 264, 40)])
def test_quant_bit_for_bit(dtype, block_rows, rows, C, pad):
    """Same formula, same IEEE roundings: values and scales are equal."""
    need_gpu()
    g = O.gen(rows * 7 + C)
    x = O.randn((rows, C), g) * torch.exp(O.randn((1, C), g))
    x[:, :8] *= torch.tensor(SPECIAL * 2)[:8]
    x[rows // 2] = 0.0
    x = x.to(dtype)
    q, s = O.quantise(x, block_rows)
    dx, _ = guarded(rows, C, C + pad, dtype)
    dx.copy_(x)
    dq = torch.full((rows, C + pad), 0x55, dtype=torch.uint8, device="cuda")
    nb = -(-C // 128)
    ld = rows + 5 if block_rows == 1 else nb + 3
    sr = nb if block_rows == 1 else -(-rows // 128)
    ds, base = guarded(sr, ld - (5 if block_rows == 1 else 3), ld, F32)
    abi.ff_quant_q8(q_desc(dx, dq, ds, block_rows), O.ptr(dx), O.ptr(dq), O.ptr(ds), O.stream())
    assert torch.equal(ds.cpu(), s.t() if block_rows == 1 else s)
    assert torch.equal(dq[:, :C].cpu(), q.view(torch.uint8))
    if pad:
        assert (dq[:, C:] == 0x55).all()
    untouched(base, sr, ds.shape[1], ld)


def test_quant_nan_and_infinity():
    """A NaN stays in its place; an infinity makes its block's values NaN; other blocks are as ever."""
    need_gpu()
    x = O.randn((4, 384), O.gen(1))
    x[1, 5] = math.nan
    x[2, 130] = math.inf
    dx = x.cuda()
    dq, ds = torch.empty(4, 384, dtype=torch.uint8, device="cuda"), torch.empty(3, 4, device="cuda")
    abi.ff_quant_q8(q_desc(dx, dq, ds, 1), O.ptr(dx), O.ptr(dq), O.ptr(ds), O.stream())
    v = dq.view(O.E4M3).float().cpu() * O.spread(ds.cpu().t(), 1, 4, 384)
    bad = torch.isnan(v)
    want = torch.zeros_like(bad)
    want[1, 5] = True
    want[2, 128:256] = True
    assert torch.equal(bad, want)
    q, s = O.quantise(x.nan_to_num(nan=0.0, posinf=0.0), 1)
    ok = ~want
    assert torch.equal(v[ok], (q.float() * O.spread(s, 1, 4, 384))[ok])


def norm_call(x, resid, gain, sum_, y, q, qs, eps=1e-6):
    p = lambda t: t.stride(0) if t is not None else 0  # noqa: E731
    d = abi.ff_norm_desc(rows=x.shape[0], C=x.shape[1], dtype=O.CODE[x.dtype], eps=eps, x_row=p(x), resid_row=p(resid),
                         sum_row=p(sum_), y_row=p(y), q_row=p(q), qs_ld=p(qs))
    abi.ff_rms_norm_q8(d, *(O.ptr(t) for t in (x, resid, gain, sum_, y, q, qs)), O.stream())


def norm_check(x, resid, gain, t_got, y_got, q_got, s_got, eps=1e-6):
    """t is exact.  v = t (1 / sqrt(mean t^2 + eps)) g: the sum of squares carries at most 40 roundings (at most
    22 of a lane's and wavefronts' additions, with margin), half of them after the root, and six more
    follow: 26 U < 2^-19.  e4m3: half a step, 2^-4 of the value or 2^-10 of the scale."""
    dt = x.dtype
    t = (x.float() + resid.float()).to(dt) if resid is not None else x
    if t_got is not None:
        assert torch.equal(t_got.cpu(), t)
    T = t.double()
    v = T / torch.sqrt((T * T).mean(1, keepdim=True) + eps) * (gain.double() if gain is not None else 1.0)
    e = 2.0 ** -19 * v.abs()
    if y_got is not None:
        O.close(y_got, v, e + (O.HALF[dt] + O.U) * (v.abs() + e) + 1e-44, "y")
    if q_got is not None:
        rows, C = x.shape
        nb = -(-C // 128)
        top = torch.nn.functional.pad(v.abs(), (0, nb * 128 - C)).view(rows, nb, 128).amax(2)
        s = top.clamp_min(O.TINY) / 448
        O.close(s_got.t(), s, 2.0 ** -18 * s, "scales")
        S = O.spread(s_got.cpu().double().t(), 1, rows, C)
        got = q_got.cpu().double() * S
        O.close(got, v, 2.0 ** -4 * v.abs() * (1 + 2.0 ** -18) + 2.0 ** -10 * S + e, "q")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,C", [(1, 8), (1, 2048), (5, 136), (3, 1480), (2, 4096), (2, 8200), (1, 16384), (1025, 256), (1500, 1032),
                                    (1027, 2048)])
def test_norm_against_64_bits(dtype, rows, C):
    need_gpu()
    g = O.gen(rows + C)
    x = (O.randn((rows, C), g) * torch.exp(O.randn((1, C), g))).to(dtype)
    r = O.randn((rows, C), g, dtype, 3.0)
    gain = (1 + 0.1 * O.randn((C,), g)).to(dtype)
    pads = (8, 16, 24, 32)
    dx, _ = guarded(rows, C, C + pads[0], dtype)
    dx.copy_(x)
    dr = r.cuda()
    t, tb = guarded(rows, C, C + pads[1], dtype)
    y, yb = guarded(rows, C, C + pads[2], dtype)
    q = torch.full((rows, C + pads[3]), 0x55, dtype=torch.uint8, device="cuda")
    qs, sb = guarded(-(-C // 128), rows, rows + 3, F32)
    norm_call(dx, dr, gain.cuda(), t, y, q[:, :C], qs)
    norm_check(x, r, gain, t, y, q[:, :C].contiguous().view(O.E4M3).float(), qs)
    for base, pad in ((tb, pads[1]), (yb, pads[2])):
        untouched(base, rows, C, C + pad)
    untouched(sb, -(-C // 128), rows, rows + 3)
    assert (q[:, C:] == 0x55).all()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_norm_optional_parts_and_in_place(dtype):
    need_gpu()
    g = O.gen(3)
    x, r, gain = O.randn((9, 264), g, dtype), O.randn((9, 264), g, dtype), O.randn((264,), g, dtype)
    e = lambda *s, t=dtype: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    dx, dr, dg = x.cuda(), r.cuda(), gain.cuda()
    y = e(9, 264)
    norm_call(dx, None, dg, None, y, None, None)            # no residual, no 8 bits
    norm_check(x, None, gain, None, y, None, None)
    q, qs = e(9, 264, t=torch.uint8), e(3, 9, t=F32)
    norm_call(dx, dr, None, None, None, q, qs)              # no gain, sum not kept
    norm_check(x, r, None, None, None, q.view(O.E4M3).float(), qs)
    for into in (dx, dr):                                   # the sum in either addend's place
        a, b = dx.clone(), dr.clone()
        norm_call(a, b, dg, a if into is dx else b, y, q, qs)
        norm_check(x, r, gain, a if into is dx else b, y, q.view(O.E4M3).float(), qs)
    z = torch.zeros(2, 264, dtype=dtype)                    # rows of zeros
    norm_call(z.cuda(), None, None, None, y[:2], q[:2], qs[:, :2].contiguous())
    assert (y[:2] == 0).all() and (q[:2] & 0x7f == 0).all()


# ------------------------------------------------------------------ products

def operands(M, N, K, g, pads=(0, 0)):
    """8-bit operands on the CPU and the GPU (their rows at a longer pitch), a_s with a longer pitch too."""
    a, s = O.quantise(O.randn((M, K), g) * torch.exp(0.5 * O.randn((1, K), g)), 1)
    w, ws = O.quantise(O.randn((N, K), g, std=1 / math.sqrt(K)), 128)
    da = torch.full((M, K + pads[0]), 0x7f, dtype=torch.uint8, device="cuda")   # NaN between the rows
    dw = torch.full((N, K + pads[1]), 0x7f, dtype=torch.uint8, device="cuda")
    da[:, :K] = a.view(torch.uint8).cuda()
    dw[:, :K] = w.view(torch.uint8).cuda()
    ds = torch.full((s.shape[1], M + 3), math.nan, device="cuda")
    ds[:, :M] = s.t().cuda()
    return (a, s.t().contiguous(), w, ws), (da[:, :K], ds[:, :M], dw[:, :K], ws.cuda())


# every kernel and split (few rows; 64 x 64 tiles alone and with K split; 128 x 128; 256 x 256), odd rows,
# N and K off every tile, K shorter than a block, one, two and three blocks
SHAPES = [(1, 8, 16), (1, 2048, 8192), (1, 520, 4112), (2, 24, 144), (16, 136, 272), (17, 72, 128), (33, 1160, 1152), (63, 264, 400),
          (64, 2048, 2064), (100, 1480, 4608), (130, 2056, 8192), (200, 1160, 2960), (257, 6152, 400), (300, 72, 48),
          (520, 2056, 1168), (1003, 1480, 2960), (1100, 2048, 256), (5000, 2600, 400), (4700, 2312, 2064)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_against_64_bits(dtype, M, N, K):
    need_gpu()
    g = O.gen(M + N + K)
    h, d = operands(M, N, K, g, (16, 48))
    bias, resid = O.randn((N,), g, dtype), O.randn((M, N), g, dtype)
    out, base = guarded(M, N, N + 8, dtype)
    O.gemm_call(*d, bias.cuda(), False, resid.cuda(), dtype, out)
    ref, tol = O.gemm_ref(*h, bias, False, resid, dtype)
    O.close(out, ref, tol, "gemm")
    untouched(base, M, N, N + 8)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("bias,gelu,resid", [(0, 0, 0), (1, 0, 0), (0, 1, 0), (1, 1, 0), (1, 1, 1), (0, 0, 1)])
@pytest.mark.parametrize("M,N,K", [(5, 200, 272), (130, 2056, 8192), (600, 520, 528), (4500, 2568, 400)])
def test_gemm_epilogues(dtype, bias, gelu, resid, M, N, K):
    need_gpu()
    g = O.gen(M)
    h, d = operands(M, N, K, g)
    b = O.randn((N,), g, dtype) if bias else None
    r = O.randn((M, N), g, dtype) if resid else None
    dr = r.cuda() if resid else None
    got = O.gemm_call(*d, b.cuda() if bias else None, gelu, dr, dtype, dr if resid else None)   # the residual in place
    ref, tol = O.gemm_ref(*h, b, gelu, r, dtype)
    O.close(got, ref, tol, "gemm")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(5, 200, 272), (130, 1096, 528), (4500, 2568, 400)])
def test_gemm_into_other_columns(dtype, M, N, K):
    """The output beside its residual in one buffer, whose other columns stay."""
    need_gpu()
    g = O.gen(M + 1)
    h, d = operands(M, N, K, g)
    r = O.randn((M, 2 * N + 8), g, dtype)
    buf = r.cuda()
    O.gemm_call(*d, None, False, buf[:, :N], dtype, buf[:, N:2 * N])
    ref, tol = O.gemm_ref(*h, None, False, r[:, :N], dtype)
    O.close(buf[:, N:2 * N], ref, tol, "gemm")
    assert torch.equal(buf[:, :N].cpu(), r[:, :N]) and torch.equal(buf[:, 2 * N:].cpu(), r[:, 2 * N:])


def test_gemm_kernels_that_shapes_reach():
    """The sizes above reach every kernel: splits of K where there are few tiles and a long K."""
    need_gpu()
    d = lambda M, N, K: abi.ff_gemm_q8_desc(M=M, N=N, K=K, out_dtype=abi.FF_BF16, gelu=0, a_row=K, w_row=K, out_row=N,  # noqa: E731
                                            resid_row=N, as_ld=M, ws_ld=-(-K // 128))
    assert abi.ff_gemm_q8_workspace_bytes(d(130, 2056, 8192)) > 0
    assert abi.ff_gemm_q8_workspace_bytes(d(130, 1160, 8192)) > 0
    assert abi.ff_gemm_q8_workspace_bytes(d(4500, 2568, 400)) == 0


@pytest.mark.parametrize("M,N,K", [(1, 520, 272), (130, 1160, 8192), (700, 520, 272), (4500, 2568, 400)])
def test_gemm_rows_are_apart(M, N, K):
    """A NaN in a row of A or its scale reaches that output row, one in a weight row its column."""
    need_gpu()
    g = O.gen(M + 1)
    h, d = operands(M, N, K, g)
    d[0][M // 2, K - 1] = 0x7f
    d[2][N - 1, 0] = 0xff
    out = O.gemm_call(*d, dtype=BF).cpu()
    want = torch.zeros(M, N, dtype=torch.bool)
    want[M // 2] = True
    want[:, N - 1] = True
    assert torch.equal(torch.isnan(out), want)
    ref, tol = O.gemm_ref(*h, None, False, None, BF)
    O.close(out[~want], ref[~want], tol[~want])


def test_gemm_same_bits_again_and_on_another_stream():
    need_gpu()
    for M, N, K, dt in ((3, 520, 4096, BF), (130, 2056, 8192, F32), (700, 1160, 1168, BF), (4500, 2568, 400, BF)):
        _, d = operands(M, N, K, O.gen(9))
        a = O.gemm_call(*d, dtype=dt)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b = O.gemm_call(*d, dtype=dt)
            c = O.gemm_call(*d, dtype=dt)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(a, b) and torch.equal(b, c)


def test_gemm_offsets_past_32_bits():
    """Output rows and operand tiles more than 2^32 bytes apart."""
    need_gpu()
    g = O.gen(4)
    M, N, K, pitch = 600, 136, 256, (8 << 20) - 4096    # 600 rows of 8 MB: 4.7 GiB
    a, s = O.quantise(O.randn((M, K), g), 1)
    w, ws = O.quantise(O.randn((N, K), g), 128)
    da = torch.empty(M * pitch, dtype=torch.uint8, device="cuda").view(M, pitch)
    da[:, :K] = a.view(torch.uint8).cuda()
    out = torch.empty(M * (pitch // 2), dtype=BF, device="cuda").view(M, pitch // 2)
    O.gemm_call(da[:, :K], s.t().contiguous().cuda(), w.cuda(), ws.cuda(), dtype=BF, out=out[:, :N])
    ref, tol = O.gemm_ref(a, s.t(), w, ws, None, False, None, BF)
    O.close(out[:, :N].contiguous(), ref, tol, "far rows")


def test_graph_replays():
    """Norm, quantisation and a split product in one captured graph, replayed on new inputs with eager work
    and synchronisations between: every replay gives what eager calls give."""
    need_gpu()
    g = O.gen(11)
    M, C, N = 130, 8192, 2056
    x, r = O.randn((M, C), g, BF).cuda(), O.randn((M, C), g, BF).cuda()
    w, ws = O.quantise(O.randn((N, C), g, std=1 / 90), 128)
    w, ws = w.cuda(), ws.cuda()
    s, q, qs = torch.empty_like(x), torch.empty(M, C, dtype=torch.uint8, device="cuda"), torch.empty(C // 128, M, device="cuda")
    h, h8, hs = torch.empty(M, N, dtype=BF, device="cuda"), torch.empty(M, N, dtype=torch.uint8, device="cuda"), torch.empty(17, M, device="cuda")
    wk = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def step():
        norm_call(x, r, None, s, None, q, qs)
        O.gemm_call(q, qs, w, ws, gelu=True, out=h, ws=wk)
        abi.ff_quant_q8(q_desc(h, h8, hs, 1), O.ptr(h), O.ptr(h8), O.ptr(hs), O.stream())

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(O.randn((M, C), g, BF))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (s, q, qs, h, h8, hs)]
        for t in (s, q, qs, h, h8, hs):
            t.zero_()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (s, q, qs, h, h8, hs))), i
    say("  4 replays equal the eager calls")


def test_empty_calls_leave_outputs():
    need_gpu()
    h, d = operands(4, 64, 128, O.gen(1))
    out = torch.full((4, 64), GUARD, device="cuda")
    assert abi.ff_gemm_q8(abi.ff_gemm_q8_desc(M=0, N=64, K=128, out_dtype=abi.FF_F32, gelu=0, a_row=128, w_row=128, out_row=64,
                                              resid_row=64, as_ld=0, ws_ld=1), None, None, O.ptr(d[2]), O.ptr(d[3]), None, None,
                          O.ptr(out), None, 0, O.stream()) == 0
    torch.cuda.synchronize()
    assert (out == GUARD).all()
