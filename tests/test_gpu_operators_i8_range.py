"""Products of 8-bit integers and norms between branches near the ends of what fp32 holds."""
import math

import pytest
import torch

import i8_util as I
import op_util as O
from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
BF, F32, I8 = torch.bfloat16, torch.float32, torch.int8
TYPES = pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])


def cycle(values, n):
    return torch.tensor(values).repeat(-(-n // len(values)))[:n]


# every kernel: one and two rows, few rows, K split, the tiles, rows behind whole rounds of large tiles
@TYPES
@pytest.mark.parametrize("rows", ["i8", "float"])
@pytest.mark.parametrize("parts", [False, True], ids=["bias", "gate_and_residual_in_place"])
@pytest.mark.parametrize("M,N,K", [(1, 520, 272), (2, 24, 1040), (4, 200, 272), (16, 136, 2304), (33, 1160, 1152), (130, 2056, 8208),
                                   (520, 2056, 1168), (1100, 2056, 2064), (5000, 2600, 400), (7176, 2056, 400)])
def test_large_scales_of_rows_meet_small_ones_of_columns(dtype, parts, rows, M, N, K):
    """A sum times its row's scale is beyond fp32, the product with its column's scale is not: rows of 8-bit integers with such
    scales, and rows of values near the type's largest.  Columns with large scales have infinities, but zeros where the sum
    is zero; rows and columns of ordinary scales are as ever."""
    need_gpu()
    g = O.gen(M + N + K)
    a = torch.randint(-128, 128, (M, K), generator=g).to(I8)
    if M > 1:
        a[M // 2] = 0
    a_s = cycle([3e38, 1.0, 1e35, 2.0 ** 96, 1.5 * 2.0 ** 97, 1e-30, 2.0 ** 95], M)
    w = torch.randint(-128, 128, (N, K), generator=g).to(I8)
    w_s = cycle([1e-36, 2.0 ** -120, 1e-40, 1e-38, 1.0, 1e-33], N)
    w_s[-3] = 1e38
    bias, resid = O.randn((N,), g, dtype), O.randn((M, N), g, dtype) if parts else None
    per = max(1, 2 * M // 5 - 3)
    gate = torch.stack([cycle([1.5, -2.0, 1.0, -1.25], N + i)[i:] for i in range(-(-M // per))]) if parts else None
    out = resid.cuda() if parts else None
    more = dict(gate=gate.cuda(), gate_rows=per, resid=out, out=out) if parts else {}
    if rows == "i8":
        got = I.gemm_call(a.cuda(), a_s.cuda(), w.cuda(), w_s.cuda(), bias.cuda(), dtype=dtype, **more)
    else:
        x = (a.float() * cycle([2e36, 1.0, 1e-3, 2.0 ** 100], M)[:, None]).to(dtype)
        a, a_s = I.quantise(x)
        got = I.gemm_call(x.cuda(), None, w.cuda(), w_s.cuda(), bias.cuda(), dtype=dtype, **more)
    ref, tol = I.gemm_ref(a, a_s, w, w_s, bias, False, gate, per, resid, dtype)
    far = torch.isinf(ref.float().to(dtype))
    assert far.any() and not far.all()
    ref[far] = math.inf * ref[far].sign()
    tol[far] = 0.0
    O.close(got, ref, tol, "gemm")



@pytest.mark.parametrize("rows", ["i8", "float"])
def test_a_row_with_a_large_scale_does_not_depend_on_the_others(rows):
    """The first three rows' bits at every number of rows, whatever kernel it takes, among rows of large and small scales."""
    need_gpu()
    g = O.gen(11)
    N, K, most = 2056, 1168, 3000
    x = (torch.randint(-128, 128, (most, K), generator=g) * cycle([2e36, 1.0, 1e30, 1e-3], most)[:, None]).cuda()
    q, s = I.quant_call(x)
    w, w_s = I.quantise(O.randn((N, K), g))
    w, w_s = w.cuda(), (w_s * 1e-30).cuda()
    b, r, gate = O.randn((N,), g).cuda(), O.randn((most, N), g).cuda(), O.randn((1, N), g).cuda()
    got = {}
    for M in (1, 2, 3, 16, 40, 200, 520, 1000, 2500, 3000):
        a = (x[:M], None) if rows == "float" else (q[:M], s[:M])
        got[M] = I.gemm_call(*a, w, w_s, b, True, gate, M, r[:M], F32)
        assert torch.isfinite(got[M]).all()
        assert all(torch.equal(got[M][:n], got[n]) for n in got if n <= 3), M

SIZES = [1e18, 1e19, 2e19, 1e25, 1e37, 3e38]


def edge_rows(C, g, dtype):
    """Rows of values up to each of SIZES, one with small values beside a single large one, one of a large mean (what
    squares of its spread alone would not show), one of values all alike, an ordinary one, one whose values lie further from
    their mean than fp32 reaches."""
    x = torch.rand((len(SIZES) + 5, C), generator=g, dtype=torch.float64) * 2 - 1
    x[:len(SIZES)] *= torch.tensor(SIZES)[:, None]
    x[len(SIZES)] *= 1e-3
    x[len(SIZES), C // 2] = -1e30
    x[len(SIZES) + 1] = 1e38 + 1e37 * x[len(SIZES) + 1]
    x[len(SIZES) + 2] = 2.0 ** 100
    x[len(SIZES) + 4] = 3e38 + 3e37 * x[len(SIZES) + 4]
    x[len(SIZES) + 4, ::9] *= -1
    return x.to(dtype)


# one, two, four, eight and sixteen wavefronts a row, one and two pieces a lane
@TYPES
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("C", [264, 1032, 2048, 4096, 8192, 16384])
def test_norms_of_rows_whose_squares_leave_fp32(dtype, kind, C):
    """Both places of a norm, each followed by the other's work.  The roundings are norm_ref's; a row of equal values of a power of
    two has them as its mean, without any.  Such rows are summed at 2^-80 of their size, where a small value is off by half a
    step of the least numbers, 2^-150: after the division by at least 2^57 2^-80, 2^-127 in the result, below 1e-37."""
    need_gpu()
    g = O.gen(C)
    x = edge_rows(C, g, dtype)
    rows = x.shape[0]
    dx, zero = x.cuda(), torch.zeros_like(x).cuda()
    y, t, q, s = torch.empty_like(dx), torch.empty_like(dx), torch.empty(rows, C, dtype=I8, device="cuda"), torch.empty(rows, device="cuda")
    I.branch_call(dx, pre=kind, y=y, q=q, q_s=s)
    v, e = I.norm_ref(x.double(), kind, 1e-6)
    O.close(y, v, e + (O.HALF[dtype] + O.U) * (v.abs() + e) + 1e-37, "in front")
    I.close_q(q, s, v, e)
    I.branch_call(zero, dx, kind, sum=t, pre="rms", y=y)
    O.close(t, v, e + (O.HALF[dtype] + O.U) * (v.abs() + e) + 1e-37, "behind")
    v, e = I.norm_ref(t.cpu().double(), "rms", 1e-6)
    O.close(y, v, e + (O.HALF[dtype] + O.U) * (v.abs() + e) + 1e-37, "behind and in front")


@TYPES
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("eps", [2.0 ** -149, 2.0 ** -126, 1e-20, 1e20, 3e38])
def test_norms_with_any_eps(dtype, kind, eps):
    """Rows of zeros stay zeros with the least eps there is; rows of order one are normed; with a large eps, beside rows whose squares
    leave fp32, results are what is left of them (below 2^-103 with the digits that fp32 has there)."""
    need_gpu()
    g = O.gen(4)
    for C in (264, 2048, 16384):
        x = O.randn((5, C), g)
        x[0], x[2], x[3] = 0.0, x[2] * 1e25, x[3] * 1e18
        x = x.to(dtype)
        dx = x.cuda()
        y, q, s = torch.empty_like(dx), torch.empty(5, C, dtype=I8, device="cuda"), torch.empty(5, device="cuda")
        I.branch_call(dx, pre=kind, y=y, q=q, q_s=s, eps=eps)
        assert (y[0] == 0).all() and (q[0] == 0).all()
        v, e = I.norm_ref(x.double(), kind, torch.tensor(eps).double())
        O.close(y, v, e + (O.HALF[dtype] + O.U) * (v.abs() + e) + 1e-37, "y")
