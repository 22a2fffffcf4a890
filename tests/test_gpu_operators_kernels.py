"""Each kernel of the products and the tiled attention with 32 rows a wavefront, at the sizes where its loops
wrap, reload and end, against 64 bits."""
import math

import pytest
import torch

import op_util as O
import plan_util as P
from gpu_util import need_gpu, say
from test_gpu_attention_span import spans_of

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def operands(M, N, K, g, spread=0.5):
    """8-bit operands whose scales differ from block to block by up to 16 (a scale taken from another block
    shows), on the CPU and the GPU; scales that no block has are NaN."""
    a, s = O.quantise(O.randn((M, K), g) * torch.exp(spread * O.randn((M, K), g)), 1)
    w, ws = O.quantise(O.randn((N, K), g, std=1 / math.sqrt(K)) * torch.exp(spread * O.randn((N, K), g)), 128)
    s = s * torch.exp2(4 * torch.rand(s.shape, generator=g) - 2)
    ws = ws * torch.exp2(4 * torch.rand(ws.shape, generator=g) - 2)
    ds = torch.full((s.shape[1], M + 3), math.nan, device="cuda")
    ds[:, :M] = s.t().cuda()
    dw = torch.full((ws.shape[0], ws.shape[1] + 5), math.nan, device="cuda")
    dw[:, :ws.shape[1]] = ws.cuda()
    return (a, s.t().contiguous(), w, ws), (a.cuda(), ds[:, :M], w.cuda(), dw[:, :ws.shape[1]])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape,fp32,bf16", P.PRODUCTS)
def test_products_by_kernel(dtype, shape, fp32, bf16):
    """fp32 outputs besides: the sum over a block of 128 exact products, rounded to 24 bits at each addition, is
    off by sqrt(128 / 2) 2^-24 / sqrt(3) = 2.8e-7 of it (root mean square), the running sum of n blocks by
    sqrt(n / 2) 2^-24 / sqrt(3), 3.0e-7 for the 150 blocks of a wave group at most; 2e-6 normwise is three
    times both.  The 8-bit matrix instructions are 1.5e-5 off."""
    need_gpu()
    M, N, K = shape
    assert P.product(O.CODE[dtype], M, N, K) == (fp32 if dtype == F32 else bf16)
    h, d = operands(M, N, K, O.gen(M + N + K))
    got = O.gemm_call(*d, dtype=dtype)
    ref, tol = O.gemm_ref(*h, None, False, None, dtype)
    O.close(got, ref, tol, "gemm")
    if dtype == F32:
        err = float((got.cpu().double() - ref).norm() / ref.norm())
        say("  %s: %.2g" % (shape, err))
        assert err <= 2e-6


@pytest.mark.parametrize("M,N,K", [(33, 520, 1168), (520, 2056, 1168), (100, 1480, 4608), (1100, 2056, 2064)])
def test_fp32_products_are_exact_on_spread_exponents(M, N, K):
    """As above, on operands whose values span the format's range."""
    need_gpu()
    h, d = operands(M, N, K, O.gen(3), spread=3.0)
    got = O.gemm_call(*d, dtype=F32)
    ref, _ = O.gemm_ref(*h, None, False, None, F32)
    err = float((got.cpu().double() - ref).norm() / ref.norm())
    say("  %s: %.2g" % ((M, N, K), err))
    assert err <= 2e-6


def compare(q, k, v, sp):
    """The first, a middle and the last key head and its query heads."""
    d, G = q.shape[3], q.shape[2] // k.shape[2]
    scale = 1 / math.sqrt(d)
    out = O.attention_call(q.cuda(), k.cuda(), v.cuda(), scale, spans=sp.cuda() if sp is not None else None).cpu()
    for h in (0, k.shape[2] // 2, k.shape[2] - 1):
        hq = slice(h * G, h * G + G)
        ref, tol = O.attention_ref(q[:, :, hq], k[:, :, h:h + 1], v[:, :, h:h + 1], scale, spans=sp)
        O.close(out[:, :, hq].contiguous(), ref, tol, "head %d" % h)


def tensors(B, H, Hkv, d, n):
    g = O.gen(n + d)
    return O.randn((B, n, H, d), g, BF), O.randn((B, n, Hkv, d), g, BF), O.randn((B, n, Hkv, d), g, BF)


@pytest.mark.parametrize("B,H,Hkv,d,n", P.ROWS32)
@pytest.mark.parametrize("kind", [None, "causal", "docs", "prefix", "joint", "overlap", "wild"])
def test_32_rows_a_wavefront(kind, B, H, Hkv, d, n):
    need_gpu()
    assert P.attention(O.CODE[BF], B, Hkv, H // Hkv, d, n, n) == (32, 0)
    compare(*tensors(B, H, Hkv, d, n), spans_of(kind, B, n, n) if kind else None)


@pytest.mark.parametrize("B,H,Hkv,d,n", P.ROWS32)
@pytest.mark.parametrize("kind", ["causal", "prefix", "joint"])
def test_32_rows_a_wavefront_and_unseen_rows(kind, B, H, Hkv, d, n):
    """Infinities and NaN reach the queries that see them and no other; rows without keys get zeros."""
    need_gpu()
    q, k, v = tensors(B, H, Hkv, d, n)
    sp = spans_of(kind, B, n, n)
    at = n - 41 if kind == "causal" else n // 2
    v[:, at, :, 3] = math.inf
    v[:, at + 21, :, d - 1] = -math.inf
    if kind == "prefix":
        k[:, n - 1:], v[:, n - 1:], q[:, n - 1:] = math.nan, math.nan, math.nan
    if kind == "joint":
        t, last = n // 3, n // 3 - 5 * (B - 1) - 2
        k[B - 1, last:t], v[B - 1, last:t], q[B - 1, last:t] = math.nan, math.nan, math.inf
    compare(q, k, v, sp)


@pytest.mark.parametrize("B,H,Hkv,d,n", P.ROWS32[:2])
def test_32_rows_a_wavefront_give_the_same_bits_again(B, H, Hkv, d, n):
    need_gpu()
    q, k, v = (t.cuda() for t in tensors(B, H, Hkv, d, n))
    sp = spans_of("joint", B, n, n).cuda()
    a = O.attention_call(q, k, v, 0.1, spans=sp)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = O.attention_call(q, k, v, 0.1, spans=sp)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, b)
