"""Each kernel of the integer products at the sizes where its loops wrap and end, against 64 bits."""
import math

import pytest
import torch

import i8_plan_util as P
import i8_util as I
import op_util as O
from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
BF, F32, I8 = torch.bfloat16, torch.float32, torch.int8


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows", ["i8", "float"])
@pytest.mark.parametrize("shape,plan", P.PRODUCTS)
def test_products_by_kernel(dtype, rows, shape, plan):
    """Bias, gate vectors whose rows end inside tiles and launches, residual.  The rows compared: the first 150, 100 around
    each change of gate or launch, the last 150."""
    need_gpu()
    M, N, K = shape
    assert P.product(M, N, K) == plan
    g = O.gen(M + N + K)
    a = torch.randint(-128, 128, (M, K), generator=g).to(I8)
    w = torch.randint(-128, 128, (N, K), generator=g).to(I8)
    a_s, w_s = torch.exp(O.randn((M,), g)), torch.exp(O.randn((N,), g)) / 1e5
    b, r = O.randn((N,), g, dtype), O.randn((M, N), g, dtype)
    per = max(1, 2 * M // 5 - 3)
    gate = O.randn((-(-M // per), N), g)
    out = torch.full((M, N + 8), 77.0, device="cuda").to(dtype)
    if rows == "i8":
        I.gemm_call(a.cuda(), a_s.cuda(), w.cuda(), w_s.cuda(), b.cuda(), False, gate.cuda(), per, r.cuda(), dtype, out[:, :N])
    else:
        x = (a.float() * a_s[:, None]).to(dtype)
        I.gemm_call(x.cuda(), None, w.cuda(), w_s.cuda(), b.cuda(), False, gate.cuda(), per, r.cuda(), dtype, out[:, :N])
    assert (out[:, N:] == 77.0).all()
    near = torch.zeros(M, dtype=torch.bool)
    for at in [0, M, plan[2]] + list(range(per, M, per)):
        near[max(0, at - (150 if at == M else 50)):at + (150 if at == 0 else 50)] = True
    pick = near.nonzero().flatten()
    q, s = (a[pick], a_s[pick]) if rows == "i8" else I.quantise(x[pick])
    ref, tol = I.gemm_ref(q, s, w, w_s, b, False, gate[pick // per], 1, r[pick], dtype)
    O.close(out[:, :N][pick.cuda()], ref, tol, "gemm")
    # the other rows, by their sums: the integers' exact row sums times the columns that share a gate and scale of one
    one = torch.ones(N, device="cuda")
    plain = I.gemm_call(a.cuda(), torch.ones(M, device="cuda"), w.cuda(), one, dtype=F32)
    total = plain.double().sum(1).cpu()
    want = (a.long() * w.long().sum(0)).sum(1).double()
    # each of a row's N results is rounded once to 24 bits: at most 2^-24 of its magnitude
    assert ((total - want).abs() <= 2.0 ** -24 * (plain.double().abs().sum(1).cpu()) + 1e-6).all()


@pytest.mark.parametrize("K", [400, 2064])
def test_two_streams_at_once(K):
    """Calls on two streams with workspaces of their own, shared operands."""
    need_gpu()
    g = O.gen(3)
    M, N = 260, 2056
    x = O.randn((M, K), g, BF).cuda()
    w, w_s = I.quantise(O.randn((N, K), g, std=1 / math.sqrt(K)))
    w, w_s = w.cuda(), w_s.cuda()
    want = I.gemm_call(x, None, w, w_s)
    outs, sides = [torch.zeros_like(want) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    n = 1 << 24
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for o, s, k in zip(outs, sides, ws):
            with torch.cuda.stream(s):
                I.gemm_call(x, None, w, w_s, out=o, ws=k)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows", ["i8", "float"])
def test_a_row_does_not_depend_on_the_others(dtype, rows):
    """The first rows' bits at every number of rows, whatever kernel it takes."""
    need_gpu()
    g = O.gen(5)
    N, K, most = 2056, 1168, 3000
    x = O.randn((most, K), g, dtype).cuda()
    q, s = I.quant_call(x)
    w, w_s = I.quantise(O.randn((N, K), g, std=1 / math.sqrt(K)))
    w, w_s = w.cuda(), w_s.cuda()
    b, r, gate = O.randn((N,), g, dtype).cuda(), O.randn((most, N), g, dtype).cuda(), O.randn((1, N), g).cuda()
    first, seen = None, set()
    for M in (1, 2, 3, 16, 40, 200, 520, 1000, 2500, 3000):
        seen.add(P.product(M, N, K)[0])
        a = (x[:M], None) if rows == "float" else (q[:M], s[:M])
        got = I.gemm_call(*a, w, w_s, b, True, gate, M, r[:M], dtype)
        first = got[:1] if first is None else first
        assert torch.equal(got[:1], first), M
        if M > 3:
            assert torch.equal(got[1:3], three[1:3]), M
        elif M == 3:
            three = got
    assert {P.VEC, P.DIR, P.T64, P.T64X128, P.T128} <= seen, seen


@pytest.mark.parametrize("shape", [(5000, 2600, 400), (7268, 2056, 8208)])
def test_rows_of_large_products_in_small_ones(shape):
    """The same bits whether a row is among thousands, behind the whole rounds of tiles, or one of 130 or two."""
    need_gpu()
    M, N, K = shape
    plan = P.product(M, N, K)
    assert plan[0] == P.T256
    g = O.gen(9)
    q, s = I.quant_call(O.randn((M, K), g, BF).cuda())
    w, w_s = I.quantise(O.randn((N, K), g, std=1 / math.sqrt(K)))
    w, w_s, b, r = w.cuda(), w_s.cuda(), O.randn((N,), g, BF).cuda(), O.randn((M, N), g, BF).cuda()
    gate = O.randn((M, N), g).cuda()
    full = I.gemm_call(q, s, w, w_s, b, True, gate, 1, r)
    for at in (0, 700, min(plan[2], M - 130), M - 130):
        for n in (130, 2):
            got = I.gemm_call(q[at:at + n], s[at:at + n].clone(), w, w_s, b, True, gate[at:at + n], 1, r[at:at + n])
            assert torch.equal(got, full[at:at + n]), (at, n)


@pytest.mark.parametrize("into", ["x", "branch"])
@pytest.mark.parametrize("rows,C", [(1700, 2056), (6500, 264)])
def test_branch_in_place_on_long_walks(rows, C, into):
    """The sum in the place of what it is formed from, while the next rows are on their way."""
    need_gpu()
    g = O.gen(6)
    x, z, v = O.randn((rows, C), g, BF).cuda(), O.randn((rows, C), g, BF).cuda(), O.randn((3, C), g).cuda()
    new = lambda: torch.empty(rows, C, dtype=BF, device="cuda")  # noqa: E731
    how = dict(post="rms", gate=v, pre="layer", scale=v, shift=v, mod_rows=-(-rows // 3))
    t, y, y2 = new(), new(), new()
    I.branch_call(x, branch=z, **how, sum=t, y=y)
    I.branch_call(x, branch=z, **how, sum=x if into == "x" else z, y=y2)
    assert torch.equal(x if into == "x" else z, t) and torch.equal(y2, y)
