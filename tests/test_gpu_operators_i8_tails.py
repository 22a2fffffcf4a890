"""Products of 8-bit integers at every end of K, exactly."""
import pytest
import torch

import i8_util as I
import op_util as O
from gpu_util import need_gpu
from i8_tails_util import TAILS
from test_gpu_operators_q8 import guarded, untouched

pytestmark = pytest.mark.gpu
I8 = torch.int8


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape,kernel", TAILS)
def test_ends_of_k(dtype, shape, kernel):
    """Any byte on either side, large ones between the rows, scales of one: the sum, in the output's type.  64 bits hold the
    sums, below 2^31, on their way."""
    need_gpu()
    M, N, K = shape
    g = O.gen(M + N + K)
    a, w = (torch.randint(-128, 128, s, generator=g).to(I8) for s in ((M, K), (N, K)))
    da, dw = torch.full((M, K + 48), 127, dtype=I8, device="cuda"), torch.full((N, K + 16), -128, dtype=I8, device="cuda")
    da[:, :K], dw[:, :K] = a.cuda(), w.cuda()
    out, base = guarded(M, N, N + 8, dtype)
    I.gemm_call(da[:, :K], torch.ones(M, device="cuda"), dw[:, :K], torch.ones(N, device="cuda"), dtype=dtype, out=out)
    want = (da[:, :K].double() @ dw[:, :K].double().t()).float().to(dtype)
    assert torch.equal(out, want)
    untouched(base, M, N, N + 8)


@pytest.mark.parametrize("shape,kernel", [((5000, 2600, 272), 4), ((5000, 2600, 384), 4), ((256, 6144, 2048), 2), ((9, 40, 8256), 1), ((4, 200, 112), 0),
                                          ((8, 136, 240), 0), ((16, 2056, 2240), 0)])
def test_ends_of_k_with_rows_in_a_float_type(shape, kernel):
    """Whole numbers whose largest is 127 in every row: a scale of one, and themselves as their 8 bits."""
    need_gpu()
    M, N, K = shape
    g = O.gen(M + N + K)
    a, w = (torch.randint(-127, 128, s, generator=g).to(I8) for s in ((M, K), (N, K)))
    a[:, K - 1] = 127
    x = torch.full((M, K + 8), 1e4, dtype=torch.bfloat16, device="cuda")
    x[:, :K] = a.cuda().to(torch.bfloat16)
    got = I.gemm_call(x[:, :K], None, w.cuda(), torch.ones(N, device="cuda"), dtype=torch.float32)
    q, s = I.quantise(x[:, :K].cpu())
    assert torch.equal(q, a) and (s == s[0]).all()
    want = (a.cuda().double() @ w.cuda().double().t()).float() * s.cuda()[:, None]
    assert torch.equal(got, want)
