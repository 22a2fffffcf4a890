"""The norm between two branches in 8 bits and the product that takes it, run again and again: the same bits each time, the product exact on
the norm's integers, and these the nearest ones but where a value lies at the border of two."""
import pytest
import torch

import i8_util as I
import op_util as O
from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
BF, F32, I8 = torch.bfloat16, torch.float32, torch.int8


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,C,N", [(1, 2048, 6144), (333, 1488, 1480), (4608, 2048, 6144)])
def test_norm_and_product_repeat_themselves(dtype, rows, C, N):
    need_gpu()
    g = O.gen(rows)
    mod = O.randn((1, 3 * C), g, std=0.3)
    gains = [(1 + 0.1 * O.randn((C,), g)).to(dtype) for _ in range(2)]
    w, w_s = I.quantise(O.randn((N, C), g, std=C ** -0.5))
    dm, dg, dw, dws = mod.cuda(), [t.cuda() for t in gains], w.cuda(), w_s.cuda()
    sets = [tuple(O.randn((rows, C), g, dtype) for _ in range(2)) for _ in range(2)]
    dev = [tuple(t.cuda() for t in s) for s in sets]
    t, q, s = torch.empty(rows, C, dtype=dtype, device="cuda"), torch.empty(rows, C, dtype=I8, device="cuda"), torch.empty(rows, device="cuda")
    out, ws = torch.empty(rows, N, dtype=dtype, device="cuda"), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def run(x, z):
        I.branch_call(x, z, "rms", dg[0], dm[:, :C], False, "rms", dg[1], dm[:, C:2 * C], dm[:, 2 * C:], rows, sum=t, q=q, q_s=s)
        I.gemm_call(q, s, dw, dws, dtype=dtype, out=out, ws=ws)

    first = []
    for i in range(24):   # two sets of inputs through the same buffers, waited for now and then
        run(*dev[i % 2])
        got = [v.clone() for v in (t, q, s, out)]
        if i < 2:
            first.append(got)
        assert all(torch.equal(a, b) for a, b in zip(got, first[i % 2])), i
        if i % 5 == 0:
            torch.cuda.synchronize()
    for (x, z), (t1, q1, s1, o1) in zip(sets, first):
        total = (q1.double() @ dw.double().t()).float()          # whole numbers below 2^31
        assert torch.equal(o1, (total * s1[:, None] * dws).to(dtype))
        ref, e = I.branch_t_ref(x, z, "rms", gains[0], mod[:, :C], False, 1.0, 1e-6)
        O.close(t1, ref, e + (O.HALF[dtype] + O.U) * (ref.abs() + e) + 1e-44, "t")
        v, e = I.branch_v_ref(t1.cpu(), "rms", gains[1], mod[:, C:2 * C], mod[:, 2 * C:], 1e-6)
        I.close_q(q1, s1, v, e)
        # in steps of the row's exact scale: the nearest integer, or within the error of v, that of the scale (the same, and two
        # roundings) at up to 127 of them, and two more roundings of the border
        step = v.abs().amax(1, keepdim=True) / 127
        worst = 2 * e.amax(1, keepdim=True) / step + 127 * 8 * O.U
        exact = v / step
        other = q1.cpu().double() != torch.round(exact)
        assert ((exact - torch.floor(exact) - 0.5).abs()[other] <= worst.expand_as(v)[other]).all() and other.double().mean() < 1e-3
