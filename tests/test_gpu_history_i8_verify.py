"""The verify pass on the 8-bit history around the largest sample that one workgroup has to itself (8192 values, in up to four turns of
2048), and where several workgroups' sums meet, with the audit's error counted from the additions on a value's way."""
import math

import pytest
import torch

import i8_util as I
import op_util as O
from gpu_util import need_gpu
from paper_2607_27842_amd import abi
from test_gpu_history_i8 import COEFFS, fill

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
# N C: one turn, full and one value piece more; part of a third; four turns, full, one piece short of it and one piece more (two
# workgroups a sample or several); many turns of 2048 workgroups
SIZES = [(3, 1, 2048), (2, 257, 8), (3, 251, 24), (5, 767, 8), (2, 1023, 8), (3, 4, 2048), (2, 32, 256), (2, 1025, 8), (3, 47, 264),
         (1, 2200, 2048), (2, 4099, 1040)]


def additions(n):
    """On a value's way into its sample's sum: its lane's, 8 a turn; 6 in the wavefront, 2 in the workgroup; and where there are
    several workgroups those of a lane that adds their sums, and 6 and 4 more."""
    groups = 1 if n <= 8192 else min(-(-n // 2048), 2048)
    turns = -(-n // (groups * 2048))
    return 8 * turns + 8 + (0 if groups == 1 else -(-groups // 256) + 10)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("order", range(4))
@pytest.mark.parametrize("B,N,C", SIZES)
def test_verify_by_turns_and_workgroups(dtype, order, B, N, C):
    """All of a sum's terms are positive: its relative error is at most half a step of fp32 for each addition.  A difference is
    rounded once, and the quotient and the addition of eps once each."""
    need_gpu()
    n = N * C
    g = O.gen(n + order)
    m, S = I.model(B, N, C, dtype), 4
    cache, _ = fill(m, S, B, N, C, dtype, g)
    res = order % 2 == 1
    u, hf = (O.randn((B, N, C), g, dtype) for _ in range(2))
    du, dh = u.cuda(), hf.cuda()
    size = abi.ff_workspace_bytes(m)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    args = (m, O.ptr(cache), S, 0, order, [2, 0, 3, 1][:order + 1], COEFFS[order], O.ptr(du) if res else None)
    d = torch.empty_like(du)
    abi.ff_draft_forecast_i8(*args, O.ptr(d), O.stream())
    a, b = d.double(), dh.double()
    ref = ((a - b).abs().sum((1, 2)) / (b.abs().sum((1, 2)) + 1e-8)).cpu()
    tol = (2 * additions(n) + 3) * O.U * ref * (1 + 2.0 ** -10)
    token, channel = torch.arange(N, device="cuda"), torch.arange(C, device="cuda")
    for kind, stride in ((0, 1), (1, 1), (2, 1), (2, 2), (2, 3), (3, 2), (3, 5), (2, 1 << 30)):
        want = (d, dh, torch.where((token % stride == 0)[:, None], dh, d), torch.where(channel % stride == 0, dh, d))[kind]
        base, rel = torch.full((B * n + 64,), 77.0, device="cuda").to(dtype), torch.full((B + 2,), 77.0, device="cuda")
        out = base[:B * n].view(B, N, C)
        abi.ff_verify_replace_i8(*args, O.ptr(dh), O.ptr(out), kind, 1e-8, O.ptr(rel), O.ptr(ws), size, O.stream(), stride=stride)
        assert torch.equal(out, want), (kind, stride)
        O.close(rel[:B], ref, tol, "rel")
        assert (base[B * n:].float() == 77.0).all() and (rel[B:] == 77.0).all()


@pytest.mark.parametrize("B,N,C", [(3, 251, 24), (2, 32, 256), (3, 47, 264)])
def test_a_spoilt_sample_stays_alone(B, N, C):
    """A NaN in one sample's exact result reaches that sample's audit and value only."""
    need_gpu()
    g = O.gen(1)
    m, S = I.model(B, N, C, BF), 2
    cache, _ = fill(m, S, B, N, C, BF, g)
    u, h = (O.randn((B, N, C), g, BF).cuda() for _ in range(2))
    h[1, N - 1, C - 1] = math.nan
    size = abi.ff_workspace_bytes(m)
    ws, out, rel = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty_like(u), torch.empty(B, device="cuda")
    abi.ff_verify_replace_i8(m, O.ptr(cache), S, 0, 1, [0, 1], COEFFS[1], O.ptr(u), O.ptr(h), O.ptr(out), 1, 1e-8, O.ptr(rel), O.ptr(ws), size,
                             O.stream())
    assert torch.isnan(rel).cpu().nonzero().flatten().tolist() == [1]
    assert torch.isnan(out).cpu().nonzero().tolist() == [[1, N - 1, C - 1]]
