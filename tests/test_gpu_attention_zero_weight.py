"""Rows whose scores are all -inf: zeros, whatever the values hold that their spans reach, from every kernel."""
import math

import pytest
import torch

import op_util as O
from gpu_util import need_gpu
from paper_2607_27842_amd import abi

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
TABLE = abi.FF_BIAS_TABLE


def tensors(B, H, Hkv, d, nq, nk, dtype):
    g = O.gen(nq + 7 * nk + d)
    q, k, v = O.randn((B, nq, H, d), g, dtype), O.randn((B, nk, Hkv, d), g, dtype), O.randn((B, nk, Hkv, d), g, dtype)
    v[:, nk // 3, :, 5] = math.inf
    v[:, nk // 2, :, d - 1] = -math.inf
    v[:, nk - 1, :, 0] = math.nan
    return q, k, v


# one workgroup a row tile; keys split over workgroups; (bf16) the tiled kernel
SIZES = [(2, 4, 2, 64, 60, 60), (2, 8, 2, 128, 1, 5000), (1, 16, 16, 64, 600, 600), (1, 16, 16, 128, 600, 600)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("spans", [None, "causal", "two"])
@pytest.mark.parametrize("B,H,Hkv,d,nq,nk", SIZES)
def test_all_scores_minus_infinity(dtype, spans, B, H, Hkv, d, nq, nk):
    need_gpu()
    nq, nk = (150, 150) if dtype == F32 and nq > 200 else (nq, nk)
    q, k, v = tensors(B, H, Hkv, d, nq, nk, dtype)
    i = torch.arange(nq)
    z = torch.zeros_like(i)
    sp = {None: None, "causal": torch.stack([z, i + 1 + nk - nq], -1)[:, None],
          "two": torch.stack([torch.stack([z, z + nk // 2 + 1], -1), torch.stack([z + nk - 9, z + nk], -1)], 1)}[spans]
    sp = sp.to(torch.int32)[None].contiguous().cuda() if spans else None
    bias = torch.full((H, 1), -math.inf)
    out = O.attention_call(q.cuda(), k.cuda(), v.cuda(), 0.125, bias_kind=TABLE, bias=bias.cuda(), reach=0, spans=sp)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B,H,Hkv,d,nq,nk", [s for s in SIZES if s[1] != s[2]] + [(1, 16, 8, 64, 600, 600)])
def test_hidden_head_beside_a_seeing_one(dtype, B, H, Hkv, d, nq, nk):
    """Heads of one key head are rows of one tile: those whose table hides every key get zeros, the others
    their infinities and NaN."""
    need_gpu()
    nq, nk = (150, 150) if dtype == F32 and nq > 200 else (nq, nk)
    q, k, v = tensors(B, H, Hkv, d, nq, nk, dtype)
    bias = torch.zeros(H, 1)
    bias[::2] = -math.inf
    out = O.attention_call(q.cuda(), k.cuda(), v.cuda(), 0.125, bias_kind=TABLE, bias=bias.cuda(), reach=0).cpu()
    assert (out[:, :, ::2] == 0).all()
    ref, tol = O.attention_ref(q, k, v, 0.125, bias_kind=TABLE, bias=bias, reach=0)
    O.close(out[:, :, 1::2].contiguous(), ref[:, :, 1::2], tol[:, :, 1::2], "seeing heads")
