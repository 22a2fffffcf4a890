"""Caps from far below the scores to far above them."""
import math

import pytest
import torch

import op_util as O
from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def check(q, k, v, cap, spans=None):
    """The tolerance of attention_ref for the uncapped scores t, whose size and errors the cap only lessens,
    and tanh's own error e: cap tanh(t / cap) to 2^-20 of it, or 2^-21 of a cap up to 256.  A score's
    error moves a probability by 2.2 times as much, all relative to sum p |v|."""
    need_gpu()
    scale = 1 / math.sqrt(q.shape[3])
    ref, _ = O.attention_ref(q, k, v, scale, cap=cap, spans=spans)
    _, tol = O.attention_ref(q, k, v, scale, spans=spans)
    top = scale * float(q.double().norm(dim=-1).max() * k.double().norm(dim=-1).max())
    e = 2.0 ** -20 * min(top, cap) + (2.0 ** -21 * cap if cap <= 256 else 0.0)
    got = O.attention_call(q.cuda(), k.cuda(), v.cuda(), scale, cap=cap, spans=spans.cuda() if spans is not None else None)
    # (a small cap evens the probabilities out: the tolerance is taken at the largest |v|)
    O.close(got, ref, tol.amax() + 2.2 * e * float(v.double().abs().max()), "cap %g" % cap)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("cap", [2.0 ** -60, 1e-6, 0.5, 255.0, 257.0, 1e3, 1e4, 1e6, 1e9, 2.0 ** 60])
@pytest.mark.parametrize("B,H,Hkv,d,n,causal", [(2, 4, 2, 64, 70, False), (1, 4, 4, 128, 33, True), (1, 16, 16, 128, 600, True), (1, 16, 16, 64, 600, False)])
def test_caps_of_any_size(dtype, cap, B, H, Hkv, d, n, causal):
    n = 120 if dtype == F32 and n > 200 else n
    g = O.gen(n + d)
    q, k, v = O.randn((B, n, H, d), g, dtype, 2.0), O.randn((B, n, Hkv, d), g, dtype, 2.0), O.randn((B, n, Hkv, d), g, dtype)
    q[:, 3] = 0.0                       # scores of zero
    i = torch.arange(n)
    sp = torch.stack([torch.zeros_like(i), i + 1], -1)[None, :, None].to(torch.int32).contiguous() if causal else None
    check(q, k, v, cap, sp)


@pytest.mark.parametrize("cap", [300.0, 1e5])
def test_one_token_on_a_cache(cap):
    g = O.gen(4)
    check(*(O.randn(s, g, BF, 2.0) for s in ((2, 1, 8, 128), (2, 4000, 2, 128), (2, 4000, 2, 128))), cap)
