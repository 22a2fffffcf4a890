"""Limits of the operators' numbers, at both sides of each."""
import pytest

from paper_2607_27842_amd import abi
from test_operators_cpu import attn, refused


@pytest.mark.parametrize("o", [dict(scale=2.0 ** -61), dict(scale=2.0 ** 61), dict(scale=-0.125), dict(scale=float("nan")), dict(cap=1e-40),
                               dict(cap=2.0 ** -61), dict(cap=2.0 ** 61), dict(cap=3e38), dict(cap=float("inf"))])
def test_attention_refuses_scales_and_caps_whose_ratio_may_overflow(o):
    """With cap 1e-40 and scale 0.125 the ratio is infinite in fp32, and a score of zero times it NaN."""
    refused(abi.FF_E_RANGE, attn, n_q=0, **o)


@pytest.mark.parametrize("scale", [2.0 ** -60, 1.0, 2.0 ** 60])
@pytest.mark.parametrize("cap", [0.0, 2.0 ** -60, 50.0, 2.0 ** 60])
def test_attention_takes_scales_and_caps_within(scale, cap):
    assert attn(n_q=0, scale=scale, cap=cap) == 0
