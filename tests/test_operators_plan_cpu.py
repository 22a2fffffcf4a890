"""The shapes of the operators' GPU tests reach the kernels that they are there for."""
import pytest

import plan_util as P
from paper_2607_27842_amd import abi


@pytest.mark.parametrize("shape,fp32,bf16", P.PRODUCTS)
def test_products(shape, fp32, bf16):
    assert P.product(abi.FF_F32, *shape) == fp32
    assert P.product(abi.FF_BF16, *shape) == bf16


def test_every_kernel_and_split_is_reached():
    for i, code in ((1, abi.FF_F32), (2, abi.FF_BF16)):
        kinds = {s[i][0] for s in P.PRODUCTS}
        assert kinds == ({P.DIR, P.T64, P.T128} | ({P.T256} if code == abi.FF_BF16 else set()))
        assert {s[i][1] for s in P.PRODUCTS} == {1, 2, 4, 8}


@pytest.mark.parametrize("B,H,Hkv,d,n", P.ROWS32)
def test_attention_of_32_rows_a_wavefront(B, H, Hkv, d, n):
    assert P.attention(abi.FF_BF16, B, Hkv, H // Hkv, d, n, n) == (32, 0)
    assert P.attention(abi.FF_BF16, B, Hkv, H // Hkv, d, n, n, 1) == (16, 0)
    assert P.attention(abi.FF_F32, B, Hkv, H // Hkv, d, n, n) == (16, 1)


def test_plans_and_workspaces_agree():
    for shape, fp32, bf16 in P.PRODUCTS:
        M, N, K = shape
        for code, (_, splits) in ((abi.FF_F32, fp32), (abi.FF_BF16, bf16)):
            d = abi.ff_gemm_q8_desc(M=M, N=N, K=K, out_dtype=code, gelu=0, a_row=K, w_row=K, out_row=N, resid_row=N, as_ld=M, ws_ld=-(-K // 128))
            assert abi.ff_gemm_q8_workspace_bytes(d) == (splits * M * N * 4 if splits > 1 else 0)
