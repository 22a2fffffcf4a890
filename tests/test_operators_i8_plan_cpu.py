"""The shapes of the integer products' GPU tests reach the kernels that they are there for."""
import pytest

import i8_plan_util as P
from paper_2607_27842_amd import abi


@pytest.mark.parametrize("shape,plan", P.PRODUCTS)
def test_products(shape, plan):
    assert P.product(*shape) == plan


def test_every_kernel_split_and_tail_is_reached():
    assert {p[0] for _, p in P.PRODUCTS} == {P.DIR, P.T64, P.T64X128, P.T128, P.T256, P.VEC}
    tails = [P.product(s[0] - p[2], *s[1:]) for s, p in P.PRODUCTS if p[2] < s[0]]
    assert {p[1] for _, p in P.PRODUCTS} | {t[1] for t in tails} == {1, 2, 4, 8}
    assert len(tails) == 3 and any(t[1] > 1 for t in tails)


@pytest.mark.parametrize("shape,plan", P.PRODUCTS)
def test_workspaces(shape, plan):
    """Partial sums where K is split, of the rows that are; rows that the call puts in 8 bits, but for few short ones."""
    M, N, K = shape
    own = M <= 16 and -(-M // 8) * K <= 4608 and M * K * -(-N // 16) <= 1 << 23
    kernel, splits, head = plan
    if head < M:
        splits, head = P.product(M - head, N, K)[1], M - head
    part = splits * head * N * 4 if splits > 1 else 0
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    for a, rows in ((abi.FF_I8, 0), (abi.FF_BF16, None if kernel == P.VEC or own else up(M * K) + up(4 * M))):
        d = abi.ff_gemm_i8_desc(M=M, N=N, K=K, a_dtype=a, out_dtype=abi.FF_BF16, gelu=0, gate_rows=0, a_row=K, w_row=K, out_row=N, resid_row=N, gate_ld=0)
        assert abi.ff_gemm_i8_workspace_bytes(d) == (0 if rows is None else rows + part)
