"""The shapes of the integer products' tests of K's end reach the kernels that they are there for, and every end of each."""
import pytest

import i8_plan_util as P
from i8_tails_util import SHORTEST, TAILS


@pytest.mark.parametrize("shape,kernel", TAILS)
def test_kernel(shape, kernel):
    assert P.product(*shape)[0] == kernel


@pytest.mark.parametrize("kernel", SHORTEST)
def test_every_end_of_a_tiled_kernel(kernel):
    ks = [s[2] for s, k in TAILS if k == kernel]
    blocks = {-(-k // 128) for k in ks}
    assert {k % 128 for k in ks} >= {0, 16, 48, 64, 112}
    assert min(blocks) == SHORTEST[kernel] and {b % 2 for b in blocks} == {0, 1}
    assert any(k % 128 == 0 and k >= 2048 for k in ks)


def test_no_shorter_walk_is_taken():
    """SHORTEST over many shapes."""
    for K in (16, 128, 144, 256):
        for M in range(3, 15000, 97):
            for N in (8, 72, 208, 520, 1160, 2056, 4616):
                assert P.product(M, N, K)[0] != P.T256


def test_splits_and_rows_behind_whole_rounds():
    plans = [(P.product(*s), s) for s, _ in TAILS]
    assert {p[1] for p, _ in plans} >= {1, 2, 4}
    assert {s[2] % 128 == 0 for p, s in plans if p[2] < s[0]} == {True, False}
