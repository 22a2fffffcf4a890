"""The kernels that the library chooses for products of 8-bit integers, asked of the library itself, and shapes that
reach each of them."""
import ctypes

from paper_2607_27842_amd import abi

DIR, T64, T64X128, T128, T256, VEC = range(6)          # csrc/kernels.h: I8_DIR ..


class Plan(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("splits", ctypes.c_int32), ("head", ctypes.c_int32)]


def product(M, N, K, dtype=abi.FF_BF16):
    """(kernel, splits of K, rows it takes)"""
    f = abi.lib()._ZN2ff12gemm_i8_planEiiii
    f.restype, f.argtypes = Plan, [ctypes.c_int32] * 4
    p = f(dtype, M, N, K)
    return p.kernel, p.splits, p.head


# (M, N, K), and its plan: every kernel with partial tiles, tails of K, odd and even numbers of blocks, walks that end at
# once and long ones; rows behind whole rounds of large tiles, with and without splits of K
PRODUCTS = [
    ((1, 8, 16), (VEC, 1, 1)),
    ((1, 1032, 65536), (VEC, 1, 1)),
    ((2, 24, 1040), (VEC, 1, 2)),
    ((2, 520, 32768), (VEC, 1, 2)),
    ((1, 520, 65552), (T64, 8, 1)),
    ((3, 8, 16), (DIR, 1, 3)),
    ((2, 40, 32784), (T64, 8, 2)),
    ((16, 136, 2304), (DIR, 1, 16)),
    ((8, 2056, 4608), (DIR, 1, 8)),
    ((11, 72, 1040), (DIR, 1, 11)),
    ((16, 2056, 2320), (DIR, 1, 16)),
    ((130, 264, 144), (DIR, 1, 130)),
    ((33, 1160, 1152), (DIR, 1, 33)),
    ((300, 72, 48), (T64, 1, 300)),
    ((520, 2056, 1168), (T64X128, 1, 520)),
    ((200, 1160, 2960), (T64, 1, 200)),
    ((130, 2056, 8208), (T64, 2, 130)),
    ((100, 1480, 4608), (T64, 4, 100)),
    ((9, 40, 131056), (T64, 8, 9)),
    ((300, 4104, 4112), (T64X128, 1, 300)),
    ((1010, 1480, 1040), (T64X128, 1, 1010)),
    ((1100, 2056, 2064), (T128, 1, 1100)),
    ((3000, 1032, 1040), (T128, 1, 3000)),
    ((14566, 256, 512), (T128, 1, 14566)),
    ((5000, 2600, 400), (T256, 1, 5000)),
    ((2100, 4616, 1168), (T256, 1, 2100)),
    ((7176, 2056, 400), (T256, 1, 7168)),
    ((7268, 2056, 8208), (T256, 1, 7168)),
    ((10800, 1288, 2064), (T256, 1, 10752)),
]
