"""The kernels that the library chooses by its estimates, asked of the library itself, and shapes that reach
each of them."""
import ctypes

from paper_2607_27842_amd import abi

DIR, T64, T128, T256 = range(4)          # csrc/kernels.h: Q8_DIR ..


class Two(ctypes.Structure):
    _fields_ = [("first", ctypes.c_int32), ("second", ctypes.c_int32)]


def _ask(name, args):
    f = getattr(abi.lib(), name)
    f.restype, f.argtypes = Two, [ctypes.c_int32] * len(args)
    p = f(*args)
    return p.first, p.second


def product(dtype, M, N, K):
    """(kernel, splits of K)"""
    return _ask("_ZN2ff12gemm_q8_planEiiii", (dtype, M, N, K))


def attention(dtype, B, H_kv, G, d, n_q, n_k, mod=0):
    """(rows a wavefront, workgroups that share a row's keys; 0: the tiled kernel)"""
    return _ask("_ZN2ff19attention_span_planEiiiiiiii", (dtype, B, H_kv, G, d, n_q, n_k, mod))


# (M, N, K), then kernel and splits for fp32 and for bf16 outputs.  Beside small ones: many blocks of K with a tail;
# more than 64 blocks for a wave group (it then reloads the weights' scales), alone and behind a split
PRODUCTS = [
    ((2, 24, 144), (DIR, 1), (DIR, 1)),
    ((1, 2048, 8192), (DIR, 1), (DIR, 1)),
    ((63, 264, 400), (DIR, 1), (DIR, 1)),
    ((130, 264, 12304), (DIR, 1), (DIR, 1)),
    ((300, 72, 48), (T64, 1), (T64, 1)),
    ((520, 2056, 1168), (T64, 1), (T64, 1)),
    ((700, 1160, 16784), (T64, 1), (T64, 1)),
    ((130, 2056, 8208), (T64, 2), (T64, 2)),
    ((100, 1480, 4608), (T64, 4), (T64, 4)),
    ((260, 520, 33008), (T64, 4), (T64, 4)),
    ((300, 72, 150000), (T64, 8), (T64, 8)),
    ((1100, 2048, 256), (T128, 1), (T128, 1)),
    ((1100, 2056, 2064), (T128, 1), (T128, 1)),
    ((900, 2600, 1168), (T128, 1), (T128, 1)),
    ((1000, 2312, 16816), (T128, 1), (T128, 1)),
    ((5000, 2600, 400), (T128, 1), (T256, 1)),
    ((4000, 2312, 8400), (T128, 1), (T256, 1)),
]

# (B, H, H_kv, d, n) of bf16 calls without cap and bias whose wavefronts hold 32 rows
ROWS32 = [(1, 24, 24, 72, 1500), (1, 24, 8, 128, 1500), (2, 18, 9, 96, 1100), (3, 12, 12, 104, 1000)]
