"""The feature history in 8-bit integers against its plain form, and a block and its history in 8 bits in sequence."""
import math

import pytest
import torch

import i8_util as I
import op_util as O
from gpu_util import need_gpu, say
from paper_2607_27842_amd import abi

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
# one value piece; a part of a block; samples that end inside a block, and half-way through a lane's 16 values; whole
# blocks; many groups
SIZES = [(1, 1, 8), (1, 3, 40), (3, 5, 24), (2, 7, 136), (4, 33, 264), (8, 256, 1152), (3, 333, 1480), (1, 2100, 2048), (32, 2, 64)]
COEFFS = ([1.0], [1.5, -0.5], [1.875, -1.25, 0.375], [2.1875, -2.1875, 1.3125, -0.3125])


def cache_of(m, S, B, N, C, L=1):
    n = abi.ff_cache_i8_bytes(m, S)
    assert n == L * S * I.slot_bytes(B, N, C)
    return torch.full((n + 256,), 0x5a, dtype=torch.uint8, device="cuda")


def update(m, cache, S, layer, slot, u, h):
    abi.ff_cache_update_i8(m, O.ptr(cache), S, layer, slot, O.ptr(u), O.ptr(h), abi.FF_RESIDUAL if u is not None else abi.FF_OUTPUT, O.stream())


def fill(m, S, B, N, C, dtype, g, L=1):
    """A cache of random slots, and each slot's whole values and scales on the CPU."""
    cache, held = cache_of(m, S, B, N, C, L), {}
    for i in range(L * S):
        h = O.randn((B, N, C), g, dtype, std=2.0 ** (i - 1))
        update(m, cache, S, i // S, i % S, None, h.cuda())
        held[i] = I.quantise(I.blocks(h.float()))
    return cache, held


@TYPES
@pytest.mark.parametrize("res", [True, False], ids=["residual", "output"])
@pytest.mark.parametrize("B,N,C", SIZES)
def test_update_bit_for_bit(dtype, res, B, N, C):
    """Same formula, same IEEE roundings; the other slots and what lies behind the cache stay."""
    need_gpu()
    g = O.gen(B + N + C)
    m, S, L = I.model(B, N, C, dtype, 2), 3, 2
    u, h = O.randn((B, N, C), g, dtype), O.randn((B, N, C), g, dtype, 3.0)
    h[0, 0, :4] = torch.tensor([0.0, 1e-38, 1e30, 2.0 ** -130]).to(dtype)
    cache = cache_of(m, S, B, N, C, L)
    update(m, cache, S, 1, 2, u.cuda() if res else None, h.cuda())
    q, s = I.quantise(I.blocks(h.float() - u.float() if res else h.float()))
    at, sc = I.slot_views(cache, 5, B, N, C)
    assert torch.equal(at.cpu(), q) and torch.equal(sc.cpu(), s)
    size, used = I.slot_bytes(B, N, C), B * q.shape[1] * 132
    assert (cache[:5 * size] == 0x5a).all() and (cache[5 * size + used:] == 0x5a).all()


@TYPES
def test_nan_and_infinity_spoil_their_block(dtype):
    need_gpu()
    B, N, C = 2, 5, 72   # 360 values: blocks of 128, 128 and 104
    m = I.model(B, N, C, dtype)
    h = O.randn((B, N, C), O.gen(2), dtype)
    h[0].view(-1)[130], h[1].view(-1)[359] = math.nan, -math.inf
    cache = cache_of(m, 1, B, N, C)
    update(m, cache, 1, 0, 0, None, h.cuda())
    out = torch.empty(B, N, C, dtype=dtype, device="cuda")
    abi.ff_draft_forecast_i8(m, O.ptr(cache), 1, 0, 0, [0], [1.0], None, O.ptr(out), O.stream())
    want = torch.zeros(B, 360, dtype=torch.bool)
    want[0, 128:256], want[1, 256:] = True, True
    assert torch.equal(torch.isnan(out.cpu()).view(B, 360), want)


def draft_ref(held, slots, coeffs, u, shape):
    """The draft in 64 bits and its error before the last rounding: a product and an addition a term, the stream's."""
    B, n = shape[0], shape[1] * shape[2]
    d = torch.zeros(B, n, dtype=torch.float64)
    S = torch.zeros_like(d)
    for c, i in zip(coeffs, slots):
        q, s = held[i]
        x = c * (q.double() * s.double()[..., None]).view(B, -1)[:, :n]
        d, S = d + x, S + x.abs()
    d, S = d.view(shape), S.view(shape)
    if u is not None:
        d, S = d + u.double(), S + u.double().abs()
    return d, (2 * len(coeffs) + 2) * O.U * S


@TYPES
@pytest.mark.parametrize("order", range(4))
@pytest.mark.parametrize("res", [True, False], ids=["residual", "output"])
@pytest.mark.parametrize("B,N,C", SIZES)
def test_draft_against_64_bits(dtype, order, res, B, N, C):
    need_gpu()
    g = O.gen(B * N + C + order)
    S, L = 4, 2
    m = I.model(B, N, C, dtype, L)
    cache, held = fill(m, S, B, N, C, dtype, g, L)
    u = O.randn((B, N, C), g, dtype) if res else None
    slots = [3, 1, 0, 2][:order + 1]
    base = torch.full((B * N * C + 64,), 77.0, device="cuda").to(dtype)
    out = base[:B * N * C].view(B, N, C)
    du = u.cuda() if res else None
    abi.ff_draft_forecast_i8(m, O.ptr(cache), S, 1, order, slots, COEFFS[order], O.ptr(du), O.ptr(out), O.stream())
    ref, e = draft_ref(held, [S + i for i in slots], COEFFS[order], u, (B, N, C))
    O.close(out, ref, e + (O.HALF[dtype] + O.U) * (ref.abs() + e) + 1e-44, "draft")
    assert (base[B * N * C:].float() == 77.0).all()
    if res:   # in place, and the same slot for every term
        abi.ff_draft_forecast_i8(m, O.ptr(cache), S, 1, order, slots, COEFFS[order], O.ptr(du), O.ptr(du), O.stream())
        assert torch.equal(du, out)
        abi.ff_draft_forecast_i8(m, O.ptr(cache), S, 0, order, [2] * (order + 1), COEFFS[order], O.ptr(out), O.ptr(du), O.stream())
        ref, e = draft_ref(held, [2] * (order + 1), COEFFS[order], out.cpu(), (B, N, C))
        O.close(du, ref, e + (O.HALF[dtype] + O.U) * (ref.abs() + e) + 1e-44, "one slot")


@TYPES
@pytest.mark.parametrize("res", [True, False], ids=["residual", "output"])
@pytest.mark.parametrize("B,N,C", SIZES)
def test_verify(dtype, res, B, N, C):
    """What is forwarded is the draft's or the exact result's bits; the audit is that of the stored draft: a lane adds at
    most 16 values a step, (n / (2048 * 256 * 16) + 1) 16 of them and about 20 partial sums, each a rounding."""
    need_gpu()
    g = O.gen(N + C)
    m, S, order = I.model(B, N, C, dtype), 3, 2
    cache, held = fill(m, S, B, N, C, dtype, g)
    u, hf = (O.randn((B, N, C), g, dtype) for _ in range(2))
    du, dh = u.cuda(), hf.cuda()
    n = abi.ff_workspace_bytes(m)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    args = (m, O.ptr(cache), S, 0, order, [1, 0, 2], COEFFS[order], O.ptr(du) if res else None)
    d = torch.empty_like(du)
    abi.ff_draft_forecast_i8(*args, O.ptr(d), O.stream())
    want = {0: d, 1: dh, 2: torch.where((torch.arange(N, device="cuda") % 3 == 0)[:, None], dh, d),
            3: torch.where(torch.arange(C, device="cuda") % 3 == 0, dh, d)}
    a, b = d.cpu().double(), hf.double()
    ref = (a - b).abs().sum((1, 2)) / (b.abs().sum((1, 2)) + 1e-8)
    tol = 2 * ((N * C / (2048 * 256 * 16) + 1) * 16 + 20) * O.U * ref
    for kind, w in want.items():
        out, rel = torch.empty_like(du), torch.full((B + 2,), 77.0, device="cuda")
        abi.ff_verify_replace_i8(*args, O.ptr(dh), O.ptr(out), kind, 1e-8, O.ptr(rel), O.ptr(ws), n, O.stream(), stride=3)
        assert torch.equal(out, w), kind
        O.close(rel[:B], ref, tol, "rel")
        assert (rel[B:] == 77.0).all()
    if res:   # forwarded into u itself, without the audit
        abi.ff_verify_replace_i8(*args, O.ptr(dh), O.ptr(du), 2, 1e-8, None, O.ptr(ws), n, O.stream(), stride=3)
        assert torch.equal(du, want[2])


@TYPES
def test_the_8_bit_history_is_near_the_full_one(dtype):
    """Against ff_draft_forecast on the same features: each differs by at most half a step of its block, plus the
    roundings of both paths (two of the dtype's in bf16, whose slots are rounded as well)."""
    need_gpu()
    g = O.gen(6)
    B, N, C, S = 2, 96, 264, 2
    m = I.model(B, N, C, dtype)
    full = torch.empty(abi.ff_cache_bytes(m, S), dtype=torch.uint8, device="cuda")
    small = torch.empty(abi.ff_cache_i8_bytes(m, S), dtype=torch.uint8, device="cuda")
    top = torch.zeros(B, N * C, dtype=torch.float64)
    mag = torch.zeros(B, N * C, dtype=torch.float64)
    for i, c in enumerate(COEFFS[1]):
        u, h = O.randn((B, N, C), g, dtype), O.randn((B, N, C), g, dtype)
        du, dh = u.cuda(), h.cuda()
        abi.ff_cache_update(m, O.ptr(full), S, 0, i, O.ptr(du), O.ptr(dh), abi.FF_RESIDUAL, O.stream())
        update(m, small, S, 0, i, du, dh)
        _, s = I.quantise(I.blocks(h.float() - u.float()))
        top += abs(c) * 0.5 * s.double().repeat_interleave(128, 1)[:, :N * C]
        mag += abs(c) * (h.double() - u.double()).abs().view(B, -1)
    u = O.randn((B, N, C), g, dtype)
    du = u.cuda()
    a, b = torch.empty_like(du), torch.empty_like(du)
    abi.ff_draft_forecast(m, O.ptr(full), S, 0, 1, [0, 1], COEFFS[1], O.ptr(du), O.ptr(a), O.stream())
    abi.ff_draft_forecast_i8(m, O.ptr(small), S, 0, 1, [0, 1], COEFFS[1], O.ptr(du), O.ptr(b), O.stream())
    size = mag + u.double().abs().view(B, -1) + top
    tol = top * (1 + 2.0 ** -14) + 3.1 * O.HALF[dtype] * size + 16 * O.U * size
    O.close(b.view(B, -1), a.cpu().double().view(B, -1), tol, "drafts")


def test_a_long_history_past_32_bits():
    """Slots more than 2^32 bytes into the cache."""
    need_gpu()
    B, N, C, L, S = 1, 8192, 2048, 33, 8
    m = I.model(B, N, C, BF, L)
    size = I.slot_bytes(B, N, C)
    assert size * 263 > 1 << 32
    cache = torch.empty(abi.ff_cache_i8_bytes(m, S), dtype=torch.uint8, device="cuda")
    h = O.randn((B, N, C), O.gen(1), BF).cuda()
    update(m, cache, S, 32, 7, None, h)
    q, s = I.slot_views(cache, 263, B, N, C)
    wq, wsc = I.quantise(I.blocks(h.cpu().float()))
    assert torch.equal(q.cpu(), wq) and torch.equal(s.cpu(), wsc)
    out = torch.empty_like(h)
    abi.ff_draft_forecast_i8(m, O.ptr(cache), S, 32, 0, [7], [1.0], None, O.ptr(out), O.stream())
    assert torch.equal(out.cpu().view(-1), (wq.float() * wsc[..., None]).to(BF).view(-1))


def block_step(p, b):
    """An 8-bit MLP branch between its norms, its result into the 8-bit history, and the next draft from it."""
    I.branch_call(b["x"], b["z"], "rms", p["pg"], p["mod"][:, :p["C"]], True, "layer", None, p["mod"][:, p["C"]:2 * p["C"]],
                  p["mod"][:, 2 * p["C"]:], p["N"], sum=b["t"], q=b["q"], q_s=b["qs"])
    I.gemm_call(b["q"], b["qs"], p["w1"], p["s1"], p["b1"], True, out=b["hid"], ws=b["ws"])
    I.gemm_call(b["hid"], None, p["w2"], p["s2"], p["b2"], False, p["mod"][:, :p["C"]], p["N"], b["t"], out=b["h"], ws=b["ws"])
    update(p["m"], b["cache"], 2, 0, 1, b["x"], b["h"])
    abi.ff_draft_forecast_i8(p["m"], O.ptr(b["cache"]), 2, 0, 1, [1, 0], [1.5, -0.5], O.ptr(b["x"]), O.ptr(b["d"]), O.stream())
    abi.ff_verify_replace_i8(p["m"], O.ptr(b["cache"]), 2, 0, 1, [1, 0], [1.5, -0.5], O.ptr(b["x"]), O.ptr(b["h"]), O.ptr(b["o"]), 0, 1e-8,
                             O.ptr(b["rel"]), O.ptr(b["vws"]), b["vws"].numel(), O.stream())


def setup(B, N, C, H, dtype, seed):
    g = O.gen(seed)
    rows = B * N
    p = dict(B=B, N=N, C=C, m=I.model(B, N, C, dtype), pg=(1 + 0.1 * O.randn((C,), g)).to(dtype), mod=O.randn((B, 3 * C), g, std=0.4),
             b1=O.randn((H,), g, dtype), b2=O.randn((C,), g, dtype))
    p["w1"], p["s1"] = I.quantise(O.randn((H, C), g, std=1 / math.sqrt(C)))
    p["w2"], p["s2"] = I.quantise(O.randn((C, H), g, std=1 / math.sqrt(H)))
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in p.items()}
    e = lambda *s, t=dtype: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    b = dict(x=O.randn((rows, C), g, dtype).cuda(), z=O.randn((rows, C), g, dtype).cuda(), t=e(rows, C), q=e(rows, C, t=torch.int8),
             qs=e(rows, t=F32), hid=e(rows, H), h=e(rows, C), d=e(rows, C), o=e(rows, C), rel=e(B, t=F32),
             ws=e(1 << 24, t=torch.uint8), cache=e(abi.ff_cache_i8_bytes(p["m"], 2), t=torch.uint8), vws=e(abi.ff_workspace_bytes(p["m"]), t=torch.uint8))
    return p, dev, b


@TYPES
@pytest.mark.parametrize("B,N,C,H", [(1, 1, 64, 256), (2, 65, 272, 1040), (2, 256, 1152, 4608)])
def test_a_block_in_8_bits(dtype, B, N, C, H):
    """Each step of the run against its 64-bit form on what the step before gave."""
    need_gpu()
    p, dev, b = setup(B, N, C, H, dtype, B + N)
    block_step(dev, b)
    c = {k: v.cpu() for k, v in b.items()}
    at = torch.arange(B * N) // N
    gate, scale, shift = (p["mod"][:, i * C:(i + 1) * C] for i in range(3))
    ref, e = I.branch_t_ref(c["x"], c["z"], "rms", p["pg"], gate[at], True, 1.0, 1e-6)
    O.close(b["t"], ref, e + (O.HALF[dtype] + O.U) * (ref.abs() + e), "t")
    I.close_q(b["q"], b["qs"], *I.branch_v_ref(c["t"], "layer", None, scale[at], shift[at], 1e-6))
    ref, tol = I.gemm_ref(c["q"], c["qs"], p["w1"], p["s1"], p["b1"], True, dtype=dtype)
    O.close(b["hid"], ref, tol, "hidden")
    ref, tol = I.gemm_ref(*I.quantise(c["hid"]), p["w2"], p["s2"], p["b2"], False, gate, N, c["t"], dtype)
    O.close(b["h"], ref, tol, "h")
    q, s = I.quantise(I.blocks((c["h"].float() - c["x"].float()).view(B, N, C)))
    zero = torch.zeros_like(q), torch.zeros_like(s)
    ref, e = draft_ref({1: (q, s), 0: zero}, [1, 0], [1.5, -0.5], c["x"].view(B, N, C), (B, N, C))
    O.close(b["d"].view(B, N, C), ref, e + (O.HALF[dtype] + O.U) * (ref.abs() + e), "draft")
    assert torch.equal(b["o"], b["d"])
    x, y = c["d"].double().view(B, -1), c["h"].double().view(B, -1)
    ref = (x - y).abs().sum(1) / (y.abs().sum(1) + 1e-8)
    O.close(b["rel"], ref, 2 * 52 * O.U * ref, "rel")


def test_graph_replays():
    """The run in one captured graph, replayed on new inputs with eager work and synchronisations between."""
    need_gpu()
    for B, N, C, H in ((1, 1, 64, 256), (2, 65, 272, 8208)):
        p, dev, b = setup(B, N, C, H, BF, 7)
        g = O.gen(12)
        outs = ("t", "q", "qs", "hid", "h", "d", "o", "rel", "cache")
        block_step(dev, b)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            block_step(dev, b)
        for i in range(4):
            b["x"].copy_(O.randn((B * N, C), g, BF))
            graph.replay()
            torch.cuda.synchronize()
            got = [b[k].clone() for k in outs]
            for k in outs:
                b[k].zero_()
            block_step(dev, b)
            torch.cuda.synchronize()
            assert all(torch.equal(x, b[k]) for x, k in zip(got, outs)), i
    say("  4 replays equal the eager calls")
