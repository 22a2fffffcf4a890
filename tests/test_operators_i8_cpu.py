"""Host checks of the operators on 8-bit integers: what a call refuses, with which code, before anything is
launched; calls with nothing to do; workspace and cache sizes."""
import ctypes

import pytest

import i8_util as I
import torch
from paper_2607_27842_amd import abi
from test_operators_cpu import at, refused

E = abi


def quant(ptrs=None, **o):
    d = abi.ff_quant_i8_desc(**{**dict(rows=4, C=256, dtype=E.FF_BF16, x_row=256, q_row=256), **o})
    x = {**dict(x=at(1), q=at(2), s=at(3)), **(ptrs or {})}
    return abi.ff_quant_i8(d, x["x"], x["q"], x["s"])


def gemm_desc(**o):
    return abi.ff_gemm_i8_desc(**{**dict(M=4, N=64, K=256, a_dtype=E.FF_I8, out_dtype=E.FF_BF16, gelu=0, gate_rows=2, a_row=256,
                                         w_row=256, out_row=64, resid_row=64, gate_ld=64), **o})


def gemm(ptrs=None, bytes=1 << 30, **o):
    x = {**dict(a=at(1), a_s=at(2), w=at(3), w_s=at(4), bias=at(5), gate=at(6), resid=at(7), out=at(8), ws=at(9)), **(ptrs or {})}
    return abi.ff_gemm_i8(gemm_desc(**o), x["a"], x["a_s"], x["w"], x["w_s"], x["bias"], x["gate"], x["resid"], x["out"], x["ws"], bytes)


BRANCH = ("x", "branch", "post_gain", "gate", "pre_gain", "scale", "shift", "sum", "y", "q", "q_s")


def branch(ptrs=None, **o):
    d = abi.ff_branch_norm_desc(**{**dict(rows=4, C=256, dtype=E.FF_BF16, post=1, pre=1, gate_tanh=0, mod_rows=2, eps=1e-6,
                                          resid_scale=1.0, x_row=256, branch_row=256, sum_row=256, y_row=256, q_row=256, gate_ld=256,
                                          mod_ld=256), **o})
    x = {**{n: at(i + 1) for i, n in enumerate(BRANCH)}, **(ptrs or {})}
    return abi.ff_branch_norm_i8(d, *(x[n] for n in BRANCH))


@pytest.mark.parametrize("o,code", [
    (dict(dtype=2), E.FF_E_DTYPE), (dict(rows=-1), E.FF_E_SHAPE), (dict(rows=(1 << 23) + 1), E.FF_E_SHAPE), (dict(C=4), E.FF_E_SHAPE),
    (dict(C=252), E.FF_E_SHAPE), (dict(C=131064, x_row=131064, q_row=131064), E.FF_E_SHAPE), (dict(x_row=248), E.FF_E_SHAPE),
    (dict(x_row=260), E.FF_E_SHAPE), (dict(q_row=0), E.FF_E_SHAPE), (dict(x_row=1 << 50), E.FF_E_SHAPE)])
def test_quant_refuses(o, code):
    refused(code, quant, **o)


@pytest.mark.parametrize("p,code", [
    (dict(x=None), E.FF_E_NULL), (dict(q=None), E.FF_E_NULL), (dict(s=None), E.FF_E_NULL), (dict(x=at(1) + 8), E.FF_E_SHAPE),
    (dict(q=at(1) + 64), E.FF_E_SHAPE), (dict(s=at(2) + 512), E.FF_E_SHAPE), (dict(s=at(1)), E.FF_E_SHAPE)])
def test_quant_refuses_pointers(p, code):
    refused(code, quant, p)


@pytest.mark.parametrize("o,code", [
    (dict(a_dtype=3), E.FF_E_DTYPE), (dict(out_dtype=2), E.FF_E_DTYPE), (dict(gelu=2), E.FF_E_RANGE), (dict(gate_rows=0), E.FF_E_RANGE),
    (dict(M=-1), E.FF_E_SHAPE), (dict(M=(1 << 23) + 1), E.FF_E_SHAPE), (dict(N=60, out_row=64), E.FF_E_SHAPE), (dict(N=0), E.FF_E_SHAPE),
    (dict(N=(1 << 20) + 8, out_row=1 << 21, resid_row=1 << 21, gate_ld=0), E.FF_E_SHAPE),
    (dict(M=1 << 20, N=1 << 15, out_row=1 << 15, resid_row=1 << 15, gate_ld=0), E.FF_E_SHAPE), (dict(K=8), E.FF_E_SHAPE),
    (dict(K=250), E.FF_E_SHAPE), (dict(K=131072, a_row=131072, w_row=131072), E.FF_E_SHAPE), (dict(a_row=264), E.FF_E_SHAPE),
    (dict(a_row=240), E.FF_E_SHAPE), (dict(w_row=128), E.FF_E_SHAPE), (dict(out_row=56), E.FF_E_SHAPE), (dict(resid_row=68), E.FF_E_SHAPE),
    (dict(gate_ld=56), E.FF_E_SHAPE), (dict(gate_ld=68), E.FF_E_SHAPE), (dict(gate_ld=-64), E.FF_E_SHAPE), (dict(a_row=1 << 23), E.FF_E_SHAPE),
    (dict(w_row=1 << 23), E.FF_E_SHAPE)])
def test_gemm_refuses(o, code):
    refused(code, gemm, **o)


@pytest.mark.parametrize("p,o,code", [
    (dict(a=None), {}, E.FF_E_NULL), (dict(a_s=None), {}, E.FF_E_NULL), ({}, dict(a_dtype=E.FF_BF16), E.FF_E_NULL),
    (dict(w=None), {}, E.FF_E_NULL), (dict(w_s=None), {}, E.FF_E_NULL), (dict(out=None), {}, E.FF_E_NULL), (dict(w=at(3) + 8), {}, E.FF_E_SHAPE),
    (dict(gate=at(6) + 4), {}, E.FF_E_SHAPE), (dict(out=at(1)), {}, E.FF_E_SHAPE), (dict(out=at(2)), {}, E.FF_E_SHAPE),
    (dict(out=at(3)), {}, E.FF_E_SHAPE), (dict(out=at(4)), {}, E.FF_E_SHAPE), (dict(out=at(5)), {}, E.FF_E_SHAPE),
    (dict(out=at(6) + 256), {}, E.FF_E_SHAPE), (dict(out=at(7) + 16), {}, E.FF_E_SHAPE)])
def test_gemm_refuses_pointers(p, o, code):
    refused(code, gemm, p, **o)


def test_gemm_residual_in_place_needs_the_same_pitch():
    refused(E.FF_E_SHAPE, gemm, dict(out=at(7)), out_row=72)


def test_gemm_workspace_of_rows_in_a_float_type():
    o = dict(M=33, a_dtype=E.FF_BF16, N=72, out_row=72, resid_row=72, gate_ld=72)
    n = abi.ff_gemm_i8_workspace_bytes(gemm_desc(**o))
    assert n >= 33 * 256 + 33 * 4
    p = dict(a_s=None)
    refused(E.FF_E_WORKSPACE, gemm, p, bytes=n - 1, **o)
    refused(E.FF_E_NULL, gemm, dict(p, ws=None), **o)
    refused(E.FF_E_SHAPE, gemm, dict(p, ws=at(9) + 4), **o)
    for other in (1, 3, 4, 5, 6, 7, 8):
        refused(E.FF_E_SHAPE, gemm, dict(p, ws=at(other)), **o)
    assert abi.ff_gemm_i8_workspace_bytes(gemm_desc(M=0)) == 0
    assert abi.ff_gemm_i8_workspace_bytes(gemm_desc(K=8)) == 0


@pytest.mark.parametrize("o,code", [
    (dict(dtype=2), E.FF_E_DTYPE), (dict(post=3), E.FF_E_RANGE), (dict(pre=-1), E.FF_E_RANGE), (dict(gate_tanh=2), E.FF_E_RANGE),
    (dict(mod_rows=0), E.FF_E_RANGE), (dict(eps=0.0), E.FF_E_RANGE), (dict(eps=float("nan")), E.FF_E_RANGE),
    (dict(resid_scale=float("inf")), E.FF_E_RANGE), (dict(resid_scale=float("nan")), E.FF_E_RANGE), (dict(rows=-1), E.FF_E_SHAPE),
    (dict(rows=(1 << 23) + 1), E.FF_E_SHAPE), (dict(C=16392), E.FF_E_SHAPE), (dict(C=250), E.FF_E_SHAPE), (dict(x_row=128), E.FF_E_SHAPE),
    (dict(branch_row=257), E.FF_E_SHAPE), (dict(sum_row=8), E.FF_E_SHAPE), (dict(y_row=252), E.FF_E_SHAPE), (dict(q_row=0), E.FF_E_SHAPE),
    (dict(gate_ld=128), E.FF_E_SHAPE), (dict(mod_ld=260), E.FF_E_SHAPE), (dict(mod_ld=-8), E.FF_E_SHAPE)])
def test_branch_refuses(o, code):
    refused(code, branch, **o)


@pytest.mark.parametrize("p,code", [
    (dict(x=None), E.FF_E_NULL), (dict(sum=None, y=None, q=None, q_s=None), E.FF_E_NULL), (dict(q_s=None), E.FF_E_NULL),
    (dict(q=None), E.FF_E_NULL), (dict(branch=None), E.FF_E_NULL), (dict(branch=None, gate=None), E.FF_E_NULL),
    (dict(post_gain=at(3) + 4), E.FF_E_SHAPE), (dict(y=at(1)), E.FF_E_SHAPE), (dict(y=at(2)), E.FF_E_SHAPE), (dict(q=at(3)), E.FF_E_SHAPE),
    (dict(q=at(4) + 1024), E.FF_E_SHAPE), (dict(y=at(6) + 512), E.FF_E_SHAPE), (dict(q_s=at(7)), E.FF_E_SHAPE), (dict(y=at(8)), E.FF_E_SHAPE),
    (dict(q_s=at(9) + 16), E.FF_E_SHAPE), (dict(sum=at(1) + 16), E.FF_E_SHAPE), (dict(sum=at(5)), E.FF_E_SHAPE)])
def test_branch_refuses_pointers(p, code):
    refused(code, branch, p)


def test_branch_sum_in_place_needs_the_same_pitch():
    refused(E.FF_E_SHAPE, branch, dict(sum=at(1)), x_row=264)
    refused(E.FF_E_SHAPE, branch, dict(sum=at(2)), branch_row=264)


def test_nothing_to_do():
    none = dict.fromkeys(BRANCH + ("a", "a_s", "w", "w_s", "bias", "resid", "out", "ws", "s"))
    assert quant(none, rows=0) == 0
    assert gemm(none, bytes=0, M=0) == 0
    assert branch(none, rows=0) == 0
    refused(E.FF_E_SHAPE, gemm, none, M=0, K=8)


# ------------------------------------------------------------------ history

M2 = dict(B=2, N=5, C=24)


def model(dtype=torch.bfloat16, layers=2, **o):
    m = I.model(*{**M2, **o}.values(), dtype, layers)
    return m


def test_cache_bytes():
    for B, N, C in ((1, 1, 8), (2, 5, 24), (3, 333, 1480), (8, 256, 1152)):
        for L, S in ((1, 1), (3, 4)):
            assert abi.ff_cache_i8_bytes(model(layers=L, B=B, N=N, C=C), S) == L * S * I.slot_bytes(B, N, C)
    assert abi.ff_cache_i8_bytes(model(), 0) == 0
    bad = model()
    bad.C = 23
    assert abi.ff_cache_i8_bytes(bad, 2) == 0


def update(p=None, n_slots=3, layer=1, slot=2, mode=abi.FF_RESIDUAL, m=None):
    x = {**dict(cache=at(1), u=at(2), h=at(3)), **(p or {})}
    return abi.ff_cache_update_i8(m or model(), x["cache"], n_slots, layer, slot, x["u"], x["h"], mode)


def draft(p=None, n_slots=3, layer=1, k=1, slots=(2, 0), coeffs=(1.0, 0.5), m=None):
    x = {**dict(cache=at(1), u=at(2), h_d=at(3)), **(p or {})}
    return abi.ff_draft_forecast_i8(m or model(), x["cache"], n_slots, layer, k, slots, coeffs, x["u"], x["h_d"])


def verify(p=None, n_slots=3, layer=1, k=1, slots=(2, 0), coeffs=(1.0, 0.5), forward=1, stride=1, eps=1e-8, bytes=1 << 30, m=None):
    x = {**dict(cache=at(1), u=at(2), h_f=at(3), h_out=at(4), rel=at(5), ws=at(6)), **(p or {})}
    return abi.ff_verify_replace_i8(m or model(), x["cache"], n_slots, layer, k, slots, coeffs, x["u"], x["h_f"], x["h_out"], forward, eps,
                                    x["rel"], x["ws"], bytes, stride=stride)


def bad_model():
    m = model()
    m.dtype = 2
    return m


@pytest.mark.parametrize("o,code", [
    (dict(p=dict(cache=None)), E.FF_E_NULL), (dict(p=dict(h=None)), E.FF_E_NULL), (dict(p=dict(u=None)), E.FF_E_NULL), (dict(mode=2), E.FF_E_RANGE),
    (dict(layer=2), E.FF_E_RANGE), (dict(layer=-1), E.FF_E_RANGE), (dict(slot=3), E.FF_E_RANGE), (dict(slot=-1), E.FF_E_RANGE),
    (dict(n_slots=9), E.FF_E_RANGE), (dict(p=dict(h=at(3) + 8)), E.FF_E_SHAPE), (dict(p=dict(cache=at(1) + 8)), E.FF_E_SHAPE),
    (dict(p=dict(h=at(1) + 5 * 384)), E.FF_E_SHAPE), (dict(p=dict(u=at(1) + 5 * 384 + 16)), E.FF_E_SHAPE), (dict(m=bad_model()), E.FF_E_DTYPE)])
def test_update_refuses(o, code):
    assert I.slot_bytes(*M2.values()) == 384
    refused(code, update, **o)


@pytest.mark.parametrize("o,code", [
    (dict(p=dict(cache=None)), E.FF_E_NULL), (dict(p=dict(h_d=None)), E.FF_E_NULL), (dict(layer=2), E.FF_E_RANGE), (dict(k=4), E.FF_E_RANGE),
    (dict(k=-1), E.FF_E_RANGE), (dict(slots=(0, 3)), E.FF_E_RANGE), (dict(slots=(-1, 0)), E.FF_E_RANGE), (dict(n_slots=0), E.FF_E_RANGE),
    (dict(p=dict(h_d=at(3) + 8)), E.FF_E_SHAPE), (dict(p=dict(cache=at(1) + 4)), E.FF_E_SHAPE), (dict(p=dict(h_d=at(2) + 16)), E.FF_E_SHAPE),
    (dict(p=dict(h_d=at(1) + 6 * 384 - 16)), E.FF_E_SHAPE)])
def test_draft_refuses(o, code):
    refused(code, draft, **o)


@pytest.mark.parametrize("o,code", [
    (dict(p=dict(h_f=None)), E.FF_E_NULL), (dict(p=dict(h_out=None)), E.FF_E_NULL), (dict(p=dict(ws=None)), E.FF_E_NULL),
    (dict(forward=4), E.FF_E_RANGE), (dict(forward=2, stride=0), E.FF_E_RANGE), (dict(eps=0.0), E.FF_E_RANGE), (dict(slots=(3, 0)), E.FF_E_RANGE),
    (dict(bytes=16), E.FF_E_WORKSPACE), (dict(p=dict(h_out=at(3))), E.FF_E_SHAPE), (dict(p=dict(h_out=at(2) + 16)), E.FF_E_SHAPE),
    (dict(p=dict(h_out=at(1))), E.FF_E_SHAPE), (dict(p=dict(ws=at(2))), E.FF_E_SHAPE), (dict(p=dict(ws=at(3))), E.FF_E_SHAPE),
    (dict(p=dict(ws=at(4))), E.FF_E_SHAPE), (dict(p=dict(ws=at(1))), E.FF_E_SHAPE), (dict(p=dict(rel=at(6))), E.FF_E_SHAPE),
    (dict(p=dict(rel=at(4))), E.FF_E_SHAPE), (dict(p=dict(rel=at(1))), E.FF_E_SHAPE), (dict(p=dict(rel=at(5) + 2)), E.FF_E_SHAPE)])
def test_verify_refuses(o, code):
    refused(code, verify, **o)


def test_the_format_on_the_cpu():
    """The tests' own formula: within half a step, zeros as zeros, NaN rows kept apart."""
    x = torch.randn(7, 40, generator=torch.Generator().manual_seed(0)) * torch.tensor([1e-30, 1.0, 5e37, 0.0, 2.0 ** -120, 1.0, 1.0])[:, None]
    x[5, 3], x[6, 0] = float("nan"), float("-inf")
    q, s = I.quantise(x)
    assert torch.isfinite(x[:5]).all() and q[:5].abs().max() == 127 and (q[3] == 0).all() and (q[5:] == 0).all() and torch.isnan(s[5:]).all()
    assert ((q[:5].double() * s[:5].double()[:, None] - x[:5].double()).abs() <= 0.5 * s[:5].double()[:, None] * (1 + 2.0 ** -14)).all()
    assert ctypes.sizeof(abi.ff_gemm_i8_desc) == 72 and ctypes.sizeof(abi.ff_branch_norm_desc) == 96 and ctypes.sizeof(abi.ff_quant_i8_desc) == 32
