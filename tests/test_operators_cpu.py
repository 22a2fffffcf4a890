"""Host checks of the operators on 8-bit operands and of attention over spans: what a call refuses, with
which code, before anything is launched; calls with nothing to do; workspace sizes."""
import pytest

from paper_2607_27842_amd import abi

E = abi
P = 1 << 20        # addresses that no call here reaches: every one of them is refused, or has nothing to do
NAMES = ("quant", "norm", "gemm", "attn")


def at(i):
    return P + (i << 32)


def quant(ptrs=None, **o):
    d = abi.ff_quant_desc(**{**dict(rows=4, C=256, dtype=E.FF_BF16, block_rows=1, x_row=256, q_row=256, qs_ld=4), **o})
    x = {**dict(x=at(1), q=at(2), qs=at(3)), **(ptrs or {})}
    return abi.ff_quant_q8(d, x["x"], x["q"], x["qs"])


def norm(ptrs=None, **o):
    d = abi.ff_norm_desc(**{**dict(rows=4, C=256, dtype=E.FF_BF16, eps=1e-6, x_row=256, resid_row=256, sum_row=256, y_row=256,
                                   q_row=256, qs_ld=4), **o})
    x = {**dict(x=at(1), resid=at(2), gain=at(3), sum=at(4), y=at(5), q=at(6), qs=at(7)), **(ptrs or {})}
    return abi.ff_rms_norm_q8(d, x["x"], x["resid"], x["gain"], x["sum"], x["y"], x["q"], x["qs"])


def gemm_desc(**o):
    return abi.ff_gemm_q8_desc(**{**dict(M=4, N=64, K=256, out_dtype=E.FF_BF16, gelu=0, a_row=256, w_row=256, out_row=64,
                                         resid_row=64, as_ld=4, ws_ld=2), **o})


def gemm(ptrs=None, bytes=1 << 30, **o):
    x = {**dict(a=at(1), a_s=at(2), w=at(3), w_s=at(4), bias=at(5), resid=at(6), out=at(7), ws=at(8)), **(ptrs or {})}
    return abi.ff_gemm_q8(gemm_desc(**o), x["a"], x["a_s"], x["w"], x["w_s"], x["bias"], x["resid"], x["out"], x["ws"], bytes)


def attn_desc(**o):
    return abi.ff_attn_desc(**{**dict(
        dtype=E.FF_BF16, B=2, H=4, H_kv=2, d=64, n_q=8, n_k=8, bias_kind=E.FF_BIAS_NONE, bias_reach=0, n_spans=0, span_batch=0,
        q_batch=2048, q_row=256, q_head=64, k_batch=1024, k_row=128, k_head=64, v_batch=1024, v_row=128, v_head=64,
        o_batch=2048, o_row=256, o_head=64, scale=0.125, cap=0.0), **o})


def attn(ptrs=None, bytes=1 << 30, **o):
    x = {**dict(q=at(1), k=at(2), v=at(3), bias=None, pos=None, spans=None, out=at(7), ws=at(8)), **(ptrs or {})}
    return abi.ff_attention(attn_desc(**o), x["q"], x["k"], x["v"], x["bias"], x["pos"], x["spans"], x["out"], x["ws"], bytes)


def refused(code, call, *a, **k):
    with pytest.raises(abi.FFError) as e:
        call(*a, **k)
    assert e.value.status == code, e.value
    assert abi.ff_last_error()


@pytest.mark.parametrize("o,code", [
    (dict(dtype=7), E.FF_E_DTYPE), (dict(block_rows=2), E.FF_E_RANGE), (dict(rows=-1), E.FF_E_SHAPE), (dict(C=4), E.FF_E_SHAPE),
    (dict(C=252), E.FF_E_SHAPE), (dict(x_row=248), E.FF_E_SHAPE), (dict(x_row=260), E.FF_E_SHAPE), (dict(q_row=248), E.FF_E_SHAPE),
    (dict(rows=(1 << 23) + 1, qs_ld=1 << 24), E.FF_E_SHAPE), (dict(qs_ld=3), E.FF_E_SHAPE), (dict(block_rows=128, qs_ld=1), E.FF_E_SHAPE), (dict(x_row=1 << 50), E.FF_E_SHAPE)])
def test_quant_refuses(o, code):
    refused(code, quant, **o)


@pytest.mark.parametrize("p,code", [
    (dict(x=None), E.FF_E_NULL), (dict(q=None), E.FF_E_NULL), (dict(qs=None), E.FF_E_NULL), (dict(x=at(1) + 8), E.FF_E_SHAPE),
    (dict(q=at(1) + 64), E.FF_E_SHAPE), (dict(qs=at(2) + 512), E.FF_E_SHAPE)])
def test_quant_refuses_pointers(p, code):
    refused(code, quant, p)


@pytest.mark.parametrize("o,code", [
    (dict(dtype=2), E.FF_E_DTYPE), (dict(eps=0.0), E.FF_E_RANGE), (dict(eps=float("nan")), E.FF_E_RANGE), (dict(rows=-1), E.FF_E_SHAPE), (dict(rows=(1 << 23) + 1, qs_ld=1 << 24), E.FF_E_SHAPE),
    (dict(C=16392, x_row=16392), E.FF_E_SHAPE), (dict(C=250), E.FF_E_SHAPE), (dict(x_row=128), E.FF_E_SHAPE),
    (dict(resid_row=257), E.FF_E_SHAPE), (dict(sum_row=8), E.FF_E_SHAPE), (dict(y_row=252), E.FF_E_SHAPE),
    (dict(q_row=0), E.FF_E_SHAPE), (dict(qs_ld=3), E.FF_E_SHAPE)])
def test_norm_refuses(o, code):
    refused(code, norm, **o)


@pytest.mark.parametrize("p,code", [
    (dict(x=None), E.FF_E_NULL), (dict(y=None, q=None, qs=None), E.FF_E_NULL), (dict(qs=None), E.FF_E_NULL), (dict(q=None), E.FF_E_NULL),
    (dict(resid=None), E.FF_E_NULL), (dict(gain=at(3) + 4), E.FF_E_SHAPE), (dict(y=at(1)), E.FF_E_SHAPE), (dict(q=at(3)), E.FF_E_SHAPE),
    (dict(y=at(4)), E.FF_E_SHAPE), (dict(sum=at(1) + 16), E.FF_E_SHAPE)])
def test_norm_refuses_pointers(p, code):
    refused(code, norm, p)


def test_norm_sum_in_place_needs_the_same_pitch():
    refused(E.FF_E_SHAPE, norm, dict(sum=at(2)), resid_row=264)


@pytest.mark.parametrize("o,code", [
    (dict(out_dtype=3), E.FF_E_DTYPE), (dict(gelu=2), E.FF_E_RANGE), (dict(M=-1), E.FF_E_SHAPE), (dict(M=(1 << 23) + 1, as_ld=1 << 24), E.FF_E_SHAPE),
    (dict(N=(1 << 20) + 8, out_row=1 << 21, resid_row=1 << 21), E.FF_E_SHAPE), (dict(N=60, out_row=64), E.FF_E_SHAPE),
    (dict(N=0), E.FF_E_SHAPE), (dict(K=8), E.FF_E_SHAPE), (dict(K=250), E.FF_E_SHAPE), (dict(a_row=264), E.FF_E_SHAPE),
    (dict(w_row=128), E.FF_E_SHAPE), (dict(out_row=56), E.FF_E_SHAPE), (dict(resid_row=68), E.FF_E_SHAPE), (dict(as_ld=3), E.FF_E_SHAPE),
    (dict(ws_ld=1), E.FF_E_SHAPE), (dict(a_row=1 << 23), E.FF_E_SHAPE), (dict(as_ld=1 << 28), E.FF_E_SHAPE)])
def test_gemm_refuses(o, code):
    refused(code, gemm, **o)


@pytest.mark.parametrize("p,code", [
    (dict(a=None), E.FF_E_NULL), (dict(a_s=None), E.FF_E_NULL), (dict(w=None), E.FF_E_NULL), (dict(w_s=None), E.FF_E_NULL),
    (dict(out=None), E.FF_E_NULL), (dict(w=at(3) + 8), E.FF_E_SHAPE), (dict(out=at(1)), E.FF_E_SHAPE), (dict(out=at(6) + 16), E.FF_E_SHAPE),
    (dict(out=at(5)), E.FF_E_SHAPE)])
def test_gemm_refuses_pointers(p, code):
    refused(code, gemm, p)


def test_gemm_residual_in_place_needs_the_same_pitch():
    refused(E.FF_E_SHAPE, gemm, dict(out=at(6)), out_row=72)


@pytest.mark.parametrize("off", [8, 56, 72, 120, -8, -120])
def test_columns_of_one_buffer_that_overlap(off):
    """Rows of 64 columns every 128, `off` columns apart."""
    refused(E.FF_E_SHAPE, gemm, dict(out=at(6) + 2 * off), out_row=128, resid_row=128)
    if off > 0:
        refused(E.FF_E_SHAPE, attn, dict(out=at(1) + 8 * off), q_row=512, o_row=512, q_batch=4096, o_batch=4096)
        refused(E.FF_E_SHAPE, attn, dict(out=at(2) + 4 * off), k_row=256, o_row=256, k_batch=2048 + 128, o_batch=2048)


def test_gemm_workspace():
    big = dict(M=128, N=2048, K=8192, a_row=8192, w_row=8192, out_row=2048, resid_row=2048, as_ld=128, ws_ld=64)
    n = abi.ff_gemm_q8_workspace_bytes(gemm_desc(**big))
    assert n > 0 and n % (128 * 2048 * 4) == 0
    refused(E.FF_E_WORKSPACE, gemm, bytes=n - 1, **big)
    refused(E.FF_E_NULL, gemm, dict(ws=None), **big)
    refused(E.FF_E_SHAPE, gemm, dict(ws=at(8) + 4), **big)
    refused(E.FF_E_SHAPE, gemm, dict(ws=at(7)), **big)
    refused(E.FF_E_SHAPE, gemm, dict(ws=at(3)), **big)
    assert abi.ff_gemm_q8_workspace_bytes(gemm_desc(M=0)) == 0
    assert abi.ff_gemm_q8_workspace_bytes(gemm_desc(K=8)) == 0


@pytest.mark.parametrize("o,code", [
    (dict(dtype=5), E.FF_E_DTYPE), (dict(B=0), E.FF_E_SHAPE), (dict(H=3), E.FF_E_SHAPE), (dict(H_kv=0), E.FF_E_SHAPE),
    (dict(d=4), E.FF_E_SHAPE), (dict(d=68), E.FF_E_SHAPE), (dict(d=136), E.FF_E_SHAPE), (dict(n_q=-1), E.FF_E_SHAPE),
    (dict(n_k=-1), E.FF_E_SHAPE), (dict(n_k=1 << 30), E.FF_E_SHAPE), (dict(n_q=1 << 28), E.FF_E_SHAPE),
    (dict(B=1 << 23, n_q=1, q_batch=256, o_batch=256, q_row=256, o_row=256), E.FF_E_SHAPE), (dict(q_row=260), E.FF_E_SHAPE),
    (dict(k_head=-64), E.FF_E_SHAPE), (dict(k_row=1 << 24), E.FF_E_SHAPE), (dict(o_head=56), E.FF_E_SHAPE), (dict(o_row=192), E.FF_E_SHAPE),
    (dict(o_batch=1024), E.FF_E_SHAPE), (dict(o_batch=0), E.FF_E_SHAPE), (dict(scale=0.0), E.FF_E_RANGE),
    (dict(scale=float("inf")), E.FF_E_RANGE), (dict(cap=-1.0), E.FF_E_RANGE), (dict(cap=float("nan")), E.FF_E_RANGE),
    (dict(bias_kind=3), E.FF_E_RANGE), (dict(bias_kind=2, bias_reach=-1), E.FF_E_RANGE), (dict(n_spans=3), E.FF_E_RANGE),
    (dict(n_spans=1, span_batch=-1), E.FF_E_SHAPE)])
def test_attention_refuses(o, code):
    refused(code, attn, **o)


@pytest.mark.parametrize("p,o,code", [
    (dict(q=None), {}, E.FF_E_NULL), (dict(k=None), {}, E.FF_E_NULL), (dict(v=None), {}, E.FF_E_NULL), (dict(out=None), {}, E.FF_E_NULL),
    (dict(bias=at(4)), {}, E.FF_E_NULL), ({}, dict(bias_kind=1), E.FF_E_NULL), (dict(spans=at(4)), {}, E.FF_E_NULL),
    ({}, dict(n_spans=1), E.FF_E_NULL), (dict(k=at(2) + 2), {}, E.FF_E_SHAPE), (dict(out=at(1) + 512), {}, E.FF_E_SHAPE),
    (dict(out=at(2)), {}, E.FF_E_SHAPE), (dict(spans=at(7) + 64), dict(n_spans=1, span_batch=16), E.FF_E_SHAPE),
    (dict(pos=at(7)), {}, E.FF_E_SHAPE), (dict(bias=at(7)), dict(bias_kind=2, bias_reach=4), E.FF_E_SHAPE)])
def test_attention_refuses_pointers(p, o, code):
    refused(code, attn, p, **o)


def test_attention_workspace():
    long = dict(n_q=1, n_k=30000, k_batch=30000 * 128, v_batch=30000 * 128, q_batch=256, o_batch=256)
    n = abi.ff_attention_workspace_bytes(attn_desc(**long))
    assert n > 0
    refused(E.FF_E_WORKSPACE, attn, bytes=n - 1, **long)
    refused(E.FF_E_NULL, attn, dict(ws=None), **long)
    refused(E.FF_E_SHAPE, attn, dict(ws=at(7)), **long)
    refused(E.FF_E_SHAPE, attn, dict(ws=at(3)), **long)
    assert abi.ff_attention_workspace_bytes(attn_desc()) == 0
    assert abi.ff_attention_workspace_bytes(attn_desc(n_q=0)) == 0
    assert abi.ff_attention_workspace_bytes(attn_desc(d=4)) == 0


def test_nothing_to_do():
    """No rows: success without a launch, as long as the descriptor is right."""
    none = dict.fromkeys(("x", "resid", "gain", "sum", "y", "q", "qs", "a", "a_s", "w", "w_s", "bias", "out", "ws", "k", "v", "pos", "spans"))
    assert quant(none, rows=0, qs_ld=0) == 0
    assert norm(none, rows=0) == 0
    assert gemm(none, bytes=0, M=0) == 0
    assert attn(none, bytes=0, n_q=0) == 0
    refused(E.FF_E_SHAPE, gemm, none, M=0, K=8)
