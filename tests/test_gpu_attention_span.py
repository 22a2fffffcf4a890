"""Attention over spans against its plain 64-bit form: both kernels, types, head layouts, masks, biases,
strides, long caches, rows without keys, infinities and NaN in rows that a query does not see."""
import math

import pytest
import torch

import op_util as O
from gpu_util import need_gpu, say
from paper_2607_27842_amd import abi

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NONE, SLOPE, TABLE = abi.FF_BIAS_NONE, abi.FF_BIAS_SLOPE, abi.FF_BIAS_TABLE
LOWEST = torch.finfo(torch.float32).min


def inputs(B, H, Hkv, d, nq, nk, dtype, seed=0):
    g = O.gen(seed + nq * 31 + nk)
    return O.randn((B, nq, H, d), g, dtype), O.randn((B, nk, Hkv, d), g, dtype), O.randn((B, nk, Hkv, d), g, dtype)


def spans_of(kind, B, nq, nk, seed=0):
    """int32 [B, nq, s, 2]"""
    g = O.gen(seed + 5)
    i = torch.arange(nq)
    z = torch.zeros_like(i)
    rows = []
    for b in range(B):
        if kind == "causal":
            rows.append(torch.stack([z, i + 1 + nk - nq], -1)[:, None])
        elif kind == "docs":         # documents of 1, 3, 17, 60, 130, ... tokens
            cut = torch.tensor([1, 3, 17, 60, 130, 64, 300] * 40)
            first = (torch.cumsum(cut, 0) - cut).repeat_interleave(cut)[:nq]
            rows.append(torch.stack([first, torch.minimum(i + 1, torch.tensor(nk))], -1)[:, None])
        elif kind == "prefix":       # padded batch: rows behind the length see nothing
            n, p = nk - 3 * b - 1, nk // 3
            s = torch.stack([z, torch.maximum(i + 1, torch.tensor(p)).clamp_max(n)], -1)
            rows.append(torch.where((i < n)[:, None], s, 0)[:, None])
        elif kind == "joint":        # padded text before image rows
            t, l = nk // 3, nk // 3 - 5 * b - 2
            s = torch.tensor([[0, l], [t, nk]]).expand(nq, 2, 2)
            rows.append(torch.where(((i < l) | (i >= t))[:, None, None], s, 0))
        elif kind == "overlap":      # a window and a global prefix that may meet; order either way
            w = torch.stack([(i - 20).clamp_min(0), i + 1], -1)
            p = torch.stack([z, z + 30], -1)
            rows.append(torch.stack([w, p] if b % 2 else [p, w], 1))
        elif kind == "wild":         # any numbers: cut to the keys, first >= end sees nothing
            rows.append(torch.randint(-2 * nk, 3 * nk, (nq, 2, 2), generator=g))
        elif kind == "empty":
            rows.append(torch.stack([z + nk // 2, z + nk // 2], -1)[:, None])
    return torch.stack(rows).to(torch.int32).contiguous()


def check(q, k, v, spans=None, **o):
    need_gpu()
    d = q.shape[3]
    scale = o.pop("scale", 1 / math.sqrt(d))
    gpu = {n: t.cuda() if torch.is_tensor(t) else t for n, t in o.items()}
    out = O.attention_call(q.cuda(), k.cuda(), v.cuda(), scale, spans=spans.cuda() if spans is not None else None, **gpu)
    ref, tol = O.attention_ref(q, k, v, scale, spans=spans, **o)
    O.close(out, ref, tol, "attention")
    return out


# Few rows go through the kernel that reads keys straight from memory, many (per key head) through the tiled
# one in bf16; the sizes below lie on both sides.
FEW, MANY = (2, 4, 2), (1, 16, 16)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("d", [8, 32, 40, 64, 72, 96, 104, 128])
@pytest.mark.parametrize("heads,n", [(FEW, 1), (FEW, 2), (FEW, 33), (FEW, 65), (MANY, 577)], ids=str)
def test_head_dims(dtype, d, heads, n):
    B, H, Hkv = heads
    check(*inputs(B, H, Hkv, d, n, n, dtype))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["causal", "docs", "prefix", "joint", "overlap", "wild", "empty"])
@pytest.mark.parametrize("heads,n,d", [(FEW, 50, 64), ((2, 3, 1), 130, 40), ((2, 10, 5), 700, 64), (MANY, 650, 128)], ids=str)
def test_masks(dtype, kind, heads, n, d):
    B, H, Hkv = heads
    if dtype == F32 and n > 200:
        n = 257
    out = check(*inputs(B, H, Hkv, d, n, n, dtype), spans_of(kind, B, n, n))
    if kind == "empty":
        assert (out == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("cap", [0.0, 3.0, 50.0])
@pytest.mark.parametrize("bias,reach", [(NONE, 0), (SLOPE, 0), (TABLE, 0), (TABLE, 7), (TABLE, 100)])
@pytest.mark.parametrize("heads,n,d", [(FEW, 70, 64), (MANY, 600, 128), ((4, 12, 12), 420, 64)], ids=str)
def test_caps_and_biases(dtype, cap, bias, reach, heads, n, d):
    B, H, Hkv = heads
    if dtype == F32 and n > 200:
        n = 200
    g = O.gen(2)
    b = {NONE: None, SLOPE: torch.exp2(-8.0 * torch.arange(1, H + 1) / H), TABLE: O.randn((H, 2 * reach + 1), g)}[bias]
    pos = torch.tensor([3, -5, 0, 11][:B], dtype=torch.int32) if bias != NONE and cap != 3.0 else None
    q, k, v = inputs(B, H, Hkv, d, n, n, dtype)
    check(2 * q, k, v, spans_of("causal", B, n, n) if reach == 7 else None, cap=cap, bias_kind=bias, bias=b, reach=reach, pos=pos)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("heads,n", [(FEW, 60), (MANY, 600)], ids=str)
def test_bias_of_minus_infinity_and_of_the_lowest_value(dtype, heads, n):
    """-inf hides a key; the type's lowest value is a score: rows that have nothing else share their weight
    evenly.  A row of -inf alone gets zeros."""
    B, H, Hkv = heads
    n = 150 if dtype == F32 and n > 200 else n
    q, k, v = inputs(B, H, Hkv, 64, n, n, dtype)
    reach = n
    t = torch.zeros(H, 2 * reach + 1)
    t[:, reach + 1:] = -math.inf                    # causal by the table
    check(q, k, v, bias_kind=TABLE, bias=t, reach=reach)
    t[:, reach + 1:] = LOWEST
    check(q, k, v, bias_kind=TABLE, bias=t, reach=reach)
    t[:] = LOWEST
    check(q, k, v, bias_kind=TABLE, bias=t, reach=reach)
    t[:] = -math.inf
    out = check(q, k, v, bias_kind=TABLE, bias=t, reach=reach)
    assert (out == 0).all()
    t = torch.full((H, 1), LOWEST)
    check(q, k, v, spans_of("prefix", B, n, n), bias_kind=TABLE, bias=t, reach=0)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B,H,Hkv,d,nq,nk", [(1, 4, 1, 128, 1, 5000), (3, 16, 2, 128, 1, 3001), (2, 8, 8, 64, 1, 700), (1, 20, 5, 72, 5, 2100),
                                             (2, 4, 4, 128, 16, 1200), (1, 40, 1, 96, 1, 4097), (1, 8, 1, 40, 3, 9000)])
def test_cache_of_ragged_lengths(dtype, B, H, Hkv, d, nq, nk):
    """Single and few tokens at the end of caches whose rows behind the length hold NaN; the bias goes by the
    tokens' positions."""
    q, k, v = inputs(B, H, Hkv, d, nq, nk, dtype)
    lens = [nk, max(nq, nk // 3), nq + 1][:B]
    i = torch.arange(nq)
    sp = torch.stack([torch.stack([torch.zeros_like(i), l - nq + i + 1], -1)[:, None] for l in lens]).to(torch.int32)
    for b, l in enumerate(lens):
        k[b, l:] = math.nan
        v[b, l:] = math.nan
    pos = torch.tensor([l - nq for l in lens], dtype=torch.int32)
    check(q, k, v, sp)
    check(q, k, v, sp, cap=20.0, bias_kind=SLOPE, bias=torch.full((H,), 2.0 ** -7), pos=pos)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("heads,n,d", [(FEW, 90, 64), (FEW, 90, 40), (MANY, 600, 128), (MANY, 600, 72), ((4, 12, 12), 400, 64)], ids=str)
@pytest.mark.parametrize("kind", ["causal", "prefix", "joint"])
def test_unseen_rows_may_hold_anything(dtype, heads, n, d, kind):
    """Infinities and NaN in keys and values reach the queries that see them and no other."""
    B, H, Hkv = heads
    n = 150 if dtype == F32 and n > 200 else n
    q, k, v = inputs(B, H, Hkv, d, n, n, dtype)
    sp = spans_of(kind, B, n, n)
    at = n - 9 if kind == "causal" else n // 2
    v[:, at, :, 3] = math.inf
    v[:, at + 5, :, d - 1] = -math.inf
    if kind == "prefix":
        k[:, n - 1:], v[:, n - 1:] = math.nan, math.nan      # behind every length
        q[:, n - 1:] = math.nan                              # rows without keys: zeros all the same
    if kind == "joint":
        l, t = n // 3 - 5 * (B - 1) - 2, n // 3
        k[B - 1, l:t], v[B - 1, l:t], q[B - 1, l:t] = math.nan, math.nan, math.inf
    check(q, k, v, sp)
    if kind == "causal":                                     # a key with a NaN spoils the rows that see it
        k[:, at - 20, :, 1] = math.nan
        out = O.attention_call(q.cuda(), k.cuda(), v.cuda(), 0.125, spans=sp.cuda()).cpu()
        bad = torch.isnan(out)
        assert bad[:, at - 20:].all() and not bad[:, :at - 20].any()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("d", [8, 24, 48, 80, 96, 104, 128])
def test_unseen_rows_by_head_dim(dtype, d):
    """An infinity in each dim of V, the dims' signs mixed, in keys that part of a step's rows see."""
    q, k, v = inputs(2, 4, 2, d, 75, 75, dtype)
    for e in range(d):
        v[:, 40 + e % 30, e % 2, e] = math.inf if e % 3 else -math.inf
    v[0, 71, 1, d // 2] = math.nan
    check(q, k, v, spans_of("causal", 2, 75, 75))


@pytest.mark.parametrize("B,H", [(5, 8), (2, 12), (3, 11), (2, 10), (1, 7), (12, 8)])
@pytest.mark.parametrize("kind", ["causal", None])
def test_heads_over_the_grid(B, H, kind):
    """Every head's every row has its place, however the heads divide."""
    n = 400
    check(*inputs(B, H, H, 64, n, n, BF), spans_of(kind, B, n, n) if kind else None)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("heads,n", [((2, 4, 4), 45), ((2, 4, 4), 700)], ids=str)
def test_layouts(dtype, heads, n):
    """One projection's [B, N, 3, H, d] result; head-major keys; one sample's keys for all; head-major output
    in a wider buffer, whose other columns stay."""
    need_gpu()
    B, H, _ = heads
    n = 150 if dtype == F32 and n > 200 else n
    d = 64
    g = O.gen(n)
    qkv = O.randn((B, n, 3, H, d), g, dtype)
    dq = qkv.cuda()
    q, k, v = qkv.unbind(2)
    ref, tol = O.attention_ref(q, k, v, 0.125)
    O.close(O.attention_call(*dq.unbind(2), 0.125, out=torch.empty(B, n, H, d, dtype=dtype, device="cuda")), ref, tol, "packed")
    km, vm = (t.transpose(1, 2).contiguous().cuda().transpose(1, 2) for t in (k, v))
    buf = torch.full((B, H, n, d + 24), 5.0, dtype=dtype, device="cuda")
    O.attention_call(dq[:, :, 0], km, vm, 0.125, out=buf[..., :d].transpose(1, 2))
    O.close(buf[..., :d].transpose(1, 2), ref, tol, "head major")
    assert (buf[..., d:] == 5.0).all()
    k1, v1 = (t[:1].expand(B, n, H, d) for t in (k, v))
    ref, tol = O.attention_ref(q, k1, v1, 0.125)
    dk, dv = (t[:1].contiguous().cuda().expand(B, n, H, d) for t in (k, v))
    O.close(O.attention_call(dq[:, :, 0], dk, dv, 0.125, out=torch.empty(B, n, H, d, dtype=dtype, device="cuda")), ref, tol, "shared keys")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n,d", [(45, 72), (150, 48), (700, 64)])
def test_output_beside_its_operands(dtype, n, d):
    """A [B, N, 4, H, d] buffer whose last quarter takes the output; the fp32 kernel's loads of V run into it."""
    need_gpu()
    n = 150 if dtype == F32 and n > 200 else n
    x = O.randn((2, n, 4, 4, d), O.gen(n + d), dtype)
    x[:, :, 3] = math.nan
    dx = x.cuda()
    sp = spans_of("causal", 2, n, n)
    q, k, v, out = dx.unbind(2)
    O.attention_call(q, k, v, 0.125, spans=sp.cuda(), out=out)
    ref, tol = O.attention_ref(*x.unbind(2)[:3], 0.125, spans=sp)
    O.close(out, ref, tol, "attention")
    assert torch.equal(dx[:, :, :3].cpu(), x[:, :, :3])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_shared_spans_and_no_keys(dtype):
    need_gpu()
    q, k, v = inputs(3, 4, 2, 64, 20, 20, dtype)
    sp = spans_of("causal", 1, 20, 20)
    check(q, k, v, sp)
    out = O.attention_call(q.cuda(), k[:, :0].cuda(), v[:, :0].cuda(), 0.125)
    assert (out == 0).all()
    big, _, _ = inputs(1, 16, 16, 128, 700, 1, dtype)
    none = torch.empty(1, 0, 16, 128, dtype=dtype, device="cuda")
    assert (O.attention_call(big.cuda(), none, none, 0.125) == 0).all()
    check(big, *inputs(1, 16, 16, 128, 700, 1, dtype)[1:])


@pytest.mark.parametrize("dtype,nq", [(BF, 1), (F32, 1), (BF, 700)])
def test_keys_past_32_bit_offsets(dtype, nq):
    """Keys whose rows lie up to 5 GB apart in a cache."""
    need_gpu()
    nk, pitch, d = (70000, 40 * 1024, 64) if dtype == BF else (35000, 40 * 1024, 64)
    g = O.gen(8)
    H = 4 if nq == 1 else 2
    q = O.randn((1, nq, H, d), g, dtype)
    kv = torch.empty(nk * pitch, dtype=dtype, device="cuda").view(1, nk, pitch)
    near = torch.cat([torch.arange(0, 300), torch.arange(nk - 700, nk)])
    x = O.randn((1, len(near), 2 * d), g, dtype)
    kv[:, near, :2 * d] = x.cuda()
    k, v = (kv[..., i * d:i * d + d].unsqueeze(2) for i in (0, 1))
    sp = torch.tensor([[0, 300], [nk - 700, nk]], dtype=torch.int32).expand(1, nq, 2, 2).contiguous()
    out = O.attention_call(q.cuda(), k, v, 0.125, spans=sp.cuda())
    ref, tol = O.attention_ref(q, x[..., :d].unsqueeze(2), x[..., d:].unsqueeze(2), 0.125)
    O.close(out, ref, tol, "far keys")


def test_same_bits_again_graphs_and_streams():
    """Two calls at once on two streams (a workspace each), and a captured graph replayed on new inputs with
    eager work between."""
    need_gpu()
    g = O.gen(6)
    for B, H, Hkv, d, nq, nk in ((2, 8, 2, 128, 1, 4000), (1, 16, 16, 128, 640, 640), (2, 4, 4, 64, 40, 40)):
        q, k, v = (t.cuda() for t in inputs(B, H, Hkv, d, nq, nk, BF))
        sp = spans_of("causal", B, nq, nk).cuda()
        a = O.attention_call(q, k, v, 0.1, spans=sp)
        outs = []
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for s in streams:
            with torch.cuda.stream(s):
                outs.append([O.attention_call(q, k, v, 0.1, spans=sp) for _ in range(3)])
        torch.cuda.synchronize()
        assert all(torch.equal(a, o) for os in outs for o in os)
        out, ws = torch.empty_like(q), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            O.attention_call(q, k, v, 0.1, spans=sp, out=out, ws=ws)
            O.attention_call(out, k, v, 0.1, spans=sp, out=a, ws=ws)       # follows, in the same workspace
        for _ in range(3):
            q.copy_(O.randn(q.shape, g, BF))
            graph.replay()
            torch.cuda.synchronize()
            got = [out.clone(), a.clone()]
            one = O.attention_call(q, k, v, 0.1, spans=sp)
            two = O.attention_call(one, k, v, 0.1, spans=sp)
            torch.cuda.synchronize()
            assert torch.equal(got[0], one) and torch.equal(got[1], two)


def test_sublayers_together():
    """A text tower's attention and MLP sub-layers as they are run: norm to 8 bits, q / k / v product, packed
    prompts' attention on the product's own rows, quantisation, output product with the residual, norm,
    MLP with GELU; against 64 bits with the same 8-bit operands' formula.

    Tolerance, normwise: five results rounded to bf16 (2^-8 each), and values that their roundings carry
    over a border of e4m3: a step is 2^-3 of a value, a change of 2^-8 crosses a border for one value in
    16, which moves an operand by sqrt(1/16) 2^-3 of its norm at most; four operands, in quadrature."""
    need_gpu()
    from test_gpu_operators_q8 import norm_call
    g = O.gen(21)
    n, C, H, Hkv, d, M = 300, 512, 8, 4, 64, 1096
    x = O.randn((n, C), g, BF)
    W = {w: O.quantise(O.randn(s, g, std=1 / math.sqrt(s[1])), 128) for w, s in
         (("qkv", ((H + 2 * Hkv) * d, C)), ("o", (C, H * d)), ("up", (M, C)), ("down", (C, M + 8)))}
    g1, g2 = (1 + 0.1 * O.randn((2, C), g)).to(BF)
    sp = spans_of("docs", 1, n, n)
    D = {k: (a.cuda(), s.cuda()) for k, (a, s) in W.items()}
    new = lambda *s, t=BF: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731

    def quant(t):
        q, s = new(*t.shape, t=torch.uint8), new(-(-t.shape[1] // 128), t.shape[0], t=F32)
        abi.ff_quant_q8(abi.ff_quant_desc(rows=t.shape[0], C=t.shape[1], dtype=abi.FF_BF16, block_rows=1, x_row=t.stride(0),
                                          q_row=q.stride(0), qs_ld=s.stride(0)), O.ptr(t), O.ptr(q), O.ptr(s), O.stream())
        return q, s

    dx = x.cuda()
    q8, qs = new(n, C, t=torch.uint8), new(4, n, t=F32)
    norm_call(dx, None, g1.cuda(), None, None, q8, qs)
    qkv = O.gemm_call(q8, qs, *D["qkv"]).view(1, n, H + 2 * Hkv, d)
    att = O.attention_call(qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:], 0.125, cap=30.0, spans=sp.cuda(),
                           out=new(1, n, H, d))
    o = O.gemm_call(*quant(att.view(n, H * d)), *D["o"])
    s = new(n, C)
    norm_call(dx, o, g2.cuda(), s, None, q8, qs)
    hid = new(n, M + 8).zero_()                    # K % 16 == 0 for the second product
    O.gemm_call(q8, qs, *D["up"], gelu=True, out=hid[:, :M])
    y = O.gemm_call(*quant(hid), *D["down"], resid=s, out=s)

    def de(q, s, br):
        return q.double() * O.spread(s.double(), br, *q.shape)

    def q64(t):                                    # the values that 8 bits stand for
        return de(*O.quantise(t.float(), 1), 1)

    def rms(t, gain):
        return t / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-6) * gain.double()

    X = x.double()
    w = {k: de(*v, 128) for k, v in W.items()}
    p = (q64(rms(X, g1)) @ w["qkv"].t()).view(1, n, H + 2 * Hkv, d)
    A, _ = O.attention_ref(p[:, :, :H].to(BF), p[:, :, H:H + Hkv].to(BF), p[:, :, H + Hkv:].to(BF), 0.125, cap=30.0, spans=sp)
    S = X + q64(A.view(n, H * d)) @ w["o"].t()
    u = q64(rms(S, g2)) @ w["up"].t()
    u = u * 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3)))
    Y = S + q64(torch.nn.functional.pad(u, (0, 8))) @ w["down"].t()
    err = float((y.cpu().double() - Y).norm() / Y.norm())
    tol = 5 * 2.0 ** -8 + 2 * 2.0 ** -5            # sqrt(4) operands of sqrt(1/16) 2^-3
    say("  two sub-layers: normwise error %.3g (tolerance %.3g)" % (err, tol))
    assert err <= tol
