"""Operators of the text tower and of 8-bit inference beside the denoiser, each with its plain form.

The denoising path takes its text rows and conditioning vectors from a language model. These are
the operators that such a tower, and linears in 8 bits, are made of:

  norm   root-mean-square norm with the residual's addition; the result in the model dtype, in
         8 bits (e4m3) with a scale for each 128 columns of a row, or both   (ff_rms_norm_q8)
  quant  a tensor into 8 bits: a scale for each 128 columns of a row (activations) or for each
         128 x 128 block (weights, once)                                      (ff_quant_q8)
  gemm   out = act(A W^T + bias) + resid on such operands                     (ff_gemm_q8)
  attn   softmax attention whose queries each see one or two spans of keys, with shared key/value
         heads, scores capped by a tanh and biased by distance                (ff_attention)

8-bit format: scale s = max(largest |value| of the block, 2^-100) / 448, value ~ s * e4m3(value / s).
Scales of rows are stored block by block, [ceil(C / 128), rows]; those of 128 x 128 blocks
[ceil(rows / 128), ceil(C / 128)].

A case's "what" is one of the four.  Sizes follow synth.CONFIGS (widths 1152 and 2048, MLP 8192, 16
heads of 128, 14 310 image rows), the tests' ragged width 1480, and generic serving lengths.
"""
import math
import random

import torch

own = False

EPS = 1e-6
E4M3 = torch.float8_e4m3fn
TINY = 2.0 ** -100
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
NEG = float("-inf")


# ------------------------------------------------------------------ cases

def _norm(name, rows, C, dtype, resid, y, q):
    return dict(name=name, what="norm", rows=rows, C=C, dtype=dtype, resid=resid, y=y, q=q)


def _quant(name, rows, C, dtype, block_rows):
    return dict(name=name, what="quant", rows=rows, C=C, dtype=dtype, block_rows=block_rows)


def _gemm(name, M, N, K, out, bias, gelu, resid):
    return dict(name=name, what="gemm", M=M, N=N, K=K, out=out, bias=bias, gelu=gelu, resid=resid)


def _attn(name, B, H, Hkv, d, nq, nk, mask, part, dtype="bf16", cap=0.0, bias="none", reach=0):
    """mask: full | docs (packed prompts of about `part` tokens, causal) | prefix (causal behind a
    prefix of up to `part` tokens, padded batch) | joint (the first `part` keys are padded text) |
    cache (the nq newest of a ragged cache's tokens; the shortest holds nk / part)."""
    return dict(name=name, what="attn", B=B, H=H, Hkv=Hkv, d=d, nq=nq, nk=nk, mask=mask, part=part, dtype=dtype,
                cap=cap, bias=bias, reach=reach)


def listed():
    return [
        # one token being served: the smallest call of a layer's norm
        _norm("norm_token", 1, 2048, "bf16", True, False, True),
        # the video sequence's rows, residual kept beside the 8-bit operand of the next product
        _norm("norm_video", 14566, 2048, "bf16", True, False, True),
        # the MLP's hidden rows of a 4096 + 512 token image before the second product
        _quant("quant_hidden", 4608, 8192, "bf16", 1),
        # an fp32 weight matrix laid out once, odd in both directions (partial last blocks)
        _quant("quant_weight", 8200, 2960, "fp32", 128),
        # one token through the MLP's first product: the weight's bytes are all there is
        _gemm("gemm_token", 1, 8192, 2048, "bf16", True, True, False),
        # one prompt's rows through q, k and v
        _gemm("gemm_prompt", 256, 6144, 2048, "bf16", True, False, False),
        # odd sizes in all three directions, residual added in fp32
        _gemm("gemm_ragged", 1003, 1480, 2960, "fp32", True, False, True),
        # the video sequence through the MLP's first product
        _gemm("gemm_video", 14566, 8192, 2048, "bf16", True, True, False),
        # single tokens of eight users over ragged caches, four query heads to a key head
        _attn("attn_cache", 8, 16, 4, 128, 1, 32768, "cache", 4),
        # packed prompts, causal within each, scores capped
        _attn("attn_docs", 1, 16, 8, 128, 4096, 4096, "docs", 600, cap=50.0),
        # a padded batch of prompts with a bidirectional prefix and a bias by distance, in fp32
        _attn("attn_prefix_fp32", 4, 12, 12, 64, 333, 333, "prefix", 100, dtype="fp32", bias="table", reach=128),
        # the video sequence's joint attention with its 256 text rows padded
        _attn("attn_joint", 1, 16, 16, 128, 14566, 14566, "joint", 256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges; no larger than the largest listed one of its kind."""
    what = rng.choice(["norm", "quant", "gemm", "gemm", "attn", "attn", "attn"])
    if what == "norm":
        c = _norm("", _log(rng, 1, 14566), 8 * _log(rng, 8, 1024), rng.choice(["bf16", "bf16", "fp32"]),
                  rng.random() < 0.7, False, True)
        c["y"], c["q"] = rng.choice([(False, True), (True, True), (True, False)])
        while c["rows"] * c["C"] > 14566 * 2048:
            c["rows"] //= 2
    elif what == "quant":
        c = _quant("", _log(rng, 1, 16384), 8 * _log(rng, 8, 1024), rng.choice(["bf16", "bf16", "fp32"]),
                   rng.choice([1, 1, 128]))
        while c["rows"] * c["C"] > 4608 * 8192:
            c["rows"] //= 2
    elif what == "gemm":
        c = _gemm("", _log(rng, 1, 16384), 8 * _log(rng, 8, 1024), 16 * _log(rng, 8, 512),
                  rng.choice(["bf16", "bf16", "fp32"]), rng.random() < 0.7, rng.random() < 0.4, rng.random() < 0.4)
        while c["M"] * c["N"] * c["K"] > 14566 * 8192 * 2048:
            c["M"] //= 2
    else:
        c = _draw_attn(rng)
        while c["B"] * c["H"] * c["nq"] * c["nk"] > 16 * 14566 * 14566 or c["B"] * c["Hkv"] * c["d"] * c["nk"] > 8 * 4 * 128 * 32768:
            c["nk"] = max(c["nk"] // 2, 1)
            c["nq"] = c["nk"] if c["mask"] != "cache" else min(c["nq"], c["nk"])
            if c["mask"] in ("joint", "prefix"):
                c["part"] = max(1, min(c["part"], c["nk"] // 2))
    del c["name"]
    return c


def _draw_attn(rng):
    mask = rng.choice(["full", "docs", "prefix", "joint", "cache", "cache"])
    group = rng.choice([1, 1, 2, 4, 8])
    Hkv = rng.choice([1, 2, 4, 5, 8, 12])
    d = rng.choice([128, 128, 64, 64, 72, 96, 40])
    B = rng.choice([1, 1, 2, 3, 8])
    if mask == "cache":
        nq, nk = rng.choice([1, 1, 1, 2, 5, 16]), _log(rng, 16, 40000)
    else:
        nk = _log(rng, 1, 15000)
        nq = nk
    part = {"full": 0, "docs": _log(rng, 1, 1000), "prefix": rng.randint(1, max(1, nk // 2)),
            "joint": rng.randint(1, max(1, nk // 2)), "cache": rng.choice([1, 2, 4])}[mask]
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    if dtype == "fp32" and mask != "cache":
        nq = nk = min(nk, 1500)
        part = min(part, max(1, nk // 2)) if mask in ("prefix", "joint") else part
    bias = rng.choice(["none", "none", "slope", "table"]) if mask != "joint" else "none"
    return _attn("", B, Hkv * group, Hkv, d, min(nq, nk), nk, mask, part, dtype, rng.choice([0.0, 0.0, 30.0, 50.0]), bias,
                 rng.choice([16, 128, 1000]) if bias == "table" else 0)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, std=1.0, mean=0.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).add_(mean).to(dtype)


def _rows_like(g, rows, C, dtype):
    """A residual stream: most channels of order one, a few of them many times larger."""
    x = _randn(g, (rows, C))
    x *= torch.exp(_randn(g, (C,), 0.5))
    return x.to(dtype)


def _blocks(x, block_rows):
    """|x|'s largest value in blocks of block_rows x 128."""
    r, C = x.shape
    nb, nr = -(-C // 128), -(-r // block_rows)
    p = torch.nn.functional.pad(x.abs(), (0, nb * 128 - C, 0, nr * block_rows - r))
    return p.view(nr, block_rows, nb, 128).amax((1, 3))


def _quantise(x, block_rows):
    """(e4m3 values, scales [row blocks, column blocks]) of an fp32 matrix, by the format's formula."""
    s = _blocks(x, block_rows).clamp_min(TINY) / 448.0
    inv = (1.0 / s).repeat_interleave(block_rows, 0)[: x.shape[0]].repeat_interleave(128, 1)[:, : x.shape[1]]
    return (x * inv).to(E4M3), s


def _spread(s, block_rows, rows, C):
    return s.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :C]


def _lengths(c):
    """The case's own sequence lengths (part of the case, not of the seed)."""
    rng = random.Random("%(mask)s %(B)d %(nq)d %(nk)d %(part)d" % c)
    if c["mask"] == "docs":
        out = []
        for _ in range(c["B"]):
            cut = []
            while sum(cut) < c["nk"]:
                cut.append(min(_log(rng, max(1, c["part"] // 4), 2 * c["part"]), c["nk"] - sum(cut)))
            out.append(cut)
        return out
    if c["mask"] == "cache":
        low = max(c["nq"], c["nk"] // c["part"])
        return [rng.randint(low, c["nk"]) for _ in range(c["B"])]
    if c["mask"] == "prefix":
        return [(rng.randint(max(1, c["nk"] // 2), c["nk"]), rng.randint(1, c["part"])) for _ in range(c["B"])]
    if c["mask"] == "joint":
        return [rng.randint(0, c["part"]) for _ in range(c["B"])]
    return []


def _spans(c):
    """int32 [B, nq, spans, 2]: the key ranges [first, end) that each query sees."""
    n, i = c["nq"], torch.arange(c["nq"], device="cuda")
    rows = []
    for l in _lengths(c):
        if c["mask"] == "docs":
            size = torch.tensor(l, device="cuda")
            start = (torch.cumsum(size, 0) - size).repeat_interleave(size)
            rows.append(torch.stack([start, i + 1], -1)[:, None])
        elif c["mask"] == "cache":
            rows.append(torch.stack([torch.zeros_like(i), l - n + i + 1], -1)[:, None])
        elif c["mask"] == "prefix":
            s = torch.stack([torch.zeros_like(i), torch.maximum(i + 1, torch.tensor(l[1], device="cuda")).clamp_max(l[0])], -1)
            rows.append(torch.where((i < l[0])[:, None], s, 0)[:, None])
        else:
            s = torch.tensor([[0, l], [c["part"], c["nk"]]], device="cuda").expand(n, 2, 2)
            rows.append(torch.where(((i < l) | (i >= c["part"]))[:, None, None], s, 0))
    return torch.stack(rows).to(torch.int32).contiguous() if rows else None


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = {"case": c}
    if c["what"] == "norm":
        dt = DTYPES[c["dtype"]]
        st["x"] = _rows_like(g, c["rows"], c["C"], dt)
        st["resid"] = _rows_like(g, c["rows"], c["C"], dt) if c["resid"] else None
        st["gain"] = _randn(g, (c["C"],), 0.1, 1.0, dt)
    elif c["what"] == "quant":
        st["x"] = _rows_like(g, c["rows"], c["C"], DTYPES[c["dtype"]])
    elif c["what"] == "gemm":
        M, N, K, dt = c["M"], c["N"], c["K"], DTYPES[c["out"]]
        st["a"], s = _quantise(_rows_like(g, M, K, torch.float32), 1)
        st["a_s"] = s.t().contiguous()
        st["w"], st["w_s"] = _quantise(_randn(g, (N, K), 1.0 / math.sqrt(K)), 128)
        st["bias"] = _randn(g, (N,), 0.1, 0.0, dt) if c["bias"] else None
        st["resid"] = _randn(g, (M, N), 1.0, 0.0, dt) if c["resid"] else None
    else:
        dt = DTYPES[c["dtype"]]
        st["q"] = _randn(g, (c["B"], c["nq"], c["H"], c["d"]), 1.0, 0.0, dt)
        st["k"] = _randn(g, (c["B"], c["nk"], c["Hkv"], c["d"]), 1.0, 0.0, dt)
        st["v"] = _randn(g, (c["B"], c["nk"], c["Hkv"], c["d"]), 1.0, 0.0, dt)
        st["spans"] = _spans(c)
        # where a sample's first query stands among its keys (the bias goes by the distance)
        st["pos"] = torch.tensor([l - c["nq"] for l in _lengths(c)], dtype=torch.int32, device="cuda") if c["mask"] == "cache" else None
        h = torch.arange(1, c["H"] + 1, device="cuda", dtype=torch.float32)
        st["bias"] = {"none": None, "slope": torch.exp2(-8.0 * h / c["H"]) * (1.0 + 0.1 * torch.rand((), generator=g, device="cuda")),
                      "table": _randn(g, (c["H"], 2 * c["reach"] + 1))}[c["bias"]]
    return st


# ------------------------------------------------------------------ plain forms

def _norm_plain(st, c):
    x = st["x"].float()
    if c["resid"]:
        x = (x + st["resid"].float()).to(st["x"].dtype).float()
    y = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * st["gain"].float()
    out = {"sum": x.to(st["x"].dtype) if c["resid"] else None, "y": y.to(st["x"].dtype) if c["y"] else None}
    if c["q"]:
        out["q"], s = _quantise(y, 1)
        out["q_s"] = s.t().contiguous()
    return out


def _quant_plain(st, c):
    q, s = _quantise(st["x"].float(), c["block_rows"])
    return {"q": q, "q_s": s.t().contiguous() if c["block_rows"] == 1 else s}


def _gemm_plain(st, c):
    a = st["a"].float() * _spread(st["a_s"].t(), 1, c["M"], c["K"])
    w = st["w"].float() * _spread(st["w_s"], 128, c["N"], c["K"])
    y = a @ w.t()
    if c["bias"]:
        y += st["bias"].float()
    if c["gelu"]:
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if c["resid"]:
        y += st["resid"].float()
    return y.to(DTYPES[c["out"]])


def _distance(st, c):
    """key index - query position, [B or 1, nq, nk]"""
    i = torch.arange(c["nq"], device="cuda")[None]
    if st["pos"] is not None:
        i = i + st["pos"][:, None]
    return torch.arange(c["nk"], device="cuda") - i[..., None]


def _attn_plain(st, c):
    B, H, Hkv, d, nq, nk = (c[n] for n in ("B", "H", "Hkv", "d", "nq", "nk"))
    q = st["q"].float().view(B, nq, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    s = (q @ st["k"].float().permute(0, 2, 3, 1).contiguous()).view(B, H, nq, nk).mul_(1.0 / math.sqrt(d))
    if c["cap"]:
        s = torch.tanh(s / c["cap"]).mul_(c["cap"])
    if c["bias"] == "slope":
        s -= st["bias"][:, None, None] * _distance(st, c).abs().float()[:, None]
    elif c["bias"] == "table":
        R = c["reach"]
        s += st["bias"][:, _distance(st, c).clamp(-R, R) + R].transpose(0, 1)
    if st["spans"] is not None:
        j, lo, hi = torch.arange(nk, device="cuda"), st["spans"][..., 0, None], st["spans"][..., 1, None]
        s.masked_fill_(~((j >= lo) & (j < hi)).any(2)[:, None], NEG)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == NEG, 0.0, m))
    l = p.sum(-1, keepdim=True)
    o = p.view(B, Hkv, -1, nk) @ st["v"].float().transpose(1, 2)
    o = o.view(B, H, nq, d) / torch.where(l > 0, l, 1.0)
    return o.transpose(1, 2).contiguous().to(st["q"].dtype)


PLAIN = {"norm": _norm_plain, "quant": _quant_plain, "gemm": _gemm_plain, "attn": _attn_plain}


# ------------------------------------------------------------------ the framework's calls

def _ptr(t):
    return t.data_ptr() if t is not None else None


def _own_norm(st, c, abi, stream):
    k = st.get("kept")
    if k is None:   # descriptor and buffers that a program keeps
        x, rows, C = st["x"], c["rows"], c["C"]
        new = torch.empty_like
        k = st["kept"] = {
            "desc": abi.ff_norm_desc(rows=rows, C=C, dtype=abi.FF_BF16 if c["dtype"] == "bf16" else abi.FF_F32, eps=EPS,
                                     x_row=C, resid_row=C, sum_row=C, y_row=C, q_row=C, qs_ld=rows),
            "out": {"sum": new(x) if c["resid"] else None, "y": new(x) if c["y"] else None}}
        if c["q"]:
            k["out"]["q"] = torch.empty(rows, C, dtype=E4M3, device="cuda")
            k["out"]["q_s"] = torch.empty(-(-C // 128), rows, device="cuda")
    o = k["out"]
    abi.ff_rms_norm_q8(k["desc"], _ptr(st["x"]), _ptr(st["resid"]), _ptr(st["gain"]), _ptr(o["sum"]), _ptr(o["y"]),
                       _ptr(o.get("q")), _ptr(o.get("q_s")), stream)
    return o


def _own_quant(st, c, abi, stream):
    k = st.get("kept")
    if k is None:
        rows, C, br = c["rows"], c["C"], c["block_rows"]
        nb = -(-C // 128)
        k = st["kept"] = {
            "desc": abi.ff_quant_desc(rows=rows, C=C, dtype=abi.FF_BF16 if c["dtype"] == "bf16" else abi.FF_F32,
                                      block_rows=br, x_row=C, q_row=C, qs_ld=rows if br == 1 else nb),
            "out": {"q": torch.empty(rows, C, dtype=E4M3, device="cuda"),
                    "q_s": torch.empty((nb, rows) if br == 1 else (-(-rows // 128), nb), device="cuda")}}
    o = k["out"]
    abi.ff_quant_q8(k["desc"], _ptr(st["x"]), _ptr(o["q"]), _ptr(o["q_s"]), stream)
    return o


def _workspace(nbytes):
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")


def _own_gemm(st, c, abi, stream):
    k = st.get("kept")
    if k is None:
        M, N, K = c["M"], c["N"], c["K"]
        desc = abi.ff_gemm_q8_desc(M=M, N=N, K=K, out_dtype=abi.FF_BF16 if c["out"] == "bf16" else abi.FF_F32,
                                   gelu=int(c["gelu"]), a_row=K, w_row=K, out_row=N, resid_row=N, as_ld=M,
                                   ws_ld=-(-K // 128))
        n = abi.ff_gemm_q8_workspace_bytes(desc)
        k = st["kept"] = {"desc": desc, "bytes": n, "ws": _workspace(n),
                          "out": torch.empty(M, N, dtype=DTYPES[c["out"]], device="cuda")}
    abi.ff_gemm_q8(k["desc"], _ptr(st["a"]), _ptr(st["a_s"]), _ptr(st["w"]), _ptr(st["w_s"]), _ptr(st["bias"]),
                   _ptr(st["resid"]), _ptr(k["out"]), _ptr(k["ws"]), k["bytes"], stream)
    return k["out"]


def _own_attn(st, c, abi, stream):
    k = st.get("kept")
    if k is None:
        q, kk, v = st["q"], st["k"], st["v"]
        out, sp = torch.empty_like(q), st["spans"]
        desc = abi.ff_attn_desc(
            dtype=abi.FF_BF16 if c["dtype"] == "bf16" else abi.FF_F32, B=c["B"], H=c["H"], H_kv=c["Hkv"], d=c["d"],
            n_q=c["nq"], n_k=c["nk"],
            **{"%s_%s" % (n, w): t.stride(i) for n, t in (("q", q), ("k", kk), ("v", v), ("o", out))
               for i, w in enumerate(("batch", "row", "head"))},
            scale=1.0 / math.sqrt(c["d"]), cap=c["cap"],
            bias_kind={"none": abi.FF_BIAS_NONE, "slope": abi.FF_BIAS_SLOPE, "table": abi.FF_BIAS_TABLE}[c["bias"]],
            bias_reach=c["reach"], n_spans=sp.shape[2] if sp is not None else 0,
            span_batch=sp.stride(0) if sp is not None else 0)
        n = abi.ff_attention_workspace_bytes(desc)
        k = st["kept"] = {"desc": desc, "bytes": n, "ws": _workspace(n), "out": out}
    abi.ff_attention(k["desc"], _ptr(st["q"]), _ptr(st["k"]), _ptr(st["v"]), _ptr(st["bias"]), _ptr(st["pos"]),
                     _ptr(st["spans"]), _ptr(k["out"]), _ptr(k["ws"]), k["bytes"], stream)
    return k["out"]


OWN = {"norm": _own_norm, "quant": _own_quant, "gemm": _own_gemm, "attn": _own_attn}


def run(state):
    c = state["case"]
    if own:
        from paper_2607_27842_amd import abi
        return OWN[c["what"]](state, c, abi, torch.cuda.current_stream().cuda_stream)
    return PLAIN[c["what"]](state, c)


# ------------------------------------------------------------------ what a pass cannot do without

def _visible(c):
    """(query, key) pairs of one head that attend, and keys that some query of the sample sees."""
    B, nq, nk, L = c["B"], c["nq"], c["nk"], _lengths(c)
    if c["mask"] == "docs":
        return sum(n * (n + 1) // 2 for l in L for n in l), B * nk
    if c["mask"] == "cache":
        return sum(l * nq - nq * (nq - 1) // 2 for l in L), sum(L)
    if c["mask"] == "prefix":
        return sum(sum(min(l, max(i + 1, p)) for i in range(l)) for l, p in L), sum(l for l, _ in L)
    if c["mask"] == "joint":
        keys = [l + nk - c["part"] for l in L]
        return sum(k * k for k in keys), sum(keys)
    return B * nq * nk, B * nk


def work(case):
    c = case
    if c["what"] == "norm":
        n, es = c["rows"] * c["C"], 2 if c["dtype"] == "bf16" else 4
        b = n * es * (1 + 2 * c["resid"] + c["y"]) + c["C"] * es + c["q"] * (n + 4 * c["rows"] * -(-c["C"] // 128))
        return {"bytes": b, "flops": 5 * n}
    if c["what"] == "quant":
        n, es = c["rows"] * c["C"], 2 if c["dtype"] == "bf16" else 4
        return {"bytes": n * (es + 1) + 4 * -(-c["rows"] // c["block_rows"]) * -(-c["C"] // 128), "flops": 3 * n}
    if c["what"] == "gemm":
        M, N, K, es = c["M"], c["N"], c["K"], 2 if c["out"] == "bf16" else 4
        nb = -(-K // 128)
        b = (M + N) * K + 4 * nb * (M + -(-N // 128)) + M * N * es * (1 + c["resid"]) + N * es * c["bias"]
        return {"bytes": b, "flops": 2 * M * N * K}
    es = 2 if c["dtype"] == "bf16" else 4
    pairs, keys = _visible(c)
    return {"bytes": es * c["d"] * (2 * c["B"] * c["nq"] * c["H"] + 2 * keys * c["Hkv"]), "flops": 4 * c["d"] * c["H"] * pairs}


# ------------------------------------------------------------------ definitions in 64 bits

def _q_exact(y, block_rows):
    rows, C = y.shape
    q, s = torch.empty_like(y), torch.empty(-(-rows // block_rows), -(-C // 128), dtype=torch.float64, device="cuda")
    for j in range(s.shape[1]):
        blk = y[:, 128 * j:128 * j + 128]
        for i in range(0, rows, block_rows) if block_rows > 1 else (slice(None),):
            at = slice(i, i + block_rows) if block_rows > 1 else i
            top = blk[at].abs().amax(1, keepdim=True) if block_rows == 1 else blk[at].abs().max()
            sc = torch.maximum(top, torch.full_like(top, TINY)) / 448
            q[at, 128 * j:128 * j + 128] = (blk[at] / sc).to(E4M3).double()
            if block_rows == 1:
                s[:, j] = sc[:, 0]
            else:
                s[i // block_rows, j] = sc
    return q, s


def exact(case, seed):
    st, c = prepare(case, seed), case
    if c["what"] == "norm":
        x = st["x"].double()
        if c["resid"]:
            x = (x + st["resid"].double()).to(st["x"].dtype).double()
        y = x / torch.sqrt((x * x).sum(1, keepdim=True) / c["C"] + EPS) * st["gain"].double()
        out = {"sum": x if c["resid"] else None, "y": y if c["y"] else None}
        if c["q"]:
            out["q"], s = _q_exact(y, 1)
            out["q_s"] = s.t().contiguous()
        return out
    if c["what"] == "quant":
        q, s = _q_exact(st["x"].double(), c["block_rows"])
        return {"q": q, "q_s": s.t().contiguous() if c["block_rows"] == 1 else s}
    if c["what"] == "gemm":
        y = torch.zeros(c["M"], c["N"], dtype=torch.float64, device="cuda")
        for j in range(-(-c["K"] // 128)):
            at = slice(128 * j, 128 * j + 128)
            part = st["a"][:, at].double() @ st["w"][:, at].double().t()
            y += part * st["a_s"][j].double()[:, None] * st["w_s"][:, j].double().repeat_interleave(128)[: c["N"]]
        if c["bias"]:
            y += st["bias"].double()
        if c["gelu"]:
            y = y * 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
        return y + st["resid"].double() if c["resid"] else y
    group, out = c["H"] // c["Hkv"], torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    j, i = torch.arange(c["nk"], device="cuda"), torch.arange(c["nq"], device="cuda")
    for b in range(c["B"]):
        seen = torch.ones(c["nq"], c["nk"], dtype=torch.bool, device="cuda")
        if st["spans"] is not None:
            seen.zero_()
            for sp in st["spans"][b].unbind(1):
                seen |= (j[None] >= sp[:, :1]) & (j[None] < sp[:, 1:])
        dist = j[None] - (i + (int(st["pos"][b]) if st["pos"] is not None else 0))[:, None]
        some = seen.any(1)
        for h in range(c["H"]):
            s = st["q"][b, :, h].double() @ st["k"][b, :, h // group].double().t() / math.sqrt(c["d"])
            if c["cap"]:
                s = c["cap"] * torch.tanh(s / c["cap"])
            if c["bias"] == "slope":
                s = s - st["bias"][h].double() * dist.abs()
            elif c["bias"] == "table":
                s = s + st["bias"][h].double()[dist.clamp(-c["reach"], c["reach"]) + c["reach"]]
            p = torch.softmax(s.masked_fill(~seen, NEG)[some], -1)
            out[b, some, h] = p @ st["v"][b, :, h // group].double()
    return out
