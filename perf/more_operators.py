"""Operators of 8-bit integer inference around the denoiser's blocks, each with its plain form.

  linear   out = act(A W^T + bias) gate + resid on 8-bit integers with a scale for each row of A (token) and
           each row of W (output channel); A in 8 bits already, or in the model dtype and quantised by the
           call                                                        (ff_gemm_i8, and ff_quant_i8 for weights)
  branch   what stands between two branches of a block: the norm behind one branch, its gate and the scaled
           residual, then the norm and modulation in front of the next; the result in the model dtype, or in
           8-bit integers that a product takes                                              (ff_branch_norm_i8)
  history  the feature history in 8-bit integers with a scale for each 128 values: quantised as an exact
           block's result is written, read back by the draft                (ff_cache_update_i8, ff_draft_forecast_i8)
  verify   the draft from that history against an exact block's result      (ff_verify_replace_i8)

8-bit format: scale s = max(largest |value|, 2^-100) (1 / 127), value ~ s * round(value (1 / s)), in fp32 and to
the nearest, ties to even.

A case's "what" is one of the four.  Sizes follow synth.CONFIGS (widths 256, 1152 and 2048, MLP 8192, 14 566
rows of video and text, 4608 of image and text), the tests' ragged width 1480, and generic serving lengths.
"""
import ctypes
import math

import torch

own = False

EPS = 1e-6
REL_EPS = 1e-8
TINY = 2.0 ** -100
INV127 = 1.0 / 127.0
BLOCK = 128
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------ cases

def _linear(name, M, N, K, x, out, bias, gelu, gate, resid):
    """x: bf16 | fp32 (quantised by the call) | i8.  gate: rows that share a gate vector, 0 for none."""
    return dict(name=name, what="linear", M=M, N=N, K=K, x=x, out=out, bias=bias, gelu=gelu, gate=gate, resid=resid)


def _branch(name, B, n, C, dtype, post, pre, gate, mod, scale=1.0, N=0):
    """B samples of n rows.  post, pre: none | rms | layer.  gate: none | plain | tanh.  mod: scale and shift of
    the second norm.  scale: of the residual.  N > 0: the result goes in 8 bits through a product to N columns."""
    return dict(name=name, what="branch", B=B, n=n, C=C, dtype=dtype, post=post, pre=pre, gate=gate, mod=mod, scale=scale, N=N)


def _history(name, B, n, C, dtype, order, features):
    """features: residual | output."""
    return dict(name=name, what="history", B=B, n=n, C=C, dtype=dtype, order=order, features=features)


def _verify(name, B, n, C, dtype, order, features, forward):
    """forward: draft | exact | tokens (every second one)."""
    return dict(name=name, what="verify", B=B, n=n, C=C, dtype=dtype, order=order, features=features, forward=forward)


def listed():
    return [
        # one token being served through the MLP's first product: the weight's bytes are all there is
        _linear("linear_token", 1, 8192, 2048, "bf16", "bf16", True, True, 0, False),
        # one prompt's rows, in 8 bits already, through q, k and v
        _linear("linear_prompt", 256, 6144, 2048, "i8", "bf16", True, False, 0, False),
        # odd sizes in all three directions, three samples' gates and the residual in fp32
        _linear("linear_ragged", 1003, 1480, 2960, "fp32", "fp32", True, False, 335, True),
        # the video sequence through the MLP's first product
        _linear("linear_video", 14566, 8192, 2048, "bf16", "bf16", True, True, 0, False),
        # one token between two branches: the smallest call
        _branch("branch_token", 1, 1, 2048, "bf16", "rms", "rms", "plain", True),
        # the video sequence between two branches
        _branch("branch_video", 1, 14566, 2048, "bf16", "rms", "rms", "tanh", True),
        # adaptive LayerNorm without a norm behind the branch, odd rows and width, fp32, scaled residual
        _branch("branch_ragged", 3, 333, 1480, "fp32", "none", "layer", "plain", True, 0.875),
        # image and text rows between two branches and on through q, k and v in 8 bits
        _branch("branch_image_qkv", 1, 4608, 2048, "bf16", "rms", "rms", "plain", True, 1.0, 6144),
        # the smallest model's refresh and draft: two launches
        _history("history_tiny", 1, 64, 256, "fp32", 1, "residual"),
        # the video model's refresh and draft, first order
        _history("history_video", 1, 14566, 2048, "bf16", 1, "residual"),
        # eight class-conditional images at a paid site, second order, the exact result forwarded
        _verify("verify_images", 8, 256, 1152, "bf16", 2, "residual", "exact"),
        # samples that end inside a block of 128, output features, third order, half of the tokens forwarded
        _verify("verify_ragged", 3, 333, 1480, "bf16", 3, "output", "tokens"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges; no larger than the largest listed one of its kind."""
    what = rng.choice(["linear", "linear", "linear", "branch", "branch", "history", "verify"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if what == "linear":
        c = _linear("", _log(rng, 1, 16384), 8 * _log(rng, 8, 1024), 16 * _log(rng, 8, 512), rng.choice([dtype, "i8"]), dtype,
                    rng.random() < 0.7, rng.random() < 0.3, 0, rng.random() < 0.5)
        while c["M"] * c["N"] * c["K"] > 14566 * 8192 * 2048:
            c["M"] //= 2
        if c["resid"] and rng.random() < 0.7:
            c["gate"] = -(-c["M"] // rng.choice([1, 2, 3, 8]))
    elif what == "branch":
        c = _branch("", rng.choice([1, 1, 2, 3, 8]), _log(rng, 1, 14566), 8 * _log(rng, 8, 1024), dtype,
                    rng.choice(["none", "rms", "rms", "layer"]), rng.choice(["rms", "rms", "layer"]),
                    rng.choice(["none", "plain", "tanh"]), rng.random() < 0.6, rng.choice([1.0, 1.0, 0.875]))
        if dtype == "bf16" and rng.random() < 0.4:
            c["C"], c["N"] = 16 * (-(-c["C"] // 16)), 8 * _log(rng, 8, 768)
        while c["B"] * c["n"] * c["C"] * max(c["N"], 1) > (4608 * 2048 * 6144 if c["N"] else 14566 * 2048):
            c["n"], c["B"] = (c["n"] // 2, c["B"]) if c["n"] > 1 else (1, max(1, c["B"] // 2))
    else:
        B, n = rng.choice([1, 1, 2, 3, 8]), _log(rng, 1, 14566)
        C = 8 * _log(rng, 8, 256)
        while B * n * C > 14566 * 2048:
            n //= 2
        order, features = rng.choice([0, 1, 1, 2, 3]), rng.choice(["residual", "residual", "output"])
        c = _history("", B, n, C, dtype, order, features) if what == "history" else \
            _verify("", B, n, C, dtype, order, features, rng.choice(["draft", "exact", "tokens"]))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, std=1.0, mean=0.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).add_(mean).to(dtype)


def _rows_like(g, shape, dtype):
    """A residual stream: most channels of order one, a few of them many times larger."""
    x = _randn(g, shape)
    x *= torch.exp(_randn(g, shape[-1:], 0.5))
    return x.to(dtype)


def _quantise(x):
    """(whole values, scales) of the last axis of an fp32 tensor, by the format's formula."""
    s = x.abs().amax(-1).clamp_min(TINY) * INV127
    return torch.round(x * (1.0 / s)[..., None]), s


def _blocks(x):
    """A sample's values in blocks of 128, the last one padded with zeros: [B, blocks, 128]."""
    B = x.shape[0]
    nb = -(-x[0].numel() // BLOCK)
    return torch.nn.functional.pad(x.reshape(B, -1), (0, nb * BLOCK - x[0].numel())).view(B, nb, BLOCK)


def _coeffs(order):
    """A forecast half an interval ahead of the newest feature, by differences at unit intervals."""
    return {0: [1.0], 1: [1.5, -0.5], 2: [1.875, -1.25, 0.375], 3: [2.1875, -2.1875, 1.3125, -0.3125]}[order]


def _slot_bytes(c):
    """A slot: every sample's blocks of 128 values, then every block's scale, to a multiple of 128 bytes."""
    n = c["B"] * -(-c["n"] * c["C"] // BLOCK)
    return -(-n * (BLOCK + 4) // BLOCK) * BLOCK


def _slot(st, c, m):
    """Views of slot m of the cache: values [B, blocks, 128] and scales [B, blocks]."""
    nb, size = -(-c["n"] * c["C"] // BLOCK), _slot_bytes(c)
    at = st["cache"][m * size:(m + 1) * size]
    q = at[:c["B"] * nb * BLOCK].view(torch.int8).view(c["B"], nb, BLOCK)
    s = at[c["B"] * nb * BLOCK:c["B"] * nb * (BLOCK + 4)].view(torch.float32).view(c["B"], nb)
    return q, s


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = {"case": c}
    if c["what"] == "linear":
        M, N, K, dt = c["M"], c["N"], c["K"], DTYPES[c["out"]]
        x = _rows_like(g, (M, K), torch.float32)
        if c["x"] == "i8":
            q, st["x_s"] = _quantise(x)
            st["x"] = q.to(torch.int8)
        else:
            st["x"], st["x_s"] = x.to(DTYPES[c["x"]]), None
        q, st["w_s"] = _quantise(_randn(g, (N, K), 1.0 / math.sqrt(K)))
        st["w"] = q.to(torch.int8)
        st["bias"] = _randn(g, (N,), 0.1, 0.0, dt) if c["bias"] else None
        st["gate"] = _randn(g, (-(-M // c["gate"]), N), 0.5) if c["gate"] else None
        st["resid"] = _randn(g, (M, N), 1.0, 0.0, dt) if c["resid"] else None
    elif c["what"] == "branch":
        B, C, dt = c["B"], c["C"], DTYPES[c["dtype"]]
        rows = B * c["n"]
        st["x"], st["branch"] = _rows_like(g, (rows, C), dt), _rows_like(g, (rows, C), dt)
        st["post_gain"] = _randn(g, (C,), 0.1, 1.0, dt) if c["post"] == "rms" else None
        st["pre_gain"] = _randn(g, (C,), 0.1, 1.0, dt) if c["pre"] == "rms" else None
        # one vector of modulation per sample, as the conditioning's product gives it
        st["mod"] = _randn(g, (B, 3 * C), 0.3)
        if c["N"]:
            q, st["w_s"] = _quantise(_randn(g, (c["N"], C), 1.0 / math.sqrt(C)))
            st["w"] = q.to(torch.int8)
    else:
        shape, dt = (c["B"], c["n"], c["C"]), DTYPES[c["dtype"]]
        st["cache"] = torch.zeros((c["order"] + 1) * _slot_bytes(c), dtype=torch.uint8, device="cuda")
        base = _rows_like(g, shape, torch.float32)
        for m in range(c["order"] + 1):   # features that change slowly from refresh to refresh
            q, s = _slot(st, c, m)
            v, sc = _quantise(_blocks(base + 0.1 * _randn(g, shape)))
            q.copy_(v)
            s.copy_(sc)
        st["u"] = _rows_like(g, shape, dt)
        st["h"] = ((st["u"].float() if c["features"] == "residual" else 0.0) + base + 0.1 * _randn(g, shape)).to(dt)
        # the stream that the draft starts from: another step's, or at a site the exact block's own
        st["u1"] = _rows_like(g, shape, dt) if c["what"] == "history" else st["u"]
    return st


# ------------------------------------------------------------------ plain forms

def _gelu(y):
    return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))


def _norm(x, kind, gain):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    x = x / torch.sqrt(x.square().mean(1, keepdim=True) + EPS)
    return x * gain.to(x.dtype) if gain is not None else x


def _linear_plain(st, c):
    q, s = (st["x"].float(), st["x_s"]) if c["x"] == "i8" else _quantise(st["x"].float())
    y = (q @ st["w"].float().t()) * s[:, None] * st["w_s"]
    if c["bias"]:
        y += st["bias"].float()
    if c["gelu"]:
        y = _gelu(y)
    if c["gate"]:
        y *= st["gate"].repeat_interleave(c["gate"], 0)[:c["M"]]
    if c["resid"]:
        y += st["resid"].float()
    return y.to(DTYPES[c["out"]])


def _branch_plain(st, c):
    C, dt = c["C"], st["x"].dtype
    z = _norm(st["branch"].float(), c["post"], st["post_gain"])
    gate, scale, shift = (t.repeat_interleave(c["n"], 0) for t in st["mod"].split(C, 1))
    if c["gate"] != "none":
        z = z * (torch.tanh(gate) if c["gate"] == "tanh" else gate)
    t = (st["x"].float() * c["scale"] + z).to(dt)
    v = _norm(t.float(), c["pre"], st["pre_gain"])
    if c["mod"]:
        v = v * (1.0 + scale) + shift
    if not c["N"]:
        return {"sum": t, "y": v.to(dt)}
    q, s = _quantise(v)
    return {"sum": t, "out": ((q @ st["w"].float().t()) * s[:, None] * st["w_s"]).to(dt)}


def _draft_plain(st, c):
    f = 0.0
    for m, k in enumerate(_coeffs(c["order"])):
        q, s = _slot(st, c, m)
        f = f + k * (q.float() * s[..., None])
    f = f.view(c["B"], -1)[:, :c["n"] * c["C"]].view(st["u"].shape)
    return (st["u1"].float() + f if c["features"] == "residual" else f).to(st["u"].dtype)


def _history_plain(st, c):
    new = st["h"].float() - st["u"].float() if c["features"] == "residual" else st["h"].float()
    v, sc = _quantise(_blocks(new))
    q, s = _slot(st, c, 0)
    q.copy_(v)
    s.copy_(sc)
    return _draft_plain(st, c)


def _verify_plain(st, c):
    d, h = _draft_plain(st, c), st["h"]
    rel = (d.float() - h.float()).abs().sum((1, 2)) / (h.float().abs().sum((1, 2)) + REL_EPS)
    if c["forward"] == "tokens":
        d = torch.where((torch.arange(c["n"], device="cuda") % 2 == 0)[:, None], h, d)
    return {"out": h if c["forward"] == "exact" else d, "rel": rel}


PLAIN = {"linear": _linear_plain, "branch": _branch_plain, "history": _history_plain, "verify": _verify_plain}


# ------------------------------------------------------------------ the framework's calls

def _ptr(t):
    return t.data_ptr() if t is not None else None


def _code(abi, dtype):
    return {"bf16": abi.FF_BF16, "fp32": abi.FF_F32, "i8": abi.FF_I8}[dtype]


def _bytes(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


def _own_linear(st, c, abi, stream):
    k = st.get("kept")
    if k is None:   # descriptor, workspace and output that a program keeps
        M, N, K = c["M"], c["N"], c["K"]
        desc = abi.ff_gemm_i8_desc(M=M, N=N, K=K, a_dtype=_code(abi, c["x"]), out_dtype=_code(abi, c["out"]),
                                   gelu=int(c["gelu"]), gate_rows=c["gate"], a_row=K, w_row=K, out_row=N, resid_row=N, gate_ld=N)
        n = abi.ff_gemm_i8_workspace_bytes(desc)
        k = st["kept"] = {"desc": desc, "bytes": n, "ws": _bytes(n),
                          "out": torch.empty(M, N, dtype=DTYPES[c["out"]], device="cuda")}
    abi.ff_gemm_i8(k["desc"], _ptr(st["x"]), _ptr(st["x_s"]), _ptr(st["w"]), _ptr(st["w_s"]), _ptr(st["bias"]), _ptr(st["gate"]),
                   _ptr(st["resid"]), _ptr(k["out"]), _ptr(k["ws"]), k["bytes"], stream)
    return k["out"]


def _own_branch(st, c, abi, stream):
    k, C = st.get("kept"), c["C"]
    if k is None:
        rows, x = c["B"] * c["n"], st["x"]
        kinds = {"none": abi.FF_NORM_NONE, "rms": abi.FF_NORM_RMS, "layer": abi.FF_NORM_LAYER}
        k = st["kept"] = {
            "desc": abi.ff_branch_norm_desc(
                rows=rows, C=C, dtype=_code(abi, c["dtype"]), post=kinds[c["post"]], pre=kinds[c["pre"]],
                gate_tanh=int(c["gate"] == "tanh"), mod_rows=c["n"], eps=EPS, resid_scale=c["scale"],
                x_row=C, branch_row=C, sum_row=C, y_row=C, q_row=C, gate_ld=3 * C, mod_ld=3 * C),
            "out": {"sum": torch.empty_like(x)}}
        if c["N"]:
            k["q"], k["q_s"] = torch.empty(rows, C, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
            k["out"]["out"] = torch.empty(rows, c["N"], dtype=x.dtype, device="cuda")
            k["gemm"] = abi.ff_gemm_i8_desc(M=rows, N=c["N"], K=C, a_dtype=abi.FF_I8, out_dtype=_code(abi, c["dtype"]), gelu=0,
                                            gate_rows=0, a_row=C, w_row=C, out_row=c["N"], resid_row=0, gate_ld=0)
            k["bytes"] = abi.ff_gemm_i8_workspace_bytes(k["gemm"])
            k["ws"] = _bytes(k["bytes"])
        else:
            k["out"]["y"] = torch.empty_like(x)
    o, mod = k["out"], st["mod"]
    at = lambda i: mod.data_ptr() + 4 * C * i  # noqa: E731
    abi.ff_branch_norm_i8(k["desc"], _ptr(st["x"]), _ptr(st["branch"]), _ptr(st["post_gain"]), at(0) if c["gate"] != "none" else None,
                          _ptr(st["pre_gain"]), at(1) if c["mod"] else None, at(2) if c["mod"] else None, _ptr(o["sum"]),
                          _ptr(o.get("y")), _ptr(k.get("q")), _ptr(k.get("q_s")), stream)
    if c["N"]:
        abi.ff_gemm_i8(k["gemm"], _ptr(k["q"]), _ptr(k["q_s"]), _ptr(st["w"]), _ptr(st["w_s"]), None, None, None, _ptr(o["out"]),
                       _ptr(k["ws"]), k["bytes"], stream)
    return o


def _model(abi, c):
    """The descriptor of a model of one layer with this stream."""
    return abi.ff_model_desc(n_layers=1, kinds=(ctypes.c_int32 * 1)(abi.FF_DIT), C=c["C"], H=c["C"] // 8, d=8, mlp_hidden=64,
                             n_img=c["n"], n_txt=0, B=c["B"], lat_c=8, lat_f=1, lat_h=1, lat_w=c["n"], pt=1, ph=1, pw=1,
                             dtype=_code(abi, c["dtype"]), ln_eps=EPS)


def _own_history(st, c, abi, stream):
    k = st.get("kept")
    if k is None:
        k = st["kept"] = {"model": _model(abi, c), "out": torch.empty_like(st["u"])}
    m, n = k["model"], c["order"] + 1
    res = c["features"] == "residual"
    abi.ff_cache_update_i8(m, _ptr(st["cache"]), n, 0, 0, _ptr(st["u"]) if res else None, _ptr(st["h"]),
                           abi.FF_RESIDUAL if res else abi.FF_OUTPUT, stream)
    abi.ff_draft_forecast_i8(m, _ptr(st["cache"]), n, 0, c["order"], list(range(n)), _coeffs(c["order"]),
                             _ptr(st["u1"]) if res else None, _ptr(k["out"]), stream)
    return k["out"]


def _own_verify(st, c, abi, stream):
    k = st.get("kept")
    if k is None:
        m = _model(abi, c)
        n = abi.ff_workspace_bytes(m)
        k = st["kept"] = {"model": m, "bytes": n, "ws": _bytes(n),
                          "out": {"out": torch.empty_like(st["u"]), "rel": torch.empty(c["B"], device="cuda")}}
    n, o = c["order"] + 1, k["out"]
    kind = {"draft": abi.FF_FWD_DRAFT, "exact": abi.FF_FWD_EXACT, "tokens": abi.FF_FWD_TOKENS}[c["forward"]]
    abi.ff_verify_replace_i8(k["model"], _ptr(st["cache"]), n, 0, c["order"], list(range(n)), _coeffs(c["order"]),
                             _ptr(st["u1"]) if c["features"] == "residual" else None, _ptr(st["h"]), _ptr(o["out"]), kind, REL_EPS,
                             _ptr(o["rel"]), _ptr(k["ws"]), k["bytes"], stream, stride=2)
    return o


OWN = {"linear": _own_linear, "branch": _own_branch, "history": _own_history, "verify": _own_verify}


def run(state):
    c = state["case"]
    if own:
        from paper_2607_27842_amd import abi
        return OWN[c["what"]](state, c, abi, torch.cuda.current_stream().cuda_stream)
    return PLAIN[c["what"]](state, c)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    if c["what"] == "linear":
        M, N, K, es = c["M"], c["N"], c["K"], 2 if c["out"] == "bf16" else 4
        b = M * K * {"i8": 1, "bf16": 2, "fp32": 4}[c["x"]] + (4 * M if c["x"] == "i8" else 0) + N * K + 4 * N
        b += M * N * es * (1 + c["resid"]) + N * es * c["bias"] + (4 * N * -(-M // c["gate"]) if c["gate"] else 0)
        return {"bytes": b, "flops": 2 * M * N * K}
    n, es = c["B"] * c["n"] * c["C"], 2 if c["dtype"] == "bf16" else 4
    if c["what"] == "branch":
        vectors = c["C"] * es * ((c["post"] == "rms") + (c["pre"] == "rms")) + 4 * c["B"] * c["C"] * ((c["gate"] != "none") + 2 * c["mod"])
        if c["N"]:
            rows = c["B"] * c["n"]
            return {"bytes": 3 * n * es + vectors + c["N"] * (c["C"] + 4) + rows * c["N"] * es, "flops": 2 * n * c["N"]}
        return {"bytes": 4 * n * es + vectors, "flops": 10 * n}
    slot = n + 4 * c["B"] * -(-c["n"] * c["C"] // BLOCK)
    res = c["features"] == "residual"
    if c["what"] == "history":   # a refresh: h (and u) in, a slot out; a draft: the older slots (and its u) in, its result out
        return {"bytes": n * es * (2 + 2 * res) + slot * (1 + c["order"]), "flops": n * (4 + 2 * (c["order"] + 1))}
    return {"bytes": n * es * (2 + res) + slot * (c["order"] + 1) + 4 * c["B"], "flops": n * (4 + 2 * (c["order"] + 1))}


# ------------------------------------------------------------------ definitions in 64 bits

def _whole_exact(x):
    """The values that the format stands for along the last axis of a 64-bit tensor.  The format is defined on
    fp32 numbers: x, the scale, its reciprocal and their product are each the nearest of those."""
    near = lambda t: t.float().double()  # noqa: E731
    x = near(x)
    s = near(torch.maximum(x.abs().max(-1, keepdim=True).values, torch.full((), TINY, dtype=torch.float64, device="cuda"))
             * near(torch.full((), 1 / 127, dtype=torch.float64, device="cuda")))
    return torch.round(near(x * near(1 / s))) * s


def _product_exact(a, st):
    return a @ (st["w"].double() * st["w_s"].double()[:, None]).t()


def _norm_exact(x, kind, gain):
    if kind != "none":
        n = x.shape[1]
        x = x - (x.sum(1, keepdim=True) / n if kind == "layer" else 0.0)
        x = x / ((x * x).sum(1, keepdim=True) / n + EPS) ** 0.5
    return x if gain is None else x * gain.double()


def _features_exact(st, c, m, fresh):
    """Feature m as the cache holds it, [B, n C]."""
    size = c["n"] * c["C"]
    if fresh:
        v = st["h"].double() - (st["u"].double() if c["features"] == "residual" else 0.0)
        v = v.view(c["B"], size)
        full = size // BLOCK * BLOCK
        parts = [_whole_exact(v[:, :full].reshape(c["B"], -1, BLOCK)).view(c["B"], full)] if full else []
        if size > full:
            parts.append(_whole_exact(v[:, full:]))
        return torch.cat(parts, 1)
    q, s = _slot(st, c, m)
    return (q.double() * s.double()[..., None]).view(c["B"], -1)[:, :size]


def exact(case, seed):
    st, c = prepare(case, seed), case
    if c["what"] == "linear":
        y = _product_exact(st["x"].double() * st["x_s"].double()[:, None] if c["x"] == "i8" else _whole_exact(st["x"].double()), st)
        if c["bias"]:
            y += st["bias"].double()
        if c["gelu"]:
            y = y * 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
        if c["gate"]:
            y *= st["gate"].double()[torch.arange(c["M"], device="cuda") // c["gate"]]
        return y + st["resid"].double() if c["resid"] else y
    if c["what"] == "branch":
        C, mod = c["C"], st["mod"].double()[torch.arange(c["B"] * c["n"], device="cuda") // c["n"]]
        z = _norm_exact(st["branch"].double(), c["post"], st["post_gain"])
        gate = {"none": 1.0, "plain": mod[:, :C], "tanh": torch.tanh(mod[:, :C])}[c["gate"]]
        t = c["scale"] * st["x"].double() + gate * z
        v = _norm_exact(t.to(st["x"].dtype).double(), c["pre"], st["pre_gain"])   # the stream as it is stored
        if c["mod"]:
            v = v + v * mod[:, C:2 * C] + mod[:, 2 * C:]
        return {"sum": t, "out": _product_exact(_whole_exact(v), st)} if c["N"] else {"sum": t, "y": v}
    d = sum(k * _features_exact(st, c, m, c["what"] == "history" and m == 0) for m, k in enumerate(_coeffs(c["order"]))).view(st["u"].shape)
    if c["features"] == "residual":
        d = d + st["u1"].double()
    if c["what"] == "history":
        return d
    h, stored = st["h"].double(), d.to(st["u"].dtype).double()
    rel = torch.stack([(a - b).abs().sum() / (b.abs().sum() + REL_EPS) for a, b in zip(stored, h)])
    even = torch.arange(c["n"], device="cuda")[:, None] % 2 == 0
    return {"out": {"draft": d, "exact": h, "tokens": torch.where(even, h, d)}[c["forward"]], "rel": rel}
