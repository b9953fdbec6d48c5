"""Operators of the block around a mixture-of-experts layer, as cases that can be timed and checked: the norms before and after it with
gate and residual, a dense gated feed-forward block beside it with its gradient, what training keeps of that in 8 bits, and products in
8-bit integers.

A case is a dict of plain values. `kind` says which operator a pass goes through:

  norms        y = alpha r + gate N(f; w_after) and n = N(y; w_before), N(v; w) = v / sqrt(mean v^2 + eps) w
  norms_grad   the gradient of that with respect to f, r, the gates and both weights
  ffn          y = (silu(x w_in^T) * (x w_gate^T)) w_out^T
  ffn_grad     the gradient of that with respect to x and the three weights, from the products a, b that the forward pass left
  ffn_step8    forward and gradient in one pass, with x, a and b kept in 8 bits in between
  keep8        a tensor packed to 8 bits and unpacked: blocks of 32 columns, one power of two each
  matmul8      y = x W^T with the rows of x taken to 8-bit integers in the call, W held in them: a scale for each token and channel

`own` chooses between plain torch arithmetic and the framework's entry points.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


def listed():
    return [
        # serving: eight sequences decoded together around a Switch-base layer (width 768, fp32): latency
        dict(name="norms_batch8", kind="norms", tokens=8, d=768, f="f32", r="f32", n="f32", after=True, before=True, gate=False, alpha=1.0),
        # a prompt around a Mixtral-shaped layer: the layer's outputs are fp32, the stream and the next input bf16
        dict(name="norms_prompt_2048", kind="norms", tokens=2048, d=4096, f="f32", r="bf16", n="bf16", after=False, before=True, gate=True,
             alpha=1.0),
        # a training step's gradient: four sequences of 2048, norms on both sides and a gated branch
        dict(name="norms_grad_8192", kind="norms_grad", tokens=8192, d=4096, f="bf16", r="bf16", n="bf16", after=True, before=True, gate=True,
             alpha=0.5),
        # serving: one token through a Mixtral-shaped expert kept in bf16: every weight is read for it
        dict(name="ffn_token_1", kind="ffn", tokens=1, d=4096, f=14336, type="bf16"),
        # a ragged batch of a small fp16 model, odd widths
        dict(name="ffn_ragged_333", kind="ffn", tokens=333, d=1000, f=2731, type="f16"),
        # a prompt of 2048 tokens
        dict(name="ffn_prompt_2048", kind="ffn", tokens=2048, d=4096, f=14336, type="bf16"),
        # training: the gradient of two sequences of 2048
        dict(name="ffn_grad_4096", kind="ffn_grad", tokens=4096, d=4096, f=14336, type="bf16"),
        # training with activations kept in 8 bits, a batch of odd length through a narrower expert
        dict(name="ffn_step8_2047", kind="ffn_step8", tokens=2047, d=2048, f=5632, type="bf16"),
        # what a layer leaves for its backward pass: four sequences of 2048 at width 4096
        dict(name="keep8_8192", kind="keep8", tokens=8192, d=4096, type="bf16"),
        # serving: three tokens through a projection held in 8 bits
        dict(name="matmul8_tokens_3", kind="matmul8", tokens=3, k=4096, n=14336, type="bf16", out="bf16", base=False),
        # a ragged prompt through a projection of odd widths, beside a residual in fp32
        dict(name="matmul8_ragged_517", kind="matmul8", tokens=517, k=1000, n=4100, type="f16", out="f32", base=True),
        # long prompts through a square projection
        dict(name="matmul8_8192", kind="matmul8", tokens=8192, k=4096, n=4096, type="bf16", out="bf16", base=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Widths: mostly multiples of 8 to 128, as models have them, some odd."""
    w = _log_int(rng, lo, hi)
    by = rng.choice([1, 8, 32, 64, 128, 128])
    return max(lo, w // by * by)


def draw(rng):
    """One more case of the same ranges: one token to long batches, narrow to wide and odd widths, every kind and type."""
    kind = rng.choice(["norms", "norms_grad", "ffn", "ffn", "ffn_grad", "ffn_step8", "keep8", "matmul8", "matmul8"])
    t = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind in ("norms", "norms_grad"):
        d = _width(rng, 64, 8192)
        return dict(kind=kind, tokens=_log_int(rng, 1, min(16384, 8192 * 4096 // d)), d=d, f=rng.choice([t, "f32"]), r=rng.choice([t, t, "f32"]),
                    n=t, after=rng.random() < 0.6, before=rng.random() < 0.8, gate=rng.random() < 0.5, alpha=rng.choice([1.0, 1.0, 0.5, 1.25]))
    if kind in ("ffn", "ffn_grad", "ffn_step8"):
        t = rng.choice(["f32", "bf16", "bf16", "bf16", "f16"])
        d, f = _width(rng, 128, 4096), _width(rng, 256, 14336)
        most = 4096 * 4096 * 14336 // (d * f) // {"ffn": 2, "ffn_grad": 1, "ffn_step8": 2}[kind] // (4 if t == "f32" else 1)
        return dict(kind=kind, tokens=_log_int(rng, 1, max(1, min(8192, most))), d=d, f=f, type=t)
    if kind == "keep8":
        d = _width(rng, 64, 14336)
        return dict(kind=kind, tokens=_log_int(rng, 1, min(16384, 8192 * 4096 // d)), d=d, type=t)
    k, n = _width(rng, 128, 14336), _width(rng, 128, 14336)
    return dict(kind=kind, tokens=_log_int(rng, 1, max(1, min(8192, 8192 * 4096 * 4096 // (k * n)))), k=k, n=n, type=t,
                out=rng.choice([t, t, "f32"]), base=rng.random() < 0.4)


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed, *parts):
    g = torch.Generator(device=DEV)
    g.manual_seed(random.Random(repr((int(seed),) + parts)).getrandbits(62))
    return g


def _randn(shape, std, kind, seed, *parts):
    return (torch.randn(shape, generator=_gen(seed, *parts), device=DEV, dtype=torch.float32) * std).to(TYPES[kind])


def _stream(shape, kind, seed, *parts):
    """Hidden states: rows of uneven size, a few columns larger than the others."""
    T, d = shape
    g = _gen(seed, "sizes", *parts)
    rows = torch.randn((T, 1), generator=g, device=DEV).mul(0.3).exp()
    cols = 1.0 + 5.0 * (torch.rand((1, d), generator=g, device=DEV) < 0.01)
    return (torch.randn(shape, generator=g, device=DEV) * rows * cols).to(TYPES[kind])


def _ffn_weights(case, seed):
    d, f, t = case["d"], case["f"], case["type"]
    return (_randn((f, d), 1.0 / math.sqrt(d), t, seed, "w_in"), _randn((f, d), 1.0 / math.sqrt(d), t, seed, "w_gate"),
            _randn((d, f), 1.0 / math.sqrt(f), t, seed, "w_out"))


def prepare(case, seed):
    kind = case["kind"]
    s = {"case": case}
    if kind in ("norms", "norms_grad"):
        T, d = case["tokens"], case["d"]
        s["f"] = _stream((T, d), case["f"], seed, "f")
        s["r"] = _stream((T, d), case["r"], seed, "r")
        s["gate"] = torch.sigmoid(_randn((T,), 1.0, "f32", seed, "gate")) if case["gate"] else None
        s["w_after"] = 1.0 + _randn((d,), 0.1, "f32", seed, "w_after") if case["after"] else None
        s["w_before"] = 1.0 + _randn((d,), 0.1, "f32", seed, "w_before") if case["before"] else None
        if kind == "norms_grad":
            s["y"] = _plain_norms(s)["y"]      # (what the forward pass left)
            s["dy"] = _randn((T, d), 1.0, case["r"], seed, "dy")
            s["dn"] = _randn((T, d), 1.0, case["n"], seed, "dn") if case["before"] else None
        return s
    if kind in ("ffn", "ffn_grad", "ffn_step8"):
        T, d, t = case["tokens"], case["d"], case["type"]
        s["w_in"], s["w_gate"], s["w_out"] = _ffn_weights(case, seed)
        s["x"] = _randn((T, d), 1.0, t, seed, "x")
        if kind != "ffn":
            s["dy"] = _randn((T, d), 1.0, t, seed, "dy")
        if kind == "ffn_grad":                 # (what the forward pass left)
            x = s["x"].float()
            s["ab"] = torch.stack([(x @ s[w].float().t()).to(TYPES[t]) for w in ("w_in", "w_gate")])
        if own:
            import paper_2308_14352_amd as moeq
            s["ffn"] = moeq.GatedFfn(s["w_in"], s["w_gate"], s["w_out"])
        return s
    if kind == "keep8":
        s["x"] = _stream((case["tokens"], case["d"]), case["type"], seed, "x")
        return s
    s["x"] = _stream((case["tokens"], case["k"]), case["type"], seed, "x")
    w = _randn((case["n"], case["k"]), 1.0 / math.sqrt(case["k"]), "f32", seed, "w")
    s["w_codes"], s["w_scale"] = _plain_quantize(w)
    s["base"] = _randn((case["tokens"], case["n"]), 1.0, case["out"], seed, "base") if case["base"] else None
    if own:
        import paper_2308_14352_amd as moeq
        s["weights"] = moeq.QuantRows(s["w_codes"].to(torch.int8), s["w_scale"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2308_14352_amd as moeq
    case = s["case"]
    kind = case["kind"]
    if kind == "norms":
        y, n = moeq.moe_block_norms_forward(s["f"], s["r"], gate=s["gate"], w_after=s["w_after"], w_before=s["w_before"],
                                            residual_scale=case["alpha"], eps=EPS, dtype=TYPES[case["n"]])
        return {"y": y, "n": n}
    if kind == "norms_grad":
        df, dr, dgate, dw_after, dw_before = moeq.moe_block_norms_backward(
            s["f"], s["y"], s["dy"], s["dn"], gate=s["gate"], w_after=s["w_after"], w_before=s["w_before"], residual_scale=case["alpha"], eps=EPS)
        return {"df": df, "dr": dr, "dgate": dgate, "dw_after": dw_after, "dw_before": dw_before}
    if kind == "ffn":
        return {"y": moeq.moe_gated_ffn_forward(s["ffn"], s["x"])}
    if kind == "ffn_grad":
        dx, dw_in, dw_gate, dw_out = moeq.moe_gated_ffn_backward(s["ffn"], s["x"], s["dy"], s["ab"])
        return {"dx": dx, "dw_in": dw_in, "dw_gate": dw_gate, "dw_out": dw_out}
    if kind == "ffn_step8":
        x8 = moeq.moe_pack8(s["x"])
        y, ab8 = moeq.moe_gated_ffn_forward(s["ffn"], s["x"], keep=8)
        dx, dw_in, dw_gate, dw_out = moeq.moe_gated_ffn_backward(s["ffn"], x8, s["dy"], ab8)
        return {"y": y, "dx": dx, "dw_in": dw_in, "dw_gate": dw_gate, "dw_out": dw_out}
    if kind == "keep8":
        return {"x": moeq.moe_unpack8(moeq.moe_pack8(s["x"]))}
    rows = moeq.moe_quantize_rows(s["x"])
    return {"y": moeq.moe_matmul_q8(rows, s["weights"], base=s["base"], dtype=TYPES[case["out"]])}


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "norms":
        return _plain_norms(s)
    if kind == "norms_grad":
        return _plain_norms_grad(s)
    if kind == "ffn":
        x = s["x"].float()
        a, b = x @ s["w_in"].float().t(), x @ s["w_gate"].float().t()
        return {"y": ((a / (1.0 + torch.exp(-a)) * b) @ s["w_out"].float().t()).to(s["x"].dtype)}
    if kind == "ffn_grad":
        return _plain_ffn_grad(s, s["x"].float(), s["ab"][0].float(), s["ab"][1].float())
    if kind == "ffn_step8":
        x = s["x"].float()
        a, b = x @ s["w_in"].float().t(), x @ s["w_gate"].float().t()
        y = ((a / (1.0 + torch.exp(-a)) * b) @ s["w_out"].float().t()).to(s["x"].dtype)
        kept = [_plain_keep8(v, case["type"]) for v in (x, a, b)]
        return {"y": y, **_plain_ffn_grad(s, *kept)}
    if kind == "keep8":
        return {"x": _plain_keep8(s["x"].float(), case["type"]).to(s["x"].dtype)}
    codes, scale = _plain_quantize(s["x"].float())
    # (sums of products of two 7-bit integers: below 2^24, and so exact, at these lengths and distributions)
    y = (codes @ s["w_codes"].t()) * (scale[:, None] * s["w_scale"])
    if s["base"] is not None:
        y = s["base"].float() + y
    return {"y": y.to(TYPES[case["out"]])}


def _plain_norms(s):
    case = s["case"]
    branch = s["f"].float()
    if s["w_after"] is not None:
        branch = branch * torch.rsqrt((branch * branch).mean(-1, keepdim=True) + EPS) * s["w_after"]
    if s["gate"] is not None:
        branch = branch * s["gate"][:, None]
    y = case["alpha"] * s["r"].float() + branch
    n = None
    if s["w_before"] is not None:
        n = (y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * s["w_before"]).to(TYPES[case["n"]])
    return {"y": y.to(TYPES[case["r"]]), "n": n}


def _plain_norms_grad(s):
    case = s["case"]
    f, d_y = s["f"].float(), s["dy"].float()
    out = {"dgate": None, "dw_after": None, "dw_before": None}
    if s["w_before"] is not None:
        y, dn = s["y"].float(), s["dn"].float()
        by = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
        unit, v = y * by, dn * s["w_before"]
        out["dw_before"] = (dn * unit).sum(0)
        d_y = d_y + by * (v - unit * (v * unit).mean(-1, keepdim=True))
    branch = f
    if s["w_after"] is not None:
        by = torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
        unit = f * by
        branch = unit * s["w_after"]
    if s["gate"] is not None:
        out["dgate"] = (d_y * branch).sum(-1)
    d_f = d_y if s["gate"] is None else d_y * s["gate"][:, None]
    if s["w_after"] is not None:
        out["dw_after"] = (d_f * unit).sum(0)
        v = d_f * s["w_after"]
        d_f = by * (v - unit * (v * unit).mean(-1, keepdim=True))
    return {"df": d_f.to(s["f"].dtype), "dr": (case["alpha"] * d_y).to(TYPES[case["r"]]), **out}


def _plain_ffn_grad(s, x, a, b):
    t = s["x"].dtype
    dy = s["dy"].float()
    w_in, w_gate, w_out = (s[w].float() for w in ("w_in", "w_gate", "w_out"))
    dh = dy @ w_out
    sig = 1.0 / (1.0 + torch.exp(-a))
    silu = a * sig
    da, db = dh * b * (sig + silu * (1.0 - sig)), dh * silu
    return {"dx": (da @ w_in + db @ w_gate).to(t), "dw_in": (da.t() @ x).to(t), "dw_gate": (db.t() @ x).to(t),
            "dw_out": (dy.t() @ (silu * b)).to(t)}


def _plain_keep8(v, kind):
    """The values that stay of v [T][d] fp32: in blocks of 32 columns code 2^e, e = floor(log2(largest)) - 6, codes of 7 bits and a sign."""
    T, d = v.shape
    pad = -d % 32
    blocks = torch.cat([v, torch.zeros((T, pad), device=v.device)], 1).view(T, -1, 32)
    top = blocks.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 7).clamp(min=-24 if kind == "f16" else -126)
    codes = (blocks * _power(-e)).round().clamp(-127, 127)
    return (codes * _power(e)).view(T, d + pad)[:, :d]


def _power(e):
    """2^e as fp32, for whole e of -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _plain_quantize(x):
    """(codes as fp32 whole numbers, scale): a row's largest value is 127 of its scale. Quotients are those of fp32, through 64 bits: a
    quotient half way between two codes has to be the same one everywhere."""
    scale = (x.abs().amax(-1).double() / 127.0).float().clamp(min=2.0 ** -126)
    return (x.double() / scale.double()[:, None]).float().round(), scale


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    """Bytes: every input once and every output once. Operations: the multiply-adds of the products, and those of an element's norms."""
    kind, T = case["kind"], case["tokens"]
    if kind in ("norms", "norms_grad"):
        d = case["d"]
        f, r, n = BYTES[case["f"]], BYTES[case["r"]], BYTES[case["n"]] if case["before"] else 0
        vectors = 4 * d * (case["after"] + case["before"]) + (4 * T if case["gate"] else 0)
        if kind == "norms":
            return {"bytes": T * d * (f + 2 * r + n) + vectors, "flops": 9.0 * T * d}
        # (y is read for the norm before only)
        return {"bytes": T * d * (2 * f + 2 * r + (r if case["before"] else 0) + n) + 2 * vectors, "flops": 20.0 * T * d}
    if kind in ("ffn", "ffn_grad", "ffn_step8"):
        d, f, sz = case["d"], case["f"], BYTES[case["type"]]
        weights, rows = 3 * d * f * sz, T * d * sz
        if kind == "ffn":
            return {"bytes": weights + 2 * rows, "flops": 6.0 * T * d * f}
        if kind == "ffn_grad":
            return {"bytes": 2 * weights + 3 * rows + 2 * T * f * sz, "flops": 12.0 * T * d * f}
        return {"bytes": 2 * weights + 4 * rows, "flops": 18.0 * T * d * f}
    if kind == "keep8":
        return {"bytes": 2 * T * case["d"] * BYTES[case["type"]], "flops": 4.0 * T * case["d"]}
    k, n, so = case["k"], case["n"], BYTES[case["out"]]
    return {"bytes": T * k * BYTES[case["type"]] + n * k + 4 * n + T * n * so * (2 if case["base"] else 1), "flops": 2.0 * T * k * n}


# ---- the same in 64 bits, from the definitions ------------------------------------------------------------------------

def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    kind = case["kind"]
    if kind == "norms":
        return _exact_norms(case, s)
    if kind == "norms_grad":
        return _exact_norms_grad(case, s)
    if kind == "keep8":
        return {"x": _exact_keep8(s["x"].double(), case["type"])}
    if kind == "matmul8":
        x = s["x"].double()
        # the scale is an fp32 number, and a code the nearest whole number to an fp32 quotient
        scale = (x.abs().amax(1) / 127.0).float().clamp(min=torch.finfo(torch.float32).tiny).double()
        codes = torch.round((x / scale[:, None]).float()).double()
        y = torch.mm(codes, s["w_codes"].double().t().contiguous()) * scale[:, None] * s["w_scale"].double()
        return {"y": y if s["base"] is None else y + s["base"].double()}
    x = s["x"].double()
    w_in, w_gate, w_out = (s[w].double() for w in ("w_in", "w_gate", "w_out"))
    got = {}
    if kind == "ffn_grad":
        a, b = s["ab"].double().unbind(0)
    else:
        a, b = torch.mm(x, w_in.t().contiguous()), torch.mm(x, w_gate.t().contiguous())
        got["y"] = torch.mm(a * torch.sigmoid(a) * b, w_out.t().contiguous())
        if kind == "ffn":
            return got
        x, a, b = (_exact_keep8(v, case["type"]) for v in (x, a, b))
    dy = s["dy"].double()
    dh = torch.mm(dy, w_out)
    g = torch.sigmoid(a)
    da = dh * b * g * (1.0 + a * (1.0 - g))
    db = dh * a * g
    got["dx"] = torch.mm(da, w_in) + torch.mm(db, w_gate)
    got["dw_in"], got["dw_gate"] = torch.mm(da.t().contiguous(), x), torch.mm(db.t().contiguous(), x)
    got["dw_out"] = torch.mm(dy.t().contiguous(), a * g * b)
    return got


def _exact_norms(case, s):
    y = s["f"].double()
    if s["w_after"] is not None:
        y = y / torch.sqrt(y.square().mean(1, keepdim=True) + EPS) * s["w_after"].double()
    if s["gate"] is not None:
        y = y * s["gate"].double()[:, None]
    y = y + case["alpha"] * s["r"].double()
    n = None if s["w_before"] is None else y / torch.sqrt(y.square().mean(1, keepdim=True) + EPS) * s["w_before"].double()
    return {"y": y, "n": n}


def _exact_norms_grad(case, s):
    """Through the sizes u = sqrt(mean v^2 + eps): N(v) = v / u w has the gradient (w g - v (v . w g) / (d u^2)) / u."""
    d = case["d"]

    def back(v, w, g):
        u = torch.sqrt(v.square().mean(1, keepdim=True) + EPS)
        wg = w * g
        return (wg - v * ((v * wg).sum(1, keepdim=True) / (d * u.square()))) / u, v / u

    f, total = s["f"].double(), s["dy"].double()
    got = {"dgate": None, "dw_after": None, "dw_before": None}
    if s["w_before"] is not None:
        dn = s["dn"].double()
        more, unit = back(s["y"].double(), s["w_before"].double(), dn)
        total = total + more
        got["dw_before"] = (dn * unit).sum(0)
    gate = 1.0 if s["gate"] is None else s["gate"].double()[:, None]
    df, branch = total * gate, f
    if s["w_after"] is not None:
        w = s["w_after"].double()
        grad = df
        df, unit = back(f, w, grad)
        got["dw_after"] = (grad * unit).sum(0)
        branch = unit * w
    if s["gate"] is not None:
        got["dgate"] = (total * branch).sum(1)
    return {"df": df, "dr": case["alpha"] * total, **got}


def _exact_keep8(v, kind):
    T, d = v.shape
    out = torch.zeros_like(v)
    low = -24 if kind == "f16" else -126
    full = d // 32 * 32
    for part in ((v[:, :full].reshape(T, -1, 32), slice(0, full)), (v[:, full:].reshape(T, 1, -1), slice(full, d))):
        blocks, at = part
        if blocks.numel() == 0:
            continue
        top = blocks.abs().amax(2, keepdim=True)
        # (the unit from its exponent's bits: a power that is off in its last place moves the values half way between two codes)
        e = (torch.floor(torch.log2(top.clamp(min=2.0 ** -300))) - 6.0).clamp(min=low)
        unit = ((e.long() + 1023) << 52).view(torch.float64)
        out[:, at] = (torch.round(blocks / unit).clamp(-127.0, 127.0) * unit).reshape(T, -1)
    return out
