"""Operators around a mixture-of-experts layer, as cases that can be timed and checked: tokens sorted by expert and
back, low-rank adapters of many requests beside a shared projection, and distillation from a teacher's top logits.

A case is a dict of plain values. `kind` says which operator a pass goes through:

  dispatch      (token, choice) pairs sorted by expert, and the tokens' rows copied into that order
  combine       expert rows back to tokens, weighted by the gates (or the gradient of `dispatch`: not weighted)
  combine_grad  the gradient of the weighted combine: with respect to the rows and to the gates
  adapt         y = base + scale_a B_a A_a x, every row with its own adapter a or none
  adapt_grad    the gradient of that: with respect to x, A and B
  distill       the loss of every row and its log-sum-exp
  distill_grad  the gradient from a saved log-sum-exp and the gradients of the losses
  distill_both  the loss of every row and the gradient of their sum in one call

`own` chooses between plain torch arithmetic and the framework's entry points.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # serving: eight sequences decoded together with a Switch-base layer of 64 experts; launches and latency only
        dict(name="dispatch_batch8", kind="dispatch", tokens=8, k=1, experts=64, d=768, type="f32", drop=0.0),
        # a prompt of 2048 tokens through a Mixtral-shaped layer, two choices a token
        dict(name="dispatch_prompt_2048", kind="dispatch", tokens=2048, k=2, experts=8, d=4096, type="bf16", drop=0.0),
        # an odd prompt back from 128 experts (Switch-large width), rows as the experts write them; a few pairs were dropped
        dict(name="combine_prompt_1117", kind="combine", tokens=1117, k=2, experts=128, d=1024, type="f32", out="f32",
             gates=True, drop=0.03),
        # a training step's gradient of the combine: a batch of four sequences of 2048
        dict(name="combine_grad_8192", kind="combine_grad", tokens=8192, k=2, experts=8, d=4096, type="bf16", out="bf16",
             gates=True, drop=0.0),
        # serving: nine requests decoded together, each with an adapter of its own out of 32 resident ones
        dict(name="adapt_batch9", kind="adapt", tokens=9, adapters=32, rank=16, d_in=4096, d_out=4096, type="bf16",
             out="bf16", ids="each", base=True),
        # serving: prompts of many requests in one batch, ragged, beside the layer's fp32 outputs
        dict(name="adapt_prompts_4100", kind="adapt", tokens=4100, adapters=24, rank=16, d_in=4096, d_out=4096,
             type="bf16", out="f32", ids="runs", base=True),
        # a small fp32 model, odd rank, rows of all adapters mixed
        dict(name="adapt_mixed_500", kind="adapt", tokens=500, adapters=64, rank=5, d_in=768, d_out=1000, type="f32",
             out="f32", ids="mixed", base=False),
        # healing: the experts' adapters on rows sorted by expert, unevenly loaded
        dict(name="adapt_grad_experts_8192", kind="adapt_grad", tokens=8192, adapters=8, rank=32, d_in=4096, d_out=4096,
             type="bf16", out="bf16", ids="experts", base=True),
        # the same for a small fp16 model and a short odd batch
        dict(name="adapt_grad_777", kind="adapt_grad", tokens=777, adapters=16, rank=8, d_in=1024, d_out=1024, type="f16",
             out="f16", ids="runs", base=False),
        # evaluating a quantized model against its teacher, a few rows with a long vocabulary
        dict(name="distill_rows_13", kind="distill", tokens=13, vocab=131072, top=64, type="f32", temperature=1.0, masked=0.0),
        # the backward pass alone, odd vocabulary, padding rows masked
        dict(name="distill_grad_1000", kind="distill_grad", tokens=1000, vocab=50257, top=20, type="f16", temperature=2.0,
             masked=0.2),
        # a training step's loss and gradient
        dict(name="distill_both_4096", kind="distill_both", tokens=4096, vocab=32000, top=64, type="bf16", temperature=2.0,
             masked=0.05),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges: one token to long batches, narrow to wide and odd widths, every kind and type."""
    kind = rng.choice(["dispatch", "combine", "combine_grad", "adapt", "adapt", "adapt_grad", "adapt_grad", "distill",
                       "distill_grad", "distill_both"])
    t = rng.choice(["f32", "bf16", "bf16", "f16"])
    c = dict(kind=kind, type=t)
    if kind in ("dispatch", "combine", "combine_grad"):
        d = rng.choice([_log_int(rng, 64, 4096), 64 * rng.randint(4, 64), 128 * rng.randint(2, 32)])
        k = rng.choice([1, 1, 2, 2, 3, 4, 8])
        most = max(1, min(16384, 8192 * 2 * 4096 * 2 // (k * d * BYTES[t])))
        c.update(tokens=_log_int(rng, 1, most), k=k, experts=max(k, rng.choice([8, 16, 33, 64, 128, 256])), d=d,
                 drop=rng.choice([0.0, 0.0, 0.05]))
        if kind != "dispatch":
            c.update(out=rng.choice([t, "f32"]), gates=kind == "combine_grad" or rng.random() < 0.7)
    elif kind in ("adapt", "adapt_grad"):
        c.update(adapters=_log_int(rng, 1, 64), rank=rng.choice([4, 8, 8, 16, 16, 32, 64, rng.randint(1, 64)]),
                 d_in=rng.choice([_log_int(rng, 128, 4096), 128 * rng.randint(2, 32)]),
                 d_out=rng.choice([_log_int(rng, 128, 4096), 128 * rng.randint(2, 32)]),
                 tokens=_log_int(rng, 1, 8192 if t != "f32" else 4096), out=rng.choice([t, t, "f32"]), base=rng.random() < 0.6)
        c["ids"] = rng.choice(["each", "runs", "mixed", "experts"] if c["tokens"] <= 64 else ["runs", "mixed", "experts"])
    else:
        vocab = _log_int(rng, 1000, 131072)
        most = min(4096, 4096 * 32000 * 2 // (vocab * BYTES[t]))
        c.update(vocab=vocab, tokens=_log_int(rng, 1, most), top=_log_int(rng, 1, 128),
                 temperature=rng.choice([1.0, 1.0, 2.0, 4.0, 0.7]), masked=rng.choice([0.0, 0.1]))
    return c


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed, *parts):
    g = torch.Generator(device=DEV)
    g.manual_seed(random.Random(repr((int(seed),) + parts)).getrandbits(62))
    return g


def _randn(shape, std, kind, seed, *parts):
    return (torch.randn(shape, generator=_gen(seed, *parts), device=DEV, dtype=torch.float32) * std).to(TYPES[kind])


def _routing(case, seed):
    """idx [T][k]: distinct experts of uneven popularity, a share of the pairs dropped (-1). gate [T][k], sums of 1."""
    T, k, E = case["tokens"], case["k"], case["experts"]
    logits = _randn((E,), 0.7, "f32", seed, "popular") + _randn((T, E), 1.0, "f32", seed, "router")
    top, idx = torch.topk(logits, k, dim=-1)
    gate = torch.softmax(top, -1)
    idx = idx.to(torch.int32)
    if case["drop"]:
        idx[torch.rand((T, k), generator=_gen(seed, "drop"), device=DEV) < case["drop"]] = -1
    return idx.contiguous(), gate.contiguous()


def _adapter_ids(case, seed):
    """ids [T]: of each row, -1 for none. each: a request a row; runs: ragged requests of several rows; mixed: rows of all
    requests in any order; experts: sorted, unevenly loaded."""
    T, n = case["tokens"], case["adapters"]
    rng = random.Random(repr((int(seed), "ids")))
    if case["ids"] == "runs":
        ids = []
        while len(ids) < T:
            ids += [rng.choice([-1] + list(range(n)) * 2)] * _log_int(rng, 1, max(2, T // 4))
        ids = ids[:T]
    elif case["ids"] == "experts":
        share = [math.exp(rng.gauss(0.0, 0.7)) for _ in range(n)]
        ids = sorted(rng.choices(range(n), weights=share, k=T))
    else:
        ids = [rng.randrange(-1, n) if rng.random() < 0.1 else rng.randrange(n) for _ in range(T)]
    return torch.tensor(ids, dtype=torch.int32, device=DEV)


def _adapters(case, seed):
    n, r = case["adapters"], case["rank"]
    A = _randn((n, r, case["d_in"]), 1.0 / math.sqrt(case["d_in"]), case["type"], seed, "A")
    B = _randn((n, case["d_out"], r), 0.05, case["type"], seed, "B")
    scale = torch.rand((n,), generator=_gen(seed, "scale"), device=DEV) * 1.5 + 0.5
    return A, B, scale


def _teacher(case, seed, logits):
    """The teacher's largest logits of every row: the student's with noise on them, and the temperature of neither."""
    z = logits.float() + torch.randn(logits.shape, generator=_gen(seed, "teacher"), device=DEV) * 0.7
    val, idx = torch.topk(z, case["top"], dim=-1)
    return idx.to(torch.int32).contiguous(), val.contiguous()


def _row_weights(case, seed):
    if not case["masked"]:
        return None
    w = torch.rand((case["tokens"],), generator=_gen(seed, "weight"), device=DEV) + 0.5
    w[torch.rand((case["tokens"],), generator=_gen(seed, "masked"), device=DEV) < case["masked"]] = 0.0
    return w


def prepare(case, seed):
    kind, t = case["kind"], case["type"]
    s = {"case": case}
    if kind in ("dispatch", "combine", "combine_grad"):
        T, k, d = case["tokens"], case["k"], case["d"]
        s["idx"], gate = _routing(case, seed)
        if kind == "dispatch":
            s["x"] = _randn((T, d), 1.0, t, seed, "x")
            return s
        s["gate"] = gate if case["gates"] else None
        s["rows"] = _randn((T * k, d), 1.0, t, seed, "rows")
        if kind == "combine_grad":
            s["dy"] = _randn((T, d), 1.0, case["out"], seed, "dy")
        # (the order that the rows are in: what the same program's dispatch left behind)
        if own:
            import paper_2308_14352_amd as moeq
            s["sort"] = moeq.moe_sort_pairs(s["idx"], case["experts"])
        else:
            s["sort"] = _plain_sort(s["idx"], case["experts"])
        return s
    if kind in ("adapt", "adapt_grad"):
        T = case["tokens"]
        s["ids"] = _adapter_ids(case, seed)
        s["A"], s["B"], s["scale"] = _adapters(case, seed)
        s["x"] = _randn((T, case["d_in"]), 1.0, t, seed, "x")
        wide = case["d_out"] if kind == "adapt" else case["d_in"]
        s["base"] = _randn((T, wide), 1.0, case["out"], seed, "base") if case["base"] else None
        if kind == "adapt_grad":
            s["dy"] = _randn((T, case["d_out"]), 1.0, case["out"], seed, "dy")
        if own:
            import paper_2308_14352_amd as moeq
            s["adapters"] = moeq.Adapters(s["A"], s["B"], s["scale"])
        return s
    s["logits"] = _randn((case["tokens"], case["vocab"]), 2.5, t, seed, "logits")
    s["top_idx"], s["top_logits"] = _teacher(case, seed, s["logits"])
    s["weight"] = _row_weights(case, seed)
    if kind == "distill_grad":
        s["dloss"] = torch.rand((case["tokens"],), generator=_gen(seed, "dloss"), device=DEV) + 0.5
        s["lse"] = torch.logsumexp(s["logits"].double() / case["temperature"], -1).float()
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2308_14352_amd as moeq
    case = s["case"]
    kind = case["kind"]
    if kind == "dispatch":
        sort = moeq.moe_sort_pairs(s["idx"], case["experts"])
        rows = moeq.moe_gather_rows(sort, s["x"])
        return {"offsets": sort.offsets, "order": sort.order, "slot": sort.slot, "rows": rows}
    if kind == "combine":
        return {"y": moeq.moe_combine_rows(s["sort"], s["rows"], s["gate"], dtype=TYPES[case["out"]])}
    if kind == "combine_grad":
        drows, dgate = moeq.moe_combine_rows_backward(s["sort"], s["dy"], s["rows"], s["gate"])
        return {"drows": drows, "dgate": dgate}
    if kind == "adapt":
        y = torch.empty((case["tokens"], case["d_out"]), dtype=TYPES[case["out"]], device=DEV)
        return {"y": moeq.moe_adapters_forward(s["adapters"], s["x"], s["ids"], base=s["base"], y=y)}
    if kind == "adapt_grad":
        dx = torch.empty((case["tokens"], case["d_in"]), dtype=TYPES[case["out"]], device=DEV)
        dx, dA, dB = moeq.moe_adapters_backward(s["adapters"], s["x"], s["ids"], s["dy"], dx_base=s["base"], dx=dx)
        return {"dx": dx, "dA": dA, "dB": dB}
    teacher = (s["top_idx"], s["top_logits"])
    if kind == "distill":
        loss, lse = moeq.moe_distill_forward(s["logits"], *teacher, temperature=case["temperature"], weight=s["weight"])
        return {"loss": loss, "lse": lse}
    if kind == "distill_grad":
        return {"dlogits": moeq.moe_distill_backward(s["logits"], *teacher, s["lse"], s["dloss"],
                                                     temperature=case["temperature"], weight=s["weight"])}
    loss, dlogits = moeq.moe_distill_loss_grad(s["logits"], *teacher, temperature=case["temperature"], weight=s["weight"])
    return {"loss": loss, "dlogits": dlogits}


def _plain_sort(idx, E):
    """offsets [E + 1], order [P] (the pair in every place) and slot [P] (the place of every pair). Pairs without an
    expert come last, as ~pair and ~place."""
    e = idx.flatten().long()
    e = torch.where((e < 0) | (e >= E), torch.full_like(e, E), e)
    key, order = torch.sort(e, stable=True)
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=idx.device)
    offsets[1:] = (e[:, None] == torch.arange(E, device=idx.device)).sum(0).cumsum(0)
    place = torch.arange(e.numel(), device=idx.device)
    slot = torch.empty_like(place)
    slot[order] = torch.where(key == E, ~place, place)
    return offsets.to(torch.int32), torch.where(key == E, ~order, order).to(torch.int32), slot.to(torch.int32)


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "dispatch":
        offsets, order, slot = _plain_sort(s["idx"], case["experts"])
        kept = (order >= 0)[:, None]
        rows = torch.where(kept, s["x"][order.clamp(min=0).long() // case["k"]], torch.zeros((), dtype=s["x"].dtype, device=DEV))
        return {"offsets": offsets, "order": order, "slot": slot, "rows": rows}
    if kind in ("combine", "combine_grad"):
        T, k, d = case["tokens"], case["k"], case["d"]
        offsets, order, slot = s["sort"]
        kept = (slot >= 0).view(T, k)
        at = torch.where(slot >= 0, slot, ~slot).long()
        gate = s["gate"] if s["gate"] is not None else torch.ones((T, k), device=DEV)
        gate = torch.where(kept, gate, torch.zeros_like(gate))
        rows = s["rows"].float()[at].view(T, k, d)
        if kind == "combine":
            return {"y": (gate[:, :, None] * rows).sum(1).to(TYPES[case["out"]])}
        dy = s["dy"].float()[:, None, :]
        dgate = torch.where(kept, (dy * rows).sum(-1), torch.zeros_like(gate))
        drows = torch.empty_like(s["rows"])
        drows[at] = (gate[:, :, None] * dy).reshape(T * k, d).to(drows.dtype)
        return {"drows": drows, "dgate": dgate}
    if kind in ("adapt", "adapt_grad"):
        return _plain_adapters(s)
    return _plain_distill(s)


def _plain_adapters(s):
    case = s["case"]
    wide = case["d_out"] if case["kind"] == "adapt" else case["d_in"]
    out = s["base"].float() if s["base"] is not None else torch.zeros((case["tokens"], wide), device=DEV)
    groups = [(a, (s["ids"] == a).nonzero()[:, 0]) for a in torch.unique(s["ids"]).tolist() if a >= 0]
    x, scale = s["x"].float(), s["scale"].tolist()
    if case["kind"] == "adapt":
        add = torch.zeros_like(out)
        for a, t in groups:
            add[t] = scale[a] * ((x[t] @ s["A"][a].float().t()) @ s["B"][a].float().t())
        return {"y": (out + add).to(TYPES[case["out"]])}
    dy = s["dy"].float()
    add = torch.zeros_like(out)
    dA = torch.zeros(s["A"].shape, device=DEV)
    dB = torch.zeros(s["B"].shape, device=DEV)
    for a, t in groups:
        A, B = s["A"][a].float(), s["B"][a].float()
        xt, dyt = x[t], dy[t]
        g = scale[a] * (dyt @ B)
        dA[a] = g.t() @ xt
        dB[a] = scale[a] * (dyt.t() @ (xt @ A.t()))
        add[t] = g @ A
    return {"dx": (out + add).to(TYPES[case["out"]]), "dA": dA, "dB": dB}


def _plain_distill(s):
    case = s["case"]
    tau = case["temperature"]
    sc = s["logits"].float() / tau
    idx = s["top_idx"].long()
    zt = s["top_logits"] / tau
    zt = zt - zt.amax(-1, keepdim=True)
    log_p = zt - zt.exp().sum(-1, keepdim=True).log()
    p = log_p.exp()
    w = s["weight"] if s["weight"] is not None else torch.ones(case["tokens"], device=DEV)
    if case["kind"] == "distill_grad":
        lse, w = s["lse"], w * s["dloss"]
    else:
        top = sc.amax(-1)
        lse = (sc - top[:, None]).exp().sum(-1).log() + top
    out = {}
    if case["kind"] != "distill_grad":
        out["loss"] = w * tau * tau * (p * (log_p - sc.gather(1, idx) + lse[:, None])).sum(-1)
    if case["kind"] == "distill":
        return {"loss": out["loss"], "lse": lse}
    grad = (sc - lse[:, None]).exp()
    grad.scatter_add_(1, idx, -p)
    out["dlogits"] = (grad * (w * tau)[:, None]).to(s["logits"].dtype)
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    """Bytes: every input once and every output once (of adapters those that the rows are expected to use). Operations:
    the multiply-adds, and for distillation four for an element of a sum of exponentials or of a gradient."""
    kind, sz = case["kind"], BYTES[case["type"]]
    T = case["tokens"]
    if kind in ("dispatch", "combine", "combine_grad"):
        d, k = case["d"], case["k"]
        P = T * k
        if kind == "dispatch":
            return {"bytes": T * d * sz + P * d * sz + 12 * P + 4 * (case["experts"] + 1), "flops": 1.0 * P}
        so = BYTES[case["out"]]
        one = T * d * so + P * d * sz + P * (8 if case["gates"] else 4)
        if kind == "combine":
            return {"bytes": one, "flops": 2.0 * P * d}
        return {"bytes": one + P * d * sz + 4 * P, "flops": 3.0 * P * d}
    if kind in ("adapt", "adapt_grad"):
        n, r, di, do, so = case["adapters"], case["rank"], case["d_in"], case["d_out"], BYTES[case["out"]]
        used = n * (1.0 - (1.0 - 1.0 / n) ** T)
        weights = used * r * (di + do) * sz + 4 * T
        if kind == "adapt":
            return {"bytes": weights + T * di * sz + T * do * so * (2 if case["base"] else 1),
                    "flops": 2.0 * T * r * (di + do)}
        return {"bytes": weights + T * di * sz + T * do * so + T * di * so * (2 if case["base"] else 1) + n * r * (di + do) * 4,
                "flops": 2.0 * T * r * (3 * di + 2 * do)}
    V, K = case["vocab"], case["top"]
    kept = T * (1.0 - case["masked"])
    read, teacher = kept * V * sz, kept * K * 8 + T * 8
    if kind == "distill":
        return {"bytes": read + teacher, "flops": 4.0 * kept * V}
    return {"bytes": read + teacher + T * V * sz, "flops": (4.0 if kind == "distill_grad" else 8.0) * kept * V}


# ---- the same in 64 bits, from the definitions ------------------------------------------------------------------------

def exact(case, seed):
    kind = case["kind"]
    was = prepare_inputs(case, seed)
    if kind in ("dispatch", "combine", "combine_grad"):
        return _exact_rows(case, was)
    if kind in ("adapt", "adapt_grad"):
        return _exact_adapters(case, was)
    return _exact_distill(case, was)


def prepare_inputs(case, seed):
    """The inputs alone, without what the framework keeps."""
    global own
    before, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = before


def _exact_rows(case, s):
    T, k, d, E = case["tokens"], case["k"], case["d"], case["experts"]
    flat = s["idx"].flatten().tolist()
    places = [[] for _ in range(E + 1)]
    for i, e in enumerate(flat):
        places[e if 0 <= e < E else E].append(i)
    order, offsets = [], [0]
    for e in range(E):
        order += places[e]
        offsets.append(len(order))
    n_kept = len(order)
    order += places[E]
    place = [0] * len(flat)
    for p, i in enumerate(order):
        place[i] = p
    pair = torch.tensor(order, device=DEV)
    place = torch.tensor(place, device=DEV)
    if case["kind"] == "dispatch":
        rows = s["x"].double()[pair // k]
        rows[n_kept:] = 0.0
        signed = torch.tensor([i if p < n_kept else ~i for p, i in enumerate(order)], dtype=torch.int32, device=DEV)
        slot = torch.where(place < n_kept, place, -1 - place).to(torch.int32)
        return {"offsets": torch.tensor(offsets, dtype=torch.int32, device=DEV), "order": signed, "slot": slot, "rows": rows}
    kept = (place < n_kept).view(T, k).double()
    gate = kept if s["gate"] is None else kept * s["gate"].double()
    if case["kind"] == "combine":
        y = torch.zeros((T, d), dtype=torch.float64, device=DEV)
        for j in range(k):
            y += gate[:, j, None] * s["rows"][place.view(T, k)[:, j]].double()
        return {"y": y}
    dy = s["dy"].double()
    drows = torch.zeros((T * k, d), dtype=torch.float64, device=DEV)
    dgate = torch.zeros((T, k), dtype=torch.float64, device=DEV)
    for j in range(k):
        at = place.view(T, k)[:, j]
        drows[at] = gate[:, j, None] * dy
        dgate[:, j] = kept[:, j] * (dy * s["rows"][at].double()).sum(1)
    return {"drows": drows, "dgate": dgate}


def _exact_adapters(case, s):
    forward = case["kind"] == "adapt"
    x, ids = s["x"].double(), s["ids"].tolist()
    out = torch.zeros((case["tokens"], case["d_out"] if forward else case["d_in"]), dtype=torch.float64, device=DEV)
    if s["base"] is not None:
        out += s["base"].double()
    dA = torch.zeros(s["A"].shape, dtype=torch.float64, device=DEV)
    dB = torch.zeros(s["B"].shape, dtype=torch.float64, device=DEV)
    for a in range(case["adapters"]):
        t = [i for i, v in enumerate(ids) if v == a]
        if not t:
            continue
        t = torch.tensor(t, device=DEV)
        A, B, c = s["A"][a].double(), s["B"][a].double(), s["scale"][a].double()
        h = torch.mm(x[t], A.t().contiguous())
        if forward:
            out[t] += c * torch.mm(h, B.t().contiguous())
            continue
        dy = s["dy"].double()[t]
        g = c * torch.mm(dy, B)
        out[t] += torch.mm(g, A)
        dA[a] = torch.mm(g.t().contiguous(), x[t])
        dB[a] = c * torch.mm(dy.t().contiguous(), h)
    return {"y": out} if forward else {"dx": out, "dA": dA, "dB": dB}


def _exact_distill(case, s):
    T, tau, kind = case["tokens"], case["temperature"], case["kind"]
    w = torch.ones(T, dtype=torch.float64, device=DEV) if s["weight"] is None else s["weight"].double()
    p = torch.softmax(s["top_logits"].double() / tau, -1)
    idx = s["top_idx"].long()
    loss = torch.empty(T, dtype=torch.float64, device=DEV)
    lse = torch.empty(T, dtype=torch.float64, device=DEV)
    grad = None if kind == "distill" else torch.empty((T, case["vocab"]), dtype=torch.float64, device=DEV)
    step = max(1, (1 << 26) // case["vocab"])
    for a in range(0, T, step):
        b = min(T, a + step)
        sc = s["logits"][a:b].double() / tau
        lse[a:b] = torch.logsumexp(sc, -1)
        at = s["lse"][a:b].double() if kind == "distill_grad" else lse[a:b]
        log_q = sc - at[:, None]
        loss[a:b] = w[a:b] * tau ** 2 * (torch.xlogy(p[a:b], p[a:b]) - p[a:b] * log_q.gather(1, idx[a:b])).sum(-1)
        if grad is not None:
            q = log_q.exp()
            q.scatter_add_(1, idx[a:b], -p[a:b])
            by = w[a:b] * tau * (s["dloss"][a:b].double() if kind == "distill_grad" else 1.0)
            grad[a:b] = q * by[:, None]
    if kind == "distill":
        return {"loss": loss, "lse": lse}
    return {"dlogits": grad} if kind == "distill_grad" else {"loss": loss, "dlogits": grad}
