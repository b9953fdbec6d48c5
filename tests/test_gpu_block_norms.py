"""The norms around a block with gate and residual, and their gradient, against plain arithmetic in 64 bits on the host."""
import numpy as np
import pytest
import torch

import paper_2308_14352_amd as moeq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
STEP = 2.0**-24                          # a rounding of fp32, relative
# Roundings on the way of a value: at most 32 additions in a thread, 6 in a wavefront, 8 between wavefronts, and some 20 operations on
# either side of the two sums; the bounds below take every one of them with its largest error and the same sign.
CHAIN = 128


def strided(t, pad, shift):
    buf = torch.full((t.shape[0] * (t.shape[1] + pad) + shift,), float("nan"), dtype=t.dtype, device=t.device)
    v = buf[shift:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
    v.copy_(t)
    return v


def make(T, d, f, r, n, seed=0):
    g = np.random.default_rng([T, d, seed])
    t = lambda kind, *s, by=1.0, at=0.0: torch.from_numpy(g.normal(size=s) * by + at).to(TYPES[kind])
    return dict(f=t(f, T, d, by=2.0), r=t(r, T, d), dy=t(r, T, d), dn=t(n, T, d), gate=t("f32", T, at=0.5), w_after=t("f32", d, at=1.0),
                w_before=t("f32", d, at=1.0))


def norm(v, eps):
    return 1 / np.sqrt((v * v).mean(1, keepdims=True) + eps)


def forward(m, parts, alpha, eps):
    """y, n and the magnitudes of what they are made of."""
    d = {k: v.double().numpy() for k, v in m.items()}
    b, mag = d["f"], np.abs(d["f"])
    if "a" in parts:
        by = norm(d["f"], eps) * d["w_after"]
        b, mag = b * by, mag * np.abs(by)
    if "g" in parts:
        b, mag = b * d["gate"][:, None], mag * np.abs(d["gate"][:, None])
    y, mag = alpha * d["r"] + b, np.abs(alpha * d["r"]) + mag
    n = y * norm(y, eps) * d["w_before"]
    # (the size that n is divided by is off by its own roundings and by those of y: both relative to the row's)
    spread = np.sqrt((mag * mag).mean(1, keepdims=True)) * norm(y, eps)
    return y, mag, n, (mag * norm(y, eps) + np.abs(y) * norm(y, eps) * spread) * np.abs(d["w_before"])


def close(got, want, mag, kind, what):
    got = got.detach().cpu().double().numpy()
    # half a step of the type; fp16 below its normal numbers: half of 2^-24
    tol = np.abs(want) * torch.finfo(TYPES[kind]).eps / 2 + CHAIN * STEP * mag + (2.0**-25 if kind == "f16" else 1e-37)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, bad.sum(), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])


SHAPES = [(1, 1), (1, 64), (3, 8), (5, 33), (7, 511), (2, 513), (4, 1000), (9, 1025), (3, 2048), (2, 2051), (3, 4096), (2, 4104), (2, 8192), (3, 8200), (2, 16384), (1, 16381)]
KINDS = [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "bf16"), ("f16", "f16", "f16"), ("bf16", "f32", "bf16"),
         ("bf16", "bf16", "f32"), ("f32", "f32", "f16"), ("f16", "f32", "f32"), ("f32", "f16", "f32")]
PARTS = ["ab", "agb", "gb", "b", "a", "ag", "g", ""]


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("kinds", KINDS[:3])
def test_forward_and_gradient_over_shapes(T, d, kinds):
    one(T, d, kinds, "agb", 0.5, 1e-5, 0)


@pytest.mark.parametrize("kinds", KINDS)
@pytest.mark.parametrize("parts", PARTS)
def test_forward_and_gradient_over_types_and_parts(kinds, parts):
    one(6, 200, kinds, parts, 1.25, 1e-6, 3)
    one(2, 1030, kinds, parts, 1.0, 1e-5, 1)


def test_many_rows_share_a_stream():
    one(5000, 72, KINDS[0], "agb", 1.0, 1e-5, 0)
    one(1100, 2056, KINDS[1], "agb", 1.0, 1e-5, 8)
    one(4097, 1, KINDS[0], "agb", 1.0, 1e-5, 0)


def one(T, d, kinds, parts, alpha, eps, pad):
    f, r, n = kinds
    m = make(T, d, *kinds)
    dev = {k: v.to(DEV) for k, v in m.items()}
    fs, rs = strided(dev["f"], pad, pad), strided(dev["r"], 2 * pad, 1)
    kw = dict(gate=dev["gate"] if "g" in parts else None, w_after=dev["w_after"] if "a" in parts else None,
              w_before=dev["w_before"] if "b" in parts else None, residual_scale=alpha, eps=eps)
    y, nn = moeq.moe_block_norms_forward(fs, rs, dtype=TYPES[n], **kw)
    wy, ymag, wn, nmag = forward(m, parts, alpha, eps)
    close(y, wy, ymag, r, "y")
    assert y.dtype == TYPES[r] and (nn is None) == ("b" not in parts)
    if nn is not None:
        close(nn, wn, nmag, n, "n")
        assert nn.dtype == TYPES[n]

    # the gradient, from the y that was left
    df, dr, dg, da, db = moeq.moe_block_norms_backward(fs, y if "b" in parts else None, strided(dev["dy"], pad, 1),
                                                       strided(dev["dn"], 3, pad) if "b" in parts else None, **kw)
    q = {k: v.double().numpy() for k, v in m.items()}
    yq = y.cpu().double().numpy()
    dY, dYm = q["dy"], np.abs(q["dy"])
    if "b" in parts:
        by = norm(yq, eps)
        u, v = yq * by, q["dn"] * q["w_before"]
        dY = dY + by * (v - u * (v * u).mean(1, keepdims=True))
        dYm = dYm + by * (np.abs(v) + np.abs(u) * np.abs(v * u).mean(1, keepdims=True))
        close(db, (q["dn"] * u).sum(0), np.abs(q["dn"] * u).sum(0) * np.sqrt(T), "f32", "dw_before")
    else:
        assert db is None
    close(dr, alpha * dY, abs(alpha) * dYm, r, "dr")
    gate = q["gate"][:, None] if "g" in parts else 1.0
    bf = norm(q["f"], eps) if "a" in parts else 1.0
    w = q["w_after"] if "a" in parts else 1.0
    S, Sm = (dY * q["f"] * bf * w).sum(1), (dYm * np.abs(q["f"] * bf * w)).sum(1)
    if "g" in parts:
        close(dg, S, Sm, "f32", "dgate")
    else:
        assert dg is None
    if "a" in parts:
        u = q["f"] * bf
        close(da, (dY * gate * u).sum(0), (dYm * np.abs(gate * u)).sum(0) * np.sqrt(T), "f32", "dw_after")
        df_w = bf * (dY * gate * w - u * gate * S[:, None] / d)
        df_m = bf * (dYm * np.abs(gate * w) + np.abs(u * gate) * Sm[:, None] / d)
    else:
        assert da is None
        df_w, df_m = dY * gate, dYm * np.abs(gate)
    close(df, df_w, df_m, f, "df")


def test_gradient_against_differences():
    T, d, eps, h = 3, 40, 1e-3, 1e-5
    m = {k: v.double() for k, v in make(T, d, "f32", "f32", "f32").items()}
    dev = {k: v.float().to(DEV) for k, v in m.items()}
    kw = dict(gate=dev["gate"], w_after=dev["w_after"], w_before=dev["w_before"], residual_scale=0.7, eps=eps)
    y, _ = moeq.moe_block_norms_forward(dev["f"], dev["r"], **kw)
    got = dict(zip(("f", "r", "gate", "w_after", "w_before"), moeq.moe_block_norms_backward(dev["f"], y, dev["dy"], dev["dn"], **kw)))

    def loss(p):
        yy, _, n, _ = forward(p, "agb", 0.7, eps)
        return (yy * m["dy"].numpy()).sum() + (n * m["dn"].numpy()).sum()

    g = np.random.default_rng(5)
    for name, grad in got.items():
        for _ in range(4):
            at = tuple(int(g.integers(s)) for s in grad.shape)
            p = {k: v.clone() for k, v in m.items()}
            p[name][at] += h
            up = loss(p)
            p[name][at] -= 2 * h
            # differences: h^2 of the third derivative, 2^-53 of the loss / h; the kernel: fp32 of the terms, of which the largest is some 30
            assert abs((up - loss(p)) / (2 * h) - grad[at].item()) < 1e-4, name


def test_in_place_and_given_outputs():
    m = {k: v.to(DEV) for k, v in make(9, 520, "bf16", "bf16", "bf16").items()}
    kw = dict(gate=m["gate"], w_after=m["w_after"], w_before=m["w_before"])
    y, n = moeq.moe_block_norms_forward(m["f"], m["r"], **kw)
    f, r = m["f"].clone(), m["r"].clone()
    y2, n2 = moeq.moe_block_norms_forward(f, r, y=r, n=f, **kw)
    assert y2 is r and n2 is f and torch.equal(r, y) and torch.equal(f, n)
    df, dr, *_ = moeq.moe_block_norms_backward(m["f"], y, m["dy"], m["dn"], **kw)
    buf = torch.full((9, 2, 520), 7.0, dtype=torch.bfloat16, device=DEV)
    moeq.moe_block_norms_backward(m["f"], y, m["dy"], m["dn"], df=buf[:, 0], dr=buf[:, 1], **kw)
    assert torch.equal(buf[:, 0], df) and torch.equal(buf[:, 1], dr)


def test_rows_of_nan_and_of_zeros_stay_with_themselves():
    m = make(6, 300, "f32", "f32", "f32")
    m["f"][2, 5], m["r"][4, 0] = float("nan"), float("inf")
    m["f"][1], m["r"][1] = 0, 0
    dev = {k: v.to(DEV) for k, v in m.items()}
    kw = dict(gate=dev["gate"], w_after=dev["w_after"], w_before=dev["w_before"])
    y, n = moeq.moe_block_norms_forward(dev["f"], dev["r"], **kw)
    assert n[2].isnan().all() and not n[4].isfinite().all() and y[[0, 1, 3, 5]].isfinite().all() and n[[0, 1, 3, 5]].isfinite().all()
    assert (y[1] == 0).all() and (n[1] == 0).all()
    df, dr, dg, _, _ = moeq.moe_block_norms_backward(dev["f"], y, dev["dy"], dev["dn"], **kw)
    keep = [0, 1, 3, 5]
    assert df[keep].isfinite().all() and dr[keep].isfinite().all() and dg[keep].isfinite().all() and dg[2].isnan()


def test_no_rows():
    e = torch.empty((0, 40), device=DEV)
    w = torch.ones(40, device=DEV)
    y, n = moeq.moe_block_norms_forward(e, e.clone(), w_before=w)
    assert y.shape == n.shape == (0, 40)
    df, dr, dg, da, db = moeq.moe_block_norms_backward(e, y, e.clone(), n, gate=torch.empty(0, device=DEV), w_after=w, w_before=w)
    assert df.shape == (0, 40) and dg.shape == (0,) and (da == 0).all() and (db == 0).all()


def test_same_bits_again_and_on_another_stream_and_in_a_graph():
    m = {k: v.to(DEV) for k, v in make(700, 1500, "bf16", "bf16", "bf16").items()}
    kw = dict(gate=m["gate"], w_after=m["w_after"], w_before=m["w_before"])
    run = lambda stream=None: (lambda yn: yn + moeq.moe_block_norms_backward(m["f"], yn[0], m["dy"], m["dn"], stream=stream, **kw))(
        moeq.moe_block_norms_forward(m["f"], m["r"], stream=stream, **kw))
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    for _ in range(3):
        for t in got:
            t.fill_(3.0)
        g.replay()
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
