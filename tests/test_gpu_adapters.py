"""Low-rank adapters of many requests and their gradient against plain arithmetic in 64 bits on the host: one row to many, every rank
class, widths that end inside a vector or tile, rows without an adapter, adapters without rows, every pair of types."""
import threading

import numpy as np
import pytest
import torch

import paper_2308_14352_amd as moeq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
PAIRS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")]


def rng_of(*parts):
    return np.random.default_rng([ord(c) for c in repr(parts)])


def strided(t, pad, shift):
    buf = torch.full((t.shape[0] * (t.shape[1] + pad) + shift,), float("nan"), dtype=t.dtype, device=t.device)
    v = buf[shift:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
    v.copy_(t)
    return v


def make(rng, T, n, r, d_in, d_out, t, out):
    f = lambda *s, by=1.0: torch.from_numpy(rng.normal(size=s) * by)
    return dict(A=f(n, r, d_in, by=d_in**-0.5).to(t), B=f(n, d_out, r, by=0.3).to(t), scale=(f(n) * 0.5 + 1).float(),
                x=f(T, d_in).to(t), dy=f(T, d_out).to(out), base=f(T, d_out).to(out), dx_base=f(T, d_in).to(out))


def ids_of(rng, T, n, how):
    if how == "none":
        return rng.choice(np.array([-1, n, 2**31 - 1, -2**31]), size=T).astype(np.int32)
    if how == "one":
        return np.full(T, n - 1, np.int32)
    if how == "sorted":
        return np.sort(rng.integers(0, n, size=T)).astype(np.int32)
    ids = rng.integers(-1, n + 1, size=T)                 # -1 and n: none
    return ids.astype(np.int32)


def reference(m, ids, n):
    """Outputs in 64 bits, and the sums of the magnitudes that they are made of (for the tolerances)."""
    d = {k: v.double().numpy() for k, v in m.items()}
    y, dx = d["base"].copy(), d["dx_base"].copy()
    ym, dxm = np.abs(y), np.abs(dx)
    dA, dB = np.zeros_like(d["A"]), np.zeros_like(d["B"])
    dAm, dBm = np.zeros_like(dA), np.zeros_like(dB)
    for a in range(n):
        t = np.nonzero(ids == a)[0]
        if not t.size:
            continue
        A, B, c, x, dy = d["A"][a], d["B"][a], d["scale"][a], d["x"][t], d["dy"][t]
        h, g = x @ A.T, dy @ B
        hm, gm = np.abs(x) @ np.abs(A).T, np.abs(dy) @ np.abs(B)
        y[t] += c * h @ B.T
        ym[t] += abs(c) * hm @ np.abs(B).T
        dx[t] += c * g @ A
        dxm[t] += abs(c) * gm @ np.abs(A)
        dA[a], dAm[a] = c * g.T @ x, abs(c) * gm.T @ np.abs(x)
        dB[a], dBm[a] = c * dy.T @ h, abs(c) * np.abs(dy).T @ hm
    return dict(y=(y, ym), dx=(dx, dxm), dA=(dA, dAm), dB=(dB, dBm))


def check(got, want, mag, steps):
    """Sums of `steps` fp32 roundings in a row, independent of each other: each is at most half a step (2^-24) of a partial sum that
    the magnitudes bound, together the square root of their number, 8 times that for the largest of all; and the output's own."""
    half = torch.finfo(got.dtype).eps / 2
    tol = 8 * (steps + 16) ** 0.5 * 2.0**-24 * mag + half * np.abs(want) * 1.001 + (2.0**-25 if got.dtype == torch.float16 else 0)
    err = np.abs(got.double().cpu().numpy() - want)
    off = float((err / np.maximum(tol, 1e-300)).max()) if np.isfinite(err).all() else float("nan")
    assert off <= 1.0


CASES = [  # T, n, r, d_in, d_out, ids
    (1, 1, 1, 1, 1, "one"), (1, 4, 8, 64, 32, "mixed"), (2, 3, 5, 7, 9, "mixed"), (9, 32, 16, 256, 512, "mixed"), (16, 2, 4, 100, 129, "one"),
    (17, 2, 32, 130, 64, "one"), (33, 1, 64, 96, 200, "one"), (64, 9, 33, 128, 65, "mixed"), (65, 5, 16, 1000, 36, "mixed"),
    (64, 3, 17, 40, 1100, "none"), (80, 3, 2, 31, 33, "none"), (200, 70, 3, 65, 640, "mixed"), (333, 4, 64, 513, 257, "sorted"),
    (777, 16, 8, 1024, 96, "sorted"), (1500, 2, 12, 64, 128, "one"), (2500, 1, 48, 72, 520, "mixed"), (300, 1024, 1, 16, 24, "mixed")]


@pytest.mark.parametrize("kind,out", PAIRS)
@pytest.mark.parametrize("T,n,r,d_in,d_out,how", CASES)
def test_forward_and_backward(T, n, r, d_in, d_out, how, kind, out):
    rng = rng_of(T, n, r, d_in, d_out, how, kind, out)
    m = make(rng, T, n, r, d_in, d_out, TYPES[kind], TYPES[out])
    ids = ids_of(rng, T, n, how)
    want = reference(m, ids, n)
    # rows without an adapter and adapters without rows may hold anything
    off = (ids < 0) | (ids >= n)
    m["x"][torch.from_numpy(off)], m["dy"][torch.from_numpy(off)] = float("nan"), float("inf")
    unused = torch.tensor([a not in set(ids.tolist()) for a in range(n)])
    m["A"][unused], m["B"][unused], m["scale"][unused] = float("inf"), float("nan"), float("nan")
    g = {k: v.to(DEV) for k, v in m.items()}
    ids = torch.from_numpy(ids).to(DEV)
    ad = moeq.Adapters(g["A"], g["B"], g["scale"])
    y = moeq.moe_adapters_forward(ad, g["x"], ids, base=g["base"])
    check(y, *want["y"], d_in + r)
    dx, dA, dB = moeq.moe_adapters_backward(ad, g["x"], ids, g["dy"], dx_base=g["dx_base"])
    check(dx, *want["dx"], d_out + r)
    check(dA, *want["dA"], d_out + T)
    check(dB, *want["dB"], d_in + T)
    assert (dA[unused.to(DEV)] == 0).all() and (dB[unused.to(DEV)] == 0).all()
    # rows at another stride and alignment, in place of the base, without the gradient of x, twice: the same bits
    s = {k: strided(g[k], 5, 3) for k in ("x", "dy", "base", "dx_base")}
    y2 = moeq.moe_adapters_forward(ad, s["x"], ids, base=s["base"], y=s["base"])
    dx2, dA2, dB2 = moeq.moe_adapters_backward(ad, s["x"], ids, s["dy"], dx_base=s["dx_base"], dx=s["dx_base"])
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dA, dA2) and torch.equal(dB, dB2)
    none, dA2, dB2 = moeq.moe_adapters_backward(ad, g["x"], ids, g["dy"], want_dx=False)
    assert none is None and torch.equal(dA, dA2) and torch.equal(dB, dB2)


@pytest.mark.parametrize("kind,out", PAIRS)
def test_without_a_base_and_with_a_shared_one(kind, out):
    rng = rng_of("base", kind, out)
    T, n, r, d_in, d_out = 70, 4, 8, 72, 136
    m = make(rng, T, n, r, d_in, d_out, TYPES[kind], TYPES[out])
    ids = ids_of(rng, T, n, "mixed")
    m["dx_base"].zero_()
    m["base"][:] = m["base"][:1].clone()
    want = reference(m, ids, n)
    g = {k: v.to(DEV) for k, v in m.items()}
    ad, ids = moeq.Adapters(g["A"], g["B"], g["scale"]), torch.from_numpy(ids).to(DEV)
    check(moeq.moe_adapters_forward(ad, g["x"], ids, base=g["base"][:1].expand(T, d_out)), *want["y"], d_in + r)
    check(moeq.moe_adapters_backward(ad, g["x"], ids, g["dy"])[0], *want["dx"], d_out + r)
    y0 = moeq.moe_adapters_forward(ad, g["x"], ids, y=torch.empty((T, d_out), dtype=TYPES[out], device=DEV))
    b = m["base"].double().numpy()
    check(y0, want["y"][0] - b, want["y"][1] - np.abs(b), d_in + r)
    # all rows one row, of x and of dy: the gradients of a broadcast input
    x1, dy1 = g["x"][:1].expand(T, d_in), g["dy"][:1].expand(T, d_out)
    m2 = dict(m, x=m["x"][:1].expand(T, d_in), dy=m["dy"][:1].expand(T, d_out))
    want = reference(m2, ids.cpu().numpy(), n)
    dx, dA, dB = moeq.moe_adapters_backward(ad, x1, ids, dy1)
    check(dx, *want["dx"], d_out + r)
    check(dA, *want["dA"], d_out + T)
    check(dB, *want["dB"], d_in + T)


@pytest.mark.parametrize("kind", sorted(TYPES))
def test_a_row_that_is_not_finite_stays_alone(kind):
    rng = rng_of("nan", kind)
    T, n, r, d = 100, 3, 16, 256
    m = make(rng, T, n, r, d, d, TYPES[kind], TYPES[kind])
    g = {k: v.to(DEV) for k, v in m.items()}
    ids = torch.from_numpy(ids_of(rng, T, n, "mixed")).to(DEV)
    ids[5], ids[50] = 1, 1
    ad = moeq.Adapters(g["A"], g["B"], g["scale"])
    y = moeq.moe_adapters_forward(ad, g["x"], ids, base=g["base"])
    _, dA, dB = moeq.moe_adapters_backward(ad, g["x"], ids, g["dy"])
    g["x"][5, 7], g["x"][50, 200] = float("nan"), float("inf")
    y2 = moeq.moe_adapters_forward(ad, g["x"], ids, base=g["base"])
    rest = [t for t in range(T) if t not in (5, 50)]
    assert torch.equal(y[rest], y2[rest]) and not y2[[5, 50]].isfinite().any()
    _, dA2, dB2 = moeq.moe_adapters_backward(ad, g["x"], ids, g["dy"])
    others = [0, 2]
    assert torch.equal(dA[others], dA2[others]) and torch.equal(dB[others], dB2[others])
    assert not dB2[1].isfinite().any() and not dA2[1][:, [7, 200]].isfinite().any()


def test_no_rows():
    A, B, s = torch.randn((3, 4, 8), device=DEV), torch.randn((3, 16, 4), device=DEV), torch.ones(3, device=DEV)
    ad = moeq.Adapters(A, B, s)
    none = torch.empty((0,), dtype=torch.int32, device=DEV)
    assert moeq.moe_adapters_forward(ad, A.new_empty((0, 8)), none).shape == (0, 16)
    dx, dA, dB = moeq.moe_adapters_backward(ad, A.new_empty((0, 8)), none, A.new_empty((0, 16)))
    assert dx.shape == (0, 8) and (dA == 0).all() and (dB == 0).all() and dA.shape == A.shape and dB.shape == B.shape


def test_gradient_against_differences():
    """sum(y * c) is linear in x, in A and in B: differences along a direction have no error of their own but the roundings."""
    rng = rng_of("differences")
    T, n, r, d_in, d_out = 90, 4, 8, 64, 96
    new = lambda *s: torch.from_numpy(rng.normal(size=s).astype(np.float32)).to(DEV)
    A, B, scale, x, c = new(n, r, d_in), new(n, d_out, r), new(n), new(T, d_in), new(T, d_out)
    ids = torch.from_numpy(ids_of(rng, T, n, "mixed")).to(DEV)
    loss = lambda a, b, v: (moeq.moe_adapters_forward(moeq.Adapters(a, b, scale), v, ids).double() * c.double()).sum().item()
    dx, dA, dB = moeq.moe_adapters_backward(moeq.Adapters(A, B, scale), x, ids, c)
    vA, vB, vx = new(n, r, d_in), new(n, d_out, r), new(T, d_in)
    # elements of y are sums of 64 x 8 products of either sign, some 23 in size with the largest partial sums some 100: half a step
    # of those in each of T * d_out, added up as their square root, and the gradients' roundings against directions of size 1
    tol = 4 * 100 * 2.0**-23 * (T * d_out) ** 0.5 * 2
    for plus, minus, grad, v in ((loss(A + vA, B, x), loss(A - vA, B, x), dA, vA), (loss(A, B + vB, x), loss(A, B - vB, x), dB, vB),
                                 (loss(A, B, x + vx), loss(A, B, x - vx), dx, vx)):
        assert abs((plus - minus) / 2 - (grad.double() * v.double()).sum().item()) < tol


@pytest.mark.parametrize("T", (9, 700))
def test_replays_of_a_graph(T):
    rng = rng_of("graph", T)
    n, r, d_in, d_out = 5, 16, 256, 384
    m = make(rng, T, n, r, d_in, d_out, torch.bfloat16, torch.bfloat16)
    g = {k: v.to(DEV) for k, v in m.items()}
    ids = torch.from_numpy(ids_of(rng, T, n, "mixed")).to(DEV)
    ad = moeq.Adapters(g["A"], g["B"], g["scale"])
    ws = torch.empty(ad.workspace_bytes(T, True), dtype=torch.uint8, device=DEV)
    step = lambda w: [moeq.moe_adapters_forward(ad, g["x"], ids, base=g["base"], ws=w),
                      *moeq.moe_adapters_backward(ad, g["x"], ids, g["dy"], dx_base=g["dx_base"], ws=w)]
    step(ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(ws)
    other = torch.empty_like(ws)
    for k in range(4):
        g["x"].normal_()
        g["A"].normal_(std=0.1)
        ids.copy_(torch.from_numpy(ids_of(rng, T, n, ("mixed", "one", "none", "sorted")[k])).to(DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step(other)))


def test_another_stream_and_wide_offsets():
    """Rows far apart: the last begins more than 2^32 bytes behind the first."""
    T, n, r, d = 3, 2, 8, 64
    far = 300_000_000
    buf = torch.empty(far * 4 * (T - 1) // 2 + 2 * d, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (T, d), (far * 2, 1))
    A, B, s = (torch.randn(k, device=DEV).to(torch.bfloat16) for k in ((n, r, d), (n, d, r), (n,)))
    ad = moeq.Adapters(A, B, s.float())
    v = torch.randn((T, d), device=DEV).to(torch.bfloat16)
    ids = torch.tensor([0, 1, 0], dtype=torch.int32, device=DEV)
    want = moeq.moe_adapters_forward(ad, v, ids)
    gA, gB = moeq.moe_adapters_backward(ad, v, ids, want)[1:]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        x.copy_(v)
    got = moeq.moe_adapters_forward(ad, x, ids, stream=side)
    dx, dA, dB = moeq.moe_adapters_backward(ad, x, ids, got, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(dA, gA) and torch.equal(dB, gB)


def test_a_graph_keeps_the_workspace_that_it_was_captured_with():
    """The adapters' own workspace grows with a longer call: what a graph was captured with is not given away."""
    rng = rng_of("outgrown")
    n, r, d = 5, 16, 256
    m = make(rng, 200, n, r, d, d, torch.bfloat16, torch.bfloat16)
    g = {k: v.to(DEV) for k, v in m.items()}
    ids = torch.from_numpy(ids_of(rng, 200, n, "mixed")).to(DEV)
    ad = moeq.Adapters(g["A"], g["B"], g["scale"])
    step = lambda k: moeq.moe_adapters_forward(ad, g["x"][:k], ids[:k])
    want = step(200).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(200)
    size, place = ad._ws.numel(), ad._ws.data_ptr()
    long = torch.randn((5000, d), device=DEV).to(torch.bfloat16)
    moeq.moe_adapters_forward(ad, long, torch.zeros(5000, dtype=torch.int32, device=DEV))
    assert ad._ws.numel() >= 2 * size
    others = [torch.full((size,), 7, dtype=torch.uint8, device=DEV) for _ in range(4)]
    assert all(t.data_ptr() != place for t in others)
    for _ in range(3):
        held.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want) and torch.equal(step(200), want)
    assert all(bool((t == 7).all()) for t in others)


# rows that several workgroups plan, in tiles of every size, and the longest call
LONG = [(8192, 3, 16, 72, 64, "mixed"), (8193, 40, 20, 64, 72, "mixed"), (16384, 4, 33, 40, 64, "sorted"), (17003, 300, 8, 48, 40, "mixed"),
        (20000, 3, 64, 64, 24, "sorted"), (33000, 1, 17, 24, 40, "one"), (12289, 1024, 2, 16, 24, "mixed"), (65535, 7, 4, 16, 24, "mixed")]


@pytest.mark.parametrize("kind,out", PAIRS)
@pytest.mark.parametrize("T,n,r,d_in,d_out,how", LONG)
def test_long_calls(T, n, r, d_in, d_out, how, kind, out):
    rng = rng_of("long", T, n, r, d_in, d_out, how, kind, out)
    m = make(rng, T, n, r, d_in, d_out, TYPES[kind], TYPES[out])
    ids = ids_of(rng, T, n, how)
    want = reference(m, ids, n)
    g = {k: v.to(DEV) for k, v in m.items()}
    ids = torch.from_numpy(ids).to(DEV)
    ad = moeq.Adapters(g["A"], g["B"], g["scale"])
    y = moeq.moe_adapters_forward(ad, g["x"], ids, base=g["base"])
    check(y, *want["y"], d_in + r)
    dx, dA, dB = moeq.moe_adapters_backward(ad, g["x"], ids, g["dy"], dx_base=g["dx_base"])
    check(dx, *want["dx"], d_out + r)
    check(dA, *want["dA"], d_out + T)
    check(dB, *want["dB"], d_in + T)
    again = moeq.moe_adapters_backward(ad, g["x"], ids, g["dy"], dx_base=g["dx_base"])
    assert torch.equal(moeq.moe_adapters_forward(ad, g["x"], ids, base=g["base"]), y)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dA, dB)))


def mixed_calls(n_calls, seed):
    """Adapters, and calls of different rows and lengths on them, with what each gives when it runs alone."""
    rng = rng_of("calls", seed)
    n, r, d = 6, 16, 256
    m = make(rng, 2000, n, r, d, d, torch.bfloat16, torch.bfloat16)
    g = {k: v.to(DEV) for k, v in m.items()}
    ad = moeq.Adapters(g["A"], g["B"], g["scale"])
    calls = []
    for T in rng.integers(65, 2000, size=n_calls).tolist():
        ids = torch.from_numpy(ids_of(rng, T, n, "mixed")).to(DEV)
        x, dy = g["x"][:T], g["dy"][-T:]
        calls.append(lambda x=x, dy=dy, ids=ids, **kw: [moeq.moe_adapters_forward(ad, x, ids, **kw), *moeq.moe_adapters_backward(ad, x, ids, dy, **kw)])
    want = []
    for c in calls:
        want.append(c())
        torch.cuda.synchronize()
    return ad, calls, want


def test_calls_on_two_streams_have_workspaces_of_their_own():
    ad, calls, want = mixed_calls(16, "streams")
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    places = []
    for s in streams:
        calls[0](stream=s)
        places.append(ad._ws)                             # (held: the allocator cannot give the same place twice)
    assert places[0].data_ptr() != places[1].data_ptr() and all(t.device == ad.a.device for t in places)
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)                 # both queues fill up before either runs
    got = [c(stream=streams[i % 2]) for i, c in enumerate(calls)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_calls_of_two_threads_have_workspaces_of_their_own():
    """On the same stream: the launches of their calls may come between each other."""
    ad, calls, want = mixed_calls(12, "threads")
    got = {}

    def work(k):
        for turn in range(20):
            for i in range(k, len(calls), 2):
                got[turn, i] = calls[i]()

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    [t.start() for t in threads]
    [t.join(60) for t in threads]
    torch.cuda.synchronize()
    assert len(got) == 20 * len(calls)
    assert all(torch.equal(a, b) for (_, i), g in got.items() for a, b in zip(g, want[i]))


def test_a_workspace_is_not_given_away_while_its_stream_works():
    ad, calls, want = mixed_calls(2, "dropped")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = calls[1](stream=side)
    size = ad._ws.numel()
    ad._ws = None                                         # the last reference
    others = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[1])) and all(bool((t == 255).all()) for t in others)


def test_a_graph_and_calls_beside_it():
    """A graph has the workspace of its capture to itself: calls on another stream run beside its replays."""
    ad, calls, want = mixed_calls(8, "graph")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls[0]()
    side = torch.cuda.Stream()
    for i in range(1, 8):
        for h in held:
            h.zero_()
        torch.cuda.synchronize()
        graph.replay()
        got = calls[i](stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want[0])) and all(torch.equal(a, b) for a, b in zip(got, want[i]))


# columns that several workgroups share: in the backward pass two shares from 993 fp32 or 1985 16-bit columns of the narrower side, four
# from twice as many, eight from four times; in the forward pass, by d_in, eight from 4065 fp32 or 8129 16-bit columns
SHARED = [("f32", "f32", 70, 5, 992, 1500), ("f32", "f32", 70, 5, 993, 1500), ("f32", "f32", 300, 17, 1501, 994), ("f32", "f32", 130, 40, 2049, 1987),
          ("f32", "f32", 33, 16, 4001, 4099), ("bf16", "bf16", 70, 3, 1984, 2500), ("bf16", "bf16", 200, 33, 1985, 2500),
          ("bf16", "f32", 90, 16, 2505, 1986), ("bf16", "bf16", 1100, 32, 4096, 4097), ("bf16", "bf16", 40, 64, 8000, 7937), ("f16", "f16", 70, 8, 2047, 1984),
          ("f16", "f16", 70, 20, 2047, 1985), ("f16", "f32", 160, 50, 1985, 4096), ("f16", "f16", 520, 1, 4096, 4096), ("bf16", "bf16", 9, 16, 8128, 64),
          ("bf16", "bf16", 9, 16, 8129, 64), ("bf16", "f32", 66, 48, 8129, 72), ("f16", "f16", 64, 7, 8200, 40), ("f32", "f32", 64, 20, 4064, 64),
          ("f32", "f32", 64, 20, 4065, 64), ("f32", "f32", 150, 64, 4070, 33), ("bf16", "bf16", 5, 9, 32768, 64), ("bf16", "bf16", 70, 9, 64, 32768), ("f32", "f32", 40, 33, 4064, 4500), ("f32", "f32", 40, 33, 4500, 4065),
          ("bf16", "bf16", 100, 64, 8129, 8150), ("bf16", "f32", 35, 8, 8200, 8129), ("f16", "f16", 80, 24, 8128, 8300), ("f16", "f32", 80, 24, 8300, 8129)]


@pytest.mark.parametrize("kind,out,T,r,d_in,d_out", SHARED)
def test_columns_shared_among_workgroups(kind, out, T, r, d_in, d_out):
    n = 3
    rng = rng_of("shared", kind, out, T, r, d_in, d_out)
    m = make(rng, T, n, r, d_in, d_out, TYPES[kind], TYPES[out])
    ids = ids_of(rng, T, n, "mixed")
    want = reference(m, ids, n)
    g = {k: v.to(DEV) for k, v in m.items()}
    ids = torch.from_numpy(ids).to(DEV)
    ad = moeq.Adapters(g["A"], g["B"], g["scale"])
    y = moeq.moe_adapters_forward(ad, g["x"], ids, base=g["base"])
    check(y, *want["y"], d_in + r)
    dx, dA, dB = moeq.moe_adapters_backward(ad, g["x"], ids, g["dy"], dx_base=g["dx_base"])
    check(dx, *want["dx"], d_out + r)
    check(dA, *want["dA"], d_out + T)
    check(dB, *want["dB"], d_in + T)
    s = {k: strided(g[k], 3, 1) for k in ("x", "dy", "base", "dx_base")}
    y2 = moeq.moe_adapters_forward(ad, s["x"], ids, base=s["base"], y=s["base"])
    again = moeq.moe_adapters_backward(ad, s["x"], ids, s["dy"], dx_base=s["dx_base"], dx=s["dx_base"])
    assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(again, (dx, dA, dB)))


def test_replays_of_a_graph_with_shared_columns():
    """The gradient whose pieces come from shares joined in the workspace."""
    rng = rng_of("graph of shares")
    T, n, r, d = 200, 3, 24, 4096
    m = make(rng, T, n, r, d, d, torch.bfloat16, torch.bfloat16)
    g = {k: v.to(DEV) for k, v in m.items()}
    ids = torch.from_numpy(ids_of(rng, T, n, "mixed")).to(DEV)
    ad = moeq.Adapters(g["A"], g["B"], g["scale"])
    step = lambda: [moeq.moe_adapters_forward(ad, g["x"], ids, base=g["base"]), *moeq.moe_adapters_backward(ad, g["x"], ids, g["dy"], dx_base=g["dx_base"])]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for how in ("mixed", "one", "none", "sorted"):
        g["x"].normal_()
        g["dy"].normal_()
        ids.copy_(torch.from_numpy(ids_of(rng, T, n, how)).to(DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))
