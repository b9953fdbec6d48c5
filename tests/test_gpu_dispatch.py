"""Pairs sorted by expert, rows in that order and back, and the gradient, against plain arithmetic in 64 bits on the host: one token
to several chunks of pairs, widths that end inside a vector, strided and shared rows, dropped pairs, entries out of range."""
import numpy as np
import pytest
import torch

import paper_2308_14352_amd as moeq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def rng_of(*parts):
    return np.random.default_rng([ord(c) for c in repr(parts)])


def routing(rng, T, k, E, drop):
    """Distinct experts of uneven popularity where there are enough; a share out of range, below and above."""
    score = rng.normal(size=(T, E)) + rng.normal(size=E)
    idx = np.argsort(-score, axis=1)[:, :k] if k <= E else rng.integers(0, E, size=(T, k))
    idx = idx.astype(np.int32)
    out = rng.random((T, k)) < drop
    idx[out] = rng.choice(np.array([-1, E, -2**31, 2**31 - 1, E + 7], dtype=np.int64), size=int(out.sum())).astype(np.int32)
    return idx


def sorted_on_host(idx, E):
    e = idx.reshape(-1).astype(np.int64)
    key = np.where((e < 0) | (e >= E), E, e)
    order = np.argsort(key, kind="stable")
    offsets = np.zeros(E + 1, np.int64)
    offsets[1:] = np.cumsum(np.bincount(key, minlength=E + 1)[:E])
    place = np.empty_like(order)
    place[order] = np.arange(order.size)
    return offsets, np.where(key[order] == E, ~order, order), np.where(key == E, ~place, place)


@pytest.mark.parametrize("T,k,E,drop", [
    (1, 1, 1, 0.0), (1, 1, 1, 1.0), (8, 1, 64, 0.0), (3, 2, 33, 0.3), (64, 1, 7, 0.0), (65, 1, 64, 0.1), (500, 4, 512, 0.05),
    (700, 3, 513, 0.2), (1117, 2, 128, 0.03), (1000, 1, 1024, 0.0), (16384, 1, 256, 0.05), (16385, 1, 8, 0.05), (9000, 8, 1024, 0.1),
    (20001, 2, 3, 1.0), (33000, 4, 16, 0.0)])
def test_sort(T, k, E, drop):
    rng = rng_of("sort", T, k, E, drop)
    idx = routing(rng, T, k, E, drop)
    s = moeq.moe_sort_pairs(torch.from_numpy(idx).to(DEV), E)
    for got, want in zip((s.offsets, s.order, s.slot), sorted_on_host(idx, E)):
        assert got.dtype == torch.int32 and np.array_equal(got.cpu().numpy(), want)


def test_sort_of_nothing():
    s = moeq.moe_sort_pairs(torch.empty((0, 2), dtype=torch.int32, device=DEV), 5)
    assert s.offsets.tolist() == [0] * 6 and s.order.numel() == 0 and s.slot.numel() == 0


def test_sort_into_one_expert_and_ties_keep_the_order():
    idx = torch.full((5000, 1), 3, dtype=torch.int32, device=DEV)
    s = moeq.moe_sort_pairs(idx, 9)
    assert torch.equal(s.order, torch.arange(5000, dtype=torch.int32, device=DEV))
    assert s.offsets.tolist() == [0, 0, 0, 0] + [5000] * 6


def strided(t, pad, shift):
    """The same values in rows `pad` elements apart, beginning `shift` elements into their memory."""
    buf = torch.full((t.shape[0] * (t.shape[1] + pad) + shift,), float("nan"), dtype=t.dtype, device=t.device)
    v = buf[shift:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
    v.copy_(t)
    return v


CASES = [(1, 1, 1, 1, 0.0), (2, 1, 4, 7, 0.5), (8, 1, 64, 768, 0.0), (5, 2, 3, 64, 0.0), (9, 3, 16, 65, 0.2), (4, 8, 33, 100, 0.1),
         (130, 2, 8, 127, 0.0), (33, 4, 16, 1000, 0.3), (17, 1, 8, 1025, 0.0), (65, 2, 128, 2049, 0.05), (3, 2, 8, 4096, 1.0),
         (700, 2, 8, 33, 0.03)]


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("T,k,E,d,drop", CASES)
def test_rows_there_and_back(T, k, E, d, drop, kind):
    rng = rng_of("rows", T, k, E, d, kind)
    idx = routing(rng, T, k, E, drop)
    offsets, order, slot = sorted_on_host(idx, E)
    kept, at = slot.reshape(T, k) >= 0, np.where(slot < 0, ~slot, slot).reshape(T, k)
    sort = moeq.moe_sort_pairs(torch.from_numpy(idx).to(DEV), E)
    t = TYPES[kind]
    x = torch.from_numpy(rng.normal(size=(T, d))).to(t)
    rows = torch.from_numpy(rng.normal(size=(T * k, d))).to(t)
    gate = torch.from_numpy(rng.normal(size=(T, k)).astype(np.float32))
    # the rows and gates of dropped pairs may hold anything
    for i, j in zip(*np.nonzero(~kept)):
        rows[at[i, j]] = float("nan")
        gate[i, j] = float("inf")
    r64, g64 = np.nan_to_num(rows.double().numpy()), np.where(kept, gate.double().numpy(), 0.0)
    half = torch.finfo(t).eps / 2
    for pad, shift in ((0, 0), (3, 1)):
        put = lambda v: strided(v.to(DEV), pad, shift) if pad else v.to(DEV)
        # gather: copies
        want = x.numpy(force=True) if t != torch.bfloat16 else x.float().numpy()
        got = moeq.moe_gather_rows(sort, put(x), rows=None if not pad else strided(torch.zeros((T * k, d), dtype=t, device=DEV), pad, shift))
        full = np.zeros((T * k, d))
        full[at[kept]] = np.repeat(want, k, axis=0).reshape(T, k, d)[kept]
        assert np.array_equal(got.double().cpu().numpy(), full)
        for g in (gate, None):
            w = g64 if g is not None else kept.astype(np.float64)
            terms = w[:, :, None] * r64[at]
            y64, mag = terms.sum(1), np.abs(terms).sum(1)
            for yt in {t, torch.float32}:
                y = moeq.moe_combine_rows(sort, put(rows), None if g is None else g.to(DEV), dtype=yt)
                assert y.dtype == yt
                # k roundings of fp32 sums, each at most half a step of the largest partial sum, and that of the output
                tol = (k + 1) * 2.0**-24 * mag * 1.001 + torch.finfo(yt).eps / 2 * np.abs(y64) * 1.001 + (2.0**-25 if yt == torch.float16 else 0)
                assert (np.abs(y.double().cpu().numpy() - y64) <= tol).all()
                dy = torch.from_numpy(rng.normal(size=(T, d))).to(yt)
                drows, dgate = moeq.moe_combine_rows_backward(sort, put(dy), put(rows), None if g is None else g.to(DEV))
                dy64 = dy.double().numpy()
                want = np.zeros((T * k, d))
                want[at] = w[:, :, None] * dy64[:, None, :]
                assert drows.dtype == t
                tol = (2.0**-24 + half) * np.abs(want) * 1.001 + (2.0**-25 if t == torch.float16 else 0)
                assert (np.abs(drows.double().cpu().numpy() - want) <= tol).all()
                dots = dy64[:, None, :] * r64[at]
                # chains of at most d / 16 products in a thread and 8 joins
                tol = (d / 16 + 16) * 2.0**-24 * np.abs(dots).sum(-1) * 1.001
                want = np.where(kept, dots.sum(-1), 0.0)
                assert (np.abs(dgate.double().cpu().numpy() - want) <= tol).all()
                assert (dgate.cpu().numpy()[~kept] == 0).all()


def test_gradient_against_differences():
    """The loss sum(y * c) is linear in the rows and in the gates: differences along any direction have no error of their own."""
    rng = rng_of("differences")
    T, k, E, d = 40, 2, 8, 96
    sort = moeq.moe_sort_pairs(torch.from_numpy(routing(rng, T, k, E, 0.1)).to(DEV), E)
    new = lambda *s: torch.from_numpy(rng.normal(size=s).astype(np.float32)).to(DEV)
    rows, gate, c, v, u = new(T * k, d), new(T, k), new(T, d), new(T * k, d), new(T, k)
    loss = lambda r, g: (moeq.moe_combine_rows(sort, r, g).double() * c.double()).sum().item()
    drows, dgate = moeq.moe_combine_rows_backward(sort, c, rows, gate)
    size = T * d * k
    # fp32 results of a few units, 7680 of them summed with factors of either sign: the roundings add up as their square root
    tol = 40 * 2.0**-24 * size**0.5
    assert abs((loss(rows + v, gate) - loss(rows - v, gate)) / 2 - (drows.double() * v.double()).sum().item()) < tol
    assert abs((loss(rows, gate + u) - loss(rows, gate - u)) / 2 - (dgate.double() * u.double()).sum().item()) < tol
    # gather and the combine without gates are each other's transposes
    x = new(T, d)
    there = (moeq.moe_gather_rows(sort, x).double() * v.double()).sum().item()
    back = (moeq.moe_combine_rows(sort, v).double() * x.double()).sum().item()
    assert abs(there - back) < tol


def test_shared_rows_and_slots_out_of_range():
    T, k, d = 6, 2, 40
    sort = moeq.moe_sort_pairs(torch.zeros((T, k), dtype=torch.int32, device=DEV), 4)
    one = torch.randn((1, d), device=DEV)
    assert torch.equal(moeq.moe_gather_rows(sort, one.expand(T, d)), one.expand(T * k, d))
    # places that point nowhere are left alone, and add nothing
    sort.slot[3], sort.slot[4] = 1 << 30, -(1 << 30)
    rows = torch.full((T * k, d), 7.0, device=DEV)
    moeq.moe_gather_rows(sort, torch.ones((T, d), device=DEV), rows=rows)
    assert rows[3].eq(7).all() and rows[4].eq(7).all() and rows[5].eq(1).all()
    y = moeq.moe_combine_rows(sort, torch.ones((T * k, d), device=DEV))
    assert y[:, 0].tolist() == [2, 1, 1, 2, 2, 2]
    _, dgate = moeq.moe_combine_rows_backward(sort, torch.ones((T, d), device=DEV), torch.ones((T * k, d), device=DEV))
    assert dgate.flatten().tolist() == [d, d, d, 0, 0] + [d] * 7


def test_replays_of_a_graph_and_another_stream():
    rng = rng_of("graph")
    T, k, E, d = 3000, 6, 64, 128
    idx = torch.from_numpy(routing(rng, T, k, E, 0.1)).to(DEV)
    x, gate = torch.randn((T, d), device=DEV), torch.rand((T, k), device=DEV)

    def step():
        s = moeq.moe_sort_pairs(idx, E)
        rows = moeq.moe_gather_rows(s, x)
        y = moeq.moe_combine_rows(s, rows, gate)
        return [s.offsets, s.order, s.slot, rows, y, *moeq.moe_combine_rows_backward(s, y, rows, gate)]

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = step()
    for n in range(4):
        new = torch.from_numpy(routing(rng, T, k, E, 0.1 * n)).to(DEV)
        idx.copy_(new)
        x.normal_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))
    side = torch.cuda.Stream()
    want = step()
    late = torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late.copy_(x)
    s = moeq.moe_sort_pairs(idx, E, stream=side)
    rows = moeq.moe_gather_rows(s, late, stream=side)
    y = moeq.moe_combine_rows(s, rows, gate, stream=side)
    got = [s.offsets, s.order, s.slot, rows, y, *moeq.moe_combine_rows_backward(s, y, rows, gate, stream=side)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("T,k,E", [(6144, 1, 8), (6145, 1, 8), (4096, 1, 1024), (4097, 2, 300), (2048, 3, 64), (2049, 3, 64), (4096, 4, 128)])
def test_sort_around_the_chunks(T, k, E):
    rng = rng_of("chunks", T, k, E)
    idx = routing(rng, T, k, E, 0.02)
    s = moeq.moe_sort_pairs(torch.from_numpy(idx).to(DEV), E)
    for got, want in zip((s.offsets, s.order, s.slot), sorted_on_host(idx, E)):
        assert np.array_equal(got.cpu().numpy(), want)


def order_backwards(T):
    """A sort of one choice a token whose places run backwards, without the sort itself."""
    slot = torch.arange(T - 1, -1, -1, dtype=torch.int32, device=DEV)
    return moeq.PairSort(torch.tensor([0, T], dtype=torch.int32, device=DEV), slot, slot, T, 1, 1)


def test_as_many_pairs_as_there_may_be():
    """2^28 rows of one element: 2^32 threads, more than a launch may have."""
    T = 1 << 28
    sort = order_backwards(T)
    x = torch.randn(T, device=DEV).to(torch.float16)[:, None]
    rows = moeq.moe_gather_rows(sort, x)
    assert torch.equal(rows, x.flip(0))
    assert torch.equal(moeq.moe_combine_rows(sort, rows), x)
    drows, dgate = moeq.moe_combine_rows_backward(sort, x, rows)
    assert torch.equal(drows, rows) and torch.equal(dgate, x.float() ** 2)
    torch.cuda.empty_cache()


def test_as_many_wide_rows_as_pass_a_launch():
    """2^24 rows of a workgroup each: outputs of 34 GB from inputs whose rows are all one."""
    T, d = 1 << 24, 1025
    sort = order_backwards(T)
    one = torch.randn((1, d), device=DEV).to(torch.bfloat16)
    buf = torch.zeros((T, d), dtype=torch.bfloat16, device=DEV)
    same = lambda: all(bool((part == one).all()) for part in buf.split(1 << 21))
    moeq.moe_gather_rows(sort, one.expand(T, d), rows=buf)
    assert same()
    buf.zero_()
    moeq.moe_combine_rows(sort, one.expand(T, d), y=buf)
    assert same()
    buf.zero_()
    _, dgate = moeq.moe_combine_rows_backward(sort, one.expand(T, d), one.expand(T, d), drows=buf)
    assert same() and bool((dgate == dgate[0]).all())
    # 1025 squares of positive sum: a chain of at most 1025 / 256 + 16 roundings
    assert abs(dgate[0].item() / (one.double() ** 2).sum().item() - 1) < (1025 / 256 + 16) * 2.0**-24
    del buf
    torch.cuda.empty_cache()


# chunks of 4096 pairs on both sides of where their counts are scanned ahead, and as many as make adding them up in every chunk too long
@pytest.mark.parametrize("P,E,drop", [(96 * 4096, 8, 0.02), (96 * 4096 + 1, 8, 0.02), (19 * 4096, 256, 0.0), (19 * 4096 + 5, 256, 0.1),
                                      (4 * 4096, 1024, 0.02), (4 * 4096 + 1, 1024, 0.02), (1000001, 63, 0.3), (5000003, 1024, 0.0)])
def test_sort_of_many_chunks(P, E, drop):
    rng = rng_of("many", P, E, drop)
    idx = rng.integers(0, E, size=(P, 1)).astype(np.int32)
    idx[rng.random((P, 1)) < drop] = -1
    s = moeq.moe_sort_pairs(torch.from_numpy(idx).to(DEV), E)
    for got, want in zip((s.offsets, s.order, s.slot), sorted_on_host(idx, E)):
        assert np.array_equal(got.cpu().numpy(), want)


def test_sort_takes_time_in_proportion_to_its_pairs():
    """16 times the pairs, 4.2 million to 67 million of 256 experts: some 16 times the time, where counts that every chunk adds up for
    itself would take 256 times."""
    def least(P):
        idx = torch.randint(0, 256, (P, 1), dtype=torch.int32, device=DEV)
        times = []
        for _ in range(4):
            a, b = torch.cuda.Event(True), torch.cuda.Event(True)
            a.record()
            moeq.moe_sort_pairs(idx, 256)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    assert least(1 << 26) < 64 * least(1 << 22)


def test_sort_of_as_many_pairs_as_there_may_be():
    P, E = 1 << 28, 5
    idx = torch.randint(-1, E, (P // 2, 2), dtype=torch.int32, device=DEV)
    s = moeq.moe_sort_pairs(idx, E)
    key = torch.where(idx < 0, E, idx).flatten().to(torch.int8)
    counts = [int((key == e).sum()) for e in range(E)]
    assert s.offsets.tolist() == [sum(counts[:e]) for e in range(E + 1)]
    order = torch.where(s.order < 0, ~s.order, s.order)
    got = key[order.long()]
    assert bool((got[1:] >= got[:-1]).all()) and bool(((got == E) == (s.order < 0)).all())
    assert bool(((order[1:] > order[:-1]) | (got[1:] > got[:-1])).all())           # stable, and so every pair once
    place = torch.where(s.slot < 0, ~s.slot, s.slot)
    assert bool((place[order.long()] == torch.arange(P, dtype=torch.int32, device=DEV)).all()) and bool(((s.slot < 0) == (key == E)).all())
    del order, got, place, key
    torch.cuda.empty_cache()


def test_a_single_row_may_have_any_stride():
    """The stride of a single row says nothing: torch gives it what the row was cut out of."""
    x = torch.randn((1, 40), device=DEV)
    far, sort = torch.as_strided(x, (1, 40), (1 << 40, 1)), moeq.moe_sort_pairs(torch.zeros((1, 1), dtype=torch.int32, device=DEV), 3)
    assert torch.equal(moeq.moe_gather_rows(sort, far), x)
    assert torch.equal(moeq.moe_combine_rows(sort, far, y=torch.as_strided(torch.empty_like(x), (1, 40), (1 << 40, 1))), x)
    ids, top = torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.zeros((1, 1), device=DEV)
    for a, b in zip(moeq.moe_distill_loss_grad(far, ids, top), moeq.moe_distill_loss_grad(x, ids, top)):
        assert torch.equal(a, b)
    ad = moeq.Adapters(torch.randn((1, 4, 40), device=DEV), torch.randn((1, 24, 4), device=DEV), torch.ones(1, device=DEV))
    assert torch.equal(moeq.moe_adapters_forward(ad, far, ids[0]), moeq.moe_adapters_forward(ad, x, ids[0]))


@pytest.mark.parametrize("kind,dy_kind", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("T,k,d", [(1, 1, 3), (37, 2, 100), (65, 3, 1025), (9, 8, 4096), (5, 5, 16)])
def test_gradient_of_the_rows_alone(T, k, d, kind, dy_kind):
    """The C call without dgate, whose rows are not read: the same gradient of the rows."""
    rng = rng_of("alone", T, k, d, kind)
    sort = moeq.moe_sort_pairs(torch.from_numpy(routing(rng, T, k, 8, 0.2)).to(DEV), 8)
    dy, gate = torch.randn((T, d), device=DEV).to(TYPES[dy_kind]), torch.rand((T, k), device=DEV)
    rows = torch.randn((T * k, d), device=DEV).to(TYPES[kind])
    B = moeq.binding
    for g in (gate, None):
        want, _ = moeq.moe_combine_rows_backward(sort, dy, rows, g)
        got = torch.full_like(rows, float("nan"))
        assert B.lib().moe_combine_rows_backward(sort.slot.data_ptr(), None if g is None else g.data_ptr(), T, k, d, B._DTYPES[TYPES[kind]], None, 0,
                                                 B._DTYPES[TYPES[dy_kind]], dy.data_ptr(), d, got.data_ptr(), d, None, B._stream(None)) == B.MOEQ_OK
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_replays_of_a_graph_with_scanned_counts():
    rng = rng_of("graph of chunks")
    P, E = 20 * 4096, 300
    idx = torch.empty((P, 1), dtype=torch.int32, device=DEV)
    fill = lambda n: idx.copy_(torch.from_numpy(np.sort(rng.integers(-1, E - 40 * n, size=(P, 1)), axis=0 if n == 2 else 1).astype(np.int32)))
    step = lambda: (lambda s: [s.offsets, s.order, s.slot])(moeq.moe_sort_pairs(idx, E))
    fill(0)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = step()
    for n in range(4):
        fill(n)
        g.replay()
        torch.cuda.synchronize()
        want = sorted_on_host(idx.cpu().numpy(), E)
        assert all(np.array_equal(a.cpu().numpy(), w) for a, w in zip(held, want))
        assert all(torch.equal(a, b) for a, b in zip(held, step()))
