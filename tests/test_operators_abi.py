"""CPU-only checks of the operators beside the layer: sizes of workspaces, and refusals before any device call."""
import ctypes as C

import pytest
import torch

import paper_2308_14352_amd as moeq
from paper_2308_14352_amd import binding as B

P, Q, R = 1 << 20, 1 << 30, 1 << 40          # addresses far apart; nothing is read in a refused call
INVALID, UNSUPPORTED, WORKSPACE = B.MOEQ_EINVAL, B.MOEQ_EUNSUPPORTED, B.MOEQ_EWORKSPACE
F32, BF16, F16 = B.MOEQ_F32, B.MOEQ_BF16, B.MOEQ_F16


def call(name, good, **bad):
    args = dict(good, **bad)
    assert set(args) == set(good)
    return getattr(B.lib(), name)(*args.values())


SORT = dict(idx=P, T=20000, k=1, E=8, offsets=Q, order=Q + 4096, slot=R, ws=None, ws_bytes=0, stream=None)
GATHER = dict(slot=P, T=4, k=2, d=8, dtype=F32, x=Q, x_stride=8, rows=R, rows_stride=8, stream=None)
COMBINE = dict(slot=P, gate=None, T=4, k=2, d=8, dtype=BF16, rows=Q, rows_stride=8, y_dtype=F32, y=R, y_stride=8, stream=None)
COMBINE_GRAD = dict(slot=P, gate=None, T=4, k=2, d=8, dtype=BF16, rows=Q, rows_stride=8, dy_dtype=F32, dy=Q + 4096, dy_stride=8,
                    drows=R, drows_stride=8, dgate=None, stream=None)
DISTILL = dict(logits=Q, stride=100, dtype=F32, T=4, V=100, idx=P, top=P, K=3, tau=1.0, weight=None, loss=R, lse=None, ws=None,
               ws_bytes=0, stream=None)
DISTILL_GRAD = dict(logits=Q, stride=100, dtype=F32, T=4, V=100, idx=P, top=P, K=3, tau=1.0, weight=None, lse=P, dloss=P, dlogits=R,
                    dstride=100, stream=None)


@pytest.mark.parametrize("name,good,bad,status", [
    ("moe_sort_pairs", SORT, dict(E=0), INVALID), ("moe_sort_pairs", SORT, dict(k=0), INVALID),
    ("moe_sort_pairs", SORT, dict(T=-1), INVALID), ("moe_sort_pairs", SORT, dict(idx=None), INVALID),
    ("moe_sort_pairs", SORT, dict(offsets=None), INVALID), ("moe_sort_pairs", SORT, dict(slot=R + 2), INVALID),
    ("moe_sort_pairs", SORT, dict(E=1025), UNSUPPORTED), ("moe_sort_pairs", SORT, dict(T=1 << 28, k=2), UNSUPPORTED),
    ("moe_sort_pairs", SORT, dict(), WORKSPACE), ("moe_sort_pairs", SORT, dict(ws=R + 2, ws_bytes=1 << 20), INVALID),
    ("moe_gather_rows", GATHER, dict(dtype=3), INVALID), ("moe_gather_rows", GATHER, dict(x_stride=7), INVALID),
    ("moe_gather_rows", GATHER, dict(rows_stride=0), INVALID), ("moe_gather_rows", GATHER, dict(x=Q + 2), INVALID),
    ("moe_gather_rows", GATHER, dict(d=0), INVALID), ("moe_gather_rows", GATHER, dict(rows=Q + 16), INVALID),
    ("moe_gather_rows", GATHER, dict(x=None), INVALID), ("moe_gather_rows", GATHER, dict(slot=None), INVALID),
    ("moe_gather_rows", GATHER, dict(T=1 << 28), UNSUPPORTED),
    ("moe_combine_rows", COMBINE, dict(y_dtype=F16), INVALID), ("moe_combine_rows", COMBINE, dict(y=Q + 64), INVALID),
    ("moe_combine_rows", COMBINE, dict(gate=P + 1), INVALID), ("moe_combine_rows", COMBINE, dict(rows=Q + 1), INVALID),
    ("moe_combine_rows", COMBINE, dict(y_stride=4), INVALID), ("moe_combine_rows", COMBINE, dict(y=None), INVALID),
    ("moe_combine_rows_backward", COMBINE_GRAD, dict(dy_dtype=F16), INVALID),
    ("moe_combine_rows_backward", COMBINE_GRAD, dict(drows=Q + 4096), INVALID),
    ("moe_combine_rows_backward", COMBINE_GRAD, dict(rows=None, dgate=P), INVALID),
    ("moe_combine_rows_backward", COMBINE_GRAD, dict(dy=None), INVALID),
    ("moe_distill_forward", DISTILL, dict(tau=0.0), INVALID), ("moe_distill_forward", DISTILL, dict(tau=float("nan")), INVALID),
    ("moe_distill_forward", DISTILL, dict(tau=float("inf")), INVALID), ("moe_distill_forward", DISTILL, dict(tau=-1.0), INVALID),
    ("moe_distill_forward", DISTILL, dict(K=0), INVALID), ("moe_distill_forward", DISTILL, dict(V=0), INVALID),
    ("moe_distill_forward", DISTILL, dict(K=1025), UNSUPPORTED), ("moe_distill_forward", DISTILL, dict(stride=99), INVALID),
    ("moe_distill_forward", DISTILL, dict(top=None), INVALID), ("moe_distill_forward", DISTILL, dict(idx=P + 2), INVALID),
    ("moe_distill_forward", DISTILL, dict(T=1 << 25), UNSUPPORTED), ("moe_distill_forward", DISTILL, dict(dtype=7), INVALID),
    ("moe_distill_backward", DISTILL_GRAD, dict(dlogits=Q), INVALID), ("moe_distill_backward", DISTILL_GRAD, dict(lse=None), INVALID),
    ("moe_distill_backward", DISTILL_GRAD, dict(dloss=None), INVALID), ("moe_distill_backward", DISTILL_GRAD, dict(dstride=0), INVALID),
])
def test_refusals(name, good, bad, status):
    assert call(name, good, **bad) == status


def desc(**kw):
    d = dict(n_adapters=3, rank=8, d_in=64, d_out=32, dtype=BF16, a=P, b=P, scale=P)
    d.update(kw)
    return B.moeq_adapters(**d)


@pytest.mark.parametrize("kw,bad,status", [
    (dict(n_adapters=0), {}, INVALID), (dict(rank=0), {}, INVALID), (dict(d_in=0), {}, INVALID), (dict(dtype=5), {}, INVALID),
    (dict(a=None), {}, INVALID), (dict(b=P + 1), {}, INVALID), (dict(scale=None), {}, INVALID),
    (dict(rank=65), {}, UNSUPPORTED), (dict(n_adapters=1025), {}, UNSUPPORTED), (dict(d_out=32769), {}, UNSUPPORTED),
    ({}, dict(T=-1), INVALID), ({}, dict(T=65536), UNSUPPORTED), ({}, dict(dtype=F16), INVALID), ({}, dict(ids=None), INVALID),
    ({}, dict(x=None), INVALID), ({}, dict(x_stride=63), INVALID), ({}, dict(out=Q), INVALID), ({}, dict(out_stride=0), INVALID),
    ({}, dict(base=R + 8, base_stride=32), INVALID), ({}, dict(ws=None), WORKSPACE), ({}, dict(ws_bytes=8), WORKSPACE),
    ({}, dict(ws=P + 8), INVALID),
])
def test_refusals_of_adapters(kw, bad, status):
    d = desc(**kw)
    a = dict(x=Q, x_stride=64, ids=P, T=5, base=None, base_stride=0, dtype=F32, out=R, out_stride=32, ws=P, ws_bytes=1 << 24)
    a.update(bad)
    L = B.lib()
    assert L.moe_adapters_forward(C.addressof(d), a["x"], a["x_stride"], a["ids"], a["T"], a["base"], a["base_stride"], a["dtype"],
                                  a["out"], a["out_stride"], a["ws"], a["ws_bytes"], None) == status
    # in the backward pass the outputs are dx [T][d_in]
    wide = {32: 64, 0: 0}
    assert L.moe_adapters_backward(C.addressof(d), a["x"], a["x_stride"], a["ids"], a["T"], a["dtype"], Q + 65536, 32, a["base"],
                                   wide[a["base_stride"]], a["out"], wide[a["out_stride"]], R + 65536, R + (1 << 20), a["ws"],
                                   a["ws_bytes"], None) == status


def test_refusals_of_null_handles_and_gradients():
    L, d = B.lib(), desc()
    assert L.moe_adapters_forward(None, Q, 64, P, 5, None, 0, F32, R, 32, P, 1 << 24, None) == INVALID
    assert L.moe_adapters_backward(C.addressof(d), Q, 64, P, 5, F32, Q + 65536, 32, None, 0, None, 0, None, R, P, 1 << 24, None) == INVALID
    assert L.moe_adapters_backward(C.addressof(d), Q, 64, P, 5, F32, R, 32, None, 0, R + 64, 64, R, R, P, 1 << 24, None) == INVALID
    assert L.moe_adapters_workspace_bytes(None, 5, 0) == 0 and L.moe_adapters_workspace_bytes(C.addressof(desc(rank=65)), 5, 0) == 0
    sizes = [L.moe_adapters_workspace_bytes(C.addressof(d), T, b) for b in (0, 1) for T in (1, 16, 17, 64, 65, 1000, 65535)]
    assert sizes[:7] == sorted(sizes[:7]) and sizes[7:] == sorted(sizes[7:]) and all(a <= b for a, b in zip(sizes, sizes[7:]))


def test_calls_without_tokens_are_no_ops_without_pointers():
    L, d = B.lib(), desc()
    assert L.moe_gather_rows(None, 0, 2, 8, F32, None, 8, None, 8, None) == B.MOEQ_OK
    assert L.moe_combine_rows(None, None, 0, 2, 8, F32, None, 8, F32, None, 8, None) == B.MOEQ_OK
    assert L.moe_adapters_forward(C.addressof(d), None, 64, None, 0, None, 0, F32, None, 32, None, 0, None) == B.MOEQ_OK
    assert L.moe_distill_forward(None, 100, F32, 0, 100, None, None, 3, 1.0, None, None, None, None, 0, None) == B.MOEQ_OK


def test_sort_workspace_of_small_calls_is_empty():
    L = B.lib()
    assert L.moe_sort_bytes(8, 1, 64) == 0 and L.moe_sort_bytes(65535, 8, 256) > 0 and L.moe_sort_bytes(65535, 8, 1025) == 0
    assert L.moe_distill_workspace_bytes(0, 100, F32) == 0 and L.moe_distill_workspace_bytes(4, 100, 9) == 0


def test_binding_refuses_tensors_that_are_not_on_the_device_or_of_another_form():
    x = torch.zeros((4, 8))
    for call_ in (lambda: moeq.moe_sort_pairs(torch.zeros((4, 2), dtype=torch.int32), 8),
                  lambda: moeq.moe_distill_forward(x, torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2))),
                  lambda: moeq.Adapters(torch.zeros((2, 4, 8)), torch.zeros((2, 8, 4)), torch.zeros(2)),
                  lambda: moeq.Adapters(torch.zeros((2, 4, 8)), torch.zeros((2, 8, 5)), torch.zeros(2))):
        with pytest.raises(moeq.MoeqError) as e:
            call_()
        assert e.value.status == INVALID


def test_binding_takes_the_stream_of_the_current_device_only(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device)
    assert B._stream_on(1) == 101
    with pytest.raises(moeq.MoeqError) as e:
        B._stream_on(0)
    assert e.value.status == INVALID


# outputs that are no matrices: each over an input, or over another output, by its last element
GOOD_SORT, GOOD_GRAD = dict(SORT, T=4), dict(COMBINE_GRAD, dgate=P + (1 << 19))


@pytest.mark.parametrize("name,good,bad", [
    ("moe_sort_pairs", GOOD_SORT, dict(offsets=P - 32)), ("moe_sort_pairs", GOOD_SORT, dict(order=P + 12)),
    ("moe_sort_pairs", GOOD_SORT, dict(slot=Q + 4096 + 12)), ("moe_sort_pairs", GOOD_SORT, dict(offsets=Q + 4096 - 32)),
    ("moe_gather_rows", GATHER, dict(rows=P - 7 * 32)), ("moe_combine_rows", COMBINE, dict(gate=R + 3 * 32)),
    ("moe_combine_rows", COMBINE, dict(y=P + 7 * 4)), ("moe_combine_rows_backward", GOOD_GRAD, dict(dgate=Q + 8 * 16 - 4)),
    ("moe_combine_rows_backward", GOOD_GRAD, dict(dgate=P + 7 * 4)), ("moe_combine_rows_backward", GOOD_GRAD, dict(dgate=R - 7 * 4)),
    ("moe_combine_rows_backward", GOOD_GRAD, dict(gate=P + (1 << 19))), ("moe_combine_rows_backward", GOOD_GRAD, dict(dgate=Q + 4096 - 28)),
    ("moe_distill_forward", DISTILL, dict(loss=Q + 4 * 400 - 4)), ("moe_distill_forward", DISTILL, dict(loss=P + 4 * 12 - 4)),
    ("moe_distill_forward", DISTILL, dict(lse=R + 12)), ("moe_distill_forward", DISTILL, dict(weight=R - 12)),
    ("moe_distill_forward", DISTILL, dict(lse=P - 12)), ("moe_distill_backward", DISTILL_GRAD, dict(lse=R + 4 * 400 - 4)),
    ("moe_distill_backward", DISTILL_GRAD, dict(dloss=R - 12)), ("moe_distill_backward", DISTILL_GRAD, dict(dlogits=P - 3 * 400)),
])
def test_refusals_of_outputs_that_overlap(name, good, bad):
    assert call(name, good, **bad) == INVALID


@pytest.mark.parametrize("bad", [
    dict(dA=Q + 5 * 64 * 2 - 4), dict(dA=Q + 65536 - 4 * (3 * 8 * 64 - 1)), dict(dB=P + 4 * 4), dict(dA=R + (1 << 20) + 4 * 3 * 8 * 32 - 4),
    dict(dx=R + 65536 - 4), dict(dx_base=R + 65536 - 4), dict(dx=P - 4 * 4 * 64)])
def test_refusals_of_gradients_that_overlap(bad):
    d = desc(a=P + (1 << 16), b=P + (1 << 18), scale=P + (1 << 12))
    a = dict(x=Q, ids=P, dy=Q + 65536, dx_base=None, dx=R, dA=R + 65536, dB=R + (1 << 20))
    a.update(bad)
    assert B.lib().moe_adapters_backward(C.addressof(d), a["x"], 64, a["ids"], 5, F32, a["dy"], 32, a["dx_base"], 64, a["dx"], 64, a["dA"], a["dB"],
                                         P + (1 << 19), 1 << 24, None) == INVALID
    for over in (dict(a=R - 2), dict(b=R + 4), dict(scale=R - 8)):
        e = desc(**dict(dict(a=P + (1 << 16), b=P + (1 << 18), scale=P + (1 << 12)), **over))
        assert B.lib().moe_adapters_forward(C.addressof(e), Q, 64, P, 5, None, 0, F32, R, 32, P + (1 << 19), 1 << 24, None) == INVALID


@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("vocab", (100, 32000, 40000, 70001, 131072, 1000003))
def test_workspace_of_many_rows_serves_fewer(vocab, dtype):
    sizes = [B.lib().moe_distill_workspace_bytes(T, vocab, dtype) for T in [*range(1, 2100), 5000, 65535, 65536, 1 << 20, 1 << 24]]
    assert sizes == sorted(sizes)
    # what calls in shorter chunks need: those of as many rows as leave a compute unit less than four workgroups
    ve, step = 4 if dtype == F32 else 8, 256 * 8
    for T in [t for t in range(1, 2100) if sizes[0]]:
        n = -(-(vocab // ve) // step)
        while n * T < 1024 and vocab // ve // (2 * n) >= 256:
            n *= 2
        assert sizes[T - 1] >= 8 * T * -(-(vocab // ve) // -(-(vocab // ve) // n))
