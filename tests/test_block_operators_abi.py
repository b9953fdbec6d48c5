"""CPU-only checks of the norms around a block, the gated feed-forward block, packed tensors and 8-bit products: sizes, and refusals
before any device call."""
import ctypes as C

import pytest
import torch

import paper_2308_14352_amd as moeq
from paper_2308_14352_amd import binding as B

P, Q, R, S = 1 << 20, 1 << 30, 1 << 40, 1 << 44          # addresses far apart; nothing is read in a refused call
OK, INVALID, UNSUPPORTED, WORKSPACE = B.MOEQ_OK, B.MOEQ_EINVAL, B.MOEQ_EUNSUPPORTED, B.MOEQ_EWORKSPACE
F32, BF16, F16 = B.MOEQ_F32, B.MOEQ_BF16, B.MOEQ_F16


def call(name, good, **bad):
    args = dict(good, **bad)
    assert set(args) == set(good)
    return getattr(B.lib(), name)(*args.values())


NORMS = dict(T=4, d=8, alpha=1.0, eps=1e-5, f_dtype=F32, f=Q, f_stride=8, r_dtype=BF16, r=R, r_stride=8, gate=P, w_after=P + 4096, w_before=P + 8192,
             y=S, y_stride=8, n_dtype=BF16, n=S + 4096, n_stride=8, stream=None)
GRAD = dict(T=4, d=8, alpha=1.0, eps=1e-5, f_dtype=F32, f=Q, f_stride=8, r_dtype=BF16, y=R, y_stride=8, dy=R + 4096, dy_stride=8, n_dtype=BF16, dn=R + 8192,
            dn_stride=8, gate=P, w_after=P + 4096, w_before=P + 8192, df=S, df_stride=8, dr=S + 4096, dr_stride=8, dgate=S + 8192, dw_after=S + 12288,
            dw_before=S + 16384, ws=None, ws_bytes=0, stream=None)
PACK = dict(x=Q, x_stride=40, dtype=BF16, rows=4, d=40, codes=R, exps=S, stream=None)
UNPACK = dict(codes=R, exps=S, rows=4, d=40, dtype=BF16, x=Q, x_stride=40, stream=None)
ROWS = dict(x=Q, x_stride=40, dtype=BF16, rows=4, d=40, codes=R, scale=S, stream=None)
Q8 = dict(x=P, xs=P + 65536, T=4, w=Q, ws=Q + (1 << 20), n=100, k=300, base=None, base_stride=0, dtype=F32, y=R, y_stride=100, room=None, room_bytes=0, stream=None)


@pytest.mark.parametrize("name,good,bad,status", [
    ("moe_block_norms_forward", NORMS, dict(T=-1), INVALID), ("moe_block_norms_forward", NORMS, dict(d=0), INVALID),
    ("moe_block_norms_forward", NORMS, dict(d=16385, f_stride=16385, r_stride=16385, y_stride=16385, n_stride=16385), UNSUPPORTED),
    ("moe_block_norms_forward", NORMS, dict(f_dtype=3), INVALID), ("moe_block_norms_forward", NORMS, dict(f_dtype=F16), INVALID),
    ("moe_block_norms_forward", NORMS, dict(n_dtype=F16), INVALID), ("moe_block_norms_forward", NORMS, dict(eps=-1.0), INVALID),
    ("moe_block_norms_forward", NORMS, dict(eps=float("nan")), INVALID), ("moe_block_norms_forward", NORMS, dict(alpha=float("inf")), INVALID),
    ("moe_block_norms_forward", NORMS, dict(f=None), INVALID), ("moe_block_norms_forward", NORMS, dict(r=None), INVALID),
    ("moe_block_norms_forward", NORMS, dict(y=None), INVALID), ("moe_block_norms_forward", NORMS, dict(n=None), INVALID),
    ("moe_block_norms_forward", NORMS, dict(f_stride=7), INVALID), ("moe_block_norms_forward", NORMS, dict(y_stride=0), INVALID),
    ("moe_block_norms_forward", NORMS, dict(f=Q + 2), INVALID), ("moe_block_norms_forward", NORMS, dict(gate=P + 2), INVALID),
    ("moe_block_norms_forward", NORMS, dict(y=R + 2), INVALID), ("moe_block_norms_forward", NORMS, dict(y=Q), INVALID),
    ("moe_block_norms_forward", NORMS, dict(n=Q), INVALID), ("moe_block_norms_forward", NORMS, dict(n=S), INVALID),
    ("moe_block_norms_forward", NORMS, dict(y=P), INVALID), ("moe_block_norms_forward", NORMS, dict(n=R), INVALID),
    ("moe_block_norms_backward", GRAD, dict(), WORKSPACE), ("moe_block_norms_backward", GRAD, dict(ws=S + (1 << 30), ws_bytes=64), WORKSPACE),
    ("moe_block_norms_backward", GRAD, dict(ws=S + (1 << 30) + 2, ws_bytes=1 << 20), INVALID), ("moe_block_norms_backward", GRAD, dict(y=None), INVALID),
    ("moe_block_norms_backward", GRAD, dict(dn=None), INVALID), ("moe_block_norms_backward", GRAD, dict(dy=None), INVALID),
    ("moe_block_norms_backward", GRAD, dict(df=Q), INVALID), ("moe_block_norms_backward", GRAD, dict(dr=R), INVALID),
    ("moe_block_norms_backward", GRAD, dict(dr=R + 4096), INVALID), ("moe_block_norms_backward", GRAD, dict(dgate=None), INVALID),
    ("moe_block_norms_backward", GRAD, dict(dw_after=None), INVALID), ("moe_block_norms_backward", GRAD, dict(dw_before=S + 12288), INVALID),
    ("moe_block_norms_backward", GRAD, dict(dgate=P), INVALID), ("moe_block_norms_backward", GRAD, dict(df_stride=7), INVALID),
    ("moe_pack8", PACK, dict(rows=-1), INVALID), ("moe_pack8", PACK, dict(d=0), INVALID), ("moe_pack8", PACK, dict(codes=None), INVALID),
    ("moe_pack8", PACK, dict(x=Q + 1), INVALID), ("moe_pack8", PACK, dict(x_stride=39), INVALID), ("moe_pack8", PACK, dict(exps=R + 159), INVALID),
    ("moe_pack8", PACK, dict(codes=Q + 300), INVALID), ("moe_pack8", PACK, dict(dtype=9), INVALID),
    ("moe_unpack8", UNPACK, dict(exps=None), INVALID), ("moe_unpack8", UNPACK, dict(x=R - 100), INVALID), ("moe_unpack8", UNPACK, dict(x_stride=0), INVALID),
    ("moe_quantize_rows", ROWS, dict(d=65537, x_stride=65537), UNSUPPORTED), ("moe_quantize_rows", ROWS, dict(codes=R + 8), INVALID),
    ("moe_quantize_rows", ROWS, dict(scale=None), INVALID), ("moe_quantize_rows", ROWS, dict(scale=R + 508), INVALID), ("moe_quantize_rows", ROWS, dict(x=None), INVALID),
    ("moe_matmul_q8", Q8, dict(T=-1), INVALID), ("moe_matmul_q8", Q8, dict(n=0), INVALID), ("moe_matmul_q8", Q8, dict(k=0), INVALID),
    ("moe_matmul_q8", Q8, dict(k=65537), UNSUPPORTED), ("moe_matmul_q8", Q8, dict(T=(1 << 20) + 1), UNSUPPORTED), ("moe_matmul_q8", Q8, dict(n=(1 << 20) + 1), UNSUPPORTED),
    ("moe_matmul_q8", Q8, dict(T=1 << 18, n=(1 << 18) + 1), UNSUPPORTED), ("moe_pack8", PACK, dict(d=(1 << 30) + 1, x_stride=1 << 31), UNSUPPORTED),
    ("moe_unpack8", UNPACK, dict(d=(1 << 30) + 1, x_stride=1 << 31), UNSUPPORTED),
    ("moe_matmul_q8", Q8, dict(x=None), INVALID), ("moe_matmul_q8", Q8, dict(w=Q + 8), INVALID), ("moe_matmul_q8", Q8, dict(xs=P + 2), INVALID),
    ("moe_matmul_q8", Q8, dict(y=Q + 128), INVALID), ("moe_matmul_q8", Q8, dict(y_stride=99), INVALID), ("moe_matmul_q8", Q8, dict(base=R + 4, base_stride=100), INVALID),
    ("moe_matmul_q8", Q8, dict(dtype=4), INVALID),
])
def test_refusals(name, good, bad, status):
    assert call(name, good, **bad) == status


def desc(**kw):
    d = dict(d_model=64, d_ff=96, dtype=BF16, w_in=P, w_gate=P + 65536, w_out=P + 131072)
    d.update(kw)
    return B.moeq_gated_ffn(*d.values())


@pytest.mark.parametrize("kw,bad,status", [
    (dict(d_model=0), {}, INVALID), (dict(d_ff=-1), {}, INVALID), (dict(dtype=7), {}, INVALID), (dict(w_in=None), {}, INVALID), (dict(w_gate=P + 1), {}, INVALID),
    (dict(w_out=None), {}, INVALID), (dict(d_model=65537), {}, UNSUPPORTED), (dict(d_ff=65537), {}, UNSUPPORTED),
    (dict(d_ff=65536), dict(T=(1 << 19) + 1), UNSUPPORTED), ({}, dict(T=-1), INVALID), ({}, dict(T=(1 << 20) + 1), UNSUPPORTED), ({}, dict(keep=2), INVALID), ({}, dict(x=None), INVALID), ({}, dict(x_stride=63), INVALID),
    ({}, dict(out=None), INVALID), ({}, dict(out=Q), INVALID), ({}, dict(out_stride=0), INVALID), ({}, dict(ab=None), INVALID), ({}, dict(ab=S + 1), INVALID),
    ({}, dict(keep=8, exps=None), INVALID), ({}, dict(ws=None), WORKSPACE), ({}, dict(ws_bytes=100), WORKSPACE), ({}, dict(ws=S + (1 << 30) + 16), INVALID),
])
def test_refusals_of_the_gated_block(kw, bad, status):
    d = desc(**kw)
    a = dict(x=Q, x_stride=64, T=5, out=R, out_stride=64, keep=1, ab=S, exps=S + (1 << 20), ws=S + (1 << 30), ws_bytes=1 << 24)
    a.update(bad)
    L = B.lib()
    assert L.moe_gated_ffn_forward(C.addressof(d), a["x"], a["x_stride"], a["T"], None, 0, BF16, a["out"], a["out_stride"], a["keep"], a["ab"], a["exps"], a["ws"],
                                   a["ws_bytes"], None) == status
    if bad.get("out", 0) is None:
        return                                # (dx need not be wanted)
    dw = R + (1 << 20)
    assert L.moe_gated_ffn_backward(C.addressof(d), a["x"], a["x_stride"], None, None, a["T"], Q + 65536, 64, a["keep"], a["ab"], a["exps"], a["out"], a["out_stride"],
                                    dw, dw + 65536, dw + 131072, a["ws"], a["ws_bytes"], None) == status


def test_more_refusals_of_the_gated_block():
    L, d = B.lib(), desc()
    h, ws, dw = C.addressof(d), S + (1 << 30), R + (1 << 20)
    fwd = lambda base=None, dtype=BF16, ab=S, y=R: L.moe_gated_ffn_forward(h, Q, 64, 5, base, 64, dtype, y, 64, 1, ab, None, ws, 256, None)
    assert fwd() == WORKSPACE                      # (the good call but for its workspace)
    assert fwd(dtype=F16) == INVALID and fwd(base=R + 2) == INVALID and fwd(base=S) == INVALID and fwd(ab=R) == INVALID and fwd(y=P + 64) == INVALID
    assert fwd(base=R) == WORKSPACE
    bwd = lambda x=Q, xc=None, xe=None, dx=R, g=dw, o=dw + 131072: L.moe_gated_ffn_backward(h, x, 64, xc, xe, 5, Q + 65536, 64, 0, None, None, dx, 64, g, dw + 65536, o, ws, 256, None)
    assert bwd() == WORKSPACE and bwd(dx=None) == WORKSPACE and bwd(x=None, xc=Q, xe=Q + 4096) == WORKSPACE
    assert bwd(x=None) == INVALID and bwd(xc=Q, xe=Q + 4096) == INVALID and bwd(x=None, xc=Q) == INVALID
    assert bwd(g=None) == INVALID and bwd(o=dw) == INVALID and bwd(g=P) == INVALID and bwd(dx=Q) == INVALID and bwd(dx=dw) == INVALID
    assert L.moe_gated_ffn_forward(None, Q, 64, 5, None, 0, BF16, R, 64, 0, None, None, ws, 1 << 24, None) == INVALID


def test_calls_without_rows_are_no_ops_without_pointers():
    L, d = B.lib(), desc()
    assert call("moe_block_norms_forward", NORMS, T=0, f=None, r=None, y=None, n=None, gate=None) == OK
    assert call("moe_pack8", PACK, rows=0, x=None, codes=None, exps=None) == OK and call("moe_unpack8", UNPACK, rows=0, x=None, codes=None, exps=None) == OK
    assert call("moe_quantize_rows", ROWS, rows=0, x=None, codes=None, scale=None) == OK
    assert call("moe_matmul_q8", Q8, T=0, x=None, xs=None, y=None) == OK
    assert L.moe_gated_ffn_forward(C.addressof(d), None, 64, 0, None, 0, BF16, None, 64, 1, None, None, None, 0, None) == OK


def test_sizes():
    L = B.lib()
    assert [L.moe_q8_pitch(k) for k in (0, 1, 128, 129, 4096)] == [0, 128, 128, 256, 4096]
    assert L.moe_block_norms_workspace_bytes(0, 64) == 0 and L.moe_block_norms_workspace_bytes(4, 16385) == 0 and L.moe_block_norms_workspace_bytes(4, 64) >= 4 * 2 * 64 * 4
    d = desc()
    size = lambda T, back, packed, keep: L.moe_gated_ffn_workspace_bytes(C.addressof(d), T, back, packed, keep)
    assert size(0, 0, 0, 0) == 0 and size(5, 0, 0, 3) == 0 and L.moe_gated_ffn_workspace_bytes(None, 5, 0, 0, 0) == 0
    assert 0 < size(5, 0, 0, 0) <= size(65, 0, 0, 0) < size(65, 1, 0, 1) < size(65, 1, 1, 1) < size(65, 1, 1, 0)
    assert L.moe_matmul_q8_workspace_bytes(0, 5, 5) == 0 and L.moe_matmul_q8_workspace_bytes(4, 5, 65537) == 0


def test_binding_refuses_tensors_that_are_not_on_the_device_or_of_another_form():
    x, w = torch.zeros((4, 8)), torch.zeros(8)
    codes = torch.zeros((4, 8), dtype=torch.int8)
    for call_ in (lambda: moeq.moe_block_norms_forward(x, x), lambda: moeq.moe_block_norms_backward(x, None, x), lambda: moeq.moe_pack8(x),
                  lambda: moeq.moe_unpack8(moeq.Packed8(codes, codes, torch.float32)), lambda: moeq.moe_quantize_rows(x),
                  lambda: moeq.GatedFfn(x, x, x.t()), lambda: moeq.GatedFfn(x, x, x), lambda: moeq.QuantRows(codes, w), lambda: moeq.QuantRows(x, w)):
        with pytest.raises(moeq.MoeqError) as e:
            call_()
        assert e.value.status == INVALID
    with pytest.raises(moeq.MoeqError):
        B._keep(16)
