"""Calls whose tensors have more than 2^31 elements: their last rows against a call of those rows alone."""
import pytest
import torch

import paper_2308_14352_amd as moeq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def noise(*shape, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def test_packed():
    x = noise(65600, 32800)
    assert x.numel() > 2**31
    p, tail = moeq.moe_pack8(x), moeq.moe_pack8(x[-5:])
    assert torch.equal(p.codes[-5:], tail.codes) and torch.equal(p.exps[-5:], tail.exps)
    assert torch.equal(moeq.moe_unpack8(p)[-5:], moeq.moe_unpack8(tail))


def test_norms():
    f, r = noise(262400, 8200), noise(262400, 8200, seed=1)
    assert f.numel() > 2**31
    w = torch.rand(8200, device=DEV) + 0.5
    y, n = moeq.moe_block_norms_forward(f, r, w_after=w, w_before=w)
    y2, n2 = moeq.moe_block_norms_forward(f[-7:], r[-7:], w_after=w, w_before=w)
    assert torch.equal(y[-7:], y2) and torch.equal(n[-7:], n2)
    df, dr, *_ = moeq.moe_block_norms_backward(f, y, r, n, w_after=w, w_before=w)
    df2, dr2, *_ = moeq.moe_block_norms_backward(f[-7:], y2, r[-7:], n2, w_after=w, w_before=w)
    assert torch.equal(df[-7:], df2) and torch.equal(dr[-7:], dr2)


@pytest.mark.parametrize("keep", ["own", 8])
def test_gated_block(keep):
    T, D, F, last = 131200, 64, 16448, 600
    assert T * F > 2**31
    x, dy = noise(T, D), noise(T, D, seed=1)
    ffn = moeq.GatedFfn(noise(F, D, seed=2) / 8, noise(F, D, seed=3) / 8, noise(D, F, seed=4) / 128)
    y, ab = moeq.moe_gated_ffn_forward(ffn, x, keep=keep)
    y2, ab2 = moeq.moe_gated_ffn_forward(ffn, x[-last:], keep=keep)
    dx = moeq.moe_gated_ffn_backward(ffn, x, dy, ab)[0]
    dx2 = moeq.moe_gated_ffn_backward(ffn, x[-last:], dy[-last:], ab2)[0]
    # a sum in shares or in tiles of another size adds in another order: what two fp32 sums of 2 x 16448 products differ by is far below a
    # step of bf16, which a value beside a border may differ by; fp32 sums relative to the row's largest: 8 sqrt(32896) 2^-24 times its terms
    for a, b in ((y[-last:], y2), (dx[-last:], dx2)):
        a, b = a.float(), b.float()
        assert ((a - b).abs() <= 2.0**-7 * b.abs() + 2.0**-12 * b.abs().amax(1, keepdim=True)).all()
        assert (a == b).float().mean() > 0.9
    if keep == "own":
        assert torch.equal(ab[:, -last:], ab2)
    else:
        assert torch.equal(ab.codes[:, -last:], ab2.codes) and torch.equal(ab.exps[:, -last:], ab2.exps)


def test_products():
    T, N = 16500, 131072
    assert T * N > 2**31
    q, w = moeq.moe_quantize_rows(noise(T, 128)), moeq.moe_quantize_rows(noise(N, 128, seed=1))
    y = moeq.moe_matmul_q8(q, w, dtype=torch.bfloat16)
    tail = moeq.moe_quantize_rows(noise(T, 128)[-40:])
    assert torch.equal(y[-40:], moeq.moe_matmul_q8(tail, w, dtype=torch.bfloat16))
