"""The operators around a block together, as block.py uses them: gradients of the whole path against differences of its loss, the forms in
8 bits against the same path on the values that they stand for, serving against training's forward pass, a captured step."""
import pytest
import torch

import paper_2308_14352_amd as moeq
from paper_2308_14352_amd import block, healing

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def setup(tokens, keep, seed=3, d=128, f=96):
    layer, _, g = healing.teacher_and_student(d=d, f=256, n_experts=6, seed=seed)
    w = lambda *s, by=1.0: torch.randn(s, device=DEV, generator=g) * by
    dense = moeq.GatedFfn(w(f, d, by=d**-0.5), w(f, d, by=d**-0.5), w(d, f, by=f**-0.5))
    b = block.Block(layer, dense, 1 + w(d, by=0.1), 1 + w(d, by=0.1), residual_scale=0.5, keep=keep)
    head = w(1000, d, by=0.3)
    n, r = w(tokens, d), w(tokens, d)
    top, idx = torch.topk(w(tokens, 1000, by=4.0), 16, dim=-1)
    return b, head, n, r, idx.to(torch.int32).contiguous(), top.contiguous(), g


@pytest.mark.parametrize("keep", ["own", None])
def test_gradients_against_differences(keep):
    """Central differences along a direction v with two steps h and 2 h: what the step leaves is a third of their difference (the error
    grows with h^2), and fp32 losses of up to 20 from sums of some 400 products are off by 2^-20 of themselves, over 2 h."""
    T = 40
    b, head, n, r, idx, top, g = setup(T, keep)
    _, grads = block.loss_and_gradients(b, head, n, r, idx, top)
    tensors = dict(w_in=b.dense.w_in, w_gate=b.dense.w_gate, w_out=b.dense.w_out, w_after=b.w_after, w_before=b.w_before)

    def total(t, v, by):
        old = t.clone()
        t.add_(v, alpha=by)
        _, after = b.forward(n, r)
        t.copy_(old)
        return moeq.moe_distill_forward(after @ head.t(), idx, top)[0].double().sum().item()

    for name, t in tensors.items():
        v = torch.randn(t.shape, device=DEV, generator=g)
        v *= 1.0 / v.norm()
        diff = lambda h: (total(t, v, h) - total(t, v, -h)) / (2 * h)
        h = 2.0**-5
        one, two = diff(h), diff(2 * h)
        tol = abs(one - two) + T**0.5 * 20 * 2.0**-20 / (2 * h) * 4
        assert abs(one - (grads[name].double() * v.double()).sum().item()) < tol, name


def test_kept_in_8_bits_is_the_path_on_the_values_that_are_kept():
    b, head, n, r, idx, top, _ = setup(70, 8)
    y, after, (f, y2, x8, ab8) = b.forward_kept(n, r)
    dy, dn = torch.randn_like(y), torch.randn_like(y)
    dr, dx, grads = b.backward(dy, dn, (f, y2, x8, ab8))
    same = block.Block(b.layer, b.dense, b.w_after, b.w_before, 0.5, keep="own")
    dr2, dx2, grads2 = same.backward(dy, dn, (f, y2, moeq.moe_unpack8(x8), moeq.moe_unpack8(ab8)))
    assert torch.equal(dr, dr2) and torch.equal(dx, dx2) and all(torch.equal(grads[k], grads2[k]) for k in grads)
    assert x8.nbytes() * 3 < n.numel() * 4


@pytest.mark.parametrize("tokens", [1, 8, 33, 200])
def test_serving_is_trainings_forward_pass(tokens):
    b, head, n, r, *_ = setup(tokens, 8)
    y, after = b.forward(n, r)
    y2, after2, _ = b.forward_kept(n, r)
    assert torch.equal(y, y2) and torch.equal(after, after2)
    # the head in 8 bits: a code is off by half a step, 1/254 of a row's largest value
    head8, logits = block.head_in_8_bits(head), after @ head.t()
    got = block.logits_in_8_bits(after, head8)
    a, h = after.abs().double(), head.abs().double()
    ua, uh = a.amax(1, keepdim=True) / 254, h.amax(1, keepdim=True) / 254
    bound = a @ uh.expand_as(h).t() + ua.expand_as(a) @ (h + uh).t()
    assert ((got - logits).abs().double() <= bound * 1.001).all()


def test_a_fresh_dense_expert_changes_nothing():
    b, _, n, r, *_ = setup(30, 8)
    g = torch.Generator(device=DEV).manual_seed(1)
    fresh = block.Block(b.layer, block.dense_expert(128, 64, g), b.w_after, b.w_before, 0.5)
    y, after = fresh.forward(n, r)
    f = moeq.moe_layer_forward(b.layer, n)
    y2, after2 = moeq.moe_block_norms_forward(f, r, w_after=b.w_after, w_before=b.w_before, residual_scale=0.5)
    assert torch.equal(y, y2) and torch.equal(after, after2)


def test_training_runs():
    teacher, student, g = healing.teacher_and_student(d=128, f=256, n_experts=6)
    head = torch.randn((500, 128), device=DEV, generator=g) * 0.3
    ones = lambda: torch.ones(128, device=DEV)
    t = block.Block(teacher, block.dense_expert(128, 64, g), ones(), ones())
    s = block.Block(student, block.dense_expert(128, 64, g), ones(), ones())
    before = s.dense.w_out.clone()
    losses = list(block.train(s, head, block.teacher_batches(t, head, g, 3, tokens=64, top=8)))
    assert len(losses) == 3 and all(l.isfinite() for l in losses) and not torch.equal(before, s.dense.w_out)
    empty = (torch.empty((0, 128), device=DEV), torch.empty((0, 128), device=DEV), torch.empty((0, 8), dtype=torch.int32, device=DEV), torch.empty((0, 8), device=DEV))
    assert [l.item() for l in block.train(s, head, [empty])] == [0.0]


def test_graph_of_a_training_step():
    """The path's own calls are captured; what lies between them are torch's products."""
    b, head, n, r, idx, top, _ = setup(64, 8)
    run = lambda: (lambda loss, grads: (loss, *grads.values()))(*block.loss_and_gradients(b, head, n, r, idx, top))
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(3):
        for t in got:
            t.fill_(3.0)
        graph.replay()
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def calls(dev, other):
    """Every operator as a call without arguments: of tensors on `dev`, one of the inputs on `other`."""
    f = lambda *s, at=dev: torch.ones(s, device=at)
    ffn, rows, packed = moeq.GatedFfn(f(8, 16), f(8, 16), f(16, 8)), moeq.moe_quantize_rows(f(4, 16)), moeq.moe_pack8(f(4, 16))
    return [lambda: moeq.moe_block_norms_forward(f(4, 16), f(4, 16, at=other)), lambda: moeq.moe_block_norms_backward(f(4, 16), None, f(4, 16, at=other)),
            lambda: moeq.moe_pack8(f(4, 16)), lambda: moeq.moe_unpack8(packed), lambda: moeq.moe_gated_ffn_forward(ffn, f(4, 16, at=other)),
            lambda: moeq.moe_gated_ffn_backward(ffn, f(4, 16), f(4, 16, at=other)), lambda: moeq.moe_quantize_rows(f(4, 16)), lambda: moeq.moe_matmul_q8(rows, rows)]


def test_another_device_is_the_current_one_and_tensors_of_the_host(monkeypatch):
    for call in calls(DEV, DEV):
        call()
    torch.cuda.synchronize()
    for i, call in enumerate(calls(DEV, "cpu")):
        if i in (0, 1, 4, 5):
            with pytest.raises(moeq.MoeqError):
                call()
    made = calls(DEV, DEV)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in made:
        with pytest.raises(moeq.MoeqError) as e:
            call()
        assert e.value.status == moeq.binding.MOEQ_EINVAL
