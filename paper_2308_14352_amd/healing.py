"""Healing a quantized mixture-of-experts layer: a low-rank adapter for every expert, trained against a teacher's top logits.

The layer's experts stay as they are, packed at 2, 4 or 8 bits. What their rounding cost is learned by adapters on the rows that the
router sends to each expert: the pairs are sorted by expert, the tokens' rows copied into that order, multiplied by their expert's
adapter, and combined back with the gates beside the layer's own output. The loss is the distance to the teacher's largest logits, which
is what a data set of teacher outputs stores.

    python -m paper_2308_14352_amd.healing        heals a small layer of 2-bit experts and prints the loss
"""
import torch

from . import binding as B


class AdaptedLayer:
    """A binding.Layer with an adapter a [E][rank][d], b [E][d][rank] for each of its experts, in the type of the layer's hidden
    states. b starts at zero: a fresh layer computes what the layer computes."""

    def __init__(self, layer, rank, scale=1.0, generator=None):
        self.layer = layer
        E, d, dev = layer.n_experts, layer.d_model, layer.router_w.device
        dtype = torch.bfloat16 if layer.x_dtype == B.MOEQ_BF16 else torch.float32
        a = torch.randn((E, rank, d), device=dev, generator=generator) / d**0.5
        self.adapters = B.Adapters(a.to(dtype), torch.zeros((E, d, rank), dtype=dtype, device=dev), torch.full((E,), float(scale), device=dev))

    def forward(self, x):
        """x [T][d] in the layer's type -> (y [T][d] fp32, what backward needs)."""
        y, idx, gate = B.moe_layer_forward(self.layer, x, want_routing=True)
        sort = B.moe_sort_pairs(idx, self.layer.n_experts)
        rows = B.moe_gather_rows(sort, x)
        ids = idx.flatten()[torch.where(sort.order < 0, ~sort.order, sort.order).long()]
        out = B.moe_adapters_forward(self.adapters, rows, ids)
        y += B.moe_combine_rows(sort, out, gate, dtype=torch.float32)
        return y, (sort, rows, ids, out, gate)

    def backward(self, dy, saved):
        """dy [T][d] fp32 -> (dA, dB, dgate, dx): the gradients of the adapters, and of the gates and the hidden states as far as they
        come through the adapters."""
        sort, rows, ids, out, gate = saved
        dout, dgate = B.moe_combine_rows_backward(sort, dy, out, gate)
        drows, dA, dB = B.moe_adapters_backward(self.adapters, rows, ids, dout)
        return dA, dB, dgate, B.moe_combine_rows(sort, drows, dtype=torch.float32)


def loss_and_gradients(adapted, head, x, top_idx, top_logits, temperature=1.0, weight=None):
    """(loss [T], dA, dB) of the sum of the losses for logits y head^T, head [V][d]."""
    y, saved = adapted.forward(x)
    loss, dlogits = B.moe_distill_loss_grad(y @ head.t(), top_idx, top_logits, temperature, weight)
    dA, dB, _, _ = adapted.backward(dlogits @ head, saved)
    return loss, dA, dB


def heal(adapted, head, batches, temperature=1.0, lr=1e-3):
    """One pass over batches of (x, top_idx, top_logits), by Adam on fp32 copies of the adapters. Yields the mean loss of every batch."""
    ad = adapted.adapters
    params = [torch.nn.Parameter(t.float()) for t in (ad.a, ad.b)]
    opt = torch.optim.Adam(params, lr=lr)
    for x, top_idx, top_logits in batches:
        if x.shape[0] == 0:
            yield torch.zeros((), device=x.device)      # (nothing to learn from, and no mean)
            continue
        loss, dA, dB = loss_and_gradients(adapted, head, x, top_idx, top_logits, temperature)
        for p, g, t in zip(params, (dA, dB), (ad.a, ad.b)):
            p.grad = g / x.shape[0]
        opt.step()
        for p, t in zip(params, (ad.a, ad.b)):
            t.copy_(p.detach())                # (in place: the adapters borrow these tensors)
        yield loss.mean()


def _pack(w_in, w_out, bits, group):
    q_in, s_in = B.moe_quantize_pack(w_in, bits, group)
    q_out, s_out = B.moe_quantize_pack(w_out, bits, group)
    return B.PackedExpert(bits, q_in, s_in, q_out, s_out)


def teacher_and_student(d=256, f=512, n_experts=8, top_k=2, bits=2, group=32, device="cuda:0", seed=0):
    """Two ReLU layers of the same random weights and router: the experts at 8 bits, and at `bits`."""
    g = torch.Generator(device=device).manual_seed(seed)
    weights = [(torch.randn((f, d), device=device, generator=g) / d**0.5, torch.randn((d, f), device=device, generator=g) / f**0.5)
               for _ in range(n_experts)]
    router = torch.randn((n_experts, d), device=device, generator=g) / d**0.5
    make = lambda b: B.Layer(d, f, top_k, group, B.MOEQ_ACT_RELU, True, B.MOEQ_F32, router, None, [_pack(wi, wo, b, group) for wi, wo in weights])
    return make(8), make(bits), g


def teacher_batches(teacher, head, g, n, tokens=1024, top=32):
    """n batches of (x, top_idx, top_logits): what a stored set of teacher outputs holds."""
    for _ in range(n):
        x = torch.randn((tokens, teacher.d_model), device=head.device, generator=g)
        top_logits, top_idx = torch.topk(B.moe_layer_forward(teacher, x) @ head.t(), top, dim=-1)
        yield x, top_idx.to(torch.int32).contiguous(), top_logits.contiguous()


def main():
    teacher, student, g = teacher_and_student()
    head = torch.randn((4096, teacher.d_model), device="cuda:0", generator=g) * 0.3
    adapted = AdaptedLayer(student, rank=16, generator=g)
    for i, loss in enumerate(heal(adapted, head, teacher_batches(teacher, head, g, 201), lr=3e-3)):
        if i % 25 == 0:
            print(f"batch {i:4d}  loss {loss.item():.4f}")


if __name__ == "__main__":
    main()
