"""The operators beside the layer refuse tensors on a device that is not the current one, and tensors of several devices, before they
launch anything."""
import pytest
import torch

import paper_2308_14352_amd as moeq

pytestmark = pytest.mark.gpu


def calls(dev, other=None):
    """Every operator as a call without arguments: of tensors on `dev`, one of the inputs on `other`."""
    other = dev if other is None else other
    f = lambda *s, at=dev: torch.ones(s, device=at)
    i = lambda *s, at=dev: torch.zeros(s, dtype=torch.int32, device=at)
    T, k, d = 4, 2, 16
    slot = torch.arange(T * k, dtype=torch.int32, device=dev)
    sort = moeq.PairSort(i(4), slot, slot, T, k, 3)
    ad = moeq.Adapters(f(3, 4, d), f(3, d, 4), f(3))
    return [lambda: moeq.moe_sort_pairs(i(T, k), 3), lambda: moeq.moe_gather_rows(sort, f(T, d, at=other)),
            lambda: moeq.moe_combine_rows(sort, f(T * k, d), f(T, k, at=other)),
            lambda: moeq.moe_combine_rows_backward(sort, f(T, d, at=other), f(T * k, d)),
            lambda: moeq.moe_adapters_forward(ad, f(T, d), i(T, at=other)),
            lambda: moeq.moe_adapters_backward(ad, f(T, d), i(T), f(T, d, at=other)),
            lambda: moeq.moe_distill_forward(f(T, d), i(T, k, at=other), f(T, k)),
            lambda: moeq.moe_distill_backward(f(T, d), i(T, k), f(T, k), f(T), f(T, at=other)),
            lambda: moeq.moe_distill_loss_grad(f(T, d), i(T, k), f(T, k, at=other))]


def test_another_device_is_the_current_one(monkeypatch):
    for call in calls("cuda:0"):
        call()
    torch.cuda.synchronize()
    made = calls("cuda:0")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in made:
        with pytest.raises(moeq.MoeqError) as e:
            call()
        assert e.value.status == moeq.binding.MOEQ_EINVAL


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_tensors_of_two_devices():
    for call in calls("cuda:0", "cuda:1")[1:]:
        with pytest.raises(moeq.MoeqError):
            call()
    with pytest.raises(moeq.MoeqError):
        moeq.Adapters(torch.ones(3, 4, 8, device="cuda:0"), torch.ones(3, 8, 4, device="cuda:1"), torch.ones(3, device="cuda:0"))
    with torch.cuda.device(1):
        for call in calls("cuda:1"):
            call()
        torch.cuda.synchronize()
