"""Which device a layer belongs to: one named without a number is the device that is current when the layer is made, whatever is
current later, and weights have to lie on it."""
import contextlib
import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2602_21140_amd import ReviveLayer, binding

H, I, K, P, T = 128, 64, 2, 3, 5
CFG = SimpleNamespace(T=T, H=H, E=P, k=K, I=I, I_shared=0, n_ranks=1, slots_per_rank=P, max_replicas=1, score_fn="softmax", n_group=1, topk_group=1,
                      dtype="bf16")
GATE_UP, DOWN = 2 * binding.mx8_packed_bytes(I, H), binding.mx8_packed_bytes(H, I)


def tensors_of(place):
    """Makes tensors that say they are in the memory of device `place`."""
    class There(torch.Tensor):
        is_cuda = property(lambda self: True)

        def get_device(self):
            return place

    def make(*shape, dtype=torch.uint8):
        return torch.zeros(*shape, dtype=dtype).as_subclass(There)
    return make


@pytest.fixture
def on_device_1(monkeypatch):
    """Two devices, of which 1 is current, and a library that takes every call."""
    real = binding.lib()

    def bytes_needed(ctx, n):
        ctypes.cast(n, ctypes.POINTER(ctypes.c_size_t))[0] = 256
        return 0

    calls = {n: lambda *a: 0 for n in ("revive_create", "revive_bind_workspace", "revive_destroy", "revive_mx_eight_expert_ffn")}
    monkeypatch.setattr(binding, "lib", lambda: SimpleNamespace(revive_workspace_bytes=bytes_needed, revive_mx_eight_packed_bytes=real.revive_mx_eight_packed_bytes,
                                                            revive_last_error=real.revive_last_error, **calls))
    monkeypatch.setattr(binding, "_get_device", lambda: 1)
    monkeypatch.setattr(binding, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "device", lambda device: contextlib.nullcontext())
    plain, to = torch.empty, torch.Tensor.to
    monkeypatch.setattr(torch, "empty", lambda *shape, dtype=None, device=None: plain(*shape, dtype=dtype))
    monkeypatch.setattr(torch.Tensor, "to", lambda self, *a, **kw: self if a and isinstance(a[0], torch.device) else to(self, *a, **kw))


def call(layer, make):
    i32 = torch.int32
    return layer.mx8_expert_ffn(make(T, H), make(T, H // 32), make(T * K, dtype=i32), make(P + 1, dtype=i32), T,
                                out=(make(T * K, H, dtype=torch.bfloat16), None), stream=SimpleNamespace(cuda_stream=0, device_index=1))


@pytest.mark.parametrize("device", ["cuda", "cuda:1"])
def test_a_layer_on_the_current_device_takes_its_tensors(on_device_1, device):
    layer, make = ReviveLayer(CFG, device=device), tensors_of(1)
    layer.set_mx8_expert_weights([make(GATE_UP)] * P, [make(DOWN)] * P)
    call(layer, make)
    assert layer.device == torch.device("cuda:1")


def test_a_layer_on_another_device_than_the_current_one_is_refused(on_device_1):
    layer = ReviveLayer(CFG, device="cuda:0")
    layer._mx8_tabs = (torch.zeros(P), torch.zeros(P))
    with pytest.raises(ValueError, match="the layer is on cuda:0"):
        call(layer, tensors_of(1))


def test_weights_on_another_device_than_the_layer_are_refused(on_device_1):
    layer, here, there = ReviveLayer(CFG, device="cuda"), tensors_of(1), tensors_of(0)
    for gate_up, down in ((there, here), (here, there), (there, there)):
        with pytest.raises(AssertionError, match="weights in the memory of cuda:1"):
            layer.set_mx8_expert_weights([here(GATE_UP), None, gate_up(GATE_UP)], [here(DOWN), None, down(DOWN)])
    layer.set_mx8_expert_weights([here(GATE_UP), None, None], [here(DOWN), None, None])
