"""What the 4-bit FFN of the binding refuses before the library is called, on tensors that only say that they are in device memory."""
from types import SimpleNamespace

import pytest
import torch

from paper_2602_21140_amd import ReviveLayer, binding


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)


def on_device(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


def no_library(*_args):
    raise AssertionError("the library was called")


H, I, I_SHARED, K, P, T = 128, 64, 192, 2, 3, 5
GATE_UP, DOWN = 2 * binding.mx_packed_bytes(I, H), binding.mx_packed_bytes(H, I)
SHARED = [2 * binding.mx_packed_bytes(I_SHARED, H), binding.mx_packed_bytes(H, I_SHARED)]


def bytes_(n):
    return on_device(n, dtype=torch.uint8)


def layer(I_shared=I_SHARED):
    L = object.__new__(ReviveLayer)
    L.cfg = SimpleNamespace(H=H, I=I, I_shared=I_shared, k=K)
    L.P, L.T_max, L.device, L.dtype, L._ctx, L._mx_tabs = P, T, "cpu", torch.bfloat16, None, None
    L.L = SimpleNamespace(revive_mx_expert_ffn=lambda *a: 0)
    L.set_mx_expert_weights([bytes_(GATE_UP), None, bytes_(GATE_UP)], [bytes_(DOWN), None, bytes_(DOWN)])
    return L


def arguments(**change):
    a = dict(x=on_device(T, H), src_of=on_device(T * K, dtype=torch.int32), slot_offsets=on_device(P + 1, dtype=torch.int32), T=T,
             w_sh_gate_up=bytes_(SHARED[0]), w_sh_down=bytes_(SHARED[1]), out=(on_device(T * K, H), on_device(T, H)), stream=SimpleNamespace(cuda_stream=0))
    return {**a, **change}


def test_ffn_takes_what_fits():
    L = layer()
    L.mx_expert_ffn(**arguments())
    L.mx_expert_ffn(**arguments(w_sh_gate_up=None, w_sh_down=None, out=(on_device(T * K, H), None)))
    L.mx_expert_ffn(**arguments(T=2))  # the first tokens of more
    layer(0).mx_expert_ffn(**arguments(w_sh_gate_up=None, w_sh_down=None, out=(on_device(T * K, H), None)))


@pytest.mark.parametrize("change", [
    dict(x=torch.zeros(T, H, dtype=torch.bfloat16)), dict(x=on_device(T - 1, H)), dict(x=on_device(T, H + 64)), dict(x=on_device(T * H)),
    dict(x=on_device(T, H, dtype=torch.float32)),
    dict(src_of=on_device(T * K, dtype=torch.int64)), dict(src_of=on_device(T * K - 1, dtype=torch.int32)), dict(src_of=torch.zeros(T * K, dtype=torch.int32)),
    dict(src_of=on_device(2 * T * K, dtype=torch.int32)[::2]),
    dict(slot_offsets=on_device(P + 1, dtype=torch.int64)), dict(slot_offsets=on_device(P, dtype=torch.int32)),
    dict(slot_offsets=torch.zeros(P + 1, dtype=torch.int32)),
    dict(w_sh_gate_up=bytes_(SHARED[0] - 16)), dict(w_sh_gate_up=bytes_(SHARED[0] + 16)), dict(w_sh_down=bytes_(SHARED[1] - 16)), dict(w_sh_gate_up=on_device(SHARED[0])),
    dict(w_sh_gate_up=torch.zeros(SHARED[0], dtype=torch.uint8)), dict(w_sh_down=None),
    dict(out=(on_device(T * K, H), None)), dict(out=(on_device(T * K - 1, H), on_device(T, H))), dict(out=(on_device(T * K, H), on_device(T - 1, H))),
    dict(out=(on_device(T * K, H, dtype=torch.float32), on_device(T, H))), dict(out=(torch.zeros(T * K, H, dtype=torch.bfloat16), on_device(T, H)))])
def test_ffn_refuses(change):
    L = layer()
    L.L = SimpleNamespace(revive_mx_expert_ffn=no_library)
    with pytest.raises(ValueError):
        L.mx_expert_ffn(**arguments(**change))


def test_ffn_refuses_a_shared_expert_that_the_layer_does_not_have():
    L = layer(0)
    L.L = SimpleNamespace(revive_mx_expert_ffn=no_library)
    with pytest.raises(ValueError):
        L.mx_expert_ffn(**arguments())
