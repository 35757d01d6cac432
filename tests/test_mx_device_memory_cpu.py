"""Memory that is not the device's is refused as 4-bit weights, on tensors that only say that they are in device memory or not."""
from types import SimpleNamespace

import pytest
import torch

from paper_2602_21140_amd import binding, mx_pack
from test_mx_binding_cpu import DOWN, GATE_UP, bytes_, layer, no_library, on_device


def test_weights_that_are_not_in_device_memory():
    L = layer()
    for gate_up, down in ((torch.zeros(GATE_UP, dtype=torch.uint8), bytes_(DOWN)), (bytes_(GATE_UP), torch.zeros(DOWN, dtype=torch.uint8))):
        with pytest.raises(AssertionError):
            L.set_mx_expert_weights([gate_up, None, None], [down, None, None])


def test_weights_of_one_matrix_without_the_other():
    L = layer()
    for gate_up, down in ((None, bytes_(DOWN)), (bytes_(GATE_UP), None)):
        with pytest.raises(AssertionError):
            L.set_mx_expert_weights([gate_up, None, None], [down, None, None])


def test_pack_into_memory_that_is_not_the_devices(monkeypatch):
    monkeypatch.setattr(binding, "lib", lambda real=binding.lib(): SimpleNamespace(revive_mx_packed_bytes=real.revive_mx_packed_bytes, revive_mx_pack=no_library))
    with pytest.raises(ValueError):
        mx_pack(on_device(4, 32, dtype=torch.uint8), on_device(4, 2, dtype=torch.uint8), out=torch.zeros(binding.mx_packed_bytes(4, 64), dtype=torch.uint8))
