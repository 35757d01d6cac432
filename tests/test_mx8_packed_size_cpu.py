"""The size of packed weights that mx8_linear works out by itself is the library's, for panels and steps that are whole and broken."""
from types import SimpleNamespace

import pytest
import torch

from paper_2602_21140_amd import binding, mx8_linear


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def t(*shape, dtype=torch.uint8):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


@pytest.mark.parametrize("K", [32, 96, 128, 160, 1024, 1056])
@pytest.mark.parametrize("N", [1, 127, 128, 129, 300])
def test_packed_size_is_the_librarys(monkeypatch, N, K):
    n = binding.mx8_packed_bytes(N, K)
    monkeypatch.setattr(binding, "lib", lambda: SimpleNamespace(revive_mx_eight_linear=lambda *a: 0))
    monkeypatch.setattr(binding, "_get_device", lambda: 0)
    form, how = (t(2, K), t(2, K // 32)), dict(out=t(2, N, dtype=torch.bfloat16), stream=SimpleNamespace(cuda_stream=0, device_index=0))
    mx8_linear(*form, t(n), N, **how)
    for other in (n - 1, n + 1, n - 128 * 132, n + 128 * 132):
        with pytest.raises(ValueError):
            mx8_linear(*form, t(max(other, 0)), N, **how)
