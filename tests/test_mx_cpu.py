"""Sizes and refusals of the microscaled 4-bit calls that reach no device."""
import pytest
import torch

from paper_2602_21140_amd import ReviveError, binding, mx_dequantize, mx_quantize


@pytest.mark.parametrize("rows,K", [(1, 32), (128, 128), (129, 160), (2048, 7168), (7168, 2048), (1 << 16, (1 << 16) - 32)])
def test_packed_bytes(rows, K):
    up = lambda v, to: -(-v // to) * to
    assert binding.mx_packed_bytes(rows, K) == up(rows, 128) * (up(K, 128) // 2 + up(K, 512) // 32)


@pytest.mark.parametrize("rows,K", [(0, 32), (-1, 32), (4, 0), (4, 33), (4, -32), (1 << 16, 1 << 16)])
def test_packed_bytes_refuses(rows, K):
    with pytest.raises(ReviveError):
        binding.mx_packed_bytes(rows, K)


def test_quantize_refuses_before_any_launch():
    with pytest.raises(TypeError):
        mx_quantize(torch.zeros(2, 64, dtype=torch.float16))
    with pytest.raises(ValueError):
        mx_quantize(torch.zeros(64, 2).t())
    with pytest.raises(ValueError):
        mx_quantize(torch.zeros(2, 64))  # not in device memory
    with pytest.raises(ValueError):
        mx_dequantize(torch.zeros(2, 32, dtype=torch.uint8), torch.zeros(2, 3, dtype=torch.uint8))
    lib = binding.lib()
    assert lib.revive_mx_quantize(None, 1, 4, 64, 64, None, None, None) == -1
    assert lib.revive_mx_dequantize(None, None, 4, 64, 1, None, 64, None) == -1
    assert lib.revive_mx_pack(None, None, 4, 64, None, None) == -1
    assert lib.revive_last_error(None)
