"""4-bit floats of more rows than one launch has threads for."""
import pytest
import torch

from paper_2602_21140_amd import mx_dequantize, mx_quantize

pytestmark = pytest.mark.gpu


def test_more_rows_than_a_launch_has_threads_for():
    """Four threads a row, and at most 2^32 - 1 threads in a grid."""
    rows = 2 ** 30 + 4099
    value = torch.tensor([0.0, 1.0, -2.0, 3.0, 0.5, -6.0, 1.5, 4.0, -24.0, 2.0 ** -20, 48.0], dtype=torch.bfloat16, device="cuda")
    x = value.repeat(rows // 11 + 1)[:rows].view(rows, 1)
    codes, scales = mx_quantize(x)
    back = mx_dequantize(codes, scales, 1)
    assert torch.equal(back, x)
    del back
    assert torch.equal(scales[-11 * 400:], scales[(rows - 11 * 400) % 11:][:11 * 400])
    some, some_scales = mx_quantize(x[:11])
    for part in range(0, rows, 2 ** 28):
        a = part - part % 11
        b = min(rows, a + 2 ** 28)
        n = (b - a) // 11 * 11
        assert bool((codes[a:a + n].view(-1, 11, 16) == some).all()) and bool((scales[a:a + n].view(-1, 11, 1) == some_scales).all())
