"""Which sums the 8-bit FFN rounds h from: with a down matrix of ones on its diagonal y is h itself, exactly (one number times 1 and
zeros beside it; four bits of mantissa fit bf16), and codes that differ from those of exact sums are counted.

Few rows to a slot, and few numbers of h, have fp32 sums of bf16 products; the tiles those of the 8-bit instruction.  The same sums cut off
on the CPU (test_mx8_moved_codes_cpu.py) move 2^-8.8 of the numbers, what the tiles may move at most."""
import numpy as np
import pytest
import torch

from harness import f64
from oracle import mx8_oracle as mx
from test_gpu_mx8 import Ffn
from test_mx8_moved_codes_cpu import K as H
from test_mx8_moved_codes_cpu import MOVED_BY_FP32_SUMS, moved

pytestmark = pytest.mark.gpu

MOVED_BY_TILES = 2.0 ** -8.7


class FfnOfOnes(Ffn):
    def _draw(self, rng, I):
        w = super()._draw(rng, I)
        w["down"] = torch.eye(I, self.H, device="cuda")
        return w


def share(y, x, w):
    I = w["gate"].shape[1]
    assert not y[:, I:].any()
    return moved(y[:, :I], x, w["gate"], w["up"])


# 131 072, 368 640 and 1 105 920 numbers of h: 16 rows to a slot; 30, which the tiles would take if there were 2^20 numbers; 90, which they take
@pytest.mark.parametrize("slots,rows,I,bound", [(32, 16, 256, MOVED_BY_FP32_SUMS), (48, 30, 256, MOVED_BY_FP32_SUMS), (48, 90, 256, MOVED_BY_TILES)])
def test_routed_rows(slots, rows, I, bound):
    f = FfnOfOnes(H, I, 1, [rows] * slots, seed=rows)
    y, x = f64(f.run()[0]), mx.rounded(f64(f.x))
    off = [share(y[a:a + rows], x[f.src_of[a:a + rows]], w) for a, w in zip(f.offsets, f.experts)]
    print("moved", float(np.mean(off)), "bound", bound)
    assert np.mean(off) <= bound
    f.L.close()


# the shared expert of 4320 tokens with fewer than 2^20 numbers beside routed rows by tiles
def test_shared_expert_with_few_numbers():
    f = FfnOfOnes(H, 256, 1, [90] * 48, I_shared=192, seed=1)
    off = share(f64(f.run()[1]), mx.rounded(f64(f.x)), f.shared)
    print("moved", off, "bound", MOVED_BY_FP32_SUMS)
    assert off <= MOVED_BY_FP32_SUMS
    f.L.close()
