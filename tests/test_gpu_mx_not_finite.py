"""The 4-bit FFN by tiles on rows that are not finite."""
import numpy as np
import pytest

from harness import f64
from test_gpu_mx import Ffn

pytestmark = pytest.mark.gpu


# more than 64 tokens and more than 32 rows per slot; K that ends inside a group of steps, and inside a step
@pytest.mark.parametrize("H,I,I_shared,k,rows", [(576, 320, 192, 2, [100, 0, 130, 37]), (192, 704, 64, 2, [257, 40, 0, 3]), (1088, 64, 576, 1, [200, 300])])
def test_ffn_by_tiles_of_rows_that_are_not_finite(H, I, I_shared, k, rows):
    f = Ffn(H, I, k, rows, I_shared, seed=H)
    n = int(f.offsets[-1])
    assert f.T > 64 and f.N > 32 * f.P
    f.check(*f.run())
    clean, clean_shared = (f64(t) for t in f.run())
    last = [int(f.src_of[e - 1]) // k for e in f.offsets[1:] if e]  # of every slot's last row, which rows past a tile read again
    bad = sorted({0, 17, f.T - 1, *last})
    for i, t in enumerate(bad):
        f.x[t, (i * 61) % H] = (float("nan"), float("inf"), -float("inf"))[i % 3]
    f.x[bad[-1], H - 1] = float("nan")
    y, shared = (f64(t) for t in f.run())
    touched = np.isin(f.src_of[:n] // k, bad)
    assert np.isnan(y[:n][touched]).all() and np.array_equal(y[:n][~touched], clean[:n][~touched]) and (y[n:] == 5.0).all()
    others = [t for t in range(f.T) if t not in bad]
    assert np.isnan(shared[bad]).all() and np.array_equal(shared[others], clean_shared[others])
    f.L.close()
