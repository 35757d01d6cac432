"""The oracle of the 4-bit form of the layer, pinned by closed forms and by search."""
import numpy as np
import pytest

from oracle import mx_oracle as mx
from oracle import revive_oracle as orc


def test_hand_worked_block():
    # largest 7 -> floor(log2 7) = 2 -> scale 2^0; midpoints go to the even code, 7 saturates
    x = np.zeros((1, 32))
    x[0, :14] = [7, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -0.25, -0.75, -2.5, 0.24]
    codes, scales = mx.quantize(x)
    assert scales.tolist() == [[127]]
    assert mx.values(codes, scales)[0, :14].tolist() == [6, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, 0, -1, -2, 0]
    assert codes[0, 0] == 0x07 and codes[0, 5] == 0xA8  # two codes a byte, the lower k below: (7, 0), (-0, -1)


@pytest.mark.parametrize("exponent", [-126, -30, 0, 5, 127])
def test_scale_is_a_power_of_two_that_puts_the_largest_into_4_to_8(exponent):
    rng = np.random.default_rng(0)
    for largest in (1.0, 1.5, 1.999):
        x = rng.uniform(-1, 1, (1, 32))
        x[0, 3] = largest
        s = int(mx.scale_bytes(x * 2.0 ** exponent)[0, 0])
        assert s == max(exponent + 125, 0)


def test_zeros_tiny_and_not_finite_blocks():
    x = np.zeros((5, 32))
    x[1, 4] = 2.0 ** -140
    x[2, 0] = np.inf
    x[3, 31] = np.nan
    x[4, 1] = 3 * 2.0 ** -128
    codes, scales = mx.quantize(x)
    assert scales[:, 0].tolist() == [0, 0, 255, 255, 0]
    v = mx.values(codes, scales)
    assert not v[:2].any() and np.isnan(v[2:4]).all() and v[4, 1] == 3 * 2.0 ** -128


def test_rounding_is_the_nearest_by_search_and_odd():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 70)) * np.exp(rng.standard_normal((50, 1)))
    v, s = mx.rounded(x), mx.scale_bytes(x)
    scale = np.repeat(2.0 ** (s.astype(float) - 127), 32, axis=1)[:, :70]
    grid = np.concatenate([-mx.GRID, mx.GRID])
    best = np.abs(x[..., None] - grid * scale[..., None]).min(axis=-1)
    assert np.allclose(np.abs(x - v), best, rtol=0, atol=0)
    assert np.array_equal(mx.rounded(-x), -v)
    assert np.array_equal(mx.rounded(v), v)             # numbers on the grid stay
    assert np.array_equal(mx.rounded(4 * x), 4 * v)     # powers of two pass through


def test_ffn_is_the_layers_on_rounded_operands_when_h_is_on_the_grid():
    # up = 0: h = 0, y = 0; and with h already representable the rounding in between changes nothing
    rng = np.random.default_rng(2)
    w = {n: rng.standard_normal(s) for n, s in (("gate", (64, 32)), ("up", (64, 32)), ("down", (32, 64)))}
    q = mx.expert_values(w)
    x = mx.rounded(rng.standard_normal((3, 64)))
    assert not mx.swiglu_ffn(x, q["gate"], 0 * q["up"], q["down"]).any()
    h = orc.silu(x @ q["gate"]) * (x @ q["up"])
    assert np.allclose(mx.swiglu_ffn(x, q["gate"], q["up"], q["down"]), mx.rounded(h) @ q["down"], rtol=1e-14)
    err = np.abs(mx.rounded(h) - h).reshape(3, 1, 32).max(axis=2) / np.abs(h).reshape(3, 1, 32).max(axis=2)
    assert (err <= 0.25 + 1e-12).all()                  # half a step at the top, or a saturated 8 - 6 of 8


def test_biased_gate():
    s = np.array([[0.5, 0.4, 0.3, 0.2]])
    count = np.array([1, 1, 0, 1])
    assert orc.select_topk(mx.biased_keys(s, np.zeros(4), count), 2).tolist() == [[0, 1]]
    top = orc.select_topk(mx.biased_keys(s, np.array([0, -0.3, 1, 0.2]), count), 2)
    assert top.tolist() == [[0, 3]]                     # expert 2 is lost whatever its bias
    assert np.allclose(mx.biased_weights(s, top, True), [[0.5 / 0.7, 0.2 / 0.7]])
    assert np.allclose(mx.biased_weights(s, top, False, 2.5), [[1.25, 0.5]])
    # a bias that is the same for all changes nothing
    assert orc.select_topk(mx.biased_keys(s, np.full(4, 7.0), count), 2).tolist() == [[0, 1]]
