"""The oracle of the 8-bit form of the layer, pinned by closed forms, by search and by torch's own 8-bit floats."""
import numpy as np
import pytest
import torch

from oracle import mx8_oracle as mx


def test_grid_is_the_8_bit_floats():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(mx.grid_values(codes.numpy()), want, equal_nan=True)
    assert mx.GRID[-1] == 448 and mx.GRID[1] == 2.0 ** -9 and mx.GRID[8] == 2.0 ** -6


def test_hand_worked_block():
    # largest 448 -> scale 1; midpoints go to the even code
    x = np.zeros((1, 32))
    x[0, :10] = [448, 1.0625, 1.1875, 1.07, -17, 19, 2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -9, 430]
    codes, scales = mx.quantize(x)
    assert scales.tolist() == [[127]]
    assert mx.values(codes, scales)[0, :10].tolist() == [448, 1.0, 1.25, 1.125, -16, 20, 0, 2.0 ** -8, -2.0 ** -9, 416]


@pytest.mark.parametrize("exponent", [-118, -30, 0, 5, 127])
def test_scale_is_the_smallest_that_holds_the_largest(exponent):
    rng = np.random.default_rng(0)
    for largest, byte in ((1.0, 119), (1.75, 119), (np.nextafter(1.75, 2), 120), (1.999, 120)):
        x = rng.uniform(-1, 1, (1, 32))
        x[0, 3] = largest
        assert int(mx.scale_bytes(x * 2.0 ** exponent)[0, 0]) == max(exponent + byte, 0)


def test_zeros_tiny_and_not_finite_blocks():
    x = np.zeros((5, 32))
    x[1, 4] = 2.0 ** -140
    x[2, 0] = np.inf
    x[3, 31] = np.nan
    x[4, 1] = 3 * 2.0 ** -136
    codes, scales = mx.quantize(x)
    assert scales[:, 0].tolist() == [0, 0, 255, 255, 0]
    v = mx.values(codes, scales)
    assert not v[:2].any() and np.isnan(v[2:4]).all() and v[4, 1] == 3 * 2.0 ** -136


def test_rounding_is_the_nearest_by_search_and_odd():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((20, 70)) * np.exp(rng.standard_normal((20, 1)))
    v, s = mx.rounded(x), mx.scale_bytes(x)
    scale = np.repeat(2.0 ** (s.astype(float) - 127), 32, axis=1)[:, :70]
    grid = np.concatenate([-mx.GRID, mx.GRID])
    best = np.abs(x[..., None] - grid * scale[..., None]).min(axis=-1)
    assert np.array_equal(np.abs(x - v), best)
    # half a step, of a number of its binade or below the smallest one: nothing is cut off
    assert (np.abs(x - v) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * scale)).all()
    assert np.array_equal(mx.rounded(-x), -v) and np.array_equal(mx.rounded(v), v) and np.array_equal(mx.rounded(4 * x), 4 * v)


def test_norm_and_activations_by_torch():
    rng = np.random.default_rng(2)
    s, w = rng.standard_normal((5, 37)), rng.standard_normal(37)
    want = torch.nn.functional.rms_norm(torch.from_numpy(s), (37,), torch.from_numpy(w), 1e-3).numpy()
    assert np.allclose(mx.rms_norm(s, w, 1e-3), want, rtol=1e-13)
    z = np.linspace(-9, 9, 181)
    for name, f in (("relu", torch.relu), ("silu", torch.nn.functional.silu), ("gelu", torch.nn.functional.gelu), ("none", lambda v: v)):
        assert np.allclose(mx.activated(z, name), f(torch.from_numpy(z)).numpy(), rtol=1e-12, atol=1e-15)


def test_ffn_of_a_rounded_h_is_the_plain_one():
    rng = np.random.default_rng(3)
    w = {n: rng.standard_normal(s) for n, s in (("gate", (64, 32)), ("up", (64, 32)), ("down", (32, 64)))}
    q = mx.expert_values(w)
    x = mx.rounded(rng.standard_normal((3, 64)))
    assert not mx.swiglu_ffn(x, q["gate"], 0 * q["up"], q["down"]).any()
    g, u = x @ q["gate"], x @ q["up"]
    h = mx.rounded(g / (1 + np.exp(-g)) * u)
    assert np.allclose(mx.swiglu_ffn(x, q["gate"], q["up"], q["down"]), h @ q["down"], rtol=1e-12)
