"""CPU oracle of the 4-bit form of the layer (TEST INFRASTRUCTURE ONLY): microscaled 4-bit floats, the expert FFN on them
and the gate with a balance bias, in fp64 numpy.

Microscaled floats (the OCP formats' MXFP4): blocks of 32 numbers along a row, a scale 2^e per block with e =
floor(log2(largest magnitude)) - 2 held to -127..127, numbers as x / 2^e rounded to the nearest of GRID, ties to the even
index, at most 6.  A block with an infinity or a NaN stands for NaNs (scale byte 255); zeros have scale byte 0.
"""
from __future__ import annotations

from typing import Dict, Tuple

import numpy as np

from . import revive_oracle as orc

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def blocks(x: np.ndarray) -> np.ndarray:
    """[rows, K] -> [rows, ceil(K / 32), 32] in fp64, the last block filled up with zeros."""
    x = np.asarray(x, dtype=np.float64)
    rows, K = x.shape
    n = -(-K // BLOCK)
    out = np.zeros((rows, n * BLOCK))
    out[:, :K] = x
    return out.reshape(rows, n, BLOCK)


def scale_bytes(x: np.ndarray) -> np.ndarray:
    """uint8 [rows, n]: exponent + 127 of every block's scale, 255 for a block that is not all finite."""
    largest = np.abs(blocks(x)).max(axis=2)
    finite = np.isfinite(largest)
    floor_log2 = np.frexp(np.where(finite, largest, 1.0))[1] - 1      # largest = m 2^e with m in [0.5, 1)
    e = np.clip(np.where(largest == 0, -200, floor_log2) - 2, -127, 127)
    return np.where(finite, e + 127, 255).astype(np.uint8)


def codes_for(x: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """uint8 [rows, n, 32]: codes of x under given scale bytes (0 in blocks of byte 255)."""
    b = blocks(x)
    with np.errstate(invalid="ignore"):
        a = np.abs(b) / np.exp2(scales.astype(np.float64) - 127)[:, :, None]
    a = np.where((scales == 255)[:, :, None], 0.0, a)
    distance = np.abs(a[..., None] - GRID)
    nearest = distance.min(axis=-1, keepdims=True)
    hit = distance == nearest                                         # two where a is a midpoint
    even = np.arange(8) % 2 == 0
    code = np.where((hit & even).any(axis=-1), np.argmax(hit & even, axis=-1), np.argmax(hit, axis=-1))
    return (code + 8 * np.signbit(b)).astype(np.uint8)


def quantize(x: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """(bytes of two codes [rows, 16 n], the lower k in the lower half; scale bytes [rows, n])."""
    s = scale_bytes(x)
    c = codes_for(x, s).reshape(len(s), -1)
    return c[:, 0::2] | (c[:, 1::2] << 4), s


def values(packed: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """fp64 [rows, 32 n]: what codes and scale bytes stand for."""
    c = np.stack([packed & 15, packed >> 4], axis=2).reshape(len(packed), -1)
    v = np.where(c >= 8, -GRID[c & 7], GRID[c & 7]).reshape(*scales.shape, BLOCK)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (v * s[:, :, None]).reshape(len(packed), -1)


def rounded(x: np.ndarray) -> np.ndarray:
    """x [rows, K] as its microscaled form stands for it."""
    return values(*quantize(x))[:, :np.shape(x)[1]]


def swiglu_ffn(v: np.ndarray, gate: np.ndarray, up: np.ndarray, down: np.ndarray) -> np.ndarray:
    """Q(silu(v @ gate) * (v @ up)) @ down on matrices that are values of microscaled numbers already."""
    return rounded(orc.silu(v @ gate) * (v @ up)) @ down


def expert_values(w: Dict[str, np.ndarray]) -> Dict[str, np.ndarray]:
    """Math-layout matrices (gate, up [H, I], down [I, H]) rounded along the K of their product."""
    return {n: rounded(np.asarray(m).T).T for n, m in w.items()}


def biased_keys(s: np.ndarray, bias: np.ndarray, l2p_count: np.ndarray) -> np.ndarray:
    """Selection keys of the gate with a balance bias: score + bias, -inf for an expert with no replica left."""
    return orc.masked_selection_scores(s + np.asarray(bias, dtype=np.float64)[None, :], l2p_count)


def biased_weights(s: np.ndarray, topk_logical: np.ndarray, renormalise: bool, route_scale: float = 1.0) -> np.ndarray:
    """The chosen experts' scores without the bias, over their sum or as they are, times route_scale."""
    if renormalise:
        return orc.gate_weights(s, topk_logical, route_scale)
    return np.take_along_axis(s, topk_logical.astype(np.int64), axis=1) * route_scale
