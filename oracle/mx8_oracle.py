"""CPU oracle of the 8-bit form of the layer (TEST INFRASTRUCTURE ONLY): microscaled 8-bit floats, the residual norm, the product
with its epilogue and the expert FFN on them, in fp64 numpy.

Microscaled floats (the OCP formats' MXFP8 with E4M3 elements): blocks of 32 numbers along a row, a scale 2^e per block with e the
smallest for which the largest magnitude is at most 448 * 2^e, at least -127, numbers as x / 2^e rounded to the nearest of GRID,
ties to the even index.  A block with an infinity or a NaN stands for NaNs (scale byte 255); zeros have scale byte 0.
"""
from __future__ import annotations

from math import erfc
from typing import Dict, Tuple

import numpy as np

from . import revive_oracle as orc
from .mx_oracle import BLOCK, blocks

# code c: exponent field c >> 3, mantissa c & 7; field 0 counts in steps of 2^-9; 127 is NaN
GRID = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])
_erfc = np.vectorize(erfc, otypes=[np.float64])


def scale_bytes(x: np.ndarray) -> np.ndarray:
    """uint8 [rows, n]: exponent + 127 of every block's scale, 255 for a block that is not all finite."""
    largest = np.abs(blocks(x)).max(axis=2)
    finite = np.isfinite(largest)
    safe = np.where(finite, largest, 0.0)
    e = np.maximum(np.ceil(np.log2(np.maximum(safe, 2.0 ** -140) / 448)), -127)  # the logarithm may be off by its last bit
    e = np.where(safe > 448 * np.exp2(e), e + 1, e)
    e = np.where((e > -127) & (safe <= 448 * np.exp2(e - 1)), e - 1, e)
    return np.where(finite, e + 127, 255).astype(np.uint8)


def codes_for(x: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """uint8 [rows, n, 32]: codes of x under given scale bytes (127, a NaN, in blocks of byte 255)."""
    b = blocks(x)
    with np.errstate(invalid="ignore", over="ignore"):
        a = np.abs(b) / np.exp2(scales.astype(np.float64) - 127)[:, :, None]
    a = np.where((scales == 255)[:, :, None], 0.0, a)
    middle = (GRID[1:] + GRID[:-1]) / 2
    low, high = np.searchsorted(middle, a, side="left"), np.searchsorted(middle, a, side="right")  # they differ on a midpoint
    code = np.where(low % 2 == 0, low, high)
    return np.where((scales == 255)[:, :, None], 127, code + 128 * np.signbit(b)).astype(np.uint8)


def quantize(x: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """(codes [rows, 32 n], scale bytes [rows, n])."""
    s = scale_bytes(x)
    return codes_for(x, s).reshape(len(s), -1), s


def grid_values(codes: np.ndarray) -> np.ndarray:
    """What codes are in units of their scale (127 and 255: NaN)."""
    table = np.append(GRID, np.nan)
    return np.where(codes >= 128, -table[codes & 127], table[codes & 127])


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """fp64 [rows, 32 n]: what codes and scale bytes stand for."""
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (grid_values(codes).reshape(*scales.shape, BLOCK) * s[:, :, None]).reshape(codes.shape)


def rounded(x: np.ndarray) -> np.ndarray:
    """x [rows, K] as its microscaled form stands for it."""
    return values(*quantize(x))[:, :np.shape(x)[1]]


def rms_norm(s: np.ndarray, weight: np.ndarray, eps: float) -> np.ndarray:
    """s / sqrt(mean(s^2) + eps) * weight along the rows."""
    s = np.asarray(s, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        return s / np.sqrt(np.mean(s * s, axis=1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)


def activated(z: np.ndarray, activation: str) -> np.ndarray:
    if activation == "relu":
        return np.where(z < 0, 0.0, z)
    if activation == "silu":
        return orc.silu(z)
    return 0.5 * z * _erfc(-z / np.sqrt(2.0)) if activation == "gelu" else z


def swiglu_ffn(v: np.ndarray, gate: np.ndarray, up: np.ndarray, down: np.ndarray) -> np.ndarray:
    """Q(silu(v @ gate) * (v @ up)) @ down on matrices that are values of microscaled numbers already."""
    return rounded(orc.silu(v @ gate) * (v @ up)) @ down


def expert_values(w: Dict[str, np.ndarray]) -> Dict[str, np.ndarray]:
    """Math-layout matrices (gate, up [H, I], down [I, H]) rounded along the K of their product."""
    return {n: rounded(np.asarray(m).T).T for n, m in w.items()}
