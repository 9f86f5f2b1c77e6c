"""CPU oracle of rows and weights in 8 bits with a scale for each 128 columns (128 x 128 elements of a weight), of the norm that makes such
rows, and of their product: numpy float64 from the definitions in include/vvs.h, plain loops over the blocks.  Nothing here is shared with
the CUDA path but e4m3 itself, which is the cache's oracle's.

No counterpart in the paper: there is nothing to be unpinned against.  Pins: tests/test_oracle_block_quant.py."""
from __future__ import annotations

import numpy as np

from oracle.quant_cache_oracle import E4M3_MAX, e4m3_decode, e4m3_encode

BLOCK = 128


def scale_of(block: np.ndarray) -> float:
    """Largest finite magnitude / 448, 2^-60 at least."""
    mag = np.abs(block[np.isfinite(block)])
    return max(float(mag.max()) / E4M3_MAX if mag.size else 0.0, 2.0 ** -60)


def quantise(y: np.ndarray, block_rows: int = 1):
    """y [rows, cols] -> (codes uint8, scale [ceil(rows / block_rows), ceil(cols / 128)]); block_rows 1: rows, 128: a weight."""
    y = np.asarray(y, dtype=np.float64)
    rows, cols = y.shape
    codes = np.zeros((rows, cols), np.uint8)
    scale = np.zeros((-(-rows // block_rows), -(-cols // BLOCK)))
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            at = np.s_[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK]
            scale[i, j] = scale_of(y[at])
            codes[at] = e4m3_encode(y[at] / scale[i, j])
    return codes, scale


def dequantise(codes: np.ndarray, scale: np.ndarray, block_rows: int = 1) -> np.ndarray:
    rows, cols = codes.shape
    out = e4m3_decode(codes)
    for i in range(rows):
        for j in range(scale.shape[1]):
            out[i, j * BLOCK:(j + 1) * BLOCK] *= float(scale[i // block_rows, j])
    return out


def norm(x: np.ndarray, residual: np.ndarray | None, weight: np.ndarray, eps: float):
    """(s, y): the sum, and the sum over its root mean square times the weight."""
    s = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    y = np.zeros_like(s)
    for i, row in enumerate(s):
        y[i] = row / np.sqrt(np.sum(row * row) / row.size + eps) * weight
    return s, y


def gated(x: np.ndarray, gate: np.ndarray) -> np.ndarray:
    gate = np.asarray(gate, np.float64)
    with np.errstate(over="ignore"):
        return gate / (1.0 + np.exp(-gate)) * x


def product(a_codes, a_scale, w_codes, w_scale):
    """(out, sum of magnitudes): [rows, outputs] in float64."""
    a, w = dequantise(a_codes, a_scale), dequantise(w_codes, w_scale, BLOCK)
    return a @ w.T, np.abs(a) @ np.abs(w).T
