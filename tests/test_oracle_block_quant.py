"""Pins of the oracle of 8-bit rows, weights and products: what the definitions say of cases that can be worked out by hand."""
import numpy as np
import pytest

from oracle import block_quant_oracle as B
from oracle.quant_cache_oracle import e4m3_decode


def test_scale_is_the_largest_over_448():
    y = np.zeros((1, 300))
    y[0, 5], y[0, 130], y[0, 299] = -3.5, 448.0, 1e-30
    codes, scale = B.quantise(y)
    assert scale.shape == (1, 3) and scale[0, 0] == 3.5 / 448 and scale[0, 1] == 1.0 and scale[0, 2] == 2.0 ** -60
    assert codes[0, 5] == 0xFE and codes[0, 130] == 0x7E and codes[0, 299] == 0          # -448, 448; 1e-30 / 2^-60 rounds to nothing
    assert B.dequantise(codes, scale)[0, 5] == -3.5


def test_weights_share_a_scale_in_both_directions():
    w = np.ones((200, 130))
    w[150, 3], w[10, 129] = 896.0, -448.0
    codes, scale = B.quantise(w, 128)
    assert scale.shape == (2, 2) and (scale == [[1 / 448, 1.0], [2.0, 1 / 448]]).all()
    back = B.dequantise(codes, scale, 128)
    assert back[150, 3] == 896 and back[10, 129] == -448 and back[0, 129] == 1 and back[199, 0] == 1 and back[199, 129] == 1


def test_what_is_not_finite():
    codes, scale = B.quantise(np.array([[np.inf, -np.inf, np.nan, 2.0]]))
    assert scale[0, 0] == 2 / 448 and codes.tolist() == [[0x7E, 0xFE, 0, 0x7E]]


@pytest.mark.parametrize("seed", [0, 1])
def test_a_code_is_within_half_a_step(seed):
    y = np.random.default_rng(seed).standard_normal((3, 144))
    codes, scale = B.quantise(y)
    x = y / np.repeat(scale, 128, axis=1)[:, :144]
    assert (np.abs(e4m3_decode(codes) - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10)).all()


def test_norm_of_equal_elements_and_of_a_residual():
    s, y = B.norm(np.full((1, 16), 3.0), np.full((1, 16), -5.0), np.arange(16.0), 0.0)
    assert (s == -2).all() and (y == -np.arange(16.0)).all()
    s, y = B.norm(np.zeros((1, 16)), None, np.ones(16), 1e-5)
    assert (s == 0).all() and (y == 0).all()


def test_gate():
    assert B.gated(np.array([2.0, 2.0, 2.0]), np.array([0.0, 1e4, -1e4])).tolist() == [0.0, 2e4, 0.0]


def test_product_by_its_blocks():
    rng = np.random.default_rng(3)
    a, w = B.quantise(rng.standard_normal((2, 160))), B.quantise(rng.standard_normal((130, 160)), 128)
    out, room = B.product(*a, *w)
    by_hand = sum(float(a[1][1, k // 128]) * float(w[1][1, k // 128]) * e4m3_decode(a[0])[1, k] * e4m3_decode(w[0])[129, k] for k in range(160))
    assert abs(out[1, 129] - by_hand) <= 1e-12 * room[1, 129] and (np.abs(out) <= room).all()
