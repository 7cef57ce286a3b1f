"""Pins of the oracle's 4-bit format and of its grouped product that are not their own formulas (CPU only)."""
import numpy as np
import pytest

from oracle import regione_oracle as orc


def _values():
    return np.concatenate([orc.E2M1, -orc.E2M1])


def test_every_value_of_the_format_is_its_own_code():
    v = np.concatenate([_values(), _values()])                         # 32 elements with maximum 6: k = 0
    codes, scales = orc.mxfp4_quantize(v)
    assert scales.tolist() == [127]
    nibbles = np.stack([codes & 15, codes >> 4], -1).reshape(-1)
    assert np.array_equal(nibbles[1:8], np.arange(1, 8)) and np.array_equal(nibbles[9:16], np.arange(9, 16))
    assert np.array_equal(orc.mxfp4_dequantize(codes, scales), v)


@pytest.mark.parametrize("x,want", [(0.25, 0.0), (0.75, 1.0), (1.25, 1.0), (1.75, 2.0), (2.5, 2.0), (3.5, 4.0), (5.0, 4.0),
                                    (0.26, 0.5), (4.99, 4.0), (5.01, 6.0)])
def test_ties_go_to_the_even_code(x, want):
    t = np.zeros(32)
    t[0], t[1], t[2] = 6.0, x, -x
    assert orc.mxfp4_dequantize(*orc.mxfp4_quantize(t))[:3].tolist() == [6.0, want, -want]


@pytest.mark.parametrize("top,k", [(6.0, 0), (6.03125, 1), (3.0, -1), (3.015625, 0), (0.0, 0), (2.0 ** -133, -127), (12.0 * 2.0 ** 100, 101)])
def test_scale_is_the_smallest_that_covers(top, k):
    t = np.zeros(32)
    t[17] = -top
    codes, scales = orc.mxfp4_quantize(t)
    assert int(scales[0]) - 127 == k
    if k > -127 and top:
        got = orc.mxfp4_dequantize(codes, scales)
        assert abs(got[17] + top) <= top / 6.0                         # never saturates: half of the widest step, 1 of 6


def test_relative_error_of_a_block_is_at_most_half_a_step():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((64, 256))
    d = np.abs(orc.mxfp4_dequantize(*orc.mxfp4_quantize(x)) - x).reshape(64, -1, 32)
    s = 2.0 ** (orc.mxfp4_quantize(x)[1] - 127.0)[..., None]
    a = np.abs(x).reshape(64, -1, 32) / s
    half = np.where(a < 2, 0.25, np.where(a < 4, 0.5, 1.0)) * s
    assert np.all(d <= half)


def test_grouped_product_against_numpy_and_untouched_rows():
    rng = np.random.default_rng(1)
    x, w, bias = rng.standard_normal((11, 24)), rng.standard_normal((2, 16, 24)), rng.standard_normal((2, 16))
    begin, end, old = [0, 4, 4, 9], [3, 4, 8, 11], np.full((11, 16), 7.0)
    got = orc.grouped_matmul(x, w, begin, end, old, bias)
    assert np.allclose(got[0:3], x[0:3] @ w[0].T + bias[0]) and np.allclose(got[4:8], x[4:8] @ w[0].T + bias[0])
    assert np.allclose(got[9:11], x[9:11] @ w[1].T + bias[1])
    assert np.all(got[[3, 8]] == 7.0)
    y = np.linspace(-6, 6, 25)
    g = orc.grouped_matmul(y[:, None], np.ones((1, 1, 1)), [0], [25], np.zeros((25, 1)), gelu=True)[:, 0]
    assert g[12] == 0.0 and abs(g[-1] - 6.0) < 1e-8 and np.allclose(g - g[::-1], y)      # gelu(y) - gelu(-y) = y
