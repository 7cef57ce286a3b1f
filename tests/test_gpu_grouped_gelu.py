"""GELU of the grouped products over the whole range of bf16, infinities and NaN among ordinary rows.

A sum is one product, x[r, 0] * 1, so that it is exact.  Bound: half a bf16 step, 2^-8 |want|.  In front of it, in fp32: the exponent of
exp(-2 u) is at most 128 and off by at most 8 * 2^-24 of itself (3 roundings in the constant, 2 in the cubic term's, the square, the
sum, the product), so that its power is off by at most 128 ln 2 * 2^-21 < 2^-14.5; the power itself, the sum, the reciprocal and three
products 2^-20 in all: 2^-14 |want|.  And 2^-122: the factor is 0 where 1 + exp(-2 u) is beyond 2^126, from |y| = 10.1 on (10.1 * 2^-126)."""
import numpy as np
import pytest

from gpu_util import dev_bf16, dev_i32, host_f64
from oracle import regione_oracle as orc
from paper_2510_25590_b200 import binding, synth

pytestmark = pytest.mark.gpu

SPECIAL = [-np.inf, np.inf, np.nan, -3.3895314e38, 3.3895314e38, -3e38, -1e30, -1e20, -1e18, -1e10, -1e4, -100.0, -20.0, -12.0, -10.1, -10.0, -9.9,
           -9.0, -8.0, -7.5, -7.3, -7.0, -6.0, -5.0, -3.0, -1.0, -1e-3, -1e-30, -0.0, 0.0, 1e-30, 1e-3, 0.5, 3.0, 7.5, 10.0, 20.0, 1e10, 1e30]


def _check(y, got):
    """y [rows], got [rows, N]"""
    with np.errstate(all="ignore"):
        y = y.astype(np.float64)
        want = y / (1.0 + np.exp(-2.0 * np.sqrt(2.0 / np.pi) * (y + 0.044715 * y ** 3)))
    for column in got.T:
        assert np.array_equal(np.isnan(column), np.isnan(want))
        assert np.array_equal(column == np.inf, want == np.inf) and not np.any(column == -np.inf)
        fin = np.isfinite(want)
        assert np.all(np.abs(column[fin] - want[fin]) <= (2.0 ** -8 + 2.0 ** -14) * np.abs(want[fin]) + 2.0 ** -122)


def _call(y, K, N):
    import torch
    x = torch.zeros((len(y), K), dtype=torch.bfloat16, device="cuda")
    x[:, 0] = dev_bf16(y)
    w = torch.zeros((1, N, K), dtype=torch.bfloat16, device="cuda")
    w[:, :, 0] = 1.0
    out = torch.empty((len(y), N), dtype=torch.bfloat16, device="cuda")
    binding.grouped_matmul(x, w, dev_i32([0]), dev_i32([len(y)]), out, activation=binding.ACT_GELU_TANH)
    return host_f64(out)


@pytest.mark.parametrize("N", [8, 520])
def test_every_bf16_value(N):
    """Shuffled: a value shares its reciprocal with any other."""
    bits = np.random.default_rng(N).permutation(2 ** 16).astype(np.uint16)
    y = synth.bf16_bits_to_f32(bits)
    _check(y, _call(y, 16, N)[:, [0, 1, N - 1]])


# a tile of lone CTAs; slices of K that meet in a cluster; pairs, whole and in slices
@pytest.mark.parametrize("copies,K,N", [(1, 64, 8), (1, 4096, 8), (20, 64, 2048), (40, 4096, 264)])
def test_special_values_beside_each_other(copies, K, N):
    y = synth.bf16_round(np.array(SPECIAL * copies, np.float32))
    np.random.default_rng(copies).shuffle(y)
    _check(y, _call(y, K, N)[:, [0, N - 1]])


@pytest.mark.parametrize("copies,K,N", [(1, 128, 8), (30, 128, 2048), (40, 8192, 264)])
def test_4_bit_products(copies, K, N):
    """One element of a row is not zero, -6 to 6 times 2^k with k up to 124."""
    import torch
    k = np.array([-100, -60, -20, -5, -3, -2, -1, 0, 1, 2, 5, 20, 60, 100, 124])
    y = (np.array([-6.0, -4.0, -3.0, -1.0, -0.5, 0.0, 2.0, 6.0])[:, None] * np.exp2(k)).astype(np.float32).ravel()
    y = np.tile(y, copies)
    np.random.default_rng(copies).shuffle(y)
    x, w = np.zeros((len(y), K), np.float32), np.zeros((1, N, K), np.float32)
    x[:, 0], w[:, :, 0] = y, 1.0
    dev = lambda a: [torch.from_numpy(v).cuda() for v in orc.mxfp4_quantize(a)]
    out = torch.empty((len(y), N), dtype=torch.bfloat16, device="cuda")
    binding.mxfp4_grouped_matmul(*dev(x), *dev(w), dev_i32([0]), dev_i32([len(y)]), out, activation=binding.ACT_GELU_TANH)
    _check(y, host_f64(out)[:, [0, N - 1]])
