"""Every scale byte with every code, widened and multiplied: 2^(byte - 127), and NaN for 255, as the E8M0 format has it."""
import numpy as np
import pytest

from gpu_util import dev_i32, host_f64
from oracle import regione_oracle as orc
from paper_2510_25590_b200 import binding

pytestmark = pytest.mark.gpu


def _rows(bytes_):
    """A row of 128 elements per scale byte: every code in each of its four blocks."""
    code = np.tile(np.arange(16, dtype=np.uint8), 8)
    codes = np.tile(code[0::2] | (code[1::2] << 4), (len(bytes_), 1))
    return codes, np.repeat(np.asarray(bytes_, np.uint8)[:, None], 4, 1)


def test_widened():
    import torch
    codes, scales = _rows(np.arange(256))
    back = torch.empty((1, 256, 128), dtype=torch.bfloat16, device="cuda")
    binding.mxfp4_dequantize(torch.from_numpy(codes).cuda()[None], torch.from_numpy(scales).cuda()[None], back)
    want = orc.mxfp4_dequantize(codes, scales)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)        # (beyond bf16)
    assert np.array_equal(host_f64(back)[0], want, equal_nan=True) and np.isnan(want[255]).all() and not np.isnan(want[:255]).any()


def test_multiplied():
    """Rows times the unit vectors: one element of each row comes out, exactly; NaN scales make their rows NaN and no other."""
    import torch
    bytes_ = [2, 20, 126, 127, 128, 200, 250, 255, 127, 255, 60]
    codes, scales = _rows(bytes_)
    w = np.zeros((1, 16, 128), np.float32)
    w[0, np.arange(16), np.arange(16)] = 1.0                                             # (the first block's sixteen codes)
    out = torch.empty((len(bytes_), 16), dtype=torch.bfloat16, device="cuda")
    wq, ws = (torch.from_numpy(a).cuda() for a in orc.mxfp4_quantize(w))
    binding.mxfp4_grouped_matmul(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), wq, ws, dev_i32([0]), dev_i32([len(bytes_)]), out)
    assert np.array_equal(host_f64(out), orc.mxfp4_dequantize(codes, scales)[:, :16], equal_nan=True)
