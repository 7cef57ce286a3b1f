"""GPU parity of the products of ragged groups of rows, in bf16 and in the 4-bit format.

Small whole numbers make every product and every sum exact in fp32, whatever the order of the additions, so those outputs have to be
the correctly rounded ones, bit for bit.  With other numbers the bound is half a bf16 step of the result, 2^-8 |y|, plus K additions
that each lose at most 2^-23 of the sum of magnitudes."""
import numpy as np
import pytest

from gpu_util import dev_bf16, dev_i32, host_f64
from oracle import regione_oracle as orc
from paper_2510_25590_b200 import binding, synth

pytestmark = pytest.mark.gpu

OLD = -3.0


def _whole(rng, shape, top=4):
    return rng.integers(-top, top + 1, shape).astype(np.float32)


def _dev_codes(x):
    import torch
    c, s = orc.mxfp4_quantize(x)
    return torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()


def _run(fp4, x, w, begin, end, bias=None, gelu=False, status=0, stream=None):
    import torch
    out = torch.full((x.shape[0], w.shape[1]), OLD, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    act = binding.ACT_GELU_TANH if gelu else binding.ACT_NONE
    b = None if bias is None else dev_bf16(bias)
    if fp4:
        xq, xs = _dev_codes(x); wq, ws = _dev_codes(w)
        binding.mxfp4_grouped_matmul(xq, xs, wq, ws, dev_i32(begin), dev_i32(end), out, bias=b, activation=act, dev_status=st)
    else:
        binding.grouped_matmul(dev_bf16(x), dev_bf16(w), dev_i32(begin), dev_i32(end), out, bias=b, activation=act, dev_status=st)
    torch.cuda.synchronize()
    assert int(st[0]) == status
    return host_f64(out)


def _whole_case(fp4, begin, end, rows, sets, K, N, seed=0):
    rng = np.random.default_rng(seed)
    x, w = _whole(rng, (rows, K)), _whole(rng, (sets, N, K))
    if fp4:                                                            # (5 has no code; blocks of other scales: still whole numbers)
        x[np.abs(x) == 5] = 6
        x.reshape(-1, 32)[::3] *= 8; w.reshape(-1, 32)[::5] *= 4
    bias = _whole(rng, (sets, N), 16)
    want = np.full((rows, N), OLD)
    for g, (b, e) in enumerate(zip(begin, end)):
        want[b:e] = synth.bf16_round((x[b:e].astype(np.float64) @ w[g % sets].T.astype(np.float64) + bias[g % sets]).astype(np.float32))
    return x, w, bias, want


# few rows: the slices of K of a tile meet in a cluster
FEW = [([0], [1], 1, 1, 128, 8), ([0], [1], 1, 1, 2048, 128), ([0, 1], [1, 2], 2, 2, 1024, 1000), ([0], [17], 17, 1, 640, 264),
       ([0], [100], 100, 1, 4096, 128), ([0, 40], [33, 77], 80, 2, 896, 520), ([3], [50], 64, 1, 8192, 16),
       ([0, 5, 5, 9], [5, 5, 9, 9], 12, 4, 384, 136)]
# many: pairs of CTAs
MANY = [([0], [700], 700, 1, 512, 2048), ([0, 256], [256, 1075], 1300, 2, 1024, 1544), ([0], [2049], 2049, 1, 256, 1000),
        ([0, 600, 1300, 1900], [600, 1200, 1900, 2333], 2400, 2, 384, 768)]


# the slices of K of a pair's tiles meet, also over several rounds of tiles (groups far from alike)
SLICED = [([0], [640], 640, 1, 4096, 1024), ([0, 60, 70], [60, 70, 2000], 2000, 3, 8192, 264), ([0, 10], [10, 4000], 4000, 2, 4224, 136),
          ([0, 1, 2, 3, 4, 5, 6, 7], [1, 2, 3, 4, 5, 6, 7, 3000], 3000, 8, 2176, 72)]


@pytest.mark.parametrize("case", FEW + MANY + SLICED, ids=lambda c: f"{c[2]}x{c[4]}x{c[5]}g{len(c[0])}")
@pytest.mark.parametrize("fp4", [False, True], ids=["bf16", "mxfp4"])
def test_whole_numbers_are_exact(fp4, case):
    begin, end, rows, sets, K, N = case
    x, w, bias, want = _whole_case(fp4, begin, end, rows, sets, K, N)
    assert np.array_equal(_run(fp4, x, w, begin, end, bias), want)
