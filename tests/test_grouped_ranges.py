"""What a grouped product takes of the ranges it is given: every pair of 32-bit numbers is cut to the buffer."""
import ctypes

import numpy as np
import pytest

from paper_2510_25590_b200 import binding

LOW, HIGH = -2 ** 31, 2 ** 31 - 1
CAPS = [0, 1, 40, 4096, 2 ** 24]


@pytest.mark.parametrize("cap", CAPS)
def test_ranges_are_cut_to_the_buffer(cap):
    """The function that the kernel runs, on the host, over the corners (Python's numbers do not wrap)."""
    near = {LOW, LOW + 1, LOW + cap, LOW + 2 * cap + 1, -cap - 1, -cap, -1, 0, 1, 9, 20, 200, 300, cap // 2, cap - 1, cap, cap + 1, HIGH - cap, HIGH - 1, HIGH}
    ends = sorted(v for v in near if LOW <= v <= HIGH)
    pairs = [(b, e) for b in ends for e in ends]
    b, e = (np.array(v, np.int32) for v in zip(*pairs))
    begin, rows = np.full(len(pairs), -9, np.int32), np.full(len(pairs), -9, np.int32)
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    outside = binding.load().regione_selftest_group_ranges(p(b), p(e), cap, len(pairs), p(begin), p(rows))
    cut = lambda v: min(max(v, 0), cap)
    assert outside == sum(not 0 <= b <= e <= cap for b, e in pairs)
    for at, (b, e) in enumerate(pairs):
        assert (begin[at], rows[at]) == (cut(b), max(cut(e) - cut(b), 0)), (b, e)


def test_refusals():
    f, fake = binding.load().regione_selftest_group_ranges, ctypes.c_void_p(4096)
    assert f(None, fake, 1, 1, fake, fake) == f(fake, None, 1, 1, fake, fake) == f(fake, fake, 1, 1, None, fake) == -1
    assert f(fake, fake, -1, 1, fake, fake) == f(fake, fake, 1, -1, fake, fake) == f(fake, fake, 1, 1, fake, None) == -1
    assert f(fake, fake, 1, 0, fake, fake) == 0


# ---- on the GPU: the ends of 32 bits beside groups whose rows have to come out ----------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("rows,K,N", [(400, 64, 24), (4000, 512, 1032)])     # CTAs of their own, pairs of CTAs
@pytest.mark.parametrize("fp4", [False, True], ids=["bf16", "mxfp4"])
def test_far_ends_beside_valid_groups(fp4, rows, K, N):
    import torch
    from gpu_util import dev_bf16, dev_i32, host_f64
    from oracle import regione_oracle as orc
    K *= 2 if fp4 else 1
    rng = np.random.default_rng(rows + fp4)
    x, w = (rng.integers(-4, 5, s).astype(np.float32) for s in ((rows, K), (1, N, K)))
    full = x.astype(np.float64) @ w[0].T.astype(np.float64)
    dev = (lambda a: tuple(torch.from_numpy(v).cuda() for v in orc.mxfp4_quantize(a))) if fp4 else lambda a: (dev_bf16(a),)
    dx, dw = dev(x), dev(w)
    call = binding.mxfp4_grouped_matmul if fp4 else binding.grouped_matmul
    third = rows // 3
    for b, e in ((20, LOW), (200, LOW), (rows // 2, LOW + 3), (rows, LOW), (1, LOW + rows), (HIGH, LOW), (9, -1), (HIGH, HIGH), (LOW, LOW)):
        out = torch.full((rows, N), -3.0, dtype=torch.bfloat16, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        call(*dx, *dw, dev_i32([0, b, 2 * third]), dev_i32([third, e, rows]), out, dev_status=st)
        want = np.full((rows, N), -3.0)
        want[:third], want[2 * third:] = full[:third], full[2 * third:]      # (sums below 2^14 need more than 8 bits: rounded below)
        assert np.array_equal(host_f64(out), host_f64(torch.from_numpy(want).float().to(torch.bfloat16)))
        assert int(st[0]) == binding.DEV_BOUNDS
