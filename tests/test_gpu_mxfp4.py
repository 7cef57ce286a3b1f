"""GPU parity of the 4-bit microscaled format: codes, scales and widened rows bit-exact against the oracle."""
import numpy as np
import pytest

from gpu_util import dev_bf16, dev_i32, host_f64
from oracle import regione_oracle as orc
from paper_2510_25590_b200 import binding, synth

pytestmark = pytest.mark.gpu


def _rand(rng, shape):
    """bf16 rows of very different size, with zeros, ties and the ends of the scale's range among their blocks."""
    x = rng.standard_normal(shape).astype(np.float32) * np.exp2(rng.integers(-20, 20, shape[:-1] + (1,))).astype(np.float32)
    x = synth.bf16_round(x).reshape(-1, 32)
    x[0] = 0.0
    if len(x) > 6:
        x[1, :10] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0, -0.25]
        x[1, 10:] = 0.0
        x[2] = 0.0; x[2, 3] = 2.0 ** -133                            # smallest bf16 subnormal: the scale's floor
        x[3] = 0.0; x[3, 0], x[3, 1] = 255.0 * 2.0 ** 120, -(2.0 ** 127)   # largest finite bf16
        x[4] *= np.float32(0.0); x[4, 31] = 12.0 * 2.0 ** -127
        x[5, :] = synth.bf16_round(np.float32(6.03125))
    return x.reshape(shape)


def _same_codes(got, want):
    """Equal codes; +0 and -0 are one value."""
    a = np.stack([got & 15, got >> 4], -1); b = np.stack([want & 15, want >> 4], -1)
    return np.all((a == b) | (((a & 7) == 0) & ((b & 7) == 0)))


def _widened(codes, scales):
    """The format's values as bf16 holds them: exactly, except that 4 * 2^126 (the largest finite bf16 is rounded up to it) is
    beyond bf16 and becomes infinite."""
    v = orc.mxfp4_dequantize(codes, scales)
    return np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)


@pytest.mark.parametrize("B,rows,K", [(1, 1, 32), (1, 3, 64), (2, 5, 96), (1, 7, 1024), (3, 33, 1056), (1, 130, 2080), (2, 9, 8192)])
def test_all_rows(B, rows, K):
    import torch
    x = _rand(np.random.default_rng(B * 1000 + rows + K), (B, rows, K))
    codes = torch.full((B, rows, K // 2), 0x5a, dtype=torch.uint8, device="cuda")
    scales = torch.full((B, rows, K // 32), 0x5a, dtype=torch.uint8, device="cuda")
    back = torch.full((B, rows, K), -3.0, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.mxfp4_quantize(dev_bf16(x), codes, scales, dev_status=st)
    binding.mxfp4_dequantize(codes, scales, back, dev_status=st)
    want_c, want_s = orc.mxfp4_quantize(x)
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert _same_codes(codes.cpu().numpy(), want_c)
    assert np.array_equal(host_f64(back), _widened(want_c, want_s))
    assert int(st[0]) == 0


@pytest.mark.parametrize("K", [32, 96, 2048, 1184])
def test_gathered_rows_with_counts(K):
    import torch
    rng = np.random.default_rng(K)
    B, src, cap = 3, 50, 20
    x = _rand(rng, (B, src, K))
    idx = rng.integers(0, src, (B, cap)).astype(np.int32)             # (a row may be named twice)
    n = np.array([cap, 0, 7], np.int32)
    idx[2, 7:] = -5                                                    # behind the count: never looked at
    codes = torch.full((B, cap, K // 2), 0x5a, dtype=torch.uint8, device="cuda")
    scales = torch.full((B, cap, K // 32), 0x5a, dtype=torch.uint8, device="cuda")
    back = torch.full((B, cap, K), -3.0, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.mxfp4_quantize(dev_bf16(x), codes, scales, idx=dev_i32(idx), n=dev_i32(n), dev_status=st)
    binding.mxfp4_dequantize(codes, scales, back, n=dev_i32(n), dev_status=st)
    for b in range(B):
        c, s = orc.mxfp4_quantize(x[b][idx[b, :n[b]]])
        assert _same_codes(codes[b, :n[b]].cpu().numpy(), c) and np.array_equal(scales[b, :n[b]].cpu().numpy(), s)
        assert np.array_equal(host_f64(back)[b, :n[b]], _widened(c, s))
        assert np.all(codes[b, n[b]:].cpu().numpy() == 0x5a) and np.all(scales[b, n[b]:].cpu().numpy() == 0x5a)
        assert np.all(host_f64(back)[b, n[b]:] == -3.0)
    assert int(st[0]) == 0


def test_bad_indices_and_counts_are_recorded_and_skipped():
    import torch
    x = _rand(np.random.default_rng(3), (1, 8, 64))
    for idx, n in (([[0, 8, 2, 3]], [4]), ([[0, -1, 2, 3]], [4]), ([[0, 1, 2, 3]], [5]), ([[0, 1, 2, 3]], [-1])):
        codes = torch.full((1, 4, 32), 0x5a, dtype=torch.uint8, device="cuda")
        scales = torch.full((1, 4, 2), 0x5a, dtype=torch.uint8, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        binding.mxfp4_quantize(dev_bf16(x), codes, scales, idx=dev_i32(idx), n=dev_i32(n), dev_status=st)
        assert int(st[0]) == binding.DEV_BOUNDS
        c, s = orc.mxfp4_quantize(x[0])
        for j in range(4):
            live = j < min(n[0], 4) and 0 <= idx[0][j] < 8
            if live:
                assert _same_codes(codes[0, j].cpu().numpy(), c[j]) and np.array_equal(scales[0, j].cpu().numpy(), s[j])
            else:
                assert np.all(codes[0, j].cpu().numpy() == 0x5a)


def test_infinite_and_nan_elements_stay_in_their_block():
    import torch
    x = _rand(np.random.default_rng(4), (1, 9, 64))
    x[0, 7, 5], x[0, 7, 40] = np.inf, np.nan
    codes = torch.zeros((1, 9, 32), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((1, 9, 2), dtype=torch.uint8, device="cuda")
    binding.mxfp4_quantize(dev_bf16(x), codes, scales)
    y = x.copy(); y[0, 7, 5] = 255.0 * 2.0 ** 120; y[0, 7, 40] = 0.0
    c, s = orc.mxfp4_quantize(y)
    assert np.array_equal(scales.cpu().numpy(), s)
    got = codes.cpu().numpy()
    got[0, 7, 20] = (got[0, 7, 20] & 0xf0) | (c[0, 7, 20] & 15)        # the NaN element itself: any code
    got[0, 7, 2] = (got[0, 7, 2] & 0x0f) | (c[0, 7, 2] & 0xf0) if (got[0, 7, 2] >> 4) == 7 else 0xff
    assert _same_codes(got, c)


@pytest.mark.parametrize("H,D", [(3, 64), (5, 128), (24, 128)])
def test_cache_store_and_load(H, D):
    import torch
    rng = np.random.default_rng(H + D)
    B, N, cap = 2, 120, 90
    k, v = _rand(rng, (B, N, H, D)), _rand(rng, (B, N, H, D))
    keep = np.stack([np.sort(rng.permutation(N)[:cap]) for _ in range(B)]).astype(np.int32)
    n = np.array([cap, 31], np.int32)
    q = lambda d: torch.full((B, cap, H, D // d), 0x5a, dtype=torch.uint8, device="cuda")
    kq, vq, ks, vs = q(2), q(2), q(32), q(32)
    kc, vc = (torch.full((B, cap, H, D), -3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.rikv_store_mxfp4(dev_bf16(k), dev_bf16(v), dev_i32(keep), dev_i32(n), kq, vq, ks, vs, dev_status=st)
    binding.rikv_load_mxfp4(kq, vq, ks, vs, dev_i32(n), kc, vc, dev_status=st)
    for b in range(B):
        for full, codes, scales, cache in ((k, kq, ks, kc), (v, vq, vs, vc)):
            c, s = orc.mxfp4_quantize(full[b][keep[b, :n[b]]])
            assert _same_codes(codes[b, :n[b]].cpu().numpy(), c) and np.array_equal(scales[b, :n[b]].cpu().numpy(), s)
            assert np.array_equal(host_f64(cache)[b, :n[b]], _widened(c, s))
            assert np.all(host_f64(cache)[b, n[b]:] == -3.0) and np.all(codes[b, n[b]:].cpu().numpy() == 0x5a)
    assert int(st[0]) == 0
