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


def test_rows_on_16_bytes_only_and_captured():
    """A base that is not on 32 bytes takes the narrower loads; a captured call follows the counts."""
    import torch
    x = _rand(np.random.default_rng(5), (1, 40, 160))
    buf = torch.empty(8 + x.size, dtype=torch.bfloat16, device="cuda")
    dx = buf[8:].view(1, 40, 160)
    dx.copy_(dev_bf16(x))
    assert dx.data_ptr() % 32 == 16
    n = dev_i32([40])
    codes = torch.full((1, 40, 80), 0x5a, dtype=torch.uint8, device="cuda")
    scales = torch.full((1, 40, 5), 0x5a, dtype=torch.uint8, device="cuda")
    want_c, want_s = orc.mxfp4_quantize(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.mxfp4_quantize(dx, codes, scales, n=n)
        side.synchronize()
        assert _same_codes(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            binding.mxfp4_quantize(dx, codes, scales, n=n)
    codes.fill_(0x5a)
    n.fill_(17)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert _same_codes(codes[:, :17].cpu().numpy(), want_c[:, :17]) and bool((codes[:, 17:] == 0x5a).all())


def test_offsets_beyond_32_bits():
    import torch
    rows, K = 2_200_000, 1024
    x = torch.zeros((1, rows, K), dtype=torch.bfloat16, device="cuda")
    tail = _rand(np.random.default_rng(6), (1, 9, K))
    x[:, -9:] = dev_bf16(tail)
    codes = torch.empty((1, rows, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((1, rows, K // 32), dtype=torch.uint8, device="cuda")
    binding.mxfp4_quantize(x, codes, scales)
    c, s = orc.mxfp4_quantize(tail)
    assert _same_codes(codes[:, -9:].cpu().numpy(), c) and np.array_equal(scales[:, -9:].cpu().numpy(), s)
    idx = torch.arange(rows - 9, rows, dtype=torch.int32, device="cuda")[None]
    few = torch.empty((1, 9, K // 2), dtype=torch.uint8, device="cuda"), torch.empty((1, 9, K // 32), dtype=torch.uint8, device="cuda")
    binding.mxfp4_quantize(x, *few, idx=idx)
    assert torch.equal(few[0], codes[:, -9:]) and torch.equal(few[1], scales[:, -9:])
    binding.mxfp4_dequantize(codes, scales, x)
    assert np.array_equal(host_f64(x[:, -9:]), _widened(c, s))


def test_refusals_and_nothing_to_do():
    import torch
    t = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    u = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
    for x, c, s, kw in ((t(1, 4, 48), u(1, 4, 24), u(1, 4, 1), {}), (t(1, 4, 64), u(1, 4, 32), u(1, 4, 3), {}), (t(1, 4, 64), u(1, 5, 32), u(1, 5, 2), {}),
                        (t(1, 4, 64), u(1, 4, 32), u(1, 4, 2), dict(idx=dev_i32([[0, 1]]))), (t(1, 4, 128)[:, :, :64], u(1, 4, 32), u(1, 4, 2), {}),
                        (t(1, 4, 64).half(), u(1, 4, 32), u(1, 4, 2), {}), (t(1, 4, 64), u(1, 4, 32), u(1, 4, 2), dict(n=dev_i32([1, 2])))):
        with pytest.raises(binding.RegionEError):
            binding.mxfp4_quantize(x, c, s, **kw)
    before = binding.kernel_launches()
    binding.mxfp4_quantize(t(1, 0, 64), u(1, 0, 32), u(1, 0, 2))
    binding.mxfp4_dequantize(u(1, 0, 32), u(1, 0, 2), t(1, 0, 64))
    assert binding.kernel_launches() == before
