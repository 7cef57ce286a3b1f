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


# ---- other numbers -----------------------------------------------------------------------------------------------------
def _gelu(y):
    return 0.5 * y * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (y + 0.044715 * y ** 3)))


@pytest.mark.parametrize("fp4,rows,K,N", [(False, 37, 328, 72), (False, 900, 1000, 520), (True, 37, 384, 72), (True, 900, 1152, 520),
                                          (False, 3, 4096, 264), (True, 3, 4096, 264)])
@pytest.mark.parametrize("gelu", [False, True])
def test_normal_numbers(fp4, rows, K, N, gelu):
    rng = np.random.default_rng(rows + K)
    x, w = (synth.bf16_round(rng.standard_normal(s).astype(np.float32)) for s in ((rows, K), (1, N, K)))
    w = synth.bf16_round(w * np.float32(4 * K ** -0.5))                # sums of standard deviation 4: gelu's whole range
    bias = synth.bf16_round(rng.standard_normal((1, N)).astype(np.float32))
    got = _run(fp4, x, w, [0], [rows], bias, gelu)
    if fp4:
        x, w = orc.mxfp4_dequantize(*orc.mxfp4_quantize(x)), orc.mxfp4_dequantize(*orc.mxfp4_quantize(w))
    y = x.astype(np.float64) @ w[0].T.astype(np.float64) + bias[0]
    sums = np.abs(x.astype(np.float64)) @ np.abs(w[0].T.astype(np.float64)) + np.abs(bias[0])
    want = _gelu(y) if gelu else y
    # half a bf16 step, the additions, and with gelu (slope at most 1.13) six fp32 operations of at most 2^-20 each
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 1.13 * K * 2.0 ** -23 * sums + (6 * 2.0 ** -20 * np.abs(want) if gelu else 0)
                  + 1e-30)


def test_gelu_far_out():
    x = synth.bf16_round(np.array([[-1e4, -100, -20, -8, -7.3, -6, -3, -1e-3, -1e-30, 0, 1e-30, 1e-3, 3, 6, 8, 1e4, 3e38]], np.float32).T)
    x = np.concatenate([x, np.zeros((len(x), 7), np.float32)], 1)
    w = np.zeros((1, 8, 8), np.float32); w[0, :, 0] = 1.0
    got = _run(False, x, w, [0], [len(x)], None, True)
    # (y / 2 (1 + tanh u) cancels in 64 bits as well from -5 on: the same function as y / (1 + exp(-2 u)))
    y = x[:, :1].astype(np.float64)
    with np.errstate(over="ignore"):
        want = y / (1.0 + np.exp(-2.0 * np.sqrt(2.0 / np.pi) * (y + 0.044715 * y ** 3)))
    tiny = 2.0 ** -62 * np.abs(x[:, :1].astype(np.float64))            # what is kept of exp(-2 u) at most
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2 * tiny + 6 * 2.0 ** -20 * np.abs(want) + 2.0 ** -133)


# ---- which rows ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fp4", [False, True], ids=["bf16", "mxfp4"])
@pytest.mark.parametrize("rows", [24, 1500])
def test_rows_of_no_group_stay_and_do_not_leak(fp4, rows):
    """NaN and infinite rows between the groups, whose tiles reach over them."""
    q = rows // 8
    begin, end = [0, 2 * q, 3 * q, 6 * q], [q, 3 * q, 5 * q + 1, 8 * q - 3]
    K, N = 256, 136
    x, w, bias, want = _whole_case(False, begin, end, rows, 2, K, N, seed=rows)
    live = np.zeros(rows, bool)
    for b, e in zip(begin, end):
        live[b:e] = True
    bad = np.where(~live)[0]
    if not fp4:
        x[bad[::2]] = np.nan
        x[bad[1::2]] = np.inf
        assert np.array_equal(_run(False, x, w, begin, end, bias), want)
        return
    import torch
    xq, xs = _dev_codes(x)
    xs[torch.from_numpy(bad).cuda()] = 255                             # NaN scales
    wq, ws = _dev_codes(w)
    out = torch.full((rows, N), OLD, dtype=torch.bfloat16, device="cuda")
    binding.mxfp4_grouped_matmul(xq, xs, wq, ws, dev_i32(begin), dev_i32(end), out, bias=dev_bf16(bias))
    assert np.array_equal(host_f64(out), want)


@pytest.mark.parametrize("fp4", [False, True], ids=["bf16", "mxfp4"])
def test_many_groups_empty_and_uneven(fp4):
    rng = np.random.default_rng(11)
    for G, sets in ((512, 1), (300, 300), (64, 64)):
        count = rng.integers(0, 9, G) * (rng.random(G) < 0.6)
        count[G // 2] = 333
        end = np.cumsum(count); begin = end - count
        x, w, bias, want = _whole_case(fp4, begin, end, int(end[-1]) + 5, sets, 128, 40, seed=G)
        assert np.array_equal(_run(fp4, x, w, begin, end, bias), want)
    none = np.zeros(64, np.int64)
    assert np.all(_run(fp4, x, w, none, none, bias) == OLD)


def test_ranges_outside_the_buffer_are_cut_and_recorded():
    x, w, bias, _ = _whole_case(False, [0], [40], 40, 1, 64, 24)
    for begin, end in (([-3], [7]), ([30], [41]), ([9], [4]), ([2 ** 31 - 1], [2 ** 31 - 1]), ([-2 ** 31], [3])):
        want = np.full((40, 24), OLD)
        b, e = max(begin[0], 0), min(end[0], 40)
        if e > b:
            want[b:e] = synth.bf16_round((x[b:e] @ w[0].T + bias[0]).astype(np.float32))
        assert np.array_equal(_run(False, x, w, begin, end, bias, status=binding.DEV_BOUNDS), want)


# ---- how it is called -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,K,N", [(5, 64, 24), (800, 256, 520), (1, 8, 8)])
def test_rows_that_lie_apart(rows, K, N):
    import torch
    x, w, bias, want = _whole_case(False, [0], [rows], rows, 1, K, N)
    wide = torch.full((rows, K + 40), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 16:16 + K] = dev_bf16(x)
    out = torch.full((rows, N + 24), OLD, dtype=torch.bfloat16, device="cuda")
    binding.grouped_matmul(wide[:, 16:16 + K], dev_bf16(w), dev_i32([0]), dev_i32([rows]), out[:, 8:8 + N], bias=dev_bf16(bias))
    got = host_f64(out)
    assert np.array_equal(got[:, 8:8 + N], want) and np.all(got[:, :8] == OLD) and np.all(got[:, 8 + N:] == OLD)


def test_offsets_beyond_32_bits():
    import torch
    rows, K, N, far = 66000, 16, 8, 40000
    x, w, bias, want = _whole_case(False, [0], [rows], rows, 1, K, N)
    wide = torch.empty((rows, far), dtype=torch.bfloat16, device="cuda")
    out = torch.empty((rows, far), dtype=torch.bfloat16, device="cuda")
    wide[:, :K] = dev_bf16(x)
    binding.grouped_matmul(wide[:, :K], dev_bf16(w), dev_i32([0]), dev_i32([rows]), out[:, :N], bias=dev_bf16(bias))
    assert np.array_equal(host_f64(out[:, :N].contiguous()), want)


@pytest.mark.parametrize("fp4", [False, True], ids=["bf16", "mxfp4"])
@pytest.mark.parametrize("case", [FEW[4], MANY[1], SLICED[1]], ids=["few", "many", "sliced"])
def test_captured_and_replayed_with_other_counts(fp4, case):
    """The ranges are read when the kernel runs: a captured call follows them; runs repeat bit for bit."""
    import torch
    begin, end, rows, sets, K, N = case
    x, w, bias, want = _whole_case(fp4, begin, end, rows, sets, K, N)
    b, e = dev_i32(begin), dev_i32(end)
    out = torch.full((rows, N), OLD, dtype=torch.bfloat16, device="cuda")
    dx, dw, db = (_dev_codes(x), _dev_codes(w), dev_bf16(bias)) if fp4 else ((dev_bf16(x),), (dev_bf16(w),), dev_bf16(bias))
    call = lambda: (binding.mxfp4_grouped_matmul if fp4 else binding.grouped_matmul)(*dx, *dw, b, e, out, bias=db)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        assert np.array_equal(host_f64(out), want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
            call()
    out.fill_(OLD)
    e[-1] -= 1
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    want[end[-1] - 1] = OLD
    assert np.array_equal(host_f64(out), want)


def test_two_streams_at_once():
    import torch
    cases = [_whole_case(False, *MANY[0]), _whole_case(False, *FEW[3]), _whole_case(True, *MANY[1]), _whole_case(True, *SLICED[2])]
    begins, streams, outs = (MANY[0], FEW[3], MANY[1], SLICED[2]), [torch.cuda.Stream() for _ in range(4)], []
    calls = []
    for i, ((x, w, bias, want), c) in enumerate(zip(cases, begins)):
        out = torch.full((c[2], c[5]), OLD, dtype=torch.bfloat16, device="cuda")
        ops = (dev_bf16(x), dev_bf16(w)) if i < 2 else (*_dev_codes(x), *_dev_codes(w))
        calls.append((binding.grouped_matmul if i < 2 else binding.mxfp4_grouped_matmul, ops, dev_i32(c[0]), dev_i32(c[1]), out, dev_bf16(bias)))
    torch.cuda.synchronize()
    for _ in range(20):
        for st, (f, ops, b, e, out, bias) in zip(streams, calls):
            f(*ops, b, e, out, bias=bias, stream=st)
    torch.cuda.synchronize()
    for (x, w, bias, want), call in zip(cases, calls):
        assert np.array_equal(host_f64(call[4]), want)


def test_nothing_to_do():
    import torch
    t = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    before = binding.kernel_launches()
    binding.grouped_matmul(t(0, 64), t(1, 8, 64), dev_i32([0]), dev_i32([0]), t(0, 8))
    binding.grouped_matmul(t(4, 64), t(1, 8, 64), dev_i32([]), dev_i32([]), t(4, 8))
    assert binding.kernel_launches() == before


def test_refusals_of_the_binding():
    import torch
    t = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    r = dev_i32([0]), dev_i32([1])
    for x, w, out, kw in ((t(4, 64), t(1, 8, 72), t(4, 8), {}), (t(4, 64), t(1, 8, 64), t(4, 16), {}), (t(4, 64), t(1, 12, 64), t(4, 12), {}),
                          (t(4, 60), t(1, 8, 60), t(4, 8), {}), (t(64, 4).T, t(1, 8, 64), t(4, 8), {}),
                          (t(4, 64).float(), t(1, 8, 64), t(4, 8), {}), (t(4, 64).cpu(), t(1, 8, 64), t(4, 8), {}),
                          (t(4, 64), t(1, 8, 64), t(4, 8), dict(bias=t(1, 16))), (t(4, 64), t(1, 8, 64), t(4, 8), dict(activation=7))):
        with pytest.raises(binding.RegionEError):
            binding.grouped_matmul(x, w, *r, out, **kw)
    with pytest.raises(binding.RegionEError):
        binding.grouped_matmul(t(4, 64), t(1, 8, 64), dev_i32([0, 1]), dev_i32([1]), t(4, 8))
    u = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    for xq, xs, wq, ws in ((u(4, 32), u(4, 2), u(1, 8, 32), u(1, 8, 2)), (u(4, 64), u(4, 4), u(1, 8, 64), u(1, 8, 5)),
                           (u(4, 64), u(4, 3), u(1, 8, 64), u(1, 8, 4))):     # K = 64; scales of another shape
        with pytest.raises(binding.RegionEError):
            binding.mxfp4_grouped_matmul(xq, xs, wq, ws, *r, t(4, 8))


@pytest.mark.parametrize("rows,N", [(64, 24), (900, 264)])
def test_ranges_that_overlap_end_and_are_recorded(rows, N):
    """Not allowed, and which result stands is not said; no more is run than there can be rows."""
    import torch
    x, w, bias, _ = _whole_case(False, [0], [rows], rows, 1, 64, N)
    G = 512
    _run(False, x, w, [0] * G, [rows] * G, bias, status=binding.DEV_BOUNDS)


def test_first_call_of_a_process_may_be_captured():
    """Setting the kernels up is no work on a stream."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2510_25590_b200 import binding as b
t = lambda *s: torch.ones(s, dtype=torch.bfloat16, device="cuda")
x, w, out = t(3, 64), t(1, 8, 64), torch.zeros((3, 8), dtype=torch.bfloat16, device="cuda")
r = torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    b.grouped_matmul(x, w, *r, out)
g.replay()
torch.cuda.synchronize()
assert bool((out == 64).all()), out
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", code], check=True, cwd=root, timeout=120)
