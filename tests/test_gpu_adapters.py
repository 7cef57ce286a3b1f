"""GPU parity of the product with low-rank adapters with the oracle in 64 bits.

Small whole numbers whose sums stay below 2^8 in front of the second factor (what bf16 holds exactly) make every product and sum exact in
fp32, so those outputs have to be the correctly rounded ones, bit for bit.  With other numbers the bound is half a bf16 step of the
result, 2^-8 |y|, plus K + rank additions that each lose at most 2^-23 of the sum of magnitudes, plus, where x A^T is rounded
on the way (groups of more than 32 rows on average, 8 where there are several weight sets), 2^-8 of the magnitudes of the second product's terms."""
import numpy as np
import pytest

from gpu_util import dev_bf16, dev_i32, host_f64
from oracle import regione_oracle as orc
from paper_2510_25590_b200 import binding, synth

pytestmark = pytest.mark.gpu

OLD = -3.0


def _rand(rng, shape, std=1.0):
    return synth.bf16_round((rng.standard_normal(shape) * std).astype(np.float32))


def _f32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


class Case:
    def __init__(self, rows, ranges, sets, K, N, rank, adapters, which, whole=True, seed=0):
        rng = np.random.default_rng([seed, rows, K, N, rank])
        self.rows, self.ranges, self.which, self.N, self.K, self.rank = rows, ranges, which, N, K, rank
        if whole:
            self.x = rng.integers(-2, 3, (rows, K)).astype(np.float32)
            self.w = rng.integers(-3, 4, (sets, N, K)).astype(np.float32)
            # few elements of A, so that its sums stay below 2^8 with a scale of 1 or 2
            self.a = np.zeros((adapters, rank, K), np.float32)
            for m in self.a.reshape(-1, K):
                m[rng.integers(0, K, 24)] = rng.integers(-1, 2, 24)
            self.b = rng.integers(-2, 3, (adapters, N, rank)).astype(np.float32)
            self.scale = rng.integers(1, 3, adapters).astype(np.float32)
            self.bias = rng.integers(-9, 10, (sets, N)).astype(np.float32)
        else:
            self.x, self.w = _rand(rng, (rows, K)), _rand(rng, (sets, N, K), 2 * K ** -0.5)
            self.a, self.b = _rand(rng, (adapters, rank, K), K ** -0.5), _rand(rng, (adapters, N, rank), rank ** -0.5)
            self.scale, self.bias = rng.uniform(0.5, 2, adapters).astype(np.float32), _rand(rng, (sets, N))
        self.live = np.zeros(rows, bool)
        for b, e in ranges:
            self.live[b:e] = True
        self.x[~self.live] = np.nan                                    # rows of no group are not read, or nothing comes of it

    def args(self, extra=0):
        import torch
        x, out = dev_bf16(self.x), torch.full((self.rows, self.N + extra), OLD, dtype=torch.bfloat16, device="cuda")[:, :self.N]
        if extra:
            wide = torch.full((self.rows, self.K + extra), float("nan"), dtype=torch.bfloat16, device="cuda")
            wide[:, :self.K] = x
            x = wide[:, :self.K]
        ws = torch.full((binding.adapter_matmul_workspace(self.rows, len(self.ranges), self.K, self.N, self.rank),), 255, dtype=torch.uint8,
                        device="cuda")
        return (x, dev_bf16(self.w), dev_bf16(self.a), dev_bf16(self.b), dev_i32(self.which), dev_i32([b for b, _ in self.ranges]),
                dev_i32([e for _, e in self.ranges]), out, ws)

    def run(self, extra=0, gelu=False, status=0, scale=True, bias=True, stream=None):
        import torch
        args = self.args(extra)
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        binding.adapter_matmul(*args, scale=_f32(self.scale) if scale else None, bias=dev_bf16(self.bias) if bias else None,
                               activation=binding.ACT_GELU_TANH if gelu else binding.ACT_NONE, dev_status=st, stream=stream)
        torch.cuda.synchronize()
        assert int(st[0]) == status
        return host_f64(args[7])

    def want(self, **kw):
        x = np.where(self.live[:, None], self.x, 0.0)
        return orc.adapter_matmul(x, self.w, self.a, self.b, self.which, self.ranges, kw.get("scale", self.scale), kw.get("bias", self.bias),
                                  kw.get("gelu", False))

    def check_exact(self, got, **kw):
        want = synth.bf16_round(self.want(**kw).astype(np.float32))
        assert np.all(got[~self.live] == OLD)
        assert np.array_equal(got[self.live], want[self.live].astype(np.float64))


def _tokens(n, sets=1):
    return [(i, i + 1) for i in range(n)]


def _streams(batch, text, room, live):
    out = []
    for b in range(batch):
        at = b * (text + room)
        out += [(at, at + text), (at + text, at + text + live[b])]
    return out


def _which(rng, groups, adapters):
    w = rng.integers(-1, adapters, groups)
    w[0] = adapters - 1
    return [int(v) for v in w]


# groups of few rows on average, side by side or not
FEW = [(1, [(0, 1)], 1, 64, 8, 8, 1), (1, [(0, 1)], 1, 2048, 264, 16, 3), (64, _tokens(64), 1, 512, 520, 16, 24), (200, _tokens(200), 1, 264, 136, 8, 40),
       (48, [(i * 16, i * 16 + n) for i, n in enumerate((16, 3, 11))], 1, 1000, 72, 40, 4), (32, _tokens(32), 2, 384, 200, 64, 5),
       (30, [(0, 7), (7, 7), (7, 20), (22, 30)], 1, 8192, 64, 128, 3), (512, _tokens(512), 1, 128, 1024, 24, 9), (300, _tokens(300), 4, 192, 2048, 256, 6),
       (8, [(4 * (i % 2) + i // 2, 4 * (i % 2) + i // 2 + 1) for i in range(8)], 2, 640, 392, 32, 4)]
# sizes of one piece; many groups of the same few adapters, whose rows are dealt out eight at a time; one adapter for all
FEW += [(3, _tokens(3), 1, 8, 8, 8, 2), (1000, [(2 * i, 2 * i + 2) for i in range(500)], 1, 64, 64, 8, 3), (512, _tokens(512), 1, 72, 24, 16, 1),
        (96, [(3 * i, 3 * i + 2) for i in range(32)], 1, 136, 40, 48, 2)]
# groups of many rows
MANY = [(70, [(0, 70)], 1, 8, 8, 8, 1), (40, [(0, 40)], 1, 64, 8, 8, 1), (300, [(0, 300)], 1, 2048, 520, 16, 2), (1200, _streams(2, 77, 523, [523, 400]), 2, 512, 1544, 32, 3),
        (2400, _streams(2, 256, 944, [901, 944]), 2, 384, 768, 64, 8), (700, [(0, 700)], 1, 8192, 136, 72, 1), (500, [(3, 50), (50, 50), (60, 490)], 3, 1000, 264, 200, 4),
        (4000, [(0, 60), (60, 70), (70, 4000)], 3, 4096, 264, 128, 2), (640, [(0, 640)], 1, 4096, 1024, 256, 1), (100, [(0, 100)], 1, 4096, 128, 8, 1),
        (2049, [(0, 2049)], 1, 256, 1000, 48, 1)]


@pytest.mark.parametrize("shape", FEW + MANY, ids=lambda s: f"{s[0]}x{s[3]}x{s[4]}r{s[5]}g{len(s[1])}")
def test_whole_numbers_are_exact(shape):
    rows, ranges, sets, K, N, rank, adapters = shape
    c = Case(*shape[:6], adapters, _which(np.random.default_rng(rows), len(ranges), adapters))
    c.check_exact(c.run())
    c.check_exact(c.run(extra=16, scale=False, bias=False), scale=None, bias=None)


@pytest.mark.parametrize("shape", [FEW[2], FEW[4], FEW[6], FEW[11], MANY[2], MANY[3], MANY[5], MANY[8]], ids=lambda s: f"{s[0]}x{s[3]}x{s[4]}r{s[5]}")
@pytest.mark.parametrize("gelu", [False, True])
def test_normal_numbers(shape, gelu):
    rows, ranges, sets, K, N, rank, adapters = shape
    c = Case(*shape[:6], adapters, _which(np.random.default_rng(rows), len(ranges), adapters), whole=False)
    got, want = c.run(gelu=gelu), c.want(gelu=gelu)
    x = np.abs(np.where(c.live[:, None], c.x, 0.0).astype(np.float64))
    sums, second = np.zeros(want.shape), np.zeros(want.shape)
    few = rows <= (32 if sets == 1 else 8) * len(ranges)
    for g, ((b, e), j) in enumerate(zip(c.ranges, c.which)):
        i = g % len(c.w)
        sums[b:e] = x[b:e] @ np.abs(c.w[i].T.astype(np.float64)) + np.abs(c.bias[i])
        if j >= 0:
            u = c.scale[j] * (np.where(c.live[b:e, None], c.x[b:e], 0.0).astype(np.float64) @ c.a[j].T.astype(np.float64))
            sums[b:e] += c.scale[j] * (x[b:e] @ np.abs(c.a[j].T.astype(np.float64))) @ np.abs(c.b[j].T.astype(np.float64))
            second[b:e] = np.abs(u) @ np.abs(c.b[j].T.astype(np.float64))
    tol = 2.0 ** -8 * np.abs(want) + 1.13 * ((K + rank) * 2.0 ** -23 * sums + (0 if few else 2.0 ** -8 * second)) + 1e-30
    tol += 6 * 2.0 ** -20 * np.abs(want) if gelu else 0
    assert np.all(np.abs(got - want)[c.live] <= tol[c.live])
    assert np.all(got[~c.live] == OLD)
    # and on average: roundings of the output and of up to `rank` terms, each uniform within half a step
    d = (got - want)[c.live]
    assert np.sqrt((d * d).mean()) <= 2.5e-3 * np.sqrt((want[c.live] ** 2).mean())


@pytest.mark.parametrize("shape", [FEW[2], FEW[9], MANY[3], MANY[9]], ids=["tokens", "sets", "streams", "slices"])
def test_without_an_adapter_it_is_the_grouped_product(shape):
    import torch
    c = Case(*shape[:6], shape[6], [-1] * len(shape[1]), whole=False)
    args = c.args()
    binding.adapter_matmul(*args, bias=dev_bf16(c.bias))
    c.which = [0] * len(c.ranges)
    with_one = c.run(scale=False)
    live = torch.from_numpy(c.live).cuda()
    want = torch.full_like(args[7], OLD)
    binding.grouped_matmul(args[0], args[1], args[5], args[6], want, bias=dev_bf16(c.bias))
    # (tiles, and with them the order of additions, may be others)
    a, b = host_f64(args[7]), host_f64(want)
    assert np.all(np.abs(a - b) <= 2.0 ** -7 * np.abs(b) + c.K * 2.0 ** -22 * 8) and np.array_equal(a[~c.live], b[~c.live])
    assert not np.array_equal(with_one, a)


@pytest.mark.parametrize("rows,ranges", [(40, _tokens(40)), (1300, [(0, 600), (600, 1300)])])
def test_an_adapter_that_does_not_exist_is_none(rows, ranges):
    which = [0, 7] * (len(ranges) // 2)
    c = Case(rows, ranges, 1, 256, 136, 16, 2, [0 if v == 0 else -1 for v in which])
    want = c.run()
    c.check_exact(want)
    for bad in (7, 2, -2, 2 ** 31 - 1, -2 ** 31):
        c.which = [0 if v == 0 else bad for v in which]
        assert np.array_equal(c.run(status=binding.DEV_BOUNDS), want)


@pytest.mark.parametrize("rows,ranges", [(48, [(0, 10), (10, 30), (30, 48)]), (900, [(0, 300), (300, 600), (600, 900)])])
def test_what_is_not_finite_stays_with_its_group(rows, ranges):
    """An adapter with NaN or infinite elements, and rows that have them, next to groups with others: tiles are shared where rows are few."""
    c = Case(rows, ranges, 1, 256, 136, 16, 3, [0, 1, 2])
    want = c.run()
    c.a[1, 3, 5], c.b[1, 7, 2] = np.inf, np.nan
    c.x[ranges[2][0]] = np.inf
    got = c.run()
    (b1, e1), (b2, e2) = ranges[1], ranges[2]
    same = np.ones(rows, bool)
    same[b1:e1], same[b2] = False, False
    assert np.array_equal(got[same], want[same])
    assert np.all(np.isnan(got[b1:e1, 7]))


@pytest.mark.parametrize("begin,end,cut", [([-3, 20], [10, 500], [(0, 10), (20, 128)]), ([5, 30], [20, 10], [(5, 20)]),
                                           ([-2 ** 31, 7], [2 ** 31 - 1, 7], [(0, 128)])])
@pytest.mark.parametrize("rows", [64, 128], ids=["few", "many"])
def test_ranges_outside_the_buffer_are_cut(begin, end, cut, rows):
    import torch
    cut = [(b, min(e, rows)) for b, e in cut]
    c = Case(rows, cut, 1, 128, 64, 16, 2, [0, 1][:len(cut)])
    args = list(c.args())
    args[4], args[5], args[6] = dev_i32([0, 1]), dev_i32(begin), dev_i32(end)
    args[8] = torch.empty(binding.adapter_matmul_workspace(rows, 2, 128, 64, 16), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.adapter_matmul(*args, scale=_f32(c.scale), bias=dev_bf16(c.bias), dev_status=st)
    torch.cuda.synchronize()
    assert int(st[0]) == binding.DEV_BOUNDS
    c.check_exact(host_f64(args[7]))


def test_ranges_that_overlap_stay_in_bounds():
    """Which result stands is not said; nothing outside the buffers is touched and the call ends."""
    import torch
    for rows, n in ((16, 40), (640, 3)):
        c = Case(rows, [(0, rows)] * n, 1, 128, 64, 16, 2, [0, 1] * (n // 2) + [0] * (n % 2))
        args = c.args()
        binding.adapter_matmul(*args)
    torch.cuda.synchronize()


@pytest.mark.parametrize("shape", [FEW[2], MANY[3]], ids=["few", "many"])
def test_repeats_captured_two_graphs_and_another_stream(shape):
    import torch
    c = Case(*shape[:6], shape[6], _which(np.random.default_rng(0), len(shape[1]), shape[6]), whole=False)
    want = c.run()
    assert np.array_equal(c.run(), want)
    assert np.array_equal(c.run(stream=torch.cuda.Stream()), want)
    graphs = []
    for _ in range(2):
        args = c.args()
        extra = dict(scale=_f32(c.scale), bias=dev_bf16(c.bias))
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            binding.adapter_matmul(*args, stream=torch.cuda.current_stream(), **extra)
        graphs.append((graph, args, extra))
    side = torch.cuda.Stream()
    for _ in range(3):
        graphs[0][0].replay()
        with torch.cuda.stream(side):
            graphs[1][0].replay()
    torch.cuda.synchronize()
    for _, args, _ in graphs:
        assert np.array_equal(host_f64(args[7]), want)


def test_offsets_beyond_32_bits():
    """Many adapters: the last one's factors lie beyond 2^31 elements."""
    import torch
    n, rank, K, N = 4200, 64, 8192, 64                                 # A: 2.2e9 elements
    a = torch.zeros((n, rank, K), dtype=torch.bfloat16, device="cuda")
    b = torch.zeros((n, N, rank), dtype=torch.bfloat16, device="cuda")
    for rows, ranges in ((3, _tokens(3)), (150, [(0, 50), (50, 100), (100, 150)])):
        c = Case(rows, ranges, 1, K, N, rank, 3, [0, 1, 2])
        at = [0, 4100, n - 1]
        for i, j in enumerate(at):
            a[j], b[j] = dev_bf16(c.a[i]), dev_bf16(c.b[i])
        scale = torch.ones(n, device="cuda")
        scale[at] = _f32(c.scale)
        args = list(c.args())
        args[2], args[3], args[4] = a, b, dev_i32(at)
        binding.adapter_matmul(*args, scale=scale, bias=dev_bf16(c.bias))
        torch.cuda.synchronize()
        c.check_exact(host_f64(args[7]))


@pytest.mark.parametrize("shape", [FEW[2], FEW[11], MANY[3]], ids=["few", "few_adapters", "many"])
def test_buffers_that_are_used_again_with_other_contents(shape):
    """The same buffers and workspace call after call, everything in them written anew on the stream: rows, ranges, adapters, bias, factors."""
    import torch
    rng = np.random.default_rng(1)
    cases = [Case(*shape[:6], shape[6], _which(rng, len(shape[1]), shape[6]), seed=s) for s in range(4)]
    for c in cases[1::2]:                                              # every second time some rows less
        c.ranges = [(b, max(b, e - 1)) if i % 3 == 2 else (b, e) for i, (b, e) in enumerate(c.ranges)]
        c.live = np.zeros(c.rows, bool)
        for b, e in c.ranges:
            c.live[b:e] = True
    sources = [c.args()[:7] + (_f32(c.scale), dev_bf16(c.bias)) for c in cases]
    held, (out, ws) = [t.clone() for t in sources[0]], cases[0].args()[7:9]
    torch.cuda.synchronize()
    got = []
    for turn in range(12):
        for to, t in zip(held, sources[turn % 4]):
            to.copy_(t)
        out.fill_(OLD)
        binding.adapter_matmul(*held[:7], out, ws, scale=held[7], bias=held[8])
        got.append(out.clone())
    torch.cuda.synchronize()
    for turn in range(12):
        cases[turn % 4].check_exact(host_f64(got[turn]))
