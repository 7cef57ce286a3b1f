"""GPU parity of the layer norm of ragged groups of rows and of its backward pass with the oracle in 64 bits.

Bounds.  An output in bf16 is off by half a step, 2^-8 of its value.  In front of that, in fp32: a sum of a row has no more than 160
additions one behind the other (16 pieces of 8 to a lane, the warp, the warps), each off by 2^-24 of what is added up so far, so that
sums and means of a row are off by less than 2^-16 of the mean magnitude of their terms, and so is the variance; a handful of operations
on one element are off by less than 2^-20 of their magnitudes.  Distances z - m are off by 2^-24 (|z| + |m|) and by what the mean is off.
A gradient of a parameter adds up N rows, one behind the other at the worst: N 2^-24 of the sum of magnitudes."""
import numpy as np
import pytest

from gpu_util import dev_bf16, dev_i32, host_f64
from oracle import regione_oracle as orc
from paper_2510_25590_b200 import binding, synth

pytestmark = pytest.mark.gpu

OLD, EPS = -3.0, 1e-6


def _rand(rng, shape, std=1.0, mean=0.0):
    return synth.bf16_round((rng.standard_normal(shape) * std + mean).astype(np.float32))


def _dev_f32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


def _apart(a, extra):
    """The matrix on the device, its rows `extra` elements further apart than they are wide; what lies between is NaN."""
    import torch
    t = dev_bf16(a)
    if not extra:
        return t
    wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _old(rows, C, extra=0):
    import torch
    return torch.full((rows, C + extra), OLD, dtype=torch.bfloat16, device="cuda")[:, :C]


class Case:
    def __init__(self, rows, C, ranges, sets=1, residual=False, gate=True, weight=True, bias=True, modulated=False, mean=0.25, seed=0):
        rng = np.random.default_rng([seed, rows, C])
        self.rows, self.C, self.ranges, self.sets, self.modulated = rows, C, ranges, sets, modulated
        self.x = _rand(rng, (rows, C), 1.0, mean) * synth.bf16_round(np.exp2(rng.integers(-2, 3, C)).astype(np.float32))
        self.weight = _rand(rng, (sets, C), 0.3, 0.0 if modulated else 1.0) if weight else None
        self.bias = _rand(rng, (sets, C), 0.2) if bias else None
        self.r = _rand(rng, (rows, C)) if residual else None
        self.gate = _rand(rng, (sets, C), 0.5) if residual and gate else None
        self.dy, self.dz = _rand(rng, (rows, C), 0.1), _rand(rng, (rows, C), 0.1)
        self.live = np.zeros(rows, bool)
        for b, e in ranges:
            self.live[b:e] = True
        for a in (self.x, self.r, self.dy, self.dz):                   # rows of no group are not read
            if a is not None:
                a[~self.live] = np.nan

    def dev_ranges(self):
        return dev_i32([b for b, _ in self.ranges]), dev_i32([e for _, e in self.ranges])


def _forward(c, extra=0, status=0, in_place=False):
    import torch
    opt = lambda a: None if a is None else _apart(a, extra)
    x, out = _apart(c.x, extra), _old(c.rows, c.C, extra)
    mean, rstd = (torch.full((c.rows,), OLD, device="cuda") for _ in range(2))
    z = None if c.r is None else x if in_place else _old(c.rows, c.C, extra)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.layer_norm(x, opt(c.weight), opt(c.bias), *c.dev_ranges(), out, EPS, modulated=c.modulated, residual=opt(c.r), gate=opt(c.gate),
                       x_out=z, mean=mean, rstd=rstd, dev_status=st)
    torch.cuda.synchronize()
    assert int(st[0]) == status
    return None if z is None else host_f64(z), host_f64(out), host_f64(mean).astype(np.float64), host_f64(rstd).astype(np.float64)


def _check_forward(c, got, in_place=False):
    z, out, mean, rstd = got
    live = c.live
    if c.r is not None:
        want = c.x.astype(np.float64)
        for g, (b, e) in enumerate(c.ranges):
            want[b:e] += (1.0 if c.gate is None else c.gate[g % c.sets].astype(np.float64)) * c.r[b:e].astype(np.float64)
        if not in_place:
            assert np.all(z[~live] == OLD)
        assert np.all(np.abs(z[live] - want[live]) <= 2.0 ** -8 * np.abs(want[live]) * (1 + 2.0 ** -15))
        row = z                                                        # the norm is that of the row as it is kept
    else:
        row = c.x.astype(np.float64)
    _, want, m, s = orc.layer_norm(row, c.weight, c.bias, c.ranges, EPS, c.modulated)
    assert np.all(out[~live] == OLD) and np.all(mean[~live] == OLD) and np.all(rstd[~live] == OLD)
    size = np.abs(np.where(live[:, None], row, 0.0))
    off = 2.0 ** -16 * size.mean(1)                                    # of the mean
    assert np.all(np.abs(mean - m)[live] <= off[live])
    assert np.all(np.abs(rstd - s)[live] <= 2.0 ** -15 * s[live] + s[live] ** 3 * off[live] ** 2)
    w = np.zeros((c.rows, c.C))
    for g, (b, e) in enumerate(c.ranges):
        w[b:e] = (0.0 if c.modulated else 1.0) if c.weight is None else c.weight[g % c.sets]
    w = np.abs(w + (1.0 if c.modulated else 0.0))
    h = np.abs(row - m[:, None]) * s[:, None]
    tol = 2.0 ** -8 * np.abs(want) + w * (2.0 ** -14 * h + s[:, None] * (off[:, None] + 2.0 ** -22 * (size + np.abs(m)[:, None]))) + 2.0 ** -20
    assert np.all(np.abs(out - want)[live] <= tol[live]), np.max((np.abs(out - want) / tol)[live])


def _ragged(rows, groups):
    """Ranges with gaps and an empty group between them."""
    cut = np.linspace(0, rows, groups + 1).astype(int)
    out = [(int(b) + (i % 3 == 1), int(e)) for i, (b, e) in enumerate(zip(cut[:-1], cut[1:]))]
    out = [(min(b, e), e) for b, e in out]
    if groups > 2:
        out[2] = (out[2][0], out[2][0])
    return out


# few rows: several warps to a row; many: a warp each; long rows
SHAPES = [(1, 8, 1), (1, 1024, 1), (5, 24, 2), (33, 264, 4), (77, 1000, 3), (130, 2048, 4), (64, 2056, 40), (19, 4096, 2), (21, 4104, 2), (40, 8192, 5),
          (2500, 8, 3), (2500, 264, 70), (2400, 512, 2), (2401, 1000, 4), (2500, 1544, 8), (2400, 2056, 3), (2390, 4096, 2)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}g{s[2]}")
@pytest.mark.parametrize("form", ["affine", "modulated", "residual", "plain_residual", "bare"])
def test_forward(shape, form):
    rows, C, groups = shape
    sets = {"affine": 1, "modulated": groups, "residual": groups, "plain_residual": 2, "bare": 1}[form]
    c = Case(rows, C, _ragged(rows, groups), sets, residual="residual" in form, gate=form == "residual", weight=form != "bare",
             bias=form != "bare", modulated=form in ("modulated", "residual"))
    _check_forward(c, _forward(c))


@pytest.mark.parametrize("rows,C", [(40, 1000), (2500, 264), (9, 8192)])
def test_forward_rows_and_sets_apart_and_in_place(rows, C):
    c = Case(rows, C, _ragged(rows, 4), 4, residual=True, modulated=True)
    _check_forward(c, _forward(c, extra=24))
    _check_forward(c, _forward(c, extra=24, in_place=True), in_place=True)


def test_a_mean_far_from_zero_and_rows_without_variance():
    c = Case(50, 1024, [(0, 50)], mean=0.0)
    c.x = synth.bf16_round(1000.0 + np.random.default_rng(1).standard_normal((50, 1024)).astype(np.float32) * 8)
    c.x[7] = 3.0
    c.x[8] = 0.0
    got = _forward(c)
    _check_forward(c, got)
    assert np.array_equal(got[1][7], synth.bf16_round(c.bias[0]).astype(np.float64)) and got[3][7] == np.float32(1e3)


def test_what_is_not_finite_stays_in_its_row():
    c = Case(2400, 264, [(0, 2400)])
    want = _forward(c)[1]
    c.x[5, 3], c.x[77, 100] = np.inf, np.nan
    got = _forward(c)[1]
    other = np.ones(2400, bool)
    other[[5, 77]] = False
    assert np.array_equal(got[other], want[other]) and np.all(np.isnan(got[5])) and np.all(np.isnan(got[77]))


@pytest.mark.parametrize("begin,end,want", [([-3, 20], [10, 500], [(0, 10), (20, 64)]), ([30], [10], []), ([-2 ** 31, 5], [2 ** 31 - 1, 5], [(0, 64)])])
def test_ranges_outside_the_buffer_are_cut(begin, end, want):
    import torch
    c = Case(64, 264, want or [(0, 0)])
    c.dev_ranges = lambda: (dev_i32(begin), dev_i32(end))
    _check_forward(c, _forward(c, status=binding.DEV_BOUNDS))


def test_overlapping_ranges_stay_in_bounds():
    c = Case(64, 264, [(0, 64)] * 40)
    _forward(c, status=binding.DEV_BOUNDS)


def test_more_ranges_than_rows_and_no_rows():
    import torch
    c = Case(40, 72, [(r, r + 1) if r < 40 else (40, 40) for r in range(512)], 512, modulated=True)
    _check_forward(c, _forward(c))
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    binding.layer_norm(x, None, None, dev_i32([]), dev_i32([]), x, EPS)
    torch.cuda.synchronize()


def test_offsets_beyond_32_bits():
    import torch
    apart, rows, C = 1 << 24, 300, 264                                 # 5.0e9 elements
    c = Case(rows, C, [(0, 1), (1, 200), (290, 300)])
    wide = torch.empty(rows * apart, dtype=torch.bfloat16, device="cuda").view(rows, apart)
    wide[:, :C] = dev_bf16(c.x)
    wide[:, 512:512 + C] = OLD
    x, out = wide[:, :C], wide[:, 512:512 + C]
    binding.layer_norm(x, dev_bf16(c.weight), dev_bf16(c.bias), *c.dev_ranges(), out, EPS)
    near = _old(rows, C)
    binding.layer_norm(dev_bf16(c.x), dev_bf16(c.weight), dev_bf16(c.bias), *c.dev_ranges(), near, EPS)
    assert torch.equal(out, near)


# ---- backward ----------------------------------------------------------------------------------------------------------------------
def _stats(c):
    _, _, m, s = orc.layer_norm(np.where(c.live[:, None], c.x, 0.0), None, None, c.ranges, EPS)
    return m.astype(np.float32), s.astype(np.float32)


def _backward(c, dz=False, extra=0, status=0, in_place=False, workspace=None):
    import torch
    opt = lambda a: None if a is None else _apart(a, extra)
    m, s = _stats(c)
    dy = _apart(c.dy, extra)
    dx = dy if in_place else _old(c.rows, c.C, extra)
    dr = None if c.gate is None else _old(c.rows, c.C, extra)
    grads = [torch.full((c.sets, c.C), float("nan"), device="cuda") for _ in range(3)]
    ws = workspace
    if ws is None:
        ws = torch.full((binding.layer_norm_backward_workspace(c.rows, len(c.ranges), c.C),), 255, dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.layer_norm_backward(opt(c.x), _dev_f32(m), _dev_f32(s), dy, opt(c.weight), *c.dev_ranges(), dx, grads[0], grads[1], ws,
                                modulated=c.modulated, dx_out=opt(c.dz) if dz else None, residual=None if dr is None else opt(c.r),
                                gate=opt(c.gate), dresidual=dr, dgate=None if dr is None else grads[2], dev_status=st)
    torch.cuda.synchronize()
    assert int(st[0]) == status
    return host_f64(dx), None if dr is None else host_f64(dr), *[host_f64(t).astype(np.float64) for t in grads]


def _check_backward(c, got, dz=False, in_place=False):
    m, s = (a.astype(np.float64) for a in _stats(c))
    gated = c.gate is not None
    z = np.where(c.live[:, None], c.x, 0.0).astype(np.float64)
    dy = np.where(c.live[:, None], c.dy, 0.0).astype(np.float64)
    r = np.where(c.live[:, None], c.r, 0.0).astype(np.float64) if gated else None
    want = orc.layer_norm_backward(z, m, s, dy, c.weight, c.ranges, c.sets, c.modulated, c.dz if dz else None, r, c.gate)
    live = c.live
    if not in_place:
        assert np.all(got[0][~live] == OLD)
    # magnitudes of what is added up to d
    w, gate = np.zeros((c.rows, c.C)), np.zeros((c.rows, c.C))
    for g, (b, e) in enumerate(c.ranges):
        w[b:e] = ((0.0 if c.modulated else 1.0) if c.weight is None else c.weight[g % c.sets]) + (1.0 if c.modulated else 0.0)
        if gated:
            gate[b:e] = np.abs(c.gate[g % c.sets])
    h = (np.abs(z) + np.abs(m)[:, None]) * s[:, None]
    a = np.abs(dy * w)
    off = 2.0 ** -16 * s[:, None] * (a + a.mean(1, keepdims=True) + h * (a * h).mean(1, keepdims=True))
    off += 2.0 ** -23 * np.abs(want[0])
    tol = 2.0 ** -8 * np.abs(want[0]) + off + 2.0 ** -120
    assert np.all(np.abs(got[0] - want[0])[live] <= tol[live]), np.max((np.abs(got[0] - want[0]) / tol)[live])
    if gated:
        assert np.all(got[1][~live] == OLD)
        assert np.all(np.abs(got[1] - want[1])[live] <= (2.0 ** -8 * np.abs(want[1]) + gate * off + 2.0 ** -120)[live])
    N = c.rows
    for i in range(c.sets):
        mine = np.zeros(c.rows, bool)
        for b, e in c.ranges[i::c.sets]:
            mine[b:e] = True
        assert np.all(np.abs(got[2][i] - want[2][i]) <= (N + 4) * 2.0 ** -24 * (np.abs(dy) * h)[mine].sum(0))
        assert np.all(np.abs(got[3][i] - want[3][i]) <= N * 2.0 ** -24 * np.abs(dy)[mine].sum(0))
        if gated:
            terms = np.abs(r) * off + (N + 4) * 2.0 ** -24 * np.abs(want[0] * r)
            assert np.all(np.abs(got[4][i] - want[4][i]) <= terms[mine].sum(0))


BACK = [(1, 8, 1), (1, 2048, 1), (5, 24, 2), (33, 264, 4), (300, 1000, 3), (700, 2048, 4), (64, 2056, 40), (500, 4096, 2), (21, 4104, 2), (400, 8192, 5),
        (2500, 72, 70), (1201, 512, 2)]


@pytest.mark.parametrize("shape", BACK, ids=lambda s: f"{s[0]}x{s[1]}g{s[2]}")
@pytest.mark.parametrize("form", ["affine", "modulated", "residual", "plain_residual"])
def test_backward(shape, form):
    rows, C, groups = shape
    sets = {"affine": 1, "modulated": groups, "residual": groups, "plain_residual": 2}[form]
    c = Case(rows, C, _ragged(rows, groups), sets, residual=form == "residual", modulated=form in ("modulated", "residual"))
    dz = "residual" in form
    _check_backward(c, _backward(c, dz), dz)


def test_backward_without_weight_rows_apart_and_in_place():
    c = Case(60, 1000, _ragged(60, 4), 2, residual=True, weight=False)
    _check_backward(c, _backward(c, True, extra=8), True)
    _check_backward(c, _backward(c, True, extra=8, in_place=True), True, in_place=True)


def test_sets_without_rows_get_zeros():
    c = Case(64, 264, [(0, 10), (10, 10), (20, 64)], 5, residual=True)
    got = _backward(c)
    _check_backward(c, got)
    assert all(np.all(got[k][i] == 0) for k in (2, 3, 4) for i in (1, 3, 4))
    import torch
    none = torch.empty((0, 264), dtype=torch.bfloat16, device="cuda")
    dw = torch.full((5, 264), float("nan"), device="cuda")
    f = torch.empty(0, device="cuda")
    binding.layer_norm_backward(none, f, f, none, dev_bf16(c.weight), dev_i32([]), dev_i32([]), none, dw, None, None)
    assert torch.equal(dw, torch.zeros_like(dw))


def test_backward_of_ranges_outside_the_buffer():
    c = Case(64, 264, [(0, 10), (20, 64)])
    c.dev_ranges = lambda: (dev_i32([-3, 20]), dev_i32([10, 500]))
    _check_backward(c, _backward(c, status=binding.DEV_BOUNDS))
    c = Case(64, 264, [(0, 64)] * 40)
    _backward(c, status=binding.DEV_BOUNDS)                            # ranges that overlap: nothing out of bounds


def test_a_mostly_empty_buffer():
    c = Case(6000, 264, [(10, 40), (5000, 5003)], 2, residual=True, modulated=True)
    _check_forward(c, _forward(c))
    c.gate = c.gate
    _check_backward(c, _backward(c, True), True)


def test_calls_repeat_bit_for_bit_captured_and_on_another_stream():
    import torch
    c = Case(900, 1544, _ragged(900, 5), 5, residual=True, modulated=True)
    m, s = (_dev_f32(a) for a in _stats(c))
    x, r, dy, w, b, gate = (dev_bf16(a) for a in (c.x, c.r, c.dy, c.weight, c.bias, c.gate))
    begin, end = c.dev_ranges()
    n = binding.layer_norm_backward_workspace(900, 5, 1544)

    def buffers():
        return ([_old(900, 1544) for _ in range(4)], [torch.zeros((5, 1544), device="cuda") for _ in range(3)],
                torch.empty(n, dtype=torch.uint8, device="cuda"))

    def run(bufs, stream=None):
        (z, y, dx, dr), grads, ws = bufs
        binding.layer_norm(x, w, b, begin, end, y, EPS, modulated=True, residual=r, gate=gate, x_out=z, stream=stream)
        binding.layer_norm_backward(x, m, s, dy, w, begin, end, dx, *grads[:2], ws, modulated=True, residual=r, gate=gate, dresidual=dr,
                                    dgate=grads[2], stream=stream)

    first, again, other, captured = buffers(), buffers(), buffers(), buffers()
    run(first)
    run(again)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    run(other, side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(captured, torch.cuda.current_stream())
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for bufs in (again, other, captured):
        for a, b_ in zip(first[0] + first[1], bufs[0] + bufs[1]):
            assert torch.equal(a, b_)


def test_two_calls_at_one_time():
    """Forward and backward of two batches on two streams, a workspace each."""
    import torch
    cases = [Case(1800, 1032, _ragged(1800, 3), 3, residual=True, modulated=True, seed=s) for s in (1, 2)]
    want = [(_forward(c), _backward(c, True)) for c in cases]
    for _ in range(3):
        held, streams = [], [torch.cuda.Stream() for _ in cases]
        for c in cases:
            m, s = (_dev_f32(a) for a in _stats(c))
            held.append(dict(x=dev_bf16(c.x), w=dev_bf16(c.weight), b=dev_bf16(c.bias), r=dev_bf16(c.r), q=dev_bf16(c.gate), dy=dev_bf16(c.dy),
                             dz=dev_bf16(c.dz), m=m, s=s, at=c.dev_ranges(), z=_old(1800, 1032), y=_old(1800, 1032), dx=_old(1800, 1032),
                             dr=_old(1800, 1032), g=[torch.zeros((3, 1032), device="cuda") for _ in range(3)],
                             ws=torch.empty(binding.layer_norm_backward_workspace(1800, 3, 1032), dtype=torch.uint8, device="cuda")))
        torch.cuda.synchronize()
        for h, st in zip(held, streams):
            binding.layer_norm(h["x"], h["w"], h["b"], *h["at"], h["y"], EPS, modulated=True, residual=h["r"], gate=h["q"], x_out=h["z"], stream=st)
            binding.layer_norm_backward(h["x"], h["m"], h["s"], h["dy"], h["w"], *h["at"], h["dx"], h["g"][0], h["g"][1], h["ws"], modulated=True,
                                        dx_out=h["dz"], residual=h["r"], gate=h["q"], dresidual=h["dr"], dgate=h["g"][2], stream=st)
        torch.cuda.synchronize()
        for h, (f, b) in zip(held, want):
            assert np.array_equal(host_f64(h["z"]), f[0]) and np.array_equal(host_f64(h["y"]), f[1])
            assert np.array_equal(host_f64(h["dx"]), b[0]) and np.array_equal(host_f64(h["dr"]), b[1])
            for i in range(3):
                assert np.array_equal(host_f64(h["g"][i]).astype(np.float64), b[2 + i])


def test_buffers_that_are_used_again_with_other_contents():
    """The same buffers and workspace call after call, rows, ranges and parameters written anew on the stream."""
    import torch
    cases = [Case(1500, 520, _ragged(1500 - 200 * (i % 2), 4), 4, residual=True, modulated=True, seed=i) for i in range(3)]
    for c in cases:
        c.live = np.zeros(1500, bool)
        for b, e in c.ranges:
            c.live[b:e] = True
        for a in (c.x, c.r, c.dy, c.dz):
            a[~c.live] = np.nan
    want = [_backward(c, True) for c in cases]
    sources = []
    for c in cases:
        m, s = _stats(c)
        sources.append([dev_bf16(a) for a in (c.x, c.dy, c.dz, c.r, c.gate, c.weight)] + [_dev_f32(m), _dev_f32(s), *c.dev_ranges()])
    x, dy, dz, r, gate, w, m, s, begin, end = held = [t.clone() for t in sources[0]]
    dx, dr, grads = _old(1500, 520), _old(1500, 520), [torch.zeros((4, 520), device="cuda") for _ in range(3)]
    ws = torch.empty(binding.layer_norm_backward_workspace(1500, 4, 520), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    got = []
    for turn in range(9):
        for to, t in zip(held, sources[turn % 3]):
            to.copy_(t)
        dx.fill_(OLD); dr.fill_(OLD)
        binding.layer_norm_backward(x, m, s, dy, w, begin, end, dx, grads[0], grads[1], ws, modulated=True, dx_out=dz, residual=r, gate=gate,
                                    dresidual=dr, dgate=grads[2])
        got.append([t.clone() for t in (dx, dr, *grads)])
    torch.cuda.synchronize()
    for turn in range(9):
        for t, a in zip(got[turn], want[turn % 3]):
            assert np.array_equal(host_f64(t).astype(np.float64), a)
