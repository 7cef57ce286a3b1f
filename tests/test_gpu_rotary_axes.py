"""GPU parity of the rotary positions with several axes with the oracle's turns of complex numbers in 64 bits.

Bounds.  The output is off by half a bf16 step, 2^-8 of its value.  In front of that each of the two products is off by what the angle is
off, 2 pi 2^-22, by the cosine (2^-21) and by a few fp32 operations, and the normalised element by 2^-20: less than 2^-17 of |a| + |b|."""
import numpy as np
import pytest

from gpu_util import dev_bf16, dev_i32, host_f64
from oracle import regione_oracle as orc
from paper_2510_25590_b200 import binding, synth

pytestmark = pytest.mark.gpu

OLD, EPS = -3.0, 1e-6


def _rand(rng, shape, std=1.0):
    return synth.bf16_round((rng.standard_normal(shape) * std).astype(np.float32))


def _f32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


def _heads(a, extra=0):
    """[B, rows, H, D] on the device, its rows `extra` elements further apart."""
    import torch
    t = dev_bf16(a)
    B, n, H, D = t.shape
    wide = torch.full((B, n, H * D + extra), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :, :H * D] = t.flatten(2)
    return wide[:, :, :H * D].unflatten(-1, (H, D))


def _partner(x, interleaved):
    x = np.abs(x)
    if interleaved:
        return x.reshape(*x.shape[:-1], x.shape[-1] // 2, 2)[..., ::-1].reshape(x.shape)
    return np.roll(x, x.shape[-1] // 2, -1)


def _run(widths, B, places, cap, Hq, Hk, layout, normalise=True, inverse=False, idx=None, n=None, compact=False, extra=0, shared=False,
         positions=None, weights=True, status=0, seed=0, freq=None, stream=None):
    import torch
    rng = np.random.default_rng([seed, places, Hq, sum(widths)])
    D = sum(widths)
    f, axis = binding.rotary_frequencies(widths)
    f = f if freq is None else freq
    src = cap if compact or idx is None else places
    q, k = _rand(rng, (B, src, Hq, D)), _rand(rng, (B, src, max(Hk, 1), D))
    qw, kw = ((_rand(rng, (D,), 0.3) + np.float32(1)).astype(np.float32) for _ in range(2))
    qw, kw = synth.bf16_round(qw), synth.bf16_round(kw)
    if positions is None:
        positions = rng.integers(0, 90, (1 if shared else B, places, len(widths))).astype(np.float32) + np.float32(0.3125)
    qo, ko = (np.full((B, cap, h, D), OLD, np.float32) for h in (Hq, max(Hk, 1)))
    qt, kt, qot, kot = (_heads(a, extra) for a in (q, k, qo, ko))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    opt = dict(q_weight=dev_bf16(qw) if weights else None, k_weight=dev_bf16(kw) if weights else None, eps=EPS) if normalise else {}
    binding.rotary_axes(qt, kt if Hk else None, _f32(positions), f, axis, qot, kot if Hk else None, layout,
                        idx=None if idx is None else dev_i32(idx), n=None if n is None else dev_i32(n), src_compact=compact,
                        inverse=inverse, dev_status=st, stream=stream, **opt)
    torch.cuda.synchronize()
    assert int(st[0]) == status
    inter = layout == binding.ROPE_INTERLEAVED
    for x, got, w, H in ((q, qot, qw, Hq), (k, kot, kw, Hk)):
        if H == 0:
            continue
        got = host_f64(got)
        for b in range(B):
            live = cap if n is None else min(max(int(n[b]), 0), cap)
            at = np.arange(live) if idx is None else np.asarray(idx)[b, :live].astype(np.int64)
            ok = (at >= 0) & (at < places)
            assert np.all(got[b, live:] == OLD) and np.all(got[b, :live][~ok] == OLD)
            rows = np.arange(live)[ok] if compact or idx is None else at[ok]
            place = positions[0 if len(positions) == 1 else b][at[ok]]
            args = dict(weight=w if normalise and weights else None, eps=EPS if normalise else None)
            want = orc.rotary_axes(x[b][rows], place, f, axis, inter, inverse=inverse, **args)
            y = orc.rotary_axes(x[b][rows], 0 * place, f, axis, inter, **args)
            tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -17 * (np.abs(y) + _partner(y, inter)) + 2.0 ** -130
            d = np.abs(got[b, :live][ok] - want)
            assert np.all(d <= tol), np.max(d / tol)


LAYOUTS = [binding.ROPE_INTERLEAVED, binding.ROPE_HALF]
WIDTHS = [(16,), (8, 8, 16), (32, 32), (16, 24, 24), (32, 32, 32), (32, 24, 24), (44, 42, 42), (16, 56, 56), (48, 48, 48), (64, 64, 64, 64)]


@pytest.mark.parametrize("layout", LAYOUTS, ids=["pairs", "halves"])
@pytest.mark.parametrize("widths", WIDTHS, ids=lambda w: "_".join(map(str, w)))
@pytest.mark.parametrize("normalise", [True, False])
def test_head_dimensions_and_axes(widths, layout, normalise):
    _run(widths, 2, 37, 37, 3, 2, layout, normalise)
    _run(widths, 2, 37, 37, 3, 2, layout, False, inverse=True)


@pytest.mark.parametrize("layout", LAYOUTS, ids=["pairs", "halves"])
@pytest.mark.parametrize("B,places,Hq,Hk", [(1, 1, 1, 1), (17, 1, 8, 8), (3, 5, 16, 1), (1, 700, 24, 24), (2, 1500, 5, 0), (1, 3000, 2, 2), (5, 129, 33, 7)])
def test_rows_and_heads(B, places, Hq, Hk, layout):
    _run((16, 24, 24), B, places, places, Hq, Hk, layout)
    _run((16, 56, 56), B, places, places, Hq, Hk, layout, weights=False, shared=True)


@pytest.mark.parametrize("layout", LAYOUTS, ids=["pairs", "halves"])
@pytest.mark.parametrize("compact", [True, False])
def test_row_lists_and_counts(layout, compact):
    rng = np.random.default_rng(5)
    idx = np.stack([np.sort(rng.permutation(200)[:60]) for _ in range(4)])
    _run((16, 56, 56), 4, 200, 60, 4, 4, layout, idx=idx, n=[60, 0, 1, 37], compact=compact, extra=16)


def test_the_same_place_twice():
    idx = np.array([[7, 7, 0, 7, 3, 3, 49, 0, 1, 1]]).repeat(2, 0)
    _run((16, 24, 24), 2, 50, 10, 2, 2, LAYOUTS[1], idx=idx)


def test_indices_and_counts_outside_are_skipped():
    idx = np.arange(20)[None].repeat(2, 0)
    idx[0, 3], idx[0, 4], idx[1, 19] = -1, 50, 2 ** 31 - 1
    _run((16, 24, 24), 2, 50, 20, 2, 2, LAYOUTS[0], idx=idx, n=[20, 20], status=binding.DEV_BOUNDS)
    _run((16, 24, 24), 2, 50, 20, 2, 2, LAYOUTS[0], n=[-5, 99], status=binding.DEV_BOUNDS)


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_far_positions(sign):
    """The angle is formed as well at a million as at one."""
    at = np.array([0, 1, 4095.5, 65537, 1e6 + 1, 2 ** 22 - 1], np.float32)[None, :, None].repeat(3, 2) * np.float32(sign)
    _run((16, 56, 56), 1, 6, 6, 2, 2, LAYOUTS[0], positions=at)


def test_pairs_that_are_not_turned_and_a_full_turn():
    f = [0.0] * 16 + [2 * np.pi] * 16
    _run((32, 32), 1, 9, 9, 2, 2, LAYOUTS[1], freq=f, positions=np.arange(18, dtype=np.float32).reshape(1, 9, 2))


def test_positions_that_are_not_finite_stay_in_their_row():
    import torch
    rng = np.random.default_rng(0)
    x = dev_bf16(_rand(rng, (1, 40, 2, 64)))
    at = np.ones((1, 40, 2), np.float32)
    f, axis = binding.rotary_frequencies((32, 32))
    want, got = torch.zeros_like(x), torch.zeros_like(x)
    binding.rotary_axes(x, None, _f32(at), f, axis, want, None, LAYOUTS[0])
    at[0, 7, 0] = np.nan
    at[0, 9, 1] = np.inf
    binding.rotary_axes(x, None, _f32(at), f, axis, got, None, LAYOUTS[0])
    keep = [i for i in range(40) if i not in (7, 9)]
    assert torch.equal(got[:, keep], want[:, keep])
    assert torch.isnan(got[0, 7, :, :32].float()).all() and torch.equal(got[0, 7, :, 32:], want[0, 7, :, 32:])


@pytest.mark.parametrize("layout", LAYOUTS, ids=["pairs", "halves"])
def test_in_place_parts_of_one_projection_and_back(layout):
    """Q and K as parts of one projection's rows, turned in place; turned back they are the rows again, but for two roundings."""
    import torch
    rng = np.random.default_rng(2)
    H, D, n = 3, 64, 300
    rows = dev_bf16(_rand(rng, (1, n, 3 * H * D)))
    old = rows.clone()
    q, k = (rows[:, :, i * H * D:(i + 1) * H * D].unflatten(-1, (H, D)) for i in (0, 1))
    at = _f32(rng.integers(0, 64, (1, n, 3)))
    f, axis = binding.rotary_frequencies((16, 24, 24))
    apart_q, apart_k = torch.empty((1, n, H, D), dtype=torch.bfloat16, device="cuda"), torch.empty((1, n, H, D), dtype=torch.bfloat16, device="cuda")
    binding.rotary_axes(q, k, at, f, axis, apart_q, apart_k, layout)
    binding.rotary_axes(q, k, at, f, axis, q, k, layout)
    assert torch.equal(q, apart_q) and torch.equal(k, apart_k) and torch.equal(rows[:, :, 2 * H * D:], old[:, :, 2 * H * D:])
    binding.rotary_axes(q, k, at, f, axis, q, k, layout, inverse=True)
    a, b = host_f64(rows), host_f64(old)
    pair = np.sqrt(np.abs(b) ** 2 + np.concatenate([_partner(b[:, :, :2 * H * D].reshape(1, n, 2 * H, D), layout == LAYOUTS[0]).reshape(1, n, -1),
                                                    b[:, :, 2 * H * D:] * 0], -1) ** 2)
    # two roundings: each element of a turned pair by 2^-8 of it (together 2^-8 of the pair), then the result's own
    assert np.all(np.abs(a - b) <= 2.0 ** -8 * pair * (1 + 2.0 ** -6) + 2.0 ** -8 * np.abs(b) * (1 + 2.0 ** -6) + 2.0 ** -14 * pair)


@pytest.mark.parametrize("layout", LAYOUTS, ids=["pairs", "halves"])
def test_the_same_as_the_table_form(layout):
    """What ``fresh_qkv`` gives with a table of the same angles, to a rounding: two bf16 numbers next to each other at most."""
    import torch
    rng = np.random.default_rng(3)
    B, places, cap, H, D = 2, 90, 33, 4, 128
    f, axis = binding.rotary_frequencies((16, 56, 56))
    at = rng.integers(0, 60, (1, places, 3)).astype(np.float32)
    angle = at[0].astype(np.float64)[:, axis] * np.asarray(f)
    idx = dev_i32(np.stack([np.sort(rng.permutation(places)[:cap]) for _ in range(B)]))
    n = dev_i32([cap, 20])
    q, k, v = (dev_bf16(_rand(rng, (B, places, H, D))) for _ in range(3))
    w = dev_bf16(synth.bf16_round(np.linspace(0.5, 1.5, D).astype(np.float32)))
    outs = [torch.zeros((B, cap, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(5)]
    binding.fresh_qkv(q, k, v, idx, n, w, w, EPS, _f32(np.cos(angle)), _f32(np.sin(angle)), layout, *outs[:3])
    binding.rotary_axes(q, k, _f32(at), f, axis, outs[3], outs[4], layout, idx=idx, n=n, q_weight=w, k_weight=w, eps=EPS)
    for a, b in ((outs[0], outs[3]), (outs[1], outs[4])):
        a, b = host_f64(a), host_f64(b)
        y = np.abs(a) + _partner(a, layout == LAYOUTS[0])
        assert np.all(np.abs(a - b) <= 2.0 ** -7 * np.abs(a) + 2.0 ** -16 * y)


def test_offsets_beyond_32_bits_streams_and_capture():
    import torch
    rng = np.random.default_rng(4)
    n, H, D, apart = 260, 2, 64, 1 << 24                               # 4.4e9 elements
    x = dev_bf16(_rand(rng, (1, n, H, D)))
    at = _f32(rng.integers(0, 64, (1, n, 3)))
    f, axis = binding.rotary_frequencies((16, 24, 24))
    want = torch.zeros_like(x)
    binding.rotary_axes(x, None, at, f, axis, want, None, LAYOUTS[1])
    wide = torch.empty(n * apart, dtype=torch.bfloat16, device="cuda").view(1, n, apart)
    far = wide[:, :, :H * D].unflatten(-1, (H, D))
    far.copy_(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    binding.rotary_axes(far, None, at, f, axis, far, None, LAYOUTS[1], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(far, want)
    del wide, far
    out = torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.rotary_axes(x, None, at, f, axis, out, None, LAYOUTS[1], stream=torch.cuda.current_stream())
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
