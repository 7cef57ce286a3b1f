"""Pins of the oracle's layer norm, rotary positions with several axes and products with adapters that are not their own formulas (CPU only)."""
import numpy as np
import pytest
import torch

from oracle import regione_oracle as orc

RANGES = [(0, 3), (3, 3), (5, 9)]


@pytest.mark.parametrize("modulated", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_layer_norm_and_its_gradients_against_a_library(modulated, gated):
    """Forward, and every gradient by automatic differentiation in 64 bits."""
    rng = np.random.default_rng(0)
    rows, C, sets = 9, 24, 2
    x, r, dy, dz = (rng.standard_normal((rows, C)) for _ in range(4))
    w, b, q = (rng.standard_normal((sets, C)) for _ in range(3))
    z, out, mean, rstd = orc.layer_norm(x, w, b, RANGES, 1e-5, modulated, r if gated else None, q if gated else None)
    tx, tr, tw, tb, tq = (torch.tensor(v, requires_grad=True) for v in (x, r, w, b, q))
    total = 0.0
    for g, (lo, hi) in enumerate(RANGES):
        if hi == lo:
            continue
        i = g % sets
        row = tx[lo:hi] + (tq[i] * tr[lo:hi] if gated else 0.0)
        y = torch.nn.functional.layer_norm(row, (C,), tw[i] + (1.0 if modulated else 0.0), tb[i], 1e-5)
        assert np.allclose(out[lo:hi], y.detach().numpy(), atol=1e-12) and np.allclose(z[lo:hi], row.detach().numpy(), atol=1e-14)
        total = total + (y * torch.tensor(dy[lo:hi])).sum() + (row * torch.tensor(dz[lo:hi])).sum()
    total.backward()
    dx, dr, dw, db, dq = orc.layer_norm_backward(z, mean, rstd, dy, w, RANGES, sets, modulated, dz, r if gated else None, q if gated else None)
    live = np.array([any(lo <= i < hi for lo, hi in RANGES) for i in range(rows)])
    assert np.allclose(dx[live], tx.grad.numpy()[live], atol=1e-11) and np.all(dx[~live] == 0)
    assert np.allclose(dw, tw.grad.numpy(), atol=1e-11) and np.allclose(db, tb.grad.numpy(), atol=1e-11)
    if gated:
        assert np.allclose(dr, tr.grad.numpy(), atol=1e-11) and np.allclose(dq, tq.grad.numpy(), atol=1e-11)


def test_layer_norm_gradient_by_differences():
    rng = np.random.default_rng(1)
    x, w, dy = rng.standard_normal((2, 16)), rng.standard_normal((1, 16)), rng.standard_normal((2, 16))
    value = lambda x, w: (orc.layer_norm(x, w, None, [(0, 2)], 1e-6)[1] * dy).sum()
    z, _, mean, rstd = orc.layer_norm(x, w, None, [(0, 2)], 1e-6)
    dx, _, dw, _, _ = orc.layer_norm_backward(z, mean, rstd, dy, w, [(0, 2)], 1)
    h = 1e-6
    for at in np.ndindex(x.shape):
        d = np.zeros_like(x); d[at] = h
        assert abs((value(x + d, w) - value(x - d, w)) / (2 * h) - dx[at]) < 1e-7
    for at in np.ndindex(w.shape):
        d = np.zeros_like(w); d[at] = h
        assert abs((value(x, w + d) - value(x, w - d)) / (2 * h) - dw[at]) < 1e-7


@pytest.mark.parametrize("interleaved", [True, False])
def test_rotary_axes(interleaved):
    rng = np.random.default_rng(2)
    D = 32
    freq = list(10000.0 ** (-2.0 * np.arange(4) / 8)) + list(10000.0 ** (-2.0 * np.arange(12) / 24))
    axis = [0] * 4 + [1] * 12
    x = rng.standard_normal((5, 3, D))
    at = rng.integers(0, 50, (5, 2)).astype(float)
    y = orc.rotary_axes(x, at, freq, axis, interleaved)
    # one axis with the table form
    cos, sin = (f(at[:, axis] * np.asarray(freq))[:, None] for f in (np.cos, np.sin))
    assert np.allclose(y, orc.rope(x, cos, sin, orc.ROPE_INTERLEAVED if interleaved else orc.ROPE_HALF), atol=1e-13)
    # a turn and back; lengths stay
    assert np.allclose(orc.rotary_axes(y, at, freq, axis, interleaved, inverse=True), x, atol=1e-13)
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    # products of two rows depend on the difference of their places alone, axis by axis
    k = rng.standard_normal((5, 3, D))
    score = lambda a, b: (orc.rotary_axes(x, a, freq, axis, interleaved) * orc.rotary_axes(k, b, freq, axis, interleaved)).sum(-1)
    there = at + rng.integers(0, 9, at.shape)
    assert np.allclose(score(at, there), score(at + [3, 11], there + [3, 11]), atol=1e-10)
    assert not np.allclose(score(at, there), score(at + [3, 11], there + [11, 3]), atol=1e-3)
    # the gradient of the rotation is the rotation back
    g = rng.standard_normal(x.shape)
    h = 1e-6
    back = orc.rotary_axes(g, at, freq, axis, interleaved, inverse=True)
    for where in [(0, 0, 0), (1, 2, 5), (4, 1, 31), (2, 0, 16)]:
        d = np.zeros_like(x); d[where] = h
        num = ((orc.rotary_axes(x + d, at, freq, axis, interleaved) - orc.rotary_axes(x - d, at, freq, axis, interleaved)) * g).sum() / (2 * h)
        assert abs(num - back[where]) < 1e-8


def test_adapters_step_by_step():
    rng = np.random.default_rng(3)
    x, w, bias = rng.standard_normal((9, 16)), rng.standard_normal((2, 24, 16)), rng.standard_normal((2, 24))
    a, b, s = rng.standard_normal((3, 8, 16)), rng.standard_normal((3, 24, 8)), np.array([0.5, 2.0, -1.0])
    out = orc.adapter_matmul(x, w, a, b, [2, 0, -1], RANGES, s, bias)
    for r in range(9):
        g = next((g for g, (lo, hi) in enumerate(RANGES) if lo <= r < hi), None)
        if g is None:
            assert np.all(out[r] == 0)
            continue
        want = w[g % 2] @ x[r] + bias[g % 2]
        j = [2, 0, -1][g]
        if j >= 0:
            want = want + s[j] * (b[j] @ (a[j] @ x[r]))
        assert np.allclose(out[r], want, atol=1e-12)
    gelu = orc.adapter_matmul(x, w, a, b, [2, 0, -1], RANGES, s, bias, gelu=True)
    live = [r for lo, hi in RANGES for r in range(lo, hi)]
    assert np.allclose(gelu[live], torch.nn.functional.gelu(torch.tensor(out[live]), approximate="tanh").numpy(), atol=1e-12)
