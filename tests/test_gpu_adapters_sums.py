"""What the sums x A^T are in the product with adapters: in front of the second factor as good as fp32 for an output in bf16, whether rows are
few or many.

Bound: an output is off by half a bf16 step, 2^-8 |y|, by K + rank additions that each lose at most 2^-23 of the sum of magnitudes, and by
what a sum loses where it is taken apart into bf16 numbers, 2^-15 of it."""
import numpy as np
import pytest

from test_gpu_adapters import Case, _tokens

pytestmark = pytest.mark.gpu

# few rows a group; many, whose sums one CTA takes, slices of K that meet, or a pair of CTAs
SHAPES = [(48, _tokens(48), 1, 64, 136, 16, 3), (900, [(0, 300), (300, 600), (600, 900)], 1, 64, 136, 16, 3), (700, [(0, 300), (300, 700)], 1, 256, 520, 16, 3),
          (9000, [(0, 4501), (4501, 9000)], 1, 128, 136, 200, 3), (2000, [(0, 2000)], 1, 2048, 136, 64, 3)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[3]}x{s[4]}r{s[5]}")
def test_sums_that_nearly_cancel(shape):
    """Ranks in pairs that are nearly alike, with second factors of opposite sign: what is left is far below a bf16 step of the sums."""
    c = Case(*shape[:6], shape[6], [(i + 1) % 3 for i in range(len(shape[1]))], whole=False)
    c.w[:], c.bias[:] = 0.0, 0.0
    c.a[:, 1::2] = c.a[:, ::2]
    c.a[:, 1::2, :8] = 0.0                                             # (what is left: eight of K's terms)
    c.b[:, :, 1::2] = -c.b[:, :, ::2]
    got, want = c.run(), c.want()
    x = c.x.astype(np.float64)
    tol = 2.0 ** -8 * np.abs(want)
    for (b, e), j in zip(c.ranges, c.which):
        u, terms = (c.scale[j] * (f(x[b:e]) @ f(c.a[j].T.astype(np.float64))) for f in (lambda v: v, np.abs))
        tol[b:e] += (2.0 ** -15 * np.abs(u) + 1.01 * (c.K + c.rank) * 2.0 ** -23 * terms) @ np.abs(c.b[j].T.astype(np.float64))
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)
