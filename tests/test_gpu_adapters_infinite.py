"""Infinite elements of the adapters' second factors: times a sum x A^T they are what the formula says, whatever parts that sum is taken apart into."""
import numpy as np
import pytest

from test_gpu_adapters import Case
from test_gpu_adapters_sums import SHAPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[3]}x{s[4]}r{s[5]}")
@pytest.mark.parametrize("whole", [True, False])
def test_infinite_second_factors(shape, whole):
    """Infinite where the sum is not zero, of its sign, and NaN where it is zero: whatever parts a sum is taken apart into."""
    c = Case(*shape[:6], shape[6], [(i + 1) % 3 for i in range(len(shape[1]))], whole=whole)
    c.b[1, 7, 2], c.b[1, 33, 0], c.b[1, 100, 9], c.b[2, 5, 1] = np.inf, -np.inf, np.inf, -np.inf
    got = c.run()
    with np.errstate(invalid="ignore"):
        want = c.want()
        for (b, e), j in zip(c.ranges, c.which):                       # (the oracle's folded weights do not know the order of the products)
            for f in range(c.N):
                if not np.all(np.isfinite(c.b[j, f])):
                    u = c.x[b:e].astype(np.float64) @ c.a[j].T.astype(np.float64)
                    want[b:e, f] = u @ c.b[j, f].astype(np.float64)
    odd = ~np.isfinite(want)
    assert odd.any() and np.isposinf(want).any() and np.isneginf(want).any() and (not whole or np.isnan(want).any())
    assert np.array_equal(got[odd], want[odd], equal_nan=True)
    assert np.all(np.isfinite(got[~odd]))
