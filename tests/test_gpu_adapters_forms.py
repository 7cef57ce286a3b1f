"""Forms of the product with adapters that the sizes choose beyond those of its own tests, against a product in 64 bits: pairs of CTAs in the first
launch of many rows, and for few rows a group pairs of CTAs whose slices of K meet.  Numbers and bounds are those of its own tests."""
import numpy as np
import pytest

from paper_2510_25590_b200 import synth
from test_gpu_adapters import OLD, Case, _streams, _tokens, _which

pytestmark = pytest.mark.gpu


def _want(c, scale=True, bias=True):
    """``Case.want`` with the products taken one by one in 64 bits on the device, where folding each adapter into its weights takes minutes."""
    import torch
    dev = lambda a: torch.from_numpy(np.asarray(a, np.float64)).cuda()
    out = torch.zeros((c.rows, c.N), dtype=torch.float64, device="cuda")
    x = dev(np.where(c.live[:, None], c.x, 0.0))
    for i in range(len(c.w)):
        w = dev(c.w[i])
        for g in range(i, len(c.ranges), len(c.w)):
            (b, e), a = c.ranges[g], c.which[g]
            y = x[b:e] @ w.T
            if a >= 0:
                y += (float(c.scale[a]) if scale else 1.0) * (x[b:e] @ dev(c.a[a]).T) @ dev(c.b[a]).T
            out[b:e] = y + (dev(c.bias[i]) if bias else 0.0)
    return out.cpu().numpy()


def _check(c, **kw):
    got, want = c.run(**kw), synth.bf16_round(_want(c, **kw).astype(np.float32)).astype(np.float64)
    assert np.all(got[~c.live] == OLD)
    assert np.array_equal(got[c.live], want[c.live])


# rows, ranges, weight sets, K, N, rank, adapters
MANY = [(8802, _streams(2, 301, 4100, [3333, 4099]), 2, 2048, 256, 256, 4), (12003, [(0, 1), (1, 4000), (4001, 4001), (4001, 9000), (9003, 12003)], 1, 512, 264, 200, 3),
        (20001, _streams(1, 1001, 19000, [18999]), 2, 512, 136, 256, 5), (2000, _streams(1, 77, 1923, [1900]), 1, 8192, 512, 64, 2)]
FEW = [(300, _tokens(300), 1, 4096, 2048, 16, 7), (256, _tokens(256), 1, 4096, 3000, 24, 40), (128, _tokens(128), 1, 8192, 4096, 8, 3),
       (500, _tokens(500), 1, 1024, 4096, 64, 9), (1200, [(2 * i, 2 * i + 2) for i in range(500)], 1, 1024, 1024, 16, 5)]


@pytest.mark.parametrize("shape", MANY + FEW, ids=lambda s: f"{s[0]}x{s[3]}x{s[4]}r{s[5]}g{len(s[1])}")
def test_whole_numbers_are_exact(shape):
    c = Case(*shape[:6], shape[6], _which(np.random.default_rng(shape[0]), len(shape[1]), shape[6]))
    _check(c)


@pytest.mark.parametrize("rows", [(1, 1, 400, 2, 3, 30), (150, 1, 1, 1)], ids=str)
def test_uneven_groups_of_few_rows(rows):
    """One group has most of the rows: of its adapter, of two groups with the same, of none."""
    ends = np.cumsum(rows)
    ranges = [(int(e - n), int(e)) for n, e in zip(rows, ends)] + [(int(ends[-1]),) * 2] * 30
    for which in ([0, 1, 1, -1, 0, 1], [0, 0, -1, 0, 1, 0], [1, 0, 0, 0, 0, 0]):
        c = Case(int(ends[-1]), ranges, 1, 264, 520, 24, 2, (which * 40)[:len(ranges)])
        _check(c)
