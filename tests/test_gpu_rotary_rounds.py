"""Rotary positions of more rows than there are warps, so that a warp goes through several: the angles of the row before are written over, the
factors begin with Q again, rows without a place or behind a count lie between."""
import numpy as np
import pytest

from paper_2510_25590_b200 import binding
from test_gpu_rotary_axes import LAYOUTS, _run

pytestmark = pytest.mark.gpu


def _rows():
    import torch
    return 70 * torch.cuda.get_device_properties(0).multi_processor_count       # resident: 24 warps an SM at most


WIDTHS = [(64,), (16, 24, 24), (32, 32, 32), (16, 56, 56), (8, 8, 32)]


@pytest.mark.parametrize("layout", LAYOUTS, ids=["pairs", "halves"])
@pytest.mark.parametrize("widths", WIDTHS, ids=lambda w: "_".join(map(str, w)))
@pytest.mark.parametrize("Hq,Hk", [(3, 2), (1, 0)])
def test_many_rows_of_few_heads(widths, layout, Hq, Hk):
    _run(widths, 1, _rows() + 3, _rows() + 3, Hq, Hk, layout)
    _run(widths, 1, _rows() + 3, _rows() + 3, Hq, Hk, layout, False, inverse=True)


@pytest.mark.parametrize("layout", LAYOUTS, ids=["pairs", "halves"])
@pytest.mark.parametrize("widths", [(16, 24, 24), (32, 32, 32), (16, 56, 56)], ids=lambda w: "_".join(map(str, w)))
@pytest.mark.parametrize("compact", [True, False])
def test_rows_that_are_left_out_between_others(widths, layout, compact):
    rng = np.random.default_rng(9)
    cap, places = _rows() // 5, 5000
    idx = rng.integers(0, places, (5, cap))
    idx[rng.random((5, cap)) < 0.3] = -1
    idx[rng.random((5, cap)) < 0.1] = places
    _run(widths, 5, places, cap, 3, 2, layout, idx=idx, n=[cap, cap // 3, 0, 1, cap - 1], compact=compact, status=binding.DEV_BOUNDS)
