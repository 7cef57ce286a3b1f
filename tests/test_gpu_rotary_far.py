"""Rotary positions whose angles are many turns: what is stated of them is a limit of the product of position and frequency, whichever of the two
is the large one."""
import numpy as np
import pytest

from gpu_util import dev_bf16, host_f64
from oracle import regione_oracle as orc
from paper_2510_25590_b200 import binding
from test_gpu_rotary_axes import LAYOUTS, _f32, _partner, _rand, _run

pytestmark = pytest.mark.gpu


def _places(rng, turns, log_freq, sign):
    """Frequencies of up to 2^log_freq turns a unit and positions, whose products are up to 2^turns turns."""
    freq = [float(f) for f in 2 * np.pi * 2.0 ** log_freq * rng.uniform(0.5, 1.0, 32)]
    return freq, (rng.uniform(0.5, 1.0, (1, 64, 2)) * 2.0 ** (turns - log_freq)).astype(np.float32) * np.float32(sign)


@pytest.mark.parametrize("log_freq", [0, 10, 20])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_angles_are_exact_to_2_23_turns(log_freq, sign):
    freq, at = _places(np.random.default_rng(log_freq), 23, log_freq, sign)
    _run((32, 32), 1, 64, 64, 2, 2, LAYOUTS[0], freq=freq, positions=at)


@pytest.mark.parametrize("turns,log_freq", [(26, 3), (26, 20), (32, 10), (32, 20), (36, 20)])
def test_angles_beyond_are_off_by_2_45_of_themselves(turns, log_freq):
    """The output moves by what the angle is off times the other element of the pair, beside its rounding and what the tests of nearer
    places allow.  (The oracle's angles, of 53 bits, are off by 2^-8 of that.)"""
    rng = np.random.default_rng(turns)
    freq, at = _places(rng, turns, log_freq, 1.0)
    x = _rand(rng, (1, 64, 2, 64))
    out = dev_bf16(0 * x)
    binding.rotary_axes(dev_bf16(x), None, _f32(at), freq, [0] * 16 + [1] * 16, out, None, LAYOUTS[0])
    want = orc.rotary_axes(x[0], at[0], freq, [0] * 16 + [1] * 16, True)
    both = np.abs(x[0]) + _partner(x[0], True)
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -17 + 2 * np.pi * 2.0 ** (turns - 45) * (1 + 2.0 ** -8)) * both
    assert np.all(np.abs(host_f64(out)[0] - want) <= tol)
