"""Frequencies and axes that are no numbers of their types, on the host (CPU only: stand-ins for the tensors and for the library)."""
import pytest

from paper_2510_25590_b200 import binding
from test_binding_block import D, _args
from test_binding_products import called    # noqa: F401  (a fixture)


@pytest.mark.parametrize("kw", [dict(axis=[2 ** 31] * (D // 2)), dict(axis=[-2 ** 40] * (D // 2)), dict(freq=[10 ** 400] * (D // 2)),
                                dict(freq=[None] * (D // 2)), dict(axis=[0.0] * (D // 2)), dict(freq=3.0), dict(axis=None)],
                         ids=["axis of 33 bits", "axis of 41 bits", "freq beyond a double", "freq of None", "axis of floats", "one freq", "no axis"])
def test_what_is_no_number_ends_in_the_librarys_own_error(called, kw):
    with pytest.raises(binding.RegionEError):
        binding.rotary_axes(**_args("rotary_axes", **kw))
    assert not called


@pytest.mark.parametrize("kw", [dict(axis=[2 ** 31 - 1] * (D // 2)), dict(axis=[True] * (D // 2)), dict(freq=[1] * (D // 2))],
                         ids=["largest axis", "truth values", "whole frequencies"])
def test_numbers_of_other_kinds_reach_the_library(called, kw):
    binding.rotary_axes(**_args("rotary_axes", **kw))
    assert called == ["regione_rotary_axes"]
