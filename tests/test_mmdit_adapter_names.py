"""Adapters of the stand-in stack under names that no product of it has are refused and not left out (CPU only: before anything is laid out)."""
import pytest

from paper_2510_25590_b200 import binding
from paper_2510_25590_b200.mmdit_scaffold import MMDiTScaffold


@pytest.mark.parametrize("name", ["qkv0", "q2", "fc1_0_1", "mod2", "mod0_1", "q-1", "o"])
def test_names_of_no_product(name):
    with pytest.raises(binding.RegionEError, match=name):
        MMDiTScaffold({}, 1, 4, 0, 2, 64, 2, None, None, None, None, products="grouped", adapters=({"q0": None, name: None}, None, None))


def test_names_of_the_products():
    """All of them come as far as what the stack is built from, which is not there."""
    names = [f"{name}{l}" for l in (0, 1) for name in ("q", "k", "v", "o", "fc1_", "fc2_", "mod")]
    with pytest.raises(AttributeError):
        MMDiTScaffold({}, 1, 4, 0, 2, 64, 2, None, None, None, None, products="grouped", adapters=(dict.fromkeys(names), None, None))
