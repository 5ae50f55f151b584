"""Frequencies that are asked for in a way that contradicts itself."""
import pytest

from paper_2602_02987_amd import calibrate as K
from paper_2602_02987_amd import iteration as I


@pytest.mark.parametrize("factor", [8.0, 0.5])
def test_a_factor_without_a_scaling_is_refused(factor):
    with pytest.raises(ValueError, match="factor"):
        I.rotary_frequencies(128, factor=factor)
    with pytest.raises(ValueError, match="factor"):
        K.Positions(factor=factor).turns(128, "cpu")
    assert I.rotary_frequencies(128, factor=1.0) == I.rotary_frequencies(128) == I.rotary_frequencies(128, scaling="linear", factor=1)
