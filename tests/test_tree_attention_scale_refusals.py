"""Factors of the scores that dspark_tree_attention refuses (no GPU needed: nothing is launched)."""
import pytest

from test_tree_refusals import INVALID, attend, cache


@pytest.mark.parametrize("scale", [3e38, -3e38, float("inf"), float("-inf"), float("nan")])
def test_factors_past_the_range(scale):
    assert attend(cache(), scale=scale) == INVALID
