"""Arguments that tree attention refuses, beside those of tests/test_cache_abi.py (no GPU needed)."""
import pytest

from paper_2608_03447_gb300 import asd
from test_cache_abi import attend, cache


@pytest.mark.parametrize("scale,code", [(2.4e38, 4), (-2.4e38, 4), (3.4e38, 4), (2e38, 1), (-2e38, 1)])
def test_scales_whose_binary_form_is_not_finite(scale, code):
    """Scores are kept in units of log 2, 1.44 times the given ones; with an infinite factor a score of 0 would be NaN.
    (1: the next check, a missing pointer.)"""
    assert attend(asd.load(), cache(), scale=scale, q=None) == code
