"""Sizes and numbers at the ends of what the serving operators take, without a GPU."""
import ctypes
import math

import pytest

from paper_2602_03216_amd import binding as tsa
from tests.test_cache_host import _attend, _desc


def _code(desc):
    """0 where the descriptor is taken: the only thing wrong with the call is then that O is Q, which is looked at last."""
    rc = _attend(desc)
    return 0 if "O is Q" in tsa.tsa_last_error() else rc


@pytest.mark.parametrize("scale", [2.0 ** -149, 1.0e-39, 2.0 ** -101, 2.0 ** 31, 3.0e38])
def test_scales_that_32_bits_do_not_bear(scale):
    """Their inverse, or a logit that they make out of a product of 1, is too large."""
    assert _code(_desc(scale=scale)) == tsa.TSA_ERR_UNSUPPORTED
    assert tsa.load_library().tsa_attend_cache_workspace_bytes(ctypes.byref(_desc(scale=scale))) == 0


def test_scales_that_are_taken():
    for scale in (0.0, 2.0 ** -100, 1.0e-6, 64 ** -0.5, 1.0, 2.0 ** 30):
        assert _code(_desc(scale=scale)) == 0
    assert _code(_desc(scale=-1.0)) == _code(_desc(scale=math.nan)) == tsa.TSA_ERR_ARG
