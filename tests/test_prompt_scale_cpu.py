"""Softmax scales that prompt attention and masses refuse: 0 stands for 1/sqrt(head_dim), and nothing else does."""
import math

import pytest

from paper_2608_23599_b200 import binding as B
from tests.test_rows_refusals_cpu import attn, desc, mass, room


@pytest.mark.parametrize("scale", [-0.088, math.nan, math.inf, -math.inf, 1e-42, -1e-42])
def test_scales_that_are_refused(scale):
    d = desc(softmax_scale=scale)
    assert attn(d) == mass(d) == room(d)[0] == B.ERR_INVALID_ARG


@pytest.mark.parametrize("scale", [0.0, -0.0, 1.0, 1e-30])
def test_scales_that_are_taken(scale):
    assert room(desc(softmax_scale=scale))[0] == B.OK
