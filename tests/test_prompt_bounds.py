"""Bounds of the calls that take many new tokens per sequence, on the host."""
import math

import pytest

from paper_2508_08256_amd import binding as B
from test_prompt_args import append, chunk, prefill


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_a_softmax_scale_that_has_no_logarithmic_form_is_refused(sign):
    """The kernels take sm_scale * log2(e): an infinity from 2^128 / log2(e) = 2.36e38 on."""
    for scale, status in ((2.35e38, B.OK), (2.37e38, B.EINVAL), (3.4e38, B.EINVAL), (math.inf, B.EINVAL)):
        c = B.make_config(2, 4, 2, 256, sm_scale=sign * scale)
        assert prefill(c, n=0) == chunk(c, n=0) == status, scale  # no tokens: nothing is launched
        assert append(c, n=0) == B.OK  # has no use for it
