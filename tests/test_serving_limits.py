"""Limits of the operators around the paged cache (no GPU: refused calls launch nothing, the
others run against hip_record's stand-in)."""
import math

import pytest

import hip_record
import paper_2410_12168_amd as comet
from test_serving_host import attend, batch, cache


@pytest.mark.parametrize("scale", [2.0 ** 57, -2.0 ** 57, 1e38, -3e38])
def test_scales_whose_scores_pass_the_running_maximum(scale):
    # 2^56 times the largest product of fp16 rows in 128 channels is 9e29 as a power of two,
    # and the running maximum starts at -1e30
    assert 128 * 65504.0 * 16 * 65504.0 * 2.0 ** 56 / math.log(2) < 1e30
    assert attend(cache(), batch(), scale=scale) == 2
    assert "scale" in comet.comet_last_error()
