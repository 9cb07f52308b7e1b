"""Attention next to unseen tokens whose values are far larger."""
import numpy as np
import pytest

import oracle
import paper_2410_12168_amd as comet
from paged_ref import Paged, check_attention, to16
from test_gpu_serving import dev16, handles, host16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kvh,H", [(7, 2, 8), (60, 8, 32)])
@pytest.mark.parametrize("window", [0, 40])
def test_larger_scales_that_a_row_does_not_see(n, kvh, H, window):
    """The last token's values (and, with a window, an early one's) are 2^12 times as large.  A
    weight times a scale goes in steps of 2^-34 of the largest one at least (2^-24 over the
    largest scale's 2^10): half of one, times a code's distance from 8, over the 100 tokens, is
    100 * 2^-35 * 8 of the largest scale, 2^-13 of a scale here, where the bounds allow 2^-11 of
    the values of 8 scales and more."""
    p = Paged(97 + n + window, [(n, 100)], kvh, 128, 64, 16)
    big = [99] + ([100 - n - window - 1] if window and 100 - n - window - 1 >= 0 else [])
    rows = to16(0.5 * p.rng.standard_normal((100, kvh, 128)))
    rows[big] = to16(2048.0 * np.clip(p.rng.standard_normal((len(big), kvh, 128)), -3, 3))
    c, prm = oracle.kv4_quantize(rows.reshape(-1, 128), 64)
    p.store(1, 0, np.arange(100), c.reshape(100, kvh, -1), prm.reshape(100, kvh, 2, 2))
    cache, batch = handles(p)
    q16 = to16(p.rng.standard_normal((n, H, 128)))
    out = host16(comet.kv4_attention(dev16(q16), cache, batch, window=window))
    ref, bound = p.attention(q16, H, 128 ** -0.5, window)
    check_attention(out[:-1], ref[:-1], bound[:-1])
    check_attention(out[-1:], ref[-1:], bound[-1:])
