"""Attention of queries whose channels differ by 2^22."""
import numpy as np
import pytest

import oracle
import paper_2410_12168_amd as comet
from paged_ref import Paged, check_attention, to16
from test_gpu_serving import dev16, handles, host16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kvh,H", [(3, 2, 4), (60, 8, 32)])
@pytest.mark.parametrize("D,G", [(128, 32), (128, 64), (64, 32)])
@pytest.mark.parametrize("at", [0, 1])
def test_channels_far_below_the_largest(n, kvh, H, D, G, at):
    """One channel of q is 6e4, where the keys of its group are zeros; the others, 2^-22 of
    that, make the scores with keys of about 1000.  None of their bits is lost."""
    p = Paged(101 + n + D + G, [(n, 150)], kvh, D, G, 16)
    rows = 600.0 * p.rng.standard_normal((150, kvh, D))
    rows[..., :G] = 0.0
    c, prm = oracle.kv4_quantize(to16(rows).reshape(-1, D), G)
    p.store(0, 0, np.arange(150), c.reshape(150, kvh, -1), prm.reshape(150, kvh, D // G, 2))
    q = 0.0143 * p.rng.uniform(0.5, 1.0, (n, H, D)) * p.rng.choice([-1.0, 1.0], (n, H, D))
    q[..., at] = 6e4
    q16 = to16(q)
    cache, batch = handles(p)
    out = host16(comet.kv4_attention(dev16(q16), cache, batch))
    some = np.arange(0, n, max(1, n // 12))
    ref, bound = p.attention(q16, H, D ** -0.5, rows=some)
    check_attention(out[some], ref[some], bound[some])
