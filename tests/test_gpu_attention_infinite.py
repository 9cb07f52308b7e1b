"""Attention of queries that are not finite: not-a-number where the row sees a token."""
import numpy as np
import pytest

import oracle
import paper_2410_12168_amd as comet
from paged_ref import Paged, check_attention, f64, kv_rows, to16
from test_gpu_serving import dev16, handles, host16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kvh,H", [(3, 2, 4), (60, 8, 32)])
@pytest.mark.parametrize("bits", [0x7C00, 0xFC00, 0x7E00])
def test_a_query_that_is_not_finite(n, kvh, H, bits):
    """Keys above zero, so that the scores of an infinite query are all infinities of one
    sign: the softmax of those is not-a-number, whichever it is.  The second sequence's first
    rows see nothing: zeros, as of any query."""
    D = 64
    p = Paged(81 + n, [(n, 100), (n, n - 2)], kvh, D, 64, 16)
    for b, L in ((0, 100), (1, n - 2)):
        rows = np.abs(f64(kv_rows(p.rng, L, kvh, D))) + 0.5
        c, prm = oracle.kv4_quantize(to16(rows).reshape(L * kvh, D), 64)
        p.store(0, b, np.arange(L), c.reshape(L, kvh, -1), prm.reshape(L, kvh, 1, 2))
    q16 = to16(p.rng.standard_normal((2 * n, H, D)))
    ref, bound = p.attention(q16, H, D ** -0.5)
    bad = q16.copy()
    hit = np.zeros((2 * n, H), bool)
    for m, h, c in ((0, 1, 5), (n - 1, 0, 63), (n, 2, 0), (n + 1, 1, 9), (2 * n - 1, 3, 31)):
        bad[m, h, c] = bits
        hit[m, h] = True
    cache, batch = handles(p, max_rows=n)
    out = host16(comet.kv4_attention(dev16(bad), cache, batch))
    blind = np.array([pos < 0 for _, _, pos in p.rows()])
    assert blind.sum() == 2 and hit[blind].any()
    assert not out[blind].any()
    seen = hit & ~blind[:, None]
    assert np.isnan(f64(out[seen])).all()
    check_attention(out[~seen], ref[~seen], bound[~seen])
