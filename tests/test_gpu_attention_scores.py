"""Attention where the scores are far beyond the ordinary: products of large queries and
keys, whose softmax is the value of one token, and queries that are not finite."""
import numpy as np
import pytest
import torch

import oracle
import paper_2410_12168_amd as comet
from paged_ref import HALF_STEP, Paged, f64, to16
from test_gpu_serving import dev16, handles, host16

pytestmark = pytest.mark.gpu

# (rows, kv heads, heads): the kernel for few rows, and the one for many
KERNELS = [(3, 2, 4), (60, 8, 32)]


def store_keys(p, b, exponents, sign):
    """Keys of sequence b: 6e4 * 2^exponent in every channel, with the channel's sign."""
    L = len(exponents)
    rows = 6e4 * np.exp2(exponents)[:, None, None] * np.broadcast_to(sign, (L, p.kvh, p.D))
    c, prm = oracle.kv4_quantize(to16(rows).reshape(L * p.kvh, p.D), p.G)
    p.store(0, b, np.arange(L), c.reshape(L, p.kvh, -1), prm.reshape(L, p.kvh, p.D // p.G, 2))


def decided(p, q16, H, scale, m, b, pos):
    """Per head of row m: the value of the token with the largest score, and what the output
    may be off by, where that score is further above the others than 32-bit sums can
    be off (else None)."""
    q, R, js = f64(q16), H // p.kvh, np.arange(pos + 1)
    (kc, ks, km), (vc, vs, vm) = p.tokens(0, b, js), p.tokens(1, b, js)
    out = []
    for h in range(H):
        g = h // R
        x = scale * (ks[:, g] * kc[:, g] + km[:, g]) @ q[m, h]
        terms = np.abs(scale * q[m, h]) * (ks[:, g] * kc[:, g] + np.abs(km[:, g]))
        # the rounding of a score: D + 16 steps of 2^-24 on terms of this size (the running
        # maximum is one of the scores, and differences to it are exact or as far off)
        off = (terms.sum(axis=1) * (p.D + 16) + 2 * np.abs(x)) * 2.0 ** -24
        best = int(np.argmax(x))
        others = np.delete(x + off, best)
        # the others' weights, e^-40 each, are nothing next to a rounding
        if len(others) and x[best] - off[best] - others.max() < 40:
            out.append(None)
            continue
        v = vs[best, g] * vc[best, g] + vm[best, g]
        # one weight of 1: its product with the scale and the output are rounded to fp16
        size = vs[best, g] * vc[best, g] + np.abs(vm[best, g])
        out.append((v, HALF_STEP * np.abs(v) + 2.0 ** -25 + (HALF_STEP + 2.0 ** -20) * size))
    return out


@pytest.mark.parametrize("n,kvh,H", KERNELS)
@pytest.mark.parametrize("order", ["rising", "falling", "peak"])
@pytest.mark.parametrize("D,G,size", [(128, 128, 6e4), (128, 32, 6e4), (64, 64, 6e4),
                                      (128, 64, 300.0), (128, 128, 3.0)])
def test_large_scores_give_the_largest_ones_value(n, kvh, H, order, D, G, size):
    # scores up to 4e10 for the largest queries, over 2^24 of a range within the sequence
    L = 400 if order == "peak" else 100
    j = np.arange(L)
    exponents = {"rising": -(L - 1 - j) / 4, "falling": -j / 4,
                 "peak": -np.abs(j - 200.3) / 8}[order]
    p = Paged(71 + n + D + G, [(n, L)], kvh, D, G, 16)
    sign = p.rng.choice([-1.0, 1.0], D)
    store_keys(p, 0, exponents, sign)
    q16 = to16(size * sign * p.rng.uniform(0.5, 1.0, (n, H, 1)))
    cache, batch = handles(p)
    print(f"large scores {n} {order} {D} {G} {size}", flush=True)
    out = f64(host16(comet.kv4_attention(dev16(q16), cache, batch)))
    assert np.all(np.isfinite(out))
    checked = 0
    for m, b, pos in p.rows():
        if m % 7 and m != n - 1:
            continue
        for h, want in enumerate(decided(p, q16, H, D ** -0.5, m, b, pos)):
            if want is not None:
                assert np.all(np.abs(out[m, h] - want[0]) <= want[1]), (m, h)
                checked += 1
    assert checked >= H


@pytest.mark.parametrize("n,kvh,H", KERNELS)
@pytest.mark.parametrize("scale", [-1.0, 2.0 ** 50])
def test_large_scales(n, kvh, H, scale):
    p = Paged(73 + n, [(n, 90)], kvh, 64, 32, 16)
    sign = p.rng.choice([-1.0, 1.0], 64)
    store_keys(p, 0, -np.arange(90) / 8, sign)
    q16 = to16(1e4 * sign * p.rng.uniform(0.5, 1.0, (n, H, 1)))
    cache, batch = handles(p)
    out = f64(host16(comet.kv4_attention(dev16(q16), cache, batch, scale=scale)))
    assert np.all(np.isfinite(out))
    for m, b, pos in p.rows():
        for h, want in enumerate(decided(p, q16, H, scale, m, b, pos)):
            assert want is not None and np.all(np.abs(out[m, h] - want[0]) <= want[1]), (m, h)
