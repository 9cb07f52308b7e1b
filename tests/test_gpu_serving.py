"""Rotary positions, the paged 4-bit cache and attention over it on the GPU, against
64-bit references on the CPU (paged_ref.py) and the oracle's quantizer."""
import numpy as np
import pytest
import torch

import oracle
import paper_2410_12168_amd as comet
from paged_ref import Paged, check_attention, f64, kv_rows, to16

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev16(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(DEV).view(torch.float16)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def host16(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def handles(p, M=None, max_rows=None):
    cache = comet.KV4Cache(dev(p.codes[0]), dev16(p.params[0]), dev(p.codes[1]), dev16(p.params[1]))
    batch = comet.KV4Batch(dev(p.row_start), dev(p.lens), dev(p.table), M or p.M, max_rows)
    return cache, batch


# --- rotary positions ----------------------------------------------------------------

def rope_ref(x16, pos, freqs, interleaved, mscale):
    """(out, bound) fp64."""
    x = f64(x16)
    half = freqs.size
    a = np.outer(pos.astype(np.float64), freqs)[:, None]
    c, s = mscale * np.cos(a), mscale * np.sin(a)
    i = np.arange(half)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    out = x.copy()
    out[..., ia] = x[..., ia] * c - x[..., ib] * s
    out[..., ib] = x[..., ib] * c + x[..., ia] * s
    # sine and cosine to 4 steps of 32 bits, two products and a sum, one rounding to fp16
    size = np.zeros_like(x)
    size[..., ia] = size[..., ib] = np.abs(x[..., ia]) + np.abs(x[..., ib])
    return out, 2.0 ** -11 * np.abs(out) + 2.0 ** -25 + 8 * 2.0 ** -24 * abs(mscale) * size


@pytest.mark.parametrize("M,heads,D,rot,pad,interleaved", [
    (1, 40, 128, 128, 8, False), (1, 1, 64, 64, 0, True), (7, 5, 128, 64, 1, True),
    (3, 9, 128, 32, 2, False), (513, 3, 64, 16, 0, False), (2, 2, 80, 80, 0, True),
    (5, 3, 72, 48, 0, False), (4, 2, 96, 36, 1, False), (4, 2, 10, 6, 1, True),
    (3, 1, 2, 2, 0, False), (2, 2, 1024, 1024, 0, False), (300, 40, 128, 128, 8, True),
    (2, 600, 8, 2, 0, False)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rope(M, heads, D, rot, pad, interleaved, in_place):
    rng = np.random.default_rng(M + heads + D + rot)
    x16 = to16(rng.standard_normal((M, heads + pad, D)))
    pos = rng.integers(0, 1 << 20, M).astype(np.int32)
    pos[0] = (0, 1, -5, 2 ** 31 - 1)[M % 4]
    freqs, _ = comet.rope_frequencies(rot, 500000.0)
    mscale = 1.0 if M % 2 else 1.25
    buf = dev16(x16)
    x = buf[:, :heads]
    out = x if in_place else None
    print(f"rope {M} {heads} {D} {rot} {interleaved} {in_place}", flush=True)
    y = comet.rope(x, dev(pos), dev(freqs), interleaved=interleaved, mscale=mscale, out=out)
    ref, bound = rope_ref(x16[:, :heads], pos, freqs, interleaved, mscale)
    got = f64(host16(y))
    assert np.all(np.abs(got - ref) <= bound)
    assert np.array_equal(host16(y)[..., rot:], x16[:, :heads, rot:])
    if pad:  # the other columns of the buffer
        assert np.array_equal(host16(buf[:, heads:]), x16[:, heads:])
    if not in_place:
        assert np.array_equal(host16(x), x16[:, :heads])


@pytest.mark.parametrize("offset", [1, 4])
def test_rope_of_unaligned_rows(offset):
    # rows of odd length from an odd element on, out of another alignment
    M, heads, D = 6, 2, 64
    rng = np.random.default_rng(offset)
    flat = to16(rng.standard_normal(M * (heads * D + 3) + 8))
    x = dev16(flat)[offset:offset + M * (heads * D + 3)].view(M, -1)[:, :heads * D]
    x = x.unflatten(1, (heads, D))
    pos = np.arange(M, dtype=np.int32) * 1000
    freqs, _ = comet.rope_frequencies(D)
    y = comet.rope(x, dev(pos), dev(freqs))
    ref, bound = rope_ref(host16(x), pos, freqs, False, 1.0)
    assert np.all(np.abs(f64(host16(y)) - ref) <= bound)


def test_rope_keeps_infinities_and_nans_in_their_pairs():
    x16 = to16(np.ones((2, 2, 64)))
    x16[0, 1, 3] = 0x7C00
    x16[1, 0, 40] = 0x7E00
    freqs, _ = comet.rope_frequencies(64)
    y = f64(host16(comet.rope(dev16(x16), dev(np.array([3, 4], np.int32)), dev(freqs))))
    bad = ~np.isfinite(y)
    want = np.zeros_like(bad)
    want[0, 1, [3, 35]] = want[1, 0, [8, 40]] = True
    assert np.array_equal(bad, want)


# --- the cache ---------------------------------------------------------------------------

CACHES = [
    # seqs (rows, tokens), kvh, D, G, page
    ([(1, 1)], 1, 64, 64, 16),
    ([(1, 100), (1, 16), (1, 17)], 8, 128, 128, 16),
    ([(5, 5), (0, 0), (3, 40), (0, 7), (33, 50)], 2, 128, 32, 32),
    ([(40, 70), (1, 33)], 3, 64, 32, 64),
    ([(300, 700), (7, 1030)], 4, 128, 64, 1024),
    ([(6, 4), (2, 1), (1, 0)], 2, 128, 128, 16),  # rows at negative positions
]


@pytest.mark.parametrize("seqs,kvh,D,G,page", CACHES)
def test_append(seqs, kvh, D, G, page):
    p = Paged(len(seqs) + page, seqs, kvh, D, G, page)
    cache, batch = handles(p)
    M = p.M
    qkv = to16(p.rng.standard_normal((M, 3 * kvh, D)))
    new = [kv_rows(p.rng, M, kvh, D) for _ in "kv"]
    new[0][0] = 0  # a row of zeros, one of signed zeros
    new[1][0, :, ::2] = 0x8000
    qkv[:, kvh:2 * kvh], qkv[:, 2 * kvh:] = new
    buf = dev16(qkv)
    print(f"append {seqs} {kvh} {D} {G} {page}", flush=True)
    comet.kv4_append(cache, batch, buf[:, kvh:2 * kvh], buf[:, 2 * kvh:])
    for i in (0, 1):
        c, prm = oracle.kv4_quantize(new[i].reshape(M * kvh, D), G)
        c, prm = c.reshape(M, kvh, -1), prm.reshape(M, kvh, D // G, 2)
        for m, b, pos in p.rows():
            p.store(i, b, [pos], c[m:m + 1], prm[m:m + 1])
    assert np.array_equal(cache.k_codes.cpu().numpy(), p.codes[0])
    assert np.array_equal(cache.v_codes.cpu().numpy(), p.codes[1])
    assert np.array_equal(host16(cache.k_params), p.params[0])
    assert np.array_equal(host16(cache.v_params), p.params[1])


@pytest.mark.parametrize("seqs,kvh,D,G,page", CACHES)
def test_gather(seqs, kvh, D, G, page):
    p = Paged(7 * len(seqs) + page, seqs, kvh, D, G, page)
    cache, batch = handles(p, M=p.M + 5)
    out = [torch.full((p.M + 5, kvh, D), 0x1234, dtype=torch.int16, device=DEV).view(torch.float16)
           for _ in "kv"]
    comet.kv4_gather(cache, batch, k_out=out[0], v_out=out[1])
    for i in (0, 1):  # the rows behind the last sequence as they were
        assert np.array_equal(host16(out[i]), p.dequantized(i, p.M + 5))


def test_gather_of_one_side():
    p = Paged(3, [(9, 20)], 2, 64, 32, 16)
    cache, batch = handles(p)
    for i in (0, 1):
        o = torch.zeros((p.M, 2, 64), dtype=torch.float16, device=DEV)
        comet.comet_kv4_gather(cache, batch, o if i == 0 else None, o if i else None, 128, 128)
        assert np.array_equal(host16(o), p.dequantized(i))


def test_holes_are_not_written_and_read_as_zeros():
    holes = [(0, 1), (1, 0), (1, 2), (0, 3)]
    p = Paged(5, [(64, 64), (50, 50)], 2, 64, 64, 16, holes=holes)
    cache, batch = handles(p)
    before = [host16(cache.k_params).copy(), cache.k_codes.cpu().numpy()]
    k = dev16(kv_rows(p.rng, p.M, 2, 64))
    comet.kv4_append(cache, batch, k, k)
    c, prm = oracle.kv4_quantize(host16(k).reshape(-1, 64), 64)
    for i in (0, 1):
        for m, b, pos in p.rows():
            p.store(i, b, [pos], c.reshape(p.M, 2, -1)[m:m + 1],
                    prm.reshape(p.M, 2, 1, 2)[m:m + 1])
    assert np.array_equal(host16(cache.k_params), p.params[0])
    assert np.array_equal(cache.v_codes.cpu().numpy(), p.codes[1])
    assert not np.array_equal(before[1], cache.k_codes.cpu().numpy())
    kb, vb = comet.kv4_gather(cache, batch)
    assert np.array_equal(host16(kb), p.dequantized(0))
    assert np.array_equal(host16(vb), p.dequantized(1))


def test_tokens_behind_the_table_are_holes():
    # 70 tokens, a table of 4 pages of 16
    p = Paged(6, [(20, 70), (3, 30)], 1, 64, 64, 16, max_pages=4)
    cache, batch = handles(p)
    k = dev16(kv_rows(p.rng, p.M, 1, 64))
    comet.kv4_append(cache, batch, k, k)
    kb, _ = comet.kv4_gather(cache, batch)
    got = host16(kb)
    assert not got[14:20].any() and got[:14].any()
    q16 = to16(p.rng.standard_normal((p.M, 2, 64)))
    out = comet.kv4_attention(dev16(q16), cache, batch)
    c, prm = oracle.kv4_quantize(host16(k).reshape(-1, 64), 64)
    for i in (0, 1):
        for m, b, pos in p.rows():
            p.store(i, b, [pos], c[m:m + 1].reshape(1, 1, -1), prm[m:m + 1].reshape(1, 1, 1, 2))
    ref, bound = p.attention(q16, 2, 64 ** -0.5)
    check_attention(host16(out), ref, bound)


def test_cache_beyond_32_bits():
    # 4.3e9 bytes of codes each; the last pages are used
    page, kvh, D = 1024, 8, 128
    cache = comet.KV4Cache.empty(8300, page, kvh, D)
    assert cache.k_codes.numel() > 1 << 32
    p = Paged(8, [(40, 1500)], kvh, D, 128, page, spare=0)
    table = p.table + np.int32(8300 - p.num_pages)
    last = slice(8300 - p.num_pages, 8300)
    for t, a in ((cache.k_codes, p.codes[0]), (cache.v_codes, p.codes[1])):
        t[last] = dev(a)
    for t, a in ((cache.k_params, p.params[0]), (cache.v_params, p.params[1])):
        t[last] = dev16(a)
    batch = comet.KV4Batch(dev(p.row_start), dev(p.lens), dev(table), p.M)
    k, v = comet.kv4_gather(cache, batch)
    assert np.array_equal(host16(k), p.dequantized(0))
    comet.kv4_append(cache, batch, k, v)
    q16 = to16(p.rng.standard_normal((p.M, kvh, D)))
    out = comet.kv4_attention(dev16(q16), cache, batch)
    kb, vb = comet.kv4_gather(cache, batch)
    for i, (t, a) in enumerate(((cache.k_codes, cache.k_params), (cache.v_codes, cache.v_params))):
        p.codes[i], p.params[i] = t[last].cpu().numpy(), host16(a[last])
    assert np.array_equal(host16(vb), p.dequantized(1))
    ref, bound = p.attention(q16, kvh, D ** -0.5)
    check_attention(host16(out), ref, bound)


@pytest.mark.parametrize("n,B", [(130, 1), (8, 9)])
def test_attention_in_a_cache_beyond_32_bits(n, B):
    # many rows, and few in blocks of 32
    page, kvh, D, H = 1024, 8, 128, 32
    cache = comet.KV4Cache.empty(8300, page, kvh, D)
    p = Paged(50 + n, [(n, 300 + 130 * b) for b in range(B)], kvh, D, 128, page, spare=0)
    p2 = p.num_pages
    last = slice(8300 - p2, 8300)
    for t, a in ((cache.k_codes, p.codes[0]), (cache.v_codes, p.codes[1])):
        t[last] = dev(a)
    for t, a in ((cache.k_params, p.params[0]), (cache.v_params, p.params[1])):
        t[last] = dev16(a)
    table = np.where(p.table >= 0, p.table + (8300 - p2), -1).astype(np.int32)
    batch = comet.KV4Batch(dev(p.row_start), dev(p.lens), dev(table), p.M, n)
    q16 = to16(p.rng.standard_normal((p.M, H, D)))
    out = comet.kv4_attention(dev16(q16), cache, batch)
    some = p.rng.choice(p.M, 20, replace=False)
    ref, bound = p.attention(q16, H, D ** -0.5, rows=some)
    check_attention(host16(out)[some], ref[some], bound[some])


def test_more_sequences_than_a_block_has_lanes():
    n = 1500
    seqs = [(1 if b % 3 else 0, 1 + b % 40) for b in range(n)]
    p = Paged(9, seqs, 1, 64, 64, 16)
    cache, batch = handles(p)
    kb, _ = comet.kv4_gather(cache, batch)
    assert np.array_equal(host16(kb), p.dequantized(0))
    q16 = to16(p.rng.standard_normal((p.M, 2, 64)))
    out = comet.kv4_attention(dev16(q16), cache, batch)
    ref, bound = p.attention(q16, 2, 0.125)
    check_attention(host16(out), ref, bound)


# --- attention ------------------------------------------------------------------------------

ATTENTION = [
    # seqs, H, kvh, D, G, page, window
    ([(1, 1)], 1, 1, 64, 64, 16, 0),
    ([(1, 1)], 8, 8, 128, 128, 16, 0),
    ([(1, 100)], 32, 8, 128, 128, 16, 0),
    ([(1, 63), (1, 64), (1, 65), (0, 0), (1, 128), (1, 129)], 16, 2, 128, 128, 16, 0),
    ([(1, 1000), (1, 17), (0, 50), (1, 333)], 64, 8, 128, 64, 64, 0),
    ([(1, 5000)], 16, 2, 128, 128, 128, 0),
    ([(1, 3001)], 8, 1, 64, 32, 32, 0),
    ([(1, 500), (1, 200)], 64, 1, 128, 128, 64, 0),  # 64 heads share one
    ([(5, 300), (5, 5), (3, 77)], 12, 12, 64, 32, 32, 0),
    ([(4, 200), (2, 2), (7, 1030)], 40, 8, 128, 32, 1024, 0),
    ([(17, 200), (1, 90), (16, 16)], 10, 2, 128, 128, 16, 0),
    ([(130, 130)], 4, 2, 128, 128, 16, 0),
    ([(70, 400), (1, 300), (129, 129), (1, 2)], 8, 4, 64, 64, 64, 0),
    ([(257, 600)], 7, 1, 128, 64, 256, 0),
    ([(64, 65), (200, 201), (33, 1000)], 8, 2, 128, 32, 32, 0),
    ([(6, 4), (1, 0), (40, 17)], 8, 2, 128, 128, 16, 0),  # rows without a token
    ([(1, 400), (1, 30)], 8, 2, 128, 128, 16, 1),
    ([(1, 400), (9, 30), (1, 5000)], 8, 2, 64, 64, 32, 100),
    ([(150, 300)], 8, 2, 128, 128, 16, 33),
    ([(150, 150), (90, 700)], 4, 2, 128, 128, 64, 200),
    ([(100, 120)], 4, 4, 64, 32, 16, 5000),
    ([(130, 1500)], 32, 8, 64, 64, 16, 0),  # ranges added up in threes of 128 rows
    ([(1, 900), (1, 1300), (0, 0), (1, 70), (90, 1600)], 32, 8, 64, 64, 32, 0),
]


@pytest.mark.parametrize("seqs,H,kvh,D,G,page,window", ATTENTION)
def test_attention(seqs, H, kvh, D, G, page, window):
    p = Paged(sum(L for _, L in seqs) + H, seqs, kvh, D, G, page)
    cache, batch = handles(p, max_rows=max(n for n, _ in seqs))
    buf16 = to16(p.rng.standard_normal((p.M, H + 2, D)))
    print(f"attention {seqs} {H}/{kvh} {D} {G} {page} {window}", flush=True)
    q = dev16(buf16)[:, :H]
    out = comet.kv4_attention(q, cache, batch, window=window)
    ref, bound = p.attention(buf16[:, :H], H, D ** -0.5, window)
    check_attention(host16(out), ref, bound)
    again = comet.kv4_attention(q, cache, batch, window=window)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("n", [1, 20, 100])
@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
def test_attention_in_every_form(D, G, n, page):
    # blocks of 16 rows, one and several; tiles within a page and over several; one range and
    # several
    p = Paged(D + G + n + page, [(n, 150 + n), (1, 40), (n, 700)], 2, D, G, page)
    cache, batch = handles(p, max_rows=n)
    q16 = to16(p.rng.standard_normal((p.M, 4, D)))
    out = comet.kv4_attention(dev16(q16), cache, batch)
    ref, bound = p.attention(q16, 4, D ** -0.5)
    check_attention(host16(out), ref, bound)


@pytest.mark.parametrize("window", [0, 50])
def test_more_sequences_than_lanes_of_a_wave(window):
    # 150 sequences, some idle, of one row, of some and of many; ranges and whole ones
    seqs = [((0, 1, 1, 9, 40, 90)[b % 6], 90 + 37 * (b % 30)) for b in range(150)]
    p = Paged(41, seqs, 1, 64, 64, 32)
    cache, batch = handles(p, max_rows=90)
    q16 = to16(p.rng.standard_normal((p.M, 3, 64)))
    out = comet.kv4_attention(dev16(q16), cache, batch, window=window)
    ref, bound = p.attention(q16, 3, 0.125, window)
    check_attention(host16(out), ref, bound)


# The kernel for many rows: eight heads of K and V, 52 q rows and more to each.

def some_rows(p, rows=12):
    """The first and the last of each sequence, and others."""
    ends = np.concatenate([p.row_start[:-1], p.row_start[1:] - 1])
    return np.unique(np.concatenate([ends[(ends >= 0) & (ends < p.M)],
                                     p.rng.choice(p.M, rows, replace=False)]))


@pytest.mark.parametrize("window", [0, 90])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
def test_many_rows_in_every_form(D, G, page, window):
    p = Paged(D + G + page + window, [(100, 250), (1, 40), (75, 75), (130, 700)], 8, D, G, page)
    cache, batch = handles(p, max_rows=130)
    q16 = to16(p.rng.standard_normal((p.M, 32, D)))
    out = host16(comet.kv4_attention(dev16(q16), cache, batch, window=window))
    some = some_rows(p)
    ref, bound = p.attention(q16, 32, D ** -0.5, window, some)
    check_attention(out[some], ref[some], bound[some])


def test_many_rows_around_holes():
    seqs = [(40, 200), (40, 100), (40, 150)]
    holes = [(0, 0), (0, 5), (0, 12), (2, 3), (2, 4), (2, 5), (2, 6), (2, 7)] + [
        (1, j) for j in range(7)]
    p = Paged(55, seqs, 8, 128, 64, 16, holes=holes)
    cache, batch = handles(p, max_rows=40)
    q16 = to16(p.rng.standard_normal((p.M, 32, 128)))
    out = host16(comet.kv4_attention(dev16(q16), cache, batch))
    some = some_rows(p)
    ref, bound = p.attention(q16, 32, 128 ** -0.5, rows=some)
    check_attention(out[some], ref[some], bound[some])
    assert not out[40:80].any()


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_many_rows_with_scales(scale):
    p = Paged(57, [(60, 150), (60, 17)], 8, 64, 64, 32)  # the second has rows without a token
    cache, batch = handles(p, max_rows=60)
    q16 = to16(0.3 * p.rng.standard_normal((p.M, 32, 64)))
    out = host16(comet.kv4_attention(dev16(q16), cache, batch, scale=scale))
    some = some_rows(p)
    ref, bound = p.attention(q16, 32, scale, rows=some)
    check_attention(out[some], ref[some], bound[some])
    assert not out[60:60 + 43].any()


@pytest.mark.parametrize("kind", ["large", "small", "mixed", "zero"])
def test_many_extreme_rows(kind):
    n, L, kvh, H = 60, 180, 8, 32
    p = Paged(59, [(n, L)], kvh, 128, 64, 16)
    rng = p.rng
    size = {"large": np.full(L, 2e4), "small": np.full(L, 1e-6), "zero": np.zeros(L),
            "mixed": np.where(np.arange(L) % 7 == 0, 1e3, 1e-3)}[kind]
    for i in (0, 1):
        rows = np.clip(rng.standard_normal((L, kvh, 128)), -3, 3) * size[:, None, None]
        if i == 0 and kind == "mixed":
            rows *= 1e-3
        c, prm = oracle.kv4_quantize(to16(rows).reshape(L * kvh, 128), 64)
        p.store(i, 0, np.arange(L), c.reshape(L, kvh, -1), prm.reshape(L, kvh, 2, 2))
    cache, batch = handles(p)
    q16 = to16(rng.standard_normal((n, H, 128)) * {"large": 1e-5, "small": 1e4}.get(kind, 1.0))
    out = host16(comet.kv4_attention(dev16(q16), cache, batch))
    some = some_rows(p)
    ref, bound = p.attention(q16, H, 128 ** -0.5, rows=some)
    check_attention(out[some], ref[some], bound[some], kind)


def test_what_many_rows_do_not_see_does_not_reach_them():
    n, window = 60, 30
    p = Paged(61, [(n, 100)], 8, 64, 64, 16)
    q16 = to16(p.rng.standard_normal((n, 32, 64)))
    ref, bound = p.attention(q16, 32, 0.125, window)
    for i in (0, 1):
        for j, bits in ((99, 0x7E00), (60, 0x7C00)):
            p.params[i][p.page_of(0, j), :, j % 16] = bits
    cache, batch = handles(p)
    bad = q16.copy()
    bad[0, 0, 5] = 0x7C00
    bad[0, 2, 6] = 0x7E00
    out = host16(comet.kv4_attention(dev16(bad), cache, batch, window=window))
    at = np.arange(100 - n, 100)
    blind = (at < 99) & ~((at >= 60) & (at - window < 60))
    assert blind[0] and 2 <= blind.sum() < n - 1
    others = [h for h in range(32) if h not in (0, 2)]
    check_attention(out[0, others], ref[0, others], bound[0, others])
    assert np.isnan(f64(out[~blind])).all()
    blind[0] = False
    check_attention(out[blind], ref[blind], bound[blind])


def test_many_rows_captured_and_replayed():
    p = Paged(63, [(60, 400), (1, 300), (90, 90), (20, 900)], 8, 128, 128, 64)
    cache, batch = handles(p, max_rows=90)
    q = dev16(to16(p.rng.standard_normal((p.M, 32, 128))))
    out = torch.empty_like(q)
    workspace = comet.kv4_attention_workspace(q, cache, batch)
    call = lambda: comet.kv4_attention(q, cache, batch, out=out, workspace=workspace)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    lens = batch.seq_lens.clone()
    for step in range(4):
        batch.seq_lens.copy_(lens - 11 * step)
        q.mul_(1.0 + 0.125 * step)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        call()
        assert torch.equal(got.view(torch.int16), out.view(torch.int16)), step


@pytest.mark.parametrize("n,window", [(5, 0), (8, 100), (15, 0), (15, 70)])
@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
def test_attention_of_many_short_runs_of_rows(D, G, n, window):
    # sequences enough for blocks of 32 rows (20, 32 and 60 rows of a head's group), some with
    # fewer rows or none, of one range and of several
    seqs = [((n, n, 1, n, 0, n)[b % 6], 20 + n + 90 * b) for b in range(12)]
    p = Paged(D + G + n + window, seqs, 8, D, G, 32)
    cache, batch = handles(p, max_rows=n)
    q16 = to16(p.rng.standard_normal((p.M, 32, D)))
    out = comet.kv4_attention(dev16(q16), cache, batch, window=window)
    some = p.rng.choice(p.M, 16, replace=False)
    ref, bound = p.attention(q16, 32, D ** -0.5, window, some)
    check_attention(host16(out)[some], ref[some], bound[some])


@pytest.mark.parametrize("n,H,D,G", [(1, 8, 64, 64), (1, 8, 128, 128), (1, 16, 128, 32),
                                     (16, 64, 64, 64)])
def test_attention_of_sequences_just_longer_than_a_range(n, H, D, G):
    # 9 tiles each and about 2 / 3 of the ranges that run at once: two ranges to a sequence would
    # be more than that, so a sequence stays whole; a few shorter and longer ones
    B = 60 if n == 1 else 40
    seqs = [(n, (576, 570, 576, 100, 576, 640)[b % 6] if b else 900) for b in range(B)]
    p = Paged(47 + n + D, seqs, 8, D, G, 64)
    cache, batch = handles(p, max_rows=n)
    q16 = to16(p.rng.standard_normal((p.M, H, D)))
    out = comet.kv4_attention(dev16(q16), cache, batch)
    some = p.rng.choice(p.M, min(p.M, 24), replace=False)
    ref, bound = p.attention(q16, H, D ** -0.5, rows=some)
    check_attention(host16(out)[some], ref[some], bound[some])


def test_any_device_contents_stay_within_the_buffers():
    """Row starts that fall, negative lengths and lengths beyond the table, pages out of range:
    the calls end, and write nothing outside the rows and the cache.  (All indexes are
    checked where they are made; the buffers have guards on both sides.)"""
    kvh, H, D, page, M = 2, 8, 64, 16, 40
    rng = np.random.default_rng(43)
    shape = (6, kvh, page)
    whole = [torch.full((10,) + shape[1:] + tail, 7, dtype=t, device=DEV)
             for tail, t in (((D // 2,), torch.uint8), ((2, 2), torch.float16))]
    guard = [t.clone() for t in whole]
    codes, params = whole[0][2:8], whole[1][2:8]
    rows = [torch.full((M + 4, n, D), 3.0, dtype=torch.float16, device=DEV) for n in (H, kvh)]
    for k in range(20):
        B = (1, 3, 70)[k % 3]
        start = rng.integers(-5, M + 9, B + 1).astype(np.int32)
        if k % 2:
            start.sort()
        lens = rng.integers(-40, 300, B).astype(np.int32)
        lens[0] = (2 ** 31 - 1, -2 ** 31, 1 << 30, 77)[k % 4]
        table = rng.integers(-3, 9, (B, 5)).astype(np.int32)
        batch = comet.KV4Batch(dev(start), dev(lens), dev(table), M)
        cache = comet.KV4Cache(codes, params, codes, params)
        q = torch.randn((M, H, D), device=DEV).half()
        print(f"contents {k}: {start[:4]} {lens[:3]}", flush=True)
        comet.kv4_append(cache, batch, q[:, :kvh], q[:, kvh:2 * kvh])
        comet.kv4_gather(cache, batch, k_out=rows[1][2:M + 2], v_out=rows[1][2:M + 2])
        comet.kv4_attention(q, cache, batch, out=rows[0][2:M + 2], window=(0, 3, 2 ** 31 - 1)[k % 3])
        torch.cuda.synchronize()
        for t, g in zip(whole, guard):
            assert torch.equal(t[:2], g[:2]) and torch.equal(t[8:], g[8:])
        for t in rows:
            assert (t[:2] == 3).all() and (t[M + 2:] == 3).all()


@pytest.mark.parametrize("n", [1, 40])
def test_attention_around_holes(n):
    # first, inner and last pages; the whole of one sequence
    seqs = [(n, 200), (n, 100), (n, 150)]
    holes = [(0, 0), (0, 5), (0, 12), (2, 3), (2, 4), (2, 5), (2, 6), (2, 7)] + [
        (1, j) for j in range(7)]
    p = Paged(n, seqs, 2, 128, 64, 16, holes=holes)
    cache, batch = handles(p, max_rows=n)
    q16 = to16(p.rng.standard_normal((p.M, 8, 128)))
    out = host16(comet.kv4_attention(dev16(q16), cache, batch))
    ref, bound = p.attention(q16, 8, 128 ** -0.5)
    check_attention(out, ref, bound)
    assert not out[n:2 * n].any()


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
@pytest.mark.parametrize("n", [1, 50])
def test_attention_scales(scale, n):
    p = Paged(11, [(n, 150)], 2, 64, 64, 32)
    cache, batch = handles(p)
    q16 = to16(0.3 * p.rng.standard_normal((p.M, 4, 64)))
    out = comet.kv4_attention(dev16(q16), cache, batch, scale=scale)
    ref, bound = p.attention(q16, 4, scale)
    check_attention(host16(out), ref, bound)


@pytest.mark.parametrize("n", [1, 50])
@pytest.mark.parametrize("kind", ["large", "small", "mixed", "zero"])
def test_attention_of_extreme_rows(n, kind):
    """Cached values at both ends of fp16 and differing by 1e6 between tokens, queries of 3e4 and
    of 1e-7: nothing overflows, and no weight is lost to the spread of the scales."""
    p = Paged(13, [(n, 180)], 2, 128, 64, 16)
    L = 180
    rng = p.rng
    size = {"large": np.full(L, 2e4), "small": np.full(L, 1e-6), "zero": np.zeros(L),
            "mixed": np.where(np.arange(L) % 7 == 0, 1e3, 1e-3)}[kind]
    for i in (0, 1):
        rows = np.clip(rng.standard_normal((L, 2, 128)), -3, 3) * size[:, None, None]
        if i == 0 and kind == "mixed":
            rows *= 1e-3
        c, prm = oracle.kv4_quantize(to16(rows).reshape(L * 2, 128), 64)
        p.store(i, 0, np.arange(L), c.reshape(L, 2, -1), prm.reshape(L, 2, 2, 2))
    cache, batch = handles(p)
    q = rng.standard_normal((p.M, 4, 128)) * {"large": 1e-5, "small": 1e4}.get(kind, 1.0)
    q[-1, 0] *= 1e-2
    q16 = to16(q)
    out = comet.kv4_attention(dev16(q16), cache, batch)
    ref, bound = p.attention(q16, 4, 128 ** -0.5)
    check_attention(host16(out), ref, bound, kind)


@pytest.mark.parametrize("n", [3, 60])
def test_what_a_row_does_not_see_does_not_reach_it(n):
    """Later tokens of the chunk, tokens before the window and other rows hold
    not-a-numbers and infinities."""
    p = Paged(17, [(n, 100)], 1, 64, 64, 16)
    q16 = to16(p.rng.standard_normal((n, 4, 64)))
    window = 30
    ref, bound = p.attention(q16, 4, 0.125, window)
    for i in (0, 1):
        for j, bits in ((99, 0x7E00), (60, 0x7C00)):
            p.params[i][p.page_of(0, j), 0, j % 16] = bits
    cache, batch = handles(p)
    bad = q16.copy()
    bad[0, 0, 5] = 0x7C00
    bad[0, 2, 6] = 0x7E00
    out = host16(comet.kv4_attention(dev16(bad), cache, batch, window=window))
    at = np.arange(100 - n, 100)
    blind = (at < 99) & ~((at >= 60) & (at - window < 60))
    assert blind[0] and blind.sum() >= 2
    check_attention(out[0, [1, 3]], ref[0, [1, 3]], bound[0, [1, 3]])
    blind[0] = False
    check_attention(out[blind], ref[blind], bound[blind])


def test_rows_in_no_sequence_stay():
    p = Paged(19, [(1, 40), (30, 30)], 2, 64, 64, 16)
    cache, batch = handles(p, M=p.M + 9)
    q16 = to16(p.rng.standard_normal((p.M + 9, 4, 64)))
    out = torch.full((p.M + 9, 6, 64), 0x1234, dtype=torch.int16, device=DEV).view(torch.float16)
    comet.kv4_attention(dev16(q16), cache, batch, out=out[:, 1:5])
    got = host16(out)
    ref, bound = p.attention(q16[:p.M], 4, 0.125)
    check_attention(got[:p.M, 1:5], ref, bound)
    assert (got[p.M:] == 0x1234).all() and (got[:, [0, 5]] == 0x1234).all()


@pytest.mark.parametrize("seqs", [[(1, 900), (1, 3000), (1, 50)], [(40, 900), (1, 3000), (90, 90)]])
def test_a_layer_captured_and_replayed(seqs):
    """Rotate, append, attend in one graph; between replays new rows and lengths are written
    into its inputs and eager calls of other sizes run."""
    kvh, H, D, page = 2, 8, 128, 16
    p = Paged(23, seqs, kvh, D, 64, page, max_pages=200)
    cache, batch = handles(p, max_rows=max(n for n, _ in seqs))
    other = Paged(24, [(3, 700)], kvh, D, 64, page)
    ocache, obatch = handles(other)
    oq = dev16(to16(other.rng.standard_normal((3, H, D))))
    expect = comet.kv4_attention(oq, ocache, obatch)
    freqs = dev(comet.rope_frequencies(D)[0])
    qkv = torch.empty((p.M, H + 2 * kvh, D), dtype=torch.float16, device=DEV)
    pos = torch.zeros(p.M, dtype=torch.int32, device=DEV)

    def layer(out):
        comet.rope(qkv[:, :H + kvh], pos, freqs, out=qkv[:, :H + kvh])
        comet.kv4_append(cache, batch, qkv[:, H:H + kvh], qkv[:, H + kvh:])
        return comet.kv4_attention(qkv[:, :H], cache, batch, out=out)

    def fill(step):
        g = torch.Generator(device=DEV).manual_seed(step)
        qkv.copy_(torch.randn(qkv.shape, generator=g, device=DEV))
        batch.seq_lens.copy_(dev(np.maximum(p.lens - 3 * step, [n for n, _ in seqs])))
        pos.copy_(torch.arange(p.M, device=DEV) + step)

    fill(0)
    out = torch.zeros((p.M, H, D), dtype=torch.float16, device=DEV)
    layer(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(out)
    for step in (1, 2, 3, 4):
        fill(step)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        fill(step)
        layer(out)
        assert torch.equal(got.view(torch.int16), out.view(torch.int16)), step
        assert torch.equal(expect, comet.kv4_attention(oq, ocache, obatch))


def test_calls_on_two_streams():
    p = Paged(29, [(1, 4000), (1, 700)], 2, 128, 128, 64)
    cache, batch = handles(p)
    qs = [dev16(to16(p.rng.standard_normal((p.M, 16, 128)))) for _ in range(4)]
    expect = [comet.kv4_attention(q, cache, batch) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [comet.kv4_attention(q, cache, batch, stream=streams[i % 2]) for i, q in enumerate(qs)]
    raw = comet.kv4_attention(qs[0], cache, batch, stream=streams[0].cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(expect + expect[:1], got + [raw]):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_a_prompt_in_chunks_equals_the_prompt_at_once():
    """150 tokens appended and attended in chunks of several sizes, by two sequences that share
    the pages of their first 64 tokens: the outputs of one call over all of them, within both
    bounds."""
    kvh, H, D, page = 2, 8, 128, 32
    rng = np.random.default_rng(31)
    k, v = (dev16(kv_rows(rng, 150, kvh, D)) for _ in "kv")
    q16 = to16(rng.standard_normal((150, H, D)))
    q = dev16(q16)
    cache = comet.KV4Cache.empty(12, page, kvh, D)
    tables = np.array([[3, 7, 1, 9, 4], [3, 7, 0, 5, 2]], np.int32)
    ints = lambda *a: dev(np.array(a, np.int32))  # noqa: E731
    outs, at = [], 0
    for n in (64, 1, 1, 17, 60, 7):
        if at == 0:  # the shared pages once
            batch = comet.KV4Batch(ints(0, n), ints(n), dev(tables[:1]), n)
            two = False
        else:
            batch = comet.KV4Batch(ints(0, n, 2 * n), ints(at + n, at + n), dev(tables), 2 * n, n)
            two = True
        rep = lambda t: torch.cat([t[at:at + n]] * (2 if two else 1))  # noqa: E731
        comet.kv4_append(cache, batch, rep(k), rep(v))
        o = comet.kv4_attention(rep(q), cache, batch)
        if two:
            assert torch.equal(o[:n], o[n:])
        outs.append(host16(o[:n]))
        at += n
    p = Paged(0, [(150, 150)], kvh, D, 128, page)
    p.table[:] = tables[:1]
    p.num_pages = 12
    p.codes = [cache.k_codes.cpu().numpy(), cache.v_codes.cpu().numpy()]
    p.params = [host16(cache.k_params), host16(cache.v_params)]
    ref, bound = p.attention(q16, H, D ** -0.5)
    check_attention(np.concatenate(outs), ref, bound, "in chunks")
    whole = comet.KV4Batch(ints(0, 150), ints(150), dev(tables[:1]), 150)
    check_attention(host16(comet.kv4_attention(q, cache, whole)), ref, bound, "at once")
