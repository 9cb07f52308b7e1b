"""The paged-cache operators over long token ranges and many rows: what their loops do after
the first turn."""
import numpy as np
import pytest
import torch

import oracle
import paper_2410_12168_amd as comet
from paged_ref import Paged, check_attention, kv_rows, to16
from test_gpu_serving import DEV, dev, dev16, handles, host16, rope_ref

pytestmark = pytest.mark.gpu
FORMS = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


def enlarge(p, b, tokens, factor):
    """Values of these tokens of sequence b, `factor` times as large."""
    rows = to16(factor * p.rng.standard_normal((len(tokens), p.kvh, p.D)))
    c, prm = oracle.kv4_quantize(rows.reshape(-1, p.D), p.G)
    p.store(1, b, tokens, c.reshape(len(tokens), p.kvh, -1),
            prm.reshape(len(tokens), p.kvh, p.D // p.G, 2))


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("D,G", FORMS)
def test_many_rows_over_long_ranges(D, G, page):
    # ten blocks of 128 rows share 81 tiles: ranges of 20 tiles and more, a wave holds the pages
    # of 16; the largest values come late
    n, L, kvh, H = 300, 5150, 16, 64
    p = Paged(D + G + page, [(n, L)], kvh, D, G, page)
    enlarge(p, 0, np.arange(L - 700, L - 640), 60.0)
    cache, batch = handles(p)
    q16 = to16(p.rng.standard_normal((n, H, D)))
    print(f"long ranges {D} {G} {page}", flush=True)
    out = host16(comet.kv4_attention(dev16(q16), cache, batch))
    some = np.array([0, 151, n - 1])
    ref, bound = p.attention(q16, H, D ** -0.5, rows=some)
    check_attention(out[some], ref[some], bound[some])


@pytest.mark.parametrize("kvh,H,B,page", [(64, 64, 16, 16), (64, 64, 16, 128), (32, 1024, 24, 64)])
@pytest.mark.parametrize("D,G", FORMS)
def test_single_rows_over_long_ranges(D, G, kvh, H, B, page):
    # sequences enough that each is one range of 68 tiles, of which a wave takes 17 and holds the
    # pages of 16; blocks of 16 rows and of 32.  All share one sequence's pages.
    L = 4330
    p = Paged(D + G + page, [(1, L)], kvh, D, G, page)
    enlarge(p, 0, np.arange(L - 150, L - 90), 60.0)
    cache, _ = handles(p)
    lens = np.full(B, L, np.int32)
    lens[1] = L - 200
    batch = comet.KV4Batch(dev(np.arange(B + 1, dtype=np.int32)), dev(lens),
                           dev(np.repeat(p.table, B, axis=0)), B, 1)
    q16 = to16(p.rng.standard_normal((B, H, D)))
    q16[2:] = q16[0]
    print(f"long single rows {D} {G} {page}", flush=True)
    out = host16(comet.kv4_attention(dev16(q16), cache, batch))
    heads = slice(H // kvh // 6, None, H // kvh)  # one of each kv head
    for b in (0, 1):
        p.seqs, p.lens = [(1, int(lens[b]))], lens[b:b + 1]
        ref, bound = p.attention(q16[b:b + 1, heads], kvh, D ** -0.5)
        check_attention(out[b:b + 1, heads], ref, bound)
    assert np.array_equal(out[2:], out[2:3].repeat(B - 2, axis=0))


# --- rows enough that a block walks over several heads ------------------------------------

@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("M,heads,D,rot,interleaved", [
    (7101, 52, 128, 128, False), (7101, 52, 128, 128, True), (4003, 100, 128, 64, True),
    (14050, 52, 64, 64, False), (4003, 101, 64, 32, False)])
def test_rope_of_many_rows(M, heads, D, rot, interleaved, in_place):
    rng = np.random.default_rng(M + heads + rot)
    g = torch.Generator(device=DEV).manual_seed(M + heads + rot)
    buf = torch.randn((M, heads + 3, D), generator=g, device=DEV).half()
    before = buf.clone()
    pos16 = rng.integers(0, 1 << 17, M).astype(np.int32)
    pos = dev(pos16)
    freqs_host, _ = comet.rope_frequencies(rot, 500000.0)
    freqs = dev(freqs_host)
    x = buf[:, :heads]
    print(f"rope of many rows {M} {heads} {D} {rot} {interleaved} {in_place}", flush=True)
    y = comet.rope(x, pos, freqs, interleaved=interleaved, out=x if in_place else None)
    # row by row the same as in calls of few rows, whose blocks take 8 heads
    for m in range(0, M, 500):
        few = comet.rope(before[m:m + 500, :heads], pos[m:m + 500], freqs, interleaved=interleaved)
        assert torch.equal(few.view(torch.int16), y[m:m + 500].view(torch.int16)), m
    assert torch.equal(buf[:, heads:], before[:, heads:])
    if not in_place:
        assert torch.equal(buf, before)
    some = np.unique(np.concatenate([[0, M - 1], rng.integers(0, M, 30)]))
    x16 = host16(before[torch.from_numpy(some).to(DEV)])[:, :heads]
    ref, bound = rope_ref(x16, pos16[some], freqs_host, interleaved, 1.0)
    got = host16(y[torch.from_numpy(some).to(DEV)]).view(np.float16).astype(np.float64)
    assert np.all(np.abs(got - ref) <= bound)


@pytest.mark.parametrize("in_place", [False, True])
def test_rope_of_many_unaligned_rows(in_place):
    # more rows than need their heads spread over blocks
    M, heads, D, rot = 700, 5, 72, 36
    rng = np.random.default_rng(5)
    x16 = to16(rng.standard_normal((M, heads, D)))
    pos = rng.integers(0, 1 << 17, M).astype(np.int32)
    freqs, _ = comet.rope_frequencies(rot)
    x = dev16(x16)
    y = comet.rope(x, dev(pos), dev(freqs), out=x if in_place else None)
    ref, bound = rope_ref(x16, pos, freqs, False, 1.0)
    assert np.all(np.abs(host16(y).view(np.float16).astype(np.float64) - ref) <= bound)


@pytest.mark.parametrize("kvh,D,G,page,M", [
    (3, 128, 32, 64, 22000), (6, 128, 128, 16, 22000), (10, 128, 64, 128, 13500),
    (10, 64, 32, 32, 27000), (7, 64, 64, 1024, 19000)])
def test_append_and_gather_of_many_rows(kvh, D, G, page, M):
    """Ragged prompts in a cache with holes: bit for bit the oracle's codes at the table's
    places, the rest of the cache as it was, and the same rows back."""
    rng = np.random.default_rng(kvh + D + G)
    n = np.array([M // 2, 0, M // 3 + 5, 1, M - M // 2 - M // 3 - 6])
    lens = (n + np.array([37, 9, 0, 500, 64])).astype(np.int32)
    start = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    width = int(-(-lens.max() // page))
    need = -(-lens // page)
    pages = int(need.sum()) + 3
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((5, width), -1, np.int32)
    at = 0
    for b in range(5):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    table[0, [0, need[0] // 2, need[0] - 1]] = (-1, pages, 2 ** 31 - 1)
    table[2, need[2] // 3] = -2 ** 31
    shape = (pages, kvh, page)
    codes = [np.full(shape + (D // 2,), 0xA5, np.uint8) for _ in "kv"]
    params = [np.full(shape + (D // G, 2), 0x7E00, np.uint16) for _ in "kv"]
    cache = comet.KV4Cache(dev(codes[0]), dev16(params[0]), dev(codes[1]), dev16(params[1]))
    batch = comet.KV4Batch(dev(start), dev(lens), dev(table), M, int(n.max()))
    new = [kv_rows(rng, M, kvh, D) for _ in "kv"]
    print(f"append {kvh} {D} {G} {page} {M}", flush=True)
    comet.kv4_append(cache, batch, dev16(new[0]), dev16(new[1]))
    seq = np.repeat(np.arange(5), n)
    pos = lens[seq] - n[seq] + np.arange(M) - start[seq]
    page_of = table[seq, pos // page]
    there = (page_of >= 0) & (page_of < pages)
    back = []
    for i in (0, 1):
        c, prm = oracle.kv4_quantize(new[i].reshape(M * kvh, D), G)
        c, prm = c.reshape(M, kvh, -1), prm.reshape(M, kvh, D // G, 2)
        codes[i][page_of[there], :, pos[there] % page] = c[there]
        params[i][page_of[there], :, pos[there] % page] = prm[there]
        rows = oracle.kv4_dequantize(c.reshape(M * kvh, -1), prm.reshape(M * kvh, D // G, 2), G)
        back.append(np.where(there[:, None, None], rows.reshape(M, kvh, D), 0).astype(np.uint16))
    for i, (c, prm) in enumerate(((cache.k_codes, cache.k_params), (cache.v_codes, cache.v_params))):
        assert np.array_equal(c.cpu().numpy(), codes[i])
        assert np.array_equal(host16(prm), params[i])
    k, v = comet.kv4_gather(cache, batch)
    assert np.array_equal(host16(k), back[0]) and np.array_equal(host16(v), back[1])


# --- the device that a call is for ----------------------------------------------------------

def test_tensors_of_a_device_that_is_not_the_current_one(monkeypatch):
    """With one GPU: the wrappers are told that another device is the current one."""
    p = Paged(91, [(3, 20)], 2, 64, 32, 16)
    cache, batch = handles(p)
    k = torch.zeros((3, 2, 64), dtype=torch.float16, device=DEV)
    freqs = dev(comet.rope_frequencies(64)[0])
    pos = torch.zeros(3, dtype=torch.int32, device=DEV)
    comet.kv4_append(cache, batch, k, k)
    monkeypatch.setattr(comet, "_current_device", lambda: 1)
    for call in (lambda: comet.kv4_append(cache, batch, k, k), lambda: comet.kv4_gather(cache, batch),
                 lambda: comet.kv4_attention(k, cache, batch)):
        with pytest.raises(ValueError, match="current device is 1"):
            call()
    with pytest.raises(ValueError, match="x: on device 0, the current device is 1"):
        comet.rope(k, pos, freqs)


# --- rows before the first sequence ----------------------------------------------------------

@pytest.mark.parametrize("seqs,kvh,H", [([(0, 9), (1, 70), (4, 300)], 2, 8),
                                        ([(0, 0), (70, 90), (1, 30), (64, 500)], 8, 32)])
def test_rows_before_the_first_sequence_stay(seqs, kvh, H):
    lead, D, G = 5, 64, 32
    p = Paged(95 + kvh, seqs, kvh, D, G, 16)
    cache, _ = handles(p)
    M = lead + p.M + 2
    batch = comet.KV4Batch(dev(p.row_start + np.int32(lead)), dev(p.lens), dev(p.table), M,
                           max(n for n, _ in seqs))
    new = [kv_rows(p.rng, M, kvh, D) for _ in "kv"]
    comet.kv4_append(cache, batch, dev16(new[0]), dev16(new[1]))
    for i in (0, 1):
        c, prm = oracle.kv4_quantize(new[i][lead:lead + p.M].reshape(-1, D), G)
        c, prm = c.reshape(p.M, kvh, -1), prm.reshape(p.M, kvh, D // G, 2)
        for m, b, pos in p.rows():
            p.store(i, b, [pos], c[m:m + 1], prm[m:m + 1])
    assert np.array_equal(cache.k_codes.cpu().numpy(), p.codes[0])
    assert np.array_equal(host16(cache.v_params), p.params[1])
    marked = lambda heads: torch.full((M, heads, D), 0x1234, dtype=torch.int16,  # noqa: E731
                                      device=DEV).view(torch.float16)
    k, v, out = marked(kvh), marked(kvh), marked(H)
    comet.kv4_gather(cache, batch, k_out=k, v_out=v)
    assert np.array_equal(host16(v)[lead:-2], p.dequantized(1))
    q16 = to16(p.rng.standard_normal((M, H, D)))
    comet.kv4_attention(dev16(q16), cache, batch, out=out)
    ref, bound = p.attention(q16[lead:-2], H, D ** -0.5)
    check_attention(host16(out)[lead:-2], ref, bound)
    for t in (k, v, out):
        assert (host16(t)[:lead] == 0x1234).all() and (host16(t)[-2:] == 0x1234).all()


# --- one quantizer in two kernels ------------------------------------------------------------

@pytest.mark.parametrize("D,G", FORMS)
def test_append_quantizes_as_the_flat_quantizer_does(D, G):
    """Rows of any finite fp16 bits, of all exponents and of few, constants and ties: the codes
    and parameters of comet_kv4_quantize, bit for bit."""
    rng = np.random.default_rng(D + G)
    M, kvh, page = 4096, 3, 64
    rows = rng.integers(0, 1 << 16, (M, kvh, D)).astype(np.uint16)
    rows[(rows & 0x7C00) == 0x7C00] ^= 0x4000  # finite
    rows[M // 4:M // 2] &= 0x83FF  # subnormals
    rows[M // 2:3 * M // 4] = to16(rng.integers(-8, 9, (M // 4, kvh, D)) * 2.0 ** rng.integers(
        -20, 12, (M // 4, kvh, 1)))  # multiples of a power of two
    rows[-64:] = rows[-64:, :, :1]  # constant rows
    table = rng.permutation(M // page).astype(np.int32)
    cache = comet.KV4Cache.empty(M // page, page, kvh, D, G=G)
    ints = lambda *a: dev(np.array(a, np.int32))  # noqa: E731
    batch = comet.KV4Batch(ints(0, M), ints(M), dev(table[None]), M)
    x = dev16(rows)
    comet.kv4_append(cache, batch, x, x)
    codes, params = comet.kv4_quantize(x.view(M * kvh, D), G=G)
    want = codes.view(M // page, page, kvh, D // 2).transpose(1, 2)
    want_params = params.view(M // page, page, kvh, D // G, 2).transpose(1, 2)
    at = dev(table).long()
    for c, prm in ((cache.k_codes, cache.k_params), (cache.v_codes, cache.v_params)):
        assert torch.equal(c[at], want)
        assert torch.equal(prm[at].view(torch.int16), want_params.contiguous().view(torch.int16))
    k, v = comet.kv4_gather(cache, batch)
    flat = comet.kv4_dequantize(codes, params, G=G).view(M, kvh, D)
    assert torch.equal(k.view(torch.int16), flat.view(torch.int16))
    assert torch.equal(v.view(torch.int16), flat.view(torch.int16))
