"""Rotary frequencies, and what the operators around the paged cache refuse and launch
(no GPU: refused calls launch nothing, the others run against hip_record's stand-in)."""
import ctypes
import math

import numpy as np
import pytest

import hip_record
import paper_2410_12168_amd as comet

FAKE = 0x10000  # 16-byte aligned address that is never dereferenced


# --- frequencies ---------------------------------------------------------------------

def test_plain_frequencies():
    f, m = comet.rope_frequencies(8, 10000.0)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001], rtol=1e-14, atol=0) and m == 1.0


def test_linear_frequencies():
    f, m = comet.rope_frequencies(8, 10000.0, "linear", factor=4.0)
    assert np.allclose(f, [0.25, 0.025, 0.0025, 0.00025], rtol=1e-14, atol=0) and m == 1.0


def test_base_scaling_slows_the_last_pair_by_the_factor():
    plain, _ = comet.rope_frequencies(64, 10000.0)
    f, m = comet.rope_frequencies(64, 10000.0, "base", factor=8.0)
    assert f[0] == 1.0 and m == 1.0
    assert math.isclose(f[-1], plain[-1] / 8.0, rel_tol=1e-12)
    assert np.all(np.diff(f / plain) < 0)


def test_band_scaling():
    # pairs of more than 4 turns over 8192 positions keep their speed, of less than one
    # are slowed 8 times
    plain, _ = comet.rope_frequencies(128, 500000.0)
    f, m = comet.rope_frequencies(128, 500000.0, "bands", factor=8.0, low=1.0, high=4.0,
                                  original_len=8192.0)
    turns = 8192.0 * plain / (2 * math.pi)
    assert m == 1.0 and (turns > 4).any() and (turns < 1).any()
    assert np.array_equal(f[turns >= 4], plain[turns >= 4])
    assert np.allclose(f[turns <= 1], plain[turns <= 1] / 8, rtol=1e-14, atol=0)
    mid = (turns > 1) & (turns < 4)
    assert mid.any()
    t = (turns[mid] - 1) / 3
    assert np.allclose(f[mid], (1 - t) * plain[mid] / 8 + t * plain[mid], rtol=1e-13, atol=0)


def test_ramp_scaling():
    d, base, L, factor = 128, 10000.0, 4096.0, 16.0
    plain, _ = comet.rope_frequencies(d, base)
    f, m = comet.rope_frequencies(d, base, "ramp", factor=factor, low=1.0, high=32.0,
                                  original_len=L)
    assert math.isclose(m, 0.1 * math.log(factor) + 1.0, rel_tol=1e-7)
    # pair i makes L base^(-2 i / d) / (2 pi) turns: 32 turns near pair 20, one near pair 45
    turns = L * plain / (2 * math.pi)
    first, last = np.nonzero(turns >= 32)[0][-1], np.nonzero(turns <= 1)[0][0]
    assert (first, last) == (20, 46)
    for i in range(d // 2):
        keep = min(1.0, max(0.0, 1.0 - (i - first) / (last - first)))
        assert math.isclose(f[i], plain[i] * (keep + (1 - keep) / factor), rel_tol=1e-12), i


@pytest.mark.parametrize("args,why", [
    ((7, 1e4, 0, 1, 1, 4, 100), "rot_dim"), ((0, 1e4, 0, 1, 1, 4, 100), "rot_dim"),
    ((8, 1.0, 0, 1, 1, 4, 100), "base"), ((8, math.nan, 0, 1, 1, 4, 100), "base"),
    ((8, 1e4, 5, 1, 1, 4, 100), "scaling"), ((8, 1e4, -1, 1, 1, 4, 100), "scaling"),
    ((8, 1e4, 1, 0.5, 1, 4, 100), "factor"), ((8, 1e4, 2, math.inf, 1, 4, 100), "factor"),
    ((2, 1e4, 2, 2, 1, 4, 100), "rot_dim"), ((8, 1e4, 3, 2, 4, 4, 100), "low"),
    ((8, 1e4, 4, 2, 0, 4, 100), "low"), ((8, 1e4, 4, 2, 1, 4, 0), "original_len"),
])
def test_frequency_refusals(args, why):
    f = np.zeros(600, np.float64)
    with pytest.raises(comet.CometError, match=why) as e:
        comet.comet_rope_frequencies(f, *args)
    assert e.value.status == 1
    with pytest.raises(ValueError, match="scaling"):
        comet.rope_frequencies(8, scaling="other")


def test_frequencies_need_room():
    with pytest.raises(ValueError, match="freqs"):
        comet.comet_rope_frequencies(np.zeros(3, np.float64), 8, 1e4, 0, 1, 1, 4, 100)


# --- refusals of the entry points ------------------------------------------------------

def cache(**kw):
    a = dict(k_codes=FAKE, k_params=FAKE, v_codes=FAKE, v_params=FAKE, num_pages=4, page_size=16,
             kv_heads=2, head_dim=128, G=64)
    a.update(kw)
    return comet.KV4CacheStruct(**a)


def batch(**kw):
    a = dict(row_start=FAKE, seq_lens=FAKE, block_table=FAKE, B=2, M=8, max_pages=3, max_rows=8)
    a.update(kw)
    return comet.KV4BatchStruct(**a)


BAD_CACHES = [
    (dict(k_codes=0), 1), (dict(k_params=0), 1), (dict(v_codes=0), 1), (dict(v_params=0), 1),
    (dict(k_codes=FAKE + 8), 1), (dict(v_params=FAKE + 4), 1), (dict(num_pages=0), 1),
    (dict(page_size=8), 2), (dict(page_size=48), 2), (dict(page_size=2048), 2),
    (dict(page_size=-16), 2), (dict(kv_heads=0), 1), (dict(kv_heads=1025), 2),
    (dict(head_dim=96), 2), (dict(head_dim=0), 2), (dict(G=16), 2), (dict(G=128, head_dim=64), 2),
]
BAD_BATCHES = [
    (dict(row_start=0), 1), (dict(seq_lens=0), 1), (dict(block_table=0), 1),
    (dict(seq_lens=FAKE + 2), 1), (dict(B=0), 1), (dict(M=0), 1), (dict(max_pages=0), 1),
    (dict(max_rows=0), 1), (dict(B=65537), 2), (dict(M=65535 * 32 + 1), 2),
    (dict(max_pages=(1 << 26) + 1), 2), (dict(max_pages=2 ** 31 - 1), 2),
]


def append(c, b, k=FAKE, v=FAKE, ks=256, vs=256):
    L = comet.lib()
    return L.comet_kv4_append(c and ctypes.addressof(c), b and ctypes.addressof(b), k, v, ks, vs, 0)


def gather(c, b, k=FAKE, v=FAKE, ks=256, vs=256):
    L = comet.lib()
    return L.comet_kv4_gather(c and ctypes.addressof(c), b and ctypes.addressof(b), k, v, ks, vs, 0)


def attend(c, b, q=FAKE, out=FAKE, heads=4, qs=512, os=512, scale=0.1, window=0, ws=0, n=0):
    return comet.lib().comet_kv4_attention(c and ctypes.addressof(c), b and ctypes.addressof(b), q,
                                           out, heads, qs, os, scale, window, ws, n, 0)


@pytest.mark.parametrize("call", [append, gather, attend])
def test_bad_caches_and_batches(call):
    assert call(None, batch()) == 1 and call(cache(), None) == 1
    for kw, status in BAD_CACHES:
        assert call(cache(**kw), batch()) == status, kw
        assert comet.comet_last_error() != ""
    for kw, status in BAD_BATCHES:
        assert call(cache(), batch(**kw)) == status, kw


@pytest.mark.parametrize("call", [append, gather])
@pytest.mark.parametrize("kw", [dict(k=FAKE + 2), dict(v=FAKE + 8), dict(ks=255), dict(ks=248),
                                dict(vs=260), dict(vs=-256), dict(k=0, v=0)])
def test_bad_rows(call, kw):
    assert call(cache(), batch(), **kw) == 1


def test_append_needs_both_sides():
    assert append(cache(), batch(), k=0) == 1 and append(cache(), batch(), v=0) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), 1), (dict(out=0), 1), (dict(q=FAKE + 2), 1), (dict(out=FAKE + 8), 1),
    (dict(heads=3), 1), (dict(heads=0), 1), (dict(heads=-2), 1), (dict(heads=1026, qs=1 << 20,
                                                                      os=1 << 20), 2),
    (dict(qs=504), 1), (dict(os=516), 1), (dict(scale=math.nan), 1), (dict(scale=math.inf), 1),
    (dict(window=-1), 1), (dict(ws=FAKE + 8, n=1 << 30), 1)])
def test_bad_attention_arguments(kw, status):
    assert attend(cache(), batch(), **kw) == status


def rope(X=FAKE, pos=FAKE, freqs=FAKE, out=FAKE + 65536, M=2, heads=3, D=64, rot=32, xs=192, os=192,
         mscale=1.0):
    return comet.lib().comet_rope(X, pos, freqs, out, M, heads, D, rot, xs, os, 0, mscale, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(X=0), 1), (dict(pos=0), 1), (dict(freqs=0), 1), (dict(out=0), 1), (dict(M=0), 1),
    (dict(heads=0), 1), (dict(rot=0), 1), (dict(rot=31), 1), (dict(rot=66), 1),
    (dict(D=1026, rot=32, xs=4000, os=4000), 2), (dict(xs=191), 1), (dict(os=191), 1),
    (dict(out=FAKE, os=200), 1), (dict(mscale=math.inf), 1), (dict(X=FAKE + 1), 1),
    (dict(pos=FAKE + 2), 1), (dict(freqs=FAKE + 4), 1), (dict(M=65535 * 32 + 1), 2),
    (dict(heads=65536, D=2, rot=2, xs=1 << 20, os=1 << 20), 2)])
def test_bad_rope_arguments(kw, status):
    assert rope(**kw) == status
    assert comet.comet_last_error() != ""


def test_wrappers_refuse_host_tensors_and_wrong_shapes():
    import torch

    x = torch.zeros((2, 3, 64), dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="x: need a float16 CUDA tensor"):
        comet.rope(x, i, torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError, match="k_codes: need a contiguous uint8 CUDA tensor"):
        comet.KV4Cache(x, x, x, x)
    with pytest.raises(ValueError, match="row_start: need a contiguous int32 CUDA tensor"):
        comet.KV4Batch(i, i, i, 2)
    with pytest.raises(ValueError, match="multiple of G"):
        comet.KV4Cache.empty(1, 16, 1, 64, G=128)


def test_raw_calls_need_room():
    # arrays stand in for device buffers: too small ones are refused before the call
    small = np.zeros(8 * 256 - 1, np.float16)
    with pytest.raises(ValueError, match="K: 4094 bytes, the call needs 4096"):
        comet.comet_kv4_append(cache(), batch(), small, FAKE, 256, 256, stream=0)
    with pytest.raises(ValueError, match="V: "):
        comet.comet_kv4_gather(cache(), batch(), FAKE, small, 256, 256, stream=0)
    with pytest.raises(ValueError, match="Q: "):
        comet.comet_kv4_attention(cache(), batch(), small, FAKE, 4, 512, 512, 0.1, stream=0)
    with pytest.raises(ValueError, match="out: "):
        comet.comet_kv4_attention(cache(), batch(), FAKE, small, 4, 512, 512, 0.1, stream=0)
    with pytest.raises(ValueError, match="positions: "):
        comet.comet_rope(FAKE, np.zeros(1, np.int32), FAKE, FAKE, 2, 3, 64, 32, 192, 192, stream=0)


# --- launches ------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    return hip_record.library(str(tmp_path_factory.mktemp("hip_record")))


def test_calls_only_launch_and_only_on_their_stream(shim):
    out = hip_record.run(shim, """
c = comet.KV4CacheStruct(P, P, P, P, 100, 16, 8, 128, 128)
out = []
for M, B, pages, rows in ((1, 1, 1, 1), (1, 1, 4096, 1), (64, 64, 512, 1), (600, 3, 512, 500)):
    b = comet.KV4BatchStruct(P, P, P, B, M, pages, rows)
    n = comet.comet_kv4_attention_workspace(c, b, 32, 256)
    comet.comet_rope(P, P, P, P, M, 40, 128, 128, 6144, 6144, stream=0x1000)
    comet.comet_kv4_append(c, b, P, P, 1024, 1024, stream=0x1000)
    comet.comet_kv4_gather(c, b, P, P, 1024, 1024, stream=0x1000)
    comet.comet_kv4_attention(c, b, P, P, 32, 4096, 4096, 0.1, 0, P if n else None, n, stream=0x1000)
    out.append(log())
    try:  # one byte less
        if n:
            comet.comet_kv4_attention(c, b, P, P, 32, 4096, 4096, 0.1, 0, P, n - 1, stream=0x1000)
            out[-1].append("not refused")
    except comet.CometError as e:
        out[-1] += log() if "workspace" in str(e) else [str(e)]
print(json.dumps(out))
""")
    for lines in out:
        assert len(lines) >= 4
        assert all(line.startswith(f"launch {0x1000} ") for line in lines), lines
