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


# --- numbers that do not fit the 32 bits of the interface --------------------------------

def meta_rows(rows, heads, D, stride):
    import torch

    comet._need_torch()
    return torch.empty_strided((rows, heads, D), (stride, D, 1), dtype=torch.float16, device="meta")


@pytest.mark.parametrize("stride", [2 ** 31, 2 ** 32 + 128, 2 ** 40])
def test_row_strides_beyond_32_bits(stride):
    # the last tokens of sequences of 2^18 in a padded batch, for instance
    t = meta_rows(2, 1, 64, stride)
    with pytest.raises(ValueError, match="x: .*stride"):
        comet._heads_of(t, "x", t.get_device())
    assert comet._heads_of(meta_rows(1, 1, 64, stride), "x", t.get_device())[3] == 64
    near = meta_rows(2, 1, 64, 2 ** 31 - 64)
    assert comet._heads_of(near, "x", t.get_device()) == (2, 1, 64, 2 ** 31 - 64)


@pytest.mark.parametrize("stride", [2 ** 31, 2 ** 32 + 512])
def test_raw_strides_beyond_32_bits(stride):
    F = 0x10000
    for call in (lambda: comet.comet_rope(F, F, F, 2 * F, 2, 3, 64, 32, stride, 512, stream=0),
                 lambda: comet.comet_rope(F, F, F, 2 * F, 2, 3, 64, 32, 512, stride, stream=0),
                 lambda: comet.comet_kv4_append(cache(), batch(), F, F, stride, 256, stream=0),
                 lambda: comet.comet_kv4_gather(cache(), batch(), F, F, 256, stride, stream=0),
                 lambda: comet.comet_kv4_attention(cache(), batch(), F, F, 4, stride, 512, 0.1,
                                                   stream=0),
                 lambda: comet.comet_kv4_attention(cache(), batch(), F, F, 4, 512, stride, 0.1,
                                                   stream=0)):
        with pytest.raises(ValueError, match="stride"):
            call()


def test_windows_and_row_counts_beyond_32_bits(monkeypatch):
    F = 0x10000
    with pytest.raises(ValueError, match="window"):
        comet.comet_kv4_attention(cache(), batch(), F, F, 4, 512, 512, 0.1, window=2 ** 32 + 5,
                                  stream=0)
    # a window that reaches over everything has no effect; no sequence has more rows than there are
    import torch

    seen = []

    class Library:
        def comet_kv4_attention(self, *args):
            seen.append(args)
            return 0

    class Handle:
        struct = address = None
        M, head_dim = 2, 64

    t = meta_rows(2, 4, 64, 256)
    monkeypatch.setattr(comet, "_lib", Library())
    monkeypatch.setattr(comet, "_kv4_here", lambda *a: t.get_device())
    monkeypatch.setattr(comet, "_plain", lambda *a: None)
    ws = torch.empty(0, dtype=torch.uint8)
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda self: F)
    for window in (2 ** 31 - 1, 2 ** 31, 2 ** 32 + 5, 2 ** 63):
        comet.kv4_attention(t, Handle, Handle, window=window, out=t, workspace=ws, stream=0)
        assert seen[-1][8] == 2 ** 31 - 1
    comet.kv4_attention(t, Handle, Handle, window=7, out=t, workspace=ws, stream=0)
    assert seen[-1][8] == 7
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    monkeypatch.setattr(comet, "_tensor", lambda *a: None)
    b = comet.KV4Batch(ints(0, 1, 3), ints(5, 9), ints(0, 1).view(2, 1), 3, 2 ** 32 + 1)
    assert b.max_rows == b.struct.max_rows == 3


# --- the largest launches ------------------------------------------------------------------

@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    return hip_record.library(str(tmp_path_factory.mktemp("hip_record")))


def attention_launches(shim, cases):
    """Per case (kv heads, heads, B, M, max_pages, max_rows): the kernels that a call launches,
    or why it is refused."""
    return hip_record.run(shim, f"""
out = []
for kvh, heads, B, M, pages, rows in {cases!r}:
    c = comet.KV4CacheStruct(P, P, P, P, 1 << 20, 16, kvh, 64, 64)
    b = comet.KV4BatchStruct(P, P, P, B, M, pages, rows)
    n = comet.comet_kv4_attention_workspace(c, b, heads, 256)
    try:
        comet.comet_kv4_attention(c, b, P, P, heads, 64 * heads, 64 * heads, 0.1, 0, P, n, stream=1)
        out.append([line.split()[2] for line in log()])
    except comet.CometError as e:
        out.append([str(e)] + log())
print(json.dumps(out))
""")


def test_batches_that_always_run(shim):
    """What comet.h says that is never too large for a launch, at its ends, and beyond."""
    ends = [(8, 128, 1, (1 << 27) // 128, 1, 1 << 20), (64, 64, 65536, 65536, 1, 1),
            (64, 1024, 65536, 65536 * 2, 9, 9), (1, 64, 65536, 65535 * 32, 64, 40),
            (1024, 1024, 4096, 4096 * 32, 5, 32)]
    for case, kernels in zip(ends, attention_launches(shim, ends)):
        assert len(kernels) >= 1 and all("kernel" in k for k in kernels), (case, kernels)
    beyond = [(1024, 1024, 65536, 65536, 1, 1), (8, 1024, 8, 65535 * 32, 64, 1 << 20)]
    for case, kernels in zip(beyond, attention_launches(shim, beyond)):
        assert len(kernels) == 1 and "too many rows" in kernels[0], (case, kernels)


# --- handles ---------------------------------------------------------------------------------

def test_handles_keep_the_tensors_they_were_made_of(monkeypatch):
    """Another tensor in a handle's place would leave the calls with the address of the first
    one, which nothing keeps alive any more: refused.  Its contents may change."""
    import torch

    monkeypatch.setattr(comet, "_tensor", lambda *a: None)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    b = comet.KV4Batch(ints(0, 1, 3), ints(5, 9), ints(0, 1).view(2, 1), 3)
    codes, params = torch.zeros((4, 2, 16, 32), dtype=torch.uint8), torch.zeros((4, 2, 16, 2, 2))
    c = comet.KV4Cache(codes, params, codes, params)
    for handle, name, value in ((b, "seq_lens", b.seq_lens + 1), (b, "row_start", ints(0, 1, 3)),
                                (b, "block_table", ints(0, 1).view(2, 1)), (b, "M", 2),
                                (b, "max_rows", 1), (b, "struct", None), (c, "k_codes", codes.clone()),
                                (c, "v_params", params.clone()), (c, "G", 64), (c, "address", 0)):
        before = getattr(handle, name)
        with pytest.raises(AttributeError, match=name):
            setattr(handle, name, value)
        assert getattr(handle, name) is before
    lens = b.seq_lens
    b.seq_lens.add_(1)
    b.seq_lens += 1
    assert b.seq_lens is lens and b.struct.seq_lens == lens.data_ptr() and lens.tolist() == [7, 11]
