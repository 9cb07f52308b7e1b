"""Python binding of libcomet (include/comet.h): COMET's W4Ax hot path on MI355X.

The functions named like the C entry points pass tensor data pointers, sizes
and the current HIP stream straight through ctypes; every step of the path
runs in libcomet's gfx950 kernels.  PyTorch only provides device memory and
streams.  There is no CPU fallback: if libcomet.so is missing and cannot be
built, importing a function raises.

Convenience wrappers (``quantize_act``, ``pack_w4``, ``w4ax_gemm``,
``channel_absmax``, ``plan_channel_perm``, ``kv4_quantize``, ``kv4_dequantize``,
``rope``, ``kv4_append``, ``kv4_gather``, ``kv4_attention``) allocate the outputs
with ``torch.empty`` and call the same entry points.  ``KV4Cache`` and
``KV4Batch`` hold what the calls on the paged cache share.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcomet.so")
G = 128

_lib = None


class CometError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_status_name(status)}: {message}")
        self.status = status


def _status_name(s: int) -> str:
    return {0: "COMET_OK", 1: "COMET_ERR_INVALID_ARG", 2: "COMET_ERR_UNSUPPORTED",
            3: "COMET_ERR_HIP", 4: "COMET_ERR_OOM"}.get(s, f"status {s}")


def lib():
    """The loaded libcomet.so.  A library file whose source stamp differs from
    the sources in this tree (or a missing one) is rebuilt in-tree with hipcc
    before loading, or, with COMET_NO_REBUILD=1 in the environment, refused;
    a stale build is never loaded."""
    global _lib
    if _lib is not None:
        return _lib
    from . import build as _build

    want = _build.source_stamp()
    have = _build.library_stamp(LIB_PATH)
    if have != want:
        if os.environ.get("COMET_NO_REBUILD"):
            raise RuntimeError(f"{LIB_PATH} was built from other sources (stamp {have}, sources "
                               f"{want}) and COMET_NO_REBUILD is set; rebuild it")
        _build.build()
        have = _build.library_stamp(LIB_PATH)
        if have != want:
            raise RuntimeError(f"{LIB_PATH}: stamp {have} after rebuilding, sources {want}")
    L = ctypes.CDLL(LIB_PATH)
    P, I, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    sigs = {
        "comet_act_packed_bytes": (S, [P, I, I, I]),
        "comet_fmpq_quantize_act": (I, [P, P, P, P, I, I, I, P]),
        "comet_pack_w4": (I, [P, P, P, I, I, I, P]),
        "comet_w4ax_gemm": (I, [P, P, P, P, P, P, I, I, I, I, P]),
        "comet_w4ax_gemm_acc": (I, [P, P, P, P, P, P, I, I, I, I, I, I, I, I, P]),
        "comet_schedule_query": (I, [I, I, I, I, P, I, P, I, P, P, I, P, P, P, P]),
        "comet_fmpq_quantize_act_perm": (I, [P, P, P, P, P, I, I, I, P]),
        "comet_pack_w4_perm": (I, [P, P, P, P, I, I, I, P]),
        "comet_channel_absmax": (I, [P, P, I, I, P]),
        "comet_plan_channel_perm": (I, [P, I, I, ctypes.c_float, ctypes.c_float, P, P, P]),
        "comet_kv4_quantize": (I, [P, P, P, I, I, I, P]),
        "comet_kv4_dequantize": (I, [P, P, P, I, I, I, P]),
        "comet_w4ax_gemm_swiglu_quant": (I, [P, P, P, P, P, I, I, I, I, P, P, P, P]),
        "comet_swiglu_quantize": (I, [P, P, P, P, I, I, I, P]),
        "comet_rope": (I, [P, P, P, P, I, I, I, I, I, I, I, ctypes.c_float, P]),
        "comet_rope_frequencies": (I, [P, I, ctypes.c_double, I] + [ctypes.c_double] * 4 + [P]),
        "comet_kv4_append": (I, [P, P, P, P, I, I, P]),
        "comet_kv4_gather": (I, [P, P, P, P, I, I, P]),
        "comet_kv4_attention": (I, [P, P, P, P, I, I, I, ctypes.c_float, I, P, S, P]),
        "comet_kv4_attention_workspace": (S, [P, P, I, I]),
        "comet_gemm_kernel": (I, [I, I, I, I, I]),
        "comet_w4ax_gemm_noalloc": (I, [P, P, P, P, P, P, I, I, I, I, P]),
        "comet_build_stamp": (ctypes.c_char_p, []),
        "comet_status_str": (ctypes.c_char_p, [I]),
        "comet_last_error": (ctypes.c_char_p, []),
        "comet_release_caches": (None, []),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    if L.comet_build_stamp().decode() != want:
        raise RuntimeError(f"{LIB_PATH} reports stamp {L.comet_build_stamp().decode()}, "
                           f"sources {want}")
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        raise CometError(status, lib().comet_last_error().decode())


# A decode step makes a few of these calls per layer, each for a kernel of a few
# microseconds, so the argument handling counts: addresses go to ctypes as plain
# integers and the block map as the bytes object it is checked on.  (LLaMA-3-8B
# qkv for one token, quantize and GEMM: 22.6 us a pass before, 12.0 now.)

def _ptr(t):
    """What ctypes takes as a pointer: an address, None, or the map's bytes."""
    if t is None or isinstance(t, (int, bytes)):
        return t
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


# The lookup of the current stream, once the device is initialized (in this
# process: a forked child starts over, and torch refuses it there).
_raw_stream = None


def _forget_stream():
    global _raw_stream
    _raw_stream = None


os.register_at_fork(after_in_child=_forget_stream)


def _stream(stream):
    if stream is None:
        global _raw_stream
        if _raw_stream is None:
            import torch

            torch.cuda.current_stream()  # initializes the device
            device = getattr(torch._C, "_cuda_getDevice", None)
            raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
            if device is not None and raw is not None:
                _raw_stream = lambda: raw(device())
            else:
                _raw_stream = lambda: torch.cuda.current_stream().cuda_stream
        return _raw_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _tensor(t, dtype: str, name: str):
    """A convenience wrapper's tensor argument.  The kernels read plain
    row-major device memory, so a view with strides, another dtype or a host
    tensor would be misread; they are rejected here instead."""
    import torch

    want = getattr(torch, dtype)
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != want or not t.is_contiguous():
        got = (f"{t.dtype} on {t.device}{'' if t.is_contiguous() else ', strided'}"
               if isinstance(t, torch.Tensor) else type(t).__name__)
        raise ValueError(f"{name}: need a contiguous {dtype} CUDA tensor, got {got}")
    return t


def _map(prec, K: Optional[int] = None, G: int = G, name: str = "group_prec_map") -> bytes:
    """The host block-precision map as bytes.  With K given, it must hold
    exactly K / G entries: the library reads that many from the pointer."""
    m = np.asarray(prec, dtype=np.uint8).tobytes()
    if K is not None and G > 0 and K % G == 0 and len(m) != K // G:
        raise ValueError(f"{name}: {len(m)} entries, need K/G = {K // G}")
    return m


def _nbytes(t) -> Optional[int]:
    """Size in bytes of a tensor or array argument (None for raw pointers)."""
    if t is None or isinstance(t, int):
        return None
    return t.nbytes


def _room(t, need: int, name: str) -> None:
    """A buffer passed as a tensor or array must hold at least `need` bytes
    (the kernels read or write that many); raw integer pointers are the
    caller's responsibility."""
    have = _nbytes(t)
    if have is not None and need > 0 and have < need:
        raise ValueError(f"{name}: {have} bytes, the call needs {need}")


def _act_bytes(m: bytes, M: int, G_: int) -> int:
    """Bytes of A_packed, as comet_act_packed_bytes counts them (0: an entry is
    neither 4 nor 8)."""
    n8 = m.count(8)
    if n8 + m.count(4) != len(m):
        return 0
    return M * ((len(m) - n8) * (G_ // 2) + n8 * G_)


def _gemm_room(A_packed, m, a_scales, W_packed, w_scales, M, N, K, G_):
    if M > 0 and N > 0 and K > 0 and G_ > 0 and K % G_ == 0:
        NG = K // G_
        _room(A_packed, _act_bytes(m, M, G_), "A_packed")
        _room(a_scales, 2 * NG * M, "a_scales")
        _room(W_packed, N * K // 2, "W_packed")
        _room(w_scales, 2 * NG * N, "w_scales")


# --- the C entry points ----------------------------------------------------------

def comet_act_packed_bytes(group_prec_map, M: int, K: int, G: int = G) -> int:
    m = _map(group_prec_map, K, G)
    return int(lib().comet_act_packed_bytes(_ptr(m), M, K, G))


def comet_fmpq_quantize_act(X, group_prec_map, A_packed, a_scales, M: int, K: int, G: int = G,
                            stream=None) -> None:
    m = _map(group_prec_map, K, G)
    _quant_room(X, m, A_packed, a_scales, M, K, G)
    _check(lib().comet_fmpq_quantize_act(_ptr(X), _ptr(m), _ptr(A_packed), _ptr(a_scales), M, K,
                                         G, _stream(stream)))


def _quant_room(X, m, A_packed, a_scales, M, K, G_):
    if M > 0 and K > 0 and G_ > 0 and K % G_ == 0:
        _room(X, 2 * M * K, "X")
        _room(A_packed, _act_bytes(m, M, G_), "A_packed")
        _room(a_scales, 2 * (K // G_) * M, "a_scales")


def _pack_room(W, W_packed, w_scales, N, K, G_):
    if N > 0 and K > 0 and G_ > 0 and K % G_ == 0:
        _room(W, 2 * N * K, "W")
        _room(W_packed, N * K // 2, "W_packed")
        _room(w_scales, 2 * (K // G_) * N, "w_scales")


def comet_pack_w4(W, W_packed, w_scales, N: int, K: int, G: int = G, stream=None) -> None:
    _pack_room(W, W_packed, w_scales, N, K, G)
    _check(lib().comet_pack_w4(_ptr(W), _ptr(W_packed), _ptr(w_scales), N, K, G,
                               _stream(stream)))


def comet_fmpq_quantize_act_perm(X, perm, group_prec_map, A_packed, a_scales, M: int, K: int,
                                 G: int = G, stream=None) -> None:
    m = _map(group_prec_map, K, G)
    _quant_room(X, m, A_packed, a_scales, M, K, G)
    _room(perm, 4 * K, "perm")
    _check(lib().comet_fmpq_quantize_act_perm(_ptr(X), _ptr(perm), _ptr(m), _ptr(A_packed),
                                              _ptr(a_scales), M, K, G, _stream(stream)))


def comet_pack_w4_perm(W, perm, W_packed, w_scales, N: int, K: int, G: int = G,
                       stream=None) -> None:
    _pack_room(W, W_packed, w_scales, N, K, G)
    _room(perm, 4 * K, "perm")
    _check(lib().comet_pack_w4_perm(_ptr(W), _ptr(perm), _ptr(W_packed), _ptr(w_scales), N, K, G,
                                    _stream(stream)))


def comet_channel_absmax(X, absmax, M: int, K: int, stream=None) -> None:
    if M > 0 and K > 0:
        _room(X, 2 * M * K, "X")
        _room(absmax, 4 * K, "absmax")
    _check(lib().comet_channel_absmax(_ptr(X), _ptr(absmax), M, K, _stream(stream)))


def comet_plan_channel_perm(absmax, K: int, G: int, outlier_ratio: float, max_frac_8bit: float,
                            perm, group_prec_map, n_outliers=None) -> None:
    """Host-only: absmax, perm, group_prec_map (and n_outliers) are host numpy arrays."""
    if K > 0 and G > 0 and K % G == 0:
        _room(absmax, 4 * K, "absmax")
        _room(perm, 4 * K, "perm")
        _room(group_prec_map, K // G, "group_prec_map")
        _room(n_outliers, 4, "n_outliers")
    _check(lib().comet_plan_channel_perm(_ptr(absmax), K, G, outlier_ratio, max_frac_8bit,
                                         _ptr(perm), _ptr(group_prec_map), _ptr(n_outliers)))


def _kv4_room(X, codes, params, T, C, G_, xname):
    if T > 0 and C > 0 and G_ > 0 and C % G_ == 0:
        _room(X, 2 * T * C, xname)
        _room(codes, T * C // 2, "codes")
        _room(params, 4 * T * (C // G_), "params")


def comet_kv4_quantize(X, codes, params, T: int, C: int, G: int = 128, stream=None) -> None:
    _kv4_room(X, codes, params, T, C, G, "X")
    _check(lib().comet_kv4_quantize(_ptr(X), _ptr(codes), _ptr(params), T, C, G,
                                    _stream(stream)))


def comet_kv4_dequantize(codes, params, out, T: int, C: int, G: int = 128, stream=None) -> None:
    _kv4_room(out, codes, params, T, C, G, "out")
    _check(lib().comet_kv4_dequantize(_ptr(codes), _ptr(params), _ptr(out), T, C, G,
                                      _stream(stream)))


ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}


def comet_rope(X, positions, freqs, out, M: int, heads: int, head_dim: int, rot_dim: int,
               x_stride: int, out_stride: int, interleaved: bool = False, mscale: float = 1.0,
               stream=None) -> None:
    if M > 0 and heads > 0:
        _row_room(X, M, x_stride, heads * head_dim, "X")
        _room(positions, 4 * M, "positions")
        _room(freqs, 4 * rot_dim, "freqs")
        _row_room(out, M, out_stride, heads * head_dim, "out")
    _check(lib().comet_rope(_ptr(X), _ptr(positions), _ptr(freqs), _ptr(out), M, heads, head_dim,
                            rot_dim, x_stride, out_stride, int(bool(interleaved)), mscale,
                            _stream(stream)))


def comet_rope_frequencies(freqs, rot_dim: int, base: float, scaling: int, factor: float,
                           low: float, high: float, original_len: float, mscale=None) -> None:
    """Host-only: freqs (and mscale) are host numpy arrays, float64 and float32."""
    _room(freqs, 4 * rot_dim, "freqs")
    _room(mscale, 4, "mscale")
    _check(lib().comet_rope_frequencies(_ptr(freqs), rot_dim, base, scaling, factor, low, high,
                                        original_len, _ptr(mscale)))


class KV4CacheStruct(ctypes.Structure):
    """comet_kv4_cache_t"""

    _fields_ = [(n, ctypes.c_void_p) for n in ("k_codes", "k_params", "v_codes", "v_params")] + [
        (n, ctypes.c_int) for n in ("num_pages", "page_size", "kv_heads", "head_dim", "G")]


class KV4BatchStruct(ctypes.Structure):
    """comet_kv4_batch_t"""

    _fields_ = [(n, ctypes.c_void_p) for n in ("row_start", "seq_lens", "block_table")] + [
        (n, ctypes.c_int) for n in ("B", "M", "max_pages", "max_rows")]


_INT_MAX = 2 ** 31 - 1  # larger numbers would lose their upper bits on the way


def _row_room(t, M: int, stride: int, width: int, name: str) -> None:
    """A tensor of fp16 rows must reach, from its first element to the end of its
    storage, over M rows of `width` elements, `stride` apart; the stride is an int of
    the interface."""
    if stride > _INT_MAX:
        raise ValueError(f"{name}: stride {stride} exceeds 2^31 - 1")
    if t is None or isinstance(t, int):
        return
    have = t.nbytes if isinstance(t, np.ndarray) else (
        t.untyped_storage().nbytes() - t.storage_offset() * t.element_size())
    need = 2 * ((M - 1) * stride + width)
    if have < need:
        raise ValueError(f"{name}: {have} bytes, the call needs {need}")


def _struct(s):
    """A KV4Cache or KV4Batch as the address of its struct (None stays null)."""
    if s is None:
        return None
    return s.address if hasattr(s, "address") else ctypes.addressof(s)


def _kv4_row_room(cache, batch, K, V, k_stride: int, v_stride: int) -> None:
    if cache is None or batch is None:
        return
    c, b = getattr(cache, "struct", cache), getattr(batch, "struct", batch)
    if b.M > 0 and c.kv_heads > 0:
        _row_room(K, b.M, k_stride, c.kv_heads * c.head_dim, "K")
        _row_room(V, b.M, v_stride, c.kv_heads * c.head_dim, "V")


def comet_kv4_append(cache, batch, K, V, k_stride: int, v_stride: int, stream=None) -> None:
    _kv4_row_room(cache, batch, K, V, k_stride, v_stride)
    _check(lib().comet_kv4_append(_struct(cache), _struct(batch), _ptr(K), _ptr(V), k_stride,
                                  v_stride, _stream(stream)))


def comet_kv4_gather(cache, batch, K, V, k_stride: int, v_stride: int, stream=None) -> None:
    _kv4_row_room(cache, batch, K, V, k_stride, v_stride)
    _check(lib().comet_kv4_gather(_struct(cache), _struct(batch), _ptr(K), _ptr(V), k_stride,
                                  v_stride, _stream(stream)))


def comet_kv4_attention(cache, batch, Q, out, heads: int, q_stride: int, out_stride: int,
                        scale: float, window: int = 0, workspace=None, workspace_bytes=None,
                        stream=None) -> None:
    if cache is not None and batch is not None:
        c, b = getattr(cache, "struct", cache), getattr(batch, "struct", batch)
        if b.M > 0 and heads > 0:
            _row_room(Q, b.M, q_stride, heads * c.head_dim, "Q")
            _row_room(out, b.M, out_stride, heads * c.head_dim, "out")
    if window > _INT_MAX:
        raise ValueError(f"window: {window} exceeds 2^31 - 1")
    have = _nbytes(workspace)
    if workspace_bytes is None:
        workspace_bytes = have or 0
    elif have is not None and have < workspace_bytes:
        raise ValueError(f"workspace: {have} bytes, workspace_bytes says {workspace_bytes}")
    _check(lib().comet_kv4_attention(_struct(cache), _struct(batch), _ptr(Q), _ptr(out), heads,
                                     q_stride, out_stride, scale, window, _ptr(workspace),
                                     workspace_bytes, _stream(stream)))


def comet_kv4_attention_workspace(cache, batch, heads: int, num_cus: int) -> int:
    return int(lib().comet_kv4_attention_workspace(_struct(cache), _struct(batch), heads, num_cus))


def comet_w4ax_gemm_swiglu_quant(A_packed, group_prec_map, a_scales, W_packed, w_scales, M: int,
                                 N: int, K: int, G: int, out_prec_map, out_A_packed, out_a_scales,
                                 stream=None) -> None:
    m = _map(group_prec_map, K, G)
    om = _map(out_prec_map, N // 2, G, "out_prec_map")
    _gemm_room(A_packed, m, a_scales, W_packed, w_scales, M, N, K, G)
    if M > 0 and N > 0 and (N // 2) % G == 0:
        _room(out_A_packed, _act_bytes(om, M, G), "out_A_packed")
        _room(out_a_scales, 2 * (N // 2 // G) * M, "out_a_scales")
    _check(lib().comet_w4ax_gemm_swiglu_quant(_ptr(A_packed), _ptr(m), _ptr(a_scales),
                                              _ptr(W_packed), _ptr(w_scales), M, N, K, G,
                                              _ptr(om), _ptr(out_A_packed), _ptr(out_a_scales),
                                              _stream(stream)))


def comet_swiglu_quantize(gu, out_prec_map, out_A_packed, out_a_scales, M: int, I: int,
                          G: int = G, stream=None) -> None:
    om = _map(out_prec_map, I, G, "out_prec_map")
    if M > 0 and I > 0 and I % G == 0:
        _room(gu, 4 * M * I, "gu")
        _room(out_A_packed, _act_bytes(om, M, G), "out_A_packed")
        _room(out_a_scales, 2 * (I // G) * M, "out_a_scales")
    _check(lib().comet_swiglu_quantize(_ptr(gu), _ptr(om), _ptr(out_A_packed),
                                       _ptr(out_a_scales), M, I, G, _stream(stream)))


def comet_w4ax_gemm(A_packed, group_prec_map, a_scales, W_packed, w_scales, out, M: int, N: int,
                    K: int, G: int = G, stream=None) -> None:
    m = _map(group_prec_map, K, G)
    _gemm_room(A_packed, m, a_scales, W_packed, w_scales, M, N, K, G)
    _room(out, 2 * M * N, "out")
    _check(lib().comet_w4ax_gemm(_ptr(A_packed), _ptr(m), _ptr(a_scales), _ptr(W_packed),
                                 _ptr(w_scales), _ptr(out), M, N, K, G, _stream(stream)))


def comet_w4ax_gemm_noalloc(A_packed, group_prec_map, a_scales, W_packed, w_scales, out, M: int,
                            N: int, K: int, G: int = G, stream=None) -> None:
    m = _map(group_prec_map, K, G)
    _gemm_room(A_packed, m, a_scales, W_packed, w_scales, M, N, K, G)
    _room(out, 2 * M * N, "out")
    _check(lib().comet_w4ax_gemm_noalloc(_ptr(A_packed), _ptr(m), _ptr(a_scales), _ptr(W_packed),
                                         _ptr(w_scales), _ptr(out), M, N, K, G, _stream(stream)))


def comet_w4ax_gemm_acc(A_packed, group_prec_map, a_scales, W_packed, w_scales, acc, M: int,
                        N: int, K: int, G: int, m0: int, m1: int, n0: int, n1: int,
                        stream=None) -> None:
    m = _map(group_prec_map, K, G)
    _gemm_room(A_packed, m, a_scales, W_packed, w_scales, M, N, K, G)
    if G > 0 and K % G == 0 and m1 > m0 and n1 > n0:
        _room(acc, 4 * (m1 - m0) * (n1 - n0) * (K // G), "acc")
    _check(lib().comet_w4ax_gemm_acc(_ptr(A_packed), _ptr(m), _ptr(a_scales), _ptr(W_packed),
                                     _ptr(w_scales), _ptr(acc), M, N, K, G, m0, m1, n0, n1,
                                     _stream(stream)))


def comet_schedule_query(M: int, N: int, K: int, group_prec_map, num_cus: int = 256,
                         G: int = G) -> dict:
    """Host-only view of the GEMM's tile schedule (no device needed)."""
    m = _map(group_prec_map, K, G)
    L = lib()
    nu, nw, tm, tn = ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(L.comet_schedule_query(M, N, K, G, _ptr(m), num_cus, None, 0, ctypes.byref(nu), None,
                                  0, ctypes.byref(nw), None, ctypes.byref(tm), ctypes.byref(tn)))
    units = np.zeros((nu.value, 5), np.int32)
    wgb = np.zeros(nw.value + 1, np.int32)
    order = np.zeros(K // G, np.int32)
    _check(L.comet_schedule_query(M, N, K, G, _ptr(m), num_cus, _ptr(units), nu.value,
                                  ctypes.byref(nu), _ptr(wgb), nw.value + 1, ctypes.byref(nw),
                                  _ptr(order), ctypes.byref(tm), ctypes.byref(tn)))
    return {"units": units, "wg_begin": wgb, "order": order, "tile_m": tm.value,
            "tile_n": tn.value, "num_wgs": nw.value}


def comet_gemm_kernel(M: int, N: int, K: int, num_cus: int, G: int = G) -> int:
    """Host-only: the comet_kernel_t that comet_w4ax_gemm runs for this shape."""
    k = lib().comet_gemm_kernel(M, N, K, G, num_cus)
    if k < 0:
        raise CometError(1, lib().comet_last_error().decode())
    return k


KERNEL_NAMES = {0: "skinny", 1: "skinny_shared", 2: "mid", 3: "tile", 4: "stream", 5: "pair"}


def comet_build_stamp() -> str:
    return lib().comet_build_stamp().decode()


def comet_last_error() -> str:
    return lib().comet_last_error().decode()


def comet_status_str(status: int) -> str:
    return lib().comet_status_str(status).decode()


def comet_release_caches() -> None:
    lib().comet_release_caches()


# --- allocating conveniences (torch tensors on the current device) ----------------

def quantize_act(X, group_prec_map, perm=None, stream=None):
    """X: float16 [M][K] CUDA tensor -> (A_packed uint8, a_scales float16 [K/G][M]).
    perm: optional int32 [K] CUDA tensor (channel permutation)."""
    import torch

    _tensor(X, "float16", "X")
    M, K = X.shape
    if perm is not None:
        _tensor(perm, "int32", "perm")
        _exact(perm, K, "perm")
    nbytes = comet_act_packed_bytes(group_prec_map, M, K)
    if nbytes == 0:
        raise CometError(1, "invalid map or shape")
    A = torch.empty(nbytes, dtype=torch.uint8, device=X.device)
    sa = torch.empty((K // G, M), dtype=torch.float16, device=X.device)
    comet_fmpq_quantize_act_perm(X, perm, group_prec_map, A, sa, M, K, G, stream)
    return A, sa


def pack_w4(W, perm=None, stream=None):
    """W: float16 [N][K] CUDA tensor -> (W_packed uint8 [N][K/2], w_scales float16 [K/G][N]).
    perm: optional int32 [K] CUDA tensor (the activations' channel permutation)."""
    import torch

    _tensor(W, "float16", "W")
    N, K = W.shape
    if perm is not None:
        _tensor(perm, "int32", "perm")
        _exact(perm, K, "perm")
    Wp = torch.empty((N, K // 2), dtype=torch.uint8, device=W.device)
    sw = torch.empty((K // G, N), dtype=torch.float16, device=W.device)
    comet_pack_w4_perm(W, perm, Wp, sw, N, K, G, stream)
    return Wp, sw


def channel_absmax(X, absmax=None, stream=None):
    """Running per-channel max |X| (float32 [K] CUDA tensor), accumulated into absmax."""
    import torch

    _tensor(X, "float16", "X")
    M, K = X.shape
    if absmax is None:
        absmax = torch.zeros(K, dtype=torch.float32, device=X.device)
    _tensor(absmax, "float32", "absmax")
    _exact(absmax, K, "absmax")
    comet_channel_absmax(X, absmax, M, K, stream)
    return absmax


def plan_channel_perm(absmax, G: int = G, outlier_ratio: float = 8.0, max_frac_8bit: float = 0.2):
    """Host: per-channel maxima (numpy or tensor) -> (perm int32 [K], map uint8 [K/G], n_outliers)."""
    a = np.ascontiguousarray(np.asarray(absmax.cpu() if hasattr(absmax, "cpu") else absmax,
                                        dtype=np.float32).reshape(-1))
    K = a.size
    perm = np.empty(K, np.int32)
    prec = np.empty(max(K // G, 1), np.uint8)
    nout = np.zeros(1, np.int32)
    comet_plan_channel_perm(a, K, G, outlier_ratio, max_frac_8bit, perm, prec, nout)
    return perm, prec[: K // G], int(nout[0])


def kv4_quantize(X, G: int = 128, stream=None):
    """X: float16 [T][C] CUDA tensor -> (codes uint8 [T][C/2], params float16 [T][C/G][2])."""
    import torch

    _tensor(X, "float16", "X")
    T, C = X.shape
    codes = torch.empty((T, C // 2), dtype=torch.uint8, device=X.device)
    params = torch.empty((T, C // G, 2), dtype=torch.float16, device=X.device)
    comet_kv4_quantize(X, codes, params, T, C, G, stream)
    return codes, params


def kv4_dequantize(codes, params, G: int = 128, stream=None):
    import torch

    _tensor(codes, "uint8", "codes")
    _tensor(params, "float16", "params")
    if codes.dim() != 2:
        raise ValueError(f"codes: need [T][C/2], got shape {tuple(codes.shape)}")
    T, C = codes.shape[0], codes.shape[1] * 2
    if C % G:
        raise ValueError(f"C={C} is not a multiple of G={G}")
    _exact(params, T * (C // G) * 2, "params")
    out = torch.empty((T, C), dtype=torch.float16, device=codes.device)
    comet_kv4_dequantize(codes, params, out, T, C, G, stream)
    return out


def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "none",
                     factor: float = 1.0, low: float = 1.0, high: float = 4.0,
                     original_len: float = 8192.0):
    """Host: (float64 numpy array [rot_dim / 2] of radians per position, mscale) for
    ``rope``; scaling is a key of ROPE_SCALINGS (comet_rope_scaling_t)."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling: {scaling!r}, known are {', '.join(ROPE_SCALINGS)}")
    freqs = np.empty(max(rot_dim // 2, 1), np.float64)
    mscale = np.ones(1, np.float32)
    comet_rope_frequencies(freqs, rot_dim, base, ROPE_SCALINGS[scaling], factor, low, high,
                           original_len, mscale)
    return freqs, float(mscale[0])


# torch and its lookup of the current device, once a wrapper below has needed
# them.  These wrappers run several times per layer and token, so an argument that
# is as it should be passes with few lookups.  (rope of one token: 6.7 us a call
# when each check was made by itself, of which the library's own part is 3.3.)
_torch = None
_current_device = None
_float16 = _float64 = _int32 = None


def _need_torch():
    global _torch, _current_device, _float16, _float64, _int32
    import torch

    _float16, _float64, _int32 = torch.float16, torch.float64, torch.int32
    if not torch.cuda.is_available():
        _current_device = lambda: -2  # where no tensor is
    else:
        torch.cuda.current_device()  # initializes the device
        _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _torch = torch
    return _current_device()


def _forget_torch():
    global _torch
    _torch = None


os.register_at_fork(after_in_child=_forget_torch)


def _here() -> int:
    """The current device's number, which a call's tensors must be on."""
    return _need_torch() if _torch is None else _current_device()


def _heads_of(t, name: str, here: int):
    """(rows, heads, channels, row stride) of a float16 tensor [rows][heads][channels]
    on device `here` whose heads are contiguous; the rows may lie in a wider buffer
    (the q, k or v columns of a qkv output)."""
    try:
        M, H, D = t.shape
        s0, s1, s2 = t.stride()
        fits = t.dtype is _float16 and t.get_device() == here
    except (AttributeError, TypeError, ValueError):
        fits = False
    if not fits:
        _explain(t, name, here)
        got = (f"{t.dtype} {tuple(t.shape)} on {t.device}" if isinstance(t, _torch.Tensor)
               else type(t).__name__)
        raise ValueError(f"{name}: need a float16 CUDA tensor [rows][heads][channels], got {got}")
    if s2 == 1 and s1 == D and H * D <= s0 <= _INT_MAX:
        return M, H, D, s0
    if M > 1 and s0 > _INT_MAX:
        raise ValueError(f"{name}: row stride {s0} exceeds 2^31 - 1")
    if (s2 != 1 and D > 1) or (s1 != D and H > 1) or (s0 < H * D and M > 1):
        raise ValueError(f"{name}: heads and channels must be contiguous and rows apart, got "
                         f"strides {t.stride()} for {tuple(t.shape)}")
    return M, H, D, max(s0, H * D) if M > 1 else H * D


def _explain(t, name: str, here: int) -> None:
    """Raises for a tensor on another GPU."""
    at = t.get_device() if hasattr(t, "get_device") else -1
    if at >= 0 and at != here:
        raise ValueError(f"{name}: on device {at}, the current device is {here}")


def _plain(t, dtype: str, name: str, here: int) -> None:
    """Raises unless t is what _tensor asks for, on device `here`."""
    _tensor(t, dtype, name)
    _explain(t, name, here)


def _new(shape, dtype, device, stream):
    """Memory for work on `stream`: it is taken from that stream's own pool, so that no
    other stream's work is still using it, or gets it before this work is done."""
    import torch

    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    s = torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream
    with torch.cuda.stream(s):
        return torch.empty(shape, dtype=dtype, device=device)


def rope(x, positions, freqs, interleaved: bool = False, mscale: float = 1.0, out=None,
         stream=None):
    """Rotary positions.  x: float16 CUDA tensor [M][heads][head_dim] (rows may lie in a
    wider buffer); positions: int32 [M]; freqs: float64 [rot_dim / 2], of
    ``rope_frequencies``, on the GPU.  Returns out (out=x rotates in place)."""
    here = _here()
    M, H, D, xs = _heads_of(x, "x", here)
    for t, dtype, name in ((positions, _int32, "positions"), (freqs, _float64, "freqs")):
        if not (type(t) is _torch.Tensor and t.dtype is dtype and t.get_device() == here
                and t.is_contiguous()):
            _plain(t, str(dtype)[6:], name, here)
    if positions.numel() != M:
        _exact(positions, M, "positions")
    if out is None:
        out = _new((M, H, D), _torch.float16, x.device, stream)
        os_ = H * D
    else:
        oM, oH, oD, os_ = _heads_of(out, "out", here)
        if oM != M or oH != H or oD != D:
            raise ValueError(f"out: shape {tuple(out.shape)}, expected {(M, H, D)}")
    status = (_lib or lib()).comet_rope(x.data_ptr(), positions.data_ptr(), freqs.data_ptr(),
                                        out.data_ptr(), M, H, D, 2 * freqs.numel(), xs, os_,
                                        1 if interleaved else 0, mscale, _stream(stream))
    if status:
        _check(status)
    return out


class _Handle:
    """Tensors and the struct with their addresses.  An attribute is set once: another
    tensor in its place would not reach the struct, whose address nothing kept alive."""

    def __setattr__(self, name, value):
        if self.__dict__.get(name, value) is not value:  # (not so in `handle.lens += 1`)
            raise AttributeError(f"{type(self).__name__}.{name} is fixed: write into its tensor, "
                                 "or make a new object")
        self.__dict__[name] = value


class KV4Cache(_Handle):
    """A paged 4-bit K/V cache: codes uint8 [num_pages][kv_heads][page_size][head_dim / 2]
    and params float16 [num_pages][kv_heads][page_size][head_dim / G][2] of K and of V,
    contiguous CUDA tensors that this object keeps alive."""

    def __init__(self, k_codes, k_params, v_codes, v_params):
        for name, t, dtype, dim in (("k_codes", k_codes, "uint8", 4),
                                    ("k_params", k_params, "float16", 5),
                                    ("v_codes", v_codes, "uint8", 4),
                                    ("v_params", v_params, "float16", 5)):
            _tensor(t, dtype, name)
            if t.dim() != dim:
                raise ValueError(f"{name}: {t.dim()} dimensions, expected {dim}")
        pages, heads, size, half = k_codes.shape
        groups = k_params.shape[3]
        want = {"k_params": (pages, heads, size, groups, 2), "v_codes": (pages, heads, size, half),
                "v_params": (pages, heads, size, groups, 2)}
        for name, t in (("k_params", k_params), ("v_codes", v_codes), ("v_params", v_params)):
            if tuple(t.shape) != want[name]:
                raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {want[name]}")
            if t.device != k_codes.device:
                raise ValueError(f"{name}: on {t.device}, k_codes on {k_codes.device}")
        if groups < 1 or (2 * half) % groups:
            raise ValueError(f"k_params: {groups} groups do not divide {2 * half} channels")
        self.k_codes, self.k_params = k_codes, k_params
        self.v_codes, self.v_params = v_codes, v_params
        self.num_pages, self.page_size, self.kv_heads = pages, size, heads
        self.head_dim, self.G = 2 * half, 2 * half // groups
        self.device = k_codes.device
        self.struct = KV4CacheStruct(k_codes.data_ptr(), k_params.data_ptr(), v_codes.data_ptr(),
                                     v_params.data_ptr(), pages, size, heads, self.head_dim,
                                     self.G)
        self.address = ctypes.addressof(self.struct)

    @classmethod
    def empty(cls, num_pages: int, page_size: int, kv_heads: int, head_dim: int, G: int = 128,
              device="cuda"):
        """A new cache (its contents are written before they are read)."""
        import torch

        if G < 1 or head_dim % G:
            raise ValueError(f"head_dim={head_dim} is not a multiple of G={G}")
        rows = (num_pages, kv_heads, page_size)
        codes = [torch.empty(rows + (head_dim // 2,), dtype=torch.uint8, device=device)
                 for _ in "kv"]
        params = [torch.empty(rows + (head_dim // G, 2), dtype=torch.float16, device=device)
                  for _ in "kv"]
        return cls(codes[0], params[0], codes[1], params[1])


class KV4Batch(_Handle):
    """The rows of a call and where their sequences lie: row_start int32 [B + 1], seq_lens
    int32 [B], block_table int32 [B][max_pages] (comet_kv4_batch_t), CUDA tensors that this
    object keeps alive; their contents are read when the work runs.  M: rows of the buffers;
    max_rows: the most rows of one sequence (M if not given).  It decides which kernels
    kv4_attention launches: 64 single tokens without it take 3 to 4 us more a call (1024
    tokens each, 64 heads over 8: 24.5 us, 20.7 with max_rows=1) and 65 MB more of workspace."""

    def __init__(self, row_start, seq_lens, block_table, M: int, max_rows: Optional[int] = None):
        for name, t in (("row_start", row_start), ("seq_lens", seq_lens),
                        ("block_table", block_table)):
            _tensor(t, "int32", name)
            if t.device != seq_lens.device:
                raise ValueError(f"{name}: on {t.device}, seq_lens on {seq_lens.device}")
        B = seq_lens.numel()
        _exact(row_start, B + 1, "row_start")
        if block_table.dim() != 2 or block_table.shape[0] != B:
            raise ValueError(f"block_table: shape {tuple(block_table.shape)}, expected ({B}, pages)")
        max_pages = block_table.shape[1]
        max_rows = M if max_rows is None else min(max_rows, M)
        struct = KV4BatchStruct(row_start.data_ptr(), seq_lens.data_ptr(), block_table.data_ptr(), B,
                                M, max_pages, max_rows)
        # at once: a serving program makes one of these per step
        self.__dict__.update(row_start=row_start, seq_lens=seq_lens, block_table=block_table, B=B,
                             M=M, max_pages=max_pages, max_rows=max_rows, device=seq_lens.device,
                             struct=struct, address=ctypes.addressof(struct))


def _kv4_here(cache, batch) -> int:
    """The current device's number, which the cache and the batch must be on."""
    here = _here()
    if cache.device.index != here or batch.device.index != here:
        raise ValueError(f"cache on {cache.device}, batch on {batch.device}, the current device "
                         f"is {here}")
    return here


def _kv4_rows(t, cache, batch, name: str, here: int):
    """Row stride of a K or V buffer of this cache and batch."""
    M, H, D, stride = _heads_of(t, name, here)
    if M != batch.M or H != cache.kv_heads or D != cache.head_dim:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected "
                         f"{(batch.M, cache.kv_heads, cache.head_dim)}")
    return stride


def kv4_append(cache: KV4Cache, batch: KV4Batch, k, v, stream=None) -> None:
    """Quantizes the rows k, v (float16 [M][kv_heads][head_dim], rows may lie in a wider
    buffer) into the cache, each to its sequence's last positions."""
    here = _kv4_here(cache, batch)
    ks, vs = _kv4_rows(k, cache, batch, "k", here), _kv4_rows(v, cache, batch, "v", here)
    status = (_lib or lib()).comet_kv4_append(cache.address, batch.address, k.data_ptr(),
                                              v.data_ptr(), ks, vs, _stream(stream))
    if status:
        _check(status)


def kv4_gather(cache: KV4Cache, batch: KV4Batch, k_out=None, v_out=None, stream=None):
    """Reads the last rows of each sequence back: (k, v) float16 [M][kv_heads][head_dim].
    Rows in no sequence are left as they are (uninitialized in a new tensor)."""
    here = _kv4_here(cache, batch)
    shape = (batch.M, cache.kv_heads, cache.head_dim)
    if k_out is None:
        k_out = _new(shape, _torch.float16, cache.device, stream)
    if v_out is None:
        v_out = _new(shape, _torch.float16, cache.device, stream)
    ks = _kv4_rows(k_out, cache, batch, "k_out", here)
    vs = _kv4_rows(v_out, cache, batch, "v_out", here)
    status = (_lib or lib()).comet_kv4_gather(cache.address, batch.address, k_out.data_ptr(),
                                              v_out.data_ptr(), ks, vs, _stream(stream))
    if status:
        _check(status)
    return k_out, v_out


_cus = {}


def _num_cus(device) -> int:
    n = _cus.get(device.index)
    if n is None:
        import torch

        n = _cus[device.index] = torch.cuda.get_device_properties(device).multi_processor_count
    return n


def kv4_attention_workspace(q, cache: KV4Cache, batch: KV4Batch, stream=None):
    """A workspace tensor for kv4_attention calls of these sizes that do not overlap (an empty
    one where none is needed)."""
    import torch

    n = lib().comet_kv4_attention_workspace(cache.address, batch.address, q.shape[1],
                                            _num_cus(cache.device))
    return _new(n, torch.uint8, cache.device, stream)


def kv4_attention(q, cache: KV4Cache, batch: KV4Batch, scale: Optional[float] = None,
                  window: int = 0, out=None, workspace=None, stream=None):
    """Causal attention of the batch's rows q (float16 [M][heads][head_dim], rows may lie in
    a wider buffer) over the cache, which holds their own tokens already.  scale defaults to
    head_dim ** -0.5; workspace (of ``kv4_attention_workspace``) is allocated when not given.
    Returns out; rows in no sequence are left as they are (uninitialized in a new tensor)."""
    here = _kv4_here(cache, batch)
    M, H, D, qs = _heads_of(q, "q", here)
    if M != batch.M or D != cache.head_dim:
        raise ValueError(f"q: shape {tuple(q.shape)}, expected "
                         f"({batch.M}, heads, {cache.head_dim})")
    if out is None:
        out = _new((M, H, D), _torch.float16, q.device, stream)
        os_ = H * D
    else:
        oM, oH, oD, os_ = _heads_of(out, "out", here)
        if oM != M or oH != H or oD != D:
            raise ValueError(f"out: shape {tuple(out.shape)}, expected {(M, H, D)}")
    if workspace is None:
        workspace = kv4_attention_workspace(q, cache, batch, stream)
    else:
        _plain(workspace, "uint8", "workspace", here)
    status = (_lib or lib()).comet_kv4_attention(
        cache.address, batch.address, q.data_ptr(), out.data_ptr(), H, qs, os_,
        D ** -0.5 if scale is None else scale, min(window, _INT_MAX), workspace.data_ptr(), workspace.numel(),
        _stream(stream))
    if status:
        _check(status)
    return out


def _exact(t, numel: int, name: str) -> None:
    if t.numel() != numel:
        raise ValueError(f"{name}: {t.numel()} elements, expected {numel}")


def _gemm_operands(A_packed, a_scales, W_packed, w_scales, group_prec_map=None, M=None, N=None,
                   K=None):
    """Dtype, device and layout of the GEMM operands, and, given the shape,
    their exact sizes (the kernels read M, N and K from the arguments, not
    from the tensors)."""
    _tensor(A_packed, "uint8", "A_packed")
    _tensor(a_scales, "float16", "a_scales")
    _tensor(W_packed, "uint8", "W_packed")
    _tensor(w_scales, "float16", "w_scales")
    if M is None:
        return
    if M < 1 or N < 1 or K < G or K % G:
        raise ValueError(f"M={M}, N={N}, K={K}: need M, N >= 1 and K a positive multiple of {G}")
    m = _map(group_prec_map, K)
    nbytes = _act_bytes(m, M, G)
    if nbytes == 0:
        raise ValueError("group_prec_map: entries must be 4 or 8")
    _exact(A_packed, nbytes, "A_packed")
    _exact(a_scales, (K // G) * M, "a_scales")
    _exact(W_packed, N * K // 2, "W_packed")
    _exact(w_scales, (K // G) * N, "w_scales")


def w4ax_gemm(A_packed, group_prec_map, a_scales, W_packed, w_scales, M: int, N: int, K: int,
              out=None, stream=None):
    import torch

    _gemm_operands(A_packed, a_scales, W_packed, w_scales, group_prec_map, M, N, K)
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=A_packed.device)
    _tensor(out, "float16", "out")
    if tuple(out.shape) != (M, N):
        raise ValueError(f"out: shape {tuple(out.shape)}, expected {(M, N)}")
    comet_w4ax_gemm(A_packed, group_prec_map, a_scales, W_packed, w_scales, out, M, N, K, G,
                    stream)
    return out


def w4ax_gemm_swiglu_quant(A_packed, group_prec_map, a_scales, W_packed, w_scales, M: int, N: int,
                           K: int, out_prec_map, stream=None):
    """Fused gate/up GEMM + SwiGLU + quantization for the next layer.
    Returns (out_A_packed uint8, out_a_scales float16 [I/G][M]), I = N / 2."""
    import torch

    _gemm_operands(A_packed, a_scales, W_packed, w_scales, group_prec_map, M, N, K)
    I = N // 2
    nbytes = comet_act_packed_bytes(out_prec_map, M, I)
    if nbytes == 0:
        raise CometError(1, "invalid output map or shape")
    A2 = torch.empty(nbytes, dtype=torch.uint8, device=A_packed.device)
    sa2 = torch.empty((I // G, M), dtype=torch.float16, device=A_packed.device)
    comet_w4ax_gemm_swiglu_quant(A_packed, group_prec_map, a_scales, W_packed, w_scales, M, N, K,
                                 G, out_prec_map, A2, sa2, stream)
    return A2, sa2


def swiglu_quantize(gu, out_prec_map, stream=None):
    """gu: float16 [M][2I] CUDA tensor (256-wide gate/up groups) -> (A_packed, a_scales)."""
    import torch

    _tensor(gu, "float16", "gu")
    M, N = gu.shape
    I = N // 2
    nbytes = comet_act_packed_bytes(out_prec_map, M, I)
    if nbytes == 0:
        raise CometError(1, "invalid output map or shape")
    A2 = torch.empty(nbytes, dtype=torch.uint8, device=gu.device)
    sa2 = torch.empty((I // G, M), dtype=torch.float16, device=gu.device)
    comet_swiglu_quantize(gu, out_prec_map, A2, sa2, M, I, G, stream)
    return A2, sa2


def w4ax_gemm_acc(A_packed, group_prec_map, a_scales, W_packed, w_scales, M: int, N: int, K: int,
                  m0: int, m1: int, n0: int, n1: int, stream=None):
    import torch

    _gemm_operands(A_packed, a_scales, W_packed, w_scales, group_prec_map, M, N, K)
    if not (0 <= m0 < m1 <= M and 0 <= n0 < n1 <= N):
        raise ValueError(f"window [{m0},{m1})x[{n0},{n1}) is empty or outside {M}x{N}")
    acc = torch.empty((m1 - m0, n1 - n0, K // G), dtype=torch.int32, device=A_packed.device)
    comet_w4ax_gemm_acc(A_packed, group_prec_map, a_scales, W_packed, w_scales, acc, M, N, K, G,
                        m0, m1, n0, n1, stream)
    return acc
