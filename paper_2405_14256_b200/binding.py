"""ctypes binding of libzipcache.so: the same names as the C ABI, argument
marshalling only.  Every step of the path runs in the library's kernels."""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional, Sequence

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libzipcache.so")

ZC_F16, ZC_BF16 = 0, 1
ZC_FLAG_DEFER_APPEND = 1
ZC_FLAG_OVERLAP_CALLS = 2
ZC_FLAG_OUT_F32 = 4
ZC_FLAG_PARAMS_F16 = 8
ZC_FLAG_GROUP_ALL_HEADS = 16
ZC_K_CST, ZC_K_CHANNEL = 0, 1
ZC_PAGES_SYNC_BYTES = 1024
ZC_SCOPE_KV_HEAD, ZC_SCOPE_TOKEN = 0, 1


class ZipCacheError(RuntimeError):
    pass


class ZcConfig(C.Structure):
    _fields_ = [
        ("struct_size", C.c_int32), ("dtype", C.c_int32), ("batch", C.c_int32),
        ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("max_prefill", C.c_int32), ("max_new_tokens", C.c_int32), ("window", C.c_int32),
        ("bits_hi", C.c_int32), ("bits_lo", C.c_int32), ("flags", C.c_int32),
        ("saliency_ratio", C.c_double), ("k_scheme", C.c_int32), ("scope", C.c_int32),
    ]

    @classmethod
    def make(cls, dtype, batch, n_q_heads, n_kv_heads, max_prefill, max_new_tokens,
             saliency_ratio, bits_hi=4, bits_lo=2, window=100, head_dim=128,
             flags=0, k_scheme=0, scope=0) -> "ZcConfig":
        code = {torch.float16: ZC_F16, torch.bfloat16: ZC_BF16}.get(dtype, dtype)
        return cls(C.sizeof(cls), code, batch, n_q_heads, n_kv_heads, head_dim, max_prefill,
                   max_new_tokens, window, bits_hi, bits_lo, flags, float(saliency_ratio),
                   int(k_scheme), int(scope))


class ZcPageConfig(C.Structure):
    _fields_ = [
        ("struct_size", C.c_int32), ("dtype", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("page_size", C.c_int32), ("n_pages", C.c_int32), ("reserved", C.c_int32),
        ("strides", C.c_int64 * 3),
    ]

    @classmethod
    def make(cls, dtype, n_q_heads, n_kv_heads, page_size, n_pages, strides, head_dim=128) -> "ZcPageConfig":
        code = {torch.float16: ZC_F16, torch.bfloat16: ZC_BF16}.get(dtype, dtype)
        return cls(C.sizeof(cls), code, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, 0,
                   (C.c_int64 * 3)(*strides))


_lib = None

_SIGS = {
    "zc_cache_bytes": (C.c_int, [C.POINTER(ZcConfig), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "zc_cache_init": (C.c_int, [C.c_void_p, C.c_size_t, C.POINTER(ZcConfig), C.POINTER(C.c_void_p)]),
    "zc_cache_free": (None, [C.c_void_p]),
    "zc_probe_count": (C.c_int, [C.c_int, C.c_double, C.c_double]),
    "zc_default_probes": (C.c_int, [C.c_int, C.c_double, C.c_double, C.c_uint64,
                                    C.POINTER(C.c_int32), C.POINTER(C.c_int)]),
    "zc_prefill_compress": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                      C.POINTER(C.c_int64), C.POINTER(C.c_int64),
                                      C.POINTER(C.c_int32), C.c_int, C.c_void_p, C.c_void_p,
                                      C.c_size_t, C.c_void_p]),
    "zc_prefill_attention": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                       C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.c_void_p, C.c_void_p,
                                       C.c_void_p]),
    "zc_prefill_compress_lse": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                          C.POINTER(C.c_int64), C.POINTER(C.c_int64),
                                          C.POINTER(C.c_int32), C.c_int, C.c_void_p, C.c_void_p,
                                          C.c_size_t, C.c_void_p]),
    "zc_append": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "zc_decode_attention": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                                      C.c_size_t, C.c_void_p]),
    "zc_decode_attention_noalloc": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]),
    "zc_export_scores": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "zc_segment_tokens": (C.c_int, [C.c_void_p, C.c_int, C.c_int]),
    "zc_num_segments": (C.c_int, [C.c_void_p]),
    "zc_tail_tokens": (C.c_int, [C.c_void_p]),
    "zc_export_segment": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_void_p]),
    "zc_pages_workspace": (C.c_int, [C.POINTER(ZcPageConfig), C.c_int, C.c_int, C.POINTER(C.c_size_t)]),
    "zc_pages_init": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(ZcPageConfig), C.POINTER(C.c_void_p)]),
    "zc_pages_free": (None, [C.c_void_p]),
    "zc_pages_launch_count": (C.c_int64, [C.c_void_p]),
    "zc_page_tables": (C.c_int, [C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                                 C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p,
                                 C.c_void_p, C.c_void_p]),
    "zc_page_write": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(C.c_int64), C.c_void_p, C.c_int,
                                C.c_void_p]),
    "zc_page_read": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                               C.POINTER(C.c_int64), C.c_void_p]),
    "zc_paged_attention": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(C.c_int64), C.c_void_p, C.c_int,
                                     C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "zc_paged_attention_scored": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(C.c_int64), C.c_void_p, C.c_int,
                                            C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                            C.c_void_p, C.c_size_t, C.c_void_p]),
    "zc_scores_workspace": (C.c_int, [C.POINTER(ZcPageConfig), C.c_int, C.POINTER(C.c_size_t)]),
    "zc_paged_attention_shared": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(C.c_int64), C.c_void_p, C.c_int,
                                            C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                            C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                            C.c_void_p, C.c_size_t, C.c_void_p]),
    "zc_pages_shared_workspace": (C.c_int, [C.POINTER(ZcPageConfig), C.c_int, C.c_int, C.POINTER(C.c_size_t)]),
    "zc_page_select": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int,
                                 C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]),
    "zc_page_compact": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]),
    "zc_prefill_attention_window": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                              C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.c_int, C.c_int,
                                              C.c_void_p, C.c_void_p, C.c_void_p]),
    "zc_decode_bytes": (C.c_int64, [C.c_void_p]),
    "zc_launch_count": (C.c_int64, [C.c_void_p]),
    "zc_device_status": (C.c_int, [C.POINTER(C.c_int)]),
    "zc_order_model_reset": (None, []),
    "zc_order_model_call": (C.c_int, [C.c_uint64, C.c_int, C.POINTER(C.c_uint64), C.c_uint64, C.c_uint64,
                                      C.c_int, C.c_uint64, C.c_uint64, C.c_uint64, C.c_uint64,
                                      C.POINTER(C.c_int)]),
    "zc_strerror": (C.c_char_p, [C.c_int]),
}


def load_library(path: Optional[str] = None):
    """Load libzipcache.so and declare its signatures.  Fails loudly when the
    library has not been built: there is no fallback path."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise ZipCacheError(
            f"{p} is missing: build it with `python -m paper_2405_14256_b200.build` "
            "(there is no CPU or PyTorch fallback)")
    lib_ = C.CDLL(p)
    for name, (res, args) in _SIGS.items():
        fn = getattr(lib_, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib_
    return lib_


def lib():
    return load_library()


def _check(rc: int, what: str) -> int:
    if rc < 0:
        raise ZipCacheError(f"{what}: {zc_strerror(rc)} ({rc})")
    return rc


def _ptr(t) -> int:
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_I64x2, _I64x3 = C.c_int64 * 2, C.c_int64 * 3


@functools.lru_cache(maxsize=256)
def _strides2(a: int, b: int):
    """Two strides as the library takes them (it only reads them)."""
    return _I64x2(a, b)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(device_index: int, stream) -> int:
    """_stream for a device known to be current, without building a torch.cuda.Stream."""
    if stream is None and _raw_stream is not None:
        return _raw_stream(device_index)
    return _stream(stream)


def _stream_object(device_index: int, raw: int):
    """The torch.cuda.Stream of a raw handle."""
    return torch.cuda.ExternalStream(raw, device_index) if raw else torch.cuda.default_stream(device_index)


def _new(shape, dtype, device, stream):
    """A tensor that a kernel on `stream` writes and the current stream's work will read: it comes from that stream's
    memory, and is not given to another before the current stream's work so far is done when it is freed."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    device = _cuda_device(device)
    current = torch.cuda.current_stream(device)
    if _stream(stream) == current.cuda_stream:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(_stream_object(device.index, _stream(stream))):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(current)
    return t


class _Buffers:
    """Buffers that an object keeps for its calls, whatever stream a call runs on."""

    def _keep(self, *buffers, own: bool = True):
        """Called once they are made: whatever their memory was used for on the current stream, and their first
        fill, is over before a call on any stream can touch them.  (Made under capture, they belong to that graph.)
        own: their memory comes from the current stream; a given buffer's may come from any."""
        self._kept = buffers
        self._home = _stream_of(self._index, None) if own else None
        self._others = set()
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().synchronize()

    def _used_on(self, raw: int):
        """A call runs on a stream that is not the buffers' own: freed, they wait for its work so far."""
        if raw not in self._others:
            self._others.add(raw)
            for t in self._kept:
                t.record_stream(_stream_object(self._index, raw))


def zc_strerror(status: int) -> str:
    return lib().zc_strerror(status).decode()


def zc_cache_bytes(cfg: ZcConfig):
    cb, wb = C.c_size_t(0), C.c_size_t(0)
    _check(lib().zc_cache_bytes(C.byref(cfg), C.byref(cb), C.byref(wb)), "zc_cache_bytes")
    return cb.value, wb.value


def zc_cache_init(dev_mem, nbytes: int, cfg: ZcConfig) -> int:
    h = C.c_void_p(0)
    _check(lib().zc_cache_init(_ptr(dev_mem), nbytes, C.byref(cfg), C.byref(h)), "zc_cache_init")
    return h.value


def zc_cache_free(handle: int) -> None:
    lib().zc_cache_free(handle)


def zc_probe_count(l: int, rho_recent: float, rho_random: float) -> int:
    return _check(lib().zc_probe_count(l, rho_recent, rho_random), "zc_probe_count")


def zc_default_probes(l: int, rho_recent: float, rho_random: float, seed: int):
    n = zc_probe_count(l, rho_recent, rho_random)
    buf = (C.c_int32 * n)()
    n_out = C.c_int(0)
    _check(lib().zc_default_probes(l, rho_recent, rho_random, seed, buf, C.byref(n_out)),
           "zc_default_probes")
    return list(buf[: n_out.value])


def zc_prefill_compress(handle, Q, K, V, l: int, probe_pos: Optional[Sequence[int]],
                        salient_idx=None, workspace=None, stream=None) -> None:
    qs = (C.c_int64 * 3)(*(Q.stride()[:3] if Q is not None else (0, 0, 0)))
    ks = (C.c_int64 * 3)(*K.stride()[:3])
    if K.stride() != V.stride():
        raise ZipCacheError("K and V must share strides")
    n_probe = 0 if probe_pos is None else len(probe_pos)
    pp = (C.c_int32 * max(1, n_probe))(*(probe_pos if probe_pos is not None else [0]))
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().zc_prefill_compress(handle, _ptr(Q), _ptr(K), _ptr(V), l, qs, ks, pp, n_probe,
                                     _ptr(salient_idx), _ptr(workspace), ws_bytes,
                                     _stream(stream)), "zc_prefill_compress")


def zc_prefill_attention(handle, Q, K, V, l: int, O, row_lse, stream=None) -> None:
    qs = (C.c_int64 * 3)(*Q.stride()[:3])
    ks = (C.c_int64 * 3)(*K.stride()[:3])
    if K.stride() != V.stride():
        raise ZipCacheError("K and V must share strides")
    _check(lib().zc_prefill_attention(handle, _ptr(Q), _ptr(K), _ptr(V), l, qs, ks, _ptr(O), _ptr(row_lse),
                                      _stream(stream)), "zc_prefill_attention")


def zc_prefill_compress_lse(handle, Q, K, V, l: int, probe_pos: Sequence[int], row_lse, workspace,
                            stream=None) -> None:
    qs = (C.c_int64 * 3)(*Q.stride()[:3])
    ks = (C.c_int64 * 3)(*K.stride()[:3])
    if K.stride() != V.stride():
        raise ZipCacheError("K and V must share strides")
    pp = (C.c_int32 * max(1, len(probe_pos)))(*probe_pos)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().zc_prefill_compress_lse(handle, _ptr(Q), _ptr(K), _ptr(V), l, qs, ks, pp, len(probe_pos),
                                         _ptr(row_lse), _ptr(workspace), ws_bytes, _stream(stream)),
           "zc_prefill_compress_lse")


def zc_prefill_attention_window(handle, Q, K, V, l: int, window: int, sinks: int, O, row_lse, stream=None) -> None:
    qs = (C.c_int64 * 3)(*Q.stride()[:3])
    ks = (C.c_int64 * 3)(*K.stride()[:3])
    if K.stride() != V.stride():
        raise ZipCacheError("K and V must share strides")
    _check(lib().zc_prefill_attention_window(handle, _ptr(Q), _ptr(K), _ptr(V), l, qs, ks, window, sinks, _ptr(O),
                                             _ptr(row_lse), _stream(stream)), "zc_prefill_attention_window")


def zc_append(handle, k_new, v_new, stream=None) -> None:
    _check(lib().zc_append(handle, _ptr(k_new), _ptr(v_new), _stream(stream)), "zc_append")


def zc_decode_attention(handle, q, out, is_probe_step: bool, workspace, stream=None) -> None:
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().zc_decode_attention(handle, _ptr(q), _ptr(out), int(bool(is_probe_step)),
                                     _ptr(workspace), ws_bytes, _stream(stream)),
           "zc_decode_attention")


def zc_decode_attention_noalloc(handle, q, out, is_probe_step: bool, stream=None) -> None:
    """zc_decode_attention with the library's built-in scratch buffer instead of a caller
    workspace (for callers that cannot allocate device memory)."""
    _check(lib().zc_decode_attention_noalloc(handle, _ptr(q), _ptr(out), int(bool(is_probe_step)),
                                             _stream(stream)), "zc_decode_attention_noalloc")


def zc_export_scores(handle, p_tilde, stream=None) -> None:
    _check(lib().zc_export_scores(handle, _ptr(p_tilde), _stream(stream)), "zc_export_scores")


def zc_segment_tokens(handle, segment: int, subset: int) -> int:
    return _check(lib().zc_segment_tokens(handle, segment, subset), "zc_segment_tokens")


def zc_num_segments(handle) -> int:
    return _check(lib().zc_num_segments(handle), "zc_num_segments")


def zc_tail_tokens(handle) -> int:
    return _check(lib().zc_tail_tokens(handle), "zc_tail_tokens")


def zc_export_segment(handle, segment, tensor, subset, idx=None, codes=None, sz=None, cf=None,
                      stream=None) -> None:
    _check(lib().zc_export_segment(handle, segment, tensor, subset, _ptr(idx), _ptr(codes),
                                   _ptr(sz), _ptr(cf), _stream(stream)), "zc_export_segment")


def zc_decode_bytes(handle) -> int:
    return lib().zc_decode_bytes(handle)


def zc_launch_count(handle) -> int:
    return lib().zc_launch_count(handle)


def zc_device_status() -> int:
    code = C.c_int(0)
    _check(lib().zc_device_status(C.byref(code)), "zc_device_status")
    return code.value


# ---- full-precision pages ----
# The library's functions on tensors as they are; the classes below check theirs first and call the library themselves
# (a Python call of a microsecond less per step).
def zc_pages_workspace(cfg: ZcPageConfig, n_req: int, n_rows: int) -> int:
    nbytes = C.c_size_t(0)
    _check(lib().zc_pages_workspace(C.byref(cfg), n_req, n_rows, C.byref(nbytes)), "zc_pages_workspace")
    return nbytes.value


def zc_pages_init(k_pages, v_pages, cfg: ZcPageConfig) -> int:
    h = C.c_void_p(0)
    _check(lib().zc_pages_init(_ptr(k_pages), _ptr(v_pages), C.byref(cfg), C.byref(h)), "zc_pages_init")
    return h.value


def zc_pages_free(handle: int) -> None:
    lib().zc_pages_free(handle)


def zc_pages_launch_count(handle) -> int:
    return lib().zc_pages_launch_count(handle)


def zc_page_tables(page_size: int, past, fresh, free_pages, free_state, table, kv_len, row_start, slots, pos,
                   free_out, stream=None) -> None:
    _check(lib().zc_page_tables(page_size, past.numel(), _ptr(past), _ptr(fresh), _ptr(free_pages), free_pages.numel(),
                                _ptr(free_state), _ptr(table), table.shape[1], _ptr(kv_len), _ptr(row_start),
                                slots.numel(), _ptr(slots), _ptr(pos), _ptr(free_out), _stream(stream)),
           "zc_page_tables")


def zc_page_write(handle, k_rows, v_rows, slots, stream=None) -> None:
    if k_rows.stride() != v_rows.stride():
        raise ZipCacheError("k_rows and v_rows must share strides")
    rs = (C.c_int64 * 2)(*k_rows.stride()[:2])
    _check(lib().zc_page_write(handle, _ptr(k_rows), _ptr(v_rows), rs, _ptr(slots), k_rows.shape[0],
                               _stream(stream)), "zc_page_write")


def zc_page_read(handle, table, l: int, K, V, stream=None) -> None:
    if K.stride() != V.stride():
        raise ZipCacheError("K and V must share strides")
    ks = (C.c_int64 * 3)(*K.stride()[:3])
    _check(lib().zc_page_read(handle, _ptr(table), table.shape[1], table.shape[0], l, _ptr(K), _ptr(V), ks,
                              _stream(stream)), "zc_page_read")


def zc_paged_attention(handle, q, table, row_start, kv_len, max_rows: int, window: int, sinks: int, out, row_lse,
                       workspace, stream=None) -> None:
    qs = (C.c_int64 * 2)(*q.stride()[:2])
    _check(lib().zc_paged_attention(handle, _ptr(q), qs, _ptr(table), table.shape[1], _ptr(row_start), _ptr(kv_len),
                                    kv_len.numel(), q.shape[0], max_rows, window, sinks, _ptr(out), _ptr(row_lse),
                                    _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "zc_paged_attention")


def zc_scores_workspace(cfg: ZcPageConfig, max_rows: int) -> int:
    nbytes = C.c_size_t(0)
    _check(lib().zc_scores_workspace(C.byref(cfg), max_rows, C.byref(nbytes)), "zc_scores_workspace")
    return nbytes.value


def zc_pages_shared_workspace(cfg: ZcPageConfig, n_req: int, n_rows: int) -> int:
    nbytes = C.c_size_t(0)
    _check(lib().zc_pages_shared_workspace(C.byref(cfg), n_req, n_rows, C.byref(nbytes)), "zc_pages_shared_workspace")
    return nbytes.value


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def zc_paged_attention_scored(handle, q, table, row_start, kv_len, max_rows: int, window: int, sinks: int, first, scores,
                              out, row_lse, workspace, logits, stream=None) -> None:
    qs = (C.c_int64 * 2)(*q.stride()[:2])
    _check(lib().zc_paged_attention_scored(handle, _ptr(q), qs, _ptr(table), table.shape[1], _ptr(row_start),
                                           _ptr(kv_len), kv_len.numel(), q.shape[0], max_rows, window, sinks, _ptr(first),
                                           _ptr(scores), _ptr(out), _ptr(row_lse), _ptr(workspace), _nbytes(workspace),
                                           _ptr(logits), _nbytes(logits), _stream(stream)), "zc_paged_attention_scored")


def zc_paged_attention_shared(handle, q, table, row_start, kv_len, max_rows: int, group_start, shared_len, scores, out,
                              row_lse, workspace, logits, stream=None) -> None:
    qs = (C.c_int64 * 2)(*q.stride()[:2])
    _check(lib().zc_paged_attention_shared(handle, _ptr(q), qs, _ptr(table), table.shape[1], _ptr(row_start),
                                           _ptr(kv_len), kv_len.numel(), q.shape[0], max_rows, _ptr(group_start),
                                           _ptr(shared_len), shared_len.numel(), _ptr(scores), _ptr(out), _ptr(row_lse),
                                           _ptr(workspace), _nbytes(workspace), _ptr(logits), _nbytes(logits),
                                           _stream(stream)), "zc_paged_attention_shared")


def zc_page_select(handle, table, kv_len, scores, keep, recent: int, first, kept, kept_len, stream=None) -> None:
    _check(lib().zc_page_select(handle, _ptr(table), table.shape[1], _ptr(kv_len), kv_len.numel(), _ptr(scores), _ptr(keep),
                                recent, _ptr(first), _ptr(kept), kept.shape[2], _ptr(kept_len), _stream(stream)),
           "zc_page_select")


def zc_page_compact(handle, table, kv_len, kept, kept_len, scores=None, free_pages=None, free_state=None, free_out=None,
                    stream=None) -> None:
    _check(lib().zc_page_compact(handle, _ptr(table), table.shape[1], _ptr(kv_len), kv_len.numel(), _ptr(kept),
                                 kept.shape[2], _ptr(kept_len), _ptr(scores), _ptr(free_pages),
                                 0 if free_pages is None else free_pages.numel(), _ptr(free_state), _ptr(free_out),
                                 _stream(stream)), "zc_page_compact")


ORDER_FIELDS = ("epoch_start", "e", "need_start", "need_end", "slot", "tag", "record", "drain")


def zc_order_model_reset() -> None:
    lib().zc_order_model_reset()


def zc_order_model_call(stream_id, cache_id, q, k_new, v_new, out, io_bytes, kv_bytes, collect,
                        ws_addr, ws_bytes, need, capture_id=0) -> dict:
    """Books one call in the host-only model of the call ordering; addresses are integers."""
    addr = (C.c_uint64 * 4)(q, k_new, v_new, out)
    res = (C.c_int * 8)()
    _check(lib().zc_order_model_call(stream_id, cache_id, addr, io_bytes, kv_bytes, int(collect),
                                     ws_addr, ws_bytes, need, capture_id, res), "zc_order_model_call")
    return dict(zip(ORDER_FIELDS, list(res)))


def _want(t, name: str, shape, dtype, contiguous: bool = True) -> None:
    """Refuses a tensor whose type, shape or layout the library would misread."""
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or (contiguous and not t.is_contiguous()):
        raise ZipCacheError(f"{name}: expected {dtype} {tuple(shape)}{', contiguous' if contiguous else ''}, got "
                            f"{t.dtype} {tuple(t.shape)} with strides {t.stride()}")


def _want_i32(t, name: str, n: int, index: int) -> None:
    """Refuses anything but n contiguous int32 values on GPU `index`."""
    if t.dtype is not torch.int32 or t.numel() != n or not t.is_contiguous() or t.get_device() != index:
        raise ZipCacheError(f"{name}: expected {n} contiguous int32 values on cuda:{index}, got {t.dtype} "
                            f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _at_i32(t, name: str, n: int, index: int) -> int:
    """The address of n contiguous int32 values on GPU `index`; anything else is refused."""
    if t.dtype is not torch.int32 or t.numel() != n or t.get_device() != index or not t.is_contiguous():
        _want_i32(t, name, n, index)
    return t.data_ptr()


def _want_on(t, name: str, index: int) -> None:
    """Refuses a tensor that is not on GPU `index`."""
    if t.get_device() != index:
        raise ZipCacheError(f"{name}: expected a tensor on cuda:{index}, got one on {t.device}")


def _cuda_device(device) -> torch.device:
    if not torch.cuda.is_available():
        raise ZipCacheError("a CUDA device is required (no CPU fallback)")
    device = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device() if device.index is None else device.index)


class StepTables(_Buffers):
    """The buffers of one serving step's lengths and slots (zc_page_tables): kv_len [n_req],
    row_start [n_req + 1], slots and pos [n_rows], free_state [3], all int32, zero before the
    first build.  Made once (the constructor waits for the current stream's work) and reused from step to
    step; two steps whose free_state feeds the next one's take two of these in turn.  build may run on any
    stream; readers on another one are ordered behind it by the caller."""

    def __init__(self, n_req: int, n_rows: int, device="cuda:0"):
        self.device = _cuda_device(device)
        self.n_req, self.n_rows, self._index = n_req, n_rows, self.device.index
        new = lambda n: torch.zeros(n, dtype=torch.int32, device=self.device)  # noqa: E731
        with torch.cuda.device(self._index):
            self.kv_len, self.row_start, self.slots, self.pos = new(n_req), new(n_req + 1), new(n_rows), new(n_rows)
            self.free_state = new(3)
            self._keep(self.kv_len, self.row_start, self.slots, self.pos, self.free_state)

    def build(self, page_size: int, past, fresh, free_pages, free_state, table, stream=None) -> "StepTables":
        """past, fresh [n_req], free_pages [any], free_state [3] (next, end, -) and table [n_req, width]
        (extended in place), all int32 on this object's device."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.build(page_size, past, fresh, free_pages, free_state, table, stream)
        n = self.n_req
        _want_i32(past, "past", n, self._index)
        _want_i32(fresh, "fresh", n, self._index)
        _want_i32(free_pages, "free_pages", free_pages.numel(), self._index)
        _want_i32(free_state, "free_state", 3, self._index)
        width = table.shape[-1]
        _want_i32(table, "table", n * width, self._index)
        raw = _stream_of(self._index, stream)
        if raw != self._home:
            self._used_on(raw)
        _check(lib().zc_page_tables(page_size, n, past.data_ptr(), fresh.data_ptr(), free_pages.data_ptr(),
                                    free_pages.numel(), free_state.data_ptr(), table.data_ptr(), width,
                                    self.kv_len.data_ptr(), self.row_start.data_ptr(), self.n_rows,
                                    self.slots.data_ptr(), self.pos.data_ptr(), self.free_state.data_ptr(), raw),
               "zc_page_tables")
        return self


class PagedKV(_Buffers):
    """Keys and values at full precision in pages: a handle over the caller's tensors, both
    [n_pages, page_size, n_kv_heads, 128] with any strides of the first three dimensions (for pages
    stored [n_pages, n_kv_heads, page_size, 128] pass .transpose(1, 2)).  Holds the workspace of
    attention calls of up to max_req requests and max_rows rows: 43 MB whatever they are, so handles whose
    calls follow one another on a stream (the layers of a model) best share one: pass the first one's
    .workspace.  One made by the caller must have its first ZC_PAGES_SYNC_BYTES zeroed once.  With max_req or
    max_rows 0 and none given there is no workspace, and the handle is for all but attention: write, read, select, compact.  A handle's calls
    may run on any stream (the constructor waits for the current one's work), attention calls that share a workspace
    on one at a time.  Tensors that a call allocates may be used on the current stream, behind what orders it after
    `stream`.
    shared: the workspace serves attention_shared as well, for max_req requests and max_rows rows (11 MB more, and 1.1 KB
    for each of these rows and query heads, so max_rows is best no more than the generated tokens of a step).
    scored_rows: room for the logits of attention_scored and attention_shared calls of up to so many rows per request
    (4 bytes per slot, query head and row, in .logits, which handles over pages of one shape share as they share a
    workspace: pass the first one's); calls of more than 16 / G rows need none."""

    def __init__(self, k_pages, v_pages, n_q_heads: int, max_req: int = 256, max_rows: int = 8192,
                 workspace: Optional[torch.Tensor] = None, shared: bool = False, scored_rows: int = 0,
                 logits: Optional[torch.Tensor] = None):
        self.device = _cuda_device(k_pages.device)
        if k_pages.dim() != 4 or k_pages.stride(3) != 1 or k_pages.stride() != v_pages.stride():
            raise ZipCacheError("pages must be [n_pages, page_size, n_kv_heads, 128], the last dimension contiguous, "
                                "K and V with the same strides")
        _want(v_pages, "v_pages", k_pages.shape, k_pages.dtype, contiguous=False)
        _want_on(k_pages, "k_pages", self.device.index)
        _want_on(v_pages, "v_pages", self.device.index)
        if k_pages.dtype not in (torch.float16, torch.bfloat16):
            raise ZipCacheError("pages must be float16 or bfloat16")
        n_pages, page_size, n_kv, d = k_pages.shape
        self.cfg = ZcPageConfig.make(k_pages.dtype, n_q_heads, n_kv, page_size, n_pages, k_pages.stride()[:3], d)
        self.k_pages, self.v_pages = k_pages, v_pages
        self.dtype, self.page_size, self.n_q_heads, self.n_kv_heads = k_pages.dtype, page_size, n_q_heads, n_kv
        self._index = self.device.index
        self.workspace_bytes = (zc_pages_shared_workspace if shared else zc_pages_workspace)(self.cfg, max_req, max_rows)
        given = workspace is not None
        if not given and max_req > 0 and max_rows > 0:
            with torch.cuda.device(self._index):
                workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device)
                workspace[:ZC_PAGES_SYNC_BYTES].zero_()
        self._ws_bytes = 0
        if workspace is not None:
            _want_on(workspace, "workspace", self._index)
            if not workspace.is_contiguous():
                raise ZipCacheError("the workspace must be contiguous")
            self._ws_bytes = workspace.numel() * workspace.element_size()
            if self._ws_bytes < self.workspace_bytes:
                raise ZipCacheError("shared workspace too small")
        self.workspace, self._ws_at = workspace, 0 if workspace is None else workspace.data_ptr()
        self._lib = lib()
        self.scored_rows = int(scored_rows)
        need, given_logits = zc_scores_workspace(self.cfg, self.scored_rows), logits is not None
        if not given_logits and need > 0:
            with torch.cuda.device(self._index):
                logits = torch.empty(need, dtype=torch.uint8, device=self.device)
        if logits is not None:
            _want_on(logits, "logits", self._index)
            if not logits.is_contiguous() or _nbytes(logits) < need:
                raise ZipCacheError("shared logits too small, or not contiguous")
        self.logits = logits
        self._logits = (0, 0) if logits is None else (logits.data_ptr(), _nbytes(logits))
        self._score_shape, self._group = torch.Size((n_pages, n_kv, page_size)), n_q_heads // n_kv
        with torch.cuda.device(self._index):
            self._keep(*(t for t in (workspace, logits) if t is not None), own=not (given or given_logits))
            self.handle = zc_pages_init(k_pages, v_pages, self.cfg)

    def close(self):
        if getattr(self, "handle", None):
            zc_pages_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, t, name: str, n: int, heads: int) -> tuple:
        """The strides of t; refuses anything but [n, heads, 128] of the pages' type and device with contiguous channels."""
        strides = t.stride()
        if t.dtype is not self.dtype or t.shape != (n, heads, 128) or strides[2] != 1 or t.get_device() != self._index:
            raise ZipCacheError(f"{name}: expected {self.dtype} {(n, heads, 128)} with contiguous channels on "
                                f"{self.device}, got {t.dtype} {tuple(t.shape)} with strides {strides} on {t.device}")
        return strides

    def write(self, k_rows, v_rows, slots, stream=None):
        """Rows [n, n_kv_heads, 128] into slots [n] (int32; negative: skipped)."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.write(k_rows, v_rows, slots, stream)
        n = slots.numel()
        _want_i32(slots, "slots", n, self._index)
        strides = self._rows(k_rows, "k_rows", n, self.n_kv_heads)
        if strides != self._rows(v_rows, "v_rows", n, self.n_kv_heads):
            raise ZipCacheError("k_rows and v_rows must share strides")
        _check(self._lib.zc_page_write(self.handle, k_rows.data_ptr(), v_rows.data_ptr(), _strides2(strides[0], strides[1]),
                                       slots.data_ptr(), n, _stream_of(self._index, stream)), "zc_page_write")

    def read(self, table, l: int, K=None, V=None, stream=None):
        """The first l tokens of every request in table [n_req, width]: K, V [n_req, n_kv_heads, l, 128]."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.read(table, l, K, V, stream)
        _want(table, "table", (table.shape[0], table.shape[-1]), torch.int32)
        shape = (table.shape[0], self.n_kv_heads, l, 128)
        K = _new(shape, self.dtype, self.device, stream) if K is None else K
        V = _new(shape, self.dtype, self.device, stream) if V is None else V
        _want(K, "K", shape, self.dtype, contiguous=False)
        _want(V, "V", shape, self.dtype, contiguous=False)
        for t, name in ((table, "table"), (K, "K"), (V, "V")):
            _want_on(t, name, self._index)
        if K.stride(3) != 1:
            raise ZipCacheError("the channels of a row must be contiguous")
        zc_page_read(self.handle, table, l, K, V, stream)
        return K, V

    def attention(self, q, table, row_start, kv_len, max_rows: int, window: int = 0, sinks: int = 0, out=None,
                  row_lse=None, stream=None):
        """From q [n_rows, n_q_heads, 128], the newest tokens of the requests (rows row_start[r] ..
        row_start[r + 1] - 1 are the last of kv_len[r] tokens), to the cached keys and values: out like q
        (contiguous) and the rows' base-2 log-sum-exp [n_rows, n_q_heads].  max_rows bounds a request's
        rows; window > 0 keeps the last `window` tokens and the first `sinks` ones visible."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.attention(q, table, row_start, kv_len, max_rows, window, sinks, out, row_lse, stream)
        n_req, n, width, strides, out, row_lse, raw = self._call(q, table, row_start, kv_len, out, row_lse, stream)
        _check(self._lib.zc_paged_attention(self.handle, q.data_ptr(), strides, table.data_ptr(), width,
                                            row_start.data_ptr(), kv_len.data_ptr(), n_req, n, max_rows, window, sinks,
                                            out.data_ptr(), row_lse.data_ptr(), self._ws_at, self._ws_bytes,
                                            raw), "zc_paged_attention")
        return out, row_lse

    def _call(self, q, table, row_start, kv_len, out, row_lse, stream) -> tuple:
        """What attention calls share: their checks, outputs and stream."""
        if self.workspace is None:
            raise ZipCacheError("this handle has no workspace for attention (max_req or max_rows was 0)")
        n_req, n, heads = kv_len.numel(), q.shape[0], self.n_q_heads
        strides = self._rows(q, "q", n, heads)
        _want_i32(kv_len, "kv_len", n_req, self._index)
        _want_i32(row_start, "row_start", n_req + 1, self._index)
        width = table.shape[-1]
        _want_i32(table, "table", n_req * width, self._index)
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format) if stream is None else \
                _new(q.shape, q.dtype, self.device, stream)
        else:
            self._rows(out, "out", n, heads)
            if not out.is_contiguous():
                raise ZipCacheError("out must be contiguous")
        if row_lse is None:
            row_lse = _new((n, heads), torch.float32, self.device, stream)
        else:
            if row_lse.dtype is not torch.float32 or row_lse.numel() != n * heads or not row_lse.is_contiguous():
                _want(row_lse, "row_lse", (n, heads), torch.float32)
            _want_on(row_lse, "row_lse", self._index)
        raw = _stream_of(self._index, stream)
        if raw != self._home:
            self._used_on(raw)
        return n_req, n, width, _strides2(strides[0], strides[1]), out, row_lse, raw

    def _at_scores(self, scores) -> int:
        """The address of scores; anything but contiguous float32 [n_pages, n_kv_heads, page_size] is refused."""
        if scores.dtype is not torch.float32 or scores.shape != self._score_shape or not scores.is_contiguous() \
                or scores.get_device() != self._index:
            raise ZipCacheError(f"scores: expected contiguous float32 {tuple(self._score_shape)} on {self.device}, got "
                                f"{scores.dtype} {tuple(scores.shape)} with strides {scores.stride()} on {scores.device}")
        return scores.data_ptr()

    def _logits_for(self, max_rows: int) -> tuple:
        """The logits' scratch (address, bytes) of a call that scores."""
        if max_rows > self.scored_rows and max_rows * self._group <= 16:
            raise ZipCacheError(f"this handle has room for the logits of {self.scored_rows} rows per request (scored_rows)")
        return self._logits

    def attention_scored(self, q, table, row_start, kv_len, max_rows: int, scores, first=None, window: int = 0,
                         sinks: int = 0, out=None, row_lse=None, stream=None):
        """attention that also adds up the weight of every cached token, over the request's rows and the query heads of a KV
        head, in scores [n_pages, n_kv_heads, page_size] (float32, contiguous): the call's new tokens start from it, older
        ones add it to what they have; tokens before first[r] (int32 [n_req]; None: 0) have no score.  Tokens that requests of
        the call share belong there: a slot that two of them score ends with neither's sum."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.attention_scored(q, table, row_start, kv_len, max_rows, scores, first, window, sinks, out,
                                             row_lse, stream)
        at_scores = self._at_scores(scores)
        at_first = 0 if first is None else _at_i32(first, "first", kv_len.numel(), self._index)
        logits, size = self._logits_for(min(max_rows, q.shape[0]))
        n_req, n, width, strides, out, row_lse, raw = self._call(q, table, row_start, kv_len, out, row_lse, stream)
        _check(self._lib.zc_paged_attention_scored(self.handle, q.data_ptr(), strides, table.data_ptr(), width,
                                                   row_start.data_ptr(), kv_len.data_ptr(), n_req, n, max_rows, window, sinks,
                                                   at_first, at_scores, out.data_ptr(), row_lse.data_ptr(),
                                                   self._ws_at, self._ws_bytes, logits, size, raw),
               "zc_paged_attention_scored")
        return out, row_lse

    def attention_shared(self, q, table, row_start, kv_len, max_rows: int, group_start, shared_len, scores=None, out=None,
                         row_lse=None, stream=None):
        """attention of generated tokens (max_rows * G at most 16) for groups of consecutive requests that begin alike:
        group g, the requests group_start[g] .. group_start[g + 1] - 1, shares its first shared_len[g] tokens, whose keys
        and values are read once for all of them (int32 [n_groups + 1] and [n_groups]).  scores: as attention_scored's,
        with shared_len for `first`, which then says all that the tables share.  For handles made with shared=True."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.attention_shared(q, table, row_start, kv_len, max_rows, group_start, shared_len, scores, out,
                                             row_lse, stream)
        n_groups, index = shared_len.numel(), self._index
        at_shared = _at_i32(shared_len, "shared_len", n_groups, index)
        at_start = _at_i32(group_start, "group_start", n_groups + 1, index)
        logits = size = at_scores = 0
        if scores is not None:
            at_scores = self._at_scores(scores)
            logits, size = self._logits_for(min(max_rows, q.shape[0]))
        n_req, n, width, strides, out, row_lse, raw = self._call(q, table, row_start, kv_len, out, row_lse, stream)
        _check(self._lib.zc_paged_attention_shared(self.handle, q.data_ptr(), strides, table.data_ptr(), width,
                                                   row_start.data_ptr(), kv_len.data_ptr(), n_req, n, max_rows,
                                                   at_start, at_shared, n_groups, at_scores,
                                                   out.data_ptr(), row_lse.data_ptr(), self.workspace.data_ptr(),
                                                   self._ws_bytes, logits, size, raw), "zc_paged_attention_shared")
        return out, row_lse

    def select(self, table, kv_len, scores, keep, recent: int = 0, first=None, max_keep: Optional[int] = None, kept=None,
               kept_len=None, stream=None):
        """The tokens that each request keeps, per KV head: the first first[r] ones, the last `recent` ones, and by score as
        many between them as make keep[r] in all (int32 [n_req] each; equal scores: the lower position).  Returns
        kept [n_req, n_kv_heads, max_keep] (int32 positions, ascending, -1 behind them; max_keep is a given kept's, else
        it has to be said: no request that is thinned out keeps more) and kept_len [n_req], the requests' new lengths; what has no more than its keep stays as it is."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.select(table, kv_len, scores, keep, recent, first, max_keep, kept, kept_len, stream)
        n_req, width, index = kv_len.numel(), table.shape[-1], self._index
        if kept is None:
            if max_keep is None or max_keep < 0:
                raise ZipCacheError(f"max_keep: expected the lists' length where no kept is given, got {max_keep}")
            kept = _new((n_req, self.n_kv_heads, max_keep), torch.int32, self.device, stream)
        elif kept.dim() == 3:
            max_keep = kept.shape[2]
        if kept.dim() != 3 or kept.shape[1] != self.n_kv_heads:
            raise ZipCacheError(f"kept: expected [{n_req}, {self.n_kv_heads}, max_keep], got {tuple(kept.shape)}")
        if kept_len is None:
            kept_len = torch.empty_like(kv_len) if stream is None else _new((n_req,), torch.int32, self.device, stream)
        _check(self._lib.zc_page_select(self.handle, _at_i32(table, "table", n_req * width, index), width,
                                        _at_i32(kv_len, "kv_len", n_req, index), n_req, self._at_scores(scores),
                                        _at_i32(keep, "keep", n_req, index), recent,
                                        0 if first is None else _at_i32(first, "first", n_req, index),
                                        _at_i32(kept, "kept", n_req * self.n_kv_heads * max_keep, index), max_keep,
                                        _at_i32(kept_len, "kept_len", n_req, index), _stream_of(index, stream)), "zc_page_select")
        return kept, kept_len

    def compact(self, table, kv_len, kept, kept_len, scores=None, free_pages=None, free_state=None, free_out=None,
                stream=None):
        """Moves the rows (and scores) of the kept tokens to the front of each request's pages, in place; the requests go on
        with kept_len tokens.  The pages behind them go back in front of the free ones (free_pages, free_state as
        StepTables.build's; returns free_out [3], the new state) unless these are None."""
        if _current_device() != self._index:
            with torch.cuda.device(self._index):
                return self.compact(table, kv_len, kept, kept_len, scores, free_pages, free_state, free_out, stream)
        n_req, width, index = kv_len.numel(), table.shape[-1], self._index
        if kept.dim() != 3 or kept.shape[1] != self.n_kv_heads:
            raise ZipCacheError(f"kept: expected [{n_req}, {self.n_kv_heads}, max_keep], got {tuple(kept.shape)}")
        max_keep = kept.shape[2]
        at_free = n_free = at_state = at_out = 0
        if free_pages is not None:
            if free_state is None:
                raise ZipCacheError("free_pages come with free_state")
            if free_out is None:
                free_out = _new((3,), torch.int32, self.device, stream)
            n_free = free_pages.numel()
            at_free, at_state = _at_i32(free_pages, "free_pages", n_free, index), _at_i32(free_state, "free_state", 3, index)
            at_out = _at_i32(free_out, "free_out", 3, index)
        elif free_state is not None or free_out is not None:
            raise ZipCacheError("free_state and free_out come with free_pages")
        raw = _stream_of(index, stream)
        if n_req == 0 and at_out:        # (nothing for the library to do)
            with torch.cuda.stream(_stream_object(index, raw)):
                torch.clamp(free_state, max=n_free, out=free_out)
                free_out[:1].clamp_(min=0)
                free_out[2:].zero_()
        _check(self._lib.zc_page_compact(self.handle, _at_i32(table, "table", n_req * width, index), width,
                                         _at_i32(kv_len, "kv_len", n_req, index), n_req,
                                         _at_i32(kept, "kept", n_req * self.n_kv_heads * max_keep, index), max_keep,
                                         _at_i32(kept_len, "kept_len", n_req, index),
                                         0 if scores is None else self._at_scores(scores), at_free, n_free, at_state, at_out,
                                         raw), "zc_page_compact")
        return free_out


class ZipCache:
    """Owns the device buffers (allocated by PyTorch) of one attention layer's cache and
    forwards to the C ABI.  Marshalling and allocation only."""

    def __init__(self, dtype, batch, n_q_heads, n_kv_heads, max_prefill, max_new_tokens,
                 saliency_ratio, bits_hi=4, bits_lo=2, window=100, device="cuda:0",
                 workspace: Optional[torch.Tensor] = None, defer_append: bool = False,
                 overlap_calls: bool = False, out_f32: bool = False, k_channel: bool = False,
                 guard_bytes: int = 0, token_scope: bool = False, params_f16: bool = False,
                 group_all_heads: bool = False):
        if not torch.cuda.is_available():
            raise ZipCacheError("a CUDA device is required (no CPU fallback)")
        self.cfg = ZcConfig.make(dtype, batch, n_q_heads, n_kv_heads, max_prefill, max_new_tokens,
                                 saliency_ratio, bits_hi, bits_lo, window,
                                 flags=(ZC_FLAG_DEFER_APPEND if defer_append else 0) |
                                 (ZC_FLAG_OVERLAP_CALLS if overlap_calls else 0) |
                                 (ZC_FLAG_OUT_F32 if out_f32 else 0) |
                                 (ZC_FLAG_PARAMS_F16 if params_f16 else 0) |
                                 (ZC_FLAG_GROUP_ALL_HEADS if group_all_heads else 0),
                                 k_scheme=ZC_K_CHANNEL if k_channel else ZC_K_CST,
                                 scope=ZC_SCOPE_TOKEN if token_scope else ZC_SCOPE_KV_HEAD)
        self.k_channel = bool(k_channel)
        self.out_dtype = torch.float32 if out_f32 else dtype
        self.dtype, self.device = dtype, torch.device(device)
        self.batch, self.n_q_heads, self.n_kv_heads = batch, n_q_heads, n_kv_heads
        self.cache_bytes, self.workspace_bytes = zc_cache_bytes(self.cfg)
        # guard_bytes > 0 (a multiple of 256): the cache buffer and a workspace allocated here sit
        # between two bands filled with 0xA5, which check_guards() verifies (a debugging aid:
        # a kernel that writes outside its buffers shows up there)
        self.guard_bytes = int(guard_bytes)
        g = self.guard_bytes
        self._mem_all = torch.full((self.cache_bytes + 2 * g,), 0xA5, dtype=torch.uint8, device=self.device) \
            if g else torch.empty(self.cache_bytes, dtype=torch.uint8, device=self.device)
        self.mem = self._mem_all[g:g + self.cache_bytes]
        self._ws_all = None
        if workspace is None:
            self._ws_all = torch.full((self.workspace_bytes + 2 * g,), 0xA5, dtype=torch.uint8, device=self.device) \
                if g else torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device)
            workspace = self._ws_all[g:g + self.workspace_bytes]
        self.workspace = workspace
        if self.workspace.numel() * self.workspace.element_size() < self.workspace_bytes:
            raise ZipCacheError("shared workspace too small")
        self.handle = zc_cache_init(self.mem, self.cache_bytes, self.cfg)

    def check_guards(self) -> bool:
        """True when the guard bands around the cache buffer (and the workspace, if this object
        allocated it) still hold their fill pattern."""
        g = self.guard_bytes
        if not g:
            return True
        ok = True
        for buf in (self._mem_all, self._ws_all):
            if buf is not None:
                ok = ok and bool((buf[:g] == 0xA5).all()) and bool((buf[-g:] == 0xA5).all())
        return ok

    def close(self):
        if getattr(self, "handle", None):
            zc_cache_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def prefill_compress(self, Q, K, V, probe_pos=None, salient_idx=None, stream=None):
        zc_prefill_compress(self.handle, Q, K, V, K.shape[2], probe_pos, salient_idx,
                            self.workspace, stream)

    def prefill_attention(self, Q, K, V, stream=None):
        """Causal attention output O and the rows' log-sum-exp (Alg. 2's attention-output line)."""
        l = K.shape[2]
        O = _new((self.batch, self.n_q_heads, l, 128), self.dtype, self.device, stream)
        lse = _new((self.batch, self.n_q_heads, l), torch.float32, self.device, stream)
        zc_prefill_attention(self.handle, Q, K, V, l, O, lse, stream)
        return O, lse

    def prefill_attention_window(self, Q, K, V, window: int, sinks: int = 0, out=None, row_lse=None, stream=None):
        """prefill_attention under a sliding window: a row sees the last `window` tokens up to itself and
        the first `sinks` ones.  out and row_lse may be given (contiguous)."""
        l = K.shape[2]
        index = _cuda_device(self.device).index
        if _current_device() != index:
            with torch.cuda.device(index):
                return self.prefill_attention_window(Q, K, V, window, sinks, out, row_lse, stream)
        for t, name, heads in ((Q, "Q", self.n_q_heads), (K, "K", self.n_kv_heads), (V, "V", self.n_kv_heads)):
            _want(t, name, (self.batch, heads, l, 128), self.dtype, contiguous=False)
            _want_on(t, name, index)
            if t.stride(3) != 1:
                raise ZipCacheError(f"{name}: the channels of a row must be contiguous")
        if out is None:
            out = _new((self.batch, self.n_q_heads, l, 128), self.dtype, self.device, stream)
        if row_lse is None:
            row_lse = _new((self.batch, self.n_q_heads, l), torch.float32, self.device, stream)
        _want(out, "out", (self.batch, self.n_q_heads, l, 128), self.dtype)
        _want(row_lse, "row_lse", (self.batch, self.n_q_heads, l), torch.float32)
        _want_on(out, "out", index)
        _want_on(row_lse, "row_lse", index)
        zc_prefill_attention_window(self.handle, Q, K, V, l, window, sinks, out, row_lse, stream)
        return out, row_lse

    def prefill_compress_lse(self, Q, K, V, probe_pos, row_lse, stream=None):
        zc_prefill_compress_lse(self.handle, Q, K, V, K.shape[2], probe_pos, row_lse, self.workspace, stream)

    def append(self, k_new, v_new, stream=None):
        zc_append(self.handle, k_new, v_new, stream)

    def decode_attention(self, q, is_probe_step=False, out=None, stream=None):
        if out is None:
            out = _new(q.shape, self.out_dtype, q.device, stream)
        zc_decode_attention(self.handle, q, out, is_probe_step, self.workspace, stream)
        return out

    # ---- exports (canonical layouts) ----
    def scores(self, n: int):
        out = torch.empty((self.batch, self.n_kv_heads, n), dtype=torch.float32, device=self.device)
        zc_export_scores(self.handle, out)
        return out

    def segment(self, segment: int, tensor: int, subset: int):
        n = zc_segment_tokens(self.handle, segment, subset)
        bits = self.cfg.bits_hi if subset == 0 else self.cfg.bits_lo
        b, h = self.batch, self.n_kv_heads
        dev = self.device
        idx = torch.zeros((b, h, n), dtype=torch.int32, device=dev)
        codes = torch.zeros((b, h, n, 16 * bits), dtype=torch.uint8, device=dev)
        # channelwise keys: (scale, zero point) per channel instead of per token
        sz = torch.zeros((b, h, 128 if (self.k_channel and tensor == 0) else n, 2), dtype=torch.float32,
                         device=dev)
        cf = torch.zeros((b, h, 128), dtype=torch.float32, device=dev)
        if n > 0:
            zc_export_segment(self.handle, segment, tensor, subset, idx, codes, sz, cf)
        return idx, codes, sz, cf
