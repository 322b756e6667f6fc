"""ctypes binding of libbreadcrumbs.so: argument marshalling only.

Function names and argument order mirror include/breadcrumbs.h.  Tensors are
torch CUDA tensors used purely as device buffers; every step of the hot path
runs inside the library's kernels.  If the shared library is missing the import
of `lib()` raises: there is no CPU or PyTorch fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

from . import build as _build

# status codes and flags of breadcrumbs.h
BC_OK = 0
BC_ERR_INVALID_ARG, BC_ERR_BAD_SLOT, BC_ERR_NO_PAGES, BC_ERR_CAPACITY = -1, -2, -3, -4
BC_ERR_WINDOW_NOT_FULL, BC_ERR_WINDOW_FULL, BC_ERR_ORDER, BC_ERR_CUDA = -5, -6, -7, -8
BC_ERR_UNSUPPORTED, BC_ERR_TIMEOUT, BC_ERR_TOO_LARGE, BC_ERR_DEBUG_CHECK = -9, -10, -11, -12
BC_FLAG_OUT_F32, BC_FLAG_ATTN_REFERENCE, BC_FLAG_HOST_PIPELINED, BC_FLAG_DEBUG_BOUNDS = 1, 2, 4, 8
STATUS_NAMES = {0: "OK", -1: "INVALID_ARG", -2: "BAD_SLOT", -3: "NO_PAGES", -4: "CAPACITY",
                -5: "WINDOW_NOT_FULL", -6: "WINDOW_FULL", -7: "ORDER", -8: "CUDA",
                -9: "UNSUPPORTED", -10: "TIMEOUT", -11: "TOO_LARGE", -12: "DEBUG_CHECK"}


class BcConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("layers", "kv_heads", "q_heads", "head_dim", "c_default", "page_size", "max_seqs",
                 "num_pages", "max_pages_per_seq", "max_entries_per_seq")] + [("flags", C.c_uint32)]


class BcSeqState(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("open", "prompt_len", "n_beacons", "window_len", "c", "t",
                 "n_prompt_pages", "n_beacon_pages", "n_window_pages")]


class BreadcrumbsError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: BC_ERR_{STATUS_NAMES.get(status, status)}")


_LIB = None

# every symbol breadcrumbs.h declares: name -> (restype, argtypes)
_P, _I32, _I64, _F = C.c_void_p, C.c_int32, C.c_int64, C.c_float
SYMBOLS = {
    "bc_version": (_I32, []),
    "bc_cache_query_bytes": (_I32, [C.POINTER(BcConfig), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "bc_cache_create": (_I32, [C.POINTER(BcConfig), _P, _P, _P, _P, C.POINTER(_P)]),
    "bc_cache_destroy": (_I32, [_P]),
    "bc_seq_open": (_I32, [_P, _P, _P, _P, _I32, _P]),
    "bc_prefill": (_I32, [_P, _I32, _P, _P, _I32, _I32, _P, _P, _P]),
    "bc_restore": (_I32, [_P, _I32, _P, _I32, _P, _I32, _I32, _P, _P, _P, _P, _P]),
    "bc_append": (_I32, [_P, _I32, _P, _I32, _P, _P, _P]),
    "bc_decode_attn": (_I32, [_P, _I32, _P, _I32, _P, _P, _F, _P, _P, _P]),
    "bc_decode_step": (_I32, [_P, _I32, _P, _I32, _P, _P, _P, _P, _F, _P]),
    "bc_host_outputs_ready": (_I32, [_P, _P]),
    "bc_fill_step_host": (_I32, [_P, _I32, _P, _I32, _P, _P, _P, _P, _P, _P, _P, _P, _F, _P]),
    "bc_decode_attn_pair": (_I32, [_P, _I32, _P, _I32, _P, _P, _P, _P, _F, _P, _P, _P]),
    "bc_decode_attn_static": (_I32, [_P, _I32, _P, _I32, _P, _P, _F, _P, _P, _P]),
    "bc_mask_attn_query_bytes": (_I32, [_I32, _I32, _I32, _I32, _I64, _I64, _I64, C.POINTER(C.c_size_t)]),
    "bc_mask_attn_forward": (_I32, [_I32, _I32, _I32, _I32, _I32, C.POINTER(_I32), C.POINTER(_I32)] + [_P] * 10
                             + [_F, _P, C.c_size_t, _P]),
    "bc_mask_attn_status": (_I32, [_P, _I32, _I32, _I32, _I64, _I64, _I64, _P, C.POINTER(_I32)]),
    "bc_distill_loss": (_I32, [_I32, _P, _I64, _I32, _I32, _P, _P, _P, _P, _P, _P, _P]),
    "bc_compress": (_I32, [_P, _I32, _P, _I32, _P, _P, _P]),
    "bc_seq_close": (_I32, [_P, _P, _I32, _P]),
    "bc_decode_step_host": (_I32, [_P, _I32, _P, _I32, _P, _P, _P, _P, _F, _P]),
    "bc_compress_step_host": (_I32, [_P, _I32, _P, _I32, _P, _P, _P, _P, _F, _P]),
    "bc_get_state": (_I32, [_P, _I32, C.POINTER(BcSeqState), C.POINTER(_I32), _I32, _P]),
    "bc_get_free_list": (_I32, [_P, C.POINTER(_I32), C.POINTER(_I32), _P]),
    "bc_poll_error": (_I32, [_P, C.POINTER(_I32), C.POINTER(_I32), C.POINTER(_I64), _P]),
    "bc_clear_error": (_I32, [_P, _P]),
    "bc_export_seq": (_I32, [_P, _I32, _I32, _P, _P, _I32, _P]),
    "bc_set_attn_ctas": (_I32, [_P, _I32]),
    "bc_attn_timeline": (_I32, [_P, _P, _I32]),
    "bc_set_wait_limit": (_I32, [_P, C.c_uint32]),
    "bc_mask_attn_set_wait_limit": (_I32, [C.c_uint32]),
    "bc_profile_enable": (_I32, [_P, _I32]),
    "bc_profile_read": (_I32, [_P, C.POINTER(_I32), C.POINTER(_F)]),
    "bc_probe_read_stream": (_I32, [_P, C.c_size_t, _P]),
    "bc_fill_step": (_I32, [_P, _I32, _P, _I32, _P, _P, _P, _P, _P, _P, _P, _P, _F, _P]),
    "bc_add_rmsnorm": (_I32, [_P, _P, _P, _I32, _I32, _F, _P, _P, _P]),
    "bc_swiglu": (_I32, [_P, _I32, _I32, _P, _P]),
    "bc_argmax": (_I32, [_P, _I32, _I32, _P, _P]),
    "bc_rope_split": (_I32, [_P, _P, _P, _I32, _F, _P, _P, _P, _P]),
    "bc_rope_decode_step": (_I32, [_P, _I32, _P, _I32, _P, _P, _F, _P, _F, _P]),
    "bc_norm_rope_split": (_I32, [_I32, _I32, _I32, _I32, _P, _I64, _P, _F, _P, _P, _F, _P, _P, _P, _P]),
    "bc_norm_rope_query_bytes": (_I32, [_I32, C.POINTER(C.c_size_t)]),
    "bc_norm_rope_split_backward": (_I32, [_I32, _I32, _I32, _I32, _P, _I64, _P, _F, _P, _P, _F] + [_P] * 7 + [C.c_size_t, _P]),
    "bc_norm_rope_decode_step": (_I32, [_P, _I32, _P, _I32, _P, _P, _F, _P, _P, _F, _P, _F, _P]),
    "bc_chunk_attn": (_I32, [_P, _I32, _P, _P, _P, _I32, _I32, _P, _P, _F, _P]),
    "bc_prefill_chunk": (_I32, [_P, _I32, _P, _P, _P, _I32, _I32, _P, _P, _P, _P, _F, _P]),
    "bc_sample": (_I32, [_P, _I32, _I64, _I32, _I32, _P, _P, _P, _P, _P, _P, _P]),
    "bc_kernel_launches": (_I64, [_P]),
    "bc_last_cuda_error": (_I32, [_P]),
    "bc_status_string": (C.c_char_p, [_I32]),
}


def lib() -> C.CDLL:
    """Loads libbreadcrumbs.so (building it first if sources are newer).  Raises if unavailable."""
    global _LIB
    if _LIB is None:
        path = _build.LIB_PATH
        if not os.path.exists(path) or os.environ.get("BC_REBUILD"):
            path = _build.build_library()
        if not os.path.exists(path):
            raise RuntimeError("libbreadcrumbs.so is missing and could not be built; there is no fallback path")
        handle = C.CDLL(path)
        for name, (res, args) in SYMBOLS.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _LIB = handle
    return _LIB


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream) -> C.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _check(status, where):
    if status != BC_OK:
        raise BreadcrumbsError(status, where)


def _require(ok, where):
    if not ok:
        raise BreadcrumbsError(BC_ERR_INVALID_ARG, where)


def _on(where, ref, tensors, stream):
    """Checks that the tensors (tensor or None, dtype, shape) are contiguous, of that dtype and shape, and on the CUDA device of
    `ref`.  Returns that device's index, the raw stream, and the torch stream if one other than the device's current one was given
    (memory for the call's results is then taken from it).  Kept short: it is most of a small call's time."""
    dev = ref.get_device()
    if dev < 0:
        raise BreadcrumbsError(BC_ERR_INVALID_ARG, where)
    for t, dtype, shape in tensors:
        if t is not None and (t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous()):
            raise BreadcrumbsError(BC_ERR_INVALID_ARG, where)
    if stream is None:
        return dev, torch._C._cuda_getCurrentRawStream(dev), None
    return dev, stream.cuda_stream, _other(dev, stream)


def _call(where, dev, fn, *args):
    """A library call with the tensors' device current (a stream belongs to a device)."""
    if torch._C._cuda_getDevice() == dev:
        status = fn(*args)
    else:
        with torch.cuda.device(dev):
            status = fn(*args)
    if status != BC_OK:
        raise BreadcrumbsError(status, where)


def _at(t):
    return None if t is None else t.data_ptr()


def _other(dev, stream):
    """`stream` (anything that holds a stream's handle as cuda_stream) as a torch stream, if it is not the device's current one."""
    if stream is None or stream.cuda_stream == torch._C._cuda_getCurrentRawStream(dev):
        return None
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream, torch.device("cuda", dev))


def _new(like, shape, dtype, other):
    """Memory for results of a call on the stream `other` (None: the current one), on the device of `like`.  It is taken from that
    stream's memory, since a block that the current stream has freed may still be in use by work queued there; the caller may use it on
    the current stream."""
    if other is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(other):
        t = like.new_empty(shape, dtype=dtype)
    t.record_stream(torch.cuda.current_stream(like.device))
    return t


class Cache:
    """Owns the three device buffers (as torch tensors) and the library handle."""

    def __init__(self, layers, kv_heads, q_heads, head_dim, c_default, page_size, max_seqs, num_pages,
                 max_pages_per_seq, max_entries_per_seq=0, flags=0, device="cuda", stream=None):
        self.cfg = BcConfig(layers, kv_heads, q_heads, head_dim, c_default, page_size, max_seqs, num_pages,
                            max_pages_per_seq, max_entries_per_seq, flags)
        self.device = torch.device(device)
        sizes = [C.c_size_t() for _ in range(3)]
        _check(lib().bc_cache_query_bytes(C.byref(self.cfg), *[C.byref(s) for s in sizes]), "bc_cache_query_bytes")
        self.pool_bytes, self.meta_bytes, self.workspace_bytes = [s.value for s in sizes]
        index = torch.cuda.current_device() if self.device.index is None else self.device.index
        with torch.cuda.stream(_other(index, stream)):   # it initialises them: another stream's blocks may be in use by work queued there
            self.pool = torch.empty(self.pool_bytes, dtype=torch.uint8, device=self.device)
            self.meta = torch.empty(self.meta_bytes, dtype=torch.uint8, device=self.device)
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device)
        h = C.c_void_p()
        _check(lib().bc_cache_create(C.byref(self.cfg), _ptr(self.pool), _ptr(self.meta), _ptr(self.workspace),
                                     _stream(stream), C.byref(h)), "bc_cache_create")
        self.handle = h
        self.out_dtype = torch.float32 if flags & BC_FLAG_OUT_F32 else torch.bfloat16

    def close(self):
        if getattr(self, "handle", None) and lib is not None:   # at interpreter exit the module may be gone already
            lib().bc_cache_destroy(self.handle)
            self.handle = None

    __del__ = close

    # ---- the calls of breadcrumbs.h, same names -------------------------------------------------
    def bc_seq_open(self, slots, prompt_lens, c_per_seq=None, stream=None):
        _check(lib().bc_seq_open(self.handle, _ptr(slots), _ptr(prompt_lens), _ptr(c_per_seq), slots.numel(),
                                 _stream(stream)), "bc_seq_open")

    def bc_prefill(self, layer, slots, cu_prompt_lens, total_tokens, k, v, stream=None):
        _check(lib().bc_prefill(self.handle, layer, _ptr(slots), _ptr(cu_prompt_lens), slots.numel(), total_tokens,
                                _ptr(k), _ptr(v), _stream(stream)), "bc_prefill")

    def bc_restore(self, layer, slots, cu_tokens, total_tokens, total_beacons, tok_k, tok_v, beacon_k, beacon_v, stream=None):
        _check(lib().bc_restore(self.handle, layer, _ptr(slots), slots.numel(), _ptr(cu_tokens), total_tokens, total_beacons,
                                _ptr(tok_k), _ptr(tok_v), _ptr(beacon_k), _ptr(beacon_v), _stream(stream)), "bc_restore")

    def bc_append(self, layer, slots, k, v, stream=None):
        _check(lib().bc_append(self.handle, layer, _ptr(slots), slots.numel(), _ptr(k), _ptr(v), _stream(stream)),
               "bc_append")

    def bc_decode_attn(self, layer, slots, q, out, sm_scale, extra_k=None, extra_v=None, stream=None):
        _check(lib().bc_decode_attn(self.handle, layer, _ptr(slots), slots.numel(), _ptr(q), _ptr(out), sm_scale,
                                    _ptr(extra_k), _ptr(extra_v), _stream(stream)), "bc_decode_attn")

    def bc_host_outputs_ready(self, stream=None):
        _check(lib().bc_host_outputs_ready(self.handle, _stream(stream)), "bc_host_outputs_ready")

    def bc_fill_step_host(self, layer, slots, q, k, v, beacon_q, beacon_k, beacon_v, out, out_beacon, sm_scale, stream=None):
        _check(lib().bc_fill_step_host(self.handle, layer, _ptr(slots), slots.numel(), _ptr(q), _ptr(k), _ptr(v), _ptr(beacon_q),
                                       _ptr(beacon_k), _ptr(beacon_v), _ptr(out), _ptr(out_beacon), sm_scale, _stream(stream)),
               "bc_fill_step_host")

    def bc_decode_attn_pair(self, layer, slots, q, out, beacon_q, out_beacon, sm_scale, beacon_k, beacon_v, stream=None):
        _check(lib().bc_decode_attn_pair(self.handle, layer, _ptr(slots), slots.numel(), _ptr(q), _ptr(out), _ptr(beacon_q),
                                         _ptr(out_beacon), sm_scale, _ptr(beacon_k), _ptr(beacon_v), _stream(stream)),
               "bc_decode_attn_pair")

    def bc_decode_step(self, layer, slots, q, k, v, out, sm_scale, stream=None):
        """bc_append(k, v) + bc_decode_attn(q) in one launch."""
        _check(lib().bc_decode_step(self.handle, layer, _ptr(slots), slots.numel(), _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                    sm_scale, _stream(stream)), "bc_decode_step")

    def bc_fill_step(self, layer, slots, q, k, v, beacon_q, beacon_k, beacon_v, out, out_beacon, sm_scale, stream=None):
        """The step that fills a window: bc_append + bc_decode_attn_pair + bc_compress, the append inside the attention launch."""
        _check(lib().bc_fill_step(self.handle, layer, _ptr(slots), slots.numel(), _ptr(q), _ptr(k), _ptr(v), _ptr(beacon_q),
                                  _ptr(beacon_k), _ptr(beacon_v), _ptr(out), _ptr(out_beacon), sm_scale, _stream(stream)),
               "bc_fill_step")

    def bc_rope_split(self, qkv, positions, theta, q_out, k_out, v_out, stream=None):
        """Rotary embedding of the q and k heads of a packed QKV projection, split into the three arrays the cache calls take."""
        _check(lib().bc_rope_split(self.handle, _ptr(qkv), _ptr(positions), positions.numel(), theta, _ptr(q_out), _ptr(k_out),
                                   _ptr(v_out), _stream(stream)), "bc_rope_split")

    def bc_rope_decode_step(self, layer, slots, qkv, positions, theta, out, sm_scale, stream=None):
        """bc_rope_split + bc_decode_step: a layer's decode step straight from the packed QKV projection."""
        _check(lib().bc_rope_decode_step(self.handle, layer, _ptr(slots), slots.numel(), _ptr(qkv), _ptr(positions), theta,
                                         _ptr(out), sm_scale, _stream(stream)), "bc_rope_decode_step")

    def bc_norm_rope_decode_step(self, layer, slots, qkv, positions, theta, q_weight, k_weight, eps, out, sm_scale, stream=None):
        """bc_norm_rope_split + bc_decode_step: a layer's decode step straight from the packed QKV projection."""
        where, n, cfg = "bc_norm_rope_decode_step", slots.numel(), self.cfg
        d = cfg.head_dim
        dev, s, _ = _on(where, self.pool, (
            (slots, torch.int32, (n,)), (positions, torch.int32, (n,)), (qkv, torch.bfloat16, (n, (cfg.q_heads + 2 * cfg.kv_heads) * d)),
            (q_weight, torch.bfloat16, (d,)), (k_weight, torch.bfloat16, (d,)), (out, self.out_dtype, (n, cfg.q_heads, d))), stream)
        _call(where, dev, lib().bc_norm_rope_decode_step, self.handle, layer, _at(slots), n, _at(qkv), _at(positions), theta, _at(q_weight),
              _at(k_weight), eps, _at(out), sm_scale, s)

    def bc_chunk_attn(self, layer, slots, cu_q, total_q, q, out, sm_scale, first=None, stream=None):
        """Attention of a ragged chunk of queries per sequence (breadcrumbs.h); first None: the sequences' last entries."""
        where, n = "bc_chunk_attn", slots.numel()
        shape = (total_q, self.cfg.q_heads, self.cfg.head_dim)
        dev, s, _ = _on(where, self.pool, (
            (slots, torch.int32, (n,)), (cu_q, torch.int32, (n + 1,)), (first, torch.int32, (n,)), (q, torch.bfloat16, shape),
            (out, self.out_dtype, shape)), stream)
        _call(where, dev, lib().bc_chunk_attn, self.handle, layer, _at(slots), _at(first), _at(cu_q), n, total_q, _at(q), _at(out), sm_scale, s)

    def bc_prefill_chunk(self, layer, slots, first, cu_chunk, total, q, k, v, out, sm_scale, stream=None):
        """Stores a chunk of every prompt at positions first[i] ... and attends with its queries (breadcrumbs.h)."""
        where, n, cfg = "bc_prefill_chunk", slots.numel(), self.cfg
        shape, kv = (total, cfg.q_heads, cfg.head_dim), (total, cfg.kv_heads, cfg.head_dim)
        dev, s, _ = _on(where, self.pool, (
            (slots, torch.int32, (n,)), (cu_chunk, torch.int32, (n + 1,)), (first, torch.int32, (n,)), (q, torch.bfloat16, shape),
            (k, torch.bfloat16, kv), (v, torch.bfloat16, kv), (out, self.out_dtype, shape)), stream)
        _call(where, dev, lib().bc_prefill_chunk, self.handle, layer, _at(slots), _at(first), _at(cu_chunk), n, total, _at(q), _at(k), _at(v),
              _at(out), sm_scale, s)

    def bc_decode_attn_static(self, layer, slots, q, out, sm_scale, extra_k=None, extra_v=None, stream=None):
        """bc_decode_attn with the split-K scratch taken from the array built into the library, for callers
        that may not allocate device memory.  At most 128 sequences per call; calls share the scratch."""
        _check(lib().bc_decode_attn_static(self.handle, layer, _ptr(slots), slots.numel(), _ptr(q), _ptr(out),
                                           sm_scale, _ptr(extra_k), _ptr(extra_v), _stream(stream)),
               "bc_decode_attn_static")

    def bc_compress(self, layer, slots, beacon_k, beacon_v, stream=None):
        _check(lib().bc_compress(self.handle, layer, _ptr(slots), slots.numel(), _ptr(beacon_k), _ptr(beacon_v),
                                 _stream(stream)), "bc_compress")

    def bc_seq_close(self, slots, stream=None):
        _check(lib().bc_seq_close(self.handle, _ptr(slots), slots.numel(), _stream(stream)), "bc_seq_close")

    def bc_decode_step_host(self, layer, slots, q_host, k_host, v_host, out_host, sm_scale, stream=None):
        _check(lib().bc_decode_step_host(self.handle, layer, _ptr(slots), slots.numel(), _ptr(q_host), _ptr(k_host),
                                         _ptr(v_host), _ptr(out_host), sm_scale, _stream(stream)),
               "bc_decode_step_host")

    def bc_compress_step_host(self, layer, slots, bq_host, bk_host, bv_host, out_host, sm_scale, stream=None):
        _check(lib().bc_compress_step_host(self.handle, layer, _ptr(slots), slots.numel(), _ptr(bq_host),
                                           _ptr(bk_host), _ptr(bv_host), _ptr(out_host), sm_scale, _stream(stream)),
               "bc_compress_step_host")

    def bc_get_state(self, slot, stream=None):
        st = BcSeqState()
        cap = self.cfg.max_pages_per_seq
        pages = (C.c_int32 * cap)()
        _check(lib().bc_get_state(self.handle, slot, C.byref(st), pages, cap, _stream(stream)), "bc_get_state")
        if not st.open:
            return None
        p = list(pages)
        a, b, w = st.n_prompt_pages, st.n_beacon_pages, st.n_window_pages
        return dict(prompt_len=st.prompt_len, n_beacons=st.n_beacons, window_len=st.window_len, c=st.c, t=st.t,
                    prompt_pages=p[:a], beacon_pages=p[a:a + b], window_pages=p[a + b:a + b + w])

    def bc_get_free_list(self, stream=None):
        pages = (C.c_int32 * self.cfg.num_pages)()
        count = C.c_int32()
        _check(lib().bc_get_free_list(self.handle, pages, C.byref(count), _stream(stream)), "bc_get_free_list")
        return list(pages[:count.value])

    def bc_poll_error(self, stream=None):
        code, slot, call = C.c_int32(), C.c_int32(), C.c_int64()
        _check(lib().bc_poll_error(self.handle, C.byref(code), C.byref(slot), C.byref(call), _stream(stream)),
               "bc_poll_error")
        return code.value, slot.value, call.value

    def bc_clear_error(self, stream=None):
        _check(lib().bc_clear_error(self.handle, _stream(stream)), "bc_clear_error")

    def bc_export_seq(self, layer, slot, capacity, stream=None):
        shape = (capacity, self.cfg.kv_heads, self.cfg.head_dim)
        other = _other(self.pool.get_device(), stream)
        k, v = [_new(self.pool, shape, torch.bfloat16, other) for _ in range(2)]
        with torch.cuda.stream(other):
            k.zero_(), v.zero_()
        _check(lib().bc_export_seq(self.handle, layer, slot, _ptr(k), _ptr(v), capacity, _stream(stream)),
               "bc_export_seq")
        return k, v

    def bc_set_attn_ctas(self, ctas):
        _check(lib().bc_set_attn_ctas(self.handle, ctas), "bc_set_attn_ctas")

    def bc_set_wait_limit(self, polls):
        _check(lib().bc_set_wait_limit(self.handle, polls), "bc_set_wait_limit")

    def bc_attn_timeline(self, words, blocks=0):
        """words: uint64/int64 CUDA tensor of at least blocks * 16 elements, or None to switch it off."""
        _check(lib().bc_attn_timeline(self.handle, _ptr(words), blocks), "bc_attn_timeline")

    def bc_profile_enable(self, max_launches):
        _check(lib().bc_profile_enable(self.handle, max_launches), "bc_profile_enable")

    def bc_profile_read(self):
        n, ms = C.c_int32(), C.c_float()
        _check(lib().bc_profile_read(self.handle, C.byref(n), C.byref(ms)), "bc_profile_read")
        return n.value, ms.value

    def bc_kernel_launches(self):
        return lib().bc_kernel_launches(self.handle)

    # ---- convenience ------------------------------------------------------------------------------
    def new_out(self, n):
        return torch.empty((n, self.cfg.q_heads, self.cfg.head_dim), dtype=self.out_dtype, device=self.device)


def bc_mask_attn_forward(prompt_lens, token_lens, c, prompt_k, prompt_v, tok_q, tok_k, tok_v, beacon_q, beacon_k,
                         beacon_v, sm_scale, stream=None, check=True):
    """The mask form of a batch of trajectories (breadcrumbs.h): returns (out_tok, out_beacon).

    prompt_lens, token_lens: Python lists, one entry per sequence.  Tensors are packed bf16 CUDA
    tensors as the header describes; beacon tensors may be None when no sequence has a beacon."""
    n = len(prompt_lens)
    q_heads, kv_heads, head_dim = tok_q.shape[1], tok_k.shape[1], tok_q.shape[2]
    cu_p = (C.c_int32 * (n + 1))(0, *list(__import__("itertools").accumulate(prompt_lens)))
    cu_t = (C.c_int32 * (n + 1))(0, *list(__import__("itertools").accumulate(token_lens)))
    total_b = sum(t // c for t in token_lens) if c > 1 else 0
    size = C.c_size_t()
    _check(lib().bc_mask_attn_query_bytes(n, q_heads, kv_heads, head_dim, cu_p[n], cu_t[n], total_b, C.byref(size)),
           "bc_mask_attn_query_bytes")
    other = _other(tok_q.get_device(), stream)
    ws = _new(tok_q, size.value, torch.uint8, other)
    out_tok = _new(tok_q, tok_q.shape, tok_q.dtype, other)
    out_bea = _new(tok_q, (total_b, q_heads, head_dim), tok_q.dtype, other)
    _check(lib().bc_mask_attn_forward(n, q_heads, kv_heads, head_dim, c, cu_p, cu_t, _ptr(prompt_k), _ptr(prompt_v),
                                      _ptr(tok_q), _ptr(tok_k), _ptr(tok_v), _ptr(beacon_q), _ptr(beacon_k),
                                      _ptr(beacon_v), _ptr(out_tok), _ptr(out_bea), sm_scale, _ptr(ws), size.value,
                                      _stream(stream)), "bc_mask_attn_forward")
    if check:
        code = C.c_int32()
        _check(lib().bc_mask_attn_status(_ptr(ws), n, q_heads, kv_heads, cu_p[n], cu_t[n], total_b, _stream(stream),
                                         C.byref(code)), "bc_mask_attn_status")
        _check(code.value, "bc_mask_attn_forward (device)")
    return out_tok, out_bea


def bc_probe_read_stream(buf, stream=None):
    """Reads the CUDA tensor `buf` once with the attention kernel's copy pattern (breadcrumbs.h)."""
    _check(lib().bc_probe_read_stream(_ptr(buf), buf.numel() * buf.element_size(), _stream(stream)), "bc_probe_read_stream")


def bc_add_rmsnorm(h, delta, weight, eps, h_out, normed_out, stream=None):
    """h' = h + delta (bf16), normed_out = rmsnorm(h') * weight (breadcrumbs.h); delta, weight, h_out may be None."""
    n, hidden = h.shape[0], h.shape[-1]
    _check(lib().bc_add_rmsnorm(_ptr(h), _ptr(delta), _ptr(weight), n, hidden, eps, _ptr(h_out), _ptr(normed_out), _stream(stream)),
           "bc_add_rmsnorm")


def bc_swiglu(gate_up, out, stream=None):
    """out = silu(gate) * up for packed rows [gate | up] (breadcrumbs.h)."""
    _check(lib().bc_swiglu(_ptr(gate_up), gate_up.shape[0], gate_up.shape[-1] // 2, _ptr(out), _stream(stream)), "bc_swiglu")


def bc_argmax(logits, out, stream=None):
    """out[r] (int64) = lowest index of the maximum of row r of bf16 logits (breadcrumbs.h)."""
    _check(lib().bc_argmax(_ptr(logits), logits.shape[0], logits.shape[-1], _ptr(out), _stream(stream)), "bc_argmax")


def bc_distill_loss(cu_rows, student_logits, teacher_idx, teacher_logprob, with_grad=False, stream=None):
    """Eq. 1 (breadcrumbs.h): returns (loss [1] fp32, row_loss [rows] fp32, grad or None).

    cu_rows: int32 CUDA tensor [n_traj + 1]; student_logits bf16 [rows, vocab]; teacher_idx int32 and
    teacher_logprob fp32 [rows, top_k]."""
    rows, vocab = student_logits.shape
    top_k = teacher_idx.shape[1]
    other = _other(student_logits.get_device(), stream)
    row_loss = _new(student_logits, rows, torch.float32, other)
    loss = _new(student_logits, 1, torch.float32, other)
    grad = _new(student_logits, student_logits.shape, student_logits.dtype, other) if with_grad else None
    _check(lib().bc_distill_loss(cu_rows.numel() - 1, _ptr(cu_rows), rows, vocab, top_k, _ptr(student_logits),
                                 _ptr(teacher_idx), _ptr(teacher_logprob), _ptr(row_loss), _ptr(loss), _ptr(grad),
                                 _stream(stream)), "bc_distill_loss")
    return loss, row_loss, grad


def _norm_rope_shapes(qkv, q_heads, kv_heads, where):
    heads = q_heads + 2 * kv_heads
    if qkv.dim() != 2 or qkv.dtype is not torch.bfloat16 or q_heads < 1 or kv_heads < 1 or qkv.shape[1] % heads or qkv.stride(1) != 1:
        raise BreadcrumbsError(BC_ERR_INVALID_ARG, where)
    n, width = qkv.shape
    d = width // heads
    return n, d, qkv.stride(0) if n > 1 else max(qkv.stride(0), width), (n, q_heads, d), (n, kv_heads, d)


def bc_norm_rope_split(qkv, positions, theta, q_weight, k_weight, eps, q_heads, kv_heads, q_out=None, k_out=None, v_out=None, stream=None):
    """Norms of the q and k heads of packed QKV rows, their rotation, and the split (breadcrumbs.h): returns (q, k, v).

    qkv: [n, (q_heads + 2 kv_heads) * head_dim] bf16, rows may be strided; q_weight, k_weight: [head_dim] bf16 or None; q_out,
    k_out, v_out are allocated when not given."""
    where, bf16 = "bc_norm_rope_split", torch.bfloat16
    n, d, row_stride, qs, ks = _norm_rope_shapes(qkv, q_heads, kv_heads, where)
    dev, s, other = _on(where, qkv, ((positions, torch.int32, (n,)), (q_weight, bf16, (d,)), (k_weight, bf16, (d,)), (q_out, bf16, qs),
                                     (k_out, bf16, ks), (v_out, bf16, ks)), stream)
    q = _new(qkv, qs, bf16, other) if q_out is None else q_out
    k = _new(qkv, ks, bf16, other) if k_out is None else k_out
    v = _new(qkv, ks, bf16, other) if v_out is None else v_out
    _call(where, dev, lib().bc_norm_rope_split, n, q_heads, kv_heads, d, qkv.data_ptr(), row_stride, positions.data_ptr(), theta, _at(q_weight),
          _at(k_weight), eps, q.data_ptr(), k.data_ptr(), v.data_ptr(), s)
    return q, k, v


def bc_norm_rope_split_backward(qkv, positions, theta, q_weight, k_weight, eps, dq, dk, dv, weight_grads=True, stream=None):
    """Gradient of bc_norm_rope_split (breadcrumbs.h): returns (dqkv [n, ...] bf16, dq_weight, dk_weight [head_dim] fp32 or None)."""
    where, bf16 = "bc_norm_rope_split_backward", torch.bfloat16
    _require(dq.dim() == 3 and dk.dim() == 3, where)
    q_heads, kv_heads = dq.shape[1], dk.shape[1]
    n, d, row_stride, qs, ks = _norm_rope_shapes(qkv, q_heads, kv_heads, where)
    dev, s, other = _on(where, qkv, ((positions, torch.int32, (n,)), (q_weight, bf16, (d,)), (k_weight, bf16, (d,)), (dq, bf16, qs), (dk, bf16, ks),
                                     (dv, bf16, ks)), stream)
    size = C.c_size_t()
    _check(lib().bc_norm_rope_query_bytes(d, C.byref(size)), "bc_norm_rope_query_bytes")
    dqkv = _new(qkv, (n, qkv.shape[1]), bf16, other)
    # the weights' gradients and the scratch in one allocation
    ws = _new(qkv, size.value // 4 + 2 * d, torch.float32, other)
    at = ws.data_ptr()
    _call(where, dev, lib().bc_norm_rope_split_backward, n, q_heads, kv_heads, d, qkv.data_ptr(), row_stride, positions.data_ptr(), theta,
          _at(q_weight), _at(k_weight), eps, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dqkv.data_ptr(), at if weight_grads else None,
          at + 4 * d if weight_grads else None, at + 8 * d, size.value, s)
    return (dqkv, ws[:d], ws[d:2 * d]) if weight_grads else (dqkv, None, None)


def bc_sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, out=None, stream=None):
    """One token per row of bf16 or fp32 logits [n, vocab] (rows may be strided) from one uniform number per row, with the
    row's temperature, top-k, top-p and min-p (breadcrumbs.h): returns int64 [n]."""
    where, f32 = "bc_sample", torch.float32
    if logits.dim() != 2 or (logits.dtype is not torch.bfloat16 and logits.dtype is not f32):
        raise BreadcrumbsError(BC_ERR_INVALID_ARG, where)
    n, vocab = logits.shape
    row_stride = logits.stride(0)
    _require(vocab == 1 or logits.stride(1) == 1, where)
    dev, s, other = _on(where, logits, ((uniform, f32, (n,)), (temperature, f32, (n,)), (top_k, torch.int32, (n,)), (top_p, f32, (n,)),
                                        (min_p, f32, (n,)), (out, torch.int64, (n,))), stream)
    res = _new(logits, n, torch.int64, other) if out is None else out
    _call(where, dev, lib().bc_sample, logits.data_ptr(), 1 if logits.dtype is f32 else 0, row_stride if n > 1 else max(row_stride, vocab), n, vocab,
          _at(temperature), _at(top_k), _at(top_p), _at(min_p), uniform.data_ptr(), res.data_ptr(), s)
    return res
