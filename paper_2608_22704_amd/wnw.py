"""Python binding of the WnW decode-step library (libwnw.so), argument marshalling only.

Function names match the C ABI of include/wnw.h.  Every computation runs in the HIP library;
this module only converts arguments (torch tensors -> device pointers, torch streams -> HIP
streams) and turns error codes into exceptions.  It raises at import time when the library has
not been built: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libwnw.so")

WNW_OK, WNW_ERR_INVALID, WNW_ERR_OOM, WNW_ERR_HIP, WNW_ERR_STATE, WNW_ERR_UNSUPPORTED = 0, -1, -2, -3, -4, -5
WNW_ANCHOR, WNW_TIDAL, WNW_FIXED = 0, 1, 2
WNW_F_SELECT_NEXT_STEP, WNW_F_RECALL_MEMCPY, WNW_F_TIMING, WNW_F_OVERLAP_CHUNKS, WNW_F_PREFILL_GLOBAL = 1, 2, 4, 8, 16
WNW_F_OUT_BF16 = 32
WNW_QUANT_INT8, WNW_QUANT_E4M3 = 0, 1
WNW_ROTARY_HALVES, WNW_ROTARY_PAIRS = 0, 1

EXPORTS = ("wnw_init_cache", "wnw_set_retention", "wnw_set_roles", "wnw_prefill_scores", "wnw_prefill_scores_static",
           "wnw_set_roles_device",
           "wnw_append_kv", "wnw_decode_step", "wnw_query_geometry",
           "wnw_query_segments", "wnw_query_head_keep", "wnw_get_stats",
           "wnw_set_selection_override", "wnw_debug_read_slot", "wnw_debug_read_host_chunk",
           "wnw_debug_set_slot_offset_limit", "wnw_debug_set_recall_delay",
           "wnw_debug_read_resident", "wnw_last_error", "wnw_destroy", "wnw_voice_hits", "wnw_key_sensitivity",
           "wnw_triage", "wnw_triage_last_error",
           "wnw_quant_write", "wnw_quant_read", "wnw_quant_attend", "wnw_quant_attend_workspace", "wnw_quant_last_error",
           "wnw_rotary_frequencies", "wnw_paged_append", "wnw_paged_attend", "wnw_paged_attend_workspace", "wnw_paged_keep",
           "wnw_paged_last_error", "wnw_draft_tree", "wnw_draft_verify", "wnw_draft_verify_workspace", "wnw_draft_last_error")


class wnw_config(C.Structure):
    _fields_ = [("batch", C.c_int32), ("layers", C.c_int32), ("q_heads", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("audio_len", C.c_int32), ("text_len", C.c_int32),
                ("chunk_len", C.c_int32), ("budget_bp", C.c_int32), ("top_k", C.c_int32),
                ("evict_lag", C.c_int32), ("flags", C.c_uint32), ("max_new_tokens", C.c_int32)]


class wnw_stats(C.Structure):
    _fields_ = [("steps", C.c_int64), ("recalled_chunks", C.c_int64), ("revived_chunks", C.c_int64),
                ("recalled_bytes", C.c_int64),
                ("dropped_chunks", C.c_int64), ("resident_chunks", C.c_int64), ("peak_resident", C.c_int32),
                ("n_slots", C.c_int32), ("r_gpu", C.c_double), ("r_gpu_cpu", C.c_double),
                ("anchor_bytes", C.c_int64), ("static_bytes", C.c_int64), ("slot_rows", C.c_int64),
                ("timed_steps", C.c_int64), ("t_anchor_ms", C.c_double), ("t_select_ms", C.c_double),
                ("t_tidal_fixed_ms", C.c_double), ("t_new_ms", C.c_double), ("t_combine_ms", C.c_double),
                ("t_step_ms", C.c_double), ("t_recall_ms", C.c_double), ("slot_exhausted", C.c_int64),
                ("t_host_wait_ms", C.c_double), ("t_recall_wait_ms", C.c_double), ("kept_rows", C.c_int64),
                ("selections_in_tidal", C.c_int64)]

    def as_dict(self) -> dict:
        return {name: getattr(self, name) for name, _ in self._fields_}


class wnw_quant_config(C.Structure):
    _fields_ = [("batch", C.c_int32), ("layers", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("capacity", C.c_int32), ("block", C.c_int32), ("format", C.c_int32), ("flags", C.c_uint32)]


class wnw_quant_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class wnw_paged_config(C.Structure):
    _fields_ = [("batch", C.c_int32), ("layers", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page", C.c_int32), ("pages", C.c_int32), ("table_width", C.c_int32), ("flags", C.c_uint32)]


class wnw_paged_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("table", C.c_void_p)]


class wnw_rotary(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("dim", C.c_int32), ("layout", C.c_int32), ("amplitude", C.c_float)]


class WnwError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"wnw status {status}: {msg}")
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build the HIP library first (__graft_entry__.build())")
    lib = C.CDLL(LIB_PATH)
    P, I32, I64, SZ = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    QC, QK = C.POINTER(wnw_quant_config), C.POINTER(wnw_quant_cache)
    PC, PK = C.POINTER(wnw_paged_config), C.POINTER(wnw_paged_cache)
    sig = {
        "wnw_init_cache": ([C.POINTER(wnw_config), P, P, P, C.POINTER(P)], C.c_int),
        "wnw_set_roles": ([P, P, P], C.c_int),
        "wnw_set_retention": ([P, P, C.c_float], C.c_int),
        "wnw_prefill_scores": ([P, P, P], C.c_int),
        "wnw_prefill_scores_static": ([P, P, P, P], C.c_int),
        "wnw_append_kv": ([P, P, P, P], C.c_int),
        "wnw_voice_hits": ([I32, I32, I32, I32, I32, I32, P, P, P, I32, P, P], C.c_int),
        "wnw_key_sensitivity": ([I32, I32, I32, I32, P, P, P], C.c_int),
        "wnw_triage": ([I32, I32, I32, I32, P, P, I32, P, I32, I32, P, P, P, P], C.c_int),
        "wnw_triage_last_error": ([], C.c_char_p),
        "wnw_quant_write": ([QC, QK, I32, I32, I32, P, P, P, P, P], C.c_int),
        "wnw_quant_read": ([QC, QK, I32, I32, I32, P, P, P, P, P], C.c_int),
        "wnw_quant_attend": ([QC, QK, I32, I32, I32, I32, P, P, P, P, P, P, I32, P, SZ, P], C.c_int),
        "wnw_quant_attend_workspace": ([QC, I32, I32, I32, I32, C.POINTER(SZ)], C.c_int),
        "wnw_quant_last_error": ([], C.c_char_p),
        "wnw_rotary_frequencies": ([I32, C.c_double, C.c_double, C.c_double, C.c_double, I64, P], C.c_int),
        "wnw_paged_append": ([PC, PK, C.POINTER(wnw_rotary), I32, I32, I32, I32, P, P, P, P, P, P, P, P], C.c_int),
        "wnw_paged_attend": ([PC, PK, I32, I32, I32, I32, P, P, P, P, P, P, I32, P, SZ, P], C.c_int),
        "wnw_paged_attend_workspace": ([PC, I32, I32, I32, I32, C.POINTER(SZ)], C.c_int),
        "wnw_paged_keep": ([PC, PK, I32, I32, I32, P, P, P, P], C.c_int),
        "wnw_paged_last_error": ([], C.c_char_p),
        "wnw_draft_tree": ([I32, I32, P, P, P, P, P, P], C.c_int),
        "wnw_draft_verify": ([I32, I32, I32, P, P, P, P, P, P, P, P, P, P, SZ, P], C.c_int),
        "wnw_draft_verify_workspace": ([I32, I32, I32, C.POINTER(SZ)], C.c_int),
        "wnw_draft_last_error": ([], C.c_char_p),
        "wnw_set_roles_device": ([P, P, P], C.c_int),
        "wnw_query_head_keep": ([P, P], C.c_int),
        "wnw_decode_step": ([P, P, P, P, P, P], C.c_int),
        "wnw_query_geometry": ([P, C.POINTER(I32), C.POINTER(I32), C.POINTER(I32), C.POINTER(I32), C.POINTER(I64)], C.c_int),
        "wnw_query_segments": ([P, C.POINTER(I32)], C.c_int),
        "wnw_get_stats": ([P, C.POINTER(wnw_stats)], C.c_int),
        "wnw_set_selection_override": ([P, P], C.c_int),
        "wnw_debug_read_slot": ([P, I32, I32, P, SZ], C.c_int),
        "wnw_debug_read_host_chunk": ([P, I32, I32, P, SZ], C.c_int),
        "wnw_debug_read_resident": ([P, P], C.c_int),
        "wnw_debug_set_slot_offset_limit": ([P, I64], C.c_int),
        "wnw_debug_set_recall_delay": ([P, I32], C.c_int),
        "wnw_last_error": ([P], C.c_char_p),
        "wnw_destroy": ([P], None),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, res
    return lib


lib = _load()


def _check(status: int, ctx=None):
    if status != WNW_OK:
        raise WnwError(status, lib.wnw_last_error(ctx).decode())


def _ptr(t):
    """Device (or host) address of a tensor / numpy array / int, or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return t.ctypes.data


# element sizes the library reads or writes: bf16 bit patterns (any 2-byte dtype), fp32, int32, bytes
_BF16, _F32, _I32, _U8, _I64 = "bf16", "f32", "i32", "u8", "i64"


def _dev(t, kind, numel=None, what="tensor"):
    """Address of a device tensor after checking it holds at least `numel` contiguous elements
    of the kind the library expects (no conversion: the library reads the raw buffer)."""
    if t is None or isinstance(t, int):
        return t
    if not hasattr(t, "data_ptr"):
        raise TypeError(f"{what} must be a device tensor")
    import torch
    ok = {_BF16: t.element_size() == 2 and not t.dtype.is_complex,
          _F32: t.dtype == torch.float32, _I32: t.dtype == torch.int32, _U8: t.dtype == torch.uint8}[kind]
    if not ok:
        raise TypeError(f"{what}: expected {kind} elements, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{what}: needs {numel} elements, got {t.numel()}")
    return t.data_ptr()


def _host_in(a, dtype, numel=None, what="array"):
    """A contiguous host copy (or view) of `a` with the given numpy dtype, size checked."""
    a = np.ascontiguousarray(a, dtype=dtype)
    if numel is not None and a.size != numel:
        raise ValueError(f"{what}: expected {numel} elements, got {a.size}")
    return a


def _host_out(a, nbytes, what="host_dst"):
    """Address of a writable, contiguous host array of exactly nbytes."""
    if not isinstance(a, np.ndarray) or not a.flags.c_contiguous or not a.flags.writeable:
        raise TypeError(f"{what} must be a writable C-contiguous numpy array")
    if a.nbytes != nbytes:
        raise ValueError(f"{what}: expected {nbytes} bytes, got {a.nbytes}")
    return a.ctypes.data


_CFG = {}   # handle value -> wnw_config, for the size checks of later calls


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


# ---- the C ABI, one wrapper per entry point -------------------------------------------------

def _cache_numel(cfg):
    return cfg.batch * cfg.layers * cfg.kv_heads * (cfg.audio_len + cfg.text_len) * cfg.head_dim


def wnw_init_cache(cfg: wnw_config, k_dev, v_dev, stream=None):
    n = _cache_numel(cfg)
    h = C.c_void_p()
    _check(lib.wnw_init_cache(C.byref(cfg), _dev(k_dev, _BF16, n, "k_dev"), _dev(v_dev, _BF16, n, "v_dev"),
                              _stream(stream), C.byref(h)))
    _CFG[h.value] = wnw_config.from_buffer_copy(cfg)
    return h


def _cfg(ctx):
    return _CFG.get(getattr(ctx, "value", ctx))


def wnw_set_retention(ctx, importance, lam):
    """importance: host fp32 [L][H_kv] (or None for the uniform budget); lam: the scale."""
    c = _cfg(ctx)
    imp = None if importance is None else _host_in(importance, np.float32, c and c.layers * c.kv_heads, "importance")
    _check(lib.wnw_set_retention(ctx, _ptr(imp), float(lam)), ctx)


def wnw_set_roles(ctx, roles, prefill_scores):
    """roles: host uint8 [L][H_kv]; prefill_scores: host fp32 [B][L][H_kv][T_a]."""
    c = _cfg(ctx)
    r = _host_in(roles, np.uint8, c and c.layers * c.kv_heads, "roles")
    p = _host_in(prefill_scores, np.float32, c and c.batch * c.layers * c.kv_heads * c.audio_len, "prefill_scores")
    _check(lib.wnw_set_roles(ctx, _ptr(r), _ptr(p)), ctx)


def _tcheck(status):
    if status != WNW_OK:
        raise WnwError(status, lib.wnw_triage_last_error().decode())


def wnw_voice_hits(k_dev, q_dev, span_dev, top_k, audio_len, hits_dev, stream=None):
    """k_dev [L][H_kv][rows][d] bf16, q_dev [n_tok][L][H_q][d] bf16, span_dev int32 [n_tok][2] ->
    hits_dev int32 [n_tok][L][H_q] (tensors on the device)."""
    L, Hkv, rows, D = k_dev.shape
    n_tok, _, Hq, _ = q_dev.shape
    _tcheck(lib.wnw_voice_hits(L, Hq, Hkv, rows, audio_len, n_tok, _dev(k_dev, _BF16, None, "k_dev"),
                               _dev(q_dev, _BF16, n_tok * L * Hq * D, "q_dev"), _dev(span_dev, _I32, n_tok * 2, "span_dev"),
                               top_k, _dev(hits_dev, _I32, n_tok * L * Hq, "hits_dev"), _stream(stream)))


def wnw_key_sensitivity(grad_dev, sens_dev, stream=None):
    """grad_dev fp32 [n_tok][L][H_kv][T_a][d] -> sens_dev fp32 [n_tok][L][H_kv]."""
    n_tok, L, Hkv, Ta, _ = grad_dev.shape
    _tcheck(lib.wnw_key_sensitivity(L, Hkv, Ta, n_tok, _dev(grad_dev, _F32, None, "grad_dev"),
                                    _dev(sens_dev, _F32, n_tok * L * Hkv, "sens_dev"), _stream(stream)))


def wnw_triage(hits, top_k, sens, sample, n_voice, n_anchor):
    """Host arrays hits int32 [n][L][H_q], sens fp32 [n][L][H_kv], sample int32 [n] ->
    (roles uint8, importance fp32, vs, hs) each [L][H_kv]."""
    hits = np.ascontiguousarray(hits, dtype=np.int32)
    sens = np.ascontiguousarray(sens, dtype=np.float32)
    sample = np.ascontiguousarray(sample, dtype=np.int32)
    n, L, Hq = hits.shape
    Hkv = sens.shape[2]
    roles = np.empty((L, Hkv), dtype=np.uint8)
    imp = np.empty((L, Hkv), dtype=np.float32)
    vs, hs = np.empty((L, Hkv)), np.empty((L, Hkv))
    _tcheck(lib.wnw_triage(L, Hkv, Hq // Hkv, n, _ptr(sample), _ptr(hits), top_k, _ptr(sens), n_voice, n_anchor,
                           _ptr(roles), _ptr(imp), _ptr(vs), _ptr(hs)))
    return roles, imp, vs, hs


class QuantCache:
    """The buffers of an 8-bit cache (see wnw.h): k uint8 [B][L][H_kv][capacity][d], v uint8
    [B][L][H_kv][capacity / 64][d][64], scales fp32 [B][L][H_kv][capacity / block]."""

    def __init__(self, k, v, k_scale, v_scale):
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale

    def __setattr__(self, name, t):
        # type and layout are checked once here, device and size by every call
        _on(t.get_device(), t, _dtypes()[_F32 if name.endswith("scale") else _U8], None, name)
        object.__setattr__(self, name, t)

    def _struct(self, cfg, device):
        n = cfg.batch * cfg.layers * cfg.kv_heads * cfg.capacity
        need, scales = n * cfg.head_dim, n // (cfg.block or 1)
        k, v, ks, vs = self.k, self.v, self.k_scale, self.v_scale
        if (k.numel() < need or v.numel() < need or ks.numel() < scales or vs.numel() < scales or k.get_device() != device
                or v.get_device() != device or ks.get_device() != device or vs.get_device() != device):
            for name, t, numel in (("k", k, need), ("v", v, need), ("k_scale", ks, scales), ("v_scale", vs, scales)):
                if t.get_device() != device or t.numel() < numel:
                    raise ValueError(f"{name}: needs {numel} elements on cuda:{device}, got {t.numel()} on {t.device}")
        return wnw_quant_cache(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr())


def make_quant_config(batch, layers, kv_heads, capacity, block, format, head_dim=128, flags=0) -> wnw_quant_config:
    return wnw_quant_config(batch, layers, kv_heads, head_dim, capacity, block, format, flags)


def make_quant_cache(cfg, device="cuda") -> QuantCache:
    """New buffers for cfg on a device, uninitialised: no row is meaningful before it is written."""
    import torch
    heads = (cfg.batch, cfg.layers, cfg.kv_heads)
    scales = [torch.empty((*heads, cfg.capacity // cfg.block), dtype=torch.float32, device=device) for _ in range(2)]
    return QuantCache(torch.empty((*heads, cfg.capacity, cfg.head_dim), dtype=torch.uint8, device=device),
                      torch.empty((*heads, cfg.capacity // 64, cfg.head_dim, 64), dtype=torch.uint8, device=device), *scales)


def _qcheck(status):
    if status != WNW_OK:
        raise WnwError(status, lib.wnw_quant_last_error().decode())


_DTYPES = {}


def _dtypes():
    """Element kind -> the torch types that the calls below take for it."""
    if not _DTYPES:
        import torch
        _DTYPES.update({_BF16: (torch.bfloat16, torch.int16, torch.uint16), _F32: (torch.float32,), _I32: (torch.int32,),
                        _U8: (torch.uint8,), _I64: (torch.int64, torch.uint64)})
    return _DTYPES


def _on(device, t, kinds, numel, what):
    """Address of a tensor that must be on the GPU `device` (its index), where the call's work runs, with the checks of
    _dev(); half precision is not taken for bf16.  These calls are made for every layer and token: no detours."""
    if t is None or isinstance(t, int):
        return t
    if t.get_device() != device:
        raise ValueError(f"{what} is on {t.device}, the call's work on cuda:{device}")
    if t.dtype not in kinds:
        raise TypeError(f"{what}: expected {' or '.join(map(str, kinds))}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{what}: needs {numel} elements, got {t.numel()}")
    return t.data_ptr()


def _quant_shape(cfg, t, heads, what):
    """(layers, tokens) of rows [B][n_layers][heads][n][d]."""
    shape = t.shape
    if len(shape) != 5 or shape[0] != cfg.batch or shape[2] != heads or shape[4] != cfg.head_dim:
        raise ValueError(f"{what}: expected [{cfg.batch}][n_layers][{heads}][n][{cfg.head_dim}], got {list(shape)}")
    return shape[1], shape[3]


def _quant_place(stream):
    """(index of the current device, stream handle): where a call's work runs.  The library launches on the current device,
    so a stream of another one is refused."""
    import torch
    device = torch.cuda.current_device()
    if stream is not None:
        on = getattr(stream, "device", None)     # (a bare handle does not say)
        if on is not None and on.index != device:
            raise ValueError(f"stream is on {on}, the current device is cuda:{device}")
        return device, getattr(stream, "cuda_stream", stream)
    # the handle alone: a Stream object costs 2.5 us, as much as a launch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return device, raw(device) if raw else torch.cuda.current_stream().cuda_stream


def wnw_quant_write(cfg, cache, k_dev, v_dev, pos_dev, count_dev=None, first_layer=0, stream=None):
    """k_dev, v_dev bf16 [B][n_layers][H_kv][n][d] -> rows pos[b] .. pos[b] + count[b] - 1 of the cache
    (pos_dev, count_dev: int32 [B])."""
    nl, n = _quant_shape(cfg, k_dev, cfg.kv_heads, "k_dev")
    if v_dev.shape != k_dev.shape:
        raise ValueError(f"v_dev: expected {list(k_dev.shape)}, got {list(v_dev.shape)}")
    (dev, st), k, B = _quant_place(stream), _DTYPES or _dtypes(), cfg.batch
    _qcheck(lib.wnw_quant_write(cfg, cache._struct(cfg, dev), first_layer, nl, n, _on(dev, k_dev, k[_BF16], None, "k_dev"),
                                _on(dev, v_dev, k[_BF16], None, "v_dev"), _on(dev, pos_dev, k[_I32], B, "pos_dev"),
                                _on(dev, count_dev, k[_I32], B, "count_dev"), st))


def wnw_quant_read(cfg, cache, k_out, v_out, pos_dev, count_dev=None, first_layer=0, stream=None):
    """Rows pos[b] .. pos[b] + count[b] - 1 -> k_out, v_out [B][n_layers][H_kv][n][d], fp32 or (WNW_F_OUT_BF16)
    bf16; one of the two may be None."""
    some = k_out if k_out is not None else v_out
    if some is None:
        raise ValueError("k_out or v_out must be given")
    nl, n = _quant_shape(cfg, some, cfg.kv_heads, "k_out" if k_out is not None else "v_out")
    if v_out is not None and v_out.shape != some.shape:
        raise ValueError(f"v_out: expected {list(some.shape)}, got {list(v_out.shape)}")
    (dev, st), k, B = _quant_place(stream), _DTYPES or _dtypes(), cfg.batch
    out = k[_BF16 if cfg.flags & WNW_F_OUT_BF16 else _F32]
    _qcheck(lib.wnw_quant_read(cfg, cache._struct(cfg, dev), first_layer, nl, n, _on(dev, k_out, out, None, "k_out"),
                               _on(dev, v_out, out, None, "v_out"), _on(dev, pos_dev, k[_I32], B, "pos_dev"),
                               _on(dev, count_dev, k[_I32], B, "count_dev"), st))


def wnw_quant_attend_workspace(cfg, n_layers, q_heads, n, max_len=0) -> int:
    """Bytes of workspace that wnw_quant_attend needs for these sizes."""
    need = C.c_size_t()
    _qcheck(lib.wnw_quant_attend_workspace(cfg, n_layers, q_heads, n, max_len, C.byref(need)))
    return need.value


def wnw_quant_attend(cfg, cache, q_dev, out_dev, len_dev, count_dev=None, lse_dev=None, mass_dev=None, workspace=None,
                     max_len=0, first_layer=0, stream=None):
    """q_dev bf16 [B][n_layers][H_q][n][d] -> out_dev (same shape, fp32 or bf16), lse_dev fp32 [B][n_layers][H_q][n],
    mass_dev fp32 [B][n_layers][H_q][capacity / block] (n = 1); workspace: a uint8 tensor of
    wnw_quant_attend_workspace() bytes or more."""
    shape = q_dev.shape
    Hq = shape[2] if len(shape) == 5 else 0
    nl, n = _quant_shape(cfg, q_dev, Hq, "q_dev")
    if out_dev.shape != shape:
        raise ValueError(f"out_dev: expected {list(shape)}, got {list(out_dev.shape)}")
    (dev, st), k, B = _quant_place(stream), _DTYPES or _dtypes(), cfg.batch
    rows = B * nl * Hq
    _qcheck(lib.wnw_quant_attend(
        cfg, cache._struct(cfg, dev), first_layer, nl, Hq, n, _on(dev, q_dev, k[_BF16], None, "q_dev"),
        _on(dev, len_dev, k[_I32], B, "len_dev"), _on(dev, count_dev, k[_I32], B, "count_dev"),
        _on(dev, out_dev, k[_BF16 if cfg.flags & WNW_F_OUT_BF16 else _F32], None, "out_dev"),
        _on(dev, lse_dev, k[_F32], rows * n, "lse_dev"),
        _on(dev, mass_dev, k[_F32], rows * (cfg.capacity // max(cfg.block, 1)), "mass_dev"), max_len,
        _on(dev, workspace, k[_U8], None, "workspace"), 0 if workspace is None else workspace.numel(), st))


class PagedCache:
    """The buffers of a paged cache (see wnw.h): k, v bf16 [pages][L][H_kv][page][d], table int32 [B][table_width]."""

    def __init__(self, k, v, table):
        self.k, self.v, self.table = k, v, table

    def __setattr__(self, name, t):
        # type and layout are checked once here, device and size by every call
        _on(t.get_device(), t, _dtypes()[_I32 if name == "table" else _BF16], None, name)
        object.__setattr__(self, name, t)

    def _struct(self, cfg, device):
        need, entries = cfg.pages * cfg.layers * cfg.kv_heads * cfg.page * cfg.head_dim, cfg.batch * cfg.table_width
        k, v, table = self.k, self.v, self.table
        if (k.numel() < need or v.numel() < need or table.numel() < entries or k.get_device() != device
                or v.get_device() != device or table.get_device() != device):
            for name, t, numel in (("k", k, need), ("v", v, need), ("table", table, entries)):
                if t.get_device() != device or t.numel() < numel:
                    raise ValueError(f"{name}: needs {numel} elements on cuda:{device}, got {t.numel()} on {t.device}")
        return wnw_paged_cache(k.data_ptr(), v.data_ptr(), table.data_ptr())


def make_paged_config(batch, layers, kv_heads, page, pages, table_width, head_dim=128, flags=0) -> wnw_paged_config:
    return wnw_paged_config(batch, layers, kv_heads, head_dim, page, pages, table_width, flags)


def make_paged_cache(cfg, device="cuda") -> PagedCache:
    """New pages for cfg on a device, uninitialised, and a table without pages (-1): the caller hands them out."""
    import torch
    k, v = (torch.empty((cfg.pages, cfg.layers, cfg.kv_heads, cfg.page, cfg.head_dim), dtype=torch.bfloat16, device=device)
            for _ in range(2))
    return PagedCache(k, v, torch.full((cfg.batch, cfg.table_width), -1, dtype=torch.int32, device=device))


class Rotary:
    """How wnw_paged_append rotates (see wnw.h): freq fp32 [dim / 2] on the device, radians per position."""

    def __init__(self, freq, dim, layout, amplitude):
        if freq is None and dim:
            raise ValueError("freq must be given where dim is not 0")
        if freq is not None:
            _on(freq.get_device(), freq, _dtypes()[_F32], dim // 2, "freq")
        self.freq, self.dim, self.layout, self.amplitude = freq, dim, layout, amplitude

    def _struct(self, device):
        return wnw_rotary(_on(device, self.freq, _dtypes()[_F32], self.dim // 2, "freq"), self.dim, self.layout, self.amplitude)


def make_rotary(freq, dim, layout=WNW_ROTARY_HALVES, amplitude=1.0) -> Rotary:
    return Rotary(freq, dim, layout, amplitude)


def wnw_rotary_frequencies(dim, base, factor=1.0, low=0.0, high=0.0, original_len=0) -> np.ndarray:
    """Host fp32 [dim / 2], radians per position; for contexts longer than original_len by factor see wnw.h."""
    freq = np.empty(max(dim, 0) // 2, dtype=np.float32)
    _pcheck(lib.wnw_rotary_frequencies(dim, base, factor, low, high, original_len, _ptr(freq)))
    return freq


def _pcheck(status):
    if status != WNW_OK:
        raise WnwError(status, lib.wnw_paged_last_error().decode())


def wnw_paged_append(cfg, cache, k_dev, v_dev, at_dev, count_dev=None, q_dev=None, q_out=None, rotary=None, position_dev=None,
                     first_layer=0, stream=None):
    """k_dev, v_dev bf16 [B][n_layers][H_kv][n][d] -> rows at[b] .. at[b] + count[b] - 1 of the pages, K rotated; q_dev bf16
    [B][n_layers][H_q][n][d] -> q_out, rotated (at_dev, count_dev: int32 [B]; position_dev: int32 [B][n])."""
    some = k_dev if k_dev is not None else q_dev
    if some is None:
        raise ValueError("k_dev or q_dev must be given")
    if (k_dev is None) != (v_dev is None) or (q_dev is None) != (q_out is None):
        raise ValueError("k_dev and v_dev, and q_dev and q_out, are given together")
    shape = some.shape
    Hq = 0
    if k_dev is not None:
        nl, n = _quant_shape(cfg, k_dev, cfg.kv_heads, "k_dev")
        if v_dev.shape != shape:
            raise ValueError(f"v_dev: expected {list(shape)}, got {list(v_dev.shape)}")
    if q_dev is not None:
        Hq = q_dev.shape[2] if len(q_dev.shape) == 5 else 0
        q_nl, q_n = _quant_shape(cfg, q_dev, Hq, "q_dev")
        if k_dev is None:
            nl, n = q_nl, q_n
        if (q_nl, q_n) != (nl, n) or q_out.shape != q_dev.shape:
            raise ValueError(f"q_dev, q_out: expected {nl} layers and {n} tokens each, got {list(q_dev.shape)}, {list(q_out.shape)}")
    (dev, st), k, B = _quant_place(stream), _DTYPES or _dtypes(), cfg.batch
    _pcheck(lib.wnw_paged_append(
        cfg, cache._struct(cfg, dev), None if rotary is None else rotary._struct(dev), first_layer, nl, Hq, n,
        _on(dev, k_dev, k[_BF16], None, "k_dev"), _on(dev, v_dev, k[_BF16], None, "v_dev"), _on(dev, q_dev, k[_BF16], None, "q_dev"),
        _on(dev, q_out, k[_BF16], None, "q_out"), _on(dev, at_dev, k[_I32], B, "at_dev"), _on(dev, count_dev, k[_I32], B, "count_dev"),
        _on(dev, position_dev, k[_I32], B * n, "position_dev"), st))


def wnw_paged_attend_workspace(cfg, n_layers, q_heads, n, max_len=0) -> int:
    """Bytes of workspace that wnw_paged_attend needs for these sizes."""
    need = C.c_size_t()
    _pcheck(lib.wnw_paged_attend_workspace(cfg, n_layers, q_heads, n, max_len, C.byref(need)))
    return need.value


def wnw_paged_attend(cfg, cache, q_dev, out_dev, len_dev, count_dev=None, mask_dev=None, lse_dev=None, workspace=None, max_len=0,
                     first_layer=0, stream=None):
    """q_dev bf16 [B][n_layers][H_q][n][d] -> out_dev (same shape, fp32 or bf16), lse_dev fp32 [B][n_layers][H_q][n];
    mask_dev int64 [B][n][(n + 63) // 64] (None: causal); workspace: a uint8 tensor of wnw_paged_attend_workspace() bytes or more."""
    shape = q_dev.shape
    Hq = shape[2] if len(shape) == 5 else 0
    nl, n = _quant_shape(cfg, q_dev, Hq, "q_dev")
    if out_dev.shape != shape:
        raise ValueError(f"out_dev: expected {list(shape)}, got {list(out_dev.shape)}")
    (dev, st), k, B = _quant_place(stream), _DTYPES or _dtypes(), cfg.batch
    _pcheck(lib.wnw_paged_attend(
        cfg, cache._struct(cfg, dev), first_layer, nl, Hq, n, _on(dev, q_dev, k[_BF16], None, "q_dev"),
        _on(dev, len_dev, k[_I32], B, "len_dev"), _on(dev, count_dev, k[_I32], B, "count_dev"),
        _on(dev, mask_dev, k[_I64], B * n * ((n + 63) // 64), "mask_dev"),
        _on(dev, out_dev, k[_BF16 if cfg.flags & WNW_F_OUT_BF16 else _F32], None, "out_dev"),
        _on(dev, lse_dev, k[_F32], B * nl * Hq * n, "lse_dev"), max_len, _on(dev, workspace, k[_U8], None, "workspace"),
        0 if workspace is None else workspace.numel(), st))


def wnw_paged_keep(cfg, cache, base_dev, path_dev, count_dev=None, first_layer=0, n_layers=None, stream=None):
    """Rows base[b] + path[b][i] -> base[b] + i, i < count[b], of n_layers layers (None: all from first_layer on); path_dev int32
    [B][n], ascending."""
    if len(path_dev.shape) != 2 or path_dev.shape[0] != cfg.batch:
        raise ValueError(f"path_dev: expected [{cfg.batch}][n], got {list(path_dev.shape)}")
    (dev, st), k, B = _quant_place(stream), _DTYPES or _dtypes(), cfg.batch
    _pcheck(lib.wnw_paged_keep(cfg, cache._struct(cfg, dev), first_layer, cfg.layers - first_layer if n_layers is None else n_layers,
                               path_dev.shape[1], _on(dev, base_dev, k[_I32], B, "base_dev"), _on(dev, path_dev, k[_I32], None, "path_dev"),
                               _on(dev, count_dev, k[_I32], B, "count_dev"), st))


def _dcheck(status):
    if status != WNW_OK:
        raise WnwError(status, lib.wnw_draft_last_error().decode())


def wnw_draft_tree(parent_dev, base_dev, mask_dev=None, position_dev=None, count_dev=None, stream=None):
    """parent_dev int32 [B][n] -> mask_dev int64 [B][n][(n + 63) // 64], position_dev int32 [B][n] (either may be None);
    base_dev, count_dev int32 [B]."""
    B, n = parent_dev.shape
    (dev, st), k = _quant_place(stream), _DTYPES or _dtypes()
    _dcheck(lib.wnw_draft_tree(B, n, _on(dev, parent_dev, k[_I32], None, "parent_dev"), _on(dev, base_dev, k[_I32], B, "base_dev"),
                               _on(dev, count_dev, k[_I32], B, "count_dev"),
                               _on(dev, mask_dev, k[_I64], B * n * ((n + 63) // 64), "mask_dev"),
                               _on(dev, position_dev, k[_I32], B * n, "position_dev"), st))


def wnw_draft_verify_workspace(batch, n, vocab) -> int:
    """Bytes of workspace that wnw_draft_verify needs for these sizes."""
    need = C.c_size_t()
    _dcheck(lib.wnw_draft_verify_workspace(batch, n, vocab, C.byref(need)))
    return need.value


def wnw_draft_verify(token_dev, target_dev, uniform_dev, path_dev, accepted_dev, next_dev, draft_dev=None, parent_dev=None,
                     count_dev=None, workspace=None, stream=None):
    """token_dev int32 [B][n], target_dev fp32 [B][n + 1][vocab], uniform_dev fp32 [B][n + 1] -> path_dev int32 [B][n],
    accepted_dev, next_dev int32 [B]; draft_dev like target_dev; parent_dev int32 [B][n]; workspace: a uint8 tensor of
    wnw_draft_verify_workspace() bytes or more."""
    B, n = token_dev.shape
    shape = target_dev.shape
    if len(shape) != 3 or shape[0] != B or shape[1] != n + 1:
        raise ValueError(f"target_dev: expected [{B}][{n + 1}][vocab], got {list(shape)}")
    if draft_dev is not None and draft_dev.shape != shape:
        raise ValueError(f"draft_dev: expected {list(shape)}, got {list(draft_dev.shape)}")
    (dev, st), k = _quant_place(stream), _DTYPES or _dtypes()
    _dcheck(lib.wnw_draft_verify(
        B, n, shape[2], _on(dev, token_dev, k[_I32], None, "token_dev"), _on(dev, parent_dev, k[_I32], B * n, "parent_dev"),
        _on(dev, count_dev, k[_I32], B, "count_dev"), _on(dev, target_dev, k[_F32], None, "target_dev"),
        _on(dev, draft_dev, k[_F32], None, "draft_dev"), _on(dev, uniform_dev, k[_F32], B * (n + 1), "uniform_dev"),
        _on(dev, path_dev, k[_I32], B * n, "path_dev"), _on(dev, accepted_dev, k[_I32], B, "accepted_dev"),
        _on(dev, next_dev, k[_I32], B, "next_dev"), _on(dev, workspace, k[_U8], None, "workspace"),
        0 if workspace is None else workspace.numel(), st))


def wnw_append_kv(ctx, k_new_dev, v_new_dev, stream=None):
    c = _cfg(ctx)
    n = c and c.batch * c.layers * c.kv_heads * c.head_dim
    _check(lib.wnw_append_kv(ctx, _dev(k_new_dev, _BF16, n, "k_new_dev"), _dev(v_new_dev, _BF16, n, "v_new_dev"),
                             _stream(stream)), ctx)


def wnw_prefill_scores(ctx, q_text_dev, scores_dev):
    c = _cfg(ctx)
    nq = c and c.batch * c.layers * c.q_heads * c.text_len * c.head_dim
    ns = c and c.batch * c.layers * c.kv_heads * c.audio_len
    _check(lib.wnw_prefill_scores(ctx, _dev(q_text_dev, _BF16, nq, "q_text_dev"), _dev(scores_dev, _F32, ns, "scores_dev")),
           ctx)


def wnw_prefill_scores_static(ctx, q_text_dev, scores_dev, stream=None):
    c = _cfg(ctx)
    nq = c and c.batch * c.layers * c.q_heads * c.text_len * c.head_dim
    ns = c and c.batch * c.layers * c.kv_heads * c.audio_len
    _check(lib.wnw_prefill_scores_static(ctx, _dev(q_text_dev, _BF16, nq, "q_text_dev"),
                                         _dev(scores_dev, _F32, ns, "scores_dev"), _stream(stream)), ctx)


def wnw_set_roles_device(ctx, roles, prefill_scores_dev):
    c = _cfg(ctx)
    r = _host_in(roles, np.uint8, c and c.layers * c.kv_heads, "roles")
    ns = c and c.batch * c.layers * c.kv_heads * c.audio_len
    _check(lib.wnw_set_roles_device(ctx, _ptr(r), _dev(prefill_scores_dev, _F32, ns, "prefill_scores_dev")), ctx)


def wnw_query_head_keep(ctx, layers, kv_heads) -> np.ndarray:
    keep = np.empty((layers, kv_heads), dtype=np.int32)
    _check(lib.wnw_query_head_keep(ctx, _ptr(keep)), ctx)
    return keep


def wnw_decode_step(ctx, q_dev, out_dev, chunk_scores_dev=None, selected_dev=None, stream=None):
    c = _cfg(ctx)
    nq = c and c.batch * c.layers * c.q_heads * c.head_dim
    okind = _BF16 if c and c.flags & WNW_F_OUT_BF16 else _F32
    _check(lib.wnw_decode_step(ctx, _dev(q_dev, _BF16, nq, "q_dev"), _dev(out_dev, okind, nq, "out_dev"),
                               _dev(chunk_scores_dev, _F32, None, "chunk_scores_dev"),
                               _dev(selected_dev, _I32, None, "selected_dev"), _stream(stream)), ctx)


def wnw_query_geometry(ctx) -> dict:
    n, k, kt, ns, cb = C.c_int32(), C.c_int32(), C.c_int32(), C.c_int32(), C.c_int64(-1)
    _check(lib.wnw_query_geometry(ctx, C.byref(n), C.byref(k), C.byref(kt), C.byref(ns), None), ctx)
    out = {"n_chunks": n.value, "k": k.value, "keep_total": kt.value, "n_slots": ns.value}
    seg = C.c_int32()
    _check(lib.wnw_query_segments(ctx, C.byref(seg)), ctx)
    out["n_segments"] = seg.value
    if lib.wnw_query_geometry(ctx, None, None, None, None, C.byref(cb)) == WNW_OK:
        out["chunk_bytes"] = cb.value
    return out


def wnw_get_stats(ctx) -> dict:
    st = wnw_stats()
    _check(lib.wnw_get_stats(ctx, C.byref(st)), ctx)
    return st.as_dict()


def wnw_set_selection_override(ctx, sel_dev):
    _check(lib.wnw_set_selection_override(ctx, _dev(sel_dev, _I32, None, "sel_dev")), ctx)


def wnw_debug_set_slot_offset_limit(ctx, nbytes: int):
    _check(lib.wnw_debug_set_slot_offset_limit(ctx, nbytes), ctx)


def wnw_debug_set_recall_delay(ctx, us: int):
    _check(lib.wnw_debug_set_recall_delay(ctx, us), ctx)


def wnw_debug_read_slot(ctx, b: int, chunk: int, host_dst, nbytes: int):
    _check(lib.wnw_debug_read_slot(ctx, b, chunk, _host_out(host_dst, nbytes), nbytes), ctx)


def wnw_debug_read_host_chunk(ctx, b: int, chunk: int, host_dst, nbytes: int):
    _check(lib.wnw_debug_read_host_chunk(ctx, b, chunk, _host_out(host_dst, nbytes), nbytes), ctx)


def wnw_debug_read_resident(ctx, host_dst):
    """host_dst: writable uint8 [B][n_segments]."""
    seg = C.c_int32()
    _check(lib.wnw_query_segments(ctx, C.byref(seg)), ctx)
    c = _cfg(ctx)
    need = c.batch * seg.value if c is not None else 0
    if not isinstance(host_dst, np.ndarray) or not host_dst.flags.c_contiguous or not host_dst.flags.writeable \
            or host_dst.dtype != np.uint8 or host_dst.nbytes < need:
        raise ValueError(f"host_dst must be a writable contiguous uint8 array of at least {need} elements")
    _check(lib.wnw_debug_read_resident(ctx, _ptr(host_dst)), ctx)


def wnw_last_error(ctx=None) -> str:
    return lib.wnw_last_error(ctx).decode()


def wnw_destroy(ctx):
    _CFG.pop(getattr(ctx, "value", ctx), None)
    lib.wnw_destroy(ctx)


def make_config(batch, layers, q_heads, kv_heads, audio_len, text_len, chunk_len, budget_bp,
                head_dim=128, top_k=0, evict_lag=0, flags=0, max_new_tokens=0) -> wnw_config:
    return wnw_config(batch, layers, q_heads, kv_heads, head_dim, audio_len, text_len, chunk_len, budget_bp,
                      top_k, evict_lag, flags, max_new_tokens)
