"""Thin ctypes binding over libratsparse.so: same names as the C ABI, argument
marshalling only.  torch supplies device memory and the current HIP stream; every step
of the method runs in the library's kernels.  There is no fallback: if the library is
not built, or a call returns an error, this raises."""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libratsparse.so")

RS_F32, RS_BF16 = 0, 1
RS_WS_CTRL_BYTES = 65536
RS_STATIC_SCRATCH_BYTES = 16 << 20

_lib = None
_native = None  # the per-token calls, taken apart in C++ (csrc/native.cpp)


class RatsparseError(RuntimeError):
    pass


class rs_shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("D", ctypes.c_int32), ("Tcap", ctypes.c_int32), ("P", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class rs_pool(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("S", ctypes.c_int32), ("M", ctypes.c_int32), ("P", ctypes.c_int32)]


_vp, _i64, _i32, _f32, _sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float,
                              ctypes.c_size_t)
_shp, _pool = ctypes.POINTER(rs_shape), ctypes.POINTER(rs_pool)

# every symbol include/ratsparse.h declares: name -> (restype, argtypes)
SIGNATURES = {
    "ratsparse_status_string": (ctypes.c_char_p, [_i32]),
    "ratsparse_version": (ctypes.c_char_p, []),
    "ratsparse_workspace_init": (_i32, [_vp, _sz, _vp]),
    "ratsparse_async_status": (_i32, [_vp, _vp]),
    "ratsparse_probe_read": (_i32, [_vp, _sz, _vp, _i32, _vp]),
    "ratsparse_probe_rw": (_i32, [_vp, _vp, _vp, _sz, _i32, _vp]),
    "ratsparse_debug_set_spin_limit": (None, [_i32]),
    "ratsparse_debug_reload_knobs": (None, []),
    "rat_scan_workspace_bytes": (_sz, [_shp, _i64]),
    "rat_scan": (_i32, [_shp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _vp, _sz, _vp]),
    "quest_page_meta": (_i32, [_shp, _vp, _vp, _i64, _i64, _vp]),
    "quest_select_decode_workspace_bytes": (_sz, [_shp, _i64]),
    "quest_select_decode": (_i32, [_shp, _vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _sz, _vp]),
    "quest_select_decode_group": (_i32, [_shp, _vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _sz, _vp]),
    "sparse_attn_decode_group": (_i32, [_shp, _vp, _vp, _vp, _i64, _f32, _vp, _i32, _vp, _i32, _i32, _vp,
                                        _vp, _vp, _vp, _sz, _vp]),
    "sparse_attn_decode_workspace_bytes": (_sz, [_shp, _i64, _i32]),
    "sparse_attn_decode": (_i32, [_shp, _vp, _vp, _vp, _i64, _f32, _vp, _i32, _vp, _i32, _i32, _vp,
                                  _vp, _vp, _vp, _sz, _vp]),
    "sparse_attn_decode_static": (_i32, [_shp, _vp, _vp, _vp, _i64, _f32, _vp, _i32, _vp, _i32, _i32, _vp,
                                         _vp, _vp, _vp, _vp]),
    "rat_decode_step_workspace_bytes": (_sz, [_shp, _i64, _i32]),
    "rat_decode_state_set": (_i32, [_vp, _sz, _i64, _vp]),
    "rat_decode_state_get": (_i32, [_vp, ctypes.POINTER(ctypes.c_int64), _vp]),
    "rat_decode_step": (_i32, [_shp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _f32, _i32, _i32, _i32, _i64,
                               _vp, _vp, _vp, _vp, _sz, _vp]),
    "selection_hit_update": (_i32, [_vp, _i32, _i32, _i32, _vp, _i32, _vp, _vp]),
    "moba_select_prefill_workspace_bytes": (_sz, [_shp, _i64, _i32]),
    "moba_select_prefill": (_i32, [_shp, _vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp, _vp, _sz, _vp]),
    "sparse_attn_prefill_workspace_bytes": (_sz, [_shp, _i64, _i32, _i32]),
    "sparse_attn_prefill": (_i32, [_shp, _vp, _vp, _vp, _i64, _i32, _f32, _vp, _i32, _vp, _vp, _vp,
                                   _sz, _vp]),
    "snapkv_compress_workspace_bytes": (_sz, [_shp, _i64, _i32]),
    "snapkv_compress": (_i32, [_shp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _f32, _vp, _vp, _i64,
                               _vp, _vp, _vp, _sz, _vp]),
    "snapkv_compress_lse": (_i32, [_shp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _i64,
                                   _vp, _vp, _vp, _sz, _vp]),
    "page_pool_workspace_bytes": (_sz, [_pool]),
    "page_pool_reserve": (_i32, [_pool, _vp, _vp, _vp, _vp, _i32, _vp, _i32, _vp, _vp, _sz, _vp]),
    "page_pool_fork": (_i32, [_pool, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _sz, _vp]),
    "page_pool_free": (_i32, [_pool, _vp, _vp, _vp, _vp, _i32, _vp, _sz, _vp]),
    "page_pool_compact": (_i32, [_pool, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "page_pool_share": (_i32, [_pool, _vp, _vp, _vp, _i32, _i32, _vp, _vp]),
    "page_copy": (_i32, [_shp, _vp, _vp, _vp, _shp, _vp, _vp, _vp, _vp, _i32, _vp, _vp]),
    "rat_state_copy": (_i32, [_shp, _vp, _vp, _i32, _vp, _i32, _vp]),
    "rat_append_paged": (_i32, [_shp, _pool, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp]),
    "attn_paged_workspace_bytes": (_sz, [_shp, _pool, _i32]),
    "attn_paged": (_i32, [_shp, _pool, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _f32, _vp, _vp, _vp, _sz, _vp]),
    "kv4_append": (_i32, [_shp, _vp, _vp, _i64, _i64, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "kv4_page_meta": (_i32, [_shp, _vp, _vp, _vp, _vp, _i32, _vp, _vp]),
    "kv4_fetch": (_i32, [_shp, _vp, _vp, _vp, _vp, _vp, _i64, _i32, _vp, _vp, _vp]),
    "kv4_attn_decode_workspace_bytes": (_sz, [_shp, _i32, _i32, _i32]),
    "kv4_attn_decode": (_i32, [_shp, _vp, _vp, _vp, _vp, _vp, _vp, _f32, _vp, _i32, _i32, _vp, _i32, _vp, _vp, _vp, _sz, _vp]),
    "attn_decode_tally_workspace_bytes": (_sz, [_shp]),
    "attn_decode_tally": (_i32, [_shp, _vp, _vp, _vp, _vp, _f32, _vp, _i32, _vp, _vp, _vp, _sz, _vp]),
    "cache_evict_workspace_bytes": (_sz, [_shp, _i32]),
    "cache_evict": (_i32, [_shp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _vp, _sz, _vp]),
    "kv4_evict": (_i32, [_shp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _vp, _sz, _vp]),
}


# those of them that native.cpp takes apart too, in the order in which it is told their addresses
_POOL_CALLS = ("page_pool_reserve", "page_pool_fork", "page_pool_free", "page_pool_compact", "page_pool_share", "page_copy",
               "rat_state_copy", "rat_append_paged", "attn_paged")
_CACHE_CALLS = ("kv4_append", "kv4_page_meta", "kv4_fetch", "kv4_attn_decode", "attn_decode_tally", "cache_evict", "kv4_evict")


def load():
    """Load libratsparse.so; raises if it has not been built (no fallback exists)."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RatsparseError(
                "libratsparse.so is not built: run `python -m paper_2605_28640_amd.build` "
                "(needs hipcc); there is no CPU fallback")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        try:
            from . import _native as native
        except ImportError as e:
            raise RatsparseError("_native.so is not built: run `python -m paper_2605_28640_amd.build`") from e
        native.setup(*(ctypes.cast(getattr(lib, name), _vp).value for name in ("rat_scan", "sparse_attn_decode", "rat_decode_step")),
                     _check, torch._C._cuda_getCurrentRawStream, torch.cuda.current_device, rs_shape, Workspace)
        native.setup_pool(*(ctypes.cast(getattr(lib, name), _vp).value for name in _POOL_CALLS), rs_pool)
        native.setup_cache(*(ctypes.cast(getattr(lib, name), _vp).value for name in _CACHE_CALLS))
        _native = native
        _lib = lib  # last: another thread that finds it set goes on without a look at the rest
    return _lib


def _calls():
    """The per-token calls with plain arguments; each answers False, the call unmade, for any others."""
    if _native is None:
        load()
    return _native


def _check(status):
    if status != 0:
        raise RatsparseError("ratsparse: %s (status %d)" %
                             (load().ratsparse_status_string(status).decode(), status))


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensors only"
    return t.data_ptr()


def _stream():
    # torch.cuda.current_stream().cuda_stream without building the Stream object, which took 2.8 of the 8.6 us
    # that the host spends on a call
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return RS_BF16
    if t.dtype == torch.float32:
        return RS_F32
    raise RatsparseError("storage dtype must be float32 or bfloat16")


def make_shape(B, Hq, Hkv, D, Tcap, P, dtype):
    code = dtype if isinstance(dtype, int) else (RS_BF16 if dtype == torch.bfloat16 else RS_F32)
    return rs_shape(B, Hq, Hkv, D, Tcap, P, code)


def make_pool(N, S, M, P):
    """N pages of P tokens, rows for S sequences of at most M pages."""
    return rs_pool(N, S, M, P)


class Workspace:
    """A device scratch buffer with zeroed control words."""

    def __init__(self, nbytes, device="cuda"):
        nbytes = max(int(nbytes), RS_WS_CTRL_BYTES)
        self.buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
        _check(load().ratsparse_workspace_init(self.buf.data_ptr(), self.buf.numel(), _stream()))

    @property
    def ptr(self):
        return self.buf.data_ptr()

    @property
    def nbytes(self):
        return self.buf.numel()

    def async_status(self):
        _check(load().ratsparse_async_status(self.ptr, _stream()))


def ratsparse_probe_read(src, nbytes, sink, streaming=0):
    _check(load().ratsparse_probe_read(_ptr(src), nbytes, _ptr(sink), streaming, _stream()))


def ratsparse_probe_rw(a, b, dst, nbytes, streaming=0):
    _check(load().ratsparse_probe_rw(_ptr(a), _ptr(b), _ptr(dst), nbytes, streaming, _stream()))


def rat_scan_workspace_bytes(s, T_new):
    return load().rat_scan_workspace_bytes(ctypes.byref(s), T_new)


def rat_scan(s, k, v, g, state_k, state_v, k_cache, v_cache, t0, T_new, ws=None, meta=None):
    if _calls().rat_scan(s, k, v, g, state_k, state_v, k_cache, v_cache, t0, T_new, ws, meta):
        return
    _check(load().rat_scan(ctypes.byref(s), _ptr(k), _ptr(v), _ptr(g), _ptr(state_k), _ptr(state_v),
                           _ptr(k_cache), _ptr(v_cache), _ptr(meta), t0, T_new, ws.ptr if ws else None,
                           ws.nbytes if ws else 0, _stream()))


def quest_page_meta(s, k_cache, meta, t_begin, t_end):
    _check(load().quest_page_meta(ctypes.byref(s), _ptr(k_cache), _ptr(meta), t_begin, t_end, _stream()))


def quest_select_decode_workspace_bytes(s, T_valid):
    return load().quest_select_decode_workspace_bytes(ctypes.byref(s), T_valid)


def quest_select_decode(s, q, meta, T_valid, K, n_first, n_local, idx_out, scores_out, ws):
    _check(load().quest_select_decode(ctypes.byref(s), _ptr(q), _ptr(meta), T_valid, K, n_first, n_local,
                                      _ptr(idx_out), _ptr(scores_out), ws.ptr, ws.nbytes, _stream()))


def quest_select_decode_group(s, q, meta, T_valid, K, n_first, n_local, idx_out, scores_out, ws):
    _check(load().quest_select_decode_group(ctypes.byref(s), _ptr(q), _ptr(meta), T_valid, K, n_first, n_local,
                                            _ptr(idx_out), _ptr(scores_out), ws.ptr, ws.nbytes, _stream()))


def sparse_attn_decode_group(s, q, k_cache, v_cache, T_valid, scale, idx, K, meta, n_first, n_local, out,
                             lse_out, idx_out, ws):
    _check(load().sparse_attn_decode_group(ctypes.byref(s), _ptr(q), _ptr(k_cache), _ptr(v_cache), T_valid,
                                           scale, _ptr(idx), K, _ptr(meta), n_first, n_local, _ptr(out),
                                           _ptr(lse_out), _ptr(idx_out), ws.ptr, ws.nbytes, _stream()))


def rat_decode_step_workspace_bytes(s, T_max, K):
    return load().rat_decode_step_workspace_bytes(ctypes.byref(s), T_max, K)


def rat_decode_state_set(ws, T):
    _check(load().rat_decode_state_set(ws.ptr, ws.nbytes, T, _stream()))


def rat_decode_state_get(ws):
    T = ctypes.c_int64(0)
    _check(load().rat_decode_state_get(ws.ptr, ctypes.byref(T), _stream()))
    return T.value


def rat_decode_step(s, k, v, g, state_k, state_v, k_cache, v_cache, meta, q, scale, K, n_first, n_local, T_max,
                    out, lse_out, idx_out, ws):
    if _calls().rat_decode_step(s, k, v, g, state_k, state_v, k_cache, v_cache, meta, q, scale, K, n_first, n_local, T_max,
                                out, lse_out, idx_out, ws):
        return
    _check(load().rat_decode_step(ctypes.byref(s), _ptr(k), _ptr(v), _ptr(g), _ptr(state_k), _ptr(state_v),
                                  _ptr(k_cache), _ptr(v_cache), _ptr(meta), _ptr(q), scale, K, n_first, n_local,
                                  T_max, _ptr(out), _ptr(lse_out), _ptr(idx_out), ws.ptr, ws.nbytes, _stream()))


def selection_hit_update(idx, gold, unit, hit):
    B, H, K = idx.shape
    assert gold.shape == (B, H) and hit.shape == (B, H) and hit.dtype == torch.uint8
    _check(load().selection_hit_update(_ptr(idx), B, H, K, _ptr(gold), unit, _ptr(hit), _stream()))


def sparse_attn_decode_workspace_bytes(s, T_valid, K):
    return load().sparse_attn_decode_workspace_bytes(ctypes.byref(s), T_valid, K)


def sparse_attn_decode(s, q, k_cache, v_cache, T_valid, scale, idx, K, meta, n_first, n_local, out,
                       lse_out, idx_out, ws):
    if _calls().sparse_attn_decode(s, q, k_cache, v_cache, T_valid, scale, idx, K, meta, n_first, n_local, out, lse_out,
                                   idx_out, ws):
        return
    _check(load().sparse_attn_decode(ctypes.byref(s), _ptr(q), _ptr(k_cache), _ptr(v_cache), T_valid,
                                     scale, _ptr(idx), K, _ptr(meta), n_first, n_local, _ptr(out),
                                     _ptr(lse_out), _ptr(idx_out), ws.ptr, ws.nbytes, _stream()))


def sparse_attn_decode_static(s, q, k_cache, v_cache, T_valid, scale, idx, K, meta, n_first, n_local, out,
                              lse_out, idx_out, async_err):
    _check(load().sparse_attn_decode_static(ctypes.byref(s), _ptr(q), _ptr(k_cache), _ptr(v_cache), T_valid,
                                            scale, _ptr(idx), K, _ptr(meta), n_first, n_local, _ptr(out),
                                            _ptr(lse_out), _ptr(idx_out), _ptr(async_err), _stream()))


def moba_select_prefill_workspace_bytes(s, T, block):
    return load().moba_select_prefill_workspace_bytes(ctypes.byref(s), T, block)


def moba_select_prefill(s, q, k_cache, T, block, K, n_first, means_out, idx_out, ws):
    _check(load().moba_select_prefill(ctypes.byref(s), _ptr(q), _ptr(k_cache), T, block, K, n_first,
                                      _ptr(means_out), _ptr(idx_out), ws.ptr, ws.nbytes, _stream()))


def sparse_attn_prefill_workspace_bytes(s, T, block, K):
    return load().sparse_attn_prefill_workspace_bytes(ctypes.byref(s), T, block, K)


def sparse_attn_prefill(s, q, k_cache, v_cache, T, block, scale, idx, K, out, lse_out, ws):
    _check(load().sparse_attn_prefill(ctypes.byref(s), _ptr(q), _ptr(k_cache), _ptr(v_cache), T, block,
                                      scale, _ptr(idx), K, _ptr(out), _ptr(lse_out), ws.ptr, ws.nbytes,
                                      _stream()))


def snapkv_compress_workspace_bytes(s, T, W):
    return load().snapkv_compress_workspace_bytes(ctypes.byref(s), T, W)


def snapkv_compress(s, q_win, k_cache, v_cache, T, W, K_keep, pool_kernel, scale, kc_out, vc_out,
                    Tcap_out, idx_out, votes_out, ws):
    _check(load().snapkv_compress(ctypes.byref(s), _ptr(q_win), _ptr(k_cache), _ptr(v_cache), T, W,
                                  K_keep, pool_kernel, scale, _ptr(kc_out), _ptr(vc_out), Tcap_out,
                                  _ptr(idx_out), _ptr(votes_out), ws.ptr, ws.nbytes, _stream()))


def snapkv_compress_lse(s, q_win, k_cache, v_cache, T, W, K_keep, pool_kernel, scale, lse_win, kc_out, vc_out,
                        Tcap_out, idx_out, votes_out, ws):
    _check(load().snapkv_compress_lse(ctypes.byref(s), _ptr(q_win), _ptr(k_cache), _ptr(v_cache), T, W,
                                      K_keep, pool_kernel, scale, _ptr(lse_win), _ptr(kc_out), _ptr(vc_out),
                                      Tcap_out, _ptr(idx_out), _ptr(votes_out), ws.ptr, ws.nbytes, _stream()))


# ---- sequences in a pool of pages: the tensors' shapes and types are looked at here, since the kernels go by them ----


def _need(t, dtype, *shape):
    """The address of a device tensor of this type and shape on the current device; None: null."""
    if t is None:
        return None
    if t.dtype != dtype or tuple(t.shape) != shape:
        raise RatsparseError("a %s tensor of shape %s is needed, not %s %s" % (dtype, shape, t.dtype, tuple(t.shape)))
    p = _ptr(t)
    if t.get_device() != torch.cuda.current_device():
        raise RatsparseError("the tensors have to be on the current device")
    return p


def _scratch(ws):
    """Address and size of a workspace; one that shows its buffer has to have it on the current device."""
    buf = getattr(ws, "buf", None)
    if buf is not None:
        _ptr(buf)
        if buf.get_device() != torch.cuda.current_device():
            raise RatsparseError("the workspace has to be on the current device")
    return ws.ptr, ws.nbytes


def _sequences(p, table, len, refs):
    return (_need(table, torch.int32, p.S, p.M), _need(len, torch.int32, p.S), _need(refs, torch.int32, p.N))


def _rows(s, k, v, meta):
    """Addresses of a pool's (or one batch entry's) rows and bounds."""
    dt = torch.bfloat16 if s.dtype == RS_BF16 else torch.float32
    return (_need(k, dt, s.Hkv, s.Tcap, s.D), _need(v, dt, s.Hkv, s.Tcap, s.D), _need(meta, dt, s.Hkv, s.Tcap // s.P, 2, s.D))


def page_pool_workspace_bytes(p):
    return load().page_pool_workspace_bytes(ctypes.byref(p))


def page_pool_reserve(p, table, len, refs, seq, want, T_new, granted, ws):
    if _calls().page_pool_reserve(p, table, len, refs, seq, want, T_new, granted, ws):
        return
    n = seq.numel()
    _check(load().page_pool_reserve(ctypes.byref(p), *_sequences(p, table, len, refs), _need(seq, torch.int32, n), n,
                                    _need(want, torch.int32, n), T_new, _need(granted, torch.int32, n), *_scratch(ws),
                                    _stream()))


def page_pool_fork(p, table, len, refs, src, dst, pairs_out, carry_out, ws):
    if _calls().page_pool_fork(p, table, len, refs, src, dst, pairs_out, carry_out, ws):
        return
    n = src.numel()
    _check(load().page_pool_fork(ctypes.byref(p), *_sequences(p, table, len, refs), _need(src, torch.int32, n),
                                 _need(dst, torch.int32, n), n, _need(pairs_out, torch.int32, n, 2),
                                 _need(carry_out, torch.int32, n, 2), *_scratch(ws), _stream()))


def page_pool_free(p, table, len, refs, seq, ws):
    if _calls().page_pool_free(p, table, len, refs, seq, ws):
        return
    n = seq.numel()
    _check(load().page_pool_free(ctypes.byref(p), *_sequences(p, table, len, refs), _need(seq, torch.int32, n), n, *_scratch(ws), _stream()))


def page_pool_compact(p, table, len, refs, pairs_out, n_pairs_out, ws):
    if _calls().page_pool_compact(p, table, len, refs, pairs_out, n_pairs_out, ws):
        return
    _check(load().page_pool_compact(ctypes.byref(p), *_sequences(p, table, len, refs),
                                    _need(pairs_out, torch.int32, max(p.N // 2, 1), 2), _need(n_pairs_out, torch.int32, 1),
                                    *_scratch(ws), _stream()))


def page_pool_share(p, table, len, seq, min_pages, share_out):
    if _calls().page_pool_share(p, table, len, seq, min_pages, share_out):
        return
    n = seq.numel()
    _check(load().page_pool_share(ctypes.byref(p), _need(table, torch.int32, p.S, p.M), _need(len, torch.int32, p.S),
                                  _need(seq, torch.int32, n), n, min_pages, _need(share_out, torch.int32, n, 3), _stream()))


def page_copy(s_src, k_src, v_src, meta_src, s_dst, k_dst, v_dst, meta_dst, pairs, n_pairs):
    if _calls().page_copy(s_src, k_src, v_src, meta_src, s_dst, k_dst, v_dst, meta_dst, pairs, n_pairs):
        return
    n = pairs.shape[0]
    _check(load().page_copy(ctypes.byref(s_src), *_rows(s_src, k_src, v_src, meta_src), ctypes.byref(s_dst),
                            *_rows(s_dst, k_dst, v_dst, meta_dst), _need(pairs, torch.int32, n, 2), n,
                            _need(n_pairs, torch.int32, 1), _stream()))


def rat_state_copy(s, state_k, state_v, pairs):
    if _calls().rat_state_copy(s, state_k, state_v, pairs):
        return
    S, n = state_k.shape[0], pairs.shape[0]
    _check(load().rat_state_copy(ctypes.byref(s), _need(state_k, torch.float32, S, s.Hkv, s.D),
                                 _need(state_v, torch.float32, S, s.Hkv, s.D), S, _need(pairs, torch.int32, n, 2), n, _stream()))


def rat_append_paged(s, p, k, v, g, state_k, state_v, k_pool, v_pool, meta, table, len, seq, n_new, T_new):
    if _calls().rat_append_paged(s, p, k, v, g, state_k, state_v, k_pool, v_pool, meta, table, len, seq, n_new,
                                 T_new):
        return
    dt, new, carry = k.dtype, (s.B, s.Hkv, T_new, s.D), (p.S, s.Hkv, s.D)
    if _dtype_code(k) != s.dtype:
        raise RatsparseError("k is not of the shape's type")
    kp, vp, mp = _rows(s, k_pool, v_pool, meta)
    _check(load().rat_append_paged(ctypes.byref(s), ctypes.byref(p), _need(k, dt, *new), _need(v, dt, *new),
                                   _need(g, torch.float32, *new), _need(state_k, torch.float32, *carry),
                                   _need(state_v, torch.float32, *carry), kp, vp, mp, _need(table, torch.int32, p.S, p.M),
                                   _need(len, torch.int32, p.S), _need(seq, torch.int32, s.B), _need(n_new, torch.int32, s.B),
                                   T_new, _stream()))


def attn_paged_workspace_bytes(s, p, T_new):
    return load().attn_paged_workspace_bytes(ctypes.byref(s), ctypes.byref(p), T_new)


def attn_paged(s, p, q, k_pool, v_pool, table, len, seq, n_new, T_new, share, scale, out, lse_out, ws):
    if _calls().attn_paged(s, p, q, k_pool, v_pool, table, len, seq, n_new, T_new, share, scale, out, lse_out, ws):
        return
    dt, rows = q.dtype, (s.B, s.Hq, T_new)
    if _dtype_code(q) != s.dtype:
        raise RatsparseError("q is not of the shape's type")
    kp, vp, _ = _rows(s, k_pool, v_pool, None)
    _check(load().attn_paged(ctypes.byref(s), ctypes.byref(p), _need(q, dt, *rows, s.D), kp, vp, _need(table, torch.int32, p.S, p.M),
                             _need(len, torch.int32, p.S), _need(seq, torch.int32, s.B), _need(n_new, torch.int32, s.B), T_new,
                             _need(share, torch.int32, s.B, 3), scale, _need(out, dt, *rows, s.D),
                             _need(lse_out, torch.float32, *rows), *_scratch(ws), _stream()))


# ---- a cache in 4 bits, and caches that give up rows: sequences of lengths of their own, in device memory ----


def _four(s, k4, k4_scale, v4, v4_scale):
    rows = (s.B, s.Hkv, s.Tcap)
    return (_need(k4, torch.uint8, *rows, s.D // 2), _need(k4_scale, torch.uint8, *rows, s.D // 32), _need(v4, torch.uint8, *rows, s.D // 2),
            _need(v4_scale, torch.uint8, *rows, s.D // 32))


def _type(s):
    return torch.bfloat16 if s.dtype == RS_BF16 else torch.float32


def _bounds(s, meta):
    return _need(meta, _type(s), s.B, s.Hkv, s.Tcap // s.P if s.P > 0 else 0, 2, s.D)


def kv4_append(s, k, v, t_src, len, n_new, T_new, k4, k4_scale, v4, v4_scale, meta):
    """k, v [B, Hkv, T_src, D]: the new tokens are rows t_src .. t_src + T_new - 1."""
    if _calls().kv4_append(s, k, v, t_src, len, n_new, T_new, k4, k4_scale, v4, v4_scale, meta):
        return
    if meta is not None and meta.numel() == 0:  # its address is null: not to be taken for no bounds
        raise RatsparseError("bounds of no pages")
    T_src = k.shape[2] if k.dim() == 4 else 0
    src = (_type(s), s.B, s.Hkv, T_src, s.D)
    _check(load().kv4_append(ctypes.byref(s), _need(k, *src), _need(v, *src), T_src, t_src, _need(len, torch.int32, s.B), _need(n_new, torch.int32, s.B),
                             T_new, *_four(s, k4, k4_scale, v4, v4_scale), _bounds(s, meta), _stream()))


def kv4_page_meta(s, k4, k4_scale, len, n_new, T_new, meta):
    if _calls().kv4_page_meta(s, k4, k4_scale, len, n_new, T_new, meta):
        return
    kc, ks, _, _ = _four(s, k4, k4_scale, None, None)
    _check(load().kv4_page_meta(ctypes.byref(s), kc, ks, _need(len, torch.int32, s.B), _need(n_new, torch.int32, s.B), T_new, _bounds(s, meta),
                                _stream()))


def kv4_fetch(s, k4, k4_scale, v4, v4_scale, len, t0, T, k_out, v_out):
    if _calls().kv4_fetch(s, k4, k4_scale, v4, v4_scale, len, t0, T, k_out, v_out):
        return
    to = (_type(s), s.B, s.Hkv, T, s.D)
    _check(load().kv4_fetch(ctypes.byref(s), *_four(s, k4, k4_scale, v4, v4_scale), _need(len, torch.int32, s.B), t0, T, _need(k_out, *to),
                            _need(v_out, *to), _stream()))


def kv4_attn_decode_workspace_bytes(s, H_idx, K, with_tally):
    return load().kv4_attn_decode_workspace_bytes(ctypes.byref(s), H_idx, K, bool(with_tally))


def kv4_attn_decode(s, q, k4, k4_scale, v4, v4_scale, len, scale, idx, tally, n_fresh, out, lse_out, ws):
    """idx: [B, Hq or Hkv, K] pages or None."""
    if _calls().kv4_attn_decode(s, q, k4, k4_scale, v4, v4_scale, len, scale, idx, tally, n_fresh, out, lse_out, ws):
        return
    if idx is not None and idx.numel() == 0:  # its address is null: not to be taken for no list
        raise RatsparseError("a list of no pages")
    H, K = (idx.shape[1], idx.shape[2]) if idx is not None and idx.dim() == 3 else (0, 0)
    rows = (s.B, s.Hq)
    _check(load().kv4_attn_decode(ctypes.byref(s), _need(q, _type(s), *rows, s.D), *_four(s, k4, k4_scale, v4, v4_scale), _need(len, torch.int32, s.B),
                                  scale, _need(idx, torch.int32, s.B, H, K), H, K, _need(tally, torch.float32, s.B, s.Hkv, s.Tcap), n_fresh,
                                  _need(out, _type(s), *rows, s.D), _need(lse_out, torch.float32, *rows), *_scratch(ws), _stream()))


def attn_decode_tally_workspace_bytes(s):
    return load().attn_decode_tally_workspace_bytes(ctypes.byref(s))


def attn_decode_tally(s, q, k_cache, v_cache, len, scale, tally, n_fresh, out, lse_out, ws):
    if _calls().attn_decode_tally(s, q, k_cache, v_cache, len, scale, tally, n_fresh, out, lse_out, ws):
        return
    dt, rows, cache = _type(s), (s.B, s.Hq), (s.B, s.Hkv, s.Tcap)
    _check(load().attn_decode_tally(ctypes.byref(s), _need(q, dt, *rows, s.D), _need(k_cache, dt, *cache, s.D), _need(v_cache, dt, *cache, s.D),
                                    _need(len, torch.int32, s.B), scale, _need(tally, torch.float32, *cache), n_fresh, _need(out, dt, *rows, s.D),
                                    _need(lse_out, torch.float32, *rows), *_scratch(ws), _stream()))


def cache_evict_workspace_bytes(s, n_keep):
    return load().cache_evict_workspace_bytes(ctypes.byref(s), n_keep)


def _kept(s, tally, pos, mark, len):
    cache = (s.B, s.Hkv, s.Tcap)
    return (_need(tally, torch.float32, *cache), _need(pos, torch.int32, *cache), _need(mark, torch.int32, s.B, 2), _need(len, torch.int32, s.B))


def cache_evict(s, k_cache, v_cache, tally, pos, mark, len, n_keep, n_first, n_recent, n_slack, ws):
    if _calls().cache_evict(s, k_cache, v_cache, tally, pos, mark, len, n_keep, n_first, n_recent, n_slack, ws):
        return
    rows = (_type(s), s.B, s.Hkv, s.Tcap, s.D)
    _check(load().cache_evict(ctypes.byref(s), _need(k_cache, *rows), _need(v_cache, *rows), *_kept(s, tally, pos, mark, len), n_keep, n_first, n_recent,
                              n_slack, *_scratch(ws), _stream()))


def kv4_evict(s, k4, k4_scale, v4, v4_scale, tally, pos, mark, len, n_keep, n_first, n_recent, n_slack, ws):
    if _calls().kv4_evict(s, k4, k4_scale, v4, v4_scale, tally, pos, mark, len, n_keep, n_first, n_recent, n_slack, ws):
        return
    _check(load().kv4_evict(ctypes.byref(s), *_four(s, k4, k4_scale, v4, v4_scale), *_kept(s, tally, pos, mark, len), n_keep, n_first, n_recent, n_slack,
                            *_scratch(ws), _stream()))
