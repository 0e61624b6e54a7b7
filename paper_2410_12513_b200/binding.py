"""ctypes binding of ``libfirst.so``: the same calls as ``include/first.h``, taking torch
CUDA tensors.  Argument marshalling only -- no arithmetic happens here."""
from __future__ import annotations

import contextlib
import ctypes as C
import functools
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
_LIBPATH = _PKG / "libfirst.so"
_lib = None

FIRST_DTYPE_F32, FIRST_DTYPE_BF16 = 0, 1
MEAN_OF_SIGMOID, SIGMOID_OF_MEAN = 0, 1
FLAG_KV_FULL, FLAG_BAD_TOKEN, FLAG_BAD_MASK, FLAG_WAIT_EXPIRED, FLAG_EMPTY_SEQ, FLAG_BAD_SEQ_TABLE, FLAG_BAD_PAGE = 1, 2, 4, 8, 16, 32, 64
CACHE_INT8, CACHE_E4M3 = 0, 1


class FirstError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        msg = lib().first_status_string(status).decode()
        super().__init__(f"{what}: status {status} ({msg})")


class ModelDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "ffn_dim",
                                         "vocab")] + \
               [("rope_base", C.c_float), ("rms_eps", C.c_float), ("dtype", C.c_int32), ("max_batch", C.c_int32),
                ("max_tokens_per_seq", C.c_int32)]


class Weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p),
                ("attn_norm", C.POINTER(C.c_void_p)), ("wqkv", C.POINTER(C.c_void_p)),
                ("wo", C.POINTER(C.c_void_p)), ("ffn_norm", C.POINTER(C.c_void_p)),
                ("w_gate_up", C.POINTER(C.c_void_p)), ("w_down", C.POINTER(C.c_void_p))]


class KVCacheC(C.Structure):
    _fields_ = [("k", C.POINTER(C.c_void_p)), ("v", C.POINTER(C.c_void_p)), ("slab_off", C.c_void_p),
                ("slab_cap", C.c_void_p), ("len", C.c_void_p), ("pos", C.c_void_p), ("cap_total", C.c_int64),
                ("per_layer", C.c_int32), ("cap_total_l", C.POINTER(C.c_int64))]


class SamplingC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("temperature", "top_k", "top_p", "min_p", "uniforms")]


class AdaptersC(C.Structure):
    _fields_ = [("n_adapters", C.c_int32), ("rank", C.c_int32), ("scales", C.c_void_p), ("seq_adapter", C.c_void_p)] + \
               [(f"{t}_{m}", C.POINTER(C.c_void_p)) for t in ("qkv", "o", "gate_up", "down") for m in ("a", "b")]


class Cache8C(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("format", "n_pages", "n_kv_heads", "page", "head_dim")] + \
               [(n, C.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


class RopeSpecC(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("scaling", C.c_int32), ("base", C.c_double), ("factor", C.c_double),
                ("low", C.c_double), ("high", C.c_double), ("trained_len", C.c_int64)]


def library_path() -> Path:
    return _LIBPATH


def lib():
    """Load the CUDA library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not _LIBPATH.exists():
            raise FileNotFoundError(f"{_LIBPATH} is missing: build it with `python -m paper_2410_12513_b200.build`")
        L = C.CDLL(str(_LIBPATH))
        L.first_status_string.restype = C.c_char_p
        L.first_status_string.argtypes = [C.c_int]
        L.first_create.argtypes = [C.POINTER(ModelDesc), C.POINTER(Weights), C.POINTER(C.c_void_p)]
        L.first_destroy.argtypes = [C.c_void_p]
        L.first_prefill_route.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32,
                                          C.c_int64, C.c_void_p, C.c_void_p, C.c_float, C.c_int32, C.c_void_p,
                                          C.c_void_p, C.c_void_p]
        L.first_prefill_route_static.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p,
                                                 C.c_int32, C.c_int64, C.c_void_p, C.c_void_p, C.c_float, C.c_int32,
                                                 C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.first_prefill_route_static.restype = C.c_int
        L.first_prefill.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(KVCacheC), C.c_void_p,
                                    C.c_void_p, C.c_float, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p]
        L.first_prefill.restype = C.c_int
        L.first_set_mask.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.first_get_plan.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.first_decode_step.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(KVCacheC), C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_void_p]
        L.first_last_device_flags.argtypes = [C.c_void_p, C.POINTER(C.c_uint32), C.c_void_p]
        L.first_launch_count.restype = C.c_int64
        L.first_launch_count.argtypes = [C.c_void_p]
        L.first_set_option.argtypes = [C.c_void_p, C.c_char_p, C.c_int64]
        L.first_set_sampling.argtypes = [C.c_void_p, C.c_int32, C.c_float, C.c_void_p]
        L.first_set_sampling.restype = C.c_int
        L.first_sample_topk.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_void_p,
                                        C.c_void_p]
        L.first_sample_topk.restype = C.c_int
        L.first_profile.argtypes = [C.c_void_p, C.c_int32]
        L.first_profile.restype = C.c_int
        L.first_profile_read.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.first_profile_read.restype = C.c_int
        L.first_set_mask_host.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.first_set_mask_host.restype = C.c_int
        L.first_pool_create.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                        C.POINTER(C.c_void_p)]
        L.first_pool_destroy.argtypes = [C.c_void_p]
        L.first_seq_join.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(KVCacheC), C.c_int32, C.c_int32,
                                     C.POINTER(C.c_int32), C.c_void_p]
        L.first_seq_leave.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
        L.first_pool_commit.argtypes = [C.c_void_p, C.c_void_p]
        L.first_pool_kv.argtypes = [C.c_void_p, C.POINTER(KVCacheC)]
        L.first_pool_stats.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(C.c_int32)]
        for name in ("first_pool_create", "first_pool_destroy", "first_seq_join", "first_seq_leave", "first_pool_commit",
                     "first_pool_kv", "first_pool_stats"):
            getattr(L, name).restype = C.c_int
        L.first_graph_count.argtypes = [C.c_void_p]
        L.first_graph_count.restype = C.c_int64
        L.first_selftest_wait_expiry.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.first_selftest_wait_expiry.restype = C.c_int
        L.first_step_trace.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.first_step_trace.restype = C.c_int
        p, i32, i64, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_double
        L.first_sample.argtypes = [p, i64, i32, i32, p, p, p, p, p, p, p]
        L.first_set_sampling_rows.argtypes = [p, C.POINTER(SamplingC)]
        L.first_lora.argtypes = [p, i32, i64, p, p, i32, p, p, i32, i32, i32, p, i32, i32, i32, p, i32, i64, p]
        L.first_set_adapters.argtypes = [p, C.POINTER(AdaptersC)]
        L.first_rope_freqs.argtypes = [C.POINTER(RopeSpecC), p, p]
        L.first_rope.argtypes = [p, i64, i64, i32, p, i64, i64, i32, i32, i64, i32, i32, p, p, C.c_float, i32, p]
        L.first_set_rope.argtypes = [p, p, f64]
        cache8, pi32 = C.POINTER(Cache8C), C.POINTER(C.c_int32)
        L.first_pages_create.argtypes = [p, i32, i32, cache8, C.POINTER(C.c_void_p)]
        L.first_pages_destroy.argtypes = [p]
        L.first_pages_join.argtypes = [p, p, C.POINTER(KVCacheC), i32, i32, pi32]
        L.first_pages_fork.argtypes = [p, i32, pi32]
        L.first_pages_extend.argtypes = [p, i32, i32]
        L.first_pages_trim.argtypes = [p, i32, i32]
        L.first_pages_leave.argtypes = [p, i32]
        L.first_pages_commit.argtypes = [p, p]
        L.first_pages_compact.argtypes = [p, p]
        L.first_pages_kv.argtypes = [p, C.POINTER(KVCacheC)]
        L.first_pages_layer.argtypes = [p, i32, cache8, C.POINTER(C.c_void_p), pi32, C.POINTER(C.c_void_p)]
        L.first_pages_stats.argtypes = [p, p, p, pi32]
        L.first_pages_tokens.argtypes = [p, i32, pi32]
        L.first_set_pages.argtypes = [p, p]
        L.first_append8.argtypes = [cache8, p, i64, i64, p, i64, i64, i32, p, i32, p, i32, p, i32, i32, p, p]
        L.first_read8.argtypes = [cache8, p, i32, p, p, i32, i32, i32, p, i64, i64, p, i64, i64, i32, p, p]
        L.first_attn8.argtypes = [cache8, p, i64, i64, i32, i32, C.c_float, p, i32, p, i32, p, i32, i32, p, i64, i64, p, i64, p, p]
        L.first_attn8_workspace.argtypes = [cache8, i32, i32, i32, i32, i32, i32]
        L.first_attn8_workspace.restype = i64
        L.first_copy_pages.argtypes = [p, i32, p, i64, p, p]
        L.first_verify.argtypes = [p, i64, i64, p, i64, i64, i32, p, i32, i32, i32, p, p, p, p, p, p]
        for name in ("first_pages_create", "first_pages_destroy", "first_pages_join", "first_pages_fork", "first_pages_extend",
                     "first_pages_trim", "first_pages_leave", "first_pages_commit", "first_pages_compact", "first_pages_kv",
                     "first_pages_layer", "first_pages_stats", "first_pages_tokens", "first_set_pages",
                     "first_append8", "first_read8", "first_attn8", "first_copy_pages", "first_verify", "first_sample", "first_set_sampling_rows", "first_lora", "first_set_adapters", "first_rope_freqs",
                     "first_rope", "first_set_rope"):
            getattr(L, name).restype = C.c_int
        L.first_kernel_class_count.restype = C.c_int32
        L.first_kernel_class_name.restype = C.c_char_p
        L.first_kernel_class_name.argtypes = [C.c_int32]
        for name in ("first_create", "first_destroy", "first_prefill_route", "first_set_mask", "first_get_plan",
                     "first_decode_step", "first_last_device_flags", "first_set_option"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _dev(t, dtype=None, what="tensor"):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what} must have dtype {dtype}, got {t.dtype}")
    return C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _ptr_array(tensors, dtype, what):
    arr = (C.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = None if t is None else _dev(t, dtype, f"{what}[{i}]").value
    return arr


class KVCache:
    """Marshals caller-owned cache tensors into ``first_kv_cache``.

    k, v: lists (one per layer) of CUDA tensors [Hkv][cap_total][hd] (None allowed for
    layers no sequence keeps); slab_off int64 [B]; slab_cap int32 [B]; len int32 [L][B];
    pos int32 [B].  With two-dimensional slab_off / slab_cap ([L][B]) the tables are per
    layer and every layer's tensors may have their own height (a layer then holds slabs
    only for the sequences that keep it)."""

    def __init__(self, k, v, slab_off, slab_cap, len_, pos):
        self.k, self.v, self.slab_off, self.slab_cap, self.len, self.pos = k, v, slab_off, slab_cap, len_, pos
        first = next(t for t in k if t is not None)
        self._ka = _ptr_array(k, first.dtype, "kv.k")
        self._va = _ptr_array(v, first.dtype, "kv.v")
        per_layer = slab_off.dim() == 2
        if per_layer != (slab_cap.dim() == 2):
            raise ValueError("slab_off and slab_cap must both be [B] or both be [L][B]")
        self._heights = (C.c_int64 * len(k))(*[0 if t is None else int(t.shape[1]) for t in k])
        self.c = KVCacheC(C.cast(self._ka, C.POINTER(C.c_void_p)), C.cast(self._va, C.POINTER(C.c_void_p)),
                          _dev(slab_off, torch.int64, "slab_off"), _dev(slab_cap, torch.int32, "slab_cap"),
                          _dev(len_, torch.int32, "len"), _dev(pos, torch.int32, "pos"),
                          0 if per_layer else int(first.shape[1]), int(per_layer),
                          C.cast(self._heights, C.POINTER(C.c_int64)))


def first_create(shape, dtype, max_batch, max_tokens_per_seq, weights):
    """weights: dict with embed, lm_head, final_norm and per-layer lists attn_norm, wqkv, wo,
    ffn_norm, w_gate_up, w_down (CUDA tensors).  Returns (handle, keepalive)."""
    wd = torch.float32 if dtype == FIRST_DTYPE_F32 else torch.bfloat16
    desc = ModelDesc(shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                     shape.ffn_dim, shape.vocab, float(shape.rope_base), float(shape.rms_eps), dtype,
                     int(max_batch), int(max_tokens_per_seq))
    arrs = {k: _ptr_array(weights[k], torch.float32 if k.endswith("norm") else wd, k)
            for k in ("attn_norm", "wqkv", "wo", "ffn_norm", "w_gate_up", "w_down")}
    w = Weights(_dev(weights["embed"], wd, "embed"), _dev(weights["lm_head"], wd, "lm_head"),
                _dev(weights["final_norm"], torch.float32, "final_norm"),
                *[C.cast(arrs[k], C.POINTER(C.c_void_p)) for k in
                  ("attn_norm", "wqkv", "wo", "ffn_norm", "w_gate_up", "w_down")])
    h = C.c_void_p()
    rc = lib().first_create(C.byref(desc), C.byref(w), C.byref(h))
    if rc:
        raise FirstError(rc, "first_create")
    return h, (weights, arrs)


def first_destroy(h):
    lib().first_destroy(h)


def first_prefill_route(h, layer, hidden, cu_seqlens, router_w, router_b, tau, mode, mask, scores=None,
                        stream=None):
    if hidden.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("hidden must be float32 or bfloat16")
    hd = FIRST_DTYPE_F32 if hidden.dtype == torch.float32 else FIRST_DTYPE_BF16
    rc = lib().first_prefill_route(h, layer, _dev(hidden, None, "hidden"), hd,
                                   _dev(cu_seqlens, torch.int32, "cu_seqlens"), cu_seqlens.numel() - 1,
                                   hidden.shape[0], _dev(router_w, torch.float32, "router_w"),
                                   _dev(router_b, torch.float32, "router_b"), float(tau), int(mode),
                                   _dev(mask, torch.uint8, "mask"), _dev(scores, torch.float32, "scores"),
                                   _stream(stream))
    if rc:
        raise FirstError(rc, "first_prefill_route")


def first_prefill_route_static(layer, n_layers, hidden, cu_seqlens, router_w, router_b, tau, mode, mask,
                               scores=None, flags=None, stream=None):
    """Context-free router call that allocates nothing (built-in scratch of
    FIRST_STATIC_ROUTE_MAX_TOKENS token scores); see first.h for the limits."""
    if hidden.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("hidden must be float32 or bfloat16")
    hd = FIRST_DTYPE_F32 if hidden.dtype == torch.float32 else FIRST_DTYPE_BF16
    rc = lib().first_prefill_route_static(int(layer), int(n_layers), hidden.shape[1], _dev(hidden, None, "hidden"), hd,
                                          _dev(cu_seqlens, torch.int32, "cu_seqlens"), cu_seqlens.numel() - 1,
                                          hidden.shape[0], _dev(router_w, torch.float32, "router_w"),
                                          _dev(router_b, torch.float32, "router_b"), float(tau), int(mode),
                                          _dev(mask, torch.uint8, "mask"), _dev(scores, torch.float32, "scores"),
                                          _dev(flags, torch.int32, "flags"), _stream(stream))
    if rc:
        raise FirstError(rc, "first_prefill_route_static")


def first_prefill(h, tokens, cu_seqlens, kv: KVCache, router_w=None, router_b=None, tau=0.5, mode=0, mask=None,
                  scores=None, logits=None, next_tokens=None, stream=None):
    """Whole prompt phase of a ragged batch; cu_seqlens is a HOST int32 array (numpy or a CPU tensor)."""
    import numpy as np
    cu = np.ascontiguousarray(np.asarray(cu_seqlens), dtype=np.int32)
    rc = lib().first_prefill(h, _dev(tokens, torch.int32, "tokens"), cu.ctypes.data, cu.size - 1, C.byref(kv.c),
                             _dev(router_w, torch.float32, "router_w"), _dev(router_b, torch.float32, "router_b"),
                             float(tau), int(mode), _dev(mask, torch.uint8, "mask"),
                             _dev(scores, torch.float32, "scores"), _dev(logits, torch.float32, "logits"),
                             _dev(next_tokens, torch.int32, "next_tokens"), _stream(stream))
    if rc:
        raise FirstError(rc, "first_prefill")


def first_set_mask(h, mask, stream=None):
    rc = lib().first_set_mask(h, _dev(mask, torch.uint8, "mask"), mask.shape[0], _stream(stream))
    if rc:
        raise FirstError(rc, "first_set_mask")


def first_set_mask_host(h, mask, stream=None):
    """mask: HOST uint8 [B][L] (numpy or CPU tensor); no wait for the stream."""
    import numpy as np
    m = np.ascontiguousarray(np.asarray(mask), dtype=np.uint8)
    rc = lib().first_set_mask_host(h, m.ctypes.data, m.shape[0], _stream(stream))
    if rc:
        raise FirstError(rc, "first_set_mask_host")


class _PoolKV:
    """The pool's cache view (a first_kv_cache with per-layer tables that live in the pool)."""

    def __init__(self, c):
        self.c = c


class FirstPool:
    """Slab pool over caller-owned per-layer cache tensors for batches that change between steps
    (first_pool_* / first_seq_* in first.h).  k, v: lists of CUDA tensors [Hkv][rows_l][hd]."""

    def __init__(self, ctx, max_seqs, k, v):
        import numpy as np
        self._k, self._v, self._ctx = k, v, ctx
        self.L, self.B = len(k), int(max_seqs)
        rows = np.array([0 if t is None else int(t.shape[1]) for t in k], dtype=np.int64)
        first = next(t for t in k if t is not None)
        ka, va = _ptr_array(k, first.dtype, "pool.k"), _ptr_array(v, first.dtype, "pool.v")
        self.h = C.c_void_p()
        rc = lib().first_pool_create(ctx.h, self.B, rows.ctypes.data, C.cast(ka, C.POINTER(C.c_void_p)),
                                     C.cast(va, C.POINTER(C.c_void_p)), C.byref(self.h))
        if rc:
            raise FirstError(rc, "first_pool_create")
        c = KVCacheC()
        rc = lib().first_pool_kv(self.h, C.byref(c))
        if rc:
            raise FirstError(rc, "first_pool_kv")
        self.kv = _PoolKV(c)

    def close(self):
        if self.h:
            lib().first_pool_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def join(self, mask_row, capacity, src=None, src_seq=0, n_tokens=0, stream=None):
        import numpy as np
        m = np.ascontiguousarray(np.asarray(mask_row), dtype=np.uint8)
        slot = C.c_int32(-1)
        rc = lib().first_seq_join(self.h, m.ctypes.data, int(capacity), C.byref(src.c) if src is not None else None,
                                  int(src_seq), int(n_tokens), C.byref(slot), _stream(stream))
        if rc:
            raise FirstError(rc, "first_seq_join")
        return slot.value

    def leave(self, slot, stream=None):
        rc = lib().first_seq_leave(self.h, int(slot), _stream(stream))
        if rc:
            raise FirstError(rc, "first_seq_leave")

    def commit(self, stream=None):
        rc = lib().first_pool_commit(self.h, _stream(stream))
        if rc:
            raise FirstError(rc, "first_pool_commit")
        self._ctx.B = self.B

    def stats(self):
        import numpy as np
        held = np.zeros(self.L, dtype=np.int64)
        big = np.zeros(self.L, dtype=np.int64)
        live = C.c_int32(0)
        rc = lib().first_pool_stats(self.h, held.ctypes.data, big.ctypes.data, C.byref(live))
        if rc:
            raise FirstError(rc, "first_pool_stats")
        return held, big, live.value


class FirstPages:
    """Pages of the layers' 8-bit caches (a list of Cache8, borrowed) handed out to sequences (first_pages_* in first.h)."""

    def __init__(self, ctx, max_seqs, max_pages, caches):
        self._ctx, self.caches = ctx, list(caches)
        self.B, self.L, self.max_pages, self.h = int(max_seqs), len(self.caches), int(max_pages), None
        self._sources = []  # caches that the next commit imports from
        if self.L != ctx.shape.n_layers:
            raise ValueError(f"one cache a layer: {ctx.shape.n_layers}")
        arr = (Cache8C * self.L)(*[c.c for c in self.caches])
        h = C.c_void_p()
        rc = lib().first_pages_create(ctx.h, self.B, self.max_pages, arr, C.byref(h))
        if rc:
            raise FirstError(rc, "first_pages_create")
        self.h = h

    def close(self):
        if self.h:
            if getattr(self._ctx, "_pages", None) is self and self._ctx.h is not None:
                self._ctx.set_pages(None)
            lib().first_pages_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _call(self, name, *args):
        rc = getattr(lib(), name)(self.h, *args)
        if rc:
            raise FirstError(rc, name)

    def join(self, mask_row, src=None, src_seq=0, n_tokens=0):
        import numpy as np
        m = np.ascontiguousarray(np.asarray(mask_row), dtype=np.uint8)
        if m.size != self.L:
            raise ValueError(f"mask_row must have {self.L} entries")
        off = getattr(src, "slab_off", None)
        if off is not None and not 0 <= int(src_seq) < off.shape[-1]:
            raise ValueError(f"src has {off.shape[-1]} sequences")
        slot = C.c_int32(-1)
        self._call("first_pages_join", m.ctypes.data, C.byref(src.c) if src is not None else None, int(src_seq), int(n_tokens), C.byref(slot))
        if src is not None:
            self._sources.append(src)
        return slot.value

    def fork(self, slot):
        out = C.c_int32(-1)
        self._call("first_pages_fork", int(slot), C.byref(out))
        return out.value

    def extend(self, n_new=1, slot=-1):
        self._call("first_pages_extend", int(slot), int(n_new))

    def trim(self, slot, n_tokens):
        self._call("first_pages_trim", int(slot), int(n_tokens))

    def leave(self, slot):
        self._call("first_pages_leave", int(slot))

    def commit(self, stream=None):
        self._call("first_pages_commit", _stream(stream))
        self._sources.clear()
        self._ctx.B = self.B

    def compact(self, stream=None):
        self._call("first_pages_compact", _stream(stream))
        self._sources.clear()
        self._ctx.B = self.B

    def tokens(self, slot):
        n = C.c_int32(0)
        self._call("first_pages_tokens", int(slot), C.byref(n))
        return n.value

    def stats(self):
        """-> (pages in use per layer, highest page in use per layer, live sequences)."""
        import numpy as np
        held, top, live = np.zeros(self.L, np.int32), np.zeros(self.L, np.int32), C.c_int32(0)
        self._call("first_pages_stats", held.ctypes.data, top.ctypes.data, C.byref(live))
        return held, top, live.value

    def layer(self, layer):
        """-> (Cache8, page table, lengths) of a layer, as CUDA int32 tensors [max_seqs][max_pages] and [max_seqs] that view the manager's own."""
        table, ln = C.c_void_p(), C.c_void_p()
        self._call("first_pages_layer", int(layer), None, C.byref(table), None, C.byref(ln))
        return self.caches[layer], _view_i32(table.value, (self.B, self.max_pages), self), _view_i32(ln.value, (self.B,), self)


class _DeviceArray:
    def __init__(self, address, shape, owner):
        self.owner = owner  # (a view keeps the manager alive)
        self.__cuda_array_interface__ = {"shape": shape, "typestr": "<i4", "data": (address, False), "version": 2}


def _view_i32(address, shape, owner):
    return torch.as_tensor(_DeviceArray(address, shape, owner), device="cuda")


def first_set_pages(h, pages=None):
    rc = lib().first_set_pages(h, None if pages is None else pages.h)
    if rc:
        raise FirstError(rc, "first_set_pages")


def first_get_plan(h, B, L):
    import numpy as np
    idx = np.empty((L, B), dtype=np.int32)
    cnt = np.empty((L,), dtype=np.int32)
    slot = np.empty((L, B), dtype=np.int32)
    rc = lib().first_get_plan(h, idx.ctypes.data, cnt.ctypes.data, slot.ctypes.data)
    if rc:
        raise FirstError(rc, "first_get_plan")
    return idx, cnt, slot


def first_decode_step(h, tokens, kv: KVCache, logits=None, next_tokens=None, layer_inputs=None, stream=None):
    rc = lib().first_decode_step(h, _dev(tokens, torch.int32, "tokens"), None if kv is None else C.byref(kv.c),
                                 _dev(logits, torch.float32, "logits"),
                                 _dev(next_tokens, torch.int32, "next_tokens"),
                                 _dev(layer_inputs, torch.float32, "layer_inputs"), _stream(stream))
    if rc:
        raise FirstError(rc, "first_decode_step")


def first_last_device_flags(h, stream=None):
    fl = C.c_uint32(0)
    rc = lib().first_last_device_flags(h, C.byref(fl), _stream(stream))
    if rc not in (0, -6):
        raise FirstError(rc, "first_last_device_flags")
    return fl.value


def first_set_option(h, name, value):
    rc = lib().first_set_option(h, name.encode(), int(value))
    if rc:
        raise FirstError(rc, "first_set_option")


def first_set_sampling(h, top_k, temperature, uniforms):
    """uniforms: CUDA float32 [B] (borrowed: refresh its contents before every step), or None with
    top_k <= 1 / temperature 0 to go back to argmax."""
    rc = lib().first_set_sampling(h, int(top_k), float(temperature), _dev(uniforms, torch.float32, "uniforms"))
    if rc:
        raise FirstError(rc, "first_set_sampling")


def first_sample_topk(logits, top_k, temperature, uniforms, tokens, stream=None):
    """logits CUDA float32 [B][vocab]; uniforms CUDA float32 [B]; tokens CUDA int32 [B] (output)."""
    B, V = logits.shape
    if uniforms.numel() != B or tokens.numel() != B:
        raise ValueError("uniforms and tokens must have one entry per row of logits")
    rc = lib().first_sample_topk(_dev(logits, torch.float32, "logits"), B, V, int(top_k), float(temperature),
                                 _dev(uniforms, torch.float32, "uniforms"), _dev(tokens, torch.int32, "tokens"),
                                 _stream(stream))
    if rc:
        raise FirstError(rc, "first_sample_topk")


def _on(t, dtype, n, what, dev):
    """Address of a contiguous CUDA tensor of n elements (None: NULL) on device `dev`."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != dev:
        if t.dtype is not dtype or not t.is_cuda:
            raise TypeError(f"{what} must be a CUDA tensor of {dtype}")
        raise ValueError(f"{what} is on another device")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous with {n} elements")
    return t.data_ptr()


def _raw_stream(stream, dev):
    """The stream's handle; None: the current stream of device `dev`."""
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(dev) if _RAW else torch.cuda.current_stream(dev).cuda_stream


# (building a Stream object takes longer than a small call; without a CUDA build of torch neither is there)
_RAW = hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice")


def _device_of(t, what):
    """The device index of a CUDA tensor; the calls launch on the current device, so it has to be that one."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    dev = t.get_device()
    if dev != (torch._C._cuda_getDevice() if _RAW else torch.cuda.current_device()):
        raise ValueError(f"{what} is on device {dev}, not on the current one")
    return dev


_DTYPE_CODE = {torch.float32: FIRST_DTYPE_F32, torch.bfloat16: FIRST_DTYPE_BF16}


def _code(t, what):
    c = _DTYPE_CODE.get(t.dtype)
    if c is None:
        raise TypeError(f"{what} must be float32 or bfloat16")
    return c


def _rows_of(t, what):
    """(row stride) of a matrix whose rows may be padded; elements of a row are adjacent."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what} must be a matrix with adjacent elements in a row")
    return t.stride(0)


def first_sample(logits, uniforms, tokens, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
    """Next token of every row with settings of its own (see first.h).  logits CUDA float32 [B][vocab], rows may be
    padded; uniforms, temperature, top_p, min_p CUDA float32 [B], top_k CUDA int32 [B]; tokens CUDA int32 [B] (output)."""
    dev = _device_of(logits, "logits")
    if logits.dtype != torch.float32:
        raise TypeError("logits must be float32")
    ld = _rows_of(logits, "logits")
    B, V = logits.shape
    f32, i32 = torch.float32, torch.int32
    if uniforms is None or tokens is None:
        raise TypeError("uniforms and tokens are required")
    rc = lib().first_sample(logits.data_ptr(), ld, B, V, _on(temperature, f32, B, "temperature", dev), _on(top_k, i32, B, "top_k", dev),
                            _on(top_p, f32, B, "top_p", dev), _on(min_p, f32, B, "min_p", dev),
                            _on(uniforms, f32, B, "uniforms", dev), _on(tokens, i32, B, "tokens", dev), _raw_stream(stream, dev))
    if rc:
        raise FirstError(rc, "first_sample")


@functools.lru_cache(maxsize=256)
def _segment_array(segments):
    return (C.c_int32 * len(segments))(*segments)


def first_lora(x, a, b, row_adapter, y, scales=None, segments=None, stream=None):
    """y[r] += scales[i] * b[i] (a[i] x[r]), i = row_adapter[r], rows with an id outside 0 .. n-1 left alone (see first.h).
    x CUDA [rows][k], y CUDA [rows][n] (rows may be padded), float32 or bfloat16; a CUDA [adapters][segments*rank][k],
    b CUDA [adapters][n][rank], contiguous, of one type; segments: borders of the output segments, (0, ..., n)."""
    dev = _device_of(x, "x")
    ldx, ldy = _rows_of(x, "x"), _rows_of(y, "y")
    rows, k = x.shape
    n = y.shape[1]
    if y.shape[0] != rows or a.dim() != 3 or b.dim() != 3 or a.dtype is not b.dtype:
        raise ValueError("x and y must have one row each per row of the batch; a, b three dimensions and one type")
    segments = (0, n) if segments is None else tuple(segments)
    adapters, bn, rank = b.shape
    parts = len(segments) - 1
    if bn != n or a.shape != (adapters, parts * rank, k):
        raise ValueError("a must be [adapters][segments*rank][k] and b [adapters][n][rank]")
    if y.get_device() != dev or a.get_device() != dev or b.get_device() != dev:
        raise ValueError("x, y, a and b must be on one device")
    if not (a.is_contiguous() and b.is_contiguous()):
        raise ValueError("a and b must be contiguous")
    rc = lib().first_lora(x.data_ptr(), _code(x, "x"), ldx, a.data_ptr(), b.data_ptr(), _code(a, "a"),
                          _on(scales, torch.float32, adapters, "scales", dev), _on(row_adapter, torch.int32, rows, "row_adapter", dev),
                          adapters, rank, parts, _segment_array(segments), rows, k, n, y.data_ptr(), _code(y, "y"), ldy,
                          _raw_stream(stream, dev))
    if rc:
        raise FirstError(rc, "first_lora")


def first_rope_freqs(rot_dim, base, scaling="none", factor=1.0, low=1.0, high=None, trained_len=0):
    """-> (inv_freq numpy float64 [rot_dim/2], factor on cosines and sines) of a scheme: none, linear, llama3, yarn."""
    import numpy as np
    kinds = {"none": 0, "linear": 1, "llama3": 2, "yarn": 3}
    if scaling not in kinds:
        raise ValueError(f"unknown scaling {scaling!r}")
    if high is None:
        high = 32.0 if scaling == "yarn" else 4.0
    spec = RopeSpecC(int(rot_dim), kinds[scaling], float(base), float(factor), float(low), float(high), int(trained_len))
    inv = np.empty(max(int(rot_dim) // 2, 1), dtype=np.float64)
    out = C.c_double(1.0)
    rc = lib().first_rope_freqs(C.byref(spec), inv.ctypes.data, C.byref(out))
    if rc:
        raise FirstError(rc, "first_rope_freqs")
    return inv, out.value


def _heads_of(t, what):
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{what} must be [tokens][heads][head_dim] with adjacent elements in a head")


def first_rope(q, k, pos, inv_freq, factor=1.0, interleaved=False, stream=None):
    """Rotates q CUDA [tokens][Hq][hd] and k CUDA [tokens][Hkv][hd] (or None) in place; both may be views of a larger
    buffer.  pos CUDA int32 [tokens]; inv_freq CUDA float64 [rot/2] (rot <= hd elements of a head are rotated)."""
    dev = _device_of(q, "q")
    _heads_of(q, "q")
    T, hq, hd = q.shape
    kp, hk, ks = None, 0, (0, 0)
    if k is not None:
        _heads_of(k, "k")
        if k.shape[0] != T or k.shape[2] != hd or k.dtype != q.dtype:
            raise ValueError("q and k must agree in tokens, head size and type")
        if k.get_device() != dev:
            raise ValueError("k is on another device")
        kp, hk, ks = k.data_ptr(), k.shape[1], k.stride()
    qs = q.stride()
    rc = lib().first_rope(q.data_ptr(), qs[0], qs[1], hq, kp, ks[0], ks[1], hk, _code(q, "q"), T, hd, 2 * inv_freq.numel(),
                          _on(pos, torch.int32, T, "pos", dev), _on(inv_freq, torch.float64, inv_freq.numel(), "inv_freq", dev),
                          factor, bool(interleaved), _raw_stream(stream, dev))
    if rc:
        raise FirstError(rc, "first_rope")


class Cache8:
    """One layer's paged 8-bit cache (first_cache8 in first.h): k, v CUDA [n_pages][Hkv][page][hd] of torch.int8 or
    torch.float8_e4m3fn, k_scale, v_scale CUDA float32 [n_pages][Hkv].  Borrowed: holds on to the tensors."""

    def __init__(self, k, v, k_scale, v_scale):
        formats = {torch.int8: CACHE_INT8, torch.float8_e4m3fn: CACHE_E4M3}
        if k.dim() != 4 or v.shape != k.shape:
            raise ValueError("k and v must be [pages][heads][tokens][head_dim], alike")
        if k.dtype not in formats or v.dtype is not k.dtype:
            raise TypeError("k and v must be int8 or float8_e4m3fn, alike")
        self.device = k.get_device()
        n, heads, page, hd = k.shape
        for t in (k, v):
            if not t.is_cuda or t.get_device() != self.device or not t.is_contiguous():
                raise ValueError("k and v must be contiguous, on one CUDA device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.c = Cache8C(formats[k.dtype], n, heads, page, hd, k.data_ptr(), v.data_ptr(),
                         _on(k_scale, torch.float32, n * heads, "k_scale", self.device),
                         _on(v_scale, torch.float32, n * heads, "v_scale", self.device))
        self.ref, self.raw = C.byref(self.c), bytes(self.c)
        self.heads, self.head_dim = heads, hd
        self.sizes = (formats[k.dtype], n, heads, page, hd)


def _batch8(cache, dev, pages, len_, cu):
    """(cu, pages, width, len, sequences) of a call on an 8-bit cache."""
    if cache.device != dev:
        raise ValueError("the cache is on another device")
    if pages.dim() != 2:
        raise ValueError("pages must be [sequences][pages]")
    B, width = pages.shape
    return (_on(cu, torch.int32, B + 1, "cu", dev), _on(pages, torch.int32, B * width, "pages", dev), width,
            _on(len_, torch.int32, B, "len", dev), B)


def _kv_rows(cache, k, v, dev):
    """(rows, strides of k, strides of v, dtype code) of two tensors [rows][Hkv][hd].  (Sizes and strides are fetched once: the
    checks of a small call take as long as the call.)"""
    shape, ks, vs = k.shape, k.stride(), v.stride()
    if len(shape) != 3 or v.shape != shape or k.dtype is not v.dtype or v.get_device() != dev:
        raise ValueError("k and v must be [rows][heads][head_dim], alike, on one device")
    rows, heads, hd = shape
    if (ks[2] != 1 or vs[2] != 1) and hd > 1:
        raise ValueError("k and v must have adjacent elements in a head")
    if heads != cache.heads or hd != cache.head_dim:
        raise ValueError("k and v must have the cache's heads and head size")
    return rows, ks, vs, _code(k, "k")


def first_append8(k, v, cache, pages, len, cu_new=None, max_new=1, flags=None, stream=None):
    """Stores new keys and values, CUDA [total][Hkv][hd] (strided views are fine), in pages of a Cache8 (see first.h).  pages
    CUDA int32 [B][n] of page ids; len CUDA int32 [B], tokens before the new ones; cu_new CUDA int32 [B+1], rows of each sequence (None:
    one row each); max_new: most new tokens of a sequence; flags CUDA int32 [1] or None."""
    dev = _device_of(k, "k")
    total, ks, vs, code = _kv_rows(cache, k, v, dev)
    cu, pp, width, lp, B = _batch8(cache, dev, pages, len, cu_new)
    rc = lib().first_append8(cache.ref, k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], code, cu, total, pp, width, lp, B,
                             max_new, _on(flags, torch.int32, 1, "flags", dev), _raw_stream(stream, dev))
    if rc:
        raise FirstError(rc, "first_append8")


def first_read8(cache, pages, start, k, v, cu=None, max_rows=1, flags=None, stream=None):
    """Writes the values at positions start[b] .. of every sequence to rows cu[b] .. cu[b+1]-1 of k and v (see first.h)."""
    dev = _device_of(k, "k")
    total, ks, vs, code = _kv_rows(cache, k, v, dev)
    cp, pp, width, sp, B = _batch8(cache, dev, pages, start, cu)
    rc = lib().first_read8(cache.ref, pp, width, sp, cp, B, total, max_rows, k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1],
                           code, _on(flags, torch.int32, 1, "flags", dev), _raw_stream(stream, dev))
    if rc:
        raise FirstError(rc, "first_read8")


@functools.lru_cache(maxsize=1024)
def _workspace8(sizes, n_q_heads, code, total, width, B, max_new):
    return lib().first_attn8_workspace(C.byref(Cache8C(*sizes, 16, 16, 16, 16)), n_q_heads, code, total, width, B, max_new)


def first_attn8(q, cache, pages, len, out, scale=None, cu_new=None, max_new=1, workspace=None, flags=None, stream=None):
    """Attention of the new tokens' queries, CUDA [total][Hq][hd], over a Cache8 that holds their keys and values already; out
    like q.  len, cu_new, max_new as in first_append8.  scale None: 1/sqrt(hd).  workspace: a CUDA tensor to keep unfinished
    results in (first_attn8_workspace bytes), None: one is taken from torch's allocator where there is a use for it."""
    dev = _device_of(q, "q")
    shape, qs, os_ = q.shape, q.stride(), out.stride()
    if out.shape != shape or out.dtype is not q.dtype or out.get_device() != dev:
        raise ValueError("out must be like q")
    if q.dim() != 3 or ((qs[2] != 1 or os_[2] != 1) and shape[2] > 1):
        raise ValueError("q and out must be [rows][heads][head_dim] with adjacent elements in a head")
    total, hq, hd = shape
    if hd != cache.head_dim:
        raise ValueError("q must have the cache's head size")
    cu, pp, width, lp, B = _batch8(cache, dev, pages, len, cu_new)
    code, room = _code(q, "q"), 0
    if workspace is None:
        room = _workspace8(cache.sizes, hq, code, total, width, B, max_new)
        if room:
            with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
                workspace = torch.empty(room, dtype=torch.uint8, device=q.device)
    else:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous, on q's device")
        room = workspace.numel() * workspace.element_size()
    rc = lib().first_attn8(cache.ref, q.data_ptr(), qs[0], qs[1], hq, code, hd ** -0.5 if scale is None else scale, cu, total, pp, width,
                           lp, B, max_new, out.data_ptr(), os_[0], os_[1], workspace.data_ptr() if room else None, room,
                           _on(flags, torch.int32, 1, "flags", dev), _raw_stream(stream, dev))
    if rc:
        raise FirstError(rc, "first_attn8")


def first_copy_pages(caches, moves, flags=None, stream=None):
    """Copies pages within the layers' caches (a list of Cache8): moves CUDA int32 [n][3] of (layer, from, to)."""
    dev = _device_of(moves, "moves")
    if moves.dim() != 2 or moves.shape[1] != 3:
        raise ValueError("moves must be [n][3]")
    here = [c.raw for c in caches if c.device == dev]
    if len(here) != len(caches):
        raise ValueError("the caches are on another device")
    arr = b"".join(here)  # (an array of first_cache8)
    rc = lib().first_copy_pages(arr, len(caches), _on(moves, torch.int32, moves.numel(), "moves", dev), moves.shape[0],
                                _on(flags, torch.int32, 1, "flags", dev), _raw_stream(stream, dev))
    if rc:
        raise FirstError(rc, "first_copy_pages")


def first_verify(target, drafted, uniforms, draws, tokens, accepted, draft=None, temperature=None, probs=False, stream=None):
    """Accepts or refuses drafted tokens and draws the token after them (see first.h).  target CUDA float32
    [B][n+1][vocab], draft [B][n][vocab] or None (adjacent elements in a row): logits, or probabilities with probs;
    drafted CUDA int32 [B][n]; uniforms CUDA float32 [B][n], draws [B]; temperature CUDA float32 [B] or None.
    Output: tokens CUDA int32 [B][n+1], accepted CUDA int32 [B]."""
    dev = _device_of(target, "target")
    f32, i32 = torch.float32, torch.int32
    ts = target.stride()
    if len(ts) != 3 or (ts[2] != 1 and target.shape[2] > 1):
        raise ValueError("target must be [sequences][drafts + 1][vocab] with adjacent elements in a row")
    if target.dtype is not f32:
        raise TypeError("target must be float32")
    B, rows, V = target.shape
    n = rows - 1
    if n < 0:
        raise ValueError("target needs a row for the token after the drafts")
    dp, ds = None, (0, 0)
    if draft is not None:
        if draft.dtype is not f32 or draft.get_device() != dev:
            raise TypeError("draft must be float32, on target's device")
        ds = draft.stride()
        if draft.shape != (B, n, V) or (ds[2] != 1 and V > 1):
            raise ValueError("draft must be [sequences][drafts][vocab] with adjacent elements in a row")
        dp = draft.data_ptr()
    if draws is None or tokens is None or accepted is None:
        raise TypeError("draws, tokens and accepted are required")
    rc = lib().first_verify(target.data_ptr(), ts[0], ts[1], dp, ds[0], ds[1], bool(probs), _on(drafted, i32, B * n, "drafted", dev),
                            B, n, V, _on(temperature, f32, B, "temperature", dev), _on(uniforms, f32, B * n, "uniforms", dev),
                            _on(draws, f32, B, "draws", dev), _on(tokens, i32, B * rows, "tokens", dev),
                            _on(accepted, i32, B, "accepted", dev), _raw_stream(stream, dev))
    if rc:
        raise FirstError(rc, "first_verify")


def first_set_sampling_rows(h, uniforms=None, temperature=None, top_k=None, top_p=None, min_p=None):
    """Per-row sampling of later steps; arrays CUDA [B], borrowed.  uniforms None restores argmax."""
    if uniforms is None:
        rc = lib().first_set_sampling_rows(h, None)
    else:
        s = SamplingC(_dev(temperature, torch.float32, "temperature"), _dev(top_k, torch.int32, "top_k"),
                      _dev(top_p, torch.float32, "top_p"), _dev(min_p, torch.float32, "min_p"),
                      _dev(uniforms, torch.float32, "uniforms"))
        rc = lib().first_set_sampling_rows(h, C.byref(s))
    if rc:
        raise FirstError(rc, "first_set_sampling_rows")


def first_set_adapters(h, shape, dtype, adapters=None, seq_adapter=None, scales=None):
    """adapters: dict of per-layer lists of (a, b) pairs (None = no adapter there) under qkv, o, gate_up, down;
    seq_adapter CUDA int32 [max_batch].  Everything is borrowed.  adapters None removes them.  Returns what to keep."""
    if adapters is None:
        rc = lib().first_set_adapters(h, None)
        if rc:
            raise FirstError(rc, "first_set_adapters")
        return None
    wd = torch.float32 if dtype == FIRST_DTYPE_F32 else torch.bfloat16
    D, F, qd = shape.d_model, shape.ffn_dim, shape.n_q_heads * shape.head_dim
    sizes = {"qkv": (3, D, qd + 2 * shape.n_kv_heads * shape.head_dim), "o": (1, qd, D), "gate_up": (2, D, 2 * F), "down": (1, F, D)}
    if set(adapters) - set(sizes):
        raise ValueError(f"unknown projections {sorted(set(adapters) - set(sizes))}")
    pairs = [p for rows in adapters.values() for p in rows if p is not None]
    if not pairs:
        raise ValueError("no adapter given")
    n, _, rank = pairs[0][1].shape
    c = AdaptersC(n, rank, _dev(scales, torch.float32, "scales"), _dev(seq_adapter, torch.int32, "seq_adapter"))
    if scales is not None and scales.numel() != n:
        raise ValueError("scales must have one entry per adapter")
    keep = [adapters, seq_adapter, scales]
    for name, rows in adapters.items():
        segs, k, out = sizes[name]
        if len(rows) != shape.n_layers:
            raise ValueError(f"{name}: one entry per layer")
        for p in rows:
            if p is not None and (tuple(p[0].shape) != (n, segs * rank, k) or tuple(p[1].shape) != (n, out, rank)):
                raise ValueError(f"{name}: a must be [{n}][{segs * rank}][{k}] and b [{n}][{out}][{rank}]")
        for j, m in enumerate("ab"):
            arr = _ptr_array([None if p is None else p[j] for p in rows], wd, f"{name}.{m}")
            keep.append(arr)
            setattr(c, f"{name}_{m}", C.cast(arr, C.POINTER(C.c_void_p)))
    rc = lib().first_set_adapters(h, C.byref(c))
    if rc:
        raise FirstError(rc, "first_set_adapters")
    return keep


def first_set_rope(h, inv_freq=None, factor=1.0, head_dim=None):
    """inv_freq: HOST float64 [head_dim/2] (first_rope_freqs), or None for the description's own frequencies."""
    import numpy as np
    f = None if inv_freq is None else np.ascontiguousarray(np.asarray(inv_freq), dtype=np.float64)
    if f is not None and head_dim is not None and f.size != head_dim // 2:
        raise ValueError(f"inv_freq must have {head_dim // 2} entries")
    rc = lib().first_set_rope(h, None if f is None else f.ctypes.data, float(factor))
    if rc:
        raise FirstError(rc, "first_set_rope")


def first_profile(h, enable):
    rc = lib().first_profile(h, int(bool(enable)))
    if rc:
        raise FirstError(rc, "first_profile")


def first_profile_read(h, stream=None):
    """-> {kernel class name: (total device ms, launches)}"""
    n = lib().first_kernel_class_count()
    ms = (C.c_double * n)()
    cnt = (C.c_int64 * n)()
    rc = lib().first_profile_read(h, n, ms, cnt, _stream(stream))
    if rc:
        raise FirstError(rc, "first_profile_read")
    return {lib().first_kernel_class_name(k).decode(): (ms[k], cnt[k]) for k in range(n)}


def first_step_trace(h, stream=None, max_n=2048):
    """Launches of the last step with option "stamp" on: [(class name, start_ns, end_ns)] in launch order."""
    import numpy as np
    cls = np.zeros(max_n, dtype=np.int32)
    t0 = np.zeros(max_n, dtype=np.uint64)
    t1 = np.zeros(max_n, dtype=np.uint64)
    n = C.c_int32(0)
    rc = lib().first_step_trace(h, max_n, cls.ctypes.data, t0.ctypes.data, t1.ctypes.data, C.byref(n), _stream(stream))
    if rc:
        raise FirstError(rc, "first_step_trace")
    names = [lib().first_kernel_class_name(int(k)).decode() for k in cls[:n.value]]
    return [(names[i], int(t0[i]), int(t1[i])) for i in range(n.value)]


class FirstContext:
    """Owns one library context; methods mirror the C calls."""

    def __init__(self, shape, dtype, max_batch, max_tokens_per_seq, weights):
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required; there is no CPU path")
        self.shape, self.dtype, self.max_batch = shape, dtype, int(max_batch)
        self._sampling = ()
        self.h, self._keep = first_create(shape, dtype, max_batch, max_tokens_per_seq, weights)

    def close(self):
        if self.h is not None:
            first_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def prefill_route(self, layer, hidden, cu_seqlens, router_w, router_b, tau, mode, mask, scores=None, stream=None):
        first_prefill_route(self.h, layer, hidden, cu_seqlens, router_w, router_b, tau, mode, mask, scores, stream)

    def prefill(self, tokens, cu_seqlens, kv, router_w=None, router_b=None, tau=0.5, mode=0, mask=None, scores=None,
                logits=None, next_tokens=None, stream=None):
        self._check_sampling(len(cu_seqlens) - 1, next_tokens)
        first_prefill(self.h, tokens, cu_seqlens, kv, router_w, router_b, tau, mode, mask, scores, logits,
                      next_tokens, stream)

    def set_mask(self, mask, stream=None):
        first_set_mask(self.h, mask, stream)
        self.B = mask.shape[0]

    def set_mask_host(self, mask, stream=None):
        import numpy as np
        first_set_mask_host(self.h, mask, stream)
        self.B = np.asarray(mask).shape[0]

    def graph_count(self):
        return int(lib().first_graph_count(self.h))

    def get_plan(self):
        return first_get_plan(self.h, self.B, self.shape.n_layers)

    def decode_step(self, tokens, kv, logits=None, next_tokens=None, layer_inputs=None, stream=None):
        self._check_sampling(getattr(self, "B", 0), next_tokens)
        first_decode_step(self.h, tokens, kv, logits, next_tokens, layer_inputs, stream)

    def device_flags(self, stream=None):
        return first_last_device_flags(self.h, stream)

    def launch_count(self):
        return int(lib().first_launch_count(self.h))

    def set_option(self, name, value):
        first_set_option(self.h, name, value)

    def set_sampling(self, top_k, temperature, uniforms):
        self._uniforms = uniforms  # borrowed by the library until the next call
        self._sampling = ()
        first_set_sampling(self.h, top_k, temperature, uniforms)

    def set_sampling_rows(self, uniforms=None, temperature=None, top_k=None, top_p=None, min_p=None):
        """Arrays of one entry per batch row (borrowed until the next call); uniforms None restores argmax."""
        first_set_sampling_rows(self.h, uniforms, temperature, top_k, top_p, min_p)
        self._sampling = () if uniforms is None else tuple(t for t in (uniforms, temperature, top_k, top_p, min_p) if t is not None)

    def _check_sampling(self, rows, next_tokens):
        if next_tokens is not None and any(t.numel() < rows for t in self._sampling):
            raise ValueError(f"the sampling settings have fewer than {rows} entries")

    def set_adapters(self, adapters=None, seq_adapter=None, scales=None):
        """adapters: {"qkv" | "o" | "gate_up" | "down": [(a, b) or None per layer]}; seq_adapter CUDA int32 [max_batch]."""
        if adapters is not None and seq_adapter.numel() < self.max_batch:
            raise ValueError(f"seq_adapter must have {self.max_batch} entries")
        self._adapters = first_set_adapters(self.h, self.shape, self.dtype, adapters, seq_adapter, scales)

    def set_pages(self, pages=None):
        """Steps with kv=None run over this FirstPages (kept alive until the next call)."""
        first_set_pages(self.h, pages)
        self._pages = pages

    def set_rope(self, inv_freq=None, factor=1.0):
        first_set_rope(self.h, inv_freq, factor, self.shape.head_dim)

    def selftest_wait_expiry(self, polls=1000, stream=None):
        """Runs a bounded wait that must give up; -> (what the wait returned, the abort word)."""
        r, a = C.c_int32(-1), C.c_int32(-1)
        rc = lib().first_selftest_wait_expiry(self.h, int(polls), C.byref(r), C.byref(a), _stream(stream))
        if rc:
            raise FirstError(rc, "first_selftest_wait_expiry")
        return r.value, a.value

    def step_trace(self, stream=None):
        return first_step_trace(self.h, stream)

    def profile(self, enable):
        first_profile(self.h, enable)

    def profile_read(self, stream=None):
        return first_profile_read(self.h, stream)
