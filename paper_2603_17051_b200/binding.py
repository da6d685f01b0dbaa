"""ctypes binding of the C ABI declared in include/astro.h.

Argument marshalling only: every step of the path runs in the CUDA kernels of
libastro.so.  There is no fallback: if the library cannot be built or loaded,
or a call returns an error status, an exception is raised.  torch supplies
device memory and the current stream, nothing else.
"""
from __future__ import annotations

import contextlib
import ctypes as C

from . import build as _build

ASTRO_OK = 0
STATUS_NAMES = {0: "ASTRO_OK", 1: "ASTRO_ERR_NULL", 2: "ASTRO_ERR_SHAPE", 3: "ASTRO_ERR_ALIGN",
                4: "ASTRO_ERR_CAPACITY", 5: "ASTRO_ERR_UNDERFLOW", 6: "ASTRO_ERR_ARCH", 7: "ASTRO_ERR_CUDA",
                8: "ASTRO_ERR_TIMEOUT"}

EXPORTED = ("astro_kvcache_key_segments", "astro_selftest_wait_timeout", "astro_nft_loss", "astro_kvcache_get_state", "astro_kvcache_set_state", "astro_kvcache_storage_bytes", "astro_kvcache_create", "astro_kvcache_destroy", "astro_kvcache_reset",
            "astro_kvcache_append", "astro_kvcache_evict", "astro_kvcache_query", "astro_kvcache_export",
            "astro_chunk_attn_fwd", "astro_chunk_attn_bwd_workspace_bytes", "astro_chunk_attn_bwd",
            "astro_chunk_attn_bwd_delta", "astro_chunk_attn_bwd_dq", "astro_chunk_attn_bwd_dkv",
            "astro_chunk_attn_bwd_static", "astro_debug_forward_mode", "astro_debug_pair_flag",
            "astro_last_device_status", "astro_status_string", "astro_kvcache_fork", "astro_rope_create",
            "astro_rope_destroy", "astro_rope_frequencies", "astro_rope_apply", "astro_rope_apply_check", "astro_block_count", "astro_block_pool",
            "astro_block_select_workspace_bytes", "astro_block_select", "astro_sparse_attn_fwd_workspace_bytes",
            "astro_sparse_attn_fwd", "astro_sparse_attn_bwd_workspace_bytes", "astro_sparse_attn_bwd")


class AstroError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__("%s failed: %s (%s)" % (where, STATUS_NAMES.get(self.status, self.status),
                                                  status_string(self.status)))


class KVCacheDesc(C.Structure):
    _fields_ = [("cache_batch", C.c_int), ("heads", C.c_int), ("head_dim", C.c_int),
                ("tokens_per_frame", C.c_int), ("sink_frames", C.c_int), ("window_frames", C.c_int)]


class KVCacheState(C.Structure):
    _fields_ = [("sink_held", C.c_int), ("window_head", C.c_int), ("window_held", C.c_int),
                ("frames_seen", C.c_int64)]


class RopeDesc(C.Structure):
    _fields_ = [("head_dim", C.c_int), ("rot_dim", C.c_int), ("layout", C.c_int), ("axes", C.c_int),
                ("axis_pairs", C.c_int * 4), ("base", C.c_double), ("scaling", C.c_int), ("scaled_axes", C.c_int),
                ("factor", C.c_double), ("original_length", C.c_double), ("ramp_low", C.c_double),
                ("ramp_high", C.c_double), ("magnitude", C.c_double)]


class Strides(C.Structure):
    _fields_ = [("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


_lib = None


def lib():
    """Load (building first when stale) the shared library; raises if that is impossible."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.build()
    L = C.CDLL(path)
    vp, ci, cf, sz = C.c_void_p, C.c_int, C.c_float, C.c_size_t
    L.astro_kvcache_storage_bytes.restype = sz
    L.astro_kvcache_storage_bytes.argtypes = [C.POINTER(KVCacheDesc)]
    L.astro_kvcache_create.restype = ci
    L.astro_kvcache_create.argtypes = [C.POINTER(KVCacheDesc), vp, vp, sz, C.POINTER(vp)]
    L.astro_kvcache_destroy.restype = ci
    L.astro_kvcache_destroy.argtypes = [vp]
    L.astro_kvcache_reset.restype = ci
    L.astro_kvcache_reset.argtypes = [vp]
    L.astro_kvcache_append.restype = ci
    L.astro_kvcache_append.argtypes = [vp, vp, vp, ci, vp]
    L.astro_kvcache_evict.restype = ci
    L.astro_kvcache_evict.argtypes = [vp, ci, vp]
    L.astro_kvcache_query.restype = ci
    L.astro_kvcache_query.argtypes = [vp, C.POINTER(ci), C.POINTER(ci), C.POINTER(C.c_int64)]
    L.astro_kvcache_get_state.restype = ci
    L.astro_kvcache_get_state.argtypes = [vp, C.POINTER(KVCacheState)]
    L.astro_kvcache_set_state.restype = ci
    L.astro_kvcache_set_state.argtypes = [vp, C.POINTER(KVCacheState)]
    L.astro_kvcache_key_segments.restype = ci
    L.astro_kvcache_key_segments.argtypes = [vp, ci, C.POINTER(ci), C.POINTER(ci), C.POINTER(ci), C.POINTER(ci)]
    L.astro_kvcache_export.restype = ci
    L.astro_kvcache_export.argtypes = [vp, vp, vp, vp]
    L.astro_chunk_attn_fwd.restype = ci
    L.astro_chunk_attn_fwd.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, vp, vp]
    L.astro_chunk_attn_bwd_workspace_bytes.restype = sz
    L.astro_chunk_attn_bwd_workspace_bytes.argtypes = [ci, ci, ci, ci]
    L.astro_chunk_attn_bwd.restype = ci
    L.astro_chunk_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, vp, vp, vp, sz, vp]
    L.astro_chunk_attn_bwd_delta.restype = ci
    L.astro_chunk_attn_bwd_delta.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp]
    L.astro_chunk_attn_bwd_dq.restype = ci
    L.astro_chunk_attn_bwd_dq.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, vp]
    L.astro_chunk_attn_bwd_dkv.restype = ci
    L.astro_chunk_attn_bwd_dkv.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, vp, vp]
    L.astro_chunk_attn_bwd_static.restype = ci
    L.astro_chunk_attn_bwd_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, vp, vp, vp]
    L.astro_nft_loss.restype = ci
    L.astro_nft_loss.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, C.c_longlong, cf, vp, vp, vp, vp]
    L.astro_kvcache_fork.restype = ci
    L.astro_kvcache_fork.argtypes = [vp, vp, vp, C.POINTER(ci), ci, vp]
    L.astro_rope_create.restype = ci
    L.astro_rope_create.argtypes = [C.POINTER(RopeDesc), C.POINTER(vp)]
    L.astro_rope_destroy.restype = ci
    L.astro_rope_destroy.argtypes = [vp]
    L.astro_rope_frequencies.restype = ci
    L.astro_rope_frequencies.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_double)]
    L.astro_rope_apply.restype = ci
    L.astro_rope_apply.argtypes = [vp, ci, vp, vp, vp, ci, ci, ci, ci, ci, ci, C.POINTER(Strides), vp, vp,
                                   C.POINTER(Strides), vp]
    L.astro_rope_apply_check.restype = ci
    L.astro_rope_apply_check.argtypes = L.astro_rope_apply.argtypes[:-1]
    L.astro_block_count.restype = ci
    L.astro_block_count.argtypes = [vp, ci, ci, C.POINTER(ci), C.POINTER(ci)]
    L.astro_block_pool.restype = ci
    L.astro_block_pool.argtypes = [vp, ci, ci, ci, vp, vp]
    L.astro_block_select_workspace_bytes.restype = sz
    L.astro_block_select_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, ci]
    L.astro_block_select.restype = ci
    L.astro_block_select.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, vp, vp, sz, vp]
    L.astro_sparse_attn_fwd_workspace_bytes.restype = sz
    L.astro_sparse_attn_fwd_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, ci]
    L.astro_sparse_attn_fwd.restype = ci
    L.astro_sparse_attn_fwd.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, cf, vp, vp, vp, sz, vp]
    L.astro_sparse_attn_bwd_workspace_bytes.restype = sz
    L.astro_sparse_attn_bwd_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, ci, ci]
    L.astro_sparse_attn_bwd.restype = ci
    L.astro_sparse_attn_bwd.argtypes = [vp, vp, vp, vp, vp, ci, ci, vp, vp, vp, ci, ci, ci, ci, ci, cf, vp, vp, vp, vp, sz, vp]
    L.astro_debug_forward_mode.restype = ci
    L.astro_debug_forward_mode.argtypes = [ci]
    L.astro_debug_pair_flag.restype = ci
    L.astro_debug_pair_flag.argtypes = [C.POINTER(ci)]
    L.astro_selftest_wait_timeout.restype = ci
    L.astro_selftest_wait_timeout.argtypes = [vp]
    L.astro_last_device_status.restype = ci
    L.astro_last_device_status.argtypes = [C.POINTER(C.c_uint32)]
    L.astro_status_string.restype = C.c_char_p
    L.astro_status_string.argtypes = [ci]
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().astro_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != ASTRO_OK:
        raise AstroError(status, where)


def _int(x):
    """A whole number for a C int.  ctypes would cut off the bits behind the 32nd; a number that has any becomes one that every
    call refuses."""
    x = int(x)
    return x if -0x80000000 <= x <= 0x7fffffff else -0x80000000


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _contiguous(*tensors):
    for t in tensors:
        if t is not None and not t.is_contiguous():
            raise ValueError("tensor arguments must be contiguous")


def _where(stream, q):
    """(device, stream address) of a call on q.  Kernels run on the current device, and a given stream must belong to it: a
    tensor that lives elsewhere, on the host included, is refused before its address reaches one."""
    import torch
    dev = q.get_device()
    if dev < 0:
        raise ValueError("tensors must be on the GPU")
    if dev != torch._C._cuda_getDevice():
        raise ValueError("tensors on cuda:%d, the current device is %d" % (dev, torch._C._cuda_getDevice()))
    if stream is None:
        return dev, torch._C._cuda_getCurrentRawStream(dev)
    if stream.device.index != dev:
        raise ValueError("the stream belongs to another device than the current one")
    return dev, stream.cuda_stream


def _like(shape, kind, dev, *tensors):
    """Tensors (None passes) that a kernel reads as contiguous ones of this shape and type on this device."""
    for t in tensors:
        if t is not None and (t.dtype is not kind or t.get_device() != dev or not t.is_contiguous() or t.shape != shape):
            raise ValueError("expected a contiguous %s tensor %s on cuda:%d, got %s %s on %s%s" % (
                kind, tuple(shape), dev, t.dtype, tuple(t.shape), t.device, "" if t.is_contiguous() else ", not contiguous"))


def _scratch(workspace, dev):
    """(address, bytes) of a workspace tensor."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous and on cuda:%d" % dev)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _cache(cache):
    """Handle of a cache or None for none.  One that has been destroyed is refused: as a null handle it would be no context."""
    if cache is None:
        return None
    if cache.handle is None:
        raise ValueError("the cache has been destroyed")
    return cache.handle


def _handle(cache, dev):
    if cache is None:
        return None
    if cache.k_storage.get_device() != dev or cache.v_storage.get_device() != dev:
        raise ValueError("the cache is on %s, the call on cuda:%d" % (cache.k_storage.device, dev))
    return _cache(cache)


def _at(t):
    return None if t is None else t.data_ptr()


def _chunk(q, dev, k_chunk, v_chunk, *others):
    """n_kc of the chunk tensors, which must fit q [B, n_q, H, D]."""
    first = k_chunk if k_chunk is not None else v_chunk
    if first is None:
        return 0
    s, (B, _, H, D) = first.shape, q.shape
    if len(s) != 4 or s[0] != B or s[2] != H or s[3] != D:
        raise ValueError("chunk tensors must be [B, n_kc, H, D] like q")
    _like(s, q.dtype, dev, k_chunk, v_chunk, *others)
    return s[1]


def _lists(q, dev, blocks):
    """n_select of blocks [B, H, query blocks, n_select], which must fit q."""
    import torch
    s, (B, n_q, H, _) = blocks.shape, q.shape
    if len(s) != 4 or s[0] != B or s[1] != H or s[2] != (n_q + QUERY_BLOCK - 1) // QUERY_BLOCK:
        raise ValueError("blocks must be [B, H, query blocks, n_select]")
    _like(s, torch.int32, dev, blocks)
    return s[3]


_HERE = contextlib.nullcontext()


def _owned_by(stream):
    """Context in which a wrapper allocates: what its kernels use on `stream` comes out of that stream's memory.  torch hands
    out memory whose last use may still be queued on the stream that it belongs to, and on that one alone."""
    import torch
    return _HERE if stream is None else torch.cuda.stream(stream)


def _used_here(stream, *tensors):
    """Tensors a wrapper allocated for `stream` are for the caller, who may be on another: tell torch's caching allocator, so that
    a block that the caller drops is not handed out again on `stream` while the caller's work still uses it."""
    if stream is None:
        return
    import torch
    here = torch.cuda.current_stream(stream.device)
    for t in tensors:
        if t is not None:
            t.record_stream(here)


def _desc(cache_batch, heads, head_dim, tokens_per_frame, sink_frames, window_frames):
    return KVCacheDesc(_int(cache_batch), _int(heads), _int(head_dim), _int(tokens_per_frame), _int(sink_frames),
                       _int(window_frames))


def astro_kvcache_storage_bytes(cache_batch, heads, head_dim, tokens_per_frame, sink_frames, window_frames) -> int:
    d = _desc(cache_batch, heads, head_dim, tokens_per_frame, sink_frames, window_frames)
    return int(lib().astro_kvcache_storage_bytes(C.byref(d)))


class KVCache:
    """Handle of one layer's rolling cache plus the torch tensors that back its storage."""

    def __init__(self, handle, desc, k_storage, v_storage):
        self.handle = handle
        self.desc = desc
        self.k_storage = k_storage
        self.v_storage = v_storage

    def __del__(self):
        try:
            astro_kvcache_destroy(self)
        except Exception:
            pass


def astro_kvcache_create(cache_batch, heads, head_dim, tokens_per_frame, sink_frames, window_frames,
                         k_storage=None, v_storage=None, device="cuda") -> KVCache:
    """Bind storage (torch uint8/bf16 tensors; allocated here with torch when not given) to a new cache."""
    import torch
    d = _desc(cache_batch, heads, head_dim, tokens_per_frame, sink_frames, window_frames)
    nbytes = int(lib().astro_kvcache_storage_bytes(C.byref(d)))
    if nbytes == 0:
        raise AstroError(2, "astro_kvcache_storage_bytes")
    if k_storage is None:
        k_storage = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if v_storage is None:
        v_storage = torch.empty(nbytes, dtype=torch.uint8, device=device)
    out = C.c_void_p()
    st = lib().astro_kvcache_create(C.byref(d), _ptr(k_storage), _ptr(v_storage),
                                    min(k_storage.numel() * k_storage.element_size(),
                                        v_storage.numel() * v_storage.element_size()), C.byref(out))
    _check(st, "astro_kvcache_create")
    return KVCache(out, d, k_storage, v_storage)


def astro_kvcache_destroy(cache: KVCache) -> None:
    if cache.handle is not None and _lib is not None:
        h, cache.handle = cache.handle, None
        _check(_lib.astro_kvcache_destroy(h), "astro_kvcache_destroy")


def astro_kvcache_reset(cache: KVCache) -> None:
    _check(lib().astro_kvcache_reset(cache.handle), "astro_kvcache_reset")


def astro_kvcache_append(cache: KVCache, k, v, n_frames: int, stream=None) -> None:
    """k, v: bf16 [B_c, n_frames*T, H, D] on the device."""
    _check(lib().astro_kvcache_append(cache.handle, _ptr(k), _ptr(v), _int(n_frames), _stream(stream)),
           "astro_kvcache_append")


def astro_kvcache_evict(cache: KVCache, n_frames: int, stream=None) -> None:
    _check(lib().astro_kvcache_evict(cache.handle, _int(n_frames), None), "astro_kvcache_evict")


def astro_kvcache_query(cache: KVCache):
    """Returns (sink_held, window_held, frames_seen)."""
    a, b, c = C.c_int(), C.c_int(), C.c_int64()
    _check(lib().astro_kvcache_query(cache.handle, C.byref(a), C.byref(b), C.byref(c)), "astro_kvcache_query")
    return a.value, b.value, c.value


def astro_kvcache_get_state(cache: KVCache) -> KVCacheState:
    st = KVCacheState()
    _check(lib().astro_kvcache_get_state(cache.handle, C.byref(st)), "astro_kvcache_get_state")
    return st


def astro_kvcache_set_state(cache: KVCache, state: KVCacheState) -> None:
    _check(lib().astro_kvcache_set_state(cache.handle, C.byref(state)), "astro_kvcache_set_state")


def astro_kvcache_key_segments(cache, n_kc: int):
    """List of (first_token, token_count, from_chunk) the attention kernels would walk (host only)."""
    n = C.c_int()
    a, b, c = (C.c_int * 3)(), (C.c_int * 3)(), (C.c_int * 3)()
    _check(lib().astro_kvcache_key_segments(_cache(cache), _int(n_kc), C.byref(n), a, b, c),
           "astro_kvcache_key_segments")
    return [(a[i], b[i], c[i]) for i in range(n.value)]


def astro_kvcache_export(cache: KVCache, stream=None):
    """Held frames in logical order as two bf16 tensors [B_c, held*T, H, D]."""
    import torch
    sink, win, _ = astro_kvcache_query(cache)
    d = cache.desc
    shape = (d.cache_batch, (sink + win) * d.tokens_per_frame, d.heads, d.head_dim)
    with _owned_by(stream):
        k = torch.empty(shape, dtype=torch.bfloat16, device=cache.k_storage.device)
        v = torch.empty_like(k)
    _used_here(stream, k, v)
    if sink + win:
        _check(lib().astro_kvcache_export(cache.handle, _ptr(k), _ptr(v), _stream(stream)), "astro_kvcache_export")
    return k, v


def astro_chunk_attn_fwd(cache, q, k_chunk, v_chunk, scale: float, o=None, lse=None, stream=None):
    """q [B, n_q, H, D], k_chunk/v_chunk [B, n_kc, H, D] or None; returns (O bf16, LSE fp32 [B, H, n_q])."""
    import torch
    B, n_q, H, D = q.shape
    n_kc = 0 if k_chunk is None else k_chunk.shape[1]
    fresh = []
    with _owned_by(stream):
        if o is None:
            o = torch.empty_like(q); fresh.append(o)
        if lse is None:
            lse = torch.empty((B, H, n_q), dtype=torch.float32, device=q.device); fresh.append(lse)
    _contiguous(q, k_chunk, v_chunk, o, lse)
    _used_here(stream, *fresh)
    st = lib().astro_chunk_attn_fwd(_cache(cache), _ptr(q), _ptr(k_chunk), _ptr(v_chunk),
                                    B, H, D, n_q, n_kc, float(scale), _ptr(o), _ptr(lse), _stream(stream))
    _check(st, "astro_chunk_attn_fwd")
    return o, lse


def astro_chunk_attn_bwd_workspace_bytes(batch, heads, n_q, head_dim) -> int:
    return int(lib().astro_chunk_attn_bwd_workspace_bytes(_int(batch), _int(heads), _int(n_q), _int(head_dim)))


def astro_chunk_attn_bwd(cache, q, k_chunk, v_chunk, o, lse, d_o, scale: float, dq=None, dk_chunk=None,
                         dv_chunk=None, workspace=None, stream=None):
    """Returns (dQ, dK_chunk, dV_chunk), bf16; the cached context receives no gradient."""
    import torch
    B, n_q, H, D = q.shape
    n_kc = 0 if k_chunk is None else k_chunk.shape[1]
    fresh = []
    with _owned_by(stream):
        if dq is None:
            dq = torch.empty_like(q); fresh.append(dq)
        if n_kc and dk_chunk is None:
            dk_chunk = torch.empty_like(k_chunk); fresh.append(dk_chunk)
        if n_kc and dv_chunk is None:
            dv_chunk = torch.empty_like(v_chunk); fresh.append(dv_chunk)
        if workspace is None:
            need = astro_chunk_attn_bwd_workspace_bytes(B, H, n_q, D)
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device); fresh.append(workspace)
    _contiguous(q, k_chunk, v_chunk, o, lse, d_o, dq, dk_chunk, dv_chunk)
    _used_here(stream, *fresh)
    st = lib().astro_chunk_attn_bwd(_cache(cache), _ptr(q), _ptr(k_chunk), _ptr(v_chunk),
                                    _ptr(o), _ptr(lse), _ptr(d_o), B, H, D, n_q, n_kc, float(scale), _ptr(dq),
                                    _ptr(dk_chunk), _ptr(dv_chunk), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "astro_chunk_attn_bwd")
    return dq, dk_chunk, dv_chunk


def astro_chunk_attn_bwd_delta(o, d_o, delta=None, stream=None):
    """delta [B, H, n_q] fp32 = rowsum(dO * O)."""
    import torch
    B, n_q, H, D = o.shape
    if delta is None:
        with _owned_by(stream):
            delta = torch.empty((B, H, n_q), dtype=torch.float32, device=o.device)
        _used_here(stream, delta)
    _contiguous(o, d_o, delta)
    _check(lib().astro_chunk_attn_bwd_delta(_ptr(o), _ptr(d_o), B, H, D, n_q, _ptr(delta), _stream(stream)),
           "astro_chunk_attn_bwd_delta")
    return delta


def astro_chunk_attn_bwd_dq(cache, q, k_chunk, v_chunk, lse, delta, d_o, scale: float, dq=None, stream=None):
    import torch
    B, n_q, H, D = q.shape
    n_kc = 0 if k_chunk is None else k_chunk.shape[1]
    if dq is None:
        with _owned_by(stream):
            dq = torch.empty_like(q)
        _used_here(stream, dq)
    _contiguous(q, k_chunk, v_chunk, lse, delta, d_o, dq)
    st = lib().astro_chunk_attn_bwd_dq(_cache(cache), _ptr(q), _ptr(k_chunk), _ptr(v_chunk),
                                       _ptr(lse), _ptr(delta), _ptr(d_o), B, H, D, n_q, n_kc, float(scale), _ptr(dq),
                                       _stream(stream))
    _check(st, "astro_chunk_attn_bwd_dq")
    return dq


def astro_chunk_attn_bwd_dkv(q, k_chunk, v_chunk, lse, delta, d_o, scale: float, dk_chunk=None, dv_chunk=None,
                             stream=None):
    import torch
    B, n_q, H, D = q.shape
    n_kc = k_chunk.shape[1]
    fresh = []
    with _owned_by(stream):
        if dk_chunk is None:
            dk_chunk = torch.empty_like(k_chunk); fresh.append(dk_chunk)
        if dv_chunk is None:
            dv_chunk = torch.empty_like(v_chunk); fresh.append(dv_chunk)
    _used_here(stream, *fresh)
    _contiguous(q, k_chunk, v_chunk, lse, delta, d_o, dk_chunk, dv_chunk)
    st = lib().astro_chunk_attn_bwd_dkv(_ptr(q), _ptr(k_chunk), _ptr(v_chunk), _ptr(lse), _ptr(delta), _ptr(d_o), B, H,
                                        D, n_q, n_kc, float(scale), _ptr(dk_chunk), _ptr(dv_chunk), _stream(stream))
    _check(st, "astro_chunk_attn_bwd_dkv")
    return dk_chunk, dv_chunk


def _frame_list(frames):
    """(C array, count) of a list of frame indices, (None, -1) for all."""
    if frames is None:
        return None, -1
    n = len(frames)
    return (C.c_int * max(1, n))(*[_int(f) for f in frames]), n


def astro_kvcache_fork(dst: KVCache, src: KVCache, parents=None, frames=None, stream=None) -> None:
    """Empty `dst` and copy the listed held frames of `src` (logical indices, None = all) into it; parents: int32 [dst
    cache_batch] on the device, the sample of src that each sample of dst continues."""
    import torch
    dev, on = _where(stream, dst.k_storage)
    if parents is not None:
        _like((dst.desc.cache_batch,), torch.int32, dev, parents)
    arr, n = _frame_list(frames)
    _check(lib().astro_kvcache_fork(_handle(dst, dev), _handle(src, dev), _at(parents), arr, n, on), "astro_kvcache_fork")


ROPE_LAYOUTS = {"interleaved": 0, "halves": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "ramp": 3}


class Rope:
    """Handle of one table of rotary frequencies (host memory only)."""

    def __init__(self, handle, desc):
        self.handle = handle
        self.desc = desc

    def __del__(self):
        try:
            astro_rope_destroy(self)
        except Exception:
            pass


def astro_rope_create(head_dim, rot_dim, layout, axis_pairs, base=10000.0, scaling="none", factor=1.0, scaled_axes=None,
                      original_length=4096.0, ramp_low=1.0, ramp_high=32.0, magnitude=0.0) -> Rope:
    """axis_pairs: pairs of each position axis, e.g. (64,) or (22, 21, 21); scaled_axes: axes that `scaling` applies to
    (None = all); magnitude 0 = the scaling's own."""
    if len(axis_pairs) > 4:
        raise AstroError(2, "astro_rope_create")
    axes = range(len(axis_pairs)) if scaled_axes is None else [int(a) for a in scaled_axes]
    if any(not 0 <= a < len(axis_pairs) for a in axes):
        raise AstroError(2, "astro_rope_create")
    d = RopeDesc(_int(head_dim), _int(rot_dim), ROPE_LAYOUTS[layout], len(axis_pairs), (C.c_int * 4)(*[_int(p) for p in axis_pairs]),
                 float(base), ROPE_SCALINGS[scaling], sum({1 << a for a in axes}), float(factor), float(original_length),
                 float(ramp_low), float(ramp_high), float(magnitude))
    out = C.c_void_p()
    _check(lib().astro_rope_create(C.byref(d), C.byref(out)), "astro_rope_create")
    return Rope(out, d)


def astro_rope_destroy(rope: Rope) -> None:
    if rope.handle is not None and _lib is not None:
        h, rope.handle = rope.handle, None
        _check(_lib.astro_rope_destroy(h), "astro_rope_destroy")


def astro_rope_frequencies(rope: Rope):
    """(radians per position of every pair, factor on cosines and sines)."""
    f, m = (C.c_double * (rope.desc.rot_dim // 2))(), C.c_double()
    _check(lib().astro_rope_frequencies(rope.handle, f, C.byref(m)), "astro_rope_frequencies")
    return list(f), m.value


def _rope_strides(t):
    """(batch, token, head) strides, those of axes of size 1 as in a contiguous tensor (torch leaves them open)."""
    B, n, H, D = t.shape
    dense = (n * H * D, H * D, D)
    return tuple(s if size > 1 else d for s, size, d in zip(t.stride(), (B, n, H), dense))


def _dense_like(t):
    import torch
    # empty_like keeps the strides of a dense tensor, and is the cheaper of the two where they are the contiguous ones
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


_ROPE_TYPES = {}


def astro_rope_apply(rope: Rope, q, k, positions, inverse: bool = False, q_out=None, k_out=None, stream=None):
    """Rotate q [B, n, H, D] and k (same type; other head count allowed; None: q alone) by their tokens' positions, int32
    [B or 1, n, axes] on the device.  Inputs and outputs may be strided as long as a head's elements are contiguous;
    q_out = q and k_out = k rotate in place.  inverse=True turns back: the gradient of q and k from that of the outputs."""
    import torch
    if not _ROPE_TYPES:
        _ROPE_TYPES.update({torch.bfloat16: 0, torch.float16: 1, torch.float32: 2})
    kind = _ROPE_TYPES.get(q.dtype)
    if kind is None:
        raise ValueError("q and k must be bf16, fp16 or fp32")
    shape = q.shape
    if len(shape) != 4 or shape[3] != rope.desc.head_dim:
        raise ValueError("q must be [B, n, heads, head_dim]")
    B, n, H, _ = shape
    dev, on = _where(stream, q)
    fresh = []
    if q_out is None:
        with _owned_by(stream):
            q_out = _dense_like(q); fresh.append(q_out)
    elif q_out.shape != shape or q_out.dtype is not q.dtype or q_out.get_device() != dev:
        raise ValueError("q_out must be like q")
    if k is not None:
        if k.dim() != 4 or k.dtype is not q.dtype or k.shape[0] != B or k.shape[1] != n or k.shape[3] != shape[3] or k.get_device() != dev:
            raise ValueError("k must be [B, n, heads, head_dim] of q's type, beside it")
        if k_out is None:
            with _owned_by(stream):
                k_out = _dense_like(k); fresh.append(k_out)
        elif k_out.shape != k.shape or k_out.dtype is not k.dtype or k_out.get_device() != dev:
            raise ValueError("k_out must be like k")
    else:
        k_out = None
    pb = positions.shape[0]
    if pb != 1 and pb != B:
        raise ValueError("positions must be [B or 1, n, axes]")
    _like((pb, n, rope.desc.axes), torch.int32, dev, positions)
    _used_here(stream, *fresh)

    def arguments(x, x2, y, y2, strides):
        return (rope.handle, 1 if inverse else 0, _at(x), _at(x2), _at(positions), pb, B, _int(n), x.shape[2],
                0 if x2 is None else x2.shape[2], kind, None if strides is None else C.byref(Strides(*strides[0])), _at(y), _at(y2),
                None if strides is None else C.byref(Strides(*strides[1])))

    def call(*of):
        _check(lib().astro_rope_apply(*arguments(*of), on), "astro_rope_apply")

    dense = q.is_contiguous() and q_out.is_contiguous()
    if dense and (k is None or (k.shape == shape and k.is_contiguous() and k_out.is_contiguous())):
        call(q, k, q_out, k_out, None)
        return q_out, k_out
    pairs = [(x, y) for x, y in ((q, q_out), (k, k_out)) if x is not None]
    if n and any(z.stride(3) != 1 for pair in pairs for z in pair):
        raise ValueError("the elements of a head must be contiguous")
    layouts = [(_rope_strides(x), _rope_strides(y)) for x, y in pairs]
    if len(pairs) == 2 and layouts[0] == layouts[1]:   # one launch for q and k; two where their strides differ
        call(q, k, q_out, k_out, layouts[0])
    else:
        if len(pairs) == 2:                            # neither if one is refused, and none reads what the other has written
            if q_out.data_ptr() in (k.data_ptr(), k_out.data_ptr()) or k_out.data_ptr() == q.data_ptr():
                if n:
                    raise AstroError(2, "astro_rope_apply")
            for (x, y), layout in zip(pairs, layouts):
                _check(lib().astro_rope_apply_check(*arguments(x, None, y, None, layout)), "astro_rope_apply")
        for (x, y), layout in zip(pairs, layouts):
            call(x, None, y, None, layout)
    return q_out, k_out


QUERY_BLOCK = 128
KEEP_SINK, KEEP_CHUNK = 1, 2


def astro_block_count(cache, n_kc: int, block_tokens: int):
    """(cache blocks, chunk blocks) that a call numbers (host only)."""
    a, b = C.c_int(), C.c_int()
    _check(lib().astro_block_count(_cache(cache), _int(n_kc), _int(block_tokens), C.byref(a), C.byref(b)),
           "astro_block_count")
    return a.value, b.value


def _pooled_shape(cache, block_tokens):
    d = cache.desc
    return (d.cache_batch, d.heads, d.sink_frames + d.window_frames, -(-d.tokens_per_frame // _int(block_tokens)), d.head_dim)


def astro_block_pool(cache: KVCache, block_tokens: int, first_frame: int = 0, n_frames=None, pooled=None, stream=None):
    """Means of the keys of the blocks of `n_frames` held frames from `first_frame` on (None: all behind it), fp32 [B_c, H,
    S+L, blocks per frame, D] by storage slot; `pooled` keeps the means of the other frames."""
    import torch
    if n_frames is None:
        sink, win, _ = astro_kvcache_query(cache)
        n_frames = sink + win - _int(first_frame)
    dev, on = _where(stream, cache.k_storage)
    if _int(block_tokens) < 1:
        raise AstroError(2, "astro_block_pool")
    shape = _pooled_shape(cache, block_tokens)
    if pooled is None:
        with _owned_by(stream):   # and cleared there too: on another stream the clearing could wipe the means
            pooled = torch.zeros(shape, dtype=torch.float32, device=cache.k_storage.device)
        _used_here(stream, pooled)
    else:
        _like(shape, torch.float32, dev, pooled)
    _check(lib().astro_block_pool(_handle(cache, dev), _int(first_frame), _int(n_frames), _int(block_tokens), _at(pooled), on),
           "astro_block_pool")
    return pooled


def astro_block_select_workspace_bytes(batch, heads, head_dim, n_q, n_kc, block_tokens) -> int:
    return int(lib().astro_block_select_workspace_bytes(_int(batch), _int(heads), _int(head_dim), _int(n_q), _int(n_kc), _int(block_tokens)))


def astro_block_select(cache, pooled, q, k_chunk, block_tokens: int, n_select: int, keep: int = 0, blocks=None, workspace=None,
                       stream=None):
    """int32 [B, H, ceil(n_q / QUERY_BLOCK), n_select]: per query block the key blocks of the highest scores, ascending,
    -1 behind them.  pooled: astro_block_pool's means of every held frame (None without a cache)."""
    import torch
    dev, on = _where(stream, q)
    B, n_q, H, D = q.shape
    _like(q.shape, torch.bfloat16, dev, q)
    n_kc = _chunk(q, dev, k_chunk, None)
    shape = (B, H, (n_q + QUERY_BLOCK - 1) // QUERY_BLOCK, max(1, _int(n_select)))
    if blocks is not None:
        _like(shape, torch.int32, dev, blocks)
    fresh = []
    with _owned_by(stream):
        if blocks is None:
            blocks = q.new_empty(shape, dtype=torch.int32); fresh.append(blocks)
        if workspace is None:
            need = astro_block_select_workspace_bytes(B, H, D, n_q, n_kc, block_tokens)
            workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device); fresh.append(workspace)
    if pooled is not None and cache is not None and _int(block_tokens) >= 1:
        _like(_pooled_shape(cache, block_tokens), torch.float32, dev, pooled)
    _used_here(stream, *fresh)
    st = lib().astro_block_select(_handle(cache, dev), _at(pooled), _at(q), _at(k_chunk), B, H, D, n_q, n_kc, _int(block_tokens),
                                  _int(n_select), _int(keep), _at(blocks), *_scratch(workspace, dev), on)
    _check(st, "astro_block_select")
    return blocks


def astro_sparse_attn_fwd_workspace_bytes(batch, heads, head_dim, n_q, n_select, block_tokens) -> int:
    return int(lib().astro_sparse_attn_fwd_workspace_bytes(_int(batch), _int(heads), _int(head_dim), _int(n_q), _int(n_select),
                                                           _int(block_tokens)))


def astro_sparse_attn_fwd(cache, q, k_chunk, v_chunk, blocks, block_tokens: int, scale: float, o=None, lse=None, workspace=None,
                          stream=None):
    """Attention of every query block over the key blocks its list names (blocks: int32 [B, H, ceil(n_q / QUERY_BLOCK),
    n_select] on the device, -1 for none); returns (O bf16, LSE fp32 [B, H, n_q]); a query without a key gets 0 and
    -infinity."""
    import torch
    dev, on = _where(stream, q)
    shape = q.shape
    B, n_q, H, D = shape
    _like(shape, torch.bfloat16, dev, q, o)
    n_kc, n_select = _chunk(q, dev, k_chunk, v_chunk), _lists(q, dev, blocks)
    if lse is not None:
        _like((B, H, n_q), torch.float32, dev, lse)
    fresh = []
    with _owned_by(stream):
        if o is None:
            o = torch.empty_like(q); fresh.append(o)
        if lse is None:
            lse = q.new_empty((B, H, n_q), dtype=torch.float32); fresh.append(lse)
        if workspace is None:
            need = astro_sparse_attn_fwd_workspace_bytes(B, H, D, n_q, n_select, block_tokens)
            if need:
                workspace = torch.empty(need, dtype=torch.uint8, device=q.device); fresh.append(workspace)
    _used_here(stream, *fresh)
    st = lib().astro_sparse_attn_fwd(_handle(cache, dev), _at(q), _at(k_chunk), _at(v_chunk), _at(blocks), n_select,
                                     _int(block_tokens), B, H, D, n_q, n_kc, float(scale), _at(o), _at(lse),
                                     *_scratch(workspace, dev), on)
    _check(st, "astro_sparse_attn_fwd")
    return o, lse


def astro_sparse_attn_bwd_workspace_bytes(batch, heads, head_dim, n_q, n_kc, n_select, block_tokens) -> int:
    return int(lib().astro_sparse_attn_bwd_workspace_bytes(_int(batch), _int(heads), _int(head_dim), _int(n_q), _int(n_kc),
                                                           _int(n_select), _int(block_tokens)))


def astro_sparse_attn_bwd(cache, q, k_chunk, v_chunk, blocks, block_tokens: int, o, lse, d_o, scale: float, dq=None, dk_chunk=None,
                          dv_chunk=None, workspace=None, stream=None):
    """Returns (dQ, dK_chunk, dV_chunk), bf16, of astro_sparse_attn_fwd with the same lists; the cached context receives no
    gradient."""
    import torch
    dev, on = _where(stream, q)
    shape = q.shape
    B, n_q, H, D = shape
    _like(shape, torch.bfloat16, dev, q, o, d_o, dq)
    _like((B, H, n_q), torch.float32, dev, lse)
    n_kc, n_select = _chunk(q, dev, k_chunk, v_chunk, dk_chunk, dv_chunk), _lists(q, dev, blocks)
    fresh = []
    with _owned_by(stream):
        if dq is None:
            dq = torch.empty_like(q); fresh.append(dq)
        if n_kc and dk_chunk is None:
            dk_chunk = torch.empty_like(k_chunk); fresh.append(dk_chunk)
        if n_kc and dv_chunk is None:
            dv_chunk = torch.empty_like(v_chunk); fresh.append(dv_chunk)
        if workspace is None:
            need = astro_sparse_attn_bwd_workspace_bytes(B, H, D, n_q, n_kc, n_select, block_tokens)
            workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device); fresh.append(workspace)
    _used_here(stream, *fresh)
    st = lib().astro_sparse_attn_bwd(_handle(cache, dev), _at(q), _at(k_chunk), _at(v_chunk), _at(blocks), n_select,
                                     _int(block_tokens), _at(o), _at(lse), _at(d_o), B, H, D, n_q, n_kc, float(scale), _at(dq),
                                     _at(dk_chunk), _at(dv_chunk), *_scratch(workspace, dev), on)
    _check(st, "astro_sparse_attn_bwd")
    return dq, dk_chunk, dv_chunk


def astro_nft_loss(v_theta, v_old, v_ref, v_target, r_tilde, beta: float, w_policy=None, w_kl=None, grad=True,
                   stream=None, out=None):
    """Per-sample policy loss and squared distance to the reference, plus d/d v_theta of the weighted total.

    Velocity tensors: bf16 [B, ...] (flattened per sample); r_tilde / weights: fp32 [B].  Returns
    (policy[B], kl[B] or None, grad like v_theta or None); `out` may pass those three preallocated."""
    import torch
    B = v_theta.shape[0]
    elems = v_theta.numel() // B
    if out is not None:
        policy, kl, g = out
    else:
        with _owned_by(stream):
            policy = torch.empty(B, dtype=torch.float32, device=v_theta.device)
            kl = None if v_ref is None else torch.empty(B, dtype=torch.float32, device=v_theta.device)
            g = torch.empty_like(v_theta) if grad else None
        _used_here(stream, policy, kl, g)
    _contiguous(v_theta, v_old, v_ref, v_target, g)
    st = lib().astro_nft_loss(_ptr(v_theta), _ptr(v_old), _ptr(v_ref), _ptr(v_target), _ptr(r_tilde), _ptr(w_policy),
                              _ptr(w_kl), B, elems, float(beta), _ptr(policy), _ptr(kl), _ptr(g), _stream(stream))
    _check(st, "astro_nft_loss")
    return policy, kl, g


BWD_STATIC_MAX_ROWS = 262144


def astro_chunk_attn_bwd_static(cache, q, k_chunk, v_chunk, o, lse, d_o, scale: float, dq, dk_chunk, dv_chunk,
                                stream=None):
    """Backward for callers that may not allocate: no workspace argument, delta goes to a fixed 1 MiB
    device array inside the library (batch * heads * n_q <= BWD_STATIC_MAX_ROWS).  The caller passes every
    output tensor; this wrapper allocates nothing either.  Calls that may overlap on the GPU race on the
    shared array; issue them on one stream."""
    B, n_q, H, D = q.shape
    n_kc = 0 if k_chunk is None else k_chunk.shape[1]
    _contiguous(q, k_chunk, v_chunk, o, lse, d_o, dq, dk_chunk, dv_chunk)
    st = lib().astro_chunk_attn_bwd_static(_cache(cache), _ptr(q), _ptr(k_chunk),
                                           _ptr(v_chunk), _ptr(o), _ptr(lse), _ptr(d_o), B, H, D, n_q, n_kc,
                                           float(scale), _ptr(dq), _ptr(dk_chunk), _ptr(dv_chunk), _stream(stream))
    _check(st, "astro_chunk_attn_bwd_static")
    return dq, dk_chunk, dv_chunk


FWD_MODE_NORMAL, FWD_MODE_SAFE_ONLY, FWD_MODE_PAIR = 0, 1, 2


def astro_debug_forward_mode(mode: int) -> None:
    """Diagnostic switch: 0 normal operation, 1 every later forward runs its safe pass only, 2 head_dim 128
    forwards run the CTA-pair kernel."""
    _check(lib().astro_debug_forward_mode(_int(mode)), "astro_debug_forward_mode")


def astro_debug_pair_flag() -> int:
    """Synchronises; 1 if a CTA-pair forward since the last call had a row that needs the safe pass (cleared)."""
    f = C.c_int()
    _check(lib().astro_debug_pair_flag(C.byref(f)), "astro_debug_pair_flag")
    return f.value


def astro_selftest_wait_timeout(stream=None) -> None:
    """Enqueue the bounded-wait self-test kernel (its wait runs out on purpose; see astro_last_device_status)."""
    _check(lib().astro_selftest_wait_timeout(_stream(stream)), "astro_selftest_wait_timeout")


def astro_last_device_status() -> int:
    """Synchronises, reads and clears the device status word; raises AstroError on a recorded timeout."""
    detail = C.c_uint32()
    st = lib().astro_last_device_status(C.byref(detail))
    _check(st, "astro_last_device_status (detail 0x%x)" % detail.value)
    return detail.value
