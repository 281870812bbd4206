"""ctypes binding of libmoba.so (C ABI in include/moba.h).

Argument marshalling only: torch tensors are described to the library as
(pointer, dtype, shape, strides) and the caller's current HIP stream is passed
through; every step of the computation runs in the library's HIP kernels.
There is no fallback: if libmoba.so is missing or fails to load, every call
raises.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoba.so")

MOBA_F32, MOBA_BF16, MOBA_I32, MOBA_I64, MOBA_F8E4M3, MOBA_F64 = 0, 1, 2, 3, 4, 5
_DT = {torch.float32: MOBA_F32, torch.bfloat16: MOBA_BF16, torch.int32: MOBA_I32,
       torch.int64: MOBA_I64, torch.float8_e4m3fn: MOBA_F8E4M3}

STATUS = ["MOBA_OK", "MOBA_ERR_NULL", "MOBA_ERR_DTYPE", "MOBA_ERR_SHAPE", "MOBA_ERR_LAYOUT",
          "MOBA_ERR_BLOCK_SIZE", "MOBA_ERR_TOPK", "MOBA_ERR_SEQLENS", "MOBA_ERR_UNSUPPORTED",
          "MOBA_ERR_NO_MEMORY", "MOBA_ERR_HIP"]


class MobaTensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("ndim", ctypes.c_int32),
                ("shape", ctypes.c_int64 * 4), ("stride", ctypes.c_int64 * 4)]


class PhaseStat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 24), ("launches", ctypes.c_int64),
                ("total_ms", ctypes.c_double)]


class MobaError(RuntimeError):
    def __init__(self, fn: str, status: int):
        name = STATUS[status] if 0 <= status < len(STATUS) else str(status)
        super().__init__("%s failed: %s" % (fn, name))
        self.status = status
        self.name = name


_lib = None


def load() -> ctypes.CDLL:
    """Load libmoba.so once.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libmoba.so not found at %s; build it with "
                           "`python -m paper_2502_13189_amd.build`" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER(MobaTensor)
    vp, i32 = ctypes.c_void_p, ctypes.c_int32
    sig = {
        "moba_forward": [P, P, P, P, i32, i32, P, P, vp],
        "moba_backward": [P, P, P, P, i32, i32, P, P, P, P, P, P, vp],
        "moba_dense_backward": [P, P, P, P, P, P, P, P, P, P, vp],
        "moba_decode": [P, P, P, P, P, i32, i32, P, P, vp],
        "moba_decode_noalloc": [P, P, P, P, P, i32, i32, P, P, vp],
        "moba_dense_forward": [P, P, P, P, P, P, vp],
        "moba_pool": [P, P, i32, P, vp],
        "moba_select": [P, P, P, i32, i32, P, P, vp],
        "moba_route": [P, P, i32, i32, P, P, P, vp],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = ctypes.c_int
    i64 = ctypes.c_int64
    for name, args in {
        "moba_cache_plan": [vp] * 5 + [i32] + [vp] * 6,
        "moba_cache_write": [vp] * 5,
        "moba_cache_decode": [vp] * 4 + [i32, i32] + [vp] * 3 + [ctypes.c_size_t, vp],
        "moba_rope": [vp] * 6,
        "moba_rope_backward": [vp] * 6,
        "moba_latent_forward": [vp] * 5 + [ctypes.c_float] + [vp] * 3,
        "moba_latent_backward": [vp] * 5 + [ctypes.c_float] + [vp] * 8 + [ctypes.c_size_t, vp],
        "moba_latent_write": [vp] * 6,
        "moba_latent_decode": [vp] * 5 + [ctypes.c_float] + [vp] * 3 + [ctypes.c_size_t, vp],
    }.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = ctypes.c_int
    lib.moba_cache_decode_workspace_bytes.restype = ctypes.c_size_t
    lib.moba_cache_decode_workspace_bytes.argtypes = [i64, i64, i32, i32, i32, i32, i32]
    lib.moba_latent_backward_workspace_bytes.restype = ctypes.c_size_t
    lib.moba_latent_backward_workspace_bytes.argtypes = [i64, i32]
    lib.moba_latent_decode_workspace_bytes.restype = ctypes.c_size_t
    lib.moba_latent_decode_workspace_bytes.argtypes = [i64, i64, i32, i32]
    lib.moba_workspace_bytes.restype = ctypes.c_size_t
    lib.moba_workspace_bytes.argtypes = [i64, i32, i32, i32, i64, i32]
    lib.moba_workspace_held_bytes.restype = ctypes.c_size_t
    lib.moba_workspace_held_bytes.argtypes = []
    lib.moba_route_size.restype = ctypes.c_int
    lib.moba_route_size.argtypes = [P, i32, i32, i32, ctypes.POINTER(i64), ctypes.POINTER(i64), vp]
    lib.moba_take_wait_timeouts.restype = ctypes.c_int
    lib.moba_take_wait_timeouts.argtypes = [ctypes.POINTER(ctypes.c_uint64)]
    lib.moba_release_workspace.restype = ctypes.c_int
    lib.moba_release_workspace.argtypes = []
    lib.moba_status_string.restype = ctypes.c_char_p
    lib.moba_status_string.argtypes = [ctypes.c_int]
    lib.moba_profile_enable.argtypes = [ctypes.c_int]
    lib.moba_profile_enable.restype = None
    lib.moba_profile_read.argtypes = [ctypes.POINTER(PhaseStat), ctypes.c_int]
    lib.moba_profile_read.restype = ctypes.c_int
    _lib = lib
    return lib


def describe(t: torch.Tensor) -> MobaTensor:
    """Descriptor of a tensor (its storage stays owned by the caller)."""
    if t.dtype not in _DT:
        raise TypeError("unsupported dtype %s" % t.dtype)
    if t.dim() > 4:
        raise ValueError("at most 4 dimensions")
    d = MobaTensor()
    d.data = t.data_ptr()
    d.dtype = _DT[t.dtype]
    d.ndim = t.dim()
    for i in range(t.dim()):
        d.shape[i] = t.shape[i]
        d.stride[i] = t.stride(i)
    return d


def _ref(d):
    return None if d is None else ctypes.byref(d)


def _stream(t: torch.Tensor, stream=None) -> int:
    if stream is not None:
        return int(stream.cuda_stream if hasattr(stream, "cuda_stream") else stream)
    if t.is_cuda:
        return int(torch.cuda.current_stream(t.device).cuda_stream)
    return 0


def _check(fn: str, status: int):
    if status != 0:
        raise MobaError(fn, status)


def _cu(cu_seqlens) -> torch.Tensor:
    if not isinstance(cu_seqlens, torch.Tensor):
        cu_seqlens = torch.tensor(list(cu_seqlens), dtype=torch.int32)
    if cu_seqlens.dtype != torch.int32:
        cu_seqlens = cu_seqlens.to(torch.int32)
    return cu_seqlens.contiguous()


def forward(q, k, v, cu_seqlens, block_size: int, topk: int, out=None, lse=None, stream=None):
    """MoBA causal prefill forward.  q [T, Hq, 128], k/v [T, Hkv, 128] (bf16 or
    fp32, on the GPU); cu_seqlens [S+1] int32 (host tensor keeps the call
    asynchronous).  Returns (out [T, Hq, 128], lse [Hq, T] fp32)."""
    lib = load()
    cu = _cu(cu_seqlens)
    T, Hq = q.shape[0], q.shape[1]
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if lse is None:
        lse = torch.empty((Hq, T), dtype=torch.float32, device=q.device)
    dq, dk, dv, dc, do, dl = map(describe, (q, k, v, cu, out, lse))
    _check("moba_forward", lib.moba_forward(_ref(dq), _ref(dk), _ref(dv), _ref(dc), int(block_size),
                                            int(topk), _ref(do), _ref(dl), _stream(q, stream)))
    return out, lse


def backward(q, k, v, cu_seqlens, block_size: int, topk: int, out, lse, dout, dq=None, dk=None,
             dv=None, stream=None):
    """Gradients of forward() w.r.t. q, k, v (bf16).  out and lse are forward()'s
    results for the same inputs; dout [T, Hq, 128] is the gradient w.r.t. out.
    Returns (dq [T, Hq, 128], dk [T, Hkv, 128], dv [T, Hkv, 128])."""
    lib = load()
    cu = _cu(cu_seqlens)
    if dq is None:
        dq = torch.empty_like(q, memory_format=torch.contiguous_format)
    if dk is None:
        dk = torch.empty_like(k, memory_format=torch.contiguous_format)
    if dv is None:
        dv = torch.empty_like(v, memory_format=torch.contiguous_format)
    d = [describe(t) for t in (q, k, v, cu, out, lse, dout, dq, dk, dv)]
    _check("moba_backward", lib.moba_backward(_ref(d[0]), _ref(d[1]), _ref(d[2]), _ref(d[3]),
                                              int(block_size), int(topk), _ref(d[4]), _ref(d[5]),
                                              _ref(d[6]), _ref(d[7]), _ref(d[8]), _ref(d[9]),
                                              _stream(q, stream)))
    return dq, dk, dv


def dense_backward(q, k, v, cu_seqlens, out, lse, dout, dq=None, dk=None, dv=None, stream=None):
    """Gradients of dense_forward() (causal full attention) w.r.t. q, k, v (bf16)."""
    lib = load()
    cu = _cu(cu_seqlens)
    if dq is None:
        dq = torch.empty_like(q, memory_format=torch.contiguous_format)
    if dk is None:
        dk = torch.empty_like(k, memory_format=torch.contiguous_format)
    if dv is None:
        dv = torch.empty_like(v, memory_format=torch.contiguous_format)
    d = [describe(t) for t in (q, k, v, cu, out, lse, dout, dq, dk, dv)]
    _check("moba_dense_backward", lib.moba_dense_backward(
        _ref(d[0]), _ref(d[1]), _ref(d[2]), _ref(d[3]), _ref(d[4]), _ref(d[5]), _ref(d[6]),
        _ref(d[7]), _ref(d[8]), _ref(d[9]), _stream(q, stream)))
    return dq, dk, dv


def decode(q, k_cache, v_cache, cu_seqlens, block_size: int, topk: int, kbar=None, out=None,
           lse=None, stream=None):
    """One new query per sequence against its cache (topk == 0: full
    attention).  q [S, Hq, 128] bf16; k_cache/v_cache [T, Hkv, 128] bf16 with
    each new token's key/value last in its sequence; kbar: optional block
    means from pool().  Returns (out [S, Hq, 128], lse [Hq, S])."""
    lib = load()
    cu = _cu(cu_seqlens)
    S, Hq = q.shape[0], q.shape[1]
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if lse is None:
        lse = torch.empty((Hq, S), dtype=torch.float32, device=q.device)
    d = [describe(t) for t in (q, k_cache, v_cache, cu)]
    dkb = describe(kbar) if kbar is not None else None
    do, dl = describe(out), describe(lse)
    _check("moba_decode", lib.moba_decode(_ref(d[0]), _ref(d[1]), _ref(d[2]), _ref(d[3]),
                                          _ref(dkb), int(block_size), int(topk), _ref(do),
                                          _ref(dl), _stream(q, stream)))
    return out, lse


def decode_noalloc(q, k_cache, v_cache, cu_seqlens, block_size: int, topk: int, out, lse,
                   kbar=None, stream=None):
    """decode() through moba_decode_noalloc: the library allocates nothing;
    the caller passes out [S, Hq, 128] bf16 and lse [Hq, S] fp32, and
    cu_seqlens must be a host tensor."""
    lib = load()
    cu = _cu(cu_seqlens)
    d = [describe(t) for t in (q, k_cache, v_cache, cu)]
    dkb = describe(kbar) if kbar is not None else None
    do, dl = describe(out), describe(lse)
    _check("moba_decode_noalloc", lib.moba_decode_noalloc(_ref(d[0]), _ref(d[1]), _ref(d[2]),
                                                          _ref(d[3]), _ref(dkb), int(block_size),
                                                          int(topk), _ref(do), _ref(dl),
                                                          _stream(q, stream)))
    return out, lse


def dense_forward(q, k, v, cu_seqlens, out=None, lse=None, stream=None):
    """Dense causal attention with the same conventions as forward()."""
    lib = load()
    cu = _cu(cu_seqlens)
    T, Hq = q.shape[0], q.shape[1]
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if lse is None:
        lse = torch.empty((Hq, T), dtype=torch.float32, device=q.device)
    dq, dk, dv, dc, do, dl = map(describe, (q, k, v, cu, out, lse))
    _check("moba_dense_forward", lib.moba_dense_forward(_ref(dq), _ref(dk), _ref(dv), _ref(dc),
                                                        _ref(do), _ref(dl), _stream(q, stream)))
    return out, lse


def route_size(cu_seqlens, block_size: int, topk: int, num_q_heads: int, stream=None):
    """(nblk_total, E) as the library reports them: the batch's block count
    and its number of history selections (moba_route's entries)."""
    lib = load()
    cu = _cu(cu_seqlens)
    nb, e = ctypes.c_int64(), ctypes.c_int64()
    dc = describe(cu)
    _check("moba_route_size", lib.moba_route_size(_ref(dc), int(block_size), int(topk),
                                                  int(num_q_heads), ctypes.byref(nb),
                                                  ctypes.byref(e), _stream(cu, stream)))
    return int(nb.value), int(e.value)


def num_blocks(cu_seqlens, block_size: int) -> int:
    return route_size(cu_seqlens, block_size, 1, 1)[0]


def pool(k, cu_seqlens, block_size: int, stream=None):
    """Block keys [nblk_total, Hkv, 128] fp32."""
    lib = load()
    cu = _cu(cu_seqlens)
    nb = num_blocks(cu, block_size)
    kbar = torch.empty((nb, k.shape[1], k.shape[2]), dtype=torch.float32, device=k.device)
    dk, dc, db = map(describe, (k, cu, kbar))
    _check("moba_pool", lib.moba_pool(_ref(dk), _ref(dc), int(block_size), _ref(db),
                                      _stream(k, stream)))
    return kbar


def select(q, k, cu_seqlens, block_size: int, topk: int, nmax: int = 0, stream=None):
    """sel [T, Hq, topk] int32 (and scores [T, Hq, nmax] fp32 if nmax > 0)."""
    lib = load()
    cu = _cu(cu_seqlens)
    T, Hq = q.shape[0], q.shape[1]
    sel = torch.empty((T, Hq, topk), dtype=torch.int32, device=q.device)
    scores = torch.empty((T, Hq, nmax), dtype=torch.float32, device=q.device) if nmax > 0 else None
    dq, dk, dc, ds = map(describe, (q, k, cu, sel))
    dsc = describe(scores) if scores is not None else None
    _check("moba_select", lib.moba_select(_ref(dq), _ref(dk), _ref(dc), int(block_size), int(topk),
                                          _ref(ds), _ref(dsc), _stream(q, stream)))
    return (sel, scores) if nmax > 0 else sel


def route(sel, cu_seqlens, block_size: int, num_kv_heads: int, stream=None):
    """(counts [Hkv*nblk] int32, offsets [Hkv*nblk+1] int64, entries [E] int32)."""
    lib = load()
    cu = _cu(cu_seqlens)
    T, Hq, topk = sel.shape
    nb, E = route_size(cu, block_size, topk, Hq, stream)
    nbins = nb * num_kv_heads
    counts = torch.empty((nbins,), dtype=torch.int32, device=sel.device)
    offsets = torch.empty((nbins + 1,), dtype=torch.int64, device=sel.device)
    entries = torch.empty((E,), dtype=torch.int32, device=sel.device)
    ds, dc, dn, do, de = map(describe, (sel, cu, counts, offsets, entries))
    _check("moba_route", lib.moba_route(_ref(ds), _ref(dc), int(block_size), int(num_kv_heads),
                                        _ref(dn), _ref(do), _ref(de), _stream(sel, stream)))
    return counts, offsets, entries


class PagedCache(NamedTuple):
    """A pool of N pages of P tokens (64, 128, 192 or 256) in 8 bits, as include/moba.h
    describes it.  Every tensor may be a slice of a larger pool (a layer's) whose page
    and head strides are multiples of 16 bytes; scales and sums are contiguous, and k, v and
    k_sum begin at multiples of 16 bytes."""
    k: torch.Tensor        # [N, Hkv, P, 128] float8_e4m3fn
    v: torch.Tensor        # [N, Hkv, P // 64, 128, 64] float8_e4m3fn, token index innermost
    k_scale: torch.Tensor  # [N, Hkv] fp32: the page's keys are k * k_scale
    v_scale: torch.Tensor  # [N, Hkv] fp32
    k_sum: torch.Tensor    # [N, Hkv, 128] fp32, the sum of the page's keys


class CachePlan(NamedTuple):
    """What cache_plan() returns."""
    cu_new: torch.Tensor    # [S + 1] int32: request s's new tokens are rows cu_new[s] ..
    slots: torch.Tensor     # [num_tokens] int64: every new token's slot, -1: none
    lens: torch.Tensor      # [S] int32: lengths after the step
    num_free: torch.Tensor  # [1] int32: free pages after the step
    refused: torch.Tensor   # [1] int32: requests refused


def _cache_module():
    """The marshalling of the paged cache's calls (csrc/cache_binding.cpp).  Raises if it has not
    been built."""
    load()
    try:
        from . import _cache_binding
    except ImportError as e:
        raise RuntimeError("_cache_binding.so does not load; build it with "
                           "`python -m paper_2502_13189_amd.build`") from e
    return _cache_binding


def _latent_module():
    """The marshalling of rotary positions' and latent attention's calls
    (csrc/latent_binding.cpp).  Raises if it has not been built."""
    load()
    try:
        from . import _latent_binding
    except ImportError as e:
        raise RuntimeError("_latent_binding.so does not load; build it with "
                           "`python -m paper_2502_13189_amd.build`") from e
    return _latent_binding


def _caller(module, owner: str):
    """call(fn, t, stream, *args): fn of the module that module() loads, on `stream` or the current stream of
    t's device, which is made current.  What the call allocates is allocated for that stream, so that memory
    it drops is not given out again before the call is done with it.  A closure for each module: a
    function that both share would be a second Python call on the way, 0.15 us."""
    ext = None

    def call(fn: str, t: torch.Tensor, stream, *args):
        nonlocal ext
        if ext is None:
            ext = module()
        f = getattr(ext, fn)
        device = t.get_device()
        if device < 0:
            raise ValueError("%s tensors live on a GPU" % owner)
        if stream is not None:
            if not hasattr(stream, "cuda_stream"):
                stream = torch.cuda.ExternalStream(int(stream), device=device)
            if stream.device_index != device:
                raise ValueError("the stream is on GPU %d, the tensors on GPU %d"
                                 % (stream.device_index, device))
            with torch.cuda.stream(stream):
                return f(*args, stream.cuda_stream)
        if device == torch.cuda.current_device():
            return f(*args, torch._C._cuda_getCurrentRawStream(device))
        with torch.cuda.device(device):
            return f(*args, torch._C._cuda_getCurrentRawStream(device))

    return call


_cache_call = _caller(_cache_module, "the paged cache's")
_latent_call = _caller(_latent_module, "rotary positions' and latent attention's")


def cache_new(num_pages: int, num_kv_heads: int, page_size: int = 64, device="cuda") -> PagedCache:
    """An empty pool of pages (uninitialised memory: nothing reads what was not written)."""
    if page_size not in (64, 128, 192, 256):
        raise ValueError("page_size must be 64, 128, 192 or 256")
    f8 = dict(dtype=torch.float8_e4m3fn, device=device)
    f32 = dict(dtype=torch.float32, device=device)
    n, h = int(num_pages), int(num_kv_heads)
    return PagedCache(torch.empty((n, h, page_size, 128), **f8),
                      torch.empty((n, h, page_size // 64, 128, 64), **f8),
                      torch.empty((n, h), **f32), torch.empty((n, h), **f32),
                      torch.empty((n, h, 128), **f32))


def cache_plan(add, lens, table, free_pages, num_free, page_size: int, num_tokens: int,
               lens_out=None, num_free_out=None, cu_new=None, slots=None, refused=None,
               stream=None) -> CachePlan:
    """Block tables and slot maps of a serving step, on the GPU from the requests' lengths.

    add [S] int32: new tokens per request (0: none, negative: the request ends); lens [S]
    int32: tokens held; table [S, W] int32 and free_pages [N] int32 are updated in place (the
    first num_free[0] entries are free); num_tokens: rows of the step's arrays, at least
    the new tokens'.  Requests that do not fit are refused whole (their slots are -1).
    Who cuts a request back (lowers its length) past a page's begin appends the pages behind
    its new end to free_pages and raises num_free.
    lens_out and num_free_out may be lens and num_free themselves: a captured step then
    carries its state from replay to replay."""
    status, *out = _cache_call("plan", add, stream, add, lens, table, free_pages, num_free, page_size,
                               num_tokens, lens_out, num_free_out, cu_new, slots, refused)
    if status:
        raise MobaError("moba_cache_plan", status)
    return CachePlan(*out)


def cache_write(k, v, slots, cache: PagedCache, stream=None) -> None:
    """Quantises new keys and values [T, Hkv, 128] (bf16 or fp32) into their slots [T]
    int64 (negative: left out), as cache_plan() gives them: a page's tokens are
    consecutive rows with ascending slots."""
    _check("moba_cache_write", _cache_call("write", k, stream, k, v, slots, cache))


def cache_decode_workspace_bytes(num_requests: int, table_width: int, num_q_heads: int,
                                 num_kv_heads: int, page_size: int, block_size: int,
                                 topk: int) -> int:
    """Bytes of cache_decode()'s workspace (0: such a call would be refused)."""
    # (what does not fit 32 bits is refused for its value; ctypes would cut it off)
    return int(load().moba_cache_decode_workspace_bytes(
        *(max(-1, min(int(x), 2 ** 31 - 1))
          for x in (num_requests, table_width, num_q_heads, num_kv_heads, page_size, block_size, topk))))


def cache_decode(q, cache: PagedCache, table, lens, block_size: int, topk: int, out=None, lse=None,
                 workspace=None, stream=None):
    """decode() over a paged 8-bit cache: one new query per request (topk == 0: full
    attention) at the last position of the lens[s] tokens it holds.  q [S, Hq, 128] bf16,
    table [S, W] int32, lens [S] int32; block_size is a multiple of the page size.  A request
    with lens[s] <= 0 gets out 0 and lse -inf.  workspace: uint8, at least
    cache_decode_workspace_bytes() of it; by default a fresh one per call, so that calls on
    several streams and captured graphs share nothing.  Returns (out [S, Hq, 128], lse
    [Hq, S])."""
    status, out, lse = _cache_call("decode", q, stream, q, cache, table, lens, block_size, topk, out,
                                   lse, workspace)
    if status:
        raise MobaError("moba_cache_decode", status)
    return out, lse


class Rotation(NamedTuple):
    """How fast the pairs of a head's first 2 * len(freqs) dims turn, and which dims make a pair."""
    freqs: torch.Tensor         # [R / 2] float64 on the GPU, radians a position
    amplitude: float = 1.0      # factor of the result
    interleaved: bool = False   # pairs (2i, 2i + 1); otherwise (i, i + R / 2)


def rotation(rot_dim: int, base: float = 10000.0, scaling=None, factor: float = 1.0, original_length=None,
             low: float = 1.0, high: float = 32.0, interleaved: bool = False, device="cuda") -> Rotation:
    """Rotary frequencies base ** (-2 i / rot_dim), as they are or scaled for contexts `factor` times as
    long as the `original_length` a model was trained on:
      "linear"  divided by factor (position interpolation)
      "base"    of a base factor ** (rot_dim / (rot_dim - 2)) as large: the slowest pair is interpolated,
                the fastest is not
      "parts"   pairs that turn fewer than `low` times over original_length are interpolated, more than
                `high` times kept, and in between mixed linearly by that number; the amplitude is
                0.1 ln(factor) + 1 (NTK-by-parts with its attention temperature, arXiv 2309.00071)"""
    if rot_dim < 2 or rot_dim % 2:
        raise ValueError("rot_dim must be even and positive")
    if scaling not in (None, "linear", "base", "parts"):
        raise ValueError("scaling must be None, 'linear', 'base' or 'parts'")
    if not base > 0.0 or not factor >= 1.0:
        raise ValueError("base must be positive, factor at least 1")
    base, factor = float(base), float(factor)
    if scaling == "base":
        if rot_dim == 2:
            raise ValueError("a single pair has no slowest and fastest: scaling 'base' needs rot_dim > 2")
        base *= factor ** (rot_dim / (rot_dim - 2))
    freqs = [base ** (-2 * i / rot_dim) for i in range(rot_dim // 2)]
    amplitude = 1.0
    if scaling == "linear":
        freqs = [f / factor for f in freqs]
    if scaling == "parts":
        if not original_length or not low < high:
            raise ValueError("scaling 'parts' needs original_length, and low < high")
        turns = [original_length * f / (2 * math.pi) for f in freqs]
        keep = [min(1.0, max(0.0, (t - low) / (high - low))) for t in turns]
        freqs = [f * (k + (1.0 - k) / factor) for f, k in zip(freqs, keep)]
        amplitude = 0.1 * math.log(factor) + 1.0
    return Rotation(torch.tensor(freqs, dtype=torch.float64, device=device), amplitude, bool(interleaved))


def rope(q, k, rot: Rotation, pos=None, cu_seqlens=None, start=None, q_out=None, k_out=None, stream=None):
    """Rotary positions of queries [T, Hq, D] and keys [T, Hk, D] (bf16 or fp32; k may be None): the
    first 2 * len(rot.freqs) dims of every head are turned, the others copied.  Rows stand at pos [T] (int32
    or int64), or, packed, row t of sequence s at start[s] + t - cu_seqlens[s] (int32 on the GPU; start None:
    0), rows of no sequence left as they are.  q_out and k_out may be q and k.  Returns (q_out, k_out)."""
    status, qo, ko = _latent_call("rope", q, stream, False, q, k, rot, pos, cu_seqlens, start, q_out, k_out)
    if status:
        raise MobaError("moba_rope", status)
    return qo, ko


def rope_backward(dq_out, dk_out, rot: Rotation, pos=None, cu_seqlens=None, start=None, dq=None, dk=None,
                  stream=None):
    """Gradients of rope() w.r.t. q and k from those w.r.t. its results (dk_out may be None; dq and dk may be
    dq_out and dk_out).  Returns (dq, dk)."""
    status, gq, gk = _latent_call("rope", dq_out, stream, True, dq_out, dk_out, rot, pos, cu_seqlens, start, dq,
                                  dk)
    if status:
        raise MobaError("moba_rope_backward", status)
    return gq, gk


_LATENT_SCALE = 1.0 / math.sqrt(192.0)


def latent_forward(q, k, k_rope, v, cu_seqlens, scale=None, out=None, lse=None, stream=None):
    """Causal latent attention, expanded: q [T, H, 192] (128 dims, then 64 rotary ones), k [T, H, 128],
    k_rope [T, 64] shared by all heads, v [T, H, 128], all bf16, rotary positions applied; cu_seqlens [S + 1]
    int32 on the GPU.  scale: None for 1 / sqrt(192).  Returns (out [T, H, 128], lse [H, T] fp32)."""
    status, out, lse = _latent_call("forward", q, stream, q, k, k_rope, v, cu_seqlens,
                                    _LATENT_SCALE if scale is None else scale, out, lse)
    if status:
        raise MobaError("moba_latent_forward", status)
    return out, lse


def latent_backward_workspace_bytes(T: int, num_heads: int) -> int:
    """Bytes of latent_backward()'s workspace (0: such a call would be refused)."""
    return int(load().moba_latent_backward_workspace_bytes(*(max(-1, min(int(x), 2 ** 31 - 1))
                                                             for x in (T, num_heads))))


def latent_backward(q, k, k_rope, v, cu_seqlens, out, lse, dout, scale=None, dq=None, dk=None, dk_rope=None,
                    dv=None, workspace=None, stream=None):
    """Gradients of latent_forward() (out and lse its results, dout [T, H, 128]).  workspace: uint8, at least
    latent_backward_workspace_bytes() of it; by default a fresh one per call.  Returns (dq [T, H, 192], dk
    [T, H, 128], dk_rope [T, 64], dv [T, H, 128])."""
    status, *grads = _latent_call("backward", q, stream, q, k, k_rope, v, cu_seqlens, out, lse, dout,
                                  _LATENT_SCALE if scale is None else scale, dq, dk, dk_rope, dv, workspace)
    if status:
        raise MobaError("moba_latent_backward", status)
    return tuple(grads)


def latent_cache_new(num_pages: int, page_size: int = 64, device="cuda") -> torch.Tensor:
    """Pages [num_pages, page_size, 576] bf16 of a latent cache: a token's row is its latent vector (512)
    and its rotary key (64).  Uninitialised: nothing reads what was not written."""
    if page_size not in (64, 128, 192, 256):
        raise ValueError("page_size must be 64, 128, 192 or 256")
    return torch.empty((int(num_pages), page_size, 576), dtype=torch.bfloat16, device=device)


def latent_write(c, k_rope, slots, pages, rot=None, pos=None, cu_seqlens=None, start=None, stream=None) -> None:
    """Writes latent vectors c [T, 512] and rotary keys k_rope [T, 64] (bf16) into their slots [T] int64
    (negative: left out), as cache_plan() gives them.  With a Rotation, the keys are turned on the way;
    positions as for rope()."""
    _check("moba_latent_write", _latent_call("write", c, stream, c, k_rope, slots, pages, rot, pos, cu_seqlens,
                                             start))


def latent_decode_workspace_bytes(num_requests: int, table_width: int, num_heads: int, page_size: int) -> int:
    """Bytes of latent_decode()'s workspace (0: such a call would be refused)."""
    return int(load().moba_latent_decode_workspace_bytes(
        *(max(-1, min(int(x), 2 ** 31 - 1)) for x in (num_requests, table_width, num_heads, page_size))))


def latent_decode(q_c, q_rope, pages, table, lens, scale=None, out=None, lse=None, workspace=None, stream=None):
    """Latent attention of one new query per request, absorbed, over the lens[s] tokens its pages hold: q_c
    [S, H, 512], q_rope [S, H, 64] bf16; table [S, W], lens [S] int32.  A request with lens[s] <= 0 gets out 0
    and lse -inf.  workspace: uint8, at least latent_decode_workspace_bytes() of it; by default a fresh
    one per call.  Returns (out [S, H, 512] bf16, lse [H, S])."""
    status, out, lse = _latent_call("decode", q_c, stream, q_c, q_rope, pages, table, lens,
                                    _LATENT_SCALE if scale is None else scale, out, lse, workspace)
    if status:
        raise MobaError("moba_latent_decode", status)
    return out, lse


def workspace_bytes(T: int, num_q_heads: int, num_kv_heads: int, nblk_total: int, topk: int,
                    head_dim: int = 128) -> int:
    """Device workspace bytes a one-pass moba_forward needs (an upper bound)."""
    return int(load().moba_workspace_bytes(int(T), int(num_q_heads), int(num_kv_heads),
                                           int(head_dim), int(nblk_total), int(topk)))


def workspace_held_bytes() -> int:
    """Bytes of device workspace the library holds on the current device."""
    return int(load().moba_workspace_held_bytes())


def take_wait_timeouts() -> int:
    """Give-ups of the backward's hand-over wait since the last call (waits
    for the device)."""
    n = ctypes.c_uint64()
    _check("moba_take_wait_timeouts", load().moba_take_wait_timeouts(ctypes.byref(n)))
    return int(n.value)


def release_workspace() -> None:
    _check("moba_release_workspace", load().moba_release_workspace())


def profile_enable(on: bool = True) -> None:
    load().moba_profile_enable(1 if on else 0)


def profile_read() -> dict:
    """{phase: (launches, total_ms)} since the last read."""
    buf = (PhaseStat * 32)()
    n = load().moba_profile_read(buf, 32)
    return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms)) for i in range(n)}
