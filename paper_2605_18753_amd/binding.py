"""ctypes binding of libdash_attn.so: argument marshalling only.

Every function mirrors one entry point of include/dash_attn.h and takes torch
tensors that already live on the GPU; torch is used for device memory and the
current stream, nothing else.  There is no fallback: if the library is missing
or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import operator
import os
import struct
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("DASH_ATTN_LIB") or os.path.join(_HERE, "libdash_attn.so")

DASH_F32, DASH_BF16 = 0, 1


class DashError(RuntimeError):
    pass


class dash_params(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("h_q", ctypes.c_int32), ("h_kv", ctypes.c_int32),
        ("n_q", ctypes.c_int32), ("n_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("block_size", ctypes.c_int32), ("causal", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("alpha", ctypes.c_float), ("gamma", ctypes.c_float), ("sigma", ctypes.c_float),
        ("scale", ctypes.c_float), ("window", ctypes.c_int32),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
        ("v_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3),
    ]


class dash_paged_params(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "h_q", "h_kv", "head_dim", "dtype", "causal", "page_size", "n_pages",
                                              "max_pages", "n_rows")]
    _fields_ += [("scale", ctypes.c_float), ("reserved", ctypes.c_int32)]
    _fields_ += [(n, ctypes.c_int64 * k) for n, k in (("q_stride", 2), ("o_stride", 2), ("k_new_stride", 2), ("v_new_stride", 2),
                                                      ("k_stride", 3), ("v_stride", 3))]


_lib = None
_P = ctypes.POINTER(dash_params)
_PP = ctypes.POINTER(dash_paged_params)
_V = ctypes.c_void_p
_I = ctypes.c_int32
_SIGNATURES = {
    "dash_list_stride": (ctypes.c_int32, [_P]),
    "dash_mask_words": (ctypes.c_int32, [_P]),
    "dash_attn_workspace_bytes": (ctypes.c_int, [_P, ctypes.POINTER(ctypes.c_size_t)]),
    "dash_kbar_compress": (ctypes.c_int, [_P, _V, _V, ctypes.c_int32, ctypes.c_int32, _V]),
    "dash_kbar_summarize": (ctypes.c_int, [_P, _V, _V, ctypes.POINTER(ctypes.c_int64), _V, ctypes.c_int32,
                                           ctypes.c_int32, _V]),
    "dash_stage1_route": (ctypes.c_int, [_P, _V, _V, _V, _V, _V, _V, _V, _V, ctypes.c_size_t, _V]),
    "dash_stage2_attend": (ctypes.c_int, [_P, _V, _V, _V, _V, _V, _V, _V, ctypes.c_size_t, _V]),
    "dash_attn_prefill": (ctypes.c_int, [_P, _V, _V, _V, _V, _V, _V, _V, _V, _V, _V, _V, ctypes.c_size_t, _V]),
    "dash_attn_decode": (ctypes.c_int, [_P, _V, _V, _V, _V, _V, _V, _V, _V, _V, _V, _V, ctypes.c_size_t, _V]),
    "dash_attn_decode_static": (ctypes.c_int, [_P, _V, _V, _V, _V, _V, _V, _V, _V, _V, _V, _V]),
    "dash_attn_decode_ragged": (ctypes.c_int, [_P, _V, _V, _V, _V, _V, ctypes.c_int32, _V, _V, _V, _V, _V, _V, _V,
                                               ctypes.c_size_t, _V]),
    "dense_attn": (ctypes.c_int, [_P, _V, _V, _V, _V, _V, ctypes.c_size_t, _V]),
    "dash_attn_backward_workspace_bytes": (ctypes.c_int, [_P, ctypes.POINTER(ctypes.c_size_t)]),
    "dash_attn_backward": (ctypes.c_int, [_P] + [_V] * 13 + [ctypes.c_size_t, _V]),
    "dash_kbar_summarize_backward": (ctypes.c_int, [_P, _V, _V, ctypes.POINTER(ctypes.c_int64), _V, _V, _V, _V]),
    "dash_paged_workspace_bytes": (ctypes.c_int, [_PP, ctypes.POINTER(ctypes.c_size_t)]),
    "dash_paged_evict_workspace_bytes": (ctypes.c_int, [_PP, ctypes.POINTER(ctypes.c_size_t)]),
    "dash_paged_append": (ctypes.c_int, [_PP] + [_V] * 11),
    "dash_paged_attend": (ctypes.c_int, [_PP] + [_V] * 9 + [ctypes.c_size_t, _V]),
    "dash_paged_weigh": (ctypes.c_int, [_PP] + [_V] * 6 + [_I, _V, _V, ctypes.c_size_t, _V]),
    "dash_paged_evict": (ctypes.c_int, [_PP] + [_V] * 7 + [_I, _I, _I, _V, _V, ctypes.c_size_t, _V]),
    "dash_strerror": (ctypes.c_char_p, [ctypes.c_int]),
}


def load_library(path: Optional[str] = None):
    """Load libdash_attn.so (built in-tree by paper_2605_18753_amd.build)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise DashError(f"{p} not found: build it with `python -m paper_2605_18753_amd.build`")
    lib = ctypes.CDLL(p)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if path is None:
        _lib = lib
    return lib


def exported_symbols():
    return list(_SIGNATURES)


def _check(rc: int, what: str):
    if rc != 0:
        msg = load_library().dash_strerror(rc).decode()
        raise DashError(f"{what} failed: {msg} ({rc})")


def _ptr(t: Optional[torch.Tensor]):
    # a plain int (or None): the declared argument types convert it
    return None if t is None else t.data_ptr()


# The current stream's handle without building a torch.cuda.Stream object: 0.2 us instead of
# 2.7 us, which a decode step of a short cache would notice.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    if _raw_stream is not None and _device is not None and torch.cuda.is_initialized():
        return _raw_stream(_device())
    return torch.cuda.current_stream().cuda_stream


def make_params(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: Optional[torch.Tensor],
                block: int, alpha: float = 1.5, gamma: float = 1.0, sigma: float = 1.0,
                causal: bool = True, scale: float = 0.0, window: int = 0) -> dash_params:
    """q [B,H_q,n_q,d]; k, v [B,H_kv,n_kv,d]; last dim contiguous."""
    p = dash_params()
    p.batch, p.h_q, p.n_q, p.head_dim = q.shape
    p.h_kv, p.n_kv = k.shape[1], k.shape[2]
    p.block_size = block
    p.causal = int(causal)
    p.dtype = DASH_BF16 if q.dtype == torch.bfloat16 else DASH_F32
    p.alpha, p.gamma, p.sigma, p.scale = alpha, gamma, sigma, scale
    p.window = window
    for name, t in (("q_stride", q), ("k_stride", k), ("v_stride", v), ("o_stride", o if o is not None else q)):
        assert t.stride(3) == 1, "head_dim must be contiguous"
        getattr(p, name)[:] = [t.stride(0), t.stride(1), t.stride(2)]
    return p


def workspace_bytes(p: dash_params) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().dash_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(n)), "dash_attn_workspace_bytes")
    return n.value


def list_stride(p: dash_params) -> int:
    return load_library().dash_list_stride(ctypes.byref(p))


def mask_words(p: dash_params) -> int:
    return load_library().dash_mask_words(ctypes.byref(p))


def alloc_workspace(p: dash_params, device) -> torch.Tensor:
    return torch.empty(workspace_bytes(p) + 256, dtype=torch.uint8, device=device)


def _ws_ptr(ws: torch.Tensor):
    if not ws.is_contiguous():
        raise DashError("a workspace is contiguous")
    base = ws.data_ptr()
    aligned = (base + 255) & ~255
    return aligned, ws.numel() - (aligned - base)


@dataclass
class Lists:
    """Optional Stage-1 outputs (see dash_stage1_route in the header)."""
    mask: Optional[torch.Tensor] = None
    cnt: Optional[torch.Tensor] = None
    idx: Optional[torch.Tensor] = None
    bias: Optional[torch.Tensor] = None
    tau: Optional[torch.Tensor] = None

    @staticmethod
    def allocate(p: dash_params, device, idx: bool = True, tau: bool = True) -> "Lists":
        rows = (p.batch, p.h_kv, p.n_q)
        ls, mw = list_stride(p), mask_words(p)
        return Lists(
            mask=torch.zeros(rows + (mw,), dtype=torch.int32, device=device),
            cnt=torch.zeros(rows, dtype=torch.int32, device=device),
            idx=torch.zeros(rows + (ls,), dtype=torch.int32, device=device) if idx else None,
            bias=torch.zeros(rows + (ls,), dtype=torch.float32, device=device),
            tau=torch.zeros((p.batch, p.h_q, p.n_q), dtype=torch.float32, device=device) if tau else None,
        )


def dash_kbar_compress(p: dash_params, k: torch.Tensor, kbar: torch.Tensor,
                       first_chunk: int = 0, n_chunks: int = -1) -> None:
    _check(load_library().dash_kbar_compress(p, _ptr(k), _ptr(kbar), first_chunk, n_chunks,
                                             _stream()), "dash_kbar_compress")


def _qbar_strides(qbar: torch.Tensor):
    assert qbar.dtype == torch.float32 and qbar.stride(-1) == 1
    if qbar.dim() == 2:
        st = (0, qbar.stride(0), 0)
    elif qbar.dim() == 3:
        st = (0, qbar.stride(0), qbar.stride(1))
    else:
        st = (qbar.stride(0), qbar.stride(1), qbar.stride(2))
    return (ctypes.c_int64 * 3)(*st)


def dash_kbar_summarize(p: dash_params, k: torch.Tensor, qbar: torch.Tensor, kbar: torch.Tensor,
                        first_chunk: int = 0, n_chunks: int = -1) -> None:
    """qbar: fp32 tensor [h_kv, d] (one summary query per kv-head), [h_kv, T_c, d]
    or [batch, h_kv, T_c, d] (one per chunk); only the strides are passed on."""
    arr = _qbar_strides(qbar)
    _check(load_library().dash_kbar_summarize(p, _ptr(k), _ptr(qbar), arr, _ptr(kbar),
                                              first_chunk, n_chunks, _stream()), "dash_kbar_summarize")


def dash_stage1_route(p, q, kbar, lists: Lists, ws: torch.Tensor) -> None:
    wp, wn = _ws_ptr(ws)
    _check(load_library().dash_stage1_route(p, _ptr(q), _ptr(kbar), _ptr(lists.mask),
                                            _ptr(lists.cnt), _ptr(lists.idx), _ptr(lists.bias),
                                            _ptr(lists.tau), wp, wn, _stream()), "dash_stage1_route")


def dash_stage2_attend(p, q, k, v, o, lists: Lists, ws: torch.Tensor) -> None:
    wp, wn = _ws_ptr(ws)
    _check(load_library().dash_stage2_attend(p, _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                             _ptr(lists.mask), _ptr(lists.bias), wp, wn, _stream()),
           "dash_stage2_attend")


def dash_attn_prefill(p, q, k, v, o, kbar, lists: Lists, ws: torch.Tensor) -> None:
    wp, wn = _ws_ptr(ws)
    _check(load_library().dash_attn_prefill(p, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(kbar),
                                            _ptr(lists.mask), _ptr(lists.cnt), _ptr(lists.idx),
                                            _ptr(lists.bias), _ptr(lists.tau), wp, wn, _stream()),
           "dash_attn_prefill")


def dash_attn_decode(p, q, k_cache, v_cache, kbar_cache, o, lists: Lists, ws: torch.Tensor) -> None:
    wp, wn = _ws_ptr(ws)
    _check(load_library().dash_attn_decode(p, _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                           _ptr(kbar_cache), _ptr(o), _ptr(lists.mask), _ptr(lists.cnt),
                                           _ptr(lists.idx), _ptr(lists.bias), _ptr(lists.tau), wp, wn,
                                           _stream()), "dash_attn_decode")


def dash_attn_decode_static(p, q, k_cache, v_cache, kbar_cache, o, lists: Lists) -> None:
    """dash_attn_decode on the library's built-in scratch (no workspace, no allocation)."""
    _check(load_library().dash_attn_decode_static(p, _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                                  _ptr(kbar_cache), _ptr(o), _ptr(lists.mask), _ptr(lists.cnt),
                                                  _ptr(lists.idx), _ptr(lists.bias), _ptr(lists.tau), _stream()),
           "dash_attn_decode_static")


def dash_attn_decode_ragged(p, q, k_cache, v_cache, kbar_cache, seq_lens: torch.Tensor, o, lists: Lists,
                            ws: torch.Tensor, update_cache: bool = True) -> None:
    assert seq_lens.dtype == torch.int32 and seq_lens.is_contiguous() and seq_lens.numel() == p.batch
    wp, wn = _ws_ptr(ws)
    _check(load_library().dash_attn_decode_ragged(p, _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                                  _ptr(kbar_cache), _ptr(seq_lens), int(update_cache), _ptr(o),
                                                  _ptr(lists.mask), _ptr(lists.cnt), _ptr(lists.idx),
                                                  _ptr(lists.bias), _ptr(lists.tau), wp, wn, _stream()),
           "dash_attn_decode_ragged")


def dense_attn(p, q, k, v, o, ws: torch.Tensor) -> None:
    wp, wn = _ws_ptr(ws)
    _check(load_library().dense_attn(p, _ptr(q), _ptr(k), _ptr(v), _ptr(o), wp, wn, _stream()),
           "dense_attn")


def backward_workspace_bytes(p: dash_params) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().dash_attn_backward_workspace_bytes(ctypes.byref(p), ctypes.byref(n)),
           "dash_attn_backward_workspace_bytes")
    return n.value


def alloc_backward_workspace(p: dash_params, device) -> torch.Tensor:
    return torch.empty(backward_workspace_bytes(p) + 256, dtype=torch.uint8, device=device)


def dash_attn_backward(p, q, k, v, d_o, kbar, lists: Lists, dq, dk, dv, ws: torch.Tensor, dkbar=None) -> None:
    """Backward of dash_attn_prefill; lists.mask / bias / tau are the forward's outputs.
    dkbar None: block-mean summaries (their gradient is folded into dk)."""
    wp, wn = _ws_ptr(ws)
    if dkbar is not None:
        assert dkbar.dtype == torch.float32 and dkbar.is_contiguous() and tuple(dkbar.shape) == kbar_shape(p)
    _check(load_library().dash_attn_backward(p, _ptr(q), _ptr(k), _ptr(v), _ptr(d_o),
                                             _ptr(kbar), _ptr(lists.mask), _ptr(lists.bias), _ptr(lists.tau),
                                             _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dkbar), wp, wn, _stream()),
           "dash_attn_backward")


def dash_kbar_summarize_backward(p, k, qbar: torch.Tensor, dkbar: torch.Tensor, dk, dqbar: torch.Tensor) -> None:
    """Backward of dash_kbar_summarize; qbar as there ([h_kv,d], [h_kv,T_c,d] or [batch,h_kv,T_c,d])."""
    strides = _qbar_strides(qbar)
    assert dkbar.dtype == torch.float32 and dkbar.is_contiguous() and tuple(dkbar.shape) == kbar_shape(p)
    assert dqbar.dtype == torch.float32 and dqbar.is_contiguous() and tuple(dqbar.shape) == kbar_shape(p)
    _check(load_library().dash_kbar_summarize_backward(p, _ptr(k), _ptr(qbar), strides, _ptr(dkbar),
                                                       _ptr(dk), _ptr(dqbar), _stream()),
           "dash_kbar_summarize_backward")


def kbar_shape(p: dash_params):
    return (p.batch, p.h_kv, p.n_kv // p.block_size, p.head_dim)


# ---- paged cache -----------------------------------------------------------------------------------------------------
@dataclass
class PagedCache:
    """Keys and values of several sequences in pages of a pool (see the header's section on the paged cache).
    k, v [n_pages, h_kv, page_size, d]; table int32 [batch, max_pages]; lens int32 [batch]; for evicting callers
    weights (fp32) and pos (int32), both [n_pages, h_kv, page_size], and seen int32 [batch].
    Every call checks those that it uses."""
    k: torch.Tensor
    v: torch.Tensor
    table: torch.Tensor
    lens: torch.Tensor
    weights: Optional[torch.Tensor] = None
    pos: Optional[torch.Tensor] = None
    seen: Optional[torch.Tensor] = None

    @staticmethod
    def allocate(batch: int, h_kv: int, n_pages: int, page_size: int, head_dim: int, max_pages: int, device,
                 dtype=torch.bfloat16, evicting: bool = False) -> "PagedCache":
        """An empty cache without pages (table entries -1)."""
        whole = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)  # noqa: E731
        kv = [torch.zeros((n_pages, h_kv, page_size, head_dim), dtype=dtype, device=device) for _ in range(2)]
        c = PagedCache(*kv, whole(batch, max_pages).fill_(-1), whole(batch))
        if evicting:
            c.weights = torch.zeros((n_pages, h_kv, page_size), dtype=torch.float32, device=device)
            c.pos, c.seen = whole(n_pages, h_kv, page_size), whole(batch)
        return c


_PAGED_PARAMS = struct.Struct("10ifi14q")                  # dash_paged_params ...
_paged_sizes = operator.itemgetter(0, 2, 3, 4, 6, 7, 8, *range(20, 26))   # ... and its batch, h_kv, head_dim, dtype, page_size, n_pages, max_pages, k_stride, v_stride
_INT, _FLOAT = torch.int32, torch.float32
_PAGED_TYPES = {torch.bfloat16: DASH_BF16, _FLOAT: DASH_F32}


def _paged_layout(c: PagedCache, weights=None, pos=None, seen=None) -> tuple:
    """Device, type, and sizes and strides (as _paged_sizes has them) of a cache whose tensors fit each other, those of the optional
    ones among them that are given.  Every call looks at them anew, for a tensor can change in place."""
    k, v, t, lens = c.k, c.v, c.table, c.lens
    shape, dtype, dev = tuple(k.shape), k.dtype, k.get_device()
    if len(shape) != 4 or v.shape != shape or v.dtype is not dtype or dtype not in _PAGED_TYPES:
        raise DashError("k and v pages: two tensors [n_pages, h_kv, page_size, d] of one type, bf16 or fp32")
    n_pages, h_kv, page_size, d = shape
    kp, kh, kt, k1 = k.stride()
    vp, vh, vt, v1 = v.stride()
    if k1 != 1 or v1 != 1:
        raise DashError("k and v pages: head_dim must be contiguous")
    if t.dtype is not _INT or t.dim() != 2 or not t.is_contiguous():
        raise DashError("table [batch, max_pages]: a contiguous int32 tensor")
    batch, max_pages = t.shape
    ok = lens is not None and lens.dtype is _INT and lens.shape == (batch,) and lens.is_contiguous()
    same = v.get_device() == dev == t.get_device()
    if weights is not None:
        ok = ok and weights.dtype is _FLOAT and weights.shape == shape[:3] and weights.is_contiguous()
        same = same and weights.get_device() == dev
    if pos is not None:
        ok = ok and pos.dtype is _INT and pos.shape == shape[:3] and pos.is_contiguous()
        same = same and pos.get_device() == dev
    if seen is not None:
        ok = ok and seen.dtype is _INT and seen.shape == (batch,) and seen.is_contiguous()
        same = same and seen.get_device() == dev
    if not ok:
        raise DashError("lens and seen int32 [batch], weights (fp32) and pos (int32) [n_pages, h_kv, page_size]: contiguous tensors")
    if not same or lens.get_device() != dev:
        raise DashError("the cache's tensors lie on one device")
    return dev, dtype, (batch, h_kv, d, _PAGED_TYPES[dtype], page_size, n_pages, max_pages, kp, kh, kt, vp, vh, vt)


def _int32(**numbers):
    # ctypes takes the low 32 bits of a number without a word
    for name, x in numbers.items():
        if not -1 << 31 <= x < 1 << 31:
            raise DashError(f"{name}: {x} does not fit 32 bits")


def make_paged_params(cache: PagedCache, n_rows: int, h_q: int, causal: bool = True, scale: float = 0.0) -> dash_paged_params:
    """The parameters of calls on this cache, or on others of the same sizes, strides and type.  The strides of q, o, k_new and
    v_new are those of the tensors each call is given."""
    _paged_layout(cache, cache.weights, cache.pos, cache.seen)
    _int32(n_rows=n_rows, h_q=h_q)
    p = dash_paged_params()
    p.batch, p.max_pages = cache.table.shape
    p.n_pages, p.h_kv, p.page_size, p.head_dim = cache.k.shape
    p.h_q, p.n_rows, p.causal, p.scale = h_q, n_rows, int(causal), scale
    p.dtype = DASH_BF16 if cache.k.dtype == torch.bfloat16 else DASH_F32
    p.k_stride[:] = cache.k.stride()[:3]
    p.v_stride[:] = cache.v.stride()[:3]
    return p


def _paged_call(p: dash_paged_params, layout, row_start, rows, extra=None, ws=None):
    """The call's own copy of p, with the strides of its packed tensors, and the current stream.  layout: of the call's cache; rows: (tensor,
    heads, field of its strides); extra: (tensor, type, shape)."""
    dev, dtype, sizes = layout
    f = _PAGED_PARAMS.unpack_from(p)
    if _paged_sizes(f) != sizes:
        raise DashError("the parameters are those of a cache of other sizes, strides or type (make_paged_params)")
    p = dash_paged_params.from_buffer_copy(p)
    d, n_rows = f[3], f[9]
    if row_start is not None and (row_start.dtype is not _INT or row_start.numel() != f[0] + 1 or not row_start.is_contiguous()
                                  or row_start.get_device() != dev):
        raise DashError("row_start: a contiguous int32 tensor of batch + 1 elements on the cache's device")
    for t, heads, name in rows:
        s = t.stride()
        if t.dtype is not dtype or t.shape != (n_rows, heads, d) or s[2] != 1 or t.get_device() != dev:
            raise DashError(f"packed rows: [{n_rows}, {heads}, {d}] of the cache's type and device, head_dim contiguous")
        strides = getattr(p, name)
        strides[0], strides[1] = s[0], s[1]
    if extra is not None and extra[0] is not None:
        t, want, shape = extra
        if t.dtype is not want or t.shape != shape or not t.is_contiguous() or t.get_device() != dev:
            raise DashError(f"expected a contiguous {want} tensor of shape {tuple(shape)} on the cache's device")
    if dev < 0 or (ws is not None and ws.get_device() != dev):
        raise DashError("the cache and the workspace lie on one GPU")
    if _device is None or _raw_stream is None or not torch.cuda.is_initialized():
        return p, _stream()
    if dev != _device():
        raise DashError(f"the cache lies on cuda:{dev}, which is not the current device")
    return p, _raw_stream(dev)


def paged_workspace_bytes(p: dash_paged_params, evict: bool = False) -> int:
    n = ctypes.c_size_t(0)
    name = "dash_paged_evict_workspace_bytes" if evict else "dash_paged_workspace_bytes"
    _check(getattr(load_library(), name)(ctypes.byref(p), ctypes.byref(n)), name)
    return n.value


def alloc_paged_workspace(p: dash_paged_params, device, evict: bool = False) -> torch.Tensor:
    """Scratch of dash_paged_attend and dash_paged_weigh, or with evict=True of dash_paged_evict."""
    return torch.empty(paged_workspace_bytes(p, evict) + 256, dtype=torch.uint8, device=device)


def dash_paged_append(p: dash_paged_params, cache: PagedCache, k_new, v_new, row_start) -> None:
    """k_new, v_new [n_rows, h_kv, d]; cache.weights, pos and seen as far as they are there."""
    layout = _paged_layout(cache, cache.weights, cache.pos, cache.seen)
    p, stream = _paged_call(p, layout, row_start, ((k_new, p.h_kv, "k_new_stride"), (v_new, p.h_kv, "v_new_stride")))
    _check(load_library().dash_paged_append(p, k_new.data_ptr(), v_new.data_ptr(), cache.k.data_ptr(), cache.v.data_ptr(),
                                            row_start.data_ptr(), cache.lens.data_ptr(), cache.table.data_ptr(), _ptr(cache.weights),
                                            _ptr(cache.pos), _ptr(cache.seen), stream), "dash_paged_append")


def dash_paged_attend(p: dash_paged_params, cache: PagedCache, q, row_start, o, ws: torch.Tensor, lse=None) -> None:
    """q, o [n_rows, h_q, d]; lse fp32 [n_rows, h_q] or None."""
    p, stream = _paged_call(p, _paged_layout(cache), row_start, ((q, p.h_q, "q_stride"), (o, p.h_q, "o_stride")),
                            (lse, _FLOAT, (p.n_rows, p.h_q)), ws)
    wp, wn = _ws_ptr(ws)
    _check(load_library().dash_paged_attend(p, q.data_ptr(), cache.k.data_ptr(), cache.v.data_ptr(), row_start.data_ptr(),
                                            cache.lens.data_ptr(), cache.table.data_ptr(), o.data_ptr(), _ptr(lse), wp, wn, stream),
           "dash_paged_attend")


def dash_paged_weigh(p: dash_paged_params, cache: PagedCache, q, row_start, lse, ws: torch.Tensor, last: int = 0) -> None:
    """Adds to cache.weights; lse as dash_paged_attend wrote it."""
    if cache.weights is None or lse is None:
        raise DashError("dash_paged_weigh needs the cache's weights and the rows' lse")
    _int32(last=last)
    p, stream = _paged_call(p, _paged_layout(cache, cache.weights), row_start, ((q, p.h_q, "q_stride"),), (lse, _FLOAT, (p.n_rows, p.h_q)), ws)
    wp, wn = _ws_ptr(ws)
    _check(load_library().dash_paged_weigh(p, q.data_ptr(), cache.k.data_ptr(), row_start.data_ptr(), cache.lens.data_ptr(),
                                           cache.table.data_ptr(), _ptr(lse), last, _ptr(cache.weights), wp, wn, stream), "dash_paged_weigh")


def dash_paged_evict(p: dash_paged_params, cache: PagedCache, budget: int, ws: torch.Tensor, sinks: int = 0, recent: int = 0, src=None) -> None:
    """ws from alloc_paged_workspace(p, device, evict=True); src int32 [batch, h_kv, budget] or None."""
    if cache.weights is None or cache.pos is None or cache.seen is None:
        raise DashError("dash_paged_evict needs the cache's weights, pos and seen")
    _int32(budget=budget, sinks=sinks, recent=recent)
    layout = _paged_layout(cache, cache.weights, cache.pos, cache.seen)
    p, stream = _paged_call(p, layout, None, (), (src, _INT, (p.batch, p.h_kv, budget)), ws)
    wp, wn = _ws_ptr(ws)
    _check(load_library().dash_paged_evict(p, cache.k.data_ptr(), cache.v.data_ptr(), cache.lens.data_ptr(), _ptr(cache.seen), cache.table.data_ptr(),
                                           _ptr(cache.weights), _ptr(cache.pos), budget, sinks, recent, _ptr(src), wp, wn, stream),
           "dash_paged_evict")
