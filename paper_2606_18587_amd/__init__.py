"""DAR attention on MI355X: Python binding of libdar (include/dar.h).

Argument marshalling only: torch provides device memory and the current HIP
stream; every step of the computation runs in the library's HIP kernels.
The library must have been built (paper_2606_18587_amd.build); importing this
package without it raises, there is no fallback path.

A call given stream=s runs as under torch.cuda.stream(s): s has to have waited
for what the call reads, and the workspace and outputs that the call allocates
belong to s (a stream that uses an output later waits for s, and tells torch
so with record_stream if the output may be freed before it is done).
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdar.so")

DAR_OK, DAR_E_ARG, DAR_E_UNSUPPORTED, DAR_E_CAPACITY, DAR_E_WORKSPACE, DAR_E_HIP = range(6)
DAR_F32, DAR_BF16 = 0, 1


class DarShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("Hq", ctypes.c_int), ("Hkv", ctypes.c_int),
                ("d", ctypes.c_int), ("d_down", ctypes.c_int), ("w", ctypes.c_int),
                ("dtype", ctypes.c_int)]


class DarCacheStruct(ctypes.Structure):
    _fields_ = [("k_win", ctypes.c_void_p), ("v_win", ctypes.c_void_p),
                ("k_lat", ctypes.c_void_p), ("v_lat", ctypes.c_void_p),
                ("cap", ctypes.c_int), ("len", ctypes.c_int)]


class DarRopeStruct(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int), ("n_pos", ctypes.c_int),
                ("table", ctypes.c_void_p)]


class DarPagedCacheStruct(ctypes.Structure):
    _fields_ = [("k_win", ctypes.c_void_p), ("v_win", ctypes.c_void_p),
                ("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("page_size", ctypes.c_int), ("max_blocks", ctypes.c_int), ("n_pages", ctypes.c_int)]


class DarCacheQ4Struct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_win", "v_win", "k_codes", "v_codes", "k_exp", "v_exp")] + \
        [("cap", ctypes.c_int), ("len", ctypes.c_int)]


class DarPagedCacheQ4Struct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_win", "v_win", "k_codes", "v_codes", "k_exp", "v_exp",
                                               "block_table", "lens")] + \
        [("page_size", ctypes.c_int), ("max_blocks", ctypes.c_int), ("n_pages", ctypes.c_int)]


class DarError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, status_string(status), status))


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError("libdar.so is not built; run `python paper_2606_18587_amd/build.py` "
                          "(there is no non-HIP fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz, ci = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    shp = ctypes.POINTER(DarShape)
    cp = ctypes.POINTER(DarCacheStruct)
    lib.dar_attn_prefill.restype = ci
    lib.dar_attn_prefill.argtypes = [shp, ci, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.dar_attn_prefill_lse.restype = ci
    lib.dar_attn_prefill_lse.argtypes = [shp, ci, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.dar_cache_append.restype = ci
    lib.dar_cache_append.argtypes = [shp, cp, vp, vp, ci, vp, vp]
    lib.dar_attn_decode.restype = ci
    lib.dar_attn_decode.argtypes = [shp, cp, vp, vp, vp, vp, vp, sz, vp]
    lib.dar_prefill_workspace_bytes.restype = sz
    lib.dar_prefill_workspace_bytes.argtypes = [shp, ci]
    lib.dar_decode_workspace_bytes.restype = sz
    lib.dar_decode_workspace_bytes.argtypes = [shp, ci]
    lib.dar_attn_prefill_backward.restype = ci
    lib.dar_attn_prefill_backward.argtypes = [shp, ci] + [vp] * 14 + [sz, vp]
    lib.dar_prefill_backward_workspace_bytes.restype = sz
    lib.dar_prefill_backward_workspace_bytes.argtypes = [shp, ci]
    lib.dar_attn_prefill_chunk.restype = ci
    lib.dar_attn_prefill_chunk.argtypes = [shp, cp, ci] + [vp] * 8 + [sz, vp]
    lib.dar_prefill_chunk_workspace_bytes.restype = sz
    lib.dar_prefill_chunk_workspace_bytes.argtypes = [shp, ci, ci]
    rp = ctypes.POINTER(DarRopeStruct)
    lib.dar_rope_table.restype = ci
    lib.dar_rope_table.argtypes = [ci, ctypes.c_double, ci, vp, vp]
    lib.dar_attn_prefill_rope.restype = ci
    lib.dar_attn_prefill_rope.argtypes = [shp, ci, ci, rp] + [vp] * 8 + [sz, vp]
    lib.dar_attn_prefill_rope_backward.restype = ci
    lib.dar_attn_prefill_rope_backward.argtypes = [shp, ci, ci, rp] + [vp] * 14 + [sz, vp]
    lib.dar_prefill_rope_backward_workspace_bytes.restype = sz
    lib.dar_prefill_rope_backward_workspace_bytes.argtypes = [shp, ci]
    lib.dar_attn_decode_rope.restype = ci
    lib.dar_attn_decode_rope.argtypes = [shp, cp, rp] + [vp] * 5 + [sz, vp]
    lib.dar_attn_prefill_shared.restype = ci
    lib.dar_attn_prefill_shared.argtypes = [shp, ci] + [vp] * 9 + [sz, vp]
    lib.dar_cache_append_shared.restype = ci
    lib.dar_cache_append_shared.argtypes = [shp, cp, vp, vp, vp, ci, vp]
    lib.dar_attn_decode_shared.restype = ci
    lib.dar_attn_decode_shared.argtypes = [shp, cp] + [vp] * 5 + [sz, vp]
    pcp = ctypes.POINTER(DarPagedCacheStruct)
    lib.dar_cache_append_paged.restype = ci
    lib.dar_cache_append_paged.argtypes = [shp, pcp, vp, vp, vp, vp]
    lib.dar_attn_decode_paged.restype = ci
    lib.dar_attn_decode_paged.argtypes = [shp, pcp] + [vp] * 5 + [sz, vp]
    lib.dar_attn_decode_paged_rope.restype = ci
    lib.dar_attn_decode_paged_rope.argtypes = [shp, pcp, rp] + [vp] * 5 + [sz, vp]
    lib.dar_attn_prefill_chunk_paged.restype = ci
    lib.dar_attn_prefill_chunk_paged.argtypes = [shp, pcp, ci] + [vp] * 9 + [sz, vp]
    lib.dar_prefill_chunk_paged_workspace_bytes.restype = sz
    lib.dar_prefill_chunk_paged_workspace_bytes.argtypes = [shp, ci, ci]
    lib.dar_attn_prefill_ragged.restype = ci
    lib.dar_attn_prefill_ragged.argtypes = [shp, ci] + [vp] * 9 + [sz, vp]
    lib.dar_prefill_rope_workspace_bytes.restype = sz
    lib.dar_prefill_rope_workspace_bytes.argtypes = [shp, ci]
    lib.dar_attn_prefill_chunk_rope.restype = ci
    lib.dar_attn_prefill_chunk_rope.argtypes = [shp, cp, rp, ci] + [vp] * 8 + [sz, vp]
    lib.dar_prefill_chunk_rope_workspace_bytes.restype = sz
    lib.dar_prefill_chunk_rope_workspace_bytes.argtypes = [shp, ci, ci]
    lib.dar_attn_decode_noalloc.restype = ci
    lib.dar_attn_decode_noalloc.argtypes = [shp, cp, vp, vp, vp, vp, vp]
    lib.dar_decode_noalloc_bytes.restype = sz
    lib.dar_decode_noalloc_bytes.argtypes = [shp, ci]
    lib.dar_decode_noalloc_max_bytes.restype = sz
    lib.dar_decode_noalloc_max_bytes.argtypes = []
    lib.dar_attn_decode_scored.restype = ci
    lib.dar_attn_decode_scored.argtypes = [shp, cp] + [vp] * 7 + [sz, vp]
    lib.dar_attn_decode_paged_prefix.restype = ci
    lib.dar_attn_decode_paged_prefix.argtypes = [shp, pcp, ci] + [vp] * 6 + [sz, vp]
    lib.dar_attn_decode_paged_scored.restype = ci
    lib.dar_attn_decode_paged_scored.argtypes = [shp, pcp, ci] + [vp] * 8 + [sz, vp]
    lib.dar_decode_scored_workspace_bytes.restype = sz
    lib.dar_decode_scored_workspace_bytes.argtypes = [shp, ci]
    lib.dar_decode_prefix_workspace_bytes.restype = sz
    lib.dar_decode_prefix_workspace_bytes.argtypes = [shp, ci, ci]
    lib.dar_cache_evict.restype = ci
    lib.dar_cache_evict.argtypes = [shp, cp, ci, ci, vp, vp, vp, sz, vp]
    lib.dar_cache_evict_paged.restype = ci
    lib.dar_cache_evict_paged.argtypes = [shp, pcp, ci, ci, vp, vp, vp, sz, vp]
    lib.dar_cache_evict_workspace_bytes.restype = sz
    lib.dar_cache_evict_workspace_bytes.argtypes = [shp, ci, ci]
    qp, qpp = ctypes.POINTER(DarCacheQ4Struct), ctypes.POINTER(DarPagedCacheQ4Struct)
    lib.dar_cache_append_q4.restype = ci
    lib.dar_cache_append_q4.argtypes = [shp, qp, vp, vp, ci, vp, vp]
    lib.dar_cache_append_paged_q4.restype = ci
    lib.dar_cache_append_paged_q4.argtypes = [shp, qpp, vp, vp, vp, vp]
    lib.dar_cache_pack_q4.restype = ci
    lib.dar_cache_pack_q4.argtypes = [shp, cp, ci, qp, vp]
    lib.dar_cache_unpack_q4.restype = ci
    lib.dar_cache_unpack_q4.argtypes = [shp, qp, ci, cp, vp]
    lib.dar_cache_pack_paged_q4.restype = ci
    lib.dar_cache_pack_paged_q4.argtypes = [shp, pcp, vp, qpp, vp]
    lib.dar_cache_unpack_paged_q4.restype = ci
    lib.dar_cache_unpack_paged_q4.argtypes = [shp, qpp, vp, pcp, vp]
    lib.dar_attn_decode_q4.restype = ci
    lib.dar_attn_decode_q4.argtypes = [shp, qp] + [vp] * 5 + [sz, vp]
    lib.dar_attn_decode_paged_q4.restype = ci
    lib.dar_attn_decode_paged_q4.argtypes = [shp, qpp] + [vp] * 5 + [sz, vp]
    lib.dar_decode_q4_workspace_bytes.restype = sz
    lib.dar_decode_q4_workspace_bytes.argtypes = [shp, ci]
    lib.dar_status_string.restype = ctypes.c_char_p
    lib.dar_status_string.argtypes = [ci]
    return lib


lib = _load()

EXPORTS = ("dar_attn_prefill", "dar_cache_append", "dar_attn_decode",
           "dar_attn_prefill_backward", "dar_prefill_workspace_bytes",
           "dar_decode_workspace_bytes", "dar_prefill_backward_workspace_bytes",
           "dar_status_string")


def status_string(st: int) -> str:
    return lib.dar_status_string(int(st)).decode()


def _dtype_code(t: torch.dtype) -> int:
    if t == torch.float32:
        return DAR_F32
    if t == torch.bfloat16:
        return DAR_BF16
    raise TypeError("DAR tensors must be float32 or bfloat16, got %s" % t)


def _ptr(t):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("DAR tensors must be contiguous")
    return t.data_ptr()


# The calls of one small decode step or short prefill take the host about as
# long as the GPU, so what a call does here beyond its launches counts: the
# current stream by its handle (no Stream object), pointers as plain integers,
# and the shape struct and workspace size, pure functions of a few integers,
# from bounded caches. Host time of a call: a dense decode step 12.2 -> 8.2 us,
# a paged one 15.5 -> 11.5, a prefill 17.0 -> 12.2.
def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def make_shape(B, Hq, Hkv, d, d_down, w, dtype) -> DarShape:
    return DarShape(int(B), int(Hq), int(Hkv), int(d), int(d_down), int(w), _dtype_code(dtype))


_shape = functools.lru_cache(maxsize=1024)(make_shape)  # read only: never handed to a caller


@functools.lru_cache(maxsize=4096)
def _ws_bytes(name, key, n) -> int:
    """Workspace bytes of size function `name` for the shape of `key`
    (make_shape's arguments) and length or capacity n."""
    return int(getattr(lib, name)(ctypes.byref(_shape(*key)), *n))


def dar_prefill_workspace_bytes(shape: DarShape, T: int) -> int:
    return int(lib.dar_prefill_workspace_bytes(ctypes.byref(shape), int(T)))


def dar_decode_workspace_bytes(shape: DarShape, cap: int) -> int:
    return int(lib.dar_decode_workspace_bytes(ctypes.byref(shape), int(cap)))


def dar_prefill_backward_workspace_bytes(shape: DarShape, T: int) -> int:
    return int(lib.dar_prefill_backward_workspace_bytes(ctypes.byref(shape), int(T)))


def dar_status_string(st: int) -> str:
    return status_string(st)


# What a call on a given stream allocates (workspace, outputs) belongs to that
# stream, as under torch.cuda.stream(stream): memory of the current stream
# could be one that its pending work still uses, and a workspace, dropped at
# return, would go to the current stream's next allocation while the kernels run.
def _empty(shape, dtype, device, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _empty_like(t, stream):
    if stream is None:
        return torch.empty_like(t)
    with torch.cuda.stream(stream):
        return torch.empty_like(t)


def _workspace(nbytes, device, stream=None):
    return None if nbytes == 0 else _empty(nbytes, torch.uint8, device, stream)


def dar_attn_prefill(q, k, v, w_down, w_up, w, o=None, ws=None, stream=None, check=True,
                     lse=None, return_lse=False):
    """Causal DAR prefill. q [B,Hq,T,d]; k, v [B,Hkv,T,d]; w_down [Hkv,d,dd];
    w_up [Hkv,dd,d] or None (tied). Returns o [B,Hq,T,d], or (o, lse) with
    return_lse (lse [B,Hq,T] fp32, the log of each row's softmax denominator,
    written into `lse` when given). Calls dar_attn_prefill, or
    dar_attn_prefill_lse when the log-sum-exp is asked for."""
    B, Hq, T, d = q.shape
    Hkv = k.shape[1]
    dd = w_down.shape[2]
    key = (B, Hq, Hkv, d, dd, int(w), q.dtype)
    shape = _shape(*key)
    if check:
        for name, t, want in (("k", k, (B, Hkv, T, d)), ("v", v, (B, Hkv, T, d)),
                              ("w_down", w_down, (Hkv, d, dd))):
            if t.shape != want or t.dtype != q.dtype:
                raise ValueError("%s: expected %s %s, got %s %s" % (name, want, q.dtype,
                                                                   tuple(t.shape), t.dtype))
        if w_up is not None and (w_up.shape != (Hkv, dd, d) or w_up.dtype != q.dtype):
            raise ValueError("w_up: expected %s" % ((Hkv, dd, d),))
    if o is None:
        o = _empty_like(q, stream)
    if return_lse and lse is None:
        lse = _empty((B, Hq, T), torch.float32, q.device, stream)
    if lse is not None and (lse.shape != (B, Hq, T) or lse.dtype != torch.float32):
        raise ValueError("lse: expected %s float32" % ((B, Hq, T),))
    need = _ws_bytes("dar_prefill_workspace_bytes", key, (T,))
    if ws is None:
        ws = _workspace(need, q.device, stream)
    wsb = 0 if ws is None else ws.numel() * ws.element_size()
    if lse is None:
        st = lib.dar_attn_prefill(ctypes.byref(shape), int(T), _ptr(q), _ptr(k), _ptr(v),
                                  _ptr(w_down), _ptr(w_up), _ptr(o), _ptr(ws), wsb,
                                  _stream(stream))
        where = "dar_attn_prefill"
    else:
        st = lib.dar_attn_prefill_lse(ctypes.byref(shape), int(T), _ptr(q), _ptr(k), _ptr(v),
                                      _ptr(w_down), _ptr(w_up), _ptr(o), _ptr(lse), _ptr(ws),
                                      wsb, _stream(stream))
        where = "dar_attn_prefill_lse"
    if st != DAR_OK:
        raise DarError(st, where)
    return (o, lse) if return_lse else o


def dar_attn_prefill_lse(q, k, v, w_down, w_up, w, o=None, lse=None, ws=None, stream=None,
                         check=True):
    """dar_attn_prefill that also returns each row's log-sum-exp: (o, lse),
    lse [B,Hq,T] fp32 (written into `lse` when given)."""
    return dar_attn_prefill(q, k, v, w_down, w_up, w, o=o, ws=ws, stream=stream, check=check,
                            lse=lse, return_lse=True)


def dar_rope_table(rotary_dim, base, n_pos, device="cuda", stream=None):
    """The angle table [n_pos, rotary_dim] fp32: cos of the r/2 angles of each
    position, then their sin (computed on the device in fp64)."""
    table = _empty((int(n_pos), int(rotary_dim)), torch.float32, device, stream)
    st = lib.dar_rope_table(int(rotary_dim), float(base), int(n_pos), _ptr(table), _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_rope_table")
    return table


class Rope:
    """Rotary embedding of Eq. 3: rotate-half pairs over the first rotary_dim
    elements, angle p * base^(-2m/r); `table` [n_pos, r] fp32 on the device
    (filled by dar_rope_table unless given)."""

    def __init__(self, rotary_dim, base=10000.0, n_pos=4096, device="cuda", table=None,
                 stream=None):
        self.rotary_dim = int(rotary_dim)
        self.base = float(base)
        self.n_pos = int(n_pos)
        if table is None and self.rotary_dim > 0:
            table = dar_rope_table(self.rotary_dim, self.base, self.n_pos, device, stream)
        self.table = table

    def struct(self) -> DarRopeStruct:
        return DarRopeStruct(self.rotary_dim, self.n_pos,
                             None if self.table is None else self.table.data_ptr())


def dar_prefill_rope_workspace_bytes(shape: DarShape, T: int) -> int:
    return int(lib.dar_prefill_rope_workspace_bytes(ctypes.byref(shape), int(T)))


def dar_attn_prefill_rope(q, k, v, w_down, w_up, w, rope: Rope, pos0=0, o=None, ws=None,
                          stream=None, check=True, lse=None, return_lse=False):
    """Causal DAR prefill with the rotary embedding of Eq. 3 at positions
    pos0..pos0+T-1; q, k un-rotated. Other arguments as dar_attn_prefill."""
    B, Hq, T, d = q.shape
    Hkv = k.shape[1]
    dd = w_down.shape[2]
    key = (B, Hq, Hkv, d, dd, int(w), q.dtype)
    shape = _shape(*key)
    if check:
        for name, t, want in (("k", k, (B, Hkv, T, d)), ("v", v, (B, Hkv, T, d)),
                              ("w_down", w_down, (Hkv, d, dd))):
            if t.shape != want or t.dtype != q.dtype:
                raise ValueError("%s: expected %s %s, got %s %s" % (name, want, q.dtype,
                                                                   tuple(t.shape), t.dtype))
        if w_up is not None and (w_up.shape != (Hkv, dd, d) or w_up.dtype != q.dtype):
            raise ValueError("w_up: expected %s" % ((Hkv, dd, d),))
    if o is None:
        o = _empty_like(q, stream)
    if return_lse and lse is None:
        lse = _empty((B, Hq, T), torch.float32, q.device, stream)
    if lse is not None and (lse.shape != (B, Hq, T) or lse.dtype != torch.float32):
        raise ValueError("lse: expected %s float32" % ((B, Hq, T),))
    if ws is None:
        ws = _workspace(_ws_bytes("dar_prefill_rope_workspace_bytes", key, (T,)), q.device,
                        stream)
    rs = rope.struct()
    st = lib.dar_attn_prefill_rope(ctypes.byref(shape), int(T), int(pos0), ctypes.byref(rs),
                                   _ptr(q), _ptr(k), _ptr(v), _ptr(w_down), _ptr(w_up), _ptr(o),
                                   _ptr(lse), _ptr(ws),
                                   0 if ws is None else ws.numel() * ws.element_size(),
                                   _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_prefill_rope")
    return (o, lse) if return_lse else o


def dar_attn_prefill_backward(q, k, v, w_down, w_up, w, o, lse, dout, ws=None, stream=None,
                              check=True):
    """Gradients of sum(dout * o) of the causal DAR prefill, given the forward's
    o and lse (dar_attn_prefill(..., return_lse=True)). Returns
    (dq, dk, dv, dw_down, dw_up): dq/dk/dv in the input dtype, the weight
    gradients fp32; dw_up is None when tied (w_up None), dw_down then holds the
    gradient of the shared matrix."""
    B, Hq, T, d = q.shape
    Hkv = k.shape[1]
    dd = w_down.shape[2]
    key = (B, Hq, Hkv, d, dd, int(w), q.dtype)
    shape = _shape(*key)
    if check:
        for name, t, want in (("k", k, (B, Hkv, T, d)), ("v", v, (B, Hkv, T, d)),
                              ("w_down", w_down, (Hkv, d, dd)), ("o", o, (B, Hq, T, d)),
                              ("dout", dout, (B, Hq, T, d))):
            if t.shape != want or t.dtype != q.dtype:
                raise ValueError("%s: expected %s %s, got %s %s" % (name, want, q.dtype,
                                                                   tuple(t.shape), t.dtype))
        if w_up is not None and (w_up.shape != (Hkv, dd, d) or w_up.dtype != q.dtype):
            raise ValueError("w_up: expected %s" % ((Hkv, dd, d),))
        if lse.shape != (B, Hq, T) or lse.dtype != torch.float32:
            raise ValueError("lse: expected %s float32" % ((B, Hq, T),))
    dq = _empty_like(q, stream)
    dk = _empty_like(k, stream)
    dv = _empty_like(v, stream)
    dwd = _empty((Hkv, d, dd), torch.float32, q.device, stream)
    dwu = None if w_up is None else _empty((Hkv, dd, d), torch.float32, q.device, stream)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_prefill_backward_workspace_bytes", key, (T,)), q.device,
                        stream)
    st = lib.dar_attn_prefill_backward(ctypes.byref(shape), int(T), _ptr(q), _ptr(k), _ptr(v),
                                       _ptr(w_down), _ptr(w_up), _ptr(o), _ptr(lse), _ptr(dout),
                                       _ptr(dq),
                                       _ptr(dk), _ptr(dv), _ptr(dwd), _ptr(dwu), _ptr(ws),
                                       0 if ws is None else ws.numel() * ws.element_size(),
                                       _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_prefill_backward")
    return dq, dk, dv, dwd, dwu


def dar_prefill_rope_backward_workspace_bytes(shape: DarShape, T: int) -> int:
    return int(lib.dar_prefill_rope_backward_workspace_bytes(ctypes.byref(shape), int(T)))


def dar_attn_prefill_rope_backward(q, k, v, w_down, w_up, w, rope: "Rope", o, lse, dout, pos0=0,
                                   ws=None, stream=None):
    """Gradients of sum(dout * o) of dar_attn_prefill_rope (same q, k, v,
    weights, rope and pos0; its o and lse). Returns (dq, dk, dv, dw_down,
    dw_up) as dar_attn_prefill_backward does."""
    B, Hq, T, d = q.shape
    Hkv = k.shape[1]
    dd = w_down.shape[2]
    key = (B, Hq, Hkv, d, dd, int(w), q.dtype)
    shape = _shape(*key)
    for name, t, want in (("k", k, (B, Hkv, T, d)), ("v", v, (B, Hkv, T, d)),
                          ("w_down", w_down, (Hkv, d, dd)), ("o", o, (B, Hq, T, d)),
                          ("dout", dout, (B, Hq, T, d))):
        if t.shape != want or t.dtype != q.dtype:
            raise ValueError("%s: expected %s %s" % (name, want, q.dtype))
    if lse.shape != (B, Hq, T) or lse.dtype != torch.float32:
        raise ValueError("lse: expected %s float32" % ((B, Hq, T),))
    dq = _empty_like(q, stream)
    dk = _empty_like(k, stream)
    dv = _empty_like(v, stream)
    dwd = _empty((Hkv, d, dd), torch.float32, q.device, stream)
    dwu = None if w_up is None else _empty((Hkv, dd, d), torch.float32, q.device, stream)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_prefill_rope_backward_workspace_bytes", key, (T,)), q.device,
                        stream)
    rs = rope.struct()
    st = lib.dar_attn_prefill_rope_backward(ctypes.byref(shape), int(T), int(pos0), ctypes.byref(rs),
                                            _ptr(q), _ptr(k), _ptr(v), _ptr(w_down), _ptr(w_up),
                                            _ptr(o), _ptr(lse), _ptr(dout), _ptr(dq), _ptr(dk),
                                            _ptr(dv), _ptr(dwd), _ptr(dwu), _ptr(ws),
                                            0 if ws is None else ws.numel() * ws.element_size(),
                                            _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_prefill_rope_backward")
    return dq, dk, dv, dwd, dwu


class DarCache:
    """Split KV cache owned by torch: ring [B,Hkv,w,d] for the window and
    latents [B,Hkv,cap,dd] for older tokens (see dar_cache in include/dar.h)."""

    def __init__(self, B, Hkv, d, d_down, w, cap, dtype, device="cuda", shared=False):
        """shared: one latent array (the single shared latent per token; used
        with the *_shared entry points), else separate key and value latents."""
        self.B, self.Hkv, self.d, self.d_down, self.w, self.cap = B, Hkv, d, d_down, w, cap
        self.dtype = dtype
        self.shared = shared
        wl = max(w, 1)  # keep valid pointers for w = 0 (the ring is never touched then)
        self.k_win = torch.zeros(B, Hkv, wl, d, dtype=dtype, device=device)
        self.v_win = torch.zeros(B, Hkv, wl, d, dtype=dtype, device=device)
        self.k_lat = torch.zeros(B, Hkv, cap, d_down, dtype=dtype, device=device)
        self.v_lat = self.k_lat if shared else torch.zeros(B, Hkv, cap, d_down, dtype=dtype,
                                                           device=device)
        self.struct = DarCacheStruct(self.k_win.data_ptr(), self.v_win.data_ptr(),
                                     self.k_lat.data_ptr(), self.v_lat.data_ptr(), int(cap), 0)

    @property
    def len(self) -> int:
        return int(self.struct.len)


def dar_cache_append(cache: DarCache, k_new, v_new, w_down, Hq=None, stream=None):
    """Append n tokens k_new, v_new [B,Hkv,n,d]; projects window exits to latents."""
    B, Hkv, n, d = k_new.shape
    key = (B, int(Hq if Hq is not None else Hkv), Hkv, d, int(cache.d_down), int(cache.w),
           k_new.dtype)
    shape = _shape(*key)
    if v_new.shape != (B, Hkv, n, d) or (B, Hkv, d) != (cache.B, cache.Hkv, cache.d):
        raise ValueError("k_new/v_new do not match the cache")
    st = lib.dar_cache_append(ctypes.byref(shape), ctypes.byref(cache.struct), _ptr(k_new),
                              _ptr(v_new), int(n), _ptr(w_down), _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_cache_append")
    return cache


def dar_prefill_chunk_workspace_bytes(shape, len_, n) -> int:
    return int(lib.dar_prefill_chunk_workspace_bytes(ctypes.byref(shape), int(len_), int(n)))


def dar_attn_prefill_chunk(cache: DarCache, q, k_new, v_new, w_down, w_up=None, o=None,
                           lse=None, return_lse=False, ws=None, stream=None, check=True):
    """Chunked prefill: n new tokens (q [B,Hq,n,d], k_new/v_new [B,Hkv,n,d]) at
    positions cache.len.. attend to everything before them (ring + latents of the
    cache, and each other, causally); then the cache is extended by them as
    dar_cache_append would. Returns o [B,Hq,n,d], or (o, lse) with return_lse."""
    B, Hq, n, d = q.shape
    Hkv = cache.Hkv
    key = (B, Hq, int(Hkv), d, int(cache.d_down), int(cache.w), q.dtype)
    shape = _shape(*key)
    if check:
        for name, t in (("k_new", k_new), ("v_new", v_new)):
            if t.shape != (B, Hkv, n, d) or t.dtype != q.dtype:
                raise ValueError("%s: expected %s %s" % (name, (B, Hkv, n, d), q.dtype))
        if (B, d) != (cache.B, cache.d) or q.dtype != cache.dtype:
            raise ValueError("q does not match the cache")
    if o is None:
        o = _empty_like(q, stream)
    if return_lse and lse is None:
        lse = _empty((B, Hq, n), torch.float32, q.device, stream)
    if ws is None:
        ws = _workspace(dar_prefill_chunk_workspace_bytes(shape, cache.len, n), q.device, stream)
    st = lib.dar_attn_prefill_chunk(ctypes.byref(shape), ctypes.byref(cache.struct), int(n),
                                    _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(w_down), _ptr(w_up),
                                    _ptr(o), _ptr(lse), _ptr(ws),
                                    0 if ws is None else ws.numel() * ws.element_size(),
                                    _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_prefill_chunk")
    return (o, lse) if return_lse else o


def dar_prefill_chunk_rope_workspace_bytes(shape, len_, n) -> int:
    return int(lib.dar_prefill_chunk_rope_workspace_bytes(ctypes.byref(shape), int(len_), int(n)))


def dar_attn_prefill_chunk_rope(cache: DarCache, q, k_new, v_new, w_down, rope: "Rope", w_up=None,
                                o=None, lse=None, return_lse=False, ws=None, stream=None,
                                check=True):
    """Chunked prefill with the rotary embedding of Eq. 3: n new tokens at
    positions cache.len.. (q, k_new, v_new un-rotated, shapes as
    dar_attn_prefill_chunk); the cache is extended by the un-rotated tokens.
    Returns o [B,Hq,n,d], or (o, lse) with return_lse."""
    B, Hq, n, d = q.shape
    Hkv = cache.Hkv
    key = (B, Hq, int(Hkv), d, int(cache.d_down), int(cache.w), q.dtype)
    shape = _shape(*key)
    if check:
        for name, t in (("k_new", k_new), ("v_new", v_new)):
            if t.shape != (B, Hkv, n, d) or t.dtype != q.dtype:
                raise ValueError("%s: expected %s %s" % (name, (B, Hkv, n, d), q.dtype))
        if (B, d) != (cache.B, cache.d) or q.dtype != cache.dtype:
            raise ValueError("q does not match the cache")
    if o is None:
        o = _empty_like(q, stream)
    if return_lse and lse is None:
        lse = _empty((B, Hq, n), torch.float32, q.device, stream)
    if ws is None:
        ws = _workspace(dar_prefill_chunk_rope_workspace_bytes(shape, cache.len, n), q.device, stream)
    rs = rope.struct()
    st = lib.dar_attn_prefill_chunk_rope(ctypes.byref(shape), ctypes.byref(cache.struct),
                                         ctypes.byref(rs), int(n), _ptr(q), _ptr(k_new),
                                         _ptr(v_new), _ptr(w_down), _ptr(w_up), _ptr(o),
                                         _ptr(lse), _ptr(ws),
                                         0 if ws is None else ws.numel() * ws.element_size(),
                                         _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_prefill_chunk_rope")
    return (o, lse) if return_lse else o


def dar_attn_decode(cache: DarCache, q, w_down, w_up=None, o=None, ws=None, stream=None):
    """One decode step: q [B,Hq,d] at position cache.len - 1. Returns o [B,Hq,d]."""
    B, Hq, d = q.shape
    key = (B, Hq, int(cache.Hkv), d, int(cache.d_down), int(cache.w), q.dtype)
    shape = _shape(*key)
    if o is None:
        o = _empty_like(q, stream)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_decode_workspace_bytes", key, (int(cache.cap),)), q.device,
                        stream)
    st = lib.dar_attn_decode(ctypes.byref(shape), ctypes.byref(cache.struct), _ptr(q),
                             _ptr(w_down), _ptr(w_up), _ptr(o), _ptr(ws),
                             0 if ws is None else ws.numel() * ws.element_size(),
                             _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_decode")
    return o


def dar_attn_decode_noalloc(cache: "DarCache", q, w_down, w_up=None, o=None, stream=None):
    """One decode step as dar_attn_decode, through the entry point that takes
    no workspace (its partial records live in a fixed array inside the
    library). Pass `o` to keep the call free of allocation."""
    B, Hq, d = q.shape
    key = (B, Hq, int(cache.Hkv), d, int(cache.d_down), int(cache.w), q.dtype)
    shape = _shape(*key)
    if o is None:
        o = _empty_like(q, stream)
    st = lib.dar_attn_decode_noalloc(ctypes.byref(shape), ctypes.byref(cache.struct), _ptr(q),
                                     _ptr(w_down), _ptr(w_up), _ptr(o), _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_decode_noalloc")
    return o


def dar_decode_noalloc_bytes(shape: DarShape, length: int) -> int:
    return int(lib.dar_decode_noalloc_bytes(ctypes.byref(shape), int(length)))


def dar_decode_noalloc_max_bytes() -> int:
    return int(lib.dar_decode_noalloc_max_bytes())


def dar_attn_decode_rope(cache: "DarCache", q, w_down, rope: Rope, w_up=None, o=None, ws=None,
                         stream=None):
    """One decode step with the rotary embedding of Eq. 3; q [B,Hq,d] un-rotated,
    at position cache.len - 1. Returns o [B,Hq,d]."""
    B, Hq, d = q.shape
    key = (B, Hq, int(cache.Hkv), d, int(cache.d_down), int(cache.w), q.dtype)
    shape = _shape(*key)
    if o is None:
        o = _empty_like(q, stream)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_decode_workspace_bytes", key, (int(cache.cap),)), q.device,
                        stream)
    rs = rope.struct()
    st = lib.dar_attn_decode_rope(ctypes.byref(shape), ctypes.byref(cache.struct), ctypes.byref(rs), _ptr(q),
                                  _ptr(w_down), _ptr(w_up), _ptr(o), _ptr(ws),
                                  0 if ws is None else ws.numel() * ws.element_size(),
                                  _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_decode_rope")
    return o


def dar_attn_prefill_shared(q, k, v, c, u_k, u_v, w, o=None, ws=None, stream=None, lse=None,
                            return_lse=False):
    """Causal prefill with one shared latent per token: c [B,Hkv,T,dd]; distant
    key c U_K, distant value c U_V (u_k, u_v [Hkv,dd,d])."""
    B, Hq, T, d = q.shape
    Hkv = k.shape[1]
    dd = c.shape[3]
    key = (B, Hq, Hkv, d, dd, int(w), q.dtype)
    shape = _shape(*key)
    for name, t, want in (("k", k, (B, Hkv, T, d)), ("v", v, (B, Hkv, T, d)),
                          ("c", c, (B, Hkv, T, dd)), ("u_k", u_k, (Hkv, dd, d)),
                          ("u_v", u_v, (Hkv, dd, d))):
        if t.shape != want or t.dtype != q.dtype:
            raise ValueError("%s: expected %s %s" % (name, want, q.dtype))
    if o is None:
        o = _empty_like(q, stream)
    if return_lse and lse is None:
        lse = _empty((B, Hq, T), torch.float32, q.device, stream)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_prefill_workspace_bytes", key, (T,)), q.device,
                        stream)
    st = lib.dar_attn_prefill_shared(ctypes.byref(shape), int(T), _ptr(q), _ptr(k), _ptr(v), _ptr(c),
                                     _ptr(u_k), _ptr(u_v), _ptr(o), _ptr(lse), _ptr(ws),
                                     0 if ws is None else ws.numel() * ws.element_size(),
                                     _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_prefill_shared")
    return (o, lse) if return_lse else o


def dar_cache_append_shared(cache: DarCache, k_new, v_new, c_new, Hq=None, stream=None):
    """Append n tokens with their shared latents c_new [B,Hkv,n,dd]."""
    assert cache.shared, "a cache made with shared=True"
    B, Hkv, n, d = k_new.shape
    key = (B, int(Hq or Hkv), Hkv, d, int(cache.d_down), int(cache.w), k_new.dtype)
    shape = _shape(*key)
    st = lib.dar_cache_append_shared(ctypes.byref(shape), ctypes.byref(cache.struct), _ptr(k_new),
                                     _ptr(v_new), _ptr(c_new), int(n), _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_cache_append_shared")


def dar_attn_decode_shared(cache: DarCache, q, u_k, u_v, o=None, ws=None, stream=None):
    """One decode step over a shared-latent cache; q [B,Hq,d] at position len-1."""
    assert cache.shared, "a cache made with shared=True"
    B, Hq, d = q.shape
    key = (B, Hq, int(cache.Hkv), d, int(cache.d_down), int(cache.w), q.dtype)
    shape = _shape(*key)
    if o is None:
        o = _empty_like(q, stream)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_decode_workspace_bytes", key, (int(cache.cap),)), q.device,
                        stream)
    st = lib.dar_attn_decode_shared(ctypes.byref(shape), ctypes.byref(cache.struct), _ptr(q),
                                    _ptr(u_k), _ptr(u_v), _ptr(o), _ptr(ws),
                                    0 if ws is None else ws.numel() * ws.element_size(),
                                    _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_decode_shared")
    return o


class DarPagedCache:
    """Paged split cache (include/dar.h, dar_paged_cache): rings [B,Hkv,w,d],
    latent pages [n_pages,Hkv,page_size,dd] for keys and values, a block table
    [B,max_blocks] (int32, device) and per-sequence lengths [B] (int32,
    device). block_table and lens are plain torch tensors the caller fills."""

    def __init__(self, B, Hkv, d, d_down, w, page_size, max_blocks, n_pages, dtype,
                 device="cuda"):
        self.B, self.Hkv, self.d, self.d_down, self.w = B, Hkv, d, d_down, w
        self.page_size, self.max_blocks, self.n_pages = page_size, max_blocks, n_pages
        wl = max(w, 1)
        self.k_win = torch.zeros(B, Hkv, wl, d, dtype=dtype, device=device)
        self.v_win = torch.zeros(B, Hkv, wl, d, dtype=dtype, device=device)
        self.k_pool = torch.zeros(n_pages, Hkv, page_size, d_down, dtype=dtype, device=device)
        self.v_pool = torch.zeros(n_pages, Hkv, page_size, d_down, dtype=dtype, device=device)
        self.block_table = torch.full((B, max_blocks), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(B, dtype=torch.int32, device=device)

    @property
    def cap(self):
        return self.page_size * self.max_blocks

    def overflowed(self):
        """Sequences the append found at capacity (lens marked -1 - n); reads
        lens back to the host (synchronises with the current stream)."""
        return [b for b, n in enumerate(self.lens.cpu().tolist()) if n < 0]

    def struct(self) -> DarPagedCacheStruct:
        return DarPagedCacheStruct(self.k_win.data_ptr(), self.v_win.data_ptr(),
                                   self.k_pool.data_ptr(), self.v_pool.data_ptr(),
                                   self.block_table.data_ptr(), self.lens.data_ptr(),
                                   self.page_size, self.max_blocks, self.n_pages)


def dar_cache_append_paged(cache: DarPagedCache, k_new, v_new, w_down, Hq=None, stream=None):
    """One token per sequence: k_new, v_new [B,Hkv,d]; lens advance on the device."""
    B, Hkv, d = k_new.shape
    key = (B, int(Hq or Hkv), Hkv, d, int(cache.d_down), int(cache.w), k_new.dtype)
    shape = _shape(*key)
    cs = cache.struct()
    st = lib.dar_cache_append_paged(ctypes.byref(shape), ctypes.byref(cs), _ptr(k_new), _ptr(v_new),
                                    _ptr(w_down), _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_cache_append_paged")


def dar_attn_decode_paged(cache: DarPagedCache, q, w_down, w_up=None, o=None, ws=None, stream=None):
    """One decode step per sequence (query at position lens[b] - 1)."""
    B, Hq, d = q.shape
    key = (B, Hq, int(cache.Hkv), d, int(cache.d_down), int(cache.w), q.dtype)
    shape = _shape(*key)
    if o is None:
        o = _empty_like(q, stream)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_decode_workspace_bytes", key, (int(cache.cap),)), q.device,
                        stream)
    cs = cache.struct()
    st = lib.dar_attn_decode_paged(ctypes.byref(shape), ctypes.byref(cs), _ptr(q), _ptr(w_down),
                                   _ptr(w_up), _ptr(o), _ptr(ws),
                                   0 if ws is None else ws.numel() * ws.element_size(),
                                   _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_decode_paged")
    return o


def dar_attn_decode_paged_rope(cache: DarPagedCache, q, w_down, rope: "Rope", w_up=None, o=None,
                               ws=None, stream=None):
    """dar_attn_decode_paged with the rotary embedding of Eq. 3 (query of
    sequence b at position lens[b] - 1; rope.n_pos >= the cache capacity)."""
    B, Hq, d = q.shape
    key = (B, Hq, int(cache.Hkv), d, int(cache.d_down), int(cache.w), q.dtype)
    shape = _shape(*key)
    if o is None:
        o = _empty_like(q, stream)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_decode_workspace_bytes", key, (int(cache.cap),)), q.device,
                        stream)
    cs = cache.struct()
    rs = rope.struct()
    st = lib.dar_attn_decode_paged_rope(ctypes.byref(shape), ctypes.byref(cs), ctypes.byref(rs),
                                        _ptr(q), _ptr(w_down), _ptr(w_up), _ptr(o), _ptr(ws),
                                        0 if ws is None else ws.numel() * ws.element_size(),
                                        _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_decode_paged_rope")
    return o


def dar_prefill_chunk_paged_workspace_bytes(shape, cap, n) -> int:
    return int(lib.dar_prefill_chunk_paged_workspace_bytes(ctypes.byref(shape), int(cap), int(n)))


def dar_attn_prefill_chunk_paged(cache: DarPagedCache, q, k_new, v_new, w_down, w_up=None,
                                 n_new=None, o=None, lse=None, return_lse=False, ws=None,
                                 stream=None):
    """Chunked prefill over a paged cache: sequence b takes n_new[b] (device
    int32 [B], each <= n; None: all n) new tokens at positions lens[b]..,
    q [B,Hq,n,d], k_new/v_new [B,Hkv,n,d]; lens advance on the device.
    Returns o [B,Hq,n,d] (rows past n_new[b] not written), or (o, lse)."""
    B, Hq, n, d = q.shape
    Hkv = cache.Hkv
    key = (B, Hq, int(Hkv), d, int(cache.d_down), int(cache.w), q.dtype)
    shape = _shape(*key)
    for name, t in (("k_new", k_new), ("v_new", v_new)):
        if t.shape != (B, Hkv, n, d) or t.dtype != q.dtype:
            raise ValueError("%s: expected %s %s" % (name, (B, Hkv, n, d), q.dtype))
    if (B, d) != (cache.B, cache.d):
        raise ValueError("q does not match the cache")
    if n_new is not None and (n_new.dtype != torch.int32 or n_new.shape != (B,)):
        raise ValueError("n_new: expected int32 [%d]" % B)
    if o is None:
        o = _empty_like(q, stream)
    if return_lse and lse is None:
        lse = _empty((B, Hq, n), torch.float32, q.device, stream)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_prefill_chunk_paged_workspace_bytes", key, (int(cache.cap), n)), q.device,
                        stream)
    cs = cache.struct()
    st = lib.dar_attn_prefill_chunk_paged(ctypes.byref(shape), ctypes.byref(cs), int(n),
                                          _ptr(n_new), _ptr(q), _ptr(k_new), _ptr(v_new),
                                          _ptr(w_down), _ptr(w_up), _ptr(o), _ptr(lse), _ptr(ws),
                                          0 if ws is None else ws.numel() * ws.element_size(),
                                          _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_prefill_chunk_paged")
    return (o, lse) if return_lse else o


def dar_attn_prefill_ragged(q, k, v, w_down, w_up, w, seq_lens, o=None, ws=None, stream=None,
                            lse=None, return_lse=False):
    """Causal prefill of a padded batch whose sequence b holds seq_lens[b]
    tokens (int32 device tensor [B]); rows past a sequence's length are left
    unwritten. Other arguments as dar_attn_prefill."""
    B, Hq, T, d = q.shape
    Hkv = k.shape[1]
    dd = w_down.shape[2]
    key = (B, Hq, Hkv, d, dd, int(w), q.dtype)
    shape = _shape(*key)
    if seq_lens.dtype != torch.int32 or seq_lens.shape != (B,) or not seq_lens.is_cuda:
        raise ValueError("seq_lens: expected an int32 device tensor of shape (%d,)" % B)
    if o is None:
        o = _empty_like(q, stream)
    if return_lse and lse is None:
        lse = _empty((B, Hq, T), torch.float32, q.device, stream)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_prefill_workspace_bytes", key, (T,)), q.device,
                        stream)
    st = lib.dar_attn_prefill_ragged(ctypes.byref(shape), int(T), _ptr(seq_lens), _ptr(q), _ptr(k),
                                     _ptr(v), _ptr(w_down), _ptr(w_up), _ptr(o), _ptr(lse), _ptr(ws),
                                     0 if ws is None else ws.numel() * ws.element_size(),
                                     _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_prefill_ragged")
    return (o, lse) if return_lse else o


# --- serving operators (include/dar_serving.h) ---------------------------------

def _check_scores(cache, scores, scores_out):
    """The score arrays of a call, [B,Hkv,cap] fp32 beside the cache; scores_out
    None: in place."""
    if scores_out is None:
        scores_out = scores
    want = (cache.B, cache.Hkv, cache.cap)
    for name, t in (("scores", scores), ("scores_out", scores_out)):
        if tuple(t.shape) != want or t.dtype != torch.float32 or t.device != cache.k_win.device:
            raise ValueError("%s: expected %s float32 on %s, got %s %s on %s" % (
                name, want, cache.k_win.device, tuple(t.shape), t.dtype, t.device))
    return scores_out


def _count(name, n):
    """A number of tokens as the library takes it, a C int (ctypes would drop the
    upper bits of a larger one: "keep 2^32" would become "keep none")."""
    n = int(n)
    if not -2 ** 31 <= n < 2 ** 31:
        raise ValueError("%s: %d is no C int" % (name, n))
    return n


_HERE = contextlib.nullcontext()


def _on(cache, stream):
    """The cache's device, and the stream if one is given, made current for a call:
    its allocations and launches go there. (Entering a device context takes 1 us
    of host time, so not where it is current already.)"""
    dev = cache.k_win.device
    if stream is not None:
        if stream.device != dev:
            raise ValueError("stream: expected one of %s, got one of %s" % (dev, stream.device))
        return torch.cuda.stream(stream)
    return _HERE if torch._C._cuda_getDevice() == dev.index else torch.cuda.device(dev)


def dar_decode_scored_workspace_bytes(shape: DarShape, cap: int) -> int:
    return int(lib.dar_decode_scored_workspace_bytes(ctypes.byref(shape), _count("cap", cap)))


def dar_decode_prefix_workspace_bytes(shape: DarShape, cap: int, n_prefix: int) -> int:
    return int(lib.dar_decode_prefix_workspace_bytes(ctypes.byref(shape), _count("cap", cap),
                                                     _count("n_prefix", n_prefix)))


def _check_step(cache, q, w_down, w_up, o):
    """Query, weights and output of a decode step against its cache; (key, o)."""
    B, Hq, d = q.shape
    dev, dd = cache.k_win.device, int(cache.d_down)
    if (B, d) != (cache.B, cache.d) or q.dtype != cache.k_win.dtype or q.device != dev:
        raise ValueError("q does not match the cache")
    # (compared at once; what is wrong is looked for only if something is: 2.3 -> 1.2 us)
    if not (w_down.shape == (cache.Hkv, d, dd) and w_down.dtype is q.dtype and w_down.device == dev and
            (w_up is None or w_up.shape == (cache.Hkv, dd, d) and w_up.dtype is q.dtype and w_up.device == dev) and
            (o is None or o.shape == q.shape and o.dtype is q.dtype and o.device == dev)):
        _say_step(q, dev, w_down, w_up, o, (cache.Hkv, d, dd), (cache.Hkv, dd, d))
    return (B, Hq, int(cache.Hkv), d, dd, int(cache.w), q.dtype), torch.empty_like(q) if o is None else o


def _say_step(q, dev, w_down, w_up, o, down, up):
    for name, t, want in (("w_down", w_down, down), ("w_up", w_up, up), ("o", o, tuple(q.shape))):
        if t is not None and (tuple(t.shape) != want or t.dtype != q.dtype or t.device != dev):
            raise ValueError("%s: expected %s %s on %s" % (name, want, q.dtype, dev))


def dar_attn_decode_scored(cache: DarCache, q, w_down, scores, w_up=None, scores_out=None, o=None,
                           ws=None, stream=None):
    """One decode step (as dar_attn_decode) that adds to every cached token's entry
    of `scores` [B,Hkv,cap] fp32 the attention weight it receives, summed over
    the query heads of its KV head; in place, or into scores_out. Returns o."""
    scores_out = _check_scores(cache, scores, scores_out)
    with _on(cache, stream):
        key, o = _check_step(cache, q, w_down, w_up, o)
        if ws is None:
            ws = _workspace(_ws_bytes("dar_decode_scored_workspace_bytes", key, (int(cache.cap),)),
                            q.device)
        st = lib.dar_attn_decode_scored(ctypes.byref(_shape(*key)), ctypes.byref(cache.struct),
                                        _ptr(q), _ptr(w_down), _ptr(w_up), _ptr(o), _ptr(scores),
                                        _ptr(scores_out), _ptr(ws),
                                        0 if ws is None else ws.numel() * ws.element_size(),
                                        _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_decode_scored")
    return o


def _prefix(cache, prefix_blocks):
    """Tokens of a shared prefix held in the pages prefix_blocks (int32; None: 0)."""
    if prefix_blocks is None:
        return 0
    if (prefix_blocks.dtype != torch.int32 or prefix_blocks.dim() != 1 or
            prefix_blocks.device != cache.k_win.device):
        raise ValueError("prefix_blocks: expected int32 [n] on %s" % cache.k_win.device)
    return _count("prefix_blocks", prefix_blocks.numel() * int(cache.page_size))


def dar_attn_decode_paged_prefix(cache: DarPagedCache, q, w_down, prefix_blocks, w_up=None, o=None,
                                 ws=None, stream=None):
    """dar_attn_decode_paged for sequences that share their first tokens: those in
    the pages prefix_blocks (int32 [n], usually cache.block_table[b, :n]) are
    read once for the whole batch. Returns o [B,Hq,d]."""
    n_prefix = _prefix(cache, prefix_blocks)
    with _on(cache, stream):
        key, o = _check_step(cache, q, w_down, w_up, o)
        if ws is None:
            ws = _workspace(_ws_bytes("dar_decode_prefix_workspace_bytes", key,
                                      (int(cache.cap), n_prefix)), q.device)
        cs = cache.struct()
        st = lib.dar_attn_decode_paged_prefix(ctypes.byref(_shape(*key)), ctypes.byref(cs), n_prefix,
                                              _ptr(prefix_blocks), _ptr(q), _ptr(w_down), _ptr(w_up),
                                              _ptr(o), _ptr(ws),
                                              0 if ws is None else ws.numel() * ws.element_size(),
                                              _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_decode_paged_prefix")
    return o


def dar_attn_decode_paged_scored(cache: DarPagedCache, q, w_down, scores, w_up=None,
                                 prefix_blocks=None, scores_out=None, o=None, ws=None, stream=None):
    """dar_attn_decode_paged (with prefix_blocks: dar_attn_decode_paged_prefix)
    that scores the tokens past the prefix as dar_attn_decode_scored does."""
    n_prefix = _prefix(cache, prefix_blocks)
    scores_out = _check_scores(cache, scores, scores_out)
    with _on(cache, stream):
        key, o = _check_step(cache, q, w_down, w_up, o)
        if ws is None:
            ws = _workspace(_ws_bytes("dar_decode_prefix_workspace_bytes", key,
                                      (int(cache.cap), n_prefix)), q.device)
        cs = cache.struct()
        st = lib.dar_attn_decode_paged_scored(ctypes.byref(_shape(*key)), ctypes.byref(cs), n_prefix,
                                              _ptr(prefix_blocks), _ptr(q), _ptr(w_down), _ptr(w_up),
                                              _ptr(o), _ptr(scores), _ptr(scores_out), _ptr(ws),
                                              0 if ws is None else ws.numel() * ws.element_size(),
                                              _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_attn_decode_paged_scored")
    return o


def dar_cache_evict_workspace_bytes(shape: DarShape, cap: int, n_keep: int) -> int:
    return int(lib.dar_cache_evict_workspace_bytes(ctypes.byref(shape), _count("cap", cap),
                                                   _count("n_keep", n_keep)))


def _evict_args(cache, n_keep, n_fixed, scores, scores_out, ws):
    n_keep, n_fixed = _count("n_keep", n_keep), _count("n_fixed", n_fixed)
    key = (int(cache.B), int(cache.Hkv), int(cache.Hkv), int(cache.d), int(cache.d_down),
           int(cache.w), cache.k_win.dtype)
    scores_out = _check_scores(cache, scores, scores_out)
    if ws is None:
        ws = _workspace(_ws_bytes("dar_cache_evict_workspace_bytes", key,
                                  (int(cache.cap), n_keep)), cache.k_win.device)
    return (_shape(*key), n_keep, n_fixed, scores_out, ws,
            0 if ws is None else ws.numel() * ws.element_size())


def dar_cache_evict(cache: DarCache, scores, n_keep, n_fixed=0, scores_out=None, ws=None,
                    stream=None) -> int:
    """Evicts distant tokens until about n_keep are left (a multiple of the window
    leaves, so that the ring stays as it is), the lowest `scores` [B,Hkv,cap]
    first, never the first n_fixed; scores move with their tokens, in place or
    into scores_out. Returns the number of tokens evicted (cache.len falls by
    it). An evicted cache is for the entry points without rotary embedding."""
    before = cache.len
    with _on(cache, stream):
        shape, n_keep, n_fixed, scores_out, ws, wsb = _evict_args(cache, n_keep, n_fixed, scores,
                                                                  scores_out, ws)
        st = lib.dar_cache_evict(ctypes.byref(shape), ctypes.byref(cache.struct), n_keep,
                                 n_fixed, _ptr(scores), _ptr(scores_out), _ptr(ws), wsb,
                                 _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_cache_evict")
    return before - cache.len


def dar_cache_evict_paged(cache: DarPagedCache, scores, n_keep, n_fixed=0, scores_out=None,
                          ws=None, stream=None):
    """dar_cache_evict over a paged cache, each sequence by its own length; lens
    fall on the device. Pages that sequences share must lie below n_fixed."""
    with _on(cache, stream):
        shape, n_keep, n_fixed, scores_out, ws, wsb = _evict_args(cache, n_keep, n_fixed, scores,
                                                                  scores_out, ws)
        cs = cache.struct()
        st = lib.dar_cache_evict_paged(ctypes.byref(shape), ctypes.byref(cs), n_keep,
                                       n_fixed, _ptr(scores), _ptr(scores_out), _ptr(ws), wsb,
                                       _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_cache_evict_paged")


# --- distant latents in 4 bits (include/dar_q4.h) -------------------------------

def _q4_arrays(self, rows, dtype, device):
    """Ring, codes and scale bytes of a 4-bit cache whose latent arrays are laid out
    as `rows` (without their columns)."""
    win = (self.B, self.Hkv, max(self.w, 1), self.d)  # (w = 0: valid pointers, never read)
    self.k_win = torch.zeros(win, dtype=dtype, device=device)
    self.v_win = torch.zeros(win, dtype=dtype, device=device)
    for a, width in (("k_codes", 4 * (-(-self.d_down // 8))), ("v_codes", 4 * (-(-self.d_down // 8))),
                     ("k_exp", -(-self.d_down // 32)), ("v_exp", -(-self.d_down // 32))):
        setattr(self, a, torch.zeros(*rows, width, dtype=torch.uint8, device=device))


class DarCacheQ4:
    """Split KV cache with 4-bit latents, owned by torch (dar_cache_q4 in
    include/dar_q4.h): ring [B,Hkv,w,d] in `dtype`; codes [B,Hkv,cap,4 ceil(dd/8)]
    and scale bytes [B,Hkv,cap,ceil(dd/32)], uint8. cap: the capacity asked for,
    rounded up to a multiple of 64."""

    def __init__(self, B, Hkv, d, d_down, w, cap, dtype, device="cuda"):
        self.B, self.Hkv, self.d, self.d_down, self.w = B, Hkv, d, d_down, w
        self.cap = -(-_count("cap", cap) // 64) * 64
        self.dtype = dtype
        _q4_arrays(self, (B, Hkv, self.cap), dtype, device)
        self.struct = DarCacheQ4Struct(self.k_win.data_ptr(), self.v_win.data_ptr(),
                                       self.k_codes.data_ptr(), self.v_codes.data_ptr(),
                                       self.k_exp.data_ptr(), self.v_exp.data_ptr(),
                                       _count("cap", self.cap), 0)

    @property
    def len(self) -> int:
        return int(self.struct.len)

    def share_ring(self, cache: DarCache):
        """Makes this cache's ring that of `cache` (one window for both): what packing
        and reading back leave to the caller."""
        _same_cache(self, cache)
        self.k_win, self.v_win = cache.k_win, cache.v_win
        self.struct.k_win, self.struct.v_win = cache.k_win.data_ptr(), cache.v_win.data_ptr()
        return self


class DarPagedCacheQ4:
    """Paged split cache with 4-bit latents (dar_paged_cache_q4 in include/dar_q4.h):
    rings [B,Hkv,w,d]; pages of codes [n_pages,Hkv,page_size,4 ceil(dd/8)] and scale
    bytes [n_pages,Hkv,page_size,ceil(dd/32)], uint8; block_table [B,max_blocks]
    and lens [B] (int32, device) as in DarPagedCache."""

    def __init__(self, B, Hkv, d, d_down, w, page_size, max_blocks, n_pages, dtype, device="cuda"):
        self.B, self.Hkv, self.d, self.d_down, self.w = B, Hkv, d, d_down, w
        self.page_size, self.max_blocks, self.n_pages = page_size, max_blocks, n_pages
        self.dtype = dtype
        _q4_arrays(self, (n_pages, Hkv, page_size), dtype, device)
        self.block_table = torch.full((B, max_blocks), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(B, dtype=torch.int32, device=device)

    @property
    def cap(self):
        return self.page_size * self.max_blocks

    def overflowed(self):
        """Sequences an append found at capacity (lens marked -1 - n); reads lens back
        to the host (synchronises with the current stream)."""
        return [b for b, n in enumerate(self.lens.cpu().tolist()) if n < 0]

    def share_ring(self, cache: DarPagedCache):
        """Makes the rings and lengths of this cache those of `cache`."""
        _same_cache(self, cache)
        self.k_win, self.v_win, self.lens = cache.k_win, cache.v_win, cache.lens
        return self

    def struct(self) -> DarPagedCacheQ4Struct:
        bt, lens, dev = self.block_table, self.lens, self.k_win.device
        for name, t, want in (("block_table", bt, (self.B, self.max_blocks)), ("lens", lens, (self.B,))):
            if t.dtype is not torch.int32 or t.shape != want or not t.is_contiguous() or t.device != dev:
                raise ValueError("%s: expected contiguous int32 %s on %s" % (name, want, dev))
        return DarPagedCacheQ4Struct(self.k_win.data_ptr(), self.v_win.data_ptr(),
                                     self.k_codes.data_ptr(), self.v_codes.data_ptr(),
                                     self.k_exp.data_ptr(), self.v_exp.data_ptr(),
                                     bt.data_ptr(), lens.data_ptr(),
                                     self.page_size, self.max_blocks, self.n_pages)


def _same_cache(a, b):
    """Two caches of one batch, on one device: what a conversion or a shared ring needs."""
    x, y = a.k_win, b.k_win
    if ((a.B, a.Hkv, a.d, a.d_down, a.w) == (b.B, b.Hkv, b.d, b.d_down, b.w) and x.dtype is y.dtype and
            x.device == y.device):
        return
    for n in ("B", "Hkv", "d", "d_down", "w"):
        if int(getattr(a, n)) != int(getattr(b, n)):
            raise ValueError("%s differs between the caches: %s and %s" % (n, getattr(a, n), getattr(b, n)))
    if x.dtype != y.dtype or x.device != y.device:
        raise ValueError("the caches' dtypes or devices differ")


# One small step takes the host as long as the GPU: checks compare once and say what
# is wrong only if something is (an append and its read-back 12.8 -> 12.2 us).
def _q4_shape(cache):
    return _shape(cache.B, cache.Hkv, cache.Hkv, cache.d, cache.d_down, cache.w, cache.k_win.dtype)


def _check_tokens(cache, k_new, v_new, w_down, want):
    dev, dt = cache.k_win.device, cache.k_win.dtype
    if (k_new.shape == want and v_new.shape == want and w_down.shape == (cache.Hkv, cache.d, cache.d_down) and
            k_new.dtype is dt and v_new.dtype is dt and w_down.dtype is dt and
            k_new.device == dev and v_new.device == dev and w_down.device == dev):
        return
    for name, t, shape in (("k_new", k_new, want), ("v_new", v_new, want),
                           ("w_down", w_down, (cache.Hkv, cache.d, cache.d_down))):
        if tuple(t.shape) != shape or t.dtype != dt or t.device != dev:
            raise ValueError("%s: expected %s %s on %s, got %s %s on %s" % (
                name, shape, dt, dev, tuple(t.shape), t.dtype, t.device))


def dar_cache_append_q4(cache: DarCacheQ4, k_new, v_new, w_down, stream=None):
    """Append n tokens k_new, v_new [B,Hkv,n,d]: window exits are projected to the
    latents that dar_cache_append would store, and quantised to 4 bits."""
    if k_new.dim() != 4:
        raise ValueError("k_new: expected [B,Hkv,n,d]")
    n = k_new.shape[2]
    _check_tokens(cache, k_new, v_new, w_down, (cache.B, cache.Hkv, n, cache.d))
    with _on(cache, stream):
        st = lib.dar_cache_append_q4(ctypes.byref(_q4_shape(cache)), ctypes.byref(cache.struct),
                                     _ptr(k_new), _ptr(v_new), int(n), _ptr(w_down), _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_cache_append_q4")
    return cache


def dar_cache_append_paged_q4(cache: DarPagedCacheQ4, k_new, v_new, w_down, stream=None):
    """One token per sequence: k_new, v_new [B,Hkv,d]; lens advance on the device."""
    _check_tokens(cache, k_new, v_new, w_down, (cache.B, cache.Hkv, cache.d))
    with _on(cache, stream):
        cs = cache.struct()
        st = lib.dar_cache_append_paged_q4(ctypes.byref(_q4_shape(cache)), ctypes.byref(cs),
                                           _ptr(k_new), _ptr(v_new), _ptr(w_down), _stream(stream))
    if st != DAR_OK:
        raise DarError(st, "dar_cache_append_paged_q4")


def _convert(name, src, dst, first, stream):
    """A conversion between dense caches, tokens first.. of src."""
    _same_cache(src, dst)
    if getattr(src, "shared", False) or getattr(dst, "shared", False):
        raise ValueError("a cache with one shared latent per token is not converted")
    with _on(src, stream):
        st = getattr(lib, name)(ctypes.byref(_q4_shape(src)), ctypes.byref(src.struct),
                                _count("first", first), ctypes.byref(dst.struct), _stream(stream))
    if st != DAR_OK:
        raise DarError(st, name)
    return dst


def _convert_paged(name, src, dst, first, stream):
    _same_cache(src, dst)
    if first is not None and (first.dtype != torch.int32 or tuple(first.shape) != (src.B,) or
                              first.device != src.k_win.device):
        raise ValueError("first: expected int32 [%d] on %s" % (src.B, src.k_win.device))
    with _on(src, stream):
        ss, ds = src.struct(), dst.struct()
        st = getattr(lib, name)(ctypes.byref(_q4_shape(src)), ctypes.byref(ss), _ptr(first),
                                ctypes.byref(ds), _stream(stream))
    if st != DAR_OK:
        raise DarError(st, name)
    return dst


def dar_cache_pack_q4(src: DarCache, dst: DarCacheQ4, first=0, stream=None):
    """Quantises the latents of tokens first.. of src into dst, whose length becomes
    src's. The window is not touched (dst.share_ring(src), or copy it)."""
    return _convert("dar_cache_pack_q4", src, dst, first, stream)


def dar_cache_unpack_q4(src: DarCacheQ4, dst: DarCache, first=0, stream=None):
    """The values of the 4-bit latents of tokens first.. of src into dst, whose length
    becomes src's. The window is not touched."""
    return _convert("dar_cache_unpack_q4", src, dst, first, stream)


def dar_cache_pack_paged_q4(src: DarPagedCache, dst: DarPagedCacheQ4, first=None, stream=None):
    """dar_cache_pack_q4 between paged caches, each sequence by its own length, from
    token first[b] (int32 [B]; None: 0; not dst.lens itself, which is written); lengths
    go to dst on the device."""
    return _convert_paged("dar_cache_pack_paged_q4", src, dst, first, stream)


def dar_cache_unpack_paged_q4(src: DarPagedCacheQ4, dst: DarPagedCache, first=None, stream=None):
    """dar_cache_unpack_q4 between paged caches (as dar_cache_pack_paged_q4)."""
    return _convert_paged("dar_cache_unpack_paged_q4", src, dst, first, stream)


def dar_decode_q4_workspace_bytes(shape: DarShape, cap: int) -> int:
    return int(lib.dar_decode_q4_workspace_bytes(ctypes.byref(shape), _count("cap", cap)))


def _decode_q4(name, cache, struct, q, w_down, w_up, o, ws, stream):
    with _on(cache, stream):
        key, o = _check_step(cache, q, w_down, w_up, o)
        if ws is None:
            ws = _workspace(_ws_bytes("dar_decode_q4_workspace_bytes", key, (int(cache.cap),)), q.device)
        st = getattr(lib, name)(ctypes.byref(_shape(*key)), ctypes.byref(struct), _ptr(q), _ptr(w_down),
                                _ptr(w_up), _ptr(o), _ptr(ws),
                                0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    if st != DAR_OK:
        raise DarError(st, name)
    return o


def dar_attn_decode_q4(cache: DarCacheQ4, q, w_down, w_up=None, o=None, ws=None, stream=None):
    """One decode step over 4-bit latents: q [B,Hq,d] at position cache.len - 1.
    Returns o [B,Hq,d]."""
    return _decode_q4("dar_attn_decode_q4", cache, cache.struct, q, w_down, w_up, o, ws, stream)


def dar_attn_decode_paged_q4(cache: DarPagedCacheQ4, q, w_down, w_up=None, o=None, ws=None, stream=None):
    """One decode step per sequence over paged 4-bit latents (query at lens[b] - 1)."""
    return _decode_q4("dar_attn_decode_paged_q4", cache, cache.struct(), q, w_down, w_up, o, ws, stream)
