"""Binding of the block operators of ``libiptq.so``: attention over packed prompts, the 4-bit cache and
the attention over it, the root-mean-square norm and the requantization by row scales.

As in ``binding.py`` every function has the name of its C entry point (``include/iptq.h``) and only
marshals: counts, strides and heads that a tensor's shape says are taken from it, ``data_ptr()`` and the
current stream cross the boundary.  Tensors lie on the current device.  There is no CPU fallback.
"""

from __future__ import annotations

import ctypes

from . import binding
from .binding import Dyadic, _check, _dptr, _stream, load

GROUP = 64                        # channels that share one step of the cache


class AttentionParams(ctypes.Structure):
    _fields_ = [("variant", ctypes.c_int32), ("i0", ctypes.c_int32), ("n_shift", ctypes.c_int32),
                ("score_shift", ctypes.c_int32), ("causal", ctypes.c_int32), ("post", Dyadic)]


class RmsnormParams(ctypes.Structure):
    _fields_ = [("in_m", ctypes.c_int32), ("in_s", ctypes.c_int32), ("eps", ctypes.c_int64), ("post", Dyadic)]


class CacheI4(ctypes.Structure):
    """The cache's descriptor.  Made by cache_i4(), which keeps the four tensors alive beside it."""
    _fields_ = [("d_k_codes", ctypes.c_void_p), ("d_k_steps", ctypes.c_void_p), ("d_v_codes", ctypes.c_void_p),
                ("d_v_steps", ctypes.c_void_p), ("n_pages", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


_bound = None


def _lib():
    global _bound
    lib = load()
    if _bound is not lib:
        vp, i64, i32, p = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.POINTER
        lib.iptq_attention_i8.argtypes = [vp, i64, vp, i64, vp, i64, vp, vp, i32, i32, i64, i64, i32, i32, i32, vp, i64,
                                          p(AttentionParams), vp]
        lib.iptq_cache_store_i4.argtypes = [p(CacheI4), vp, i64, vp, i64, vp, i64, vp]
        lib.iptq_attention_cache_i4_workspace.argtypes = [p(CacheI4), i32, i32, i32, i32, p(i64)]
        lib.iptq_attention_cache_i4.argtypes = [vp, i64, p(CacheI4), vp, i32, vp, i32, i32, i32, vp, i64, vp, i64,
                                                p(AttentionParams), vp]
        lib.iptq_rmsnorm_i32.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, p(RmsnormParams), vp]
        lib.iptq_requant_rows.argtypes = [vp, vp, i32, vp, i64, i32, i32, p(Dyadic), vp]
        f64 = ctypes.c_double
        lib.iptq_attention_prepare.argtypes = [f64, f64, f64, i32, i32, i32, i32, p(AttentionParams)]
        for name in ("attention_i8", "cache_store_i4", "attention_cache_i4_workspace", "attention_cache_i4", "rmsnorm_i32",
                     "requant_rows", "attention_prepare"):
            getattr(lib, "iptq_" + name).restype = ctypes.c_int
        _bound = lib
    return lib


_native_of = None                 # the library that the native calls are bound to


def _native():
    """The native call module bound to these entry points, once the first call of the process has been made; or None."""
    global _native_of
    call = binding._fast
    if call is not None and _native_of is not binding._lib:
        lib = _lib()
        call.bind_block(*[ctypes.cast(getattr(lib, "iptq_" + n), ctypes.c_void_p).value for n in
                          ("attention_i8", "cache_store_i4", "attention_cache_i4", "rmsnorm_i32", "requant_rows")],
                        AttentionParams, RmsnormParams, CacheI4, Dyadic)
        _native_of = binding._lib
    return call


def _need(t, dtype, what, least=0):
    torch = binding.torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError("%s must be a contiguous %s tensor on the GPU" % (what, dtype))
    if t.get_device() != torch.cuda.current_device():
        raise ValueError("%s is not on the current device" % what)
    if t.numel() < least:
        raise ValueError("%s has %d elements, %d are needed" % (what, t.numel(), least))


def _rows(t, what):
    """(tokens, heads, head dimension, bytes between two tokens) of an int8 tensor of token rows."""
    torch = binding.torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != torch.int8 or t.dim() != 3:
        raise TypeError("%s must be an int8 tensor [tokens, heads, head dimension] on the GPU" % what)
    if t.get_device() != torch.cuda.current_device():
        raise ValueError("%s is not on the current device" % what)
    tokens, heads, dim = t.shape
    if tokens == 0:                                       # (an empty tensor's strides mean nothing)
        return tokens, heads, dim, heads * dim
    if (dim > 1 and t.stride(2) != 1) or (heads > 1 and t.stride(1) != dim) or (tokens > 1 and t.stride(0) < heads * dim):
        raise ValueError("the heads of a token of %s must lie side by side, and tokens must not overlap" % what)
    return tokens, heads, dim, t.stride(0) if tokens > 1 else heads * dim


def attention_prepare(s_score: float, s_v: float, s_out: float, zp_out: int, variant: int, causal: int,
                      of_cache: int = 0) -> AttentionParams:
    p = AttentionParams()
    _check(_lib().iptq_attention_prepare(s_score, s_v, s_out, zp_out, variant, causal, of_cache, ctypes.byref(p)),
           "iptq_attention_prepare")
    return p


def attention_i8(d_q, d_k, d_v, d_q_offsets, d_k_offsets, n_seq: int, max_q: int, d_out, p: AttentionParams):
    """d_q, d_out: int8 [q tokens, heads, head dimension]; d_k, d_v: [k tokens, kv heads, head dimension]; rows
    may lie apart.  Offsets: int32 [n_seq + 1] both, or None both (equal lengths)."""
    call = _native()
    if call is not None:
        rc = call.attention_i8(d_q, d_k, d_v, d_q_offsets, d_k_offsets, n_seq, max_q, d_out, p)
        if rc is not None:
            return _check(rc, "iptq_attention_i8")
    lib = _lib()
    qt, heads, dim, qs = _rows(d_q, "d_q")
    kt, kv_heads, kd, ks = _rows(d_k, "d_k")
    vt, vh, vd, vs = _rows(d_v, "d_v")
    ot, oh, od, os_ = _rows(d_out, "d_out")
    if (kt, kv_heads) != (vt, vh) or not dim == kd == vd or (qt, heads, dim) != (ot, oh, od):
        raise ValueError("the shapes of d_q, d_k, d_v and d_out do not belong together")
    for t, what in ((d_q_offsets, "d_q_offsets"), (d_k_offsets, "d_k_offsets")):
        if t is not None:
            _need(t, binding.torch.int32, what, n_seq + 1)
    _check(lib.iptq_attention_i8(_dptr(d_q), qs, _dptr(d_k), ks, _dptr(d_v), vs, _dptr(d_q_offsets), _dptr(d_k_offsets), n_seq,
                                 max_q, qt, kt, heads, kv_heads, dim, _dptr(d_out), os_, ctypes.byref(p), _stream()),
           "iptq_attention_i8")


def cache_i4(d_k_codes, d_k_steps, d_v_codes, d_v_steps, head_dim: int) -> CacheI4:
    """The descriptor of a cache whose four uint8 tensors have the shapes [pages, kv heads, page tokens, head_dim / 2],
    [pages, kv heads, page tokens, groups], [pages, kv heads, head_dim / 2, page tokens] and, again,
    [pages, kv heads, page tokens, groups]; groups = ceil(head_dim / 64)."""
    _lib()
    for t, what in ((d_k_codes, "d_k_codes"), (d_k_steps, "d_k_steps"), (d_v_codes, "d_v_codes"), (d_v_steps, "d_v_steps")):
        _need(t, binding.torch.uint8, what)
    if d_k_codes.dim() != 4 or head_dim < 2:
        raise ValueError("the codes must be 4-dimensional")
    pages, heads, tokens, half = d_k_codes.shape
    steps = (pages, heads, tokens, -(-head_dim // GROUP))
    if 2 * half != head_dim or tuple(d_v_codes.shape) != (pages, heads, half, tokens) or tuple(d_k_steps.shape) != steps or \
            tuple(d_v_steps.shape) != steps:
        raise ValueError("the shapes of the cache's tensors do not belong together")
    c = CacheI4(_dptr(d_k_codes), _dptr(d_k_steps), _dptr(d_v_codes), _dptr(d_v_steps), pages, tokens, heads, head_dim)
    c.tensors = (d_k_codes, d_k_steps, d_v_codes, d_v_steps)
    return c


def cache_store_i4(cache: CacheI4, d_k, d_v, d_slots, tokens: int):
    """d_k, d_v: int8 [tokens, kv heads, head dimension], rows may lie apart; d_slots: int32 [tokens]."""
    call = _native()
    if call is not None:
        rc = call.cache_store_i4(cache, d_k, d_v, d_slots, tokens)
        if rc is not None:
            return _check(rc, "iptq_cache_store_i4")
    lib = _lib()
    kt, kh, kd, ks = _rows(d_k, "d_k")
    vt, vh, vd, vs = _rows(d_v, "d_v")
    if kt < tokens or vt < tokens or not kh == vh == cache.kv_heads or not kd == vd == cache.head_dim:
        raise ValueError("the shapes of d_k and d_v are not the cache's")
    _need(d_slots, binding.torch.int32, "d_slots", tokens)
    _check(lib.iptq_cache_store_i4(ctypes.byref(cache), _dptr(d_k), ks, _dptr(d_v), vs, _dptr(d_slots), tokens, _stream()),
           "iptq_cache_store_i4")


def attention_cache_i4_workspace(cache: CacheI4, n_seq: int, q_tokens: int, heads: int, max_pages: int) -> int:
    size = ctypes.c_int64()
    _check(_lib().iptq_attention_cache_i4_workspace(ctypes.byref(cache), n_seq, q_tokens, heads, max_pages, ctypes.byref(size)),
           "iptq_attention_cache_i4_workspace")
    return size.value


def attention_cache_i4(d_q, cache: CacheI4, d_pages, d_lengths, n_seq: int, q_tokens: int, d_out, d_work, p: AttentionParams):
    """d_q, d_out: int8 [n_seq * q_tokens, heads, head dimension]; d_pages: int32 [n_seq, max_pages]; d_lengths: int32
    [n_seq]; d_work: uint8 of attention_cache_i4_workspace() bytes, or None."""
    call = _native()
    if call is not None:
        rc = call.attention_cache_i4(d_q, cache, d_pages, d_lengths, n_seq, q_tokens, d_out, d_work, p)
        if rc is not None:
            return _check(rc, "iptq_attention_cache_i4")
    lib = _lib()
    qt, heads, dim, qs = _rows(d_q, "d_q")
    ot, oh, od, os_ = _rows(d_out, "d_out")
    if (qt, heads, dim) != (ot, oh, od) or dim != cache.head_dim or qt < n_seq * q_tokens:
        raise ValueError("the shapes of d_q, d_out and the cache do not belong together")
    _need(d_pages, binding.torch.int32, "d_pages")
    if d_pages.dim() != 2 or d_pages.shape[0] < n_seq:
        raise ValueError("d_pages must be [n_seq, max_pages]")
    _need(d_lengths, binding.torch.int32, "d_lengths", n_seq)
    size = 0
    if d_work is not None:
        _need(d_work, binding.torch.uint8, "d_work")
        size = d_work.numel()
    _check(lib.iptq_attention_cache_i4(_dptr(d_q), qs, ctypes.byref(cache), _dptr(d_pages), d_pages.shape[1], _dptr(d_lengths), n_seq,
                                       q_tokens, heads, _dptr(d_out), os_, _dptr(d_work), size, ctypes.byref(p), _stream()),
           "iptq_attention_cache_i4")


def rmsnorm_i32(d_x, d_residual, d_gain, d_residual_out, d_out, d_row_scales, rows: int, cols: int, p: RmsnormParams):
    """d_x, d_residual, d_residual_out: int32 [rows, cols] or None (d_residual_out may be d_residual); d_gain: int16 [cols];
    d_out: int8 [rows, cols]; d_row_scales: int32 [rows] or None (codes of one scale, by p.post)."""
    call = _native()
    if call is not None:
        rc = call.rmsnorm_i32(d_x, d_residual, d_gain, d_residual_out, d_out, d_row_scales, rows, cols, p)
        if rc is not None:
            return _check(rc, "iptq_rmsnorm_i32")
    lib = _lib()
    torch = binding.torch
    n = rows * cols
    for t, what in ((d_x, "d_x"), (d_residual, "d_residual"), (d_residual_out, "d_residual_out")):
        if t is not None:
            _need(t, torch.int32, what, n)
    _need(d_gain, torch.int16, "d_gain", cols)
    _need(d_out, torch.int8, "d_out", n)
    if d_row_scales is not None:
        _need(d_row_scales, torch.int32, "d_row_scales", rows)
    _check(lib.iptq_rmsnorm_i32(_dptr(d_x), _dptr(d_residual), _dptr(d_gain), _dptr(d_residual_out), _dptr(d_out), _dptr(d_row_scales),
                                rows, cols, ctypes.byref(p), _stream()), "iptq_rmsnorm_i32")


def requant_rows(d_in, d_row_scales, d_out, rows: int, cols: int, row_shift: int, out_is_signed: int, p: Dyadic):
    call = _native()
    if call is not None:
        rc = call.requant_rows(d_in, d_row_scales, d_out, rows, cols, row_shift, out_is_signed, p)
        if rc is not None:
            return _check(rc, "iptq_requant_rows")
    lib = _lib()
    torch = binding.torch
    _need(d_in, torch.int32, "d_in", rows * cols)
    _need(d_row_scales, torch.int32, "d_row_scales", rows)
    _need(d_out, torch.int8 if out_is_signed else torch.uint8, "d_out", rows * cols)
    _check(lib.iptq_requant_rows(_dptr(d_in), _dptr(d_row_scales), row_shift, _dptr(d_out), rows, cols, out_is_signed, ctypes.byref(p),
                                 _stream()), "iptq_requant_rows")
