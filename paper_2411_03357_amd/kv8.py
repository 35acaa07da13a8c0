"""ctypes binding for include/pgcm_kv8.h: KV blocks in 8 bits and attention with a window, same names, argument marshalling only."""
import ctypes as C

import torch

from . import kv as _kv
from .binding import _check, _stream_handle
from .kv import _HALVES, _append_args, _f32, _i64, _ptr, _rows, _same_device, _strides, _u32, _vp, kv_workspace

KV8_EXPORTS = ("pgcm_kv8_append", "pgcm_kv8_store", "pgcm_kv8_load", "pgcm_kv8_attend", "pgcm_kv_window",
               "pgcm_kv_window_reserve")

_CODES = {torch.int8: 0, torch.float8_e4m3fn: 1}


class _Cache8(C.Structure):
    _fields_ = [(n, _vp) for n in ("k", "v", "k_scales", "v_scales")] + \
        [(n, _u32) for n in ("code", "half", "blocks", "block_tokens", "kv_heads", "head_dim")] + \
        [(n, _i64) for n in ("k_block", "k_token", "k_head", "v_block", "v_token", "v_head", "k_scale_block", "k_scale_head",
                             "v_scale_block", "v_scale_head")]


class _Window(C.Structure):
    _fields_ = [(n, _u32) for n in ("requests", "heads", "tokens", "most")] + \
        [("starts", _vp), ("q", _vp), ("q_token", _i64), ("q_head", _i64), ("tables", _vp), ("table_row", _i64),
         ("row_blocks", _u32), ("scale", _f32), ("lens", _vp), ("window", _u32), ("sinks", _u32), ("out", _vp),
         ("out_token", _i64), ("out_head", _i64), ("lse", _vp)]


class _Placed8(C.Structure):
    _fields_ = [("cache", _Cache8), ("device", _i64)]


_bound = None
_marshal = None     # native marshalling (csrc/kv_marshal.cpp), bound to _bound


def _lib():
    global _bound, _marshal
    if _bound is None:
        lib, m = _kv._lib(), _kv._native()
        lib.pgcm_kv8_append.argtypes = [_vp, _vp, _vp]
        lib.pgcm_kv8_store.argtypes = [_vp, _vp, _u32, _vp, _vp, _vp, _vp]
        lib.pgcm_kv8_load.argtypes = [_vp, _vp, _u32, _vp, _vp, _vp, _vp]
        lib.pgcm_kv8_attend.argtypes = [_vp] * 4
        lib.pgcm_kv_window.argtypes = [_vp] * 4
        lib.pgcm_kv_window_reserve.argtypes = [_vp] + [_u32] * 3 + [_vp]
        for name in KV8_EXPORTS:
            getattr(lib, name).restype = C.c_int
        m.bind8(*[C.cast(getattr(lib, n), _vp).value for n in KV8_EXPORTS[:5]])
        _marshal, _bound = m, lib
    return _bound


def _native():
    _lib()
    return _marshal


class KV8Cache:
    """One layer's view of a pool of blocks in 8 bits: k and v are CUDA tensors [blocks, block_tokens, kv_heads, head_dim] of
    int8 or float8_e4m3fn with any strides but for contiguous channels, k_scales and v_scales float32 [blocks, kv_heads] with any
    strides; half is the type of what goes in and comes out.  (One piece for the cipher: uint8 [blocks, bytes], of which codes
    and scales are views.)"""

    def __init__(self, k, v, k_scales, v_scales, half=torch.bfloat16):
        if k.dtype not in _CODES or k.dim() != 4 or half not in _HALVES:
            raise ValueError("a cache in 8 bits is int8 or float8_e4m3fn [blocks, block_tokens, kv_heads, head_dim], of "
                             "float16 or bfloat16 values")
        self.k, self.v, self.k_scales, self.v_scales, self.code, self.dtype = k, v, k_scales, v_scales, k.dtype, half
        self.blocks, self.block_tokens, self.kv_heads, self.head_dim = k.shape
        at = [_ptr(x, what, k.dtype, k.shape, False, anywhere=True) for x, what in ((k, "k"), (v, "v"))]
        scales = (k_scales, "k_scales"), (v_scales, "v_scales")
        for x, what in scales:
            if x.dtype != torch.float32 or tuple(x.shape) != (self.blocks, self.kv_heads) or not x.is_cuda:
                raise ValueError("%s must be a CUDA tensor, float32 %s, not %s %s" %
                                 (what, (self.blocks, self.kv_heads), x.dtype, tuple(x.shape)))
        at += [x.data_ptr() for x, _ in scales]
        self.device = k.get_device()
        if any(x.get_device() != self.device for x in (v, k_scales, v_scales)):
            raise ValueError("codes and scales must be on one device")
        steps = [0 if n == 1 else s for x, _ in scales for n, s in zip(x.shape, x.stride())]
        self._c = _Placed8(_Cache8(*at, _CODES[k.dtype], _HALVES[half], *k.shape, *_strides(k), *_strides(v), *steps), self.device)
        self._at = C.addressof(self._c)


def kv8_append(cache, q, k, v, positions, slots, q_out, q_weight=None, k_weight=None, eps=1e-6, rope=None, adjacent=False,
               stream=None):
    """pgcm_kv8_append: as kv_append, of the cache's `half`, into blocks in 8 bits.  Slots of one block follow each other, each one
    more than the one before."""
    if not k.is_cuda:
        raise ValueError("k must be a CUDA tensor")
    h = _stream_handle(stream)
    status = (_marshal or _native()).kv8_append(None, cache._at, q, k, v, positions, slots, q_out, q_weight, k_weight, eps, rope,
                                                1 if adjacent else 0, h)
    if status is None:
        a = _append_args(cache, q, k, v, positions, slots, q_out, q_weight, k_weight, eps, rope, adjacent)
        status = _lib().pgcm_kv8_append(cache._at, C.addressof(a), h)
    if status:
        _check(status)


def _move(name, cache8, cache, blocks, counts, others, stream):
    if not blocks.is_cuda:
        raise ValueError("blocks must be a CUDA tensor")
    h = _stream_handle(stream)
    status = getattr(_marshal or _native(), name)(None, cache8._at, cache._at, blocks, counts, others, h)
    if status is None:
        _same_device(cache8.device, "the cache in 8 bits", _kv._device())
        _same_device(cache.device, "the cache", _kv._device())
        n = blocks.shape[0]
        status = getattr(_lib(), "pgcm_" + name)(
            cache8._at, cache._at, n, _ptr(blocks, "blocks", torch.int32, (n,)),
            None if counts is None else _ptr(counts, "counts", torch.int32, (n,)),
            None if others is None else _ptr(others, "the other cache's blocks", torch.int32, (n,)), h)
    if status:
        _check(status)


def kv8_store(cache8, cache, blocks, counts=None, from_blocks=None, stream=None):
    """pgcm_kv8_store: from cache (KVCache) to cache8 (KV8Cache); blocks, counts, from_blocks int32 [n]"""
    _move("kv8_store", cache8, cache, blocks, counts, from_blocks, stream)


def kv8_load(cache8, cache, blocks, counts=None, to_blocks=None, stream=None):
    """pgcm_kv8_load: from cache8 to cache; blocks (of cache8), counts, to_blocks int32 [n]"""
    _move("kv8_load", cache8, cache, blocks, counts, to_blocks, stream)


def _attend(name, cache, q, tables, lens, out, lse, scale, window, sinks, starts, most, workspace, stream):
    if not q.is_cuda:
        raise ValueError("q must be a CUDA tensor")
    h = _stream_handle(stream)
    if scale is None:
        scale = cache.head_dim ** -0.5
    if most is None:
        most = 1 if starts is None else q.shape[0]
    space = (workspace or kv_workspace(h))._h
    status = getattr(_marshal or _native(), name)(None, space, cache._at, q, tables, lens, out, lse, scale, window, sinks, starts,
                                                  most, h)
    if status is None:
        _same_device(cache.device, "the cache", _kv._device())
        n, row, tables_at, lens_at = _rows(tables, lens)
        d, half = cache.head_dim, cache.dtype
        rows, heads = (n if starts is None else q.shape[0]), q.shape[1]
        if not all(0 <= x < 1 << 32 for x in (window, sinks, most)):
            raise ValueError("window, sinks and most are numbers of 32 bits")
        a = _Window(n, heads, rows, most)
        if starts is not None:
            a.starts = _ptr(starts, "starts", torch.int32, (n + 1,))
        a.q = _ptr(q, "q", half, (rows, heads, d), False)
        a.q_token, a.q_head = _strides(q)
        a.tables, a.row_blocks, a.lens = tables_at, row, lens_at
        a.table_row, = _strides(tables)
        a.scale, a.window, a.sinks = scale, window, sinks
        a.out = _ptr(out, "out", half, (rows, heads, d), False)
        a.out_token, a.out_head = _strides(out)
        if lse is not None:
            a.lse = _ptr(lse, "lse", torch.float32, (rows, heads))
        status = getattr(_lib(), "pgcm_" + name)(space, cache._at, C.addressof(a), h)
    if status:
        _check(status)


def kv8_attend(cache, q, tables, lens, out, lse=None, scale=None, window=0, sinks=0, starts=None, most=None, workspace=None,
               stream=None):
    """pgcm_kv8_attend: q, out [tokens, heads, head_dim] of the cache's half; tables int32 [requests, row_blocks]; lens int32
    [requests], new tokens included; lse float32 [tokens, heads]; starts int32 [requests + 1]: a request's new tokens are rows
    starts[b] up to starts[b + 1], at most `most` of them; None: a row for each.  scale: 1 / sqrt(head_dim) if None; window 0: all."""
    _attend("kv8_attend", cache, q, tables, lens, out, lse, scale, window, sinks, starts, most, workspace, stream)


def kv_window(cache, q, tables, lens, out, lse=None, scale=None, window=0, sinks=0, starts=None, most=None, workspace=None,
              stream=None):
    """pgcm_kv_window: the same over blocks of halves (KVCache)"""
    _attend("kv_window", cache, q, tables, lens, out, lse, scale, window, sinks, starts, most, workspace, stream)


def kv_window_reserve(workspace, heads, kv_heads, head_dim, stream=None):
    """pgcm_kv_window_reserve: sizes a KVWorkspace ahead of time, as a captured graph needs"""
    _check(_lib().pgcm_kv_window_reserve(workspace._h, heads, kv_heads, head_dim, _stream_handle(stream)))
