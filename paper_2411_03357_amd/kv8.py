"""ctypes binding for include/pgcm_kv8.h: KV blocks in 8 bits, same names, argument marshalling only."""
import ctypes as C

import torch

from . import kv as _kv
from .binding import _check, _stream_handle
from .kv import _HALVES, _append_args, _device, _i64, _ptr, _same_device, _strides, _u32, _vp

KV8_EXPORTS = ("pgcm_kv8_append", "pgcm_kv8_store", "pgcm_kv8_load")

_CODES = {torch.int8: 0, torch.float8_e4m3fn: 1}


class _Cache8(C.Structure):
    _fields_ = [(n, _vp) for n in ("k", "v", "k_scales", "v_scales")] + \
        [(n, _u32) for n in ("code", "half", "blocks", "block_tokens", "kv_heads", "head_dim")] + \
        [(n, _i64) for n in ("k_block", "k_token", "k_head", "v_block", "v_token", "v_head", "k_scale_block", "k_scale_head",
                             "v_scale_block", "v_scale_head")]


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
        for name in KV8_EXPORTS:
            getattr(lib, name).restype = C.c_int
        m.bind8(*[C.cast(getattr(lib, "pgcm_kv8_" + n), _vp).value for n in ("append", "store", "load")])
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
        _same_device(cache8.device, "the cache in 8 bits", _device())
        _same_device(cache.device, "the cache", _device())
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
