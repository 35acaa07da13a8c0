"""ctypes binding for include/pgcm_kv.h: the operators on KV blocks, same names, argument marshalling only."""
import ctypes as C
import threading

import torch

from .binding import _check, _stream_handle, load_library

KV_EXPORTS = ("pgcm_kv_create", "pgcm_kv_destroy", "pgcm_kv_reserve", "pgcm_kv_append", "pgcm_kv_attend",
              "pgcm_kv_summarize", "pgcm_kv_select", "pgcm_kv_evict")

_HALVES = {torch.float16: 0, torch.bfloat16: 1}
_u32, _i64, _vp, _f32 = C.c_uint32, C.c_int64, C.c_void_p, C.c_float


class _Cache(C.Structure):
    _fields_ = [("k", _vp), ("v", _vp)] + \
        [(n, _u32) for n in ("half", "blocks", "block_tokens", "kv_heads", "head_dim", "reserved")] + \
        [(n, _i64) for n in ("k_block", "k_token", "k_head", "v_block", "v_token", "v_head")]


class _Placed(C.Structure):
    _fields_ = [("cache", _Cache), ("device", _i64)]


class _Append(C.Structure):
    _fields_ = [("tokens", _u32), ("heads", _u32), ("q", _vp), ("k", _vp), ("v", _vp)] + \
        [(n, _i64) for n in ("q_token", "q_head", "k_token", "k_head", "v_token", "v_head")] + \
        [(n, _vp) for n in ("positions", "slots", "q_weight", "k_weight")] + \
        [("eps", _f32), ("adjacent", _u32), ("rope", _vp), ("rope_positions", _u32), ("rope_dim", _u32), ("q_out", _vp),
         ("q_out_token", _i64), ("q_out_head", _i64)]


class _Attend(C.Structure):
    _fields_ = [("requests", _u32), ("heads", _u32), ("q", _vp), ("q_request", _i64), ("q_head", _i64), ("tables", _vp),
                ("table_row", _i64), ("row_blocks", _u32), ("scale", _f32), ("lens", _vp), ("selected", _vp),
                ("keep", _u32), ("decay", _f32), ("out", _vp), ("out_request", _i64), ("out_head", _i64), ("lse", _vp),
                ("kept", _vp), ("weights", _vp)]


class _Select(C.Structure):
    _fields_ = [(n, _u32) for n in ("requests", "heads", "kv_heads", "head_dim", "half", "block_tokens")] + \
        [("q", _vp), ("q_request", _i64), ("q_head", _i64), ("tables", _vp), ("table_row", _i64), ("row_blocks", _u32),
         ("entry_count", _u32), ("lens", _vp), ("bounds", _vp), ("scales", _vp), ("keep", _u32), ("first", _u32),
         ("last", _u32), ("selected", _vp), ("counts", _vp)]


class _Evict(C.Structure):
    _fields_ = [("requests", _u32), ("row_blocks", _u32), ("block_tokens", _u32), ("blocks", _u32), ("weights", _vp),
                ("tables", _vp), ("table_row", _i64), ("lens", _vp), ("evict", _vp), ("most", _u32), ("first", _u32),
                ("last", _u32), ("victims", _vp), ("victim_blocks", _vp), ("tables_out", _vp), ("table_out_row", _i64)]


_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_bound = None
_marshal = None     # native marshalling (csrc/kv_marshal.cpp), bound to _bound


def _load_marshal():
    """the extension that reads tensors; one of another torch would read them wrongly"""
    try:
        from . import _kv_marshal as m
    except ImportError as e:
        raise ImportError("_kv_marshal.so is not built, or not for this torch: python -m paper_2411_03357_amd.build") from e
    if m.built_for != "built for torch " + torch.__version__:
        raise ImportError("_kv_marshal.so was %s, and this is torch %s: python -m paper_2411_03357_amd.build" %
                           (m.built_for, torch.__version__))
    return m


def _lib():
    global _bound
    if _bound is None:
        lib = load_library()
        lib.pgcm_kv_create.argtypes = [C.POINTER(_vp)]
        lib.pgcm_kv_destroy.argtypes = [_vp]
        lib.pgcm_kv_destroy.restype = None
        lib.pgcm_kv_reserve.argtypes = [_vp] + [_u32] * 6 + [_vp]
        lib.pgcm_kv_append.argtypes = [_vp, _vp, _vp]
        lib.pgcm_kv_attend.argtypes = [_vp] * 4
        lib.pgcm_kv_summarize.argtypes = [_vp, _u32, _vp, _vp, _vp, _u32, _vp, _vp, _vp]
        lib.pgcm_kv_select.argtypes = [_vp] * 3
        lib.pgcm_kv_evict.argtypes = [_vp] * 2
        for name in KV_EXPORTS:
            if name != "pgcm_kv_destroy":
                getattr(lib, name).restype = C.c_int
        m = _load_marshal()
        m.bind(*[C.cast(getattr(lib, "pgcm_kv_" + n), _vp).value
                 for n in ("append", "attend", "summarize", "select", "evict")])
        global _marshal
        _marshal = m
        _bound = lib
    return _bound


def _native():
    """the calls' native marshalling; like the batch calls', it leaves anything unusual, by returning None, to the code
    here, which says what is wrong"""
    _lib()
    return _marshal


def _same_device(device, what, current):
    if device != current:
        raise ValueError("%s is on cuda:%d, and the current device is cuda:%d" % (what, device, current))


def _ptr(t, what, dtype, shape, contiguous=True, anywhere=False):
    """device address of a CUDA tensor of this type and shape, on the current device; its channels, or all of it, contiguous"""
    if t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be %s %s, not %s %s" % (what, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % what)
    if not anywhere:
        _same_device(t.get_device(), what, _device())
    if contiguous:
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % what)
    elif t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("the last dimension of %s must be contiguous" % what)
    return t.data_ptr()


def _given(at):
    """for what an address says to be there: a tensor without elements has none, and nothing of it is read"""
    return at or 4096


def _strides(t):
    """strides of all dimensions but the last; a dimension of one has none that counts"""
    return [0 if n == 1 else s for n, s in zip(t.shape[:-1], t.stride())]


class KVCache:
    """One layer's view of a pool of blocks: k and v are CUDA tensors [blocks, block_tokens, kv_heads, head_dim] of one
    16-bit type, with any strides but for contiguous channels (for blocks as the cipher takes them, pool[:, 0] and
    pool[:, 1] of [blocks, 2, block_tokens, kv_heads, head_dim])."""

    def __init__(self, k, v):
        if k.dtype not in _HALVES or k.dim() != 4:
            raise ValueError("a cache is float16 or bfloat16 [blocks, block_tokens, kv_heads, head_dim]")
        self.k, self.v, self.dtype = k, v, k.dtype
        self.blocks, self.block_tokens, self.kv_heads, self.head_dim = k.shape
        at = [_ptr(x, what, k.dtype, k.shape, False, anywhere=True) for x, what in ((k, "k"), (v, "v"))]
        self.device = k.get_device()
        if v.get_device() != self.device:
            raise ValueError("k and v must be on one device")
        self._c = _Placed(_Cache(*at, _HALVES[k.dtype], *k.shape, 0, *_strides(k), *_strides(v)), self.device)
        self._at = C.addressof(self._c)


class KVWorkspace:
    """Owns a pgcm_kv_t: what kv_attend and kv_select need besides their tensors, for calls that follow each other on one
    stream.  reserve() sizes it ahead of time, as a captured graph needs."""

    def __init__(self):
        self._h = None
        h = _vp()
        _check(_lib().pgcm_kv_create(C.byref(h)))
        self._h = h.value

    def reserve(self, requests, heads, kv_heads, head_dim, block_tokens, row_blocks, stream=None):
        _check(_lib().pgcm_kv_reserve(self._h, requests, heads, kv_heads, head_dim, block_tokens, row_blocks,
                                      _stream_handle(stream)))

    def destroy(self):
        if self._h is not None:
            _lib().pgcm_kv_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


_workspaces = {}    # (device, stream handle) -> KVWorkspace, of calls that name none
_workspaces_lock = threading.Lock()
_PER_THREAD = 2     # the handle hipStreamPerThread: another stream in each thread
_of_thread = threading.local()


def kv_workspace(stream=None) -> KVWorkspace:
    """the workspace that calls on this stream use unless they are given one.  It stays for the process, or, on
    hipStreamPerThread, for the thread: a graph captured with it is replayed no longer than that.  Who destroys a stream
    waits for its calls first, as a later stream may come by the same handle and with it by the same workspace."""
    key = (_device(), _stream_handle(stream))
    if key[1] == _PER_THREAD:
        got = _of_thread.__dict__.get(key)
        if got is None:
            got = _of_thread.__dict__[key] = KVWorkspace()
        return got
    got = _workspaces.get(key)
    if got is None:
        with _workspaces_lock:
            got = _workspaces.get(key)
            if got is None:
                got = _workspaces[key] = KVWorkspace()
    return got


def _rows(tables, lens, what="tables"):
    if tables.dim() != 2:
        raise ValueError("%s must be [requests, row_blocks]" % what)
    return tables.shape[0], tables.shape[1], _ptr(tables, what, torch.int32, tables.shape, False), \
        _ptr(lens, "lens", torch.int32, tables.shape[:1])


def kv_append(cache, q, k, v, positions, slots, q_out, q_weight=None, k_weight=None, eps=1e-6, rope=None, adjacent=False,
              stream=None):
    """pgcm_kv_append: q, q_out [tokens, heads, head_dim] (or None: keys and values alone), k, v [tokens, kv_heads,
    head_dim], of the cache's type with contiguous channels; positions int32, slots int64 [tokens]; weights [head_dim]; rope
    float32 [positions, rope_dim], cosines then sines.  positions may be None if rope is."""
    if not k.is_cuda:
        raise ValueError("k must be a CUDA tensor")
    h = _stream_handle(stream)
    status = (_marshal or _native()).kv_append(None, cache._at, q, k, v, positions, slots, q_out, q_weight,
                                               k_weight, eps, rope, 1 if adjacent else 0, h)
    if status is not None:
        if status:
            _check(status)
        return
    _same_device(cache.device, "the cache", _device())
    n, kv, d, half = k.shape[0], cache.kv_heads, cache.head_dim, cache.dtype
    heads = 0 if q is None else q.shape[1]
    a = _Append(n, heads)
    a.k, a.v = _ptr(k, "k", half, (n, kv, d), False), _ptr(v, "v", half, (n, kv, d), False)
    a.k_token, a.k_head = _strides(k)
    a.v_token, a.v_head = _strides(v)
    if q is not None:
        a.q, a.q_out = _ptr(q, "q", half, (n, heads, d), False), _ptr(q_out, "q_out", half, (n, heads, d), False)
        a.q_token, a.q_head = _strides(q)
        a.q_out_token, a.q_out_head = _strides(q_out)
    a.slots = _ptr(slots, "slots", torch.int64, (n,))
    if q_weight is not None:
        a.q_weight = _ptr(q_weight, "q_weight", half, (d,))
    if k_weight is not None:
        a.k_weight = _ptr(k_weight, "k_weight", half, (d,))
    a.eps = eps
    if rope is not None:
        a.positions = _ptr(positions, "positions", torch.int32, (n,))
        a.rope = _given(_ptr(rope, "rope", torch.float32, rope.shape))
        a.rope_positions, a.rope_dim = rope.shape
        a.adjacent = 1 if adjacent else 0
    _check(_lib().pgcm_kv_append(cache._at, C.addressof(a), h))


def kv_attend(cache, q, tables, lens, out, lse=None, scale=None, selected=None, weights=None, kept=None, decay=1.0,
              workspace=None, stream=None):
    """pgcm_kv_attend: q, out [requests, heads, head_dim] of the cache's type; tables int32 [requests, row_blocks]; lens
    int32 [requests]; lse float32 [requests, heads]; selected int32 [requests, kv_heads, keep]; weights, kept float32
    [requests, row_blocks].  scale: 1 / sqrt(head_dim) if None."""
    if not q.is_cuda:
        raise ValueError("q must be a CUDA tensor")
    h = _stream_handle(stream)
    if scale is None:
        scale = cache.head_dim ** -0.5
    space = (workspace or kv_workspace(h))._h
    status = (_marshal or _native()).kv_attend(None, space, cache._at, q, tables, lens, out, lse, scale, selected,
                                               weights, kept, decay, h)
    if status is not None:
        if status:
            _check(status)
        return
    _same_device(cache.device, "the cache", _device())
    n, row, tables_at, lens_at = _rows(tables, lens)
    d, half = cache.head_dim, cache.dtype
    heads = q.shape[1]
    a = _Attend(n, heads, _ptr(q, "q", half, (n, heads, d), False), *_strides(q), tables_at, *_strides(tables), row,
                scale, lens_at)
    a.out = _ptr(out, "out", half, (n, heads, d), False)
    a.out_request, a.out_head = _strides(out)
    if lse is not None:
        a.lse = _ptr(lse, "lse", torch.float32, (n, heads))
    if selected is not None:
        a.keep = selected.shape[-1]
        a.selected = _given(_ptr(selected, "selected", torch.int32, (n, cache.kv_heads, a.keep)))
    if weights is not None:
        a.weights, a.decay = _given(_ptr(weights, "weights", torch.float32, (n, row))), decay
    if kept is not None:
        a.kept = _given(_ptr(kept, "kept", torch.float32, (n, row)))
    _check(_lib().pgcm_kv_attend(space, cache._at, C.addressof(a), h))


def kv_summarize(cache, blocks, counts, bounds, scales, entries=None, stream=None):
    """pgcm_kv_summarize: blocks, counts, entries int32 [n]; bounds int8 [entries, kv_heads, 2, head_dim]; scales float32
    [entries, kv_heads]"""
    if not blocks.is_cuda:
        raise ValueError("blocks must be a CUDA tensor")
    h = _stream_handle(stream)
    status = (_marshal or _native()).kv_summarize(None, cache._at, blocks, counts, bounds, scales, entries, h)
    if status is not None:
        if status:
            _check(status)
        return
    _same_device(cache.device, "the cache", _device())
    n, m = blocks.shape[0], bounds.shape[0]
    _check(_lib().pgcm_kv_summarize(
        cache._at, n, _ptr(blocks, "blocks", torch.int32, (n,)), _ptr(counts, "counts", torch.int32, (n,)),
        None if entries is None else _ptr(entries, "entries", torch.int32, (n,)), m,
        _ptr(bounds, "bounds", torch.int8, (m, cache.kv_heads, 2, cache.head_dim)),
        _ptr(scales, "scales", torch.float32, (m, cache.kv_heads)), h))


def kv_select(q, tables, lens, bounds, scales, block_tokens, selected, counts=None, first=0, last=1, workspace=None,
              stream=None):
    """pgcm_kv_select: q [requests, heads, head_dim] float16 or bfloat16; tables int32 [requests, row_blocks] of entries of
    bounds; selected int32 [requests, kv_heads, keep]; counts int32 [requests, kv_heads]"""
    if not q.is_cuda:
        raise ValueError("q must be a CUDA tensor")
    h = _stream_handle(stream)
    space = (workspace or kv_workspace(h))._h
    status = (_marshal or _native()).kv_select(None, space, _HALVES.get(q.dtype, 0), q, tables, lens, bounds, scales,
                                               block_tokens, selected, counts, first, last, h)
    if status is not None:
        if status:
            _check(status)
        return
    n, row, tables_at, lens_at = _rows(tables, lens)
    if q.dtype not in _HALVES or bounds.dim() != 4:
        raise ValueError("q must be float16 or bfloat16, bounds [entries, kv_heads, 2, head_dim]")
    m, kv, _, d = bounds.shape
    heads, keep = q.shape[1], selected.shape[-1]
    a = _Select(n, heads, kv, d, _HALVES[q.dtype], block_tokens, _ptr(q, "q", q.dtype, (n, heads, d), False), *_strides(q),
                tables_at, *_strides(tables), row, m, lens_at,
                _ptr(bounds, "bounds", torch.int8, (m, kv, 2, d)), _ptr(scales, "scales", torch.float32, (m, kv)), keep, first,
                last, _ptr(selected, "selected", torch.int32, (n, kv, keep)),
                None if counts is None else _ptr(counts, "counts", torch.int32, (n, kv)))
    _check(_lib().pgcm_kv_select(space, C.addressof(a), h))


def kv_evict(weights, tables, lens, block_tokens, evict, victims, victim_blocks=None, tables_out=None, first=0, last=1,
             blocks=0x7FFFFFFF, stream=None):
    """pgcm_kv_evict: weights float32, tables and tables_out int32 [requests, row_blocks]; evict int32 [requests]; victims,
    victim_blocks int32 [requests, most].  blocks: of the pool; table entries outside [0, blocks) are not on the device."""
    if not weights.is_cuda:
        raise ValueError("weights must be a CUDA tensor")
    h = _stream_handle(stream)
    status = (_marshal or _native()).kv_evict(None, weights, tables, lens, block_tokens, evict, victims, victim_blocks,
                                              tables_out, first, last, blocks, h)
    if status is not None:
        if status:
            _check(status)
        return
    n, row, tables_at, lens_at = _rows(tables, lens)
    most = victims.shape[-1]
    a = _Evict(n, row, block_tokens, blocks, _ptr(weights, "weights", torch.float32, (n, row)), tables_at, *_strides(tables),
               lens_at, _ptr(evict, "evict", torch.int32, (n,)), most, first, last,
               _ptr(victims, "victims", torch.int32, (n, most)))
    if victim_blocks is not None:
        a.victim_blocks = _ptr(victim_blocks, "victim_blocks", torch.int32, (n, most))
    if tables_out is not None:
        a.tables_out = _ptr(tables_out, "tables_out", torch.int32, (n, row), False)
        a.table_out_row, = _strides(tables_out)
    _check(_lib().pgcm_kv_evict(C.addressof(a), h))
