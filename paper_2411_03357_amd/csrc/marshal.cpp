// Argument marshalling of the batch calls, and of the calls on KV blocks, for the Python binding: the common case (descriptor arrays
// that already are contiguous numpy arrays of the right type, device memory as CUDA tensors or
// addresses) in one native step.  A call on a few chunks takes the GPU under 10 us, and converting
// nine arguments in Python took as long.  Anything unusual is left to the Python code: the
// functions return None then, having done nothing.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/pgcm.h"
#include "../../include/pgcm_kv.h"

namespace {

// names looked up on every call
PyObject *s_is_cuda, *s_is_contiguous, *s_data_ptr, *s_handle;

// the C entry points, by address
typedef int (*encrypt_fn)(void*, size_t, const void*, uint32_t, const void*, const void*,
                          const void*, const void*, const void*, void*, void*);
typedef int (*decrypt_fn)(void*, size_t, const void*, uint32_t, const void*, const void*,
                          const void*, const void*, const void*, const void*, void*, void*);
encrypt_fn g_encrypt;
decrypt_fn g_decrypt;

// A one-dimensional contiguous buffer of n unsigned items of `size` bytes; None is NULL.
class Array {
  public:
    ~Array() {
        if (held_) PyBuffer_Release(&view_);
    }
    bool take(PyObject* o, Py_ssize_t n, Py_ssize_t size) {
        if (o == Py_None) return true;
        if (PyObject_GetBuffer(o, &view_, PyBUF_FORMAT | PyBUF_ND | PyBUF_C_CONTIGUOUS) != 0) {
            PyErr_Clear();
            return false;
        }
        held_ = true;
        const char* f = view_.format;
        if (f == nullptr || f[0] == '\0' || f[1] != '\0') return false;
        const bool unsigned_int = f[0] == 'I' || f[0] == 'L' || f[0] == 'Q';
        ptr_ = view_.buf;
        return unsigned_int && view_.itemsize == size && view_.ndim == 1 &&
               (n < 0 || view_.shape[0] == n);
    }
    const void* ptr() const { return ptr_; }
    Py_ssize_t count() const { return held_ ? view_.shape[0] : -1; }

  private:
    Py_buffer view_;
    bool held_ = false;
    const void* ptr_ = nullptr;
};

// device address of an int, of None (NULL) or of a contiguous CUDA tensor
bool device_address(PyObject* o, void** out) {
    if (o == Py_None) {
        *out = nullptr;
        return true;
    }
    PyObject* value = nullptr;
    if (PyLong_CheckExact(o)) {
        Py_INCREF(o);
        value = o;
    } else {
        PyObject* cuda = PyObject_GetAttr(o, s_is_cuda);
        const bool on_gpu = cuda == Py_True;
        Py_XDECREF(cuda);
        if (on_gpu) {
            PyObject* contiguous = PyObject_CallMethodNoArgs(o, s_is_contiguous);
            if (contiguous == Py_True) value = PyObject_CallMethodNoArgs(o, s_data_ptr);
            Py_XDECREF(contiguous);
        }
    }
    bool ok = false;
    if (value != nullptr) {
        *out = PyLong_AsVoidPtr(value);
        ok = PyErr_Occurred() == nullptr;
        Py_DECREF(value);
    }
    PyErr_Clear();
    return ok;
}

// (key, ivs, iv_bytes, aad, aad_len, src, length, dst, tags[, ok], stream) -> status or None
PyObject* batch(PyObject* const* args, Py_ssize_t nargs, bool decrypt) {
    if (nargs != (decrypt ? 11 : 10)) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    void *key, *ivs, *tags, *ok = nullptr, *stream;
    PyObject* handle = PyObject_GetAttr(args[0], s_handle);
    if (handle == nullptr || !PyLong_CheckExact(handle)) {
        PyErr_Clear();
        Py_XDECREF(handle);
        Py_RETURN_NONE;
    }
    key = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    const long iv_bytes = PyLong_AsLong(args[2]);
    if (PyErr_Occurred() || iv_bytes < 0 || iv_bytes > 0x7FFFFFFF) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    Array len, src, dst, aad, aad_len;
    if (args[6] == Py_None || !len.take(args[6], -1, 8)) Py_RETURN_NONE;
    const Py_ssize_t n = len.count();
    if (!src.take(args[5], n, 8) || !dst.take(args[7], n, 8) || !aad.take(args[3], n, 8) ||
        !aad_len.take(args[4], n, 4) || !device_address(args[1], &ivs) ||
        !device_address(args[8], &tags) || (decrypt && !device_address(args[9], &ok)) ||
        !device_address(args[nargs - 1], &stream))
        Py_RETURN_NONE;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = decrypt ? g_decrypt(key, (size_t)n, ivs, (uint32_t)iv_bytes, aad.ptr(), aad_len.ptr(),
                                 src.ptr(), len.ptr(), dst.ptr(), tags, ok, stream)
                     : g_encrypt(key, (size_t)n, ivs, (uint32_t)iv_bytes, aad.ptr(), aad_len.ptr(),
                                 src.ptr(), len.ptr(), dst.ptr(), tags, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

PyObject* encrypt_batch(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return batch(args, nargs, false);
}
PyObject* decrypt_verify_batch(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return batch(args, nargs, true);
}

// ---- the operators on KV blocks (kv.py): the same, for tensors of the shapes and types that they take

PyObject *s_shape, *s_stride, *s_dtype;
PyObject *d_f16, *d_bf16, *d_i8, *d_i32, *d_i64, *d_f32;  // torch's types

struct KvCalls {
    decltype(&pgcm_kv_append) append;
    decltype(&pgcm_kv_attend) attend;
    decltype(&pgcm_kv_summarize) summarize;
    decltype(&pgcm_kv_select) select;
    decltype(&pgcm_kv_evict) evict;
} g_kv;

// A CUDA tensor; strides of dimensions of one count as zero.
struct Tensor {
    void* at = nullptr;
    int64_t shape[4] = {0, 0, 0, 0}, stride[4] = {0, 0, 0, 0};

    static bool numbers(PyObject* o, int dims, int64_t* to) {
        bool ok = o != nullptr && PyTuple_Check(o) && PyTuple_GET_SIZE(o) == dims;
        for (int i = 0; ok && i < dims; ++i) {
            to[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
            ok = !(to[i] == -1 && PyErr_Occurred());
        }
        Py_XDECREF(o);
        return ok;
    }
    // of this type and number of dimensions, contiguous as a whole or in the last of them
    bool take(PyObject* o, PyObject* dtype, int dims, bool whole) {
        PyObject* type = PyObject_GetAttr(o, s_dtype);
        const bool right = type == dtype;
        Py_XDECREF(type);
        if (!right || !numbers(PyObject_GetAttr(o, s_shape), dims, shape)) return false;
        if (!whole) {
            if (!numbers(PyObject_CallMethodNoArgs(o, s_stride), dims, stride)) return false;
            if (shape[dims - 1] > 1 && stride[dims - 1] != 1) return false;
            for (int i = 0; i < dims; ++i)
                if (shape[i] == 1) stride[i] = 0;
        } else {
            PyObject* contiguous = PyObject_CallMethodNoArgs(o, s_is_contiguous);
            const bool is = contiguous == Py_True;
            Py_XDECREF(contiguous);
            if (!is) return false;
        }
        PyObject* cuda = PyObject_GetAttr(o, s_is_cuda);
        const bool on_gpu = cuda == Py_True;
        Py_XDECREF(cuda);
        if (!on_gpu) return false;
        PyObject* value = PyObject_CallMethodNoArgs(o, s_data_ptr);
        if (value == nullptr) return false;
        at = PyLong_AsVoidPtr(value);
        Py_DECREF(value);
        return PyErr_Occurred() == nullptr;
    }
    bool is(int64_t a, int64_t b = -1, int64_t c = -1, int64_t d = -1) const {
        return shape[0] == a && (b < 0 || shape[1] == b) && (c < 0 || shape[2] == c) && (d < 0 || shape[3] == d);
    }
};

// Arguments one after the other; good() turns false for good at the first one that is unusual.
class Arguments {
  public:
    Arguments(PyObject* const* args, Py_ssize_t n) : args_(args), n_(n) {}
    ~Arguments() {
        if (!good_) PyErr_Clear();
    }
    bool good() const { return good_; }
    bool all_taken() const { return good_ && at_ == n_; }
    void* address() {
        PyObject* o = next();
        if (o == nullptr || o == Py_None) return nullptr;
        void* p = PyLong_Check(o) ? PyLong_AsVoidPtr(o) : nullptr;
        good_ = good_ && PyLong_Check(o) && PyErr_Occurred() == nullptr;
        return p;
    }
    uint32_t number() {
        PyObject* o = next();
        if (o == nullptr || !PyLong_Check(o)) return refuse();
        const long long x = PyLong_AsLongLong(o);
        if (PyErr_Occurred() || x < 0 || x > 0xFFFFFFFFll) return refuse();
        return (uint32_t)x;
    }
    float real() {
        PyObject* o = next();
        if (o == nullptr) return 0.f;
        const double x = PyFloat_AsDouble(o);
        if (PyErr_Occurred()) refuse();
        return (float)x;
    }
    // false for None, which only may be where it is allowed
    bool tensor(Tensor* t, PyObject* dtype, int dims, bool whole, bool may_be_none = false) {
        PyObject* o = next();
        if (o == nullptr) return false;
        if (o == Py_None) {
            if (!may_be_none) refuse();
            return false;
        }
        if (!t->take(o, dtype, dims, whole)) refuse();
        return good_;
    }
    void need(bool is) { good_ = good_ && is; }

  private:
    PyObject* next() {
        if (!good_ || at_ >= n_) {
            good_ = false;
            return nullptr;
        }
        return args_[at_++];
    }
    uint32_t refuse() {
        good_ = false;
        return 0;
    }
    PyObject* const* args_;
    Py_ssize_t n_, at_ = 0;
    bool good_ = true;
};

PyObject* half_of(uint32_t half) { return half == PGCM_KV_F16 ? d_f16 : d_bf16; }

template <class Call>
PyObject* called(Call call) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// (cache, q, k, v, positions, slots, q_out, q_weight, k_weight, eps, rope, adjacent, stream) -> status or None
PyObject* kv_append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    const auto* cache = (const pgcm_kv_cache*)in.address();
    if (!in.good() || cache == nullptr) Py_RETURN_NONE;
    PyObject* half = half_of(cache->half);
    const int64_t d = cache->head_dim, kv = cache->kv_heads;
    pgcm_kv_append_args a = {};
    Tensor q, k, v, positions, slots, q_out, q_weight, k_weight, rope;
    const bool has_q = in.tensor(&q, half, 3, false, true);
    in.tensor(&k, half, 3, false);
    in.tensor(&v, half, 3, false);
    const int64_t n = k.shape[0];
    const bool placed = in.tensor(&positions, d_i32, 1, true, true);
    in.tensor(&slots, d_i64, 1, true);
    const bool has_out = in.tensor(&q_out, half, 3, false, true);
    if (in.tensor(&q_weight, half, 1, true, true)) in.need(q_weight.is(d));
    if (in.tensor(&k_weight, half, 1, true, true)) in.need(k_weight.is(d));
    a.eps = in.real();
    const bool turned = in.tensor(&rope, d_f32, 2, true, true);
    a.adjacent = in.number();
    void* stream = in.address();
    in.need(k.is(n, kv, d) && v.is(n, kv, d) && slots.is(n) && has_q == has_out);
    if (has_q) in.need(q.is(n, q.shape[1], d) && q_out.is(n, q.shape[1], d));
    if (turned) in.need(placed && positions.is(n));
    in.need(n <= 0xFFFFFFFFll && q.shape[1] <= 0xFFFFFFFFll && rope.shape[0] <= 0xFFFFFFFFll && rope.shape[1] <= 0xFFFFFFFFll);
    if (!in.all_taken()) Py_RETURN_NONE;
    a.tokens = (uint32_t)n, a.heads = (uint32_t)q.shape[1];
    a.q = q.at, a.k = k.at, a.v = v.at, a.q_out = q_out.at;
    a.q_token = q.stride[0], a.q_head = q.stride[1], a.k_token = k.stride[0], a.k_head = k.stride[1];
    a.v_token = v.stride[0], a.v_head = v.stride[1], a.q_out_token = q_out.stride[0], a.q_out_head = q_out.stride[1];
    a.positions = turned ? (const int32_t*)positions.at : nullptr, a.slots = (const int64_t*)slots.at;
    a.q_weight = q_weight.at, a.k_weight = k_weight.at, a.rope = (const float*)rope.at;
    a.rope_positions = (uint32_t)rope.shape[0], a.rope_dim = (uint32_t)rope.shape[1];
    return called([&] { return g_kv.append(cache, &a, stream); });
}

// (workspace, cache, q, tables, lens, out, lse, scale, selected, weights, kept, decay, stream) -> status or None
PyObject* kv_attend(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    auto* space = (pgcm_kv_t*)in.address();
    const auto* cache = (const pgcm_kv_cache*)in.address();
    if (!in.good() || cache == nullptr) Py_RETURN_NONE;
    PyObject* half = half_of(cache->half);
    pgcm_kv_attend_args a = {};
    Tensor q, tables, lens, out, lse, selected, weights, kept;
    in.tensor(&q, half, 3, false);
    in.tensor(&tables, d_i32, 2, false);
    in.tensor(&lens, d_i32, 1, true);
    in.tensor(&out, half, 3, false);
    const int64_t n = tables.shape[0], row = tables.shape[1], heads = q.shape[1], d = cache->head_dim;
    if (in.tensor(&lse, d_f32, 2, true, true)) in.need(lse.is(n, heads));
    a.scale = in.real();
    if (in.tensor(&selected, d_i32, 3, true, true)) in.need(selected.is(n, cache->kv_heads));
    if (in.tensor(&weights, d_f32, 2, true, true)) in.need(weights.is(n, row));
    if (in.tensor(&kept, d_f32, 2, true, true)) in.need(kept.is(n, row));
    a.decay = in.real();
    void* stream = in.address();
    in.need(q.is(n, heads, d) && lens.is(n) && out.is(n, heads, d) && n <= 0xFFFFFFFFll && row <= 0xFFFFFFFFll &&
            heads <= 0xFFFFFFFFll && selected.shape[2] <= 0xFFFFFFFFll);
    if (!in.all_taken()) Py_RETURN_NONE;
    a.requests = (uint32_t)n, a.heads = (uint32_t)heads, a.row_blocks = (uint32_t)row, a.keep = (uint32_t)selected.shape[2];
    a.q = q.at, a.q_request = q.stride[0], a.q_head = q.stride[1];
    a.out = out.at, a.out_request = out.stride[0], a.out_head = out.stride[1];
    a.tables = (const int32_t*)tables.at, a.table_row = tables.stride[0], a.lens = (const int32_t*)lens.at;
    a.selected = (const int32_t*)selected.at, a.lse = (float*)lse.at;
    a.weights = (float*)weights.at, a.kept = (const float*)kept.at;
    return called([&] { return g_kv.attend(space, cache, &a, stream); });
}

// (cache, blocks, counts, bounds, scales, entries, stream) -> status or None
PyObject* kv_summarize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    const auto* cache = (const pgcm_kv_cache*)in.address();
    if (!in.good() || cache == nullptr) Py_RETURN_NONE;
    Tensor blocks, counts, bounds, scales, entries;
    in.tensor(&blocks, d_i32, 1, true);
    in.tensor(&counts, d_i32, 1, true);
    in.tensor(&bounds, d_i8, 4, true);
    in.tensor(&scales, d_f32, 2, true);
    const int64_t n = blocks.shape[0], m = bounds.shape[0];
    if (in.tensor(&entries, d_i32, 1, true, true)) in.need(entries.is(n));
    void* stream = in.address();
    in.need(counts.is(n) && bounds.is(m, cache->kv_heads, 2, cache->head_dim) && scales.is(m, cache->kv_heads) &&
            n <= 0xFFFFFFFFll && m <= 0xFFFFFFFFll);
    if (!in.all_taken()) Py_RETURN_NONE;
    return called([&] {
        return g_kv.summarize(cache, (uint32_t)n, (const int32_t*)blocks.at, (const int32_t*)counts.at,
                              (const int32_t*)entries.at, (uint32_t)m, (int8_t*)bounds.at, (float*)scales.at, stream);
    });
}

// (workspace, half, q, tables, lens, bounds, scales, block_tokens, selected, counts, first, last, stream) -> status or None
PyObject* kv_select(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    auto* space = (pgcm_kv_t*)in.address();
    pgcm_kv_select_args a = {};
    Tensor q, tables, lens, bounds, scales, selected, counts;
    a.half = in.number();
    in.tensor(&q, half_of(a.half), 3, false);
    in.tensor(&tables, d_i32, 2, false);
    in.tensor(&lens, d_i32, 1, true);
    in.tensor(&bounds, d_i8, 4, true);
    in.tensor(&scales, d_f32, 2, true);
    a.block_tokens = in.number();
    in.tensor(&selected, d_i32, 3, true);
    const int64_t n = tables.shape[0], row = tables.shape[1], heads = q.shape[1], m = bounds.shape[0], kv = bounds.shape[1],
                  d = bounds.shape[3];
    if (in.tensor(&counts, d_i32, 2, true, true)) in.need(counts.is(n, kv));
    a.first = in.number(), a.last = in.number();
    void* stream = in.address();
    in.need(q.is(n, heads, d) && lens.is(n) && bounds.is(m, kv, 2, d) && scales.is(m, kv) && selected.is(n, kv) &&
            n <= 0xFFFFFFFFll && row <= 0xFFFFFFFFll && heads <= 0xFFFFFFFFll && m <= 0xFFFFFFFFll && kv <= 0xFFFFFFFFll &&
            d <= 0xFFFFFFFFll && selected.shape[2] <= 0xFFFFFFFFll);
    if (!in.all_taken()) Py_RETURN_NONE;
    a.requests = (uint32_t)n, a.heads = (uint32_t)heads, a.kv_heads = (uint32_t)kv, a.head_dim = (uint32_t)d;
    a.q = q.at, a.q_request = q.stride[0], a.q_head = q.stride[1];
    a.tables = (const int32_t*)tables.at, a.table_row = tables.stride[0], a.row_blocks = (uint32_t)row;
    a.entry_count = (uint32_t)m, a.lens = (const int32_t*)lens.at, a.bounds = (const int8_t*)bounds.at;
    a.scales = (const float*)scales.at, a.keep = (uint32_t)selected.shape[2];
    a.selected = (int32_t*)selected.at, a.counts = (int32_t*)counts.at;
    return called([&] { return g_kv.select(space, &a, stream); });
}

// (weights, tables, lens, block_tokens, evict, victims, victim_blocks, tables_out, first, last, blocks, stream) -> status or None
PyObject* kv_evict(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    pgcm_kv_evict_args a = {};
    Tensor weights, tables, lens, evict, victims, victim_blocks, tables_out;
    in.tensor(&weights, d_f32, 2, true);
    in.tensor(&tables, d_i32, 2, false);
    in.tensor(&lens, d_i32, 1, true);
    a.block_tokens = in.number();
    in.tensor(&evict, d_i32, 1, true);
    in.tensor(&victims, d_i32, 2, true);
    const int64_t n = tables.shape[0], row = tables.shape[1], most = victims.shape[1];
    if (in.tensor(&victim_blocks, d_i32, 2, true, true)) in.need(victim_blocks.is(n, most));
    if (in.tensor(&tables_out, d_i32, 2, false, true)) in.need(tables_out.is(n, row));
    a.first = in.number(), a.last = in.number(), a.blocks = in.number();
    void* stream = in.address();
    in.need(weights.is(n, row) && lens.is(n) && evict.is(n) && victims.is(n, most) && n <= 0xFFFFFFFFll &&
            row <= 0xFFFFFFFFll && most <= 0xFFFFFFFFll);
    if (!in.all_taken()) Py_RETURN_NONE;
    a.requests = (uint32_t)n, a.row_blocks = (uint32_t)row, a.most = (uint32_t)most;
    a.weights = (const float*)weights.at, a.tables = (const int32_t*)tables.at, a.table_row = tables.stride[0];
    a.lens = (const int32_t*)lens.at, a.evict = (const int32_t*)evict.at, a.victims = (int32_t*)victims.at;
    a.victim_blocks = (int32_t*)victim_blocks.at;
    a.tables_out = (int32_t*)tables_out.at, a.table_out_row = tables_out.stride[0];
    return called([&] { return g_kv.evict(&a, stream); });
}

// kv_bind(five addresses, in the order of KvCalls; torch's float16, bfloat16, int8, int32, int64, float32)
PyObject* kv_bind(PyObject*, PyObject* args) {
    PyObject *f[5], *d[6];
    if (!PyArg_ParseTuple(args, "OOOOOOOOOOO", &f[0], &f[1], &f[2], &f[3], &f[4], &d[0], &d[1], &d[2], &d[3], &d[4], &d[5]))
        return nullptr;
    void* at[5];
    for (int i = 0; i < 5; ++i) at[i] = PyLong_AsVoidPtr(f[i]);
    if (PyErr_Occurred()) return nullptr;
    g_kv.append = reinterpret_cast<decltype(g_kv.append)>(at[0]);
    g_kv.attend = reinterpret_cast<decltype(g_kv.attend)>(at[1]);
    g_kv.summarize = reinterpret_cast<decltype(g_kv.summarize)>(at[2]);
    g_kv.select = reinterpret_cast<decltype(g_kv.select)>(at[3]);
    g_kv.evict = reinterpret_cast<decltype(g_kv.evict)>(at[4]);
    PyObject** to[6] = {&d_f16, &d_bf16, &d_i8, &d_i32, &d_i64, &d_f32};
    for (int i = 0; i < 6; ++i) {
        Py_INCREF(d[i]);
        Py_XDECREF(*to[i]);
        *to[i] = d[i];
    }
    Py_RETURN_NONE;
}

// bind(address of pgcm_encrypt_batch_iv, address of pgcm_decrypt_verify_batch_iv)
PyObject* bind(PyObject*, PyObject* args) {
    PyObject *e, *d;
    if (!PyArg_ParseTuple(args, "OO", &e, &d)) return nullptr;
    g_encrypt = reinterpret_cast<encrypt_fn>(PyLong_AsVoidPtr(e));
    g_decrypt = reinterpret_cast<decrypt_fn>(PyLong_AsVoidPtr(d));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"encrypt_batch", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(encrypt_batch)),
     METH_FASTCALL, nullptr},
    {"decrypt_verify_batch",
     reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decrypt_verify_batch)),
     METH_FASTCALL, nullptr},
    {"kv_bind", kv_bind, METH_VARARGS, nullptr},
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kv_append)), METH_FASTCALL, nullptr},
    {"kv_attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kv_attend)), METH_FASTCALL, nullptr},
    {"kv_summarize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kv_summarize)), METH_FASTCALL, nullptr},
    {"kv_select", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kv_select)), METH_FASTCALL, nullptr},
    {"kv_evict", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kv_evict)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_handle = PyUnicode_InternFromString("_h");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_dtype = PyUnicode_InternFromString("dtype");
    if (!s_is_cuda || !s_is_contiguous || !s_data_ptr || !s_handle || !s_shape || !s_stride || !s_dtype) return nullptr;
    return PyModule_Create(&module);
}
