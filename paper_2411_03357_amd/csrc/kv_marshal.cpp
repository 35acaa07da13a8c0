// Native marshalling of the operators on KV blocks (kv.py, kv8.py): a torch extension, as what a tensor is takes five calls of the
// interpreter to ask it and some nanoseconds to read (an append of nine tensors: 6.1 us of the host and 4.0).  Each call gives
// the status, or None for anything unusual, which the Python code then names.
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "../../include/pgcm.h"
#include "../../include/pgcm_kv8.h"

namespace {

struct KvCalls {
    decltype(&pgcm_kv_append) append;
    decltype(&pgcm_kv_attend) attend;
    decltype(&pgcm_kv_summarize) summarize;
    decltype(&pgcm_kv_select) select;
    decltype(&pgcm_kv_evict) evict;
} g_kv;
struct Kv8Calls {
    decltype(&pgcm_kv8_append) append;
    decltype(&pgcm_kv8_store) store;
    decltype(&pgcm_kv8_load) load;
    decltype(&pgcm_kv8_attend) attend;
    decltype(&pgcm_kv_window) window;
} g_kv8;

// A cache as kv.py hands it over: with the device that it is on.
struct Cache {
    pgcm_kv_cache c;
    int64_t device;
};

struct Cache8 {
    pgcm_kv8_cache c;
    int64_t device;
};

// A tensor on the current CUDA device; strides of dimensions of one count as zero.
struct Tensor {
    void* at = nullptr;
    bool none = true;   // not taken
    int64_t shape[4] = {0, 0, 0, 0}, stride[4] = {0, 0, 0, 0};

    // of this type and number of dimensions, contiguous as a whole or in the last of them
    bool take(PyObject* o, int64_t device, at::ScalarType dtype, int dims, bool whole) {
        if (!THPVariable_Check(o)) return false;
        try {
            const at::Tensor& t = THPVariable_Unpack(o);
            if (t.scalar_type() != dtype || t.dim() != dims || !t.is_cuda() || t.get_device() != device ||
                t.layout() != at::kStrided)
                return false;
            const auto sizes = t.sizes(), strides = t.strides();
            for (int i = 0; i < dims; ++i) {
                shape[i] = sizes[i];
                stride[i] = sizes[i] == 1 ? 0 : strides[i];
            }
            if (whole ? !t.is_contiguous() : shape[dims - 1] > 1 && stride[dims - 1] != 1) return false;
            at = t.data_ptr();
            none = false;
        } catch (...) {   // (a tensor without memory of its own)
            return false;
        }
        return true;
    }
    // for what an address says to be there: a tensor without elements has none, and nothing of it is read
    void* given() const { return at != nullptr ? at : none ? nullptr : (void*)4096; }
    bool is(int64_t a, int64_t b = -1, int64_t c = -1, int64_t d = -1) const {
        return shape[0] == a && (b < 0 || shape[1] == b) && (c < 0 || shape[2] == c) && (d < 0 || shape[3] == d);
    }
};

// Arguments one after the other, the current device or None for it first; good() turns false for good at the first one that is
// unusual.
class Arguments {
  public:
    Arguments(PyObject* const* args, Py_ssize_t n) : args_(args), n_(n) {
        if (n > 0 && args[0] == Py_None) {
            ++at_;
            try {
                device_ = c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice().index();
            } catch (...) {   // (a torch without GPUs)
                good_ = false;
            }
        } else {
            device_ = number();
        }
    }
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
    // on the current device
    const pgcm_kv_cache* cache() { return placed<Cache>(); }
    const pgcm_kv8_cache* cache8() { return placed<Cache8>(); }
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
    bool tensor(Tensor* t, at::ScalarType dtype, int dims, bool whole, bool may_be_none = false) {
        PyObject* o = next();
        if (o == nullptr) return false;
        if (o == Py_None) {
            if (!may_be_none) refuse();
            return false;
        }
        if (!t->take(o, device_, dtype, dims, whole)) refuse();
        return good_;
    }
    void need(bool is) { good_ = good_ && is; }

  private:
    template <class Placed>
    auto placed() -> decltype(&((const Placed*)nullptr)->c) {
        const auto* cache = (const Placed*)address();
        if (cache == nullptr || cache->device != device_) good_ = false;
        return good_ ? &cache->c : nullptr;
    }
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
    int64_t device_ = 0;
    bool good_ = true;
};

at::ScalarType half_of(uint32_t half) { return half == PGCM_KV_F16 ? at::kHalf : at::kBFloat16; }

template <class Call>
PyObject* called(Call call) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// the arguments of an append but for the cache, and the call with them
template <class Cache, class Call>
PyObject* append_to(Arguments& in, const Cache* cache, Call call) {
    if (cache == nullptr) Py_RETURN_NONE;
    const at::ScalarType half = half_of(cache->half);
    const int64_t d = cache->head_dim, kv = cache->kv_heads;
    pgcm_kv_append_args a = {};
    Tensor q, k, v, positions, slots, q_out, q_weight, k_weight, rope;
    const bool has_q = in.tensor(&q, half, 3, false, true);
    in.tensor(&k, half, 3, false);
    in.tensor(&v, half, 3, false);
    const int64_t n = k.shape[0];
    const bool placed = in.tensor(&positions, at::kInt, 1, true, true);
    in.tensor(&slots, at::kLong, 1, true);
    const bool has_out = in.tensor(&q_out, half, 3, false, true);
    if (in.tensor(&q_weight, half, 1, true, true)) in.need(q_weight.is(d));
    if (in.tensor(&k_weight, half, 1, true, true)) in.need(k_weight.is(d));
    a.eps = in.real();
    const bool turned = in.tensor(&rope, at::kFloat, 2, true, true);
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
    a.q_weight = q_weight.at, a.k_weight = k_weight.at, a.rope = (const float*)rope.given();
    a.rope_positions = (uint32_t)rope.shape[0], a.rope_dim = (uint32_t)rope.shape[1];
    return called([&] { return call(cache, &a, stream); });
}

// (device, cache, q, k, v, positions, slots, q_out, q_weight, k_weight, eps, rope, adjacent, stream) -> status or None
PyObject* kv_append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    return append_to(in, in.cache(), g_kv.append);
}
PyObject* kv8_append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    return append_to(in, in.cache8(), g_kv8.append);
}

// the arguments of attention with a window but for the workspace and the cache, and the call with them
template <class Cache, class Call>
PyObject* attend_in_window(Arguments& in, pgcm_kv_t* space, const Cache* cache, Call call) {
    if (cache == nullptr) Py_RETURN_NONE;
    const at::ScalarType half = half_of(cache->half);
    pgcm_kv_window_args a = {};
    Tensor q, tables, lens, out, lse, starts;
    in.tensor(&q, half, 3, false);
    in.tensor(&tables, at::kInt, 2, false);
    in.tensor(&lens, at::kInt, 1, true);
    in.tensor(&out, half, 3, false);
    const int64_t n = tables.shape[0], row = tables.shape[1], rows = q.shape[0], heads = q.shape[1], d = cache->head_dim;
    if (in.tensor(&lse, at::kFloat, 2, true, true)) in.need(lse.is(rows, heads));
    a.scale = in.real();
    a.window = in.number(), a.sinks = in.number();
    if (in.tensor(&starts, at::kInt, 1, true, true)) in.need(starts.is(n + 1));
    else in.need(rows == n);
    a.most = in.number();
    void* stream = in.address();
    in.need(q.is(rows, heads, d) && lens.is(n) && out.is(rows, heads, d) && n <= 0xFFFFFFFFll && row <= 0xFFFFFFFFll &&
            rows <= 0xFFFFFFFFll && heads <= 0xFFFFFFFFll);
    if (!in.all_taken()) Py_RETURN_NONE;
    a.requests = (uint32_t)n, a.heads = (uint32_t)heads, a.tokens = (uint32_t)rows, a.row_blocks = (uint32_t)row;
    a.q = q.at, a.q_token = q.stride[0], a.q_head = q.stride[1];
    a.out = out.at, a.out_token = out.stride[0], a.out_head = out.stride[1];
    a.tables = (const int32_t*)tables.at, a.table_row = tables.stride[0], a.lens = (const int32_t*)lens.at;
    a.starts = (const int32_t*)starts.at, a.lse = (float*)lse.at;
    return called([&] { return call(space, cache, &a, stream); });
}

// (device, workspace, cache, q, tables, lens, out, lse, scale, window, sinks, starts, most, stream) -> status or None
PyObject* kv8_attend(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    auto* space = (pgcm_kv_t*)in.address();
    return attend_in_window(in, space, in.cache8(), g_kv8.attend);
}
PyObject* kv_window(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    auto* space = (pgcm_kv_t*)in.address();
    return attend_in_window(in, space, in.cache(), g_kv8.window);
}

// (device, cache8, cache, blocks, counts, others, stream) -> status or None
template <bool kStore>
PyObject* kv8_move(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    const pgcm_kv8_cache* cache8 = in.cache8();
    const pgcm_kv_cache* cache = cache8 == nullptr ? nullptr : in.cache();
    if (cache == nullptr) Py_RETURN_NONE;
    Tensor blocks, counts, others;
    in.tensor(&blocks, at::kInt, 1, true);
    const int64_t n = blocks.shape[0];
    if (in.tensor(&counts, at::kInt, 1, true, true)) in.need(counts.is(n));
    if (in.tensor(&others, at::kInt, 1, true, true)) in.need(others.is(n));
    void* stream = in.address();
    in.need(n <= 0xFFFFFFFFll);
    if (!in.all_taken()) Py_RETURN_NONE;
    return called([&] {
        return (kStore ? g_kv8.store : g_kv8.load)(cache8, cache, (uint32_t)n, (const int32_t*)blocks.at,
                                                   (const int32_t*)counts.at, (const int32_t*)others.at, stream);
    });
}

// (device, workspace, cache, q, tables, lens, out, lse, scale, selected, weights, kept, decay, stream) -> status or None
PyObject* kv_attend(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    auto* space = (pgcm_kv_t*)in.address();
    const pgcm_kv_cache* cache = in.cache();
    if (cache == nullptr) Py_RETURN_NONE;
    const at::ScalarType half = half_of(cache->half);
    pgcm_kv_attend_args a = {};
    Tensor q, tables, lens, out, lse, selected, weights, kept;
    in.tensor(&q, half, 3, false);
    in.tensor(&tables, at::kInt, 2, false);
    in.tensor(&lens, at::kInt, 1, true);
    in.tensor(&out, half, 3, false);
    const int64_t n = tables.shape[0], row = tables.shape[1], heads = q.shape[1], d = cache->head_dim;
    if (in.tensor(&lse, at::kFloat, 2, true, true)) in.need(lse.is(n, heads));
    a.scale = in.real();
    if (in.tensor(&selected, at::kInt, 3, true, true)) in.need(selected.is(n, cache->kv_heads));
    if (in.tensor(&weights, at::kFloat, 2, true, true)) in.need(weights.is(n, row));
    if (in.tensor(&kept, at::kFloat, 2, true, true)) in.need(kept.is(n, row));
    a.decay = in.real();
    void* stream = in.address();
    in.need(q.is(n, heads, d) && lens.is(n) && out.is(n, heads, d) && n <= 0xFFFFFFFFll && row <= 0xFFFFFFFFll &&
            heads <= 0xFFFFFFFFll && selected.shape[2] <= 0xFFFFFFFFll);
    if (!in.all_taken()) Py_RETURN_NONE;
    a.requests = (uint32_t)n, a.heads = (uint32_t)heads, a.row_blocks = (uint32_t)row, a.keep = (uint32_t)selected.shape[2];
    a.q = q.at, a.q_request = q.stride[0], a.q_head = q.stride[1];
    a.out = out.at, a.out_request = out.stride[0], a.out_head = out.stride[1];
    a.tables = (const int32_t*)tables.at, a.table_row = tables.stride[0], a.lens = (const int32_t*)lens.at;
    a.selected = (const int32_t*)selected.given(), a.lse = (float*)lse.at;
    a.weights = (float*)weights.given(), a.kept = (const float*)kept.given();
    return called([&] { return g_kv.attend(space, cache, &a, stream); });
}

// (device, cache, blocks, counts, bounds, scales, entries, stream) -> status or None
PyObject* kv_summarize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    const pgcm_kv_cache* cache = in.cache();
    if (cache == nullptr) Py_RETURN_NONE;
    Tensor blocks, counts, bounds, scales, entries;
    in.tensor(&blocks, at::kInt, 1, true);
    in.tensor(&counts, at::kInt, 1, true);
    in.tensor(&bounds, at::kChar, 4, true);
    in.tensor(&scales, at::kFloat, 2, true);
    const int64_t n = blocks.shape[0], m = bounds.shape[0];
    if (in.tensor(&entries, at::kInt, 1, true, true)) in.need(entries.is(n));
    void* stream = in.address();
    in.need(counts.is(n) && bounds.is(m, cache->kv_heads, 2, cache->head_dim) && scales.is(m, cache->kv_heads) &&
            n <= 0xFFFFFFFFll && m <= 0xFFFFFFFFll);
    if (!in.all_taken()) Py_RETURN_NONE;
    return called([&] {
        return g_kv.summarize(cache, (uint32_t)n, (const int32_t*)blocks.at, (const int32_t*)counts.at,
                              (const int32_t*)entries.at, (uint32_t)m, (int8_t*)bounds.at, (float*)scales.at, stream);
    });
}

// (device, workspace, half, q, tables, lens, bounds, scales, block_tokens, selected, counts, first, last, stream)
// -> status or None
PyObject* kv_select(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    auto* space = (pgcm_kv_t*)in.address();
    pgcm_kv_select_args a = {};
    Tensor q, tables, lens, bounds, scales, selected, counts;
    a.half = in.number();
    in.tensor(&q, half_of(a.half), 3, false);
    in.tensor(&tables, at::kInt, 2, false);
    in.tensor(&lens, at::kInt, 1, true);
    in.tensor(&bounds, at::kChar, 4, true);
    in.tensor(&scales, at::kFloat, 2, true);
    a.block_tokens = in.number();
    in.tensor(&selected, at::kInt, 3, true);
    const int64_t n = tables.shape[0], row = tables.shape[1], heads = q.shape[1], m = bounds.shape[0], kv = bounds.shape[1],
                  d = bounds.shape[3];
    if (in.tensor(&counts, at::kInt, 2, true, true)) in.need(counts.is(n, kv));
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

// (device, weights, tables, lens, block_tokens, evict, victims, victim_blocks, tables_out, first, last, blocks, stream)
// -> status or None
PyObject* kv_evict(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    Arguments in(args, nargs);
    pgcm_kv_evict_args a = {};
    Tensor weights, tables, lens, evict, victims, victim_blocks, tables_out;
    in.tensor(&weights, at::kFloat, 2, true);
    in.tensor(&tables, at::kInt, 2, false);
    in.tensor(&lens, at::kInt, 1, true);
    a.block_tokens = in.number();
    in.tensor(&evict, at::kInt, 1, true);
    in.tensor(&victims, at::kInt, 2, true);
    const int64_t n = tables.shape[0], row = tables.shape[1], most = victims.shape[1];
    if (in.tensor(&victim_blocks, at::kInt, 2, true, true)) in.need(victim_blocks.is(n, most));
    if (in.tensor(&tables_out, at::kInt, 2, false, true)) in.need(tables_out.is(n, row));
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

// bind(five addresses, in the order of KvCalls)
PyObject* bind(PyObject*, PyObject* args) {
    PyObject* f[5];
    if (!PyArg_ParseTuple(args, "OOOOO", &f[0], &f[1], &f[2], &f[3], &f[4])) return nullptr;
    void* at[5];
    for (int i = 0; i < 5; ++i) at[i] = PyLong_AsVoidPtr(f[i]);
    if (PyErr_Occurred()) return nullptr;
    g_kv.append = reinterpret_cast<decltype(g_kv.append)>(at[0]);
    g_kv.attend = reinterpret_cast<decltype(g_kv.attend)>(at[1]);
    g_kv.summarize = reinterpret_cast<decltype(g_kv.summarize)>(at[2]);
    g_kv.select = reinterpret_cast<decltype(g_kv.select)>(at[3]);
    g_kv.evict = reinterpret_cast<decltype(g_kv.evict)>(at[4]);
    Py_RETURN_NONE;
}

// bind8(the addresses of Kv8Calls, in their order)
PyObject* bind8(PyObject*, PyObject* args) {
    PyObject* f[5];
    if (!PyArg_ParseTuple(args, "OOOOO", &f[0], &f[1], &f[2], &f[3], &f[4])) return nullptr;
    void* at[5];
    for (int i = 0; i < 5; ++i) at[i] = PyLong_AsVoidPtr(f[i]);
    if (PyErr_Occurred()) return nullptr;
    g_kv8.append = reinterpret_cast<decltype(g_kv8.append)>(at[0]);
    g_kv8.store = reinterpret_cast<decltype(g_kv8.store)>(at[1]);
    g_kv8.load = reinterpret_cast<decltype(g_kv8.load)>(at[2]);
    g_kv8.attend = reinterpret_cast<decltype(g_kv8.attend)>(at[3]);
    g_kv8.window = reinterpret_cast<decltype(g_kv8.window)>(at[4]);
    Py_RETURN_NONE;
}

template <PyObject* (*kCall)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction fast() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kCall));
}

PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         {"kv_append", fast<kv_append>(), METH_FASTCALL, nullptr},
                         {"kv_attend", fast<kv_attend>(), METH_FASTCALL, nullptr},
                         {"kv_summarize", fast<kv_summarize>(), METH_FASTCALL, nullptr},
                         {"kv_select", fast<kv_select>(), METH_FASTCALL, nullptr},
                         {"kv_evict", fast<kv_evict>(), METH_FASTCALL, nullptr},
                         {"bind8", bind8, METH_VARARGS, nullptr},
                         {"kv8_append", fast<kv8_append>(), METH_FASTCALL, nullptr},
                         {"kv8_store", fast<kv8_move<true>>(), METH_FASTCALL, nullptr},
                         {"kv8_load", fast<kv8_move<false>>(), METH_FASTCALL, nullptr},
                         {"kv8_attend", fast<kv8_attend>(), METH_FASTCALL, nullptr},
                         {"kv_window", fast<kv_window>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

// BUILT_FOR: torch.__version__ when this was compiled; what a tensor is in memory belongs to it
const char kBuiltFor[] = "built for torch " BUILT_FOR;

}  // namespace

PyMODINIT_FUNC PyInit__kv_marshal() {
    PyObject* m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "built_for", kBuiltFor) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
