// Workspace of the operators on KV blocks (C ABI of include/pgcm_kv.h).
#include "pgcm_kv_common.h"

#include <new>

using pgcm::hip_noted;

namespace pgcm_kv_impl {

static int grow(pgcm_kv* kv, pgcm_kv::Memory* m, size_t bytes, bool zero, hipStream_t stream) {
    if (m->bytes >= bytes) return PGCM_OK;
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hip_noted(hipStreamIsCapturing(stream, &capture))) return PGCM_ERR_HIP;
    if (capture != hipStreamCaptureStatusNone) return PGCM_ERR_CAPACITY;
    const size_t room = bytes + bytes / 2 + 4096;
    void* p = nullptr;
    try {
        kv->outgrown.reserve(kv->outgrown.size() + 1);
    } catch (const std::bad_alloc&) {
        return PGCM_ERR_NOMEM;
    }
    if (hip_noted(hipMalloc(&p, room))) {
        (void)hipGetLastError();
        return PGCM_ERR_NOMEM;
    }
    if (zero && hip_noted(hipMemsetAsync(p, 0, room, stream))) {
        (void)hipFree(p);
        return PGCM_ERR_HIP;
    }
    if (m->at != nullptr) kv->outgrown.push_back(m->at);
    m->at = (uint8_t*)p;
    m->bytes = room;
    return PGCM_OK;
}

int kv_ensure(pgcm_kv* kv, size_t counters, size_t scratch, hipStream_t stream) {
    int device = 0;
    if (hip_noted(hipGetDevice(&device))) return PGCM_ERR_HIP;
    if (device != kv->device) return PGCM_ERR_ARG;
    int rc = grow(kv, &kv->counters, counters, true, stream);
    return rc != PGCM_OK ? rc : grow(kv, &kv->scratch, scratch, false, stream);
}

}  // namespace pgcm_kv_impl

extern "C" {
#pragma GCC visibility push(default)

int pgcm_kv_create(pgcm_kv_t** out) {
    if (out == nullptr) return PGCM_ERR_ARG;
    *out = nullptr;
    pgcm_kv* kv = new (std::nothrow) pgcm_kv();
    if (kv == nullptr) return PGCM_ERR_NOMEM;
    if (hip_noted(hipGetDevice(&kv->device))) {
        delete kv;
        return PGCM_ERR_HIP;
    }
    *out = kv;
    return PGCM_OK;
}

void pgcm_kv_destroy(pgcm_kv_t* kv) {
    if (kv == nullptr) return;
    if (kv->counters.at) (void)hipFree(kv->counters.at);
    if (kv->scratch.at) (void)hipFree(kv->scratch.at);
    for (void* p : kv->outgrown) (void)hipFree(p);
    delete kv;
}

int pgcm_kv_reserve(pgcm_kv_t* kv, uint32_t requests, uint32_t heads, uint32_t kv_heads, uint32_t head_dim,
                    uint32_t block_tokens, uint32_t row_blocks, void* hip_stream) {
    using namespace pgcm_kv_impl;
    if (kv == nullptr) return PGCM_ERR_ARG;
    if (const int rc = check_sizes(requests, heads, kv_heads, head_dim, block_tokens, row_blocks)) return rc;
    const Room a = attend_room(requests, heads, kv_heads, head_dim, (uint64_t)row_blocks * (block_tokens / kPiece));
    const size_t s = select_room(requests, kv_heads, row_blocks);
    const std::lock_guard<std::mutex> held(kv->enqueue);
    return kv_ensure(kv, a.counters, a.scratch > s ? a.scratch : s, (hipStream_t)hip_stream);
}

#pragma GCC visibility pop
}  // extern "C"
