// Attention with a window: the calls (C ABI of include/pgcm_kv8.h).
#include "pgcm_kv_window.h"

#include <cmath>

using namespace pgcm_kv_impl;

namespace {

constexpr int64_t kMostTokenStride = 1 << 25;

int window_args(const pgcm_kv_window_args* args, uint32_t kv_heads, uint32_t head_dim, uint32_t block_tokens, WindowArgs* a) {
    if (args->q == nullptr || args->out == nullptr || args->lens == nullptr || !std::isfinite(args->scale) ||
        (args->tables == nullptr && args->row_blocks != 0) || args->requests > 0x7FFFFFFFu || args->tokens > 0x7FFFFFFFu)
        return PGCM_ERR_ARG;
    if (args->starts == nullptr ? args->tokens != args->requests || args->most != 1 : args->most == 0) return PGCM_ERR_ARG;
    if (const int rc = check_sizes(args->requests, args->heads, kv_heads, head_dim, block_tokens, args->row_blocks)) return rc;
    if (!aligned(args->q, args->q_token, args->q_head) || !aligned(args->out, args->out_token, args->out_head)) return PGCM_ERR_ALIGN;
    a->q = (const uint8_t*)args->q, a->out = (uint8_t*)args->out;
    a->q_token = 2 * args->q_token, a->q_head = 2 * args->q_head;
    a->out_token = 2 * args->out_token, a->out_head = 2 * args->out_head;
    a->tables = args->tables, a->lens = args->lens, a->starts = args->starts, a->lse = args->lse;
    a->table_row = args->table_row;
    a->requests = args->requests, a->tokens = args->tokens;
    a->most = args->most < args->tokens ? args->most : args->tokens;
    a->kv_heads = kv_heads, a->group = args->heads / kv_heads, a->head_dim = head_dim;
    a->block_tokens = block_tokens, a->row_blocks = args->row_blocks;
    a->window = args->window, a->sinks = args->sinks;
    a->scale = (float)((double)args->scale * 1.4426950408889634);
    return PGCM_OK;
}
// (lanes' places within sixteen rows are counted in 32 bits)
bool token_stride(int64_t x) { return x >= 0 && x <= kMostTokenStride; }

}  // namespace

extern "C" {
#pragma GCC visibility push(default)

int pgcm_kv8_attend(pgcm_kv_t* kv, const pgcm_kv8_cache* cache, const pgcm_kv_window_args* args, void* hip_stream) {
    if (kv == nullptr || args == nullptr) return PGCM_ERR_ARG;
    if (const int rc = check_cache8(cache)) return rc;
    if (args->requests == 0 || args->tokens == 0) return PGCM_OK;
    WindowArgs a{};
    if (const int rc = window_args(args, cache->kv_heads, cache->head_dim, cache->block_tokens, &a)) return rc;
    if (!token_stride(cache->k_token) || !token_stride(cache->v_token)) return PGCM_ERR_ARG;
    a.k = (const uint8_t*)cache->k, a.v = (const uint8_t*)cache->v, a.blocks = cache->blocks;
    a.k_block = cache->k_block, a.k_token = cache->k_token, a.k_head = cache->k_head;
    a.v_block = cache->v_block, a.v_token = cache->v_token, a.v_head = cache->v_head;
    a.k_scales = cache->k_scales, a.v_scales = cache->v_scales;
    a.k_scale_block = cache->k_scale_block, a.k_scale_head = cache->k_scale_head;
    a.v_scale_block = cache->v_scale_block, a.v_scale_head = cache->v_scale_head;
    const std::lock_guard<std::mutex> held(kv->enqueue);
    return window_few(kv, a, cache->half, cache->code, (hipStream_t)hip_stream);
}

int pgcm_kv_window(pgcm_kv_t* kv, const pgcm_kv_cache* cache, const pgcm_kv_window_args* args, void* hip_stream) {
    if (kv == nullptr || args == nullptr) return PGCM_ERR_ARG;
    if (const int rc = check_cache(cache)) return rc;
    if (args->requests == 0 || args->tokens == 0) return PGCM_OK;
    WindowArgs a{};
    if (const int rc = window_args(args, cache->kv_heads, cache->head_dim, cache->block_tokens, &a)) return rc;
    if (!token_stride(cache->k_token) || !token_stride(cache->v_token)) return PGCM_ERR_ARG;
    a.k = (const uint8_t*)cache->k, a.v = (const uint8_t*)cache->v, a.blocks = cache->blocks;
    a.k_block = 2 * cache->k_block, a.k_token = 2 * cache->k_token, a.k_head = 2 * cache->k_head;
    a.v_block = 2 * cache->v_block, a.v_token = 2 * cache->v_token, a.v_head = 2 * cache->v_head;
    const std::lock_guard<std::mutex> held(kv->enqueue);
    return a.most == 1 ? window_few(kv, a, cache->half, ~0u, (hipStream_t)hip_stream)
                       : window_many(kv, a, cache->half, (hipStream_t)hip_stream);
}

int pgcm_kv_window_reserve(pgcm_kv_t* kv, uint32_t heads, uint32_t kv_heads, uint32_t head_dim, void* hip_stream) {
    if (kv == nullptr) return PGCM_ERR_ARG;
    if (const int rc = check_sizes(1, heads, kv_heads, head_dim, kPiece, 1)) return rc;
    const Room few = window_few_room(heads, kv_heads, head_dim), many = window_many_room(head_dim);
    const Room room{few.counters, few.scratch > many.scratch ? few.scratch : many.scratch};
    const std::lock_guard<std::mutex> held(kv->enqueue);
    return kv_ensure(kv, room.counters, room.scratch, (hipStream_t)hip_stream);
}

#pragma GCC visibility pop
}  // extern "C"
