// New keys and values into a paged cache, and the bounds of its blocks (include/pgcm_kv.h).  Both read and write each
// element once: what bounds them is memory.
#include "pgcm_kv_common.h"

namespace pgcm_kv_impl {
namespace {

constexpr uint32_t kThreads = 256;

// A row of head_dim halves is held by 2^row_power lanes, eight channels each; lanes beyond the row hold nothing.
inline uint32_t row_power_of(uint32_t head_dim) {
    uint32_t p = 0;
    while ((8u << p) < head_dim) ++p;
    return p;
}

struct AppendArgs {
    const uint8_t *q, *k, *v, *q_weight, *k_weight;
    uint8_t *q_out, *k_cache, *v_cache;
    const int32_t* positions;
    const int64_t* slots;
    const float* rope;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, q_out_token, q_out_head;  // bytes
    int64_t kc_block, kc_token, kc_head, vc_block, vc_token, vc_head;
    uint64_t pool_tokens;
    uint32_t heads, kv_heads, head_dim, block_tokens, rope_positions, rope_dim, adjacent, row_power;
    float eps;
};

// One token, and of its rows (queries, keys, values in this order) those that blockIdx.y has.  A lane has the same
// channels of each of its rows, so cosines, sines and weights are read once.
template <class H>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
    const uint32_t token = blockIdx.x, lanes = 1u << a.row_power;
    const uint32_t part = threadIdx.x & (lanes - 1), d = 8 * part, at = threadIdx.x >> a.row_power;
    const uint32_t step = (kThreads >> a.row_power) * gridDim.y;
    const uint32_t rows = a.heads + 2 * a.kv_heads;
    const bool mine = d < a.head_dim;

    const int64_t slot = a.slots[token];
    const bool stored = (uint64_t)slot < a.pool_tokens;
    const uint64_t block = stored ? (uint64_t)slot / a.block_tokens : 0;
    const uint32_t inside = stored ? (uint32_t)((uint64_t)slot - block * a.block_tokens) : 0;

    float c[8], s[8];       // of the lane's channels; the sine with its sign
    const uint32_t half = a.rope_dim / 2;
    const bool turned = a.rope != nullptr && d < a.rope_dim;
    uint32_t partner = part;  // the lane with the other channels of the pairs
    if (a.rope != nullptr && !a.adjacent && turned) partner = d < half ? part + half / 8 : part - half / 8;
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) c[e] = 1.f, s[e] = 0.f;
    if (turned) {
        const int32_t position = a.positions[token];
        const bool known = (uint32_t)position < a.rope_positions;
        const float* line = a.rope + (known ? (size_t)position * a.rope_dim : 0);
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
            const uint32_t n = a.adjacent ? (d + e) / 2 : (d < half ? d : d - half) + e;
            const bool second = a.adjacent ? e % 2 : d >= half;
            c[e] = known ? line[n] : NAN;
            s[e] = known ? line[half + n] : NAN;
            if (!second) s[e] = -s[e];
        }
    }
    float qw[8], kw[8], qo[8], ko[8];   // weights of the lane's channels, and of their partners
    auto weights = [&](const uint8_t* from, float(&own)[8], float(&other)[8]) {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) own[e] = other[e] = 1.f;
        if (from == nullptr || !mine) return;
        const typename H::eight x = as_eight<H>(*(const uint4*)(from + 2 * d));
        const typename H::eight y = as_eight<H>(*(const uint4*)(from + 16 * partner));
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) own[e] = (float)x[e], other[e] = (float)y[e];
    };
    weights(a.q_weight, qw, qo);
    weights(a.k_weight, kw, ko);

    for (uint32_t row = blockIdx.y * (kThreads >> a.row_power) + at; row - at < rows; row += step) {
        const bool is_q = row < a.heads, is_k = !is_q && row < a.heads + a.kv_heads, there = row < rows;
        const uint32_t head = is_q ? row : is_k ? row - a.heads : row - a.heads - a.kv_heads;
        const uint8_t* from = is_q ? a.q + token * a.q_token + head * a.q_head
                              : is_k ? a.k + token * a.k_token + head * a.k_head
                                     : a.v + token * a.v_token + head * a.v_head;
        const bool wanted = there && mine && (is_q || stored);
        uint4 words = make_uint4(0, 0, 0, 0);
        if (wanted) words = *(const uint4*)(from + 2 * d);
        uint4 result = words;
        if (__any(is_q || is_k)) {
            const typename H::eight x = as_eight<H>(words);
            float sum = 0.f;
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) sum += (float)x[e] * (float)x[e];
            for (uint32_t l = 1; l < lanes; l *= 2) sum += __shfl_xor(sum, l);
            const uint32_t lane = threadIdx.x % 64, other = lane - part + partner;
            uint4 far;
            far.x = __shfl(words.x, other), far.y = __shfl(words.y, other);
            far.z = __shfl(words.z, other), far.w = __shfl(words.w, other);
            const typename H::eight z = as_eight<H>(far);
            const bool normed = (is_q ? a.q_weight : a.k_weight) != nullptr;
            const float by = normed ? 1.f / sqrtf(sum / (float)a.head_dim + a.eps) : 1.f;
            typename H::eight y;
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) {
                const float own = (float)x[e] * by * (is_q ? qw[e] : kw[e]);
                const uint32_t f = e ^ 1;
                const float pair = a.adjacent ? (float)x[f] * by * (is_q ? qw[f] : kw[f])
                                              : (float)z[e] * by * (is_q ? qo[e] : ko[e]);
                y[e] = (typename H::one)(turned ? own * c[e] + pair * s[e] : own);
            }
            if (is_q || is_k) result = as_words<H>(y);
        }
        if (wanted) {
            uint8_t* to = is_q ? a.q_out + token * a.q_out_token + head * a.q_out_head
                          : is_k ? a.k_cache + block * a.kc_block + inside * a.kc_token + head * a.kc_head
                                 : a.v_cache + block * a.vc_block + inside * a.vc_token + head * a.vc_head;
            *(uint4*)(to + 2 * d) = result;
        }
    }
}

struct SummarizeArgs {
    const uint8_t* k;
    const int32_t *blocks, *counts, *entries;
    int8_t* bounds;
    float* scales;
    int64_t k_block, k_token, k_head;  // bytes
    uint32_t n, kv_heads, head_dim, block_tokens, pool, entry_count, row_power;
};

// A wavefront for each block and head: 64 / 2^row_power tokens at a time.
template <class H>
__global__ __launch_bounds__(kThreads) void summarize_kernel(SummarizeArgs a) {
    const uint32_t lane = threadIdx.x % 64;
    const uint64_t task = (uint64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    const uint32_t n = (uint32_t)(task / a.kv_heads), head = (uint32_t)(task - (uint64_t)n * a.kv_heads);
    if (n >= a.n) return;
    const uint32_t block = (uint32_t)a.blocks[n], entry = a.entries == nullptr ? block : (uint32_t)a.entries[n];
    if (block >= a.pool || entry >= a.entry_count) return;
    const int32_t asked = a.counts[n];
    const uint32_t count = asked <= 0 ? 0u : (uint32_t)asked < a.block_tokens ? (uint32_t)asked : a.block_tokens;
    const uint32_t lanes = 1u << a.row_power, part = lane & (lanes - 1), d = 8 * part;
    const bool mine = d < a.head_dim;

    float low[8], high[8];
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) low[e] = INFINITY, high[e] = -INFINITY;
    const uint8_t* from = a.k + block * a.k_block + head * a.k_head + 2 * d;
    if (mine) {
#pragma unroll 4
        for (uint32_t t = lane >> a.row_power; t < count; t += 64 >> a.row_power) {
            const typename H::eight x = as_eight<H>(*(const uint4*)(from + t * a.k_token));
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) {
                const float y = (float)x[e], z = fabsf(y) < INFINITY ? y : 0.f;
                low[e] = fminf(low[e], z), high[e] = fmaxf(high[e], z);
            }
        }
    }
    for (uint32_t l = lanes; l < 64; l *= 2)
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
            low[e] = fminf(low[e], __shfl_xor(low[e], l));
            high[e] = fmaxf(high[e], __shfl_xor(high[e], l));
        }
    float most = 0.f;
    if (mine && count != 0)
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) most = fmaxf(most, fmaxf(fabsf(low[e]), fabsf(high[e])));
    for (uint32_t l = 1; l < lanes; l *= 2) most = fmaxf(most, __shfl_xor(most, l));
    const bool small = !(most >= 1e-30f);
    const float by = small ? 0.f : 127.f / most;
    if (lane < lanes && mine) {
        uint32_t words[4];
#pragma unroll
        for (uint32_t w = 0; w < 4; ++w) {
            words[w] = 0;
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
                const float x = w < 2 ? low[4 * w + e] : high[4 * w - 8 + e];
                const int32_t whole = small ? 0 : (int32_t)rintf(x * by);
                words[w] |= ((uint32_t)whole & 0xFF) << (8 * e);
            }
        }
        int8_t* to = a.bounds + ((uint64_t)entry * a.kv_heads + head) * 2 * a.head_dim + d;
        *(uint2*)to = make_uint2(words[0], words[1]);
        *(uint2*)(to + a.head_dim) = make_uint2(words[2], words[3]);
    }
    if (lane == 0) a.scales[(uint64_t)entry * a.kv_heads + head] = small ? 0.f : most / 127.f;
}

}  // namespace
}  // namespace pgcm_kv_impl

using namespace pgcm_kv_impl;
using pgcm::hip_noted;

extern "C" {
#pragma GCC visibility push(default)

int pgcm_kv_append(const pgcm_kv_cache* cache, const pgcm_kv_append_args* args, void* hip_stream) {
    if (args == nullptr) return PGCM_ERR_ARG;
    if (const int rc = check_cache(cache)) return rc;
    if (args->tokens == 0) return PGCM_OK;
    const uint32_t dim = cache->head_dim;
    if (args->tokens > 0x7FFFFFFFu || args->heads > kMaxHeads || args->heads % cache->kv_heads != 0 ||
        (args->q == nullptr) != (args->heads == 0) || (args->q_out == nullptr) != (args->heads == 0) || args->k == nullptr ||
        args->v == nullptr || args->slots == nullptr || !(args->eps >= 0.f))
        return PGCM_ERR_ARG;
    if (args->rope != nullptr && (args->positions == nullptr || args->rope_dim == 0 || args->rope_dim % 16 != 0 ||
                                  args->rope_dim > dim || args->rope_positions == 0 || args->rope_positions > 0x7FFFFFFFu))
        return PGCM_ERR_ARG;
    if (!aligned(args->q, args->q_token, args->q_head) || !aligned(args->k, args->k_token, args->k_head) ||
        !aligned(args->v, args->v_token, args->v_head) || !aligned(args->q_out, args->q_out_token, args->q_out_head) ||
        !aligned(args->q_weight) || !aligned(args->k_weight) || !aligned(args->rope))
        return PGCM_ERR_ALIGN;
    AppendArgs a{};
    a.q = (const uint8_t*)args->q, a.k = (const uint8_t*)args->k, a.v = (const uint8_t*)args->v;
    a.q_weight = (const uint8_t*)args->q_weight, a.k_weight = (const uint8_t*)args->k_weight;
    a.q_out = (uint8_t*)args->q_out, a.k_cache = (uint8_t*)cache->k, a.v_cache = (uint8_t*)cache->v;
    a.positions = args->positions, a.slots = args->slots, a.rope = args->rope;
    a.q_token = 2 * args->q_token, a.q_head = 2 * args->q_head, a.k_token = 2 * args->k_token, a.k_head = 2 * args->k_head;
    a.v_token = 2 * args->v_token, a.v_head = 2 * args->v_head;
    a.q_out_token = 2 * args->q_out_token, a.q_out_head = 2 * args->q_out_head;
    a.kc_block = 2 * cache->k_block, a.kc_token = 2 * cache->k_token, a.kc_head = 2 * cache->k_head;
    a.vc_block = 2 * cache->v_block, a.vc_token = 2 * cache->v_token, a.vc_head = 2 * cache->v_head;
    a.pool_tokens = (uint64_t)cache->blocks * cache->block_tokens;
    a.heads = args->heads, a.kv_heads = cache->kv_heads, a.head_dim = dim, a.block_tokens = cache->block_tokens;
    a.rope_positions = args->rope_positions, a.rope_dim = args->rope_dim, a.adjacent = args->adjacent;
    a.row_power = row_power_of(dim);
    a.eps = args->eps;
    const uint32_t at_once = kThreads >> a.row_power, passes = (a.heads + 2 * a.kv_heads + at_once - 1) / at_once;
    // a token's rows in one workgroup, or in several where tokens alone would not fill the chip
    uint32_t ways = args->tokens >= 1024 ? 1 : (1024 + args->tokens - 1) / args->tokens;
    if (ways > passes) ways = passes;
    const dim3 grid(args->tokens, ways);
    if (cache->half == PGCM_KV_F16) append_kernel<F16><<<grid, kThreads, 0, (hipStream_t)hip_stream>>>(a);
    else append_kernel<Bf16><<<grid, kThreads, 0, (hipStream_t)hip_stream>>>(a);
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

int pgcm_kv_summarize(const pgcm_kv_cache* cache, uint32_t n, const int32_t* blocks, const int32_t* counts,
                      const int32_t* entries, uint32_t entry_count, int8_t* bounds, float* scales, void* hip_stream) {
    if (const int rc = check_cache(cache)) return rc;
    if (n == 0) return PGCM_OK;
    if (n > 0x7FFFFFFFu || blocks == nullptr || counts == nullptr || entry_count == 0 || entry_count > 0x7FFFFFFFu ||
        bounds == nullptr || scales == nullptr || (uint64_t)n * cache->kv_heads > 0x7FFFFFFFull)
        return PGCM_ERR_ARG;
    if (!aligned(bounds)) return PGCM_ERR_ALIGN;
    SummarizeArgs a{};
    a.k = (const uint8_t*)cache->k;
    a.blocks = blocks, a.counts = counts, a.entries = entries, a.bounds = bounds, a.scales = scales;
    a.k_block = 2 * cache->k_block, a.k_token = 2 * cache->k_token, a.k_head = 2 * cache->k_head;
    a.n = n, a.kv_heads = cache->kv_heads, a.head_dim = cache->head_dim, a.block_tokens = cache->block_tokens;
    a.pool = cache->blocks, a.entry_count = entry_count, a.row_power = row_power_of(cache->head_dim);
    const uint32_t groups = (uint32_t)(((uint64_t)n * a.kv_heads + kThreads / 64 - 1) / (kThreads / 64));
    if (cache->half == PGCM_KV_F16) summarize_kernel<F16><<<groups, kThreads, 0, (hipStream_t)hip_stream>>>(a);
    else summarize_kernel<Bf16><<<groups, kThreads, 0, (hipStream_t)hip_stream>>>(a);
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

#pragma GCC visibility pop
}  // extern "C"
