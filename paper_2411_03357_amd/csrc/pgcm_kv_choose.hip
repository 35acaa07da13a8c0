// The best blocks of a request for attention, and the least of them for eviction (include/pgcm_kv.h): so many largest
// of a row of keys, equal ones from the front.
#include "pgcm_kv_common.h"

namespace pgcm_kv_impl {
namespace {

constexpr uint32_t kThreads = 512;
constexpr uint32_t kWaves = kThreads / 64;
constexpr uint32_t kLdsKeys = 16384;  // rows of more are read from memory at each look
constexpr uint32_t kBins = 2048;
constexpr uint32_t kNever = 0, kAlways = 0xFFFFFFFFu;  // keys of what cannot be chosen, and of what is chosen before all others

// Whole numbers in the order of numbers; those of -inf and inf are not kNever and kAlways.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);  // (-0 as 0)
    return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

struct ChooseShared {
    uint32_t bins[kBins];
    uint32_t able[kWaves], always[kWaves], least[kWaves], most[kWaves];
    uint32_t bin, in_bin, need;
};

// What is chosen: the keys above `above`, and of those equal to `equal` the first `of_equal`; `count` in all.
struct Chosen {
    uint32_t above, equal, of_equal, count;
};

// The `want` largest of keys key(0) ... key(n - 1).  All threads call it.
template <class Key>
__device__ __forceinline__ Chosen choose(Key key, uint32_t n, uint32_t want, ChooseShared& shared) {
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t able = 0, always = 0, least = kAlways, most = 0;
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t k = key(i);
        able += k != kNever;
        always += k == kAlways;
        if (k != kNever && k != kAlways) {
            least = k < least ? k : least;
            most = k > most ? k : most;
        }
    }
#pragma unroll
    for (uint32_t l = 1; l < 64; l *= 2) {
        able += __shfl_xor(able, l);
        always += __shfl_xor(always, l);
        const uint32_t x = __shfl_xor(least, l), y = __shfl_xor(most, l);
        least = x < least ? x : least;
        most = y > most ? y : most;
    }
    __syncthreads();
    if (lane == 0) shared.able[wave] = able, shared.always[wave] = always, shared.least[wave] = least, shared.most[wave] = most;
    __syncthreads();
    able = always = most = 0, least = kAlways;
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) {
        able += shared.able[w], always += shared.always[w];
        least = shared.least[w] < least ? shared.least[w] : least;
        most = shared.most[w] > most ? shared.most[w] : most;
    }
    if (able <= want) return Chosen{kNever, kNever, 0, able};
    if (want == 0) return Chosen{kAlways, kNever, 0, 0};
    if (always >= want) return Chosen{kAlways, kAlways, want, want};

    // The place of the last one chosen, within [least, most]: counts of equal pieces of that range, from the top, then
    // the piece that it is in; as a rule one or two looks, at most three.
    uint32_t need = want - always;
    while (true) {
        const uint32_t width = most - least;
        const uint32_t bits = width == 0 ? 0 : 32 - __builtin_clz(width);
        const uint32_t shift = bits > 11 ? bits - 11 : 0;
        for (uint32_t b = threadIdx.x; b < kBins; b += kThreads) shared.bins[b] = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
            const uint32_t k = key(i);
            if (k >= least && k <= most) atomicAdd(&shared.bins[(k - least) >> shift], 1u);
        }
        __syncthreads();
        // bins in threads from the top: kBins / kThreads each
        constexpr uint32_t kEach = kBins / kThreads;
        uint32_t mine[kEach], sum = 0;
#pragma unroll
        for (uint32_t e = 0; e < kEach; ++e) {
            mine[e] = shared.bins[kBins - 1 - (threadIdx.x * kEach + e)];
            sum += mine[e];
        }
        const uint32_t upto = scan(sum);
        if (lane == 63) shared.able[wave] = upto;
        __syncthreads();
        uint32_t before = upto - sum;
        for (uint32_t w = 0; w < wave; ++w) before += shared.able[w];
#pragma unroll
        for (uint32_t e = 0; e < kEach; ++e) {
            if (before < need && before + mine[e] >= need) {
                shared.bin = kBins - 1 - (threadIdx.x * kEach + e);
                shared.in_bin = mine[e];
                shared.need = need - before;
            }
            before += mine[e];
        }
        __syncthreads();
        const uint32_t bin = shared.bin, in_bin = shared.in_bin;
        need = shared.need;
        least += bin << shift;
        if (need == in_bin) return Chosen{least - 1, kNever, 0, want};   // (least is no key of kNever: at least 1)
        if (shift == 0) return Chosen{least, least, need, want};
        const uint32_t end = least + ((1u << shift) - 1);
        most = end < most ? end : most;
        __syncthreads();
    }
}

// put(i, place, chosen) for each i, with the places of the chosen ones in the order of i.
template <class Key, class Put>
__device__ __forceinline__ void put_in_order(Key key, uint32_t n, const Chosen& c, ChooseShared& shared, Put put) {
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t each = (n + kThreads - 1) / kThreads * 64;   // a wavefront's part of the row
    const uint32_t from = wave * each < n ? wave * each : n, to = from + each < n ? from + each : n;
    uint32_t above = 0, equal = 0;
    for (uint32_t i = from; i < to; i += 64) {
        const uint32_t k = i + lane < to ? key(i + lane) : kNever;
        above += __builtin_popcountll(__ballot(k > c.above));
        equal += __builtin_popcountll(__ballot(k == c.equal && c.of_equal != 0));
    }
    __syncthreads();
    if (lane == 0) shared.able[wave] = above, shared.always[wave] = equal;
    __syncthreads();
    above = equal = 0;
    for (uint32_t w = 0; w < wave; ++w) above += shared.able[w], equal += shared.always[w];
    const uint64_t before_me = (1ull << lane) - 1;
    for (uint32_t i = from; i < to; i += 64) {
        const bool there = i + lane < to;
        const uint32_t k = there ? key(i + lane) : kNever;
        const uint64_t is_above = __ballot(k > c.above), is_equal = __ballot(k == c.equal && c.of_equal != 0);
        const uint32_t rank = equal + __builtin_popcountll(is_equal & before_me);
        const bool chosen = k > c.above || ((is_equal >> lane & 1) && rank < c.of_equal);
        const uint32_t place = above + __builtin_popcountll(is_above & before_me) + (rank < c.of_equal ? rank : c.of_equal);
        if (there) put(i + lane, place, chosen);
        above += __builtin_popcountll(is_above);
        equal += __builtin_popcountll(is_equal);
    }
}

// ---------------------------------------------------------------------------------------------
struct EvictArgs {
    const float* weights;
    const int32_t *tables, *lens, *evict;
    int32_t *victims, *victim_blocks, *tables_out;
    int64_t table_row, table_out_row;
    uint32_t row_blocks, block_tokens, blocks, most, first, last;
};

__global__ __launch_bounds__(kThreads) void evict_kernel(EvictArgs a) {
    __shared__ ChooseShared shared;
    __shared__ uint32_t keys[kLdsKeys];
    const uint32_t request = blockIdx.x;
    const int32_t len = a.lens[request], asked = a.evict[request];
    const float* weights = a.weights + (size_t)request * a.row_blocks;
    const int32_t* row = a.tables + request * a.table_row;
    int32_t* row_out = a.tables_out == nullptr ? nullptr : a.tables_out + request * a.table_out_row;
    int32_t* victims = a.victims + (size_t)request * a.most;
    int32_t* victim_blocks = a.victim_blocks == nullptr ? nullptr : a.victim_blocks + (size_t)request * a.most;
    uint32_t blocks = len <= 0 ? 0u : ((uint32_t)len - 1) / a.block_tokens + 1;
    if (blocks > a.row_blocks) blocks = a.row_blocks;
    uint32_t want = asked <= 0 ? 0u : (uint32_t)asked;
    if (want > a.most) want = a.most;
    const uint32_t n = blocks > a.last ? blocks - a.last : 0;   // the last ones stay
    auto made = [&](uint32_t i, int32_t block, float w) {
        return i < a.first || (uint32_t)block >= a.blocks ? kNever : w == w ? ~ordered(w) : 1u;
    };
    auto run = [&](auto key) {
        const Chosen c = choose(key, n, want, shared);
        put_in_order(key, n, c, shared, [&](uint32_t i, uint32_t place, bool chosen) {
            if (!chosen) return;
            victims[place] = (int32_t)i;
            if (victim_blocks != nullptr) victim_blocks[place] = row[i];
            if (row_out != nullptr) row_out[i] = -1;   // (a table that is changed in place: the last look at it)
        });
        for (uint32_t i = c.count + threadIdx.x; i < a.most; i += kThreads) {
            victims[i] = -1;
            if (victim_blocks != nullptr) victim_blocks[i] = -1;
        }
    };
    const bool copied = row_out != nullptr && row_out != row;
    // eight of a thread's places at once: their loads are under way together
    for (uint32_t i0 = threadIdx.x; i0 < a.row_blocks; i0 += 8 * kThreads) {
        int32_t block[8];
        float w[8];
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
            const uint32_t i = i0 + e * kThreads;
            block[e] = i < a.row_blocks ? row[i] : -1;
            w[e] = i < n ? weights[i] : 0.f;
        }
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
            const uint32_t i = i0 + e * kThreads;
            if (i < n && i < kLdsKeys) keys[i] = made(i, block[e], w[e]);
            if (i < a.row_blocks && copied) row_out[i] = block[e];
        }
    }
    __syncthreads();
    if (n <= kLdsKeys) run([&](uint32_t i) { return keys[i]; });
    else run([&](uint32_t i) { return made(i, row[i], weights[i]); });
}

// ---------------------------------------------------------------------------------------------
struct SelectArgs {
    const uint8_t* q;
    const int32_t *tables, *lens;
    const int8_t* bounds;
    const float* scales;
    int32_t *selected, *counts;
    uint32_t *arrived, *keys;
    int64_t q_request, q_head;  // bytes
    int64_t table_row;
    uint32_t kv_heads, group, head_dim, block_tokens, row_blocks, entry_count, keep, first, last, part;
};

// Part blockIdx.x of the blocks of a request for one kv head: their keys, and by whichever workgroup is the last of the
// row the choice.  The scores are products on the matrix cores, of 2 head_dim whole numbers: the bounds of sixteen blocks
// with, for each of sixteen query heads, its negative channels (for the least values) and its positive ones.
template <class H, uint32_t kChunks>   // kChunks pieces of 64 numbers
__global__ __launch_bounds__(kThreads) void select_kernel(SelectArgs a) {
    __shared__ ChooseShared shared;
    __shared__ uint32_t keys[kLdsKeys];
    __shared__ __align__(16) int8_t q8[16][64 * kChunks + 16];
    __shared__ float q_scale[16];
    __shared__ uint32_t last;
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, g = lane / 16, i = lane % 16;
    const uint32_t head = blockIdx.y, request = blockIdx.z, list = request * a.kv_heads + head;
    const int32_t len = a.lens[request];
    uint32_t blocks = len <= 0 ? 0u : ((uint32_t)len - 1) / a.block_tokens + 1;
    if (blocks > a.row_blocks) blocks = a.row_blocks;
    const uint32_t parts = blocks == 0 ? 1 : (blocks + a.part - 1) / a.part;
    if (blockIdx.x >= parts) return;
    const uint32_t from = blockIdx.x * a.part, to = from + a.part < blocks ? from + a.part : blocks;
    const int32_t* row = a.tables + request * a.table_row;
    const uint32_t numbers = 2 * a.head_dim;
    const uint64_t entry_bytes = (uint64_t)a.kv_heads * numbers;

    for (uint32_t head0 = 0; head0 < a.group; head0 += 16) {
        const uint32_t heads = a.group - head0 < 16 ? a.group - head0 : 16;
        __syncthreads();
        for (uint32_t h = wave; h < 16; h += kWaves) {
            const uint8_t* from_q = a.q + request * a.q_request + (head * a.group + head0 + h) * a.q_head;
            float x[kChunks / 2], most = 0.f;
#pragma unroll
            for (uint32_t c = 0; c < kChunks / 2; ++c) {
                const uint32_t d = 64 * c + lane;
                x[c] = h < heads && d < a.head_dim ? (float)*(const typename H::one*)(from_q + 2 * d) : 0.f;
                if (!(fabsf(x[c]) < INFINITY)) x[c] = 0.f;
                most = fmaxf(most, fabsf(x[c]));
            }
            most = over_rows_max(row_max(most));
            const bool small = !(most >= 1e-30f);
            const float by = small ? 0.f : 127.f / most;
#pragma unroll
            for (uint32_t c = 0; c < kChunks / 2; ++c) {
                const uint32_t d = 64 * c + lane;
                const int32_t y = small ? 0 : (int32_t)rintf(x[c] * by);
                if (d < a.head_dim) {
                    q8[h][d] = (int8_t)(y < 0 ? y : 0);
                    q8[h][a.head_dim + d] = (int8_t)(y > 0 ? y : 0);
                }
            }
            for (uint32_t d = numbers + lane; d < 64 * kChunks; d += 64) q8[h][d] = 0;
            if (lane == 0) q_scale[h] = small ? 0.f : most / 127.f;
        }
        __syncthreads();
        i32x4 q[kChunks];
#pragma unroll
        for (uint32_t c = 0; c < kChunks; ++c) q[c] = *(const i32x4*)&q8[i][64 * c + 16 * g];
        const float qs = q_scale[i];

        for (uint32_t j0 = from + 64 * wave; j0 < to; j0 += 64 * kWaves) {
            const uint32_t j = j0 + lane;
            uint32_t entry = j < to ? (uint32_t)row[j] : 0;
            if (entry >= a.entry_count) entry = 0;   // not chosen, whatever its score
            const float scale = a.scales[(uint64_t)entry * a.kv_heads + head];
            const int8_t* of_head = a.bounds + (uint64_t)head * numbers;
            i32x4 x[4][kChunks];
#pragma unroll
            for (uint32_t s = 0; s < 4; ++s) {
                const int8_t* at = of_head + __shfl(entry, 16 * s + i) * entry_bytes;
#pragma unroll
                for (uint32_t c = 0; c < kChunks; ++c) {
                    x[s][c] = i32x4{0, 0, 0, 0};
                    if (64 * c + 16 * g < numbers) x[s][c] = *(const i32x4*)(at + 64 * c + 16 * g);
                }
            }
#pragma unroll
            for (uint32_t s = 0; s < 4; ++s) {
                i32x4 sum{0, 0, 0, 0};
#pragma unroll
                for (uint32_t c = 0; c < kChunks; ++c) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[s][c], q[c], sum, 0, 0, 0);
#pragma unroll
                for (uint32_t r = 0; r < 4; ++r) {   // head i, block 4 g + r
                    const uint32_t b = 16 * s + 4 * g + r;
                    float score = (float)sum[r] * __shfl(scale, b) * qs;
                    if (i >= heads) score = -INFINITY;
                    score = row_max(score);
                    if (i == 0 && j0 + b < to) {
                        uint32_t* key = &keys[j0 + b - from];
                        const uint32_t now = ordered(score);
                        *key = head0 == 0 || now > *key ? now : *key;
                    }
                }
            }
        }
    }
    __syncthreads();
    uint32_t* row_keys = a.keys + (size_t)list * a.row_blocks;
    for (uint32_t j = from + threadIdx.x; j < to; j += kThreads) {
        uint32_t key = keys[j - from];
        if ((uint32_t)row[j] >= a.entry_count) key = kNever;
        else if (j < a.first || blocks - j <= a.last) key = kAlways;
        if (parts == 1) keys[j] = key;
        else put_shared(row_keys + j, key);
    }
    int32_t* selected = a.selected + (size_t)list * a.keep;
    auto run = [&](auto key) {
        const Chosen c = choose(key, blocks, a.keep, shared);
        put_in_order(key, blocks, c, shared, [&](uint32_t j, uint32_t place, bool chosen) {
            if (chosen) selected[place] = (int32_t)j;
        });
        for (uint32_t n = c.count + threadIdx.x; n < a.keep; n += kThreads) selected[n] = -1;
        if (threadIdx.x == 0 && a.counts != nullptr) a.counts[list] = (int32_t)c.count;
    };
    if (parts > 1 && !last_to_arrive(a.arrived + list, parts, &last)) return;
    if (blocks <= kLdsKeys) {
        if (parts > 1)
            for (uint32_t j0 = threadIdx.x; j0 < blocks; j0 += 8 * kThreads) {   // eight loads under way together
                uint32_t k[8];
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) k[e] = j0 + e * kThreads < blocks ? get_shared(row_keys + j0 + e * kThreads) : 0;
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e)
                    if (j0 + e * kThreads < blocks) keys[j0 + e * kThreads] = k[e];
            }
        __syncthreads();
        run([&](uint32_t j) { return keys[j]; });
    } else {
        run([&](uint32_t j) { return get_shared(row_keys + j); });
    }
}

template <class H>
void launch(const SelectArgs& a, dim3 grid, hipStream_t stream) {
    if (a.head_dim <= 64) select_kernel<H, 2><<<grid, kThreads, 0, stream>>>(a);
    else if (a.head_dim <= 128) select_kernel<H, 4><<<grid, kThreads, 0, stream>>>(a);
    else select_kernel<H, 8><<<grid, kThreads, 0, stream>>>(a);
}

}  // namespace
}  // namespace pgcm_kv_impl

using namespace pgcm_kv_impl;
using pgcm::hip_noted;

extern "C" {
#pragma GCC visibility push(default)

int pgcm_kv_select(pgcm_kv_t* kv, const pgcm_kv_select_args* args, void* hip_stream) {
    if (kv == nullptr || args == nullptr || args->half > PGCM_KV_BF16) return PGCM_ERR_ARG;
    if (const int rc = check_sizes(args->requests, args->heads, args->kv_heads, args->head_dim, args->block_tokens,
                                   args->row_blocks))
        return rc;
    if (args->requests == 0) return PGCM_OK;
    if (args->q == nullptr || args->lens == nullptr || args->bounds == nullptr || args->scales == nullptr ||
        args->selected == nullptr || args->keep == 0 || args->keep > 0x7FFFFFFFu || args->entry_count == 0 ||
        args->entry_count > 0x7FFFFFFFu || (args->tables == nullptr && args->row_blocks != 0) || args->requests > 65535 ||
        (uint64_t)args->requests * args->kv_heads > 0x7FFFFFFFull)
        return PGCM_ERR_ARG;
    if (!aligned(args->q, args->q_request, args->q_head) || !aligned(args->bounds)) return PGCM_ERR_ALIGN;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const Room room = select_room(args->requests, args->kv_heads, args->row_blocks);
    if (const int rc = kv_ensure(kv, room.counters, room.scratch, stream)) return rc;
    SelectArgs a{};
    a.q = (const uint8_t*)args->q;
    a.tables = args->tables, a.lens = args->lens, a.bounds = args->bounds, a.scales = args->scales;
    a.selected = args->selected, a.counts = args->counts;
    a.arrived = (uint32_t*)kv->counters.at, a.keys = (uint32_t*)kv->scratch.at;
    a.q_request = 2 * args->q_request, a.q_head = 2 * args->q_head, a.table_row = args->table_row;
    a.kv_heads = args->kv_heads, a.group = args->heads / args->kv_heads, a.head_dim = args->head_dim;
    a.block_tokens = args->block_tokens, a.row_blocks = args->row_blocks, a.entry_count = args->entry_count;
    a.keep = args->keep, a.first = args->first, a.last = args->last;
    // a row in one workgroup, or in several where rows alone would not fill the chip; of whole steps of 512 blocks
    const uint64_t lists = (uint64_t)args->requests * args->kv_heads;
    const uint32_t steps = (args->row_blocks + 64 * kWaves - 1) / (64 * kWaves);
    uint32_t ways = lists >= 512 ? 1 : (uint32_t)((512 + lists - 1) / lists);
    if (ways > steps) ways = steps;
    if (ways == 0) ways = 1;
    uint32_t part = (steps + ways - 1) / ways * 64 * kWaves;
    if (part > kLdsKeys) part = kLdsKeys;
    if (part == 0) part = 64 * kWaves;
    a.part = part;
    const uint32_t parts = args->row_blocks == 0 ? 1 : (args->row_blocks + part - 1) / part;
    const dim3 grid(parts, args->kv_heads, args->requests);
    if (args->half == PGCM_KV_F16) launch<F16>(a, grid, stream);
    else launch<Bf16>(a, grid, stream);
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

int pgcm_kv_evict(const pgcm_kv_evict_args* args, void* hip_stream) {
    if (args == nullptr) return PGCM_ERR_ARG;
    if (args->block_tokens == 0 || args->block_tokens % kPiece != 0 || args->block_tokens > 4096 ||
        (uint64_t)args->row_blocks * args->block_tokens > 0x7FFFFFFFull || args->blocks > 0x7FFFFFFFu ||
        args->most > 0x7FFFFFFFu || args->requests > 0x7FFFFFFFu)
        return PGCM_ERR_ARG;
    if (args->requests == 0) return PGCM_OK;
    if (args->lens == nullptr || args->evict == nullptr || (args->victims == nullptr && args->most != 0) ||
        ((args->weights == nullptr || args->tables == nullptr) && args->row_blocks != 0))
        return PGCM_ERR_ARG;
    EvictArgs a{};
    a.weights = args->weights, a.tables = args->tables, a.lens = args->lens, a.evict = args->evict;
    a.victims = args->victims, a.victim_blocks = args->victim_blocks, a.tables_out = args->tables_out;
    a.table_row = args->table_row, a.table_out_row = args->table_out_row;
    a.row_blocks = args->row_blocks, a.block_tokens = args->block_tokens, a.blocks = args->blocks;
    a.most = args->most, a.first = args->first, a.last = args->last;
    evict_kernel<<<args->requests, kThreads, 0, (hipStream_t)hip_stream>>>(a);
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

#pragma GCC visibility pop
}  // extern "C"
