// New keys and values into a paged cache, and the bounds of its blocks (include/pgcm_kv.h).  Both read and write each
// element once: what bounds them is memory.
#include "pgcm_kv_common.h"

#include <type_traits>

namespace pgcm_kv_impl {
namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kAround = 0x128;  // DPP: eight lanes on in a row of sixteen

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
    float eps, by_dim;  // by_dim: 1 / head_dim
};

// Over the 2^power lanes of a row, so that each has the result.
template <class Of>
__device__ __forceinline__ float over_lanes(float x, uint32_t power, Of of) {
    if (power > 0) x = of(x, from_lane<kPairs>(x));
    if (power > 1) x = of(x, from_lane<kQuads>(x));
    if (power > 2) x = of(x, from_lane<kMirrorEight>(x));
    if (power > 3) x = of(x, from_lane<kMirrorRow>(x));
    if (power > 4) {
        const Two y = of_row_pairs(x);
        x = of(y.a, y.b);
    }
    return x;
}

// One token.  A wavefront takes 64 / 2^row_power of its heads at a step, of queries, keys or values alone; the steps are
// dealt out to wavefronts, and to the blockIdx.y of a token.  A lane has the same channels of each of its heads, so the
// factors of
//   x by w c + y by w' s        (by: of the norm; y, w': the other channel of the pair and its weight; s with its sign)
// are made once for a token, and a head takes five operations a channel.  What they take is asked for before anything is
// waited for, the table's line in pieces of sixteen bytes (word by word, a batch of 300 tokens took twice as long).  8191
// tokens, 40 heads and kv heads of 128 (508 MB): 104 us, 4.9 TB/s, the rate of a large copy; 64 tokens of 32 and 8: 3.8 us, the
// launch and two loads one after the other.
template <class H>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
    const uint32_t token = blockIdx.x, lane = threadIdx.x % 64, lanes = 1u << a.row_power;
    const uint32_t part = lane & (lanes - 1), d = 8 * part, in_step = lane >> a.row_power, heads_at_once = 64u >> a.row_power;
    const bool mine = d < a.head_dim;
    const uint32_t of_q = (a.heads + heads_at_once - 1) / heads_at_once, of_k = (a.kv_heads + heads_at_once - 1) / heads_at_once;
    const uint32_t steps = of_q + 2 * of_k, waves = blockDim.x / 64, stride = waves * gridDim.y;
    uint32_t step = __builtin_amdgcn_readfirstlane(blockIdx.y * waves + threadIdx.x / 64);

    const int64_t slot = a.slots[token];
    const int32_t position = a.rope == nullptr ? 0 : a.positions[token];
    const bool stored = (uint64_t)slot < a.pool_tokens;
    // the lane's head of a step, and whether it is there and wanted
    struct Head {
        uint32_t n;
        bool wanted;
    };
    auto head_of = [&](uint32_t step) {
        const uint32_t first = step < of_q ? 0 : step < of_q + of_k ? of_q : of_q + of_k;
        const uint32_t n = (step - first) * heads_at_once + in_step;
        return Head{n, mine && (step < of_q ? n < a.heads : n < a.kv_heads && stored)};
    };
    auto load = [&](uint32_t step) {
        const Head h = head_of(step);
        const uint8_t* from = step < of_q ? a.q + token * a.q_token + h.n * a.q_head
                              : step < of_q + of_k ? a.k + token * a.k_token + h.n * a.k_head
                                                   : a.v + token * a.v_token + h.n * a.v_head;
        return h.wanted ? *(const uint4*)(from + 2 * d) : make_uint4(0, 0, 0, 0);
    };
    uint4 words = make_uint4(0, 0, 0, 0);
    if (step < steps) words = load(step);      // under way while the factors are made

    const uint32_t half = a.rope_dim / 2;
    const bool turned = a.rope != nullptr && d < a.rope_dim;
    const bool halves = a.rope != nullptr && a.adjacent == 0;
    const uint32_t taken = turned ? ~0u : 0u;  // of a pair's other channel
    uint32_t partner = part;                   // the lane with the other channels of the pairs
    if (halves && turned) partner = d < half ? part + half / 8 : part - half / 8;
    // weights of queries' channels and of keys', and those of the partner's
    uint4 weight[2], far_weight[2];
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
        const uint8_t* from = k == 0 ? a.q_weight : a.k_weight;
        weight[k] = far_weight[k] = make_uint4(0, 0, 0, 0);
        if (from != nullptr && mine) weight[k] = *(const uint4*)(from + 2 * d), far_weight[k] = *(const uint4*)(from + 16 * partner);
    }
    float own[2][8], other[2][8];              // factors of queries and of keys
    {
        const bool known = (uint32_t)position < a.rope_positions;
        float c[8], s[8];
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) c[e] = 1.f, s[e] = 0.f;
        if (turned) {
            // eight pairs in a row, or four (an adjacent pair's channels have the same)
            const float* line = a.rope + (known ? (size_t)position * a.rope_dim : 0) + (a.adjacent ? d / 2 : d < half ? d : d - half);
            const float4 c0 = *(const float4*)line, s0 = *(const float4*)(line + half);
            if (a.adjacent) {
                c[0] = c[1] = c0.x, c[2] = c[3] = c0.y, c[4] = c[5] = c0.z, c[6] = c[7] = c0.w;
                s[1] = s0.x, s[3] = s0.y, s[5] = s0.z, s[7] = s0.w;
                s[0] = -s0.x, s[2] = -s0.y, s[4] = -s0.z, s[6] = -s0.w;
            } else {
                const float4 c1 = *(const float4*)(line + 4), s1 = *(const float4*)(line + half + 4);
                c[0] = c0.x, c[1] = c0.y, c[2] = c0.z, c[3] = c0.w, c[4] = c1.x, c[5] = c1.y, c[6] = c1.z, c[7] = c1.w;
                s[0] = s0.x, s[1] = s0.y, s[2] = s0.z, s[3] = s0.w, s[4] = s1.x, s[5] = s1.y, s[6] = s1.z, s[7] = s1.w;
                if (d < half)
#pragma unroll
                    for (uint32_t e = 0; e < 8; ++e) s[e] = -s[e];
            }
            if (!known)
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) c[e] = s[e] = NAN;
        }
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
            const bool there = (k == 0 ? a.q_weight : a.k_weight) != nullptr;
            const typename H::eight x = as_eight<H>(weight[k]), y = as_eight<H>(far_weight[k]);
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) {
                own[k][e] = (there ? (float)x[e] : 1.f) * c[e];
                other[k][e] = turned ? (there ? (float)(a.adjacent ? x[e ^ 1] : y[e]) : 1.f) * s[e] : 0.f;
            }
        }
    }
    const uint64_t block = stored ? (uint64_t)slot / a.block_tokens : 0;
    const uint32_t inside = stored ? (uint32_t)((uint64_t)slot - block * a.block_tokens) : 0;
    uint8_t* const k_to = a.k_cache + block * a.kc_block + inside * a.kc_token;
    uint8_t* const v_to = a.v_cache + block * a.vc_block + inside * a.vc_token;
    const bool across = halves && a.row_power == 4 && a.rope_dim == 128;   // the partner is eight lanes on, around the row

    while (step < steps) {
        const uint4 now = words;
        const uint32_t this_step = step;
        step += stride;
        if (step < steps) words = load(step);  // under way while this step is worked on
        const Head h = head_of(this_step);
        uint4 result = now;
        const uint32_t k = this_step < of_q ? 0 : 1;
        const bool normed = (k == 0 ? a.q_weight : a.k_weight) != nullptr;
        if (this_step < of_q + of_k && (normed || a.rope != nullptr)) {   // (others are copied)
            const typename H::eight x = as_eight<H>(now);
            float by = 1.f;
            if (normed) {
                float sum = 0.f;
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) sum += (float)x[e] * (float)x[e];
                sum = over_lanes(sum, a.row_power, [](float x, float y) { return x + y; });
                by = __builtin_amdgcn_rsqf(sum * a.by_dim + a.eps);   // (to one unit in the last place)
            }
            uint4 pairs = now;
            if (halves) {
                if (across) {
                    pairs.x = __builtin_amdgcn_update_dpp(0, now.x, kAround, 0xF, 0xF, true);
                    pairs.y = __builtin_amdgcn_update_dpp(0, now.y, kAround, 0xF, 0xF, true);
                    pairs.z = __builtin_amdgcn_update_dpp(0, now.z, kAround, 0xF, 0xF, true);
                    pairs.w = __builtin_amdgcn_update_dpp(0, now.w, kAround, 0xF, 0xF, true);
                } else {
                    const uint32_t at = lane - part + partner;
                    pairs.x = __shfl(now.x, at), pairs.y = __shfl(now.y, at), pairs.z = __shfl(now.z, at), pairs.w = __shfl(now.w, at);
                }
            }
            // (channels that are not rotated take nothing from others, and infinity times nothing is no number)
            pairs.x &= taken, pairs.y &= taken, pairs.z &= taken, pairs.w &= taken;
            const typename H::eight y = as_eight<H>(pairs);
            typename H::eight z;
            auto turn = [&](const float(&c)[8], const float(&s)[8]) {
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) {
                    const float pair = (float)(a.adjacent ? y[e ^ 1] : y[e]);
                    z[e] = (typename H::one)(((float)x[e] * c[e] + pair * s[e]) * by);
                }
            };
            if (k == 0) turn(own[0], other[0]);
            else turn(own[1], other[1]);
            result = as_words<H>(z);
        }
        if (h.wanted) {
            uint8_t* to = this_step < of_q ? a.q_out + token * a.q_out_token + h.n * a.q_out_head
                          : this_step < of_q + of_k ? k_to + h.n * a.kc_head
                                                    : v_to + h.n * a.vc_head;
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
    uint32_t n, kv_heads, head_dim, block_tokens, pool, entry_count, row_power, group_power;
};

typedef short s16x2 __attribute__((ext_vector_type(2)));
// Two halves as whole numbers in their order, and back: an involution.
__device__ __forceinline__ s16x2 in_order(s16x2 x) { return x ^ ((x >> 15) & (s16x2)(short)0x7FFF); }
__device__ __forceinline__ s16x2 as_two(uint32_t x) { return __builtin_bit_cast(s16x2, x); }
__device__ __forceinline__ uint32_t as_word(s16x2 x) { return __builtin_bit_cast(uint32_t, x); }
// x of the lanes whose number differs in 2^n, n < 6
__device__ __forceinline__ uint32_t opposite(uint32_t x, uint32_t n) {
    if (n == 4) {
        const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return y[0] ^ y[1] ^ x;
    }
    if (n == 5) {
        const auto y = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return y[0] ^ y[1] ^ x;
    }
    return __shfl_xor(x, 1u << n);
}

// 2^group_power lanes for each block and head: 2^(group_power - row_power) tokens at a time.  Least and largest values are those
// of the halves as whole numbers in order, two an instruction; whatever is not finite lies at the ends of that order, and if any
// is found there the block is gone through again with zeros in such places.  8192 blocks of 8 heads of 128 (286 MB): 61 us, 4.7
// TB/s, the rate of a large copy; with one token's load at a time 68.  kWhole: all lanes of the wavefront (known when compiled,
// so that the block's numbers are the wavefront's: 61 us and 63).
template <class H, bool kWhole>
__global__ __launch_bounds__(kThreads) void summarize_kernel(SummarizeArgs a) {
    const uint32_t lane = threadIdx.x % 64, group_power = kWhole ? 6 : a.group_power;
    const uint32_t in_workgroup = threadIdx.x >> group_power;
    const uint32_t task = blockIdx.x * (kThreads >> group_power) + (kWhole ? __builtin_amdgcn_readfirstlane(in_workgroup) : in_workgroup);
    const uint32_t n = task / a.kv_heads, head = task - n * a.kv_heads;
    uint32_t block = ~0u, entry = ~0u;
    int32_t asked = 0;
    if (n < a.n) {
        block = (uint32_t)a.blocks[n], entry = a.entries == nullptr ? block : (uint32_t)a.entries[n];
        asked = a.counts[n];
    }
    const bool wanted = block < a.pool && entry < a.entry_count;
    const uint32_t count = !wanted || asked <= 0 ? 0u : (uint32_t)asked < a.block_tokens ? (uint32_t)asked : a.block_tokens;
    const uint32_t lanes = 1u << a.row_power, part = lane & (lanes - 1), d = 8 * part, at_once = 1u << (group_power - a.row_power);
    const uint32_t in_turn = lane >> a.row_power & (at_once - 1);
    const bool mine = d < a.head_dim;
    const uint8_t* from = a.k + (wanted ? block * a.k_block + head * a.k_head : 0) + 2 * d;

    s16x2 low[4], high[4];
    auto walk = [&](auto careful) {
#pragma unroll
        for (uint32_t w = 0; w < 4; ++w) low[w] = (s16x2)(short)0x7FFF, high[w] = (s16x2)(short)0x8000;
        if (!mine) return;
        for (uint32_t t0 = in_turn; t0 < count; t0 += 4 * at_once) {   // four tokens' loads under way together
            uint4 x[4];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) {
                const uint32_t t = t0 + u * at_once;   // (beyond the block's tokens: the first one again)
                x[u] = *(const uint4*)(from + (t < count ? t : t0) * a.k_token);
            }
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) {
                uint32_t words[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
                for (uint32_t w = 0; w < 4; ++w) {
                    if constexpr (decltype(careful)::value) {
                        constexpr uint32_t kInf = H::kInfinity;
                        if ((words[w] & kInf) == kInf) words[w] &= 0xFFFF0000u;
                        if ((words[w] & kInf << 16) == kInf << 16) words[w] &= 0xFFFFu;
                    }
                    const s16x2 k = in_order(as_two(words[w]));
                    low[w] = __builtin_elementwise_min(low[w], k), high[w] = __builtin_elementwise_max(high[w], k);
                }
            }
        }
    };
    walk(std::false_type());
    {
        s16x2 least = low[0], most = high[0];
#pragma unroll
        for (uint32_t w = 0; w < 4; ++w)
            least = __builtin_elementwise_min(least, low[w]), most = __builtin_elementwise_max(most, high[w]);
        const short end = (short)H::kInfinity;
        const bool beyond = mine && in_turn < count && ((most.x >= end) | (most.y >= end) | (least.x <= ~end) | (least.y <= ~end));
        if (__any(beyond)) walk(std::true_type());
    }
    auto value = [](uint32_t word, uint32_t e) {   // of a half
        const uint16_t bits = (uint16_t)(word >> (16 * e));
        return (float)__builtin_bit_cast(typename H::one, bits);
    };
    for (uint32_t l = a.row_power; l < group_power; ++l)
#pragma unroll
        for (uint32_t w = 0; w < 4; ++w) {
            low[w] = __builtin_elementwise_min(low[w], as_two(opposite(as_word(low[w]), l)));
            high[w] = __builtin_elementwise_max(high[w], as_two(opposite(as_word(high[w]), l)));
        }
    uint32_t ends[8];   // the halves themselves
#pragma unroll
    for (uint32_t w = 0; w < 4; ++w) ends[w] = as_word(in_order(low[w])), ends[4 + w] = as_word(in_order(high[w]));
    // |x| is largest at an end; as whole numbers, without the sign, halves are in the order of |x|
    s16x2 size = (s16x2)(short)0;
    if (mine && count != 0)
#pragma unroll
        for (uint32_t w = 0; w < 8; ++w) size = __builtin_elementwise_max(size, as_two(ends[w] & 0x7FFF7FFFu));
    const short larger = size.x > size.y ? size.x : size.y;
    float most = value((uint32_t)(uint16_t)larger, 0);
    most = over_lanes(most, a.row_power, [](float x, float y) { return fmaxf(x, y); });
    const bool small = !(most >= 1e-30f);
    const float by = small ? 0.f : 127.f / most;
    const uint64_t to = (uint64_t)entry * a.kv_heads + head;
    // four numbers a lane at a time: words 0 and 1 of a lane's eight channels are the least values, 2 and 3 the largest
    for (uint32_t w = in_turn; w < 4; w += at_once) {
        uint32_t bytes = 0;
        const uint32_t pair0 = w == 0 ? ends[0] : w == 1 ? ends[2] : w == 2 ? ends[4] : ends[6];
        const uint32_t pair1 = w == 0 ? ends[1] : w == 1 ? ends[3] : w == 2 ? ends[5] : ends[7];
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
            const int32_t whole = small ? 0 : (int32_t)rintf(value(e < 2 ? pair0 : pair1, e % 2) * by);
            bytes |= ((uint32_t)whole & 0xFF) << (8 * e);
        }
        if (mine && wanted) *(uint32_t*)(a.bounds + to * 2 * a.head_dim + (w / 2) * a.head_dim + d + 4 * (w % 2)) = bytes;
    }
    if (part == 0 && in_turn == 0 && wanted) a.scales[to] = small ? 0.f : most / 127.f;
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
    a.eps = args->eps, a.by_dim = 1.f / (float)dim;
    // A token's workgroup: a wavefront for every eight steps, so that the factors are worth making (8000 tokens of six steps: one
    // 19.4 us, two 21.3, four 27.4; 2000 of 24 steps: two 23.8, three 21.3, four 24.1; 8191 of 30: two 108.6, four 103.2), but
    // not under 4096 in all; and several workgroups where tokens alone would not fill the chip.
    const uint32_t at_once = 64u >> a.row_power;
    const uint32_t steps = (a.heads + at_once - 1) / at_once + 2 * ((a.kv_heads + at_once - 1) / at_once);
    constexpr uint32_t kWaves = kThreads / 64;
    uint32_t waves = (steps + 7) / 8;
    if (waves < (4096 + args->tokens - 1) / args->tokens) waves = (4096 + args->tokens - 1) / args->tokens;
    if (waves > kWaves) waves = kWaves;
    const uint32_t passes = (steps + waves - 1) / waves;
    uint32_t ways = args->tokens >= 1024 ? 1 : (1024 + args->tokens - 1) / args->tokens;
    if (ways > passes) ways = passes;
    const uint32_t threads = 64 * waves;
    if (!launchable(args->tokens, threads)) return PGCM_ERR_ARG;
    const dim3 grid(args->tokens, ways);
    if (cache->half == PGCM_KV_F16) append_kernel<F16><<<grid, threads, 0, (hipStream_t)hip_stream>>>(a);
    else append_kernel<Bf16><<<grid, threads, 0, (hipStream_t)hip_stream>>>(a);
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
    // four tokens a lane, if a wavefront's lanes are too many for that (8000 blocks of 16 tokens, 4 heads of 64: 26.4 us with a
    // wavefront each, 13 with half of one)
    a.group_power = a.row_power;
    while (a.group_power < 6 && (4u << (a.group_power - a.row_power)) < a.block_tokens) ++a.group_power;
    const uint64_t threads = (uint64_t)n * a.kv_heads << a.group_power;
    if (!launchable((threads + kThreads - 1) / kThreads, kThreads)) return PGCM_ERR_ARG;
    const uint32_t groups = (uint32_t)((threads + kThreads - 1) / kThreads);
    const hipStream_t stream = (hipStream_t)hip_stream;
    if (cache->half == PGCM_KV_F16) {
        if (a.group_power == 6) summarize_kernel<F16, true><<<groups, kThreads, 0, stream>>>(a);
        else summarize_kernel<F16, false><<<groups, kThreads, 0, stream>>>(a);
    } else {
        if (a.group_power == 6) summarize_kernel<Bf16, true><<<groups, kThreads, 0, stream>>>(a);
        else summarize_kernel<Bf16, false><<<groups, kThreads, 0, stream>>>(a);
    }
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

#pragma GCC visibility pop
}  // extern "C"
