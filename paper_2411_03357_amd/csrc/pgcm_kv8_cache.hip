// KV blocks in 8 bits: new keys and values into them, whole blocks to them and back (include/pgcm_kv8.h).  All read and write
// each element once or twice, the second time from a cache: what bounds them is memory.
//
// A wavefront takes, of a block, the keys or the values of 64 / 2^row_power heads (a "unit"): a lane eight channels of one
// head in every token, so that a token's codes are written in one piece and a head's largest value is found by its lanes alone.
#include "pgcm_kv8_common.h"

namespace pgcm_kv_impl {
namespace {

constexpr uint32_t kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kTogether = 4;    // tokens whose loads are under way together

struct Side8 {   // keys or values of a cache in 8 bits
    uint8_t* at;
    float* scales;
    int64_t block, token, head, scale_block, scale_head;   // bytes; floats
};
struct Append8Args {
    const uint8_t *q, *k, *v, *q_weight, *k_weight;
    uint8_t* q_out;
    const int32_t* positions;
    const int64_t* slots;
    const float* rope;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, q_out_token, q_out_head;  // bytes
    Side8 side[2];
    uint64_t pool_tokens;
    uint32_t tokens, heads, kv_heads, head_dim, block_tokens, rope_positions, rope_dim, adjacent, row_power;
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
__device__ __forceinline__ uint32_t bits_of(float x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ float float_of(uint32_t x) { return __builtin_bit_cast(float, x); }
// |x| of floats in the order of their bits, in which whatever is not finite is largest
__device__ __forceinline__ uint32_t larger(uint32_t most, const float (&x)[8]) {
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
        const uint32_t size = bits_of(x[e]) & 0x7FFFFFFFu;
        most = most > size ? most : size;
    }
    return most;
}
__device__ __forceinline__ uint32_t over_row(uint32_t most, uint32_t power) {
    return bits_of(over_lanes(float_of(most), power, [](float x, float y) {
        return float_of(bits_of(x) > bits_of(y) ? bits_of(x) : bits_of(y));
    }));
}
template <class H>
__device__ __forceinline__ void floats_of(uint4 words, float (&x)[8]) {
    const typename H::eight y = as_eight<H>(words);
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) x[e] = (float)y[e];
}
template <class C>
__device__ __forceinline__ uint2 eight_codes(const float (&x)[8], float by) {
    return make_uint2(C::codes(x[0], x[1], x[2], x[3], by), C::codes(x[4], x[5], x[6], x[7], by));
}
// 2^-e for a scale 2^e, 0 for one that is NaN (the codes are zero then: NaN times 0 is looked for)
__device__ __forceinline__ float inverse(float scale) { return scale == scale ? 1.f / scale : 0.f; }

// Norm and rotation, as a lane needs them: x by w c + y by w' s   (by: of the norm; y, w': the other channel of the pair and its
// weight; s with its sign)
template <class H>
struct Turn {
    uint32_t lane, part, d, half, partner;
    bool mine, turned, halves;
    uint32_t taken;   // of a pair's other channel

    __device__ __forceinline__ Turn(const Append8Args& a) {
        lane = threadIdx.x % 64;
        part = lane & ((1u << a.row_power) - 1);
        d = 8 * part;
        mine = d < a.head_dim;
        half = a.rope_dim / 2;
        turned = a.rope != nullptr && d < a.rope_dim;
        halves = a.rope != nullptr && a.adjacent == 0;
        taken = turned ? ~0u : 0u;
        partner = part;
        if (halves && turned) partner = d < half ? part + half / 8 : part - half / 8;
    }
    struct Weights {
        float own[8], other[8];
    };
    __device__ __forceinline__ Weights weights(const uint8_t* from, bool adjacent) const {
        Weights w;
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) w.own[e] = w.other[e] = 1.f;
        if (from != nullptr && mine) {
            const typename H::eight x = as_eight<H>(*(const uint4*)(from + 2 * d)), y = as_eight<H>(*(const uint4*)(from + 16 * partner));
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) w.own[e] = (float)x[e], w.other[e] = (float)(adjacent ? x[e ^ 1] : y[e]);
        }
        return w;
    }
    struct Line {
        float4 c0, c1, s0, s1;
        bool known;
    };
    // a position's cosines and sines: eight pairs in a row, or four (an adjacent pair's channels have the same)
    __device__ __forceinline__ Line line(const Append8Args& a, int32_t position) const {
        Line l{};
        l.known = (uint32_t)position < a.rope_positions;
        if (turned) {
            const float* at = a.rope + (l.known ? (size_t)position * a.rope_dim : 0) + (a.adjacent ? d / 2 : d < half ? d : d - half);
            l.c0 = *(const float4*)at, l.s0 = *(const float4*)(at + half);
            if (!a.adjacent) l.c1 = *(const float4*)(at + 4), l.s1 = *(const float4*)(at + half + 4);
        }
        return l;
    }
    __device__ __forceinline__ Weights factors(const Append8Args& a, const Line& l, const Weights& w) const {
        Weights f = w;
        if (!turned) {
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) f.other[e] = 0.f;
            return f;
        }
        float c[8], s[8];
        if (a.adjacent) {
            c[0] = c[1] = l.c0.x, c[2] = c[3] = l.c0.y, c[4] = c[5] = l.c0.z, c[6] = c[7] = l.c0.w;
            s[1] = l.s0.x, s[3] = l.s0.y, s[5] = l.s0.z, s[7] = l.s0.w;
            s[0] = -l.s0.x, s[2] = -l.s0.y, s[4] = -l.s0.z, s[6] = -l.s0.w;
        } else {
            c[0] = l.c0.x, c[1] = l.c0.y, c[2] = l.c0.z, c[3] = l.c0.w, c[4] = l.c1.x, c[5] = l.c1.y, c[6] = l.c1.z, c[7] = l.c1.w;
            s[0] = l.s0.x, s[1] = l.s0.y, s[2] = l.s0.z, s[3] = l.s0.w, s[4] = l.s1.x, s[5] = l.s1.y, s[6] = l.s1.z, s[7] = l.s1.w;
            const float sign = d < half ? -1.f : 1.f;
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) s[e] *= sign;
        }
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) f.own[e] *= l.known ? c[e] : NAN, f.other[e] *= l.known ? s[e] : NAN;
        return f;
    }
    __device__ __forceinline__ void apply(const Append8Args& a, uint4 now, const Weights& f, bool normed, float (&z)[8]) const {
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
            const uint32_t at = lane - part + partner;
            pairs.x = __shfl(now.x, at), pairs.y = __shfl(now.y, at), pairs.z = __shfl(now.z, at), pairs.w = __shfl(now.w, at);
        }
        // (channels that are not rotated take nothing from others, and infinity times nothing is no number)
        pairs.x &= taken, pairs.y &= taken, pairs.z &= taken, pairs.w &= taken;
        const typename H::eight y = as_eight<H>(pairs);
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
            const float pair = (float)(a.adjacent ? y[e ^ 1] : y[e]);
            z[e] = ((float)x[e] * f.own[e] + pair * f.other[e]) * by;
        }
    }
};

// A unit's scale for these values, bits of the largest |x| in `most`, `before` what it was (0: none)
template <class C>
__device__ __forceinline__ float scale_for(uint32_t most, float before) {
    if (most >= kNotFinite || !(before == before)) return NAN;
    return fmaxf(power_of_two(C::power(most)), before);
}

// A workgroup (or several: blockIdx.y) a token.  It takes its token's queries, and a share of the units of its run: a block's new
// tokens have as many workgroups as there are tokens, which take its units in turn.
template <class H, class C>
__global__ __launch_bounds__(kThreads) void append8_kernel(Append8Args a) {
    const uint32_t token = blockIdx.x, lane = threadIdx.x % 64;
    const Turn<H> turn(a);
    const uint32_t heads_at_once = 64u >> a.row_power, in_step = lane >> a.row_power;
    const uint32_t of_q = (a.heads + heads_at_once - 1) / heads_at_once, of_kv = (a.kv_heads + heads_at_once - 1) / heads_at_once;
    const uint32_t waves = blockDim.x / 64, stride = waves * gridDim.y;
    uint32_t task = __builtin_amdgcn_readfirstlane(blockIdx.y * waves + threadIdx.x / 64);

    const int64_t slot = a.slots[token];
    const bool stored = (uint64_t)slot < a.pool_tokens;
    const uint64_t block = stored ? (uint64_t)slot / a.block_tokens : 0;
    const uint32_t inside = stored ? (uint32_t)((uint64_t)slot - block * a.block_tokens) : 0;
    // the run: how many tokens before this one, and behind it, have the slots next to its own, in the block
    uint32_t before = 0, behind = 0;
    if (stored) {
        auto count = [&](bool back) {
            const uint32_t room = back ? inside : a.block_tokens - 1 - inside, there = back ? token : a.tokens - 1 - token;
            const uint32_t most = room < there ? room : there;
            for (uint32_t n = 0; n < most; n += 64) {
                const uint32_t j = n + lane + 1;
                const bool next = j <= most && (back ? a.slots[token - j] == slot - j : a.slots[token + j] == slot + j);
                const uint64_t all = __ballot(next);
                if (~all != 0) return n + (uint32_t)__builtin_ctzll(~all);
            }
            return most;
        };
        before = __builtin_amdgcn_readfirstlane(count(true));
        behind = __builtin_amdgcn_readfirstlane(count(false));
    }
    const uint32_t m = before + 1 + behind, units = stored ? 2 * of_kv : 0;
    const uint32_t my_units = units > before ? (units - 1 - before) / m + 1 : 0, tasks = of_q + my_units;

    if (task < of_q) {
        const typename Turn<H>::Weights w =
            turn.factors(a, turn.line(a, a.rope == nullptr ? 0 : a.positions[token]), turn.weights(a.q_weight, a.adjacent != 0));
        for (; task < of_q; task += stride) {
            const uint32_t h = task * heads_at_once + in_step;
            const bool wanted = turn.mine && h < a.heads;
            uint4 words = make_uint4(0, 0, 0, 0);
            if (wanted) words = *(const uint4*)(a.q + token * a.q_token + h * a.q_head + 2 * turn.d);
            if (a.q_weight != nullptr || a.rope != nullptr) {   // (others are copied)
                float z[8];
                turn.apply(a, words, w, a.q_weight != nullptr, z);
                typename H::eight y;
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) y[e] = (typename H::one)z[e];
                words = as_words<H>(y);
            }
            if (wanted) *(uint4*)(a.q_out + token * a.q_out_token + h * a.q_out_head + 2 * turn.d) = words;
        }
    }
    if (task >= tasks) return;
    const typename Turn<H>::Weights k_weights = turn.weights(a.k_weight, a.adjacent != 0);
    const uint32_t first = token - before, first_inside = inside - before;
    for (; task < tasks; task += stride) {
        const uint32_t unit = before + (task - of_q) * m, which = unit / of_kv, h = (unit - which * of_kv) * heads_at_once + in_step;
        const Side8& side = a.side[which];
        const bool is_k = which == 0, there = h < a.kv_heads, wanted = turn.mine && there;
        const uint8_t* from = (is_k ? a.k + h * a.k_head : a.v + h * a.v_head) + 2 * turn.d;
        const int64_t from_token = is_k ? a.k_token : a.v_token;
        uint8_t* const to = side.at + block * side.block + h * side.head + turn.d;
        float* const scale_at = side.scales + block * side.scale_block + h * side.scale_head;
        const float old = first_inside != 0 && there ? *scale_at : 0.f;
        const bool worked = is_k && (a.k_weight != nullptr || a.rope != nullptr);

        float x[kTogether][8];
        auto take = [&](uint32_t j0) {
            uint4 words[kTogether];
            typename Turn<H>::Line lines[kTogether];
#pragma unroll
            for (uint32_t n = 0; n < kTogether; ++n) {
                const uint32_t t = first + (j0 + n < m ? j0 + n : j0);
                words[n] = make_uint4(0, 0, 0, 0);
                if (wanted) words[n] = *(const uint4*)(from + t * from_token);
                if (worked) lines[n] = turn.line(a, a.rope == nullptr ? 0 : a.positions[t]);
            }
#pragma unroll
            for (uint32_t n = 0; n < kTogether; ++n) {
                if (worked) turn.apply(a, words[n], turn.factors(a, lines[n], k_weights), a.k_weight != nullptr, x[n]);
                else floats_of<H>(words[n], x[n]);
            }
        };
        uint32_t most = 0;
        for (uint32_t j = 0; j < m; j += kTogether) {
            take(j);
#pragma unroll
            for (uint32_t n = 0; n < kTogether; ++n) most = larger(most, x[n]);
        }
        if (!wanted) most = 0;   // (lanes beyond the head's channels)
        most = over_row(most, a.row_power);
        const float scale = scale_for<C>(most, old), by = inverse(scale);
        const bool lost = !(scale == scale);
        for (uint32_t j = 0; j < m; j += kTogether) {
            if (m > kTogether) take(j);
#pragma unroll
            for (uint32_t n = 0; n < kTogether; ++n) {
                uint2 codes = eight_codes<C>(x[n], by);
                if (lost) codes = make_uint2(0, 0);
                if (wanted && j + n < m) *(uint2*)(to + (first_inside + j + n) * side.token) = codes;
            }
        }
        if (first_inside != 0) {
            const float ratio = old * by;
            const bool again = wanted && !lost && scale != old;
            if (__any(again)) {
                for (uint32_t t = 0; t < first_inside; t += kTogether) {
                    uint2 words[kTogether];
#pragma unroll
                    for (uint32_t n = 0; n < kTogether; ++n)
                        words[n] = again && t + n < first_inside ? *(const uint2*)(to + (t + n) * side.token) : make_uint2(0, 0);
#pragma unroll
                    for (uint32_t n = 0; n < kTogether; ++n) {
                        float low[4], high[4];
                        C::values(words[n].x, low), C::values(words[n].y, high);
                        const uint2 codes = make_uint2(C::codes(low[0], low[1], low[2], low[3], ratio),
                                                       C::codes(high[0], high[1], high[2], high[3], ratio));
                        if (again && t + n < first_inside) *(uint2*)(to + (t + n) * side.token) = codes;
                    }
                }
            }
        }
        if (turn.part == 0 && there) *scale_at = scale;
    }
}

struct MoveArgs {
    const uint8_t* half_at[2];
    int64_t half_block[2], half_token[2], half_head[2];   // bytes
    Side8 side[2];
    const int32_t *blocks, *counts, *others;
    uint32_t n, kv_heads, head_dim, block_tokens, pool8, pool, row_power, parts;   // parts: of a unit's tokens
};

// The unit of a wavefront
struct Unit {
    uint32_t which, h, d, count, part_of;   // part_of: of the unit's tokens
    bool there, wanted;
    uint8_t *half, *codes;
    int64_t half_token, code_token;
    float* scale;
    uint32_t part;
};
__device__ __forceinline__ bool unit_of(const MoveArgs& a, Unit& u) {
    const uint32_t lane = threadIdx.x % 64, at_once = 64u >> a.row_power, of_kv = (a.kv_heads + at_once - 1) / at_once;
    uint32_t task = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + threadIdx.x / 64);
    const uint32_t groups = 2 * of_kv * a.parts, i = task / groups;
    if (i >= a.n) return false;
    task -= i * groups;
    u.part_of = task / (2 * of_kv);
    task -= u.part_of * 2 * of_kv;
    u.which = task / of_kv;
    u.h = (task - u.which * of_kv) * at_once + (lane >> a.row_power);
    const uint32_t block = (uint32_t)a.blocks[i], other = a.others == nullptr ? block : (uint32_t)a.others[i];
    if (block >= a.pool8 || other >= a.pool) return false;
    const int32_t asked = a.counts == nullptr ? (int32_t)a.block_tokens : a.counts[i];
    u.count = asked <= 0 ? 0u : (uint32_t)asked < a.block_tokens ? (uint32_t)asked : a.block_tokens;
    u.part = lane & ((1u << a.row_power) - 1);
    u.d = 8 * u.part;
    u.there = u.h < a.kv_heads;
    u.wanted = u.there && u.d < a.head_dim;
    const uint32_t h = u.there ? u.h : 0;
    const Side8& s = a.side[u.which];
    u.half = (uint8_t*)a.half_at[u.which] + other * a.half_block[u.which] + h * a.half_head[u.which] + 2 * u.d;
    u.half_token = a.half_token[u.which];
    u.codes = s.at + block * s.block + h * s.head + u.d;
    u.code_token = s.token;
    u.scale = s.scales + block * s.scale_block + h * s.scale_head;
    return true;
}

template <class H, class C>
__global__ __launch_bounds__(kThreads) void store8_kernel(MoveArgs a) {
    Unit u;
    if (!unit_of(a, u)) return;
    uint4 words[kTogether];
    auto take = [&](uint32_t t) {
#pragma unroll
        for (uint32_t n = 0; n < kTogether; ++n) {
            words[n] = make_uint4(0, 0, 0, 0);
            if (u.wanted && t + n < u.count) words[n] = *(const uint4*)(u.half + (t + n) * u.half_token);
        }
    };
    uint32_t most = 0;
    float x[8];
    for (uint32_t t = 0; t < u.count; t += kTogether) {
        take(t);
#pragma unroll
        for (uint32_t n = 0; n < kTogether; ++n) {
            floats_of<H>(words[n], x);
            most = larger(most, x);
        }
    }
    most = over_row(most, a.row_power);
    const float scale = scale_for<C>(most, 0.f), by = inverse(scale);
    const bool lost = !(scale == scale);
    for (uint32_t t = 0; t < u.count; t += kTogether) {
        if (u.count > kTogether) take(t);
#pragma unroll
        for (uint32_t n = 0; n < kTogether; ++n) {
            floats_of<H>(words[n], x);
            uint2 codes = eight_codes<C>(x, by);
            if (lost) codes = make_uint2(0, 0);
            if (u.wanted && t + n < u.count) *(uint2*)(u.codes + (t + n) * u.code_token) = codes;
        }
    }
    if (u.part == 0 && u.there) *u.scale = scale;
}

template <class H, class C>
__global__ __launch_bounds__(kThreads) void load8_kernel(MoveArgs a) {
    Unit u;
    if (!unit_of(a, u)) return;
    const float scale = u.there ? *u.scale : 0.f;
    constexpr float kNearEnd = sizeof(typename H::one) == 2 && H::kInfinity == 0x7C00 ? 64.f : 0x1p118f;   // 448 times that is in range
    const bool near_end = scale > kNearEnd;
    const uint32_t from = u.count * u.part_of / a.parts, to = u.count * (u.part_of + 1) / a.parts;
    for (uint32_t t = from; t < to; t += kTogether) {
        uint2 words[kTogether];
#pragma unroll
        for (uint32_t n = 0; n < kTogether; ++n) {
            words[n] = make_uint2(0, 0);
            if (u.wanted && t + n < to) words[n] = *(const uint2*)(u.codes + (t + n) * u.code_token);
        }
#pragma unroll
        for (uint32_t n = 0; n < kTogether; ++n) {
            float low[4], high[4];
            C::values(words[n].x, low), C::values(words[n].y, high);
            typename H::eight y;
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) y[e] = (typename H::one)(low[e] * scale), y[4 + e] = (typename H::one)(high[e] * scale);
            uint4 out = as_words<H>(y);
            if (near_end) {
                auto within = [](uint32_t w) {   // the infinity of a finite product is the largest number
                    constexpr uint32_t kInf = H::kInfinity;
                    if ((w & 0x7FFFu) == kInf) w -= 1;
                    if ((w & 0x7FFF0000u) == kInf << 16) w -= 1u << 16;
                    return w;
                };
                out = make_uint4(within(out.x), within(out.y), within(out.z), within(out.w));
            }
            if (u.wanted && t + n < to) *(uint4*)(u.half + (t + n) * u.half_token) = out;
        }
    }
}

Side8 side_of(const pgcm_kv8_cache* c, bool values) {
    return values ? Side8{(uint8_t*)c->v, c->v_scales, c->v_block, c->v_token, c->v_head, c->v_scale_block, c->v_scale_head}
                  : Side8{(uint8_t*)c->k, c->k_scales, c->k_block, c->k_token, c->k_head, c->k_scale_block, c->k_scale_head};
}

}  // namespace
}  // namespace pgcm_kv_impl

using namespace pgcm_kv_impl;
using pgcm::hip_noted;

namespace {

int move_args(const pgcm_kv8_cache* c8, const pgcm_kv_cache* c, uint32_t n, const int32_t* blocks, const int32_t* counts,
              const int32_t* others, MoveArgs* a) {
    if (const int rc = check_cache8(c8)) return rc;
    if (const int rc = check_cache(c)) return rc;
    if (c8->half != c->half || c8->block_tokens != c->block_tokens || c8->kv_heads != c->kv_heads || c8->head_dim != c->head_dim)
        return PGCM_ERR_ARG;
    if (n == 0) return PGCM_OK;
    if (n > 0x7FFFFFFFu || blocks == nullptr) return PGCM_ERR_ARG;
    a->half_at[0] = (const uint8_t*)c->k, a->half_at[1] = (const uint8_t*)c->v;
    a->half_block[0] = 2 * c->k_block, a->half_token[0] = 2 * c->k_token, a->half_head[0] = 2 * c->k_head;
    a->half_block[1] = 2 * c->v_block, a->half_token[1] = 2 * c->v_token, a->half_head[1] = 2 * c->v_head;
    a->side[0] = side_of(c8, false), a->side[1] = side_of(c8, true);
    a->blocks = blocks, a->counts = counts, a->others = others;
    a->n = n, a->kv_heads = c->kv_heads, a->head_dim = c->head_dim, a->block_tokens = c->block_tokens;
    a->pool8 = c8->blocks, a->pool = c->blocks, a->row_power = row_power_of(c->head_dim), a->parts = 1;
    return PGCM_OK;
}
// workgroups, or 0: more than a launch holds
uint32_t move_groups(const MoveArgs& a) {
    const uint32_t at_once = 64u >> a.row_power, of_kv = (a.kv_heads + at_once - 1) / at_once;
    const uint64_t waves = (uint64_t)a.n * 2 * of_kv * a.parts, groups = (waves + kWaves - 1) / kWaves;
    return launchable(groups, kThreads) ? (uint32_t)groups : 0;
}

}  // namespace

extern "C" {
#pragma GCC visibility push(default)

int pgcm_kv8_append(const pgcm_kv8_cache* cache, const pgcm_kv_append_args* args, void* hip_stream) {
    if (args == nullptr) return PGCM_ERR_ARG;
    if (const int rc = check_cache8(cache)) return rc;
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
    Append8Args a{};
    a.q = (const uint8_t*)args->q, a.k = (const uint8_t*)args->k, a.v = (const uint8_t*)args->v;
    a.q_weight = (const uint8_t*)args->q_weight, a.k_weight = (const uint8_t*)args->k_weight;
    a.q_out = (uint8_t*)args->q_out;
    a.positions = args->positions, a.slots = args->slots, a.rope = args->rope;
    a.q_token = 2 * args->q_token, a.q_head = 2 * args->q_head, a.k_token = 2 * args->k_token, a.k_head = 2 * args->k_head;
    a.v_token = 2 * args->v_token, a.v_head = 2 * args->v_head;
    a.q_out_token = 2 * args->q_out_token, a.q_out_head = 2 * args->q_out_head;
    a.side[0] = side_of(cache, false), a.side[1] = side_of(cache, true);
    a.pool_tokens = (uint64_t)cache->blocks * cache->block_tokens;
    a.tokens = args->tokens, a.heads = args->heads, a.kv_heads = cache->kv_heads, a.head_dim = dim;
    a.block_tokens = cache->block_tokens;
    a.rope_positions = args->rope_positions, a.rope_dim = args->rope_dim, a.adjacent = args->adjacent;
    a.row_power = row_power_of(dim);
    a.eps = args->eps, a.by_dim = 1.f / (float)dim;
    const uint32_t at_once = 64u >> a.row_power;
    const uint32_t tasks = (a.heads + at_once - 1) / at_once + 2 * ((a.kv_heads + at_once - 1) / at_once);
    const uint32_t passes = (tasks + kWaves - 1) / kWaves;
    uint32_t ways = args->tokens >= 1024 ? 1 : (1024 + args->tokens - 1) / args->tokens;
    if (ways > passes) ways = passes;
    if (!launchable(args->tokens, kThreads)) return PGCM_ERR_ARG;
    const dim3 grid(args->tokens, ways);
    const hipStream_t stream = (hipStream_t)hip_stream;
    const bool f16 = cache->half == PGCM_KV_F16;
    if (cache->code == PGCM_KV8_INT8) {
        if (f16) append8_kernel<F16, Int8><<<grid, kThreads, 0, stream>>>(a);
        else append8_kernel<Bf16, Int8><<<grid, kThreads, 0, stream>>>(a);
    } else {
        if (f16) append8_kernel<F16, E4m3><<<grid, kThreads, 0, stream>>>(a);
        else append8_kernel<Bf16, E4m3><<<grid, kThreads, 0, stream>>>(a);
    }
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

int pgcm_kv8_store(const pgcm_kv8_cache* to, const pgcm_kv_cache* from, uint32_t n, const int32_t* blocks, const int32_t* counts,
                   const int32_t* from_blocks, void* hip_stream) {
    MoveArgs a{};
    if (const int rc = move_args(to, from, n, blocks, counts, from_blocks, &a)) return rc;
    if (n == 0) return PGCM_OK;
    const uint32_t groups = move_groups(a);
    if (groups == 0) return PGCM_ERR_ARG;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const bool f16 = from->half == PGCM_KV_F16;
    if (to->code == PGCM_KV8_INT8) {
        if (f16) store8_kernel<F16, Int8><<<groups, kThreads, 0, stream>>>(a);
        else store8_kernel<Bf16, Int8><<<groups, kThreads, 0, stream>>>(a);
    } else {
        if (f16) store8_kernel<F16, E4m3><<<groups, kThreads, 0, stream>>>(a);
        else store8_kernel<Bf16, E4m3><<<groups, kThreads, 0, stream>>>(a);
    }
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

int pgcm_kv8_load(const pgcm_kv8_cache* from, const pgcm_kv_cache* to, uint32_t n, const int32_t* blocks, const int32_t* counts,
                  const int32_t* to_blocks, void* hip_stream) {
    MoveArgs a{};
    if (const int rc = move_args(from, to, n, blocks, counts, to_blocks, &a)) return rc;
    if (n == 0) return PGCM_OK;
    a.parts = (from->block_tokens + 15) / 16;   // sixteen tokens a wavefront
    const uint32_t groups = move_groups(a);
    if (groups == 0) return PGCM_ERR_ARG;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const bool f16 = to->half == PGCM_KV_F16;
    if (from->code == PGCM_KV8_INT8) {
        if (f16) load8_kernel<F16, Int8><<<groups, kThreads, 0, stream>>>(a);
        else load8_kernel<Bf16, Int8><<<groups, kThreads, 0, stream>>>(a);
    } else {
        if (f16) load8_kernel<F16, E4m3><<<groups, kThreads, 0, stream>>>(a);
        else load8_kernel<Bf16, E4m3><<<groups, kThreads, 0, stream>>>(a);
    }
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

#pragma GCC visibility pop
}  // extern "C"
