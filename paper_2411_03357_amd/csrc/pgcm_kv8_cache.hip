// KV blocks in 8 bits: new keys and values into them, whole blocks to them and back (include/pgcm_kv8.h).  What bounds all is
// memory.  2048 blocks of 16 tokens and 40 heads of 128 (1.0 GB each way): stored in 217 us, 4.6 TB/s, read back in 182, 5.5; a
// prompt of 8191 tokens, 40 heads, 40 kv heads (420 MB): appended in 98 us, 4.3 TB/s; 64 tokens of 32 and 8 heads: 5.7 us, of
// which instructions are most, that its launch has to fetch.
//
// Store and load: a wavefront takes, of a block, the keys or the values of 64 / 2^row_power heads (a "unit"): a lane eight channels
// of one head in every token, so that a token's codes are written in one piece and a head's largest value is found by its lanes alone.
#include "pgcm_kv8_common.h"

namespace pgcm_kv_impl {
namespace {

constexpr uint32_t kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kRowsHeld = 16;   // a unit's tokens in registers; of longer ones, so many at a time, twice
constexpr int64_t kMostAppendStride = 1 << 23;
constexpr uint32_t kFewUnits = 1024;
constexpr uint32_t kTogether = 4;    // tokens whose loads are under way together
constexpr uint32_t kStepsAtOnce = 3; // of queries

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
    uint32_t kv_ways, spread;   // workgroups that share a window's keys and values; windows that a block may have
    float eps, by_dim;  // by_dim: 1 / head_dim
    double by_block;    // 1 / block_tokens
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
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 as_two(uint32_t x) { return __builtin_bit_cast(u16x2, x); }
// |x| of halves in the order of their bits
__device__ __forceinline__ u16x2 larger(u16x2 most, uint4 x) {
    const uint32_t words[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (uint32_t n = 0; n < 4; ++n) most = __builtin_elementwise_max(most, as_two(words[n] & 0x7FFF7FFFu));
    return most;
}
// the larger one's as a float's
template <class H>
__device__ __forceinline__ uint32_t as_float_bits(u16x2 most) {
    const uint16_t x = most.x > most.y ? most.x : most.y;
    return bits_of((float)__builtin_bit_cast(typename H::one, x));
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
    // a weight's own channels and the partner's
    struct Raw {
        uint4 own, other;
    };
    __device__ __forceinline__ Raw raw_weights(const uint8_t* from) const {
        Raw r{make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        if (from != nullptr && mine) r.own = *(const uint4*)(from + 2 * d), r.other = *(const uint4*)(from + 16 * partner);
        return r;
    }
    static __device__ __forceinline__ Weights weights(const Raw& raw, bool there, bool adjacent) {
        Weights w;
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) w.own[e] = w.other[e] = 1.f;
        if (there) {
            const typename H::eight x = as_eight<H>(raw.own), y = as_eight<H>(raw.other);
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
    // z: but for the norm's factor, which is returned
    __device__ __forceinline__ float apply(const Append8Args& a, uint4 now, const Weights& f, bool normed, float (&z)[8]) const {
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
            z[e] = (float)x[e] * f.own[e] + pair * f.other[e];
        }
        return by;
    }
};

// The scale for these values, as bits like all here: `most` of the largest |x|, `before` of what the scale was (0: none).  Scales
// are not below zero, so they are in the order of their bits, and NaN stays.
template <class C>
__device__ __forceinline__ uint32_t scale_for(uint32_t most, uint32_t before) {
    const int32_t needed = most >= kNotFinite ? (int32_t)0x7FC00000 : (C::power(most) + 127) << 23;
    return (uint32_t)(needed > (int32_t)before ? needed : (int32_t)before);
}
// 1 / scale, exactly for the powers of two that this library writes; for NaN anything, and the codes are to be zero
__device__ __forceinline__ float inverse(uint32_t scale) {
    if (__builtin_expect((scale & 0x7FFFFFu) != 0 || scale >= 0x7E800000u, false)) return 1.f / float_of(scale);
    return float_of(0x7F000000u - scale);
}
__device__ __forceinline__ bool is_lost(uint32_t scale) { return scale > kNotFinite; }

// Where a unit's codes go, lane by lane
struct To {
    uint8_t* at;       // of the first token
    int64_t token;
    bool wanted;       // the lane has channels of a head
};
// A unit of halves, m tokens from `from` on: their codes, and the scale's bits
// join: of the largest values of those that share it
template <class H, class C, class Join>
__device__ __forceinline__ uint32_t convert_unit(const uint8_t* from, int64_t from_token, uint32_t m, const To& to, uint32_t row_power,
                                                 Join join) {
    uint4 held[kRowsHeld];
    auto take = [&](uint32_t j0) {
#pragma unroll
        for (uint32_t n = 0; n < kRowsHeld; ++n) {
            if (n % kTogether == 0 && j0 + n >= m) break;   // (the same for all lanes)
            held[n] = make_uint4(0, 0, 0, 0);
            if (to.wanted && j0 + n < m) held[n] = *(const uint4*)(from + (j0 + n) * from_token);
        }
    };
    u16x2 largest = (u16x2)(unsigned short)0;
    for (uint32_t j0 = 0; j0 < m; j0 += kRowsHeld) {
        take(j0);
#pragma unroll
        for (uint32_t n = 0; n < kRowsHeld; ++n) {
            if (n % kTogether == 0 && j0 + n >= m) break;
            largest = larger(largest, held[n]);
        }
    }
    const uint32_t scale = scale_for<C>(join(over_row(as_float_bits<H>(largest), row_power)), 0);
    const float by = float_of(0x7F000000u - scale);   // (a power of two, or NaN)
    const bool lost = is_lost(scale);
    for (uint32_t j0 = 0; j0 < m; j0 += kRowsHeld) {
        if (m > kRowsHeld) take(j0);
#pragma unroll
        for (uint32_t n = 0; n < kRowsHeld; ++n) {
            if (n % kTogether == 0 && j0 + n >= m) break;
            float x[8];
            floats_of<H>(held[n], x);
            uint2 codes = eight_codes<C>(x, by);
            if (lost) codes = make_uint2(0, 0);
            if (to.wanted && j0 + n < m) *(uint2*)(to.at + (j0 + n) * to.token) = codes;
        }
    }
    return scale;
}

// Of floor(x / by) and the rest, x below 2^52
struct Split {
    uint64_t whole;
    uint32_t rest;
};
__device__ __forceinline__ Split split_by(uint64_t x, uint32_t by, double one_by) {   // one_by: 1 / by
    uint64_t q = (uint64_t)((double)x * one_by);   // off by one at most
    int64_t r = (int64_t)(x - q * by);
    if (r < 0) r += by, --q;
    if (r >= (int64_t)by) r -= by, ++q;
    return Split{q, (uint32_t)r};
}

// The kernel's arguments, its only ones, read where they are used: kept in scalar registers from the start on, most went to lanes of
// vector registers and back (64 tokens: 13.1 us with their read-back instead of 11.3).
typedef const Append8Args __attribute__((address_space(4))) Constant;
__device__ __forceinline__ const Append8Args& late_args() {
    Constant* at = (Constant*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(const Append8Args*)at;
}

// Keys and values of a run, m tokens from `first` on, to `block` from place `inside` on: the workgroup's share of the run's sides
// (keys of head 0, 1, ..., then values of head 0, 1, ...), [from, to), a wavefront one at a time.  A lane's rows are tokens side by
// side, kHeld times as many held in registers (a "chunk"): so a side's largest value is found in the wavefront.  The factors that
// norm and rotation multiply a chunk's tokens with are made once for all heads, in LDS.  Runs of several chunks are taken twice, for
// their largest values and for their codes.
constexpr uint32_t kSidesAtOnce = 64;    // of a wavefront, whose largest values are kept over a run
template <uint32_t kHeld>
struct AppendShared {
    float4 factors[kHeld][4][64];        // of a lane's row: own, then other
    uint32_t largest[kWaves][kSidesAtOnce];
};
template <class H, class C, uint32_t kHeld>
__device__ __forceinline__ void append_run(const Turn<H>& turn, AppendShared<kHeld>& shared, uint32_t first,
                                           uint32_t m, uint64_t block, uint32_t inside, uint32_t from, uint32_t to,
                                           const typename Turn<H>::Raw& raw, int32_t near_position, uint32_t near_from) {
    const Append8Args& a = late_args();
    const uint32_t lane = turn.lane, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t rows = 64u >> a.row_power, in_step = lane >> a.row_power, chunk = kHeld * rows;
    const bool worked = a.k_weight != nullptr || a.rope != nullptr, normed = a.k_weight != nullptr;
    const bool once = m <= chunk;
    for (uint32_t group = from; group < to; group += kSidesAtOnce * kWaves) {
        // twice: the largest values alone, then the codes
        for (uint32_t x = once ? m : 0; x < 2 * m; x = x < m && x + chunk > m ? m : x + chunk) {
            const bool writes = x >= m;
            const uint32_t j0 = once ? 0 : writes ? x - m : x, left = m - j0;
            uint4 rows_of[kHeld];
            float old_at = 0.f;   // the scale that was there
            auto take = [&](uint32_t n_side) {
                const bool is_v = n_side >= a.kv_heads;
                const uint32_t h = is_v ? n_side - a.kv_heads : n_side;
                const Append8Args& a = late_args();
                const Side8& side = a.side[is_v];
                // (where the lane's channels lie from a step's first token on: in 32 bits)
                const int64_t stride = is_v ? a.v_token : a.k_token;
                const uint32_t off = in_step * (uint32_t)stride + 2 * turn.d;
                const uint8_t* at = (is_v ? a.v + h * a.v_head : a.k + h * a.k_head) + (first + j0) * stride;
#pragma unroll
                for (uint32_t n = 0; n < kHeld; ++n) {
                    rows_of[n] = make_uint4(0, 0, 0, 0);
                    if (n * rows < left && turn.mine && n * rows + in_step < left) rows_of[n] = *(const uint4*)(at + off);
                    at += rows * stride;
                }
                if (writes && inside != 0) old_at = side.scales[block * side.scale_block + h * side.scale_head];
            };
            if (group + wave < to) take(group + wave);     // under way while the factors are made
            if (worked && group < a.kv_heads) {
                __syncthreads();   // (all have left those of before)
                for (uint32_t n = wave; n < kHeld && n * rows < left; n += kWaves) {
                    const uint32_t j = n * rows + in_step, t = first + j0 + j;
                    int32_t position = __shfl(near_position, t - near_from);
                    if (t - near_from >= 64) position = a.rope != nullptr && j < left ? a.positions[t] : 0;
                    const typename Turn<H>::Line line = turn.line(a, position);
                    const typename Turn<H>::Weights f = turn.factors(a, line, turn.weights(raw, normed, a.adjacent != 0));
                    shared.factors[n][0][lane] = make_float4(f.own[0], f.own[1], f.own[2], f.own[3]);
                    shared.factors[n][1][lane] = make_float4(f.own[4], f.own[5], f.own[6], f.own[7]);
                    shared.factors[n][2][lane] = make_float4(f.other[0], f.other[1], f.other[2], f.other[3]);
                    shared.factors[n][3][lane] = make_float4(f.other[4], f.other[5], f.other[6], f.other[7]);
                }
                __syncthreads();
            }
            for (uint32_t i = 0; i < kSidesAtOnce; ++i) {
                const uint32_t n_side = group + i * kWaves + wave;
                if (n_side >= to) break;
                if (i != 0) take(n_side);
                const bool is_v = n_side >= a.kv_heads, turned = worked && !is_v;
                float z[kHeld][8], by[kHeld];
                uint32_t most = 0;
#pragma unroll
                for (uint32_t n = 0; n < kHeld; ++n) {
                    by[n] = 1.f;
                    if (n * rows >= left) continue;   // (the same for all lanes)
                    if (turned) {
                        const float4 f0 = shared.factors[n][0][lane], f1 = shared.factors[n][1][lane];
                        const float4 f2 = shared.factors[n][2][lane], f3 = shared.factors[n][3][lane];
                        const typename Turn<H>::Weights f{{f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w},
                                                          {f2.x, f2.y, f2.z, f2.w, f3.x, f3.y, f3.z, f3.w}};
                        by[n] = turn.apply(a, rows_of[n], f, normed, z[n]);
                    } else {
                        floats_of<H>(rows_of[n], z[n]);
                    }
                    const uint32_t of_row = bits_of(float_of(larger(0, z[n])) * by[n]) & 0x7FFFFFFFu;
                    if (turn.mine && n * rows + in_step < left && of_row > most) most = of_row;
                }
                most = over_wave(most, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
                if (!once) {
                    uint32_t* const kept = &shared.largest[wave][i];   // (the wavefront's own)
                    if (!writes) *kept = j0 != 0 && *kept > most ? *kept : most;
                    else most = *kept;
                }
                if (!writes) continue;
                const uint32_t h = is_v ? n_side - a.kv_heads : n_side;
                const Append8Args& a = late_args();
                const Side8& side = a.side[is_v];
                const uint32_t old = __builtin_amdgcn_readfirstlane(bits_of(old_at));
                const uint32_t scale = scale_for<C>(__builtin_amdgcn_readfirstlane(most), old);
                const float inv = inverse(scale);
                const bool lost = is_lost(scale);
                const uint32_t off = in_step * (uint32_t)side.token + turn.d;
                uint8_t* const at = side.at + block * side.block + h * side.head;
#pragma unroll
                for (uint32_t n = 0; n < kHeld; ++n) {
                    if (n * rows >= left) continue;
                    uint2 codes = eight_codes<C>(z[n], by[n] * inv);
                    if (lost) codes = make_uint2(0, 0);
                    if (turn.mine && n * rows + in_step < left) *(uint2*)(at + (inside + j0 + n * rows) * side.token + off) = codes;
                }
                // with the first chunk: the codes that are there to the new scale
                if (j0 == 0 && inside != 0 && !lost && scale != old) {
                    const float ratio = float_of(old) * inv;
                    for (uint32_t t = 0; t < inside; t += kTogether * rows) {
                        uint2 words[kTogether];
#pragma unroll
                        for (uint32_t n = 0; n < kTogether; ++n) {
                            words[n] = make_uint2(0, 0);
                            if (turn.mine && t + n * rows + in_step < inside)
                                words[n] = *(const uint2*)(at + (t + n * rows) * side.token + off);
                        }
#pragma unroll
                        for (uint32_t n = 0; n < kTogether; ++n) {
                            float low[4], high[4];
                            C::values(words[n].x, low), C::values(words[n].y, high);
                            const uint2 codes = make_uint2(C::codes(low[0], low[1], low[2], low[3], ratio),
                                                           C::codes(high[0], high[1], high[2], high[3], ratio));
                            if (turn.mine && t + n * rows + in_step < inside)
                                *(uint2*)(at + (t + n * rows) * side.token + off) = codes;
                        }
                    }
                }
                // ... and the scale with the last, as each reads what it was
                if (left <= chunk && lane == 0) side.scales[block * side.scale_block + h * side.scale_head] = float_of(scale);
            }
        }
    }
}

// The largest value of a block's head has to be known before its first code: so a run is read once and held (with a row of the
// lanes for each head instead of each token, as the append of halves has them, sixteen tokens' factors were made for every four
// heads: 142 us instead of 103 for the prompt).
//
// The runs that begin in a window of tokens are taken by its kv_ways workgroups, whole, their sides in equal shares; the window's
// queries by the workgroups of blockIdx.y >= kv_ways, a token and some of its heads a wavefront.
constexpr uint32_t kWindow = 16;
// Four workgroups a compute unit (three: a prompt of 8191 tokens of 8 kv heads and its read-back in 47 us instead of 45).
template <class H, class C, uint32_t kHeld>
__global__ __launch_bounds__(kThreads, kHeld == 4 ? 4 : 2) void append8_kernel(Append8Args a) {
    __shared__ AppendShared<kHeld> shared;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    // windows a block apart follow each other, so that those in which a prompt's runs begin are spread over all XCDs
    const uint32_t apart = gridDim.x / a.spread, window = (blockIdx.x % apart * a.spread + blockIdx.x / apart) * kWindow;
    const Turn<H> turn(a);
    const uint32_t rows = 64u >> a.row_power, in_step = lane >> a.row_power;

    if (blockIdx.y >= a.kv_ways) {
        // a wavefront a token and some of its steps
        const uint32_t turns = (blockIdx.y - a.kv_ways) * kWaves + wave, token = window + turns % kWindow;
        const uint32_t ways = (gridDim.y - a.kv_ways) * kWaves / kWindow;
        const uint32_t of_q = (a.heads + rows - 1) / rows;
        uint32_t task = turns / kWindow;
        if (token >= a.tokens || task >= of_q || task >= ways) return;
        uint4 words[kStepsAtOnce];
        auto take = [&](uint32_t first) {
#pragma unroll
            for (uint32_t n = 0; n < kStepsAtOnce; ++n) {
                const uint32_t h = (first + n * ways) * rows + in_step;
                words[n] = make_uint4(0, 0, 0, 0);
                if (turn.mine && h < a.heads) words[n] = *(const uint4*)(a.q + token * a.q_token + h * a.q_head + 2 * turn.d);
            }
        };
        take(task);
        const typename Turn<H>::Raw raw = turn.raw_weights(a.q_weight);
        const typename Turn<H>::Weights w = turn.factors(a, turn.line(a, a.rope == nullptr ? 0 : constant(a.positions, token)),
                                                         turn.weights(raw, a.q_weight != nullptr, a.adjacent != 0));
        for (; task < of_q; task += kStepsAtOnce * ways) {
            uint4 now[kStepsAtOnce];
#pragma unroll
            for (uint32_t n = 0; n < kStepsAtOnce; ++n) now[n] = words[n];
            if (task + kStepsAtOnce * ways < of_q) take(task + kStepsAtOnce * ways);   // under way while these are worked on
#pragma unroll
            for (uint32_t n = 0; n < kStepsAtOnce; ++n) {
                if (task + n * ways >= of_q) break;
                const uint32_t h = (task + n * ways) * rows + in_step;
                if (a.q_weight != nullptr || a.rope != nullptr) {   // (others are copied)
                    float z[8];
                    const float by = turn.apply(a, now[n], w, a.q_weight != nullptr, z);
                    typename H::eight y;
#pragma unroll
                    for (uint32_t e = 0; e < 8; ++e) y[e] = (typename H::one)(z[e] * by);
                    now[n] = as_words<H>(y);
                }
                if (turn.mine && h < a.heads) *(uint4*)(a.q_out + token * a.q_out_token + h * a.q_out_head + 2 * turn.d) = now[n];
            }
        }
        return;
    }

    // Where runs begin: lane l looks at token window - 1 + l.
    auto slot_at = [&](uint32_t t) { return t < a.tokens ? a.slots[t] : (int64_t)-1; };
    auto begins = [&](uint32_t t, int64_t slot, int64_t slot_before, uint32_t inside) {   // ... or nothing does
        return t >= a.tokens || t == 0 || (uint64_t)slot >= a.pool_tokens || slot != slot_before + 1 || inside == 0;
    };
    const int64_t near = window + lane >= 1 ? slot_at(window + lane - 1) : -1;
    const Split near_place = split_by((uint64_t)near < a.pool_tokens ? (uint64_t)near : 0, a.block_tokens, a.by_block);
    const uint64_t marks = __ballot(begins(window + lane - 1, near, __shfl_up(near, 1), near_place.rest)) & ~1ull;
    // ... and its position; what is asked for here is there when the runs are known
    const uint32_t near_from = window - 1;
    const int32_t near_position = a.rope != nullptr && near_from + lane < a.tokens ? a.positions[near_from + lane] : 0;
    const typename Turn<H>::Raw raw = turn.raw_weights(a.k_weight);
    // bit i: token window + i begins a run that is stored
    const uint64_t in_pool = __ballot((uint64_t)near < a.pool_tokens && window + lane - 1 < a.tokens);
    uint64_t in_window = (marks & in_pool) >> 1 & ((1ull << kWindow) - 1);
    const uint32_t tasks = (uint32_t)__builtin_popcountll(in_window) * 2 * a.kv_heads;   // sides of all runs
    const uint32_t share = (tasks + a.kv_ways - 1) / a.kv_ways, from = share * blockIdx.y;
    const uint32_t to = from + share < tasks ? from + share : tasks;
    if (from >= tasks) return;
    for (uint32_t task = 0; in_window != 0 && task < to; in_window &= in_window - 1, task += 2 * a.kv_heads) {
        if (task + 2 * a.kv_heads <= from) continue;
        const uint32_t at = __builtin_ctzll(in_window), first = window + at;
        uint32_t m = 0;
        if (const uint64_t later = marks >> 1 & ~((2ull << at) - 1); later != 0) {
            m = __builtin_ctzll(later) - at;
        } else {
            for (uint32_t t = window + 63; m == 0; t += 64) {
                const int64_t slot = slot_at(t + lane);
                const uint32_t rest = split_by((uint64_t)slot < a.pool_tokens ? (uint64_t)slot : 0, a.block_tokens, a.by_block).rest;
                const uint64_t next = __ballot(begins(t + lane, slot, slot_at(t + lane - 1), rest));
                if (next != 0) m = t + __builtin_ctzll(next) - first;
            }
        }
        const uint32_t low = __builtin_amdgcn_readlane((uint32_t)near_place.whole, at + 1);
        const uint32_t high = __builtin_amdgcn_readlane((uint32_t)(near_place.whole >> 32), at + 1);
        append_run<H, C, kHeld>(turn, shared, first, m, (uint64_t)high << 32 | low, __builtin_amdgcn_readlane(near_place.rest, at + 1),
                                from > task ? from - task : 0, to - task < 2 * a.kv_heads ? to - task : 2 * a.kv_heads, raw, near_position,
                                near_from);
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
__device__ __forceinline__ bool unit_of(const MoveArgs& a, uint32_t task, Unit& u) {
    const uint32_t lane = threadIdx.x % 64, at_once = 64u >> a.row_power, of_kv = (a.kv_heads + at_once - 1) / at_once;
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

__device__ __forceinline__ uint32_t wave_of_grid() { return __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + threadIdx.x / 64); }

// kShared: a unit is a workgroup's, a quarter of its tokens a wavefront's; else a wavefront's.
template <class H, class C, bool kShared>
__global__ __launch_bounds__(kThreads) void store8_kernel(MoveArgs a) {
    __shared__ uint32_t largest[kShared ? kWaves : 1][64];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    Unit u;
    if (!unit_of(a, kShared ? blockIdx.x : wave_of_grid(), u)) return;
    const uint32_t from = kShared ? u.count * wave / kWaves : 0, to = kShared ? u.count * (wave + 1) / kWaves : u.count;
    const uint32_t scale = convert_unit<H, C>(u.half + from * u.half_token, u.half_token, to - from,
                                              To{u.codes + from * u.code_token, u.code_token, u.wanted}, a.row_power, [&](uint32_t most) {
        if constexpr (kShared) {
            largest[wave][lane] = most;
            __syncthreads();
#pragma unroll
            for (uint32_t w = 0; w < kWaves; ++w) most = most > largest[w][lane] ? most : largest[w][lane];
        }
        return most;
    });
    if (u.part == 0 && u.there && (!kShared || wave == 0)) *u.scale = float_of(scale);
}

template <class H, class C>
__global__ __launch_bounds__(kThreads) void load8_kernel(MoveArgs a) {
    Unit u;
    if (!unit_of(a, wave_of_grid(), u)) return;
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
uint64_t move_units(const MoveArgs& a) {
    const uint32_t at_once = 64u >> a.row_power;
    return (uint64_t)a.n * 2 * ((a.kv_heads + at_once - 1) / at_once) * a.parts;
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
    // (lanes' places within the tokens that a wavefront has side by side are counted in 32 bits)
    for (const int64_t stride : {args->k_token, args->v_token, cache->k_token, cache->v_token})
        if (stride < 0 || stride > kMostAppendStride) return PGCM_ERR_ARG;
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
    a.eps = args->eps, a.by_dim = 1.f / (float)dim, a.by_block = 1.0 / cache->block_tokens;
    const uint32_t windows = (args->tokens + kWindow - 1) / kWindow, in_window = args->tokens < kWindow ? args->tokens : kWindow;
    // about kGroups workgroups of either kind where there is that much to do
    constexpr uint32_t kGroups = 1024, kMostWays = 16384;
    auto ways = [&](uint64_t most) {   // of so many wavefronts' work
        const uint64_t groups = (most + kWaves - 1) / kWaves;
        return windows >= kGroups || groups <= 1 ? 1u : (uint32_t)(kGroups / windows < groups ? kGroups / windows : groups);
    };
    // (a prompt's runs begin in as many windows as there are blocks: the others' workgroups have nothing to do)
    const uint64_t of_kv = (uint64_t)in_window * 2 * a.kv_heads;
    a.spread = cache->block_tokens / kWindow < windows ? cache->block_tokens / kWindow : windows;
    const uint64_t most_ways = (of_kv + kWaves - 1) / kWaves < kMostWays ? (of_kv + kWaves - 1) / kWaves : kMostWays;
    const uint64_t some_ways = (uint64_t)ways(of_kv) * a.spread;
    a.kv_ways = (uint32_t)(some_ways < most_ways ? some_ways : most_ways);
    const uint32_t at_once = 64u >> a.row_power, of_q = (a.heads + at_once - 1) / at_once;
    uint32_t q_ways = of_q == 0 ? 0 : ways((uint64_t)kWindow * of_q);
    if (q_ways != 0) q_ways = (q_ways + kWindow / kWaves - 1) / (kWindow / kWaves) * (kWindow / kWaves);   // all tokens in each round
    const uint32_t groups = (windows + a.spread - 1) / a.spread * a.spread;
    if (!launchable(groups, kThreads)) return PGCM_ERR_ARG;
    const dim3 grid(groups, a.kv_ways + q_ways);
    const hipStream_t stream = (hipStream_t)hip_stream;
    // blocks of sixteen tokens fit four steps of up to 128 channels; others are worth more registers
    const bool longer = cache->block_tokens > 4 * at_once, f16 = cache->half == PGCM_KV_F16;
    auto launch = [&](auto code) {
        typedef decltype(code) C;
        if (longer) {
            if (f16) append8_kernel<F16, C, 8><<<grid, kThreads, 0, stream>>>(a);
            else append8_kernel<Bf16, C, 8><<<grid, kThreads, 0, stream>>>(a);
        } else {
            if (f16) append8_kernel<F16, C, 4><<<grid, kThreads, 0, stream>>>(a);
            else append8_kernel<Bf16, C, 4><<<grid, kThreads, 0, stream>>>(a);
        }
    };
    if (cache->code == PGCM_KV8_INT8) launch(Int8());
    else launch(E4m3());
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

int pgcm_kv8_store(const pgcm_kv8_cache* to, const pgcm_kv_cache* from, uint32_t n, const int32_t* blocks, const int32_t* counts,
                   const int32_t* from_blocks, void* hip_stream) {
    MoveArgs a{};
    if (const int rc = move_args(to, from, n, blocks, counts, from_blocks, &a)) return rc;
    if (n == 0) return PGCM_OK;
    // A wavefront a unit, or four, where one would take its tokens twice, or units are few.  Microseconds with one and with four,
    // read-back included: 16 blocks of 40 heads (320 units) 12.6 and 11.9, 64 (1280) 18.1 and 18.2, 256 41.5 and 47.3, 2048 398 and
    // 419; 1024 blocks of 32 tokens 444 and 388, 512 of 64 499 and 386.
    const bool shared = a.block_tokens > kRowsHeld || move_units(a) <= kFewUnits;
    const uint64_t units = move_units(a), groups = shared ? units : (units + kWaves - 1) / kWaves;
    if (!launchable(groups, kThreads)) return PGCM_ERR_ARG;
    const uint32_t n_groups = (uint32_t)groups;
    const hipStream_t stream = (hipStream_t)hip_stream;
    auto launch = [&](auto half, auto code) {
        typedef decltype(half) H;
        typedef decltype(code) C;
        if (shared) store8_kernel<H, C, true><<<n_groups, kThreads, 0, stream>>>(a);
        else store8_kernel<H, C, false><<<n_groups, kThreads, 0, stream>>>(a);
    };
    if (from->half == PGCM_KV_F16) to->code == PGCM_KV8_INT8 ? launch(F16(), Int8()) : launch(F16(), E4m3());
    else to->code == PGCM_KV8_INT8 ? launch(Bf16(), Int8()) : launch(Bf16(), E4m3());
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

int pgcm_kv8_load(const pgcm_kv8_cache* from, const pgcm_kv_cache* to, uint32_t n, const int32_t* blocks, const int32_t* counts,
                  const int32_t* to_blocks, void* hip_stream) {
    MoveArgs a{};
    if (const int rc = move_args(from, to, n, blocks, counts, to_blocks, &a)) return rc;
    if (n == 0) return PGCM_OK;
    a.parts = (from->block_tokens + 15) / 16;   // sixteen tokens a wavefront
    const uint64_t waves = move_units(a);
    if (!launchable((waves + kWaves - 1) / kWaves, kThreads)) return PGCM_ERR_ARG;
    const uint32_t groups = (uint32_t)((waves + kWaves - 1) / kWaves);
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
