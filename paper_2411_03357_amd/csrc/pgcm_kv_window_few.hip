// Attention of single new tokens over KV blocks, in 8 bits or in halves, with a window (include/pgcm_kv8.h), on the matrix cores.
//
// Per token, kv head and group of up to sixteen of its query heads (an "item"):
//   s[t][h] = scale k_t . q_h,   m = max s,   out = sum 2^(s - m) v_t / sum 2^(s - m)     (s in units of log 2)
// with running m and sums, one pass over K and V.  What bounds it is memory: two requests of 131 059 tokens in int8, 8 kv heads of
// 128 and 8 query heads to each (537 MB): 113 us, 4.8 TB/s; 48 requests of up to 16384 tokens in e4m3 with a window of 8192, a
// twentieth of the blocks elsewhere (416 MB): 93 us, 4.5 TB/s; 64 in bfloat16 with a window of 4096 (982 MB): 174 us, 5.6 TB/s; one
// of 33 tokens, 40 heads: 6.1 us, the launch and trips to memory one after the other (length, table, scales and rows).
//
// Codes are whole in binary16, so they are multiplied as such, and their scales are applied to sums: the keys' to scores, the
// values' to each piece of sixteen tokens' part of a sum, in binary32: so any scales do, whatever they are to each other.
//
// Rows go to registers as the products take them, two tiles by turns.  (Three under way, of codes, with a head a workgroup: 128 us
// for the long case instead of 126.)  Items are cut into parts of equal numbers of tiles, a workgroup each.
//
// A head's row is 128 or 256 bytes of a token's, and rows that lie next to each other in memory belong to the heads beside it.
// Where there is much to read, a workgroup is eight wavefronts that have four heads side by side, two wavefronts each, and as many
// workgroups as the chip has room for at once: the same loads with nothing made of them take 96 us for the long case instead of
// 121, 166 instead of 192 in bfloat16; two heads 105, workgroups of heads beside each other on one XCD 133.  It has four times as
// many results to join for a workgroup, which costs it where there is little to read: there a workgroup has one head, and about
// kTargetGroups of them even out ragged lengths.
#include "pgcm_kv_window.h"

namespace pgcm_kv_impl {
namespace {

// Wavefronts of a workgroup, and kv heads that it has side by side
constexpr uint32_t waves_of(bool wide, uint32_t dim) { return wide && dim <= 128 ? 8 : 4; }
constexpr uint32_t abreast_of(bool wide) { return wide ? 4 : 1; }
constexpr uint32_t kMergedHeads = 4;   // at a time
constexpr uint32_t kJoinedAtOnce = 8;   // parts that a thread asks for together
constexpr uint32_t kMostJoined = 24;   // parts of an item in one go, by what a thread reads of each
constexpr uint32_t kTargetGroups = 1024, kWideGroups = 256;   // workgroups that a call's work is cut for
constexpr uint32_t kWholeRows = 512;   // beyond so many rows an item is one workgroup's: each looks through them for its own

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// How channels and tokens lie in a wavefront of lanes (g = lane / 16, i = lane % 16), for a piece of sixteen tokens:
//   K as the left operand: lane has token i, a run of channels of 16 bytes from 16 (4 c + g) on, in step c
//   S comes out with head i, tokens 4 g + r: already the right operand of the second product
//   V: lane loads, of tokens 4 g + r, the kRun channels from kRun i (+ 128) on; row i of the left operand of product t is channel
//     kRun i + t
template <uint32_t kDim>
struct Layout {
    static constexpr uint32_t kRun = kDim == 64 ? 4 : 8;
    static constexpr uint32_t kParts = kDim == 256 ? 2 : 1;
};

// Codes of four bytes as binary16, as they are
__device__ __forceinline__ f16x2 two_of(Int8*, uint32_t word_x, uint32_t pick) {   // word_x: each byte xor 0x80
    // 0x64 above a byte b: 1024 + b
    const uint32_t w = __builtin_amdgcn_perm(0x64646464u, word_x, pick);
    return __builtin_bit_cast(f16x2, w) - (_Float16)1152.f;
}
template <class C>
struct Convert;
template <>
struct Convert<Int8> {
    static __device__ __forceinline__ f16x4 four(uint32_t word) {
        const uint32_t x = word ^ 0x80808080u;
        const f16x2 a = two_of((Int8*)nullptr, x, 0x04010400u), b = two_of((Int8*)nullptr, x, 0x04030402u);
        return f16x4{a[0], a[1], b[0], b[1]};
    }
};
template <>
struct Convert<E4m3> {
    static __device__ __forceinline__ f16x4 four(uint32_t word) {
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)word, 1.f, false);
        const auto b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)word, 1.f, true);
        return f16x4{(_Float16)a[0], (_Float16)a[1], (_Float16)b[0], (_Float16)b[1]};
    }
};

// Bytes of four words turned: word n of the result has byte n of each
__device__ __forceinline__ void turn_bytes(const uint32_t (&x)[4], uint32_t (&y)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
    y[0] = __builtin_amdgcn_perm(c, a, 0x05040100u), y[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    y[2] = __builtin_amdgcn_perm(d, b, 0x05040100u), y[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// What a lane needs of a piece, all of it the wavefront's
struct Here {
    uint64_t k, v;   // addresses of the rows of the piece's first token
    uint32_t mask;   // which of its tokens are seen
    float k_scale, v_scale;
};

template <class H_, class C, uint32_t kDim_>
struct Codes {
    static constexpr uint32_t kDim = kDim_, kPieces = kDim == 64 ? 4 : 2;
    static constexpr bool kScaled = true;
    typedef H_ H;
    typedef F16 M;          // multiplied as
    typedef Layout<kDim> L;
    static constexpr uint32_t kSteps = kDim / 64;
    static constexpr uint32_t kRunWords = L::kRun / 4;
    struct Held {
        uint4 k[kPieces][kSteps];
        uint32_t v[kPieces][L::kParts][4][kRunWords];
    };
    template <bool kExact>
    static __device__ __forceinline__ void load(Held& held, const WindowArgs& a, uint32_t p, const Here& at, uint32_t g, uint32_t i) {
#pragma unroll
        for (uint32_t c = 0; c < kSteps; ++c) {
            const uint32_t d = 64 * c + 16 * g;   // (beyond the channels: anything that is there; the query is zero)
            held.k[p][c] = *(const uint4*)(at.k + i * (uint32_t)a.k_token + (kExact || d < a.head_dim ? d : 0));
        }
#pragma unroll
        for (uint32_t n = 0; n < L::kParts; ++n)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                const uint32_t d = 128 * n + L::kRun * i;
                const uint64_t from = at.v + (4 * g + r) * (uint32_t)a.v_token + (kExact || d < a.head_dim ? d : 0);
                if constexpr (kRunWords == 2) {
                    const uint2 x = *(const uint2*)from;
                    held.v[p][n][r][0] = x.x, held.v[p][n][r][1] = x.y;
                } else {
                    held.v[p][n][r][0] = *(const uint32_t*)from;
                }
            }
    }
    // A query as a power of two times binary16, its largest channel in [2^14, 2^15)
    struct Query {
        f16x8 x[2 * kSteps];
        float by;
    };
    struct Raw {
        uint4 x[2 * kSteps];
    };
    template <bool kExact>
    static __device__ __forceinline__ void ask_query(Raw& q, const WindowArgs& a, const uint8_t* row, bool there, uint32_t g) {
#pragma unroll
        for (uint32_t c = 0; c < 2 * kSteps; ++c) {
            const uint32_t d = 64 * (c / 2) + 16 * g + 8 * (c % 2);
            q.x[c] = make_uint4(0, 0, 0, 0);
            if (there && (kExact || d < a.head_dim)) q.x[c] = *(const uint4*)(row + 2 * d);
        }
    }
    static __device__ __forceinline__ void make_query(Query& q, const Raw& raw) {
        float x[2 * kSteps][8];
        float most = 0.f;
        bool odd = false;
#pragma unroll
        for (uint32_t c = 0; c < 2 * kSteps; ++c) {
            const typename H::eight y = as_eight<H>(raw.x[c]);
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) {
                x[c][e] = (float)y[e];
                most = fmaxf(most, fabsf(x[c][e]));
                odd |= !(fabsf(x[c][e]) < INFINITY);
            }
        }
        most = over_rows_max(odd ? INFINITY : most);
        const uint32_t exponent = __builtin_bit_cast(uint32_t, most) >> 23;     // 255: not finite; 0: nothing to speak of
        const int32_t up = exponent == 0 || exponent == 255 ? 0 : 141 - (int32_t)exponent;   // 2^up times the largest is in [2^14, 2^15)
        // (in two steps, as 2^up may exceed the range)
        const float first = power_of_two(up / 2), second = power_of_two(up - up / 2);
        q.by = exponent == 255 ? NAN : power_of_two(-(up / 2)) * power_of_two(-(up - up / 2));
#pragma unroll
        for (uint32_t c = 0; c < 2 * kSteps; ++c)
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) q.x[c][e] = (_Float16)(exponent == 255 ? 0.f : x[c][e] * first * second);
    }
    static __device__ __forceinline__ f32x4 scores(const Held& held, uint32_t p, const Query& q) {
        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (uint32_t c = 0; c < kSteps; ++c) {
            const uint32_t words[4] = {held.k[p][c].x, held.k[p][c].y, held.k[p][c].z, held.k[p][c].w};
#pragma unroll
            for (uint32_t n = 0; n < 2; ++n) {
                const f16x4 low = Convert<C>::four(words[2 * n]), high = Convert<C>::four(words[2 * n + 1]);
                s[n] = F16::product(__builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7), q.x[2 * c + n], s[n]);
            }
        }
        return s[0] + s[1];
    }
    // sums += values by the weights of pieces p and p + 1
    static __device__ __forceinline__ void add(Held& held, uint32_t p, const float (&w)[8], const Here (&at)[kPieces],
                                               f32x4 (&sum)[L::kParts][L::kRun], uint32_t g) {
        F16::eight halves[2];
        F16::split(w, halves);
#pragma unroll
        for (uint32_t e = 0; e < 2; ++e) {
            const uint32_t piece = p + e;
            f16x4 by[2];
#pragma unroll
            for (uint32_t n = 0; n < 2; ++n)
                by[n] = f16x4{halves[n][4 * e], halves[n][4 * e + 1], halves[n][4 * e + 2], halves[n][4 * e + 3]};
            if (at[piece].mask != 0xFFFFu) {   // tokens that are not seen count as zero, whatever they hold
#pragma unroll
                for (uint32_t n = 0; n < L::kParts; ++n)
#pragma unroll
                    for (uint32_t r = 0; r < 4; ++r)
#pragma unroll
                        for (uint32_t x = 0; x < kRunWords; ++x)
                            held.v[piece][n][r][x] = at[piece].mask >> (4 * g + r) & 1 ? held.v[piece][n][r][x] : 0u;
            }
            const float scale = at[piece].mask != 0 ? at[piece].v_scale : 0.f;
#pragma unroll
            for (uint32_t n = 0; n < L::kParts; ++n)
#pragma unroll
                for (uint32_t x = 0; x < kRunWords; ++x) {
                    const uint32_t rows[4] = {held.v[piece][n][0][x], held.v[piece][n][1][x], held.v[piece][n][2][x],
                                              held.v[piece][n][3][x]};
                    uint32_t channels[4];
                    turn_bytes(rows, channels);
#pragma unroll
                    for (uint32_t t = 0; t < 4; ++t) {
                        const f16x4 v = Convert<C>::four(channels[t]);
                        f32x4 y{0.f, 0.f, 0.f, 0.f};
                        y = __builtin_amdgcn_mfma_f32_16x16x16f16(v, by[0], y, 0, 0, 0);
                        y = __builtin_amdgcn_mfma_f32_16x16x16f16(v, by[1], y, 0, 0, 0);
                        sum[n][4 * x + t] += y * scale;
                    }
                }
        }
    }
};

template <class H_, uint32_t kDim_>
struct Halves {
    static constexpr uint32_t kDim = kDim_, kPieces = 2;
    static constexpr bool kScaled = false;
    typedef H_ H;
    typedef H_ M;
    typedef Layout<kDim> L;
    static constexpr uint32_t kSteps = kDim / 32;
    static constexpr uint32_t kRunWords = L::kRun / 2;
    struct Held {
        uint4 k[kPieces][kSteps];
        uint32_t v[kPieces][L::kParts][4][kRunWords];
    };
    template <bool kExact>
    static __device__ __forceinline__ void load(Held& held, const WindowArgs& a, uint32_t p, const Here& at, uint32_t g, uint32_t i) {
#pragma unroll
        for (uint32_t c = 0; c < kSteps; ++c) {
            const uint32_t d = 32 * c + 8 * g;
            if constexpr (!kExact) held.k[p][c] = make_uint4(0, 0, 0, 0);   // (infinity times a query's zero is no number)
            if (kExact || d < a.head_dim) held.k[p][c] = *(const uint4*)(at.k + i * (uint32_t)a.k_token + 2 * d);
        }
#pragma unroll
        for (uint32_t n = 0; n < L::kParts; ++n)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                const uint32_t d = 128 * n + L::kRun * i;
                const uint64_t from = at.v + (4 * g + r) * (uint32_t)a.v_token + 2 * (kExact || d < a.head_dim ? d : 0);
                if constexpr (kRunWords == 4) {
                    const uint4 x = *(const uint4*)from;
                    held.v[p][n][r][0] = x.x, held.v[p][n][r][1] = x.y, held.v[p][n][r][2] = x.z, held.v[p][n][r][3] = x.w;
                } else {
                    const uint2 x = *(const uint2*)from;
                    held.v[p][n][r][0] = x.x, held.v[p][n][r][1] = x.y;
                }
            }
    }
    struct Query {
        uint4 x[kSteps];
        static constexpr float by = 1.f;
    };
    typedef Query Raw;
    template <bool kExact>
    static __device__ __forceinline__ void ask_query(Raw& q, const WindowArgs& a, const uint8_t* row, bool there, uint32_t g) {
#pragma unroll
        for (uint32_t c = 0; c < kSteps; ++c) {
            const uint32_t d = 32 * c + 8 * g;
            q.x[c] = make_uint4(0, 0, 0, 0);
            if (there && (kExact || d < a.head_dim)) q.x[c] = *(const uint4*)(row + 2 * d);
        }
    }
    static __device__ __forceinline__ void make_query(Query& q, const Raw& raw) { q = raw; }
    static __device__ __forceinline__ f32x4 scores(const Held& held, uint32_t p, const Query& q) {
        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (uint32_t c = 0; c < kSteps; ++c) s[c % 2] = H::product(as_eight<H>(held.k[p][c]), as_eight<H>(q.x[c]), s[c % 2]);
        return s[0] + s[1];
    }
    static __device__ __forceinline__ void add(Held& held, uint32_t p, const float (&w)[8], const Here (&at)[kPieces],
                                               f32x4 (&sum)[L::kParts][L::kRun], uint32_t g) {
        typename H::eight halves[H::kHalves];
        H::split(w, halves);
#pragma unroll
        for (uint32_t e = 0; e < 2; ++e)
            if (at[e].mask != 0xFFFFu)
#pragma unroll
                for (uint32_t n = 0; n < L::kParts; ++n)
#pragma unroll
                    for (uint32_t r = 0; r < 4; ++r)
#pragma unroll
                        for (uint32_t x = 0; x < kRunWords; ++x)
                            held.v[e][n][r][x] = at[e].mask >> (4 * g + r) & 1 ? held.v[e][n][r][x] : 0u;
#pragma unroll
        for (uint32_t n = 0; n < L::kParts; ++n)
#pragma unroll
            for (uint32_t t = 0; t < L::kRun; ++t) {
                const uint32_t x = t / 2, pick = t % 2 ? 0x07060302u : 0x05040100u;
                uint32_t y[4];
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
                    y[e] = __builtin_amdgcn_perm(held.v[e / 2][n][2 * (e % 2) + 1][x], held.v[e / 2][n][2 * (e % 2)][x], pick);
                const typename H::eight v = as_eight<H>(make_uint4(y[0], y[1], y[2], y[3]));
#pragma unroll
                for (uint32_t h = 0; h < H::kHalves; ++h) sum[n][t] = H::product(v, halves[h], sum[n][t]);
            }
    }
};

// A row's request and how many of its tokens it sees, or request ~0: none has it
struct Row {
    uint32_t request, end;
};
template <uint32_t kWaves, uint32_t kDim>
struct FewShared {
    union {
        Row row[kWholeRows];
        float sum[kWaves][kMergedHeads][kDim + 4];
    };
    float top[kWaves][16], total[kWaves][16];
    uint32_t last;
};

__device__ __forceinline__ Row row_of(const WindowArgs& a, uint32_t row) {
    const uint32_t room = a.row_blocks * a.block_tokens;
    if (a.starts == nullptr) return Row{row, clamped(a.lens[row], room)};
    // the last request that starts at this row or before it
    uint32_t low = 0, high = a.requests;   // starts[low] <= row < starts[high], if any has it
    while (high - low > 1) {
        const uint32_t mid = (low + high) / 2;
        if (clamped(a.starts[mid], a.tokens) <= row) low = mid;
        else high = mid;
    }
    const uint32_t from = clamped(a.starts[low], a.tokens), to = clamped(a.starts[low + 1], a.tokens);
    if (row < from || row >= to || row - from >= a.most) return Row{~0u, 0};
    const uint32_t count = to - from < a.most ? to - from : a.most, behind = count - 1 - (row - from);
    const uint32_t len = clamped(a.lens[low], room);
    return Row{low, len > behind ? len - behind : 0};
}

// its tiles: of the pieces that the wavefronts of an item, `slots` of them, take at once
template <class S>
__device__ __forceinline__ uint32_t tiles_of(const WindowArgs& a, Row row, uint32_t slots) {
    return row.end == 0 ? 0 : (seen_of(a, row.end, row.end).pieces() + slots * S::kPieces - 1) / (slots * S::kPieces);
}

// kCut: items are cut into parts of equal numbers of tiles; else an item is one workgroup's.  kWide: a workgroup has those of
// kAbreast kv heads.
template <class S, bool kExact, bool kCut, bool kWide>
__global__ __launch_bounds__(waves_of(kWide, S::kDim) * 64, kWide || S::kDim == 256 ? 1 : 2) void few_kernel(WindowArgs a) {
    typedef typename S::H H;
    typedef typename S::M M;
    typedef typename S::L L;
    constexpr uint32_t kDim = S::kDim, kPieces = S::kPieces, kWaves = waves_of(kWide, kDim), kThreads = kWaves * 64;
    constexpr uint32_t kAbreast = abreast_of(kWide), kSlots = kWaves / kAbreast;   // kSlots: wavefronts that share an item
    __shared__ FewShared<kWaves, kDim> shared;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t g = lane / 16, i = lane % 16, beside = wave % kAbreast, slot = wave / kAbreast;
    const uint32_t group_tiles = (a.group + 15) / 16, per_row = a.kv_heads / kAbreast * group_tiles;

    // The workgroup's items are those of kAbreast kv heads of a row, side by side.
    uint32_t row = blockIdx.x / per_row, items = blockIdx.x - row * per_row, part = 0, parts = 1, first_part = 0;
    Row of;
    if constexpr (kCut) {
        // rows and their tiles: a lane has the l-th of 64
        Row lane_row{~0u, 0};
        uint32_t mine = 0, all = 0;
        if (a.tokens <= 64) {
            if (lane < a.tokens) lane_row = row_of(a, lane);
            mine = tiles_of<S>(a, lane_row, kSlots);
            all = __builtin_amdgcn_readlane(scan(mine), 63);
        } else {
            for (uint32_t r = threadIdx.x; r < a.tokens; r += kThreads) shared.row[r] = row_of(a, r);
            __syncthreads();
        }
        auto look = [&](uint32_t r0) {
            if (a.tokens <= 64) return;
            lane_row = r0 + lane < a.tokens ? shared.row[r0 + lane] : Row{~0u, 0};
            mine = tiles_of<S>(a, lane_row, kSlots);
        };
        if (a.tokens > 64)
            for (uint32_t r0 = 0; r0 < a.tokens; r0 += 64) {
                look(r0);
                all += __builtin_amdgcn_readlane(scan(mine), 63);
            }
        // A part's tiles, at most.  One head a workgroup: so that those that are cut make about kTargetGroups; all of them are no more
        // than that and one for each item.  Heads side by side: about the least for which all are no more than kWideGroups.
        const uint32_t most_parts = kWideGroups / per_row;   // (used where items are at most half as many as kWideGroups)
        uint32_t share = kWide ? (all + most_parts - 1) / most_parts : (all * per_row + kTargetGroups - 1) / kTargetGroups;
        share = share != 0 ? share : 1;
        auto its = [&] {   // (rows without tokens are answered by one part)
            return lane_row.request == ~0u ? 0 : mine <= share ? 1 : (mine + share - 1) / share;
        };
        while (kWide) {
            uint32_t count = 0;
            for (uint32_t r0 = 0; r0 < a.tokens; r0 += 64) {
                look(r0);
                count += __builtin_amdgcn_readlane(scan(its()), 63);
            }
            if (count <= most_parts) break;
            const uint32_t more = (uint32_t)((float)share * (float)count / (float)most_parts);
            share = more > share ? more : share + 1;
        }
        uint32_t before = 0;
        bool found = false;
        for (uint32_t r0 = 0; r0 < a.tokens; r0 += 64) {
            look(r0);
            const uint32_t here = its(), upto = before + scan(here);
            const uint64_t past = __ballot(upto * per_row > blockIdx.x);
            if (past != 0) {
                const uint32_t at = __builtin_ctzll(past);
                row = r0 + at;
                parts = __builtin_amdgcn_readlane(here, at);
                const uint32_t first = (__builtin_amdgcn_readlane(upto, at) - parts) * per_row, x = blockIdx.x - first;
                // in the grid: heads next to each other, as in memory (the loads of the long case alone: 100 us, 109 with parts
                // next to each other); with one head a workgroup, parts (127 us, 139 with heads)
                part = kWide ? x / per_row : x % parts;
                items = kWide ? x - part * per_row : x / parts;
                first_part = first + items * parts;
                of = Row{(uint32_t)__builtin_amdgcn_readlane(lane_row.request, at), (uint32_t)__builtin_amdgcn_readlane(lane_row.end, at)};
                found = true;
                break;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
        }
        if (!found) return;
    } else {
        of = row_of(a, row);
        of.request = __builtin_amdgcn_readfirstlane(of.request), of.end = __builtin_amdgcn_readfirstlane(of.end);
        if (of.request == ~0u) return;
    }
    const uint32_t heads_at = items / group_tiles, head0 = (items - heads_at * group_tiles) * 16;
    const uint32_t kv_head = heads_at * kAbreast + beside, heads = a.group - head0 < 16 ? a.group - head0 : 16;
    auto first_head_of = [&](uint32_t beside) { return (heads_at * kAbreast + beside) * a.group + head0; };
    const uint32_t first_head = first_head_of(beside);
    const Seen seen = of.end == 0 ? Seen{0, 0, 0} : seen_of(a, of.end, of.end);
    const uint32_t pieces = seen.pieces(), tiles = tiles_of<S>(a, of, kSlots), low = low_of(a, of.end);
    const uint32_t even = tiles / parts, more = tiles - even * parts;   // `more` parts have one tile more
    const uint32_t from = even * part + (part < more ? part : more), to = from + even + (part < more ? 1 : 0);

    typename S::Raw raw;
    S::template ask_query<kExact>(raw, a, a.q + row * a.q_token + (first_head + (i < heads ? i : 0)) * a.q_head, i < heads, g);

    f32x4 sum[L::kParts][L::kRun];
#pragma unroll
    for (uint32_t n = 0; n < L::kParts; ++n)
#pragma unroll
        for (uint32_t t = 0; t < L::kRun; ++t) sum[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, total = 0.f;

    // Where the wavefront's pieces lie: lane l has the l-th of a batch, kPieces of each tile.
    constexpr uint32_t kBatch = 64 / kPieces;   // tiles
    struct Pieces {
        uint32_t block, inside, mask;   // block ~0: none
    };
    auto find = [&](uint32_t tile) {
        Pieces p{~0u, 0, 0};
        const uint32_t t = tile + lane / kPieces, x = (t * kSlots + slot) * kPieces + lane % kPieces;
        if (t >= to || x >= pieces) return p;
        const uint32_t token = seen.piece(x) * kPiece, place = token / a.block_tokens;
        const uint32_t end = of.end - token;   // of the tokens that are seen, from the piece's first one on
        p.mask = end < kPiece ? (1u << end) - 1 : 0xFFFFu;
        if (token < low) {
            const uint32_t from_low = low - token < kPiece ? 0xFFFFu << (low - token) & 0xFFFFu : 0u;
            const uint32_t to_sinks = a.sinks <= token ? 0u : a.sinks - token < kPiece ? (1u << (a.sinks - token)) - 1 : 0xFFFFu;
            p.mask &= from_low | to_sinks;
        }
        p.inside = token - place * a.block_tokens;
        if (p.mask != 0) p.block = (uint32_t)a.tables[of.request * a.table_row + place];
        return p;
    };
    uint64_t piece_k, piece_v, live = 0;
    uint32_t piece_mask;
    float piece_ks = 0.f, piece_vs = 0.f;
    auto use = [&](const Pieces& p) {
        const bool there = p.block < a.blocks && p.mask != 0;
        live = __ballot(there);
        piece_mask = there ? p.mask : 0;
        const uint64_t block = there ? p.block : 0;   // (a masked piece: any that is there)
        const uint32_t inside = there ? p.inside : 0;
        piece_k = (uint64_t)(uintptr_t)a.k + kv_head * a.k_head + block * a.k_block + inside * a.k_token;
        piece_v = (uint64_t)(uintptr_t)a.v + kv_head * a.v_head + block * a.v_block + inside * a.v_token;
        if constexpr (S::kScaled) {
            piece_ks = a.k_scales[block * a.k_scale_block + kv_head * a.k_scale_head];
            piece_vs = a.v_scales[block * a.v_scale_block + kv_head * a.v_scale_head];
        }
    };
    auto lane_of = [](uint64_t x, uint32_t j) {
        const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, j), hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), j);
        return (uint64_t)hi << 32 | lo;   // (what comes from a lane is an int)
    };
    uint32_t ahead = from;              // the first tile of the batch that is looked for next
    Pieces next = find(ahead);
    auto seek = [&](Here (&at)[kPieces]) {   // the next tile that is not masked as a whole, if there is one
        while (live == 0) {
            if (ahead >= to) return false;
            use(next);
            ahead += kBatch;
            next = find(ahead);
        }
        const uint32_t j = __builtin_ctzll(live) / kPieces * kPieces;
        live &= ~(((1ull << kPieces) - 1) << j);
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p) {
            at[p].k = lane_of(piece_k, j + p), at[p].v = lane_of(piece_v, j + p);
            at[p].mask = __builtin_amdgcn_readlane(piece_mask, j + p);
            at[p].k_scale = at[p].v_scale = 1.f;
            if constexpr (S::kScaled) {
                const uint32_t ks = __builtin_amdgcn_readlane(__builtin_bit_cast(uint32_t, piece_ks), j + p);
                const uint32_t vs = __builtin_amdgcn_readlane(__builtin_bit_cast(uint32_t, piece_vs), j + p);
                at[p].k_scale = __builtin_bit_cast(float, ks), at[p].v_scale = __builtin_bit_cast(float, vs);
            }
        }
        return true;
    };
    auto load = [&](typename S::Held& held, const Here (&at)[kPieces]) {
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p) S::template load<kExact>(held, a, p, at[p], g, i);
    };
    typename S::Query query;
    auto work = [&](typename S::Held& held, const Here (&at)[kPieces]) {
        float s[kPieces][4];
        float most = -INFINITY;
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p) {
            const f32x4 x = S::scores(held, p, query);
            // (the powers of two of keys and query first: either may be near the ends of the range, and their product not)
            const float scale = S::kScaled ? at[p].k_scale * query.by * a.scale : a.scale;
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                s[p][r] = x[r] * scale;
                if (at[p].mask != 0xFFFFu) s[p][r] = at[p].mask >> (4 * g + r) & 1 ? s[p][r] : -INFINITY;
                most = fmaxf(most, s[p][r]);
            }
        }
        most = over_rows_max(most);
        // Sums are kept relative to 2^top, which makes the largest weight so far 2^M::kLargest when they were last brought up to
        // it, and at most 2^M::kOverflows before the next time: a new maximum rarely takes that.
        const bool over = most > top + M::kOverflows || (top == -INFINITY && most > top);
        if (__any(over)) {   // (what other heads need changes nothing in a head)
            const float now = over ? fmaxf(most - M::kLargest, top) : top, keep = exp2_from(top, now);
            top = now;
            total *= keep;
#pragma unroll
            for (uint32_t n = 0; n < L::kParts; ++n)
#pragma unroll
                for (uint32_t t = 0; t < L::kRun; ++t) sum[n][t] *= keep;
        }
        const float down = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (uint32_t p = 0; p < kPieces; p += 2) {
            float w[8];
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f(s[p + e / 4][e % 4] - down);
                total += w[e];
            }
            S::add(held, p, w, at, sum, g);
        }
    };
    {
        // two tiles' rows in registers by turns: one under way while the other is worked on
        typename S::Held held[2];
        Here at[2][kPieces];
        if (seek(at[0])) {
            load(held[0], at[0]);
            S::make_query(query, raw);
            while (true) {
                const bool more = seek(at[1]);
                if (more) load(held[1], at[1]);
                work(held[0], at[0]);
                if (!more) break;
                const bool again = seek(at[0]);
                if (again) load(held[0], at[0]);
                work(held[1], at[1]);
                if (!again) break;
            }
        }
    }

    // The wavefronts' results as one.  A lane holds, of head i, channels kRun (4 g + r) + t.
    total = over_rows_sum(total);
    if (g == 0) shared.top[wave][i] = top, shared.total[wave][i] = total;
    auto finish = [&](uint32_t out_head, uint32_t d, float4 x, float top, float total) {
        const float by = total == 0.f ? 0.f : 1.f / total;   // (a NaN stays one)
        if (d < a.head_dim) {
            typename H::one y[4] = {(typename H::one)(x.x * by), (typename H::one)(x.y * by), (typename H::one)(x.z * by),
                                    (typename H::one)(x.w * by)};
            uint2 words;
            __builtin_memcpy(&words, y, 8);
            *(uint2*)(a.out + row * a.out_token + out_head * a.out_head + 2 * d) = words;
        }
        if (d == 0 && a.lse != nullptr)
            a.lse[(size_t)row * a.kv_heads * a.group + out_head] =
                total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * 0.693147180559945f;
    };
    constexpr uint32_t kQuads = kDim / 4;
    const uint32_t rows_kept = a.group < 16 ? a.group : 16;
    const size_t part_floats = (size_t)rows_kept * (kDim + 2);   // sums, then tops and totals
    auto part_at = [&](uint32_t place, uint32_t beside) { return a.partials + (place * kAbreast + beside) * part_floats; };
    auto put_part = [&](float* to_part, uint32_t h, uint32_t d, float4 x, float top, float total) {
        uint64_t* to_sum = (uint64_t*)(to_part + h * kDim + d);
        put_shared(to_sum, __builtin_bit_cast(uint64_t, make_float2(x.x, x.y)));
        put_shared(to_sum + 1, __builtin_bit_cast(uint64_t, make_float2(x.z, x.w)));
        if (d == 0)
            put_shared((uint64_t*)(to_part + rows_kept * kDim) + h, __builtin_bit_cast(uint64_t, make_float2(top, total)));
    };
    for (uint32_t h0 = 0; h0 < heads; h0 += kMergedHeads) {
        const uint32_t these = heads - h0 < kMergedHeads ? heads - h0 : kMergedHeads;
        __syncthreads();
        if (i - h0 < these) {
#pragma unroll
            for (uint32_t n = 0; n < L::kParts; ++n)
#pragma unroll
                for (uint32_t r = 0; r < 4; ++r)
#pragma unroll
                    for (uint32_t t = 0; t < L::kRun; t += 4)
                        *(float4*)&shared.sum[wave][i - h0][128 * n + L::kRun * (4 * g + r) + t] =
                            make_float4(sum[n][t][r], sum[n][t + 1][r], sum[n][t + 2][r], sum[n][t + 3][r]);
        }
        __syncthreads();
        for (uint32_t x = threadIdx.x; x < these * kAbreast * kQuads; x += kThreads) {
            const uint32_t d = x % kQuads * 4, b = x / kQuads % kAbreast, k = x / (kQuads * kAbreast), h = h0 + k;
            float most = shared.top[b][h];
#pragma unroll
            for (uint32_t w = 1; w < kSlots; ++w) most = fmaxf(most, shared.top[b + w * kAbreast][h]);
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            float of_all = 0.f;
#pragma unroll
            for (uint32_t w = 0; w < kSlots; ++w) {
                const float by = exp2_from(shared.top[b + w * kAbreast][h], most);
                const float4 z = *(const float4*)&shared.sum[b + w * kAbreast][k][d];
                of_all += shared.total[b + w * kAbreast][h] * by;
                y.x += z.x * by, y.y += z.y * by, y.z += z.z * by, y.w += z.w * by;
            }
            if (!kCut || parts == 1) finish(first_head_of(b) + h, d, y, most, of_all);
            else put_part(part_at(first_part + part, b), h, d, y, most, of_all);
        }
    }
    if constexpr (kCut) {
        if (parts == 1) return;
        // The parts' results as one, by the last workgroup to arrive: those of workgroups first, first + apart, ..., to the outputs
        // or to the first's place.
        constexpr uint32_t kMine = kWide && kDim != 64 ? 2 : 1;   // quads of a thread at a time
        const uint32_t quads = kAbreast * heads * kQuads;
        auto join = [&](uint32_t first, uint32_t apart, uint32_t count, bool last) {
            for (uint32_t x0 = threadIdx.x; x0 < quads; x0 += kMine * kThreads) {
                float4 y[kMine];
                float top[kMine], total[kMine];
                uint32_t b[kMine], h[kMine];
                const uint32_t d = x0 % kQuads * 4;
#pragma unroll
                for (uint32_t n = 0; n < kMine; ++n) {
                    const uint32_t x = x0 + n * kThreads < quads ? x0 + n * kThreads : x0;
                    b[n] = x / kQuads % kAbreast, h[n] = x / (kQuads * kAbreast);
                    y[n] = make_float4(0.f, 0.f, 0.f, 0.f), top[n] = -INFINITY, total[n] = 0.f;
                }
                for (uint32_t p0 = 0; p0 < count; p0 += kJoinedAtOnce) {
                    uint64_t z[kJoinedAtOnce][kMine][3];   // under way together
#pragma unroll
                    for (uint32_t e = 0; e < kJoinedAtOnce; ++e)
#pragma unroll
                        for (uint32_t n = 0; n < kMine; ++n) {
                            const float* from_part = part_at(first + (p0 + e < count ? p0 + e : p0) * apart, b[n]);
                            const uint64_t* at_sum = (const uint64_t*)(from_part + h[n] * kDim + d);
                            z[e][n][0] = get_shared(at_sum), z[e][n][1] = get_shared(at_sum + 1);
                            z[e][n][2] = get_shared((const uint64_t*)(from_part + rows_kept * kDim) + h[n]);
                        }
#pragma unroll
                    for (uint32_t n = 0; n < kMine; ++n) {
                        float most = top[n];
#pragma unroll
                        for (uint32_t e = 0; e < kJoinedAtOnce; ++e) most = fmaxf(most, __builtin_bit_cast(float2, z[e][n][2]).x);
                        const float keep = exp2_from(top[n], most);
                        top[n] = most, total[n] *= keep;
                        y[n].x *= keep, y[n].y *= keep, y[n].z *= keep, y[n].w *= keep;
#pragma unroll
                        for (uint32_t e = 0; e < kJoinedAtOnce; ++e) {
                            if (p0 + e >= count) break;
                            const float2 u = __builtin_bit_cast(float2, z[e][n][0]), v = __builtin_bit_cast(float2, z[e][n][1]);
                            const float2 of = __builtin_bit_cast(float2, z[e][n][2]);
                            const float by = exp2_from(of.x, most);
                            total[n] += of.y * by;
                            y[n].x += u.x * by, y[n].y += u.y * by, y[n].z += v.x * by, y[n].w += v.y * by;
                        }
                    }
                }
#pragma unroll
                for (uint32_t n = 0; n < kMine; ++n) {
                    if (x0 + n * kThreads >= quads) continue;
                    // (a row is a wavefront's or a part of it: what is put over the first part has been read by all)
                    if (last) finish(first_head_of(b[n]) + h[n], d, y[n], top[n], total[n]);
                    else put_part(part_at(first, b[n]), h[n], d, y[n], top[n], total[n]);
                }
            }
        };
        // in one go, or in groups of as many as there are groups
        uint32_t fan = parts;
        if (parts * ((quads + kThreads - 1) / kThreads) > kMostJoined)
            for (fan = 4; fan * fan < parts;) ++fan;
        const uint32_t mine = part / fan * fan, count = parts - mine < fan ? parts - mine : fan;
        if (last_to_arrive(a.counters + first_part + mine, count, &shared.last)) {
            join(first_part + mine, 1, count, fan >= parts);
            const uint32_t groups_of = (parts + fan - 1) / fan;
            if (fan < parts && last_to_arrive(a.counters + 2 * kTargetGroups + first_part, groups_of, &shared.last))
                join(first_part, fan, groups_of, true);
        }
    }
}

template <class S, bool kExact>
void launch(const WindowArgs& a, uint32_t groups, bool cut, bool wide, hipStream_t stream) {
    const uint32_t threads = waves_of(wide, S::kDim) * 64;
    if (cut && wide) few_kernel<S, kExact, true, true><<<groups, threads, 0, stream>>>(a);
    else if (cut) few_kernel<S, kExact, true, false><<<groups, threads, 0, stream>>>(a);
    else few_kernel<S, kExact, false, false><<<groups, threads, 0, stream>>>(a);
}
template <template <uint32_t> class S>
void launch(const WindowArgs& a, uint32_t groups, bool cut, bool wide, hipStream_t stream) {
    const uint32_t d = a.head_dim;
    if (d == 64) launch<S<64>, true>(a, groups, cut, wide, stream);
    else if (d < 64) launch<S<64>, false>(a, groups, cut, wide, stream);
    else if (d == 128) launch<S<128>, true>(a, groups, cut, wide, stream);
    else if (d < 128) launch<S<128>, false>(a, groups, cut, wide, stream);
    else if (d == 256) launch<S<256>, true>(a, groups, cut, wide, stream);
    else launch<S<256>, false>(a, groups, cut, wide, stream);
}
template <uint32_t kDim> using Int8OfF16 = Codes<F16, Int8, kDim>;
template <uint32_t kDim> using Int8OfBf16 = Codes<Bf16, Int8, kDim>;
template <uint32_t kDim> using E4m3OfF16 = Codes<F16, E4m3, kDim>;
template <uint32_t kDim> using E4m3OfBf16 = Codes<Bf16, E4m3, kDim>;
template <uint32_t kDim> using HalvesF16 = Halves<F16, kDim>;
template <uint32_t kDim> using HalvesBf16 = Halves<Bf16, kDim>;

}  // namespace

// Results of as many workgroups as there may be with more than one for an item, and two counters for each.
static_assert(abreast_of(true) * kWideGroups <= 2 * kTargetGroups, "one room for both");
Room window_few_room(uint32_t heads, uint32_t kv_heads, uint32_t head_dim) {
    return Room{4 * 2 * 2 * kTargetGroups, 4 * partial_floats(head_dim, heads / kv_heads) * 2 * kTargetGroups};
}

int window_few(pgcm_kv* kv, WindowArgs& a, uint32_t half, uint32_t code, hipStream_t stream) {
    uint64_t walked = (uint64_t)a.row_blocks * a.block_tokens;
    if (a.window != 0 && walked > (uint64_t)a.window + a.sinks + 3 * kPiece) walked = (uint64_t)a.window + a.sinks + 3 * kPiece;
    struct Cut {
        uint64_t per_row, items, tiles;   // workgroups of a row and of all, uncut; an item's tiles
        bool worth;
    };
    auto cut_of = [&](bool wide) {
        const uint32_t pieces = code != ~0u && a.head_dim <= 64 ? 4 : 2;
        const uint32_t tile = waves_of(wide, a.head_dim) / abreast_of(wide) * pieces * kPiece;
        Cut x;
        x.per_row = (uint64_t)a.kv_heads / abreast_of(wide) * ((a.group + 15) / 16);
        x.items = a.tokens * x.per_row, x.tiles = (walked + tile - 1) / tile;
        x.worth = x.tiles > 2 && x.items <= kTargetGroups && a.tokens <= kWholeRows && x.items * x.tiles < 1u << 31;
        return x;
    };
    const Cut narrow = cut_of(false), beside = cut_of(true);
    // Items are cut where that may give the chip more to do.  Heads side by side are worth it where an item has few parts to be
    // joined or many tiles: a call of them takes up to 10 us longer whatever the lengths (1 of 4096 tokens, 8 kv heads: 20 us
    // instead of 13.5; of 32768, 36 and 37; two of 131 059, 116 and 127; 48 of 500 with 8 kv heads, 15.7 and 17.1; 16, 12.5 and 8.1).
    const bool cut = narrow.worth;
    const bool wide = cut && beside.worth && a.kv_heads % abreast_of(true) == 0 && 2 * beside.items <= kWideGroups &&
                      (beside.items >= kWideGroups / 4 || beside.items * beside.tiles >= 16 * kWideGroups);
    const uint64_t items = wide ? beside.items : narrow.items;
    const uint64_t all = wide ? kWideGroups / beside.per_row * beside.per_row : narrow.items + kTargetGroups;
    const uint64_t most = items * (wide ? beside.tiles : narrow.tiles), groups = !cut ? items : most < all ? most : all;
    if (!launchable(groups, waves_of(wide, a.head_dim) * 64)) return PGCM_ERR_ARG;
    if (cut) {
        const Room room = window_few_room(a.kv_heads * a.group, a.kv_heads, a.head_dim);
        if (const int rc = kv_ensure(kv, room.counters, room.scratch, stream)) return rc;
        a.counters = (uint32_t*)kv->counters.at, a.partials = (float*)kv->scratch.at;
    }
    const uint32_t n = (uint32_t)groups;
    const bool f16 = half == PGCM_KV_F16;
    if (code == PGCM_KV8_INT8) f16 ? launch<Int8OfF16>(a, n, cut, wide, stream) : launch<Int8OfBf16>(a, n, cut, wide, stream);
    else if (code == PGCM_KV8_E4M3) f16 ? launch<E4m3OfF16>(a, n, cut, wide, stream) : launch<E4m3OfBf16>(a, n, cut, wide, stream);
    else f16 ? launch<HalvesF16>(a, n, cut, wide, stream) : launch<HalvesBf16>(a, n, cut, wide, stream);
    return pgcm::hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

}  // namespace pgcm_kv_impl
