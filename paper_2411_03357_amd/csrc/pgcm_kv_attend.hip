// Attention of one new token of each request over its KV blocks (include/pgcm_kv.h), on the matrix cores.
//
// Per request, kv head and group of up to sixteen of its query heads (an "item"):
//   s[t][h] = scale k_t . q_h,   m = max s,   out = sum 2^(s - m) v_t / sum 2^(s - m)     (s in units of log 2)
// with running m and sums, one pass over K and V.
#include "pgcm_kv_common.h"

#include <cmath>

namespace pgcm_kv_impl {
namespace {

constexpr uint32_t kWaves = 4;
constexpr uint32_t kThreads = kWaves * 64;
constexpr uint32_t kMinTiles = 2;  // a workgroup's span, where the batch has as many: less is not worth joining
static_assert(kTileTokens == kWaves * 2 * kPiece, "two pieces a wavefront");

struct AttendArgs {
    const uint8_t *k, *v, *q;
    uint8_t* out;
    const int32_t *tables, *lens, *selected;
    float *lse, *partials, *head_lse, *piece_lse;  // the last two in units of log 2; piece_lse null: no weights
    uint32_t* counters;
    int64_t k_block, k_token, k_head, v_block, v_token, v_head, q_request, q_head, out_request, out_head;  // bytes
    int64_t table_row;
    uint32_t requests, kv_heads, group, group_tiles, head_dim, block_tokens, row_blocks, blocks, keep;
    float scale;  // times log2 e
};

__device__ __forceinline__ uint32_t clamped_len(const AttendArgs& a, int32_t len) {
    const uint32_t room = a.row_blocks * a.block_tokens;
    return len <= 0 ? 0u : (uint32_t)len < room ? (uint32_t)len : room;
}
// tokens that an item of a request of this length walks over; of a selection, those of all its places
__device__ __forceinline__ uint32_t walked(const AttendArgs& a, int32_t len) {
    const uint32_t n = clamped_len(a, len);
    return a.selected == nullptr || n == 0 ? n : a.keep * a.block_tokens;
}
__device__ __forceinline__ uint32_t tiles_of(const AttendArgs& a, uint32_t request) {
    return (walked(a, a.lens[request]) + kTileTokens - 1) / kTileTokens;
}

__device__ __forceinline__ float exp2_from(float x, float top) {  // 0 for x = -inf, whatever the top
    return __builtin_amdgcn_exp2f(x - (top == -INFINITY ? 0.f : top));
}

template <uint32_t kDim>
struct AttendShared {
    float sum[kWaves][16][kDim + 4];
    float top[kWaves][16], total[kWaves][16];
    float part_top[64][16], part_total[64][16];
    uint32_t last;
};

// How channels and tokens lie in a wavefront of lanes (g = lane / 16, i = lane % 16), for a tile of 32 tokens:
//   K as the left operand, piece by piece: lane has token i, channels 32 c + 8 g ... + 7 in step c
//   S comes out with head i, tokens 4 g + r: already the right operand of the second product, which takes
//     tokens 4 g + r of the first piece and of the second as its eight of lane (g, i)
//   V: lane loads, of its eight tokens, the kRun channels from kRun i (+ 128); row i of the left operand of product
//     t is channel kRun i + t, so that the lane has all of its operands' words and only swaps halves of registers
template <class H, uint32_t kDim, bool kExact>
struct Walk {
    static constexpr uint32_t kSteps = kDim / 32;               // of the first product
    static constexpr uint32_t kRun = kDim == 64 ? 4 : 8;        // channels of V that a lane loads at once
    static constexpr uint32_t kParts = kDim == 256 ? 2 : 1;     // ... so many times
    static constexpr uint32_t kWords = kRun / 2;                // 32-bit words of that

    f32x4 sum[kParts][kRun];
    float top, total;
    uint4 q[kSteps], k[2][kSteps];
    uint32_t v[kParts][8][kWords];

    __device__ __forceinline__ void begin(const AttendArgs& a, const uint8_t* row, bool there, uint32_t g) {
#pragma unroll
        for (uint32_t p = 0; p < kParts; ++p)
#pragma unroll
            for (uint32_t t = 0; t < kRun; ++t) sum[p][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        top = -INFINITY;
        total = 0.f;
#pragma unroll
        for (uint32_t c = 0; c < kSteps; ++c) {
            const uint32_t d = 32 * c + 8 * g;
            q[c] = make_uint4(0, 0, 0, 0);
            if (there && (kExact || d < a.head_dim)) q[c] = *(const uint4*)(row + 2 * d);
        }
    }
    __device__ __forceinline__ void load_k(const AttendArgs& a, uint32_t which, const uint8_t* lane_row, uint32_t g) {
#pragma unroll
        for (uint32_t c = 0; c < kSteps; ++c) {
            const uint32_t d = 32 * c + 8 * g;
            if (kExact || d < a.head_dim)
                k[which][c] = *(const uint4*)(lane_row + 2 * d);
            else
                k[which][c] = make_uint4(0, 0, 0, 0);
        }
    }
    // first_row: of the lane's first token in the piece
    __device__ __forceinline__ void load_v(const AttendArgs& a, uint32_t which, const uint8_t* first_row, uint32_t i) {
#pragma unroll
        for (uint32_t p = 0; p < kParts; ++p) {
            const uint32_t d = 128 * p + kRun * i;
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                uint32_t(&to)[kWords] = v[p][4 * which + r];
                if (kExact || d < a.head_dim) {
                    const uint8_t* from = first_row + r * a.v_token + 2 * d;
                    if constexpr (kWords == 4) {
                        const uint4 x = *(const uint4*)from;
                        to[0] = x.x, to[1] = x.y, to[2] = x.z, to[3] = x.w;
                    } else {
                        const uint2 x = *(const uint2*)from;
                        to[0] = x.x, to[1] = x.y;
                    }
                } else {
#pragma unroll
                    for (uint32_t w = 0; w < kWords; ++w) to[w] = 0;
                }
            }
        }
    }
    // rows of tokens that are not there count as zero, whatever they hold
    __device__ __forceinline__ void drop_v(uint32_t which, uint32_t valid, uint32_t g) {
#pragma unroll
        for (uint32_t p = 0; p < kParts; ++p)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r)
#pragma unroll
                for (uint32_t w = 0; w < kWords; ++w)
                    v[p][4 * which + r][w] = 4 * g + r < valid ? v[p][4 * which + r][w] : 0u;
    }
    __device__ __forceinline__ void scores(float (&s)[8], float scale, uint32_t valid0, uint32_t valid1, uint32_t g) const {
        f32x4 s0{0.f, 0.f, 0.f, 0.f}, s1{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (uint32_t c = 0; c < kSteps; ++c) {
            s0 = H::product(as_eight<H>(k[0][c]), as_eight<H>(q[c]), s0);
            s1 = H::product(as_eight<H>(k[1][c]), as_eight<H>(q[c]), s1);
        }
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) {
            s[r] = 4 * g + r < valid0 ? s0[r] * scale : -INFINITY;
            s[4 + r] = 4 * g + r < valid1 ? s1[r] * scale : -INFINITY;
        }
    }
    // running maximum and sum; the scores become weights
    __device__ __forceinline__ void weigh(float (&s)[8]) {
        float most = s[0];
#pragma unroll
        for (uint32_t j = 1; j < 8; ++j) most = fmaxf(most, s[j]);
        most = over_rows_max(most);
        if (__any(most > top)) {
            const float now = fmaxf(most, top), keep = exp2_from(top, now);
            top = now;
            total *= keep;
#pragma unroll
            for (uint32_t p = 0; p < kParts; ++p)
#pragma unroll
                for (uint32_t t = 0; t < kRun; ++t) sum[p][t] *= keep;
        }
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            s[j] = exp2_from(s[j], top);
            total += s[j];
        }
    }
    __device__ __forceinline__ void add_v(const float (&s)[8]) {
        // A weight goes to the matrix cores as two halves, the second what the first leaves: with one, its rounding
        // would be as large as that of the output.
        typename H::eight high, low;
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            high[j] = (typename H::one)s[j];
            low[j] = (typename H::one)(s[j] - (float)high[j]);
        }
#pragma unroll
        for (uint32_t p = 0; p < kParts; ++p)
#pragma unroll
            for (uint32_t t = 0; t < kRun; ++t) {
                const uint32_t pick = t % 2 ? 0x07060302u : 0x05040100u;
                const uint4 x = make_uint4(__builtin_amdgcn_perm(v[p][1][t / 2], v[p][0][t / 2], pick),
                                           __builtin_amdgcn_perm(v[p][3][t / 2], v[p][2][t / 2], pick),
                                           __builtin_amdgcn_perm(v[p][5][t / 2], v[p][4][t / 2], pick),
                                           __builtin_amdgcn_perm(v[p][7][t / 2], v[p][6][t / 2], pick));
                sum[p][t] = H::product(as_eight<H>(x), high, sum[p][t]);
                sum[p][t] = H::product(as_eight<H>(x), low, sum[p][t]);
            }
    }
};

// Where a wavefront's pieces lie: lane l holds its l-th from `first` on (two of each tile).
struct Pieces {
    uint32_t block;   // number, or ~0: masked
    uint32_t inside;  // token of the block in the low half, how many of its sixteen are there in the high one
};
__device__ __forceinline__ Pieces find_pieces(const AttendArgs& a, const int32_t* row, const int32_t* picked, uint32_t len,
                                              uint32_t tile, uint32_t last_tile, uint32_t wave, uint32_t lane) {
    Pieces p{~0u, 0u};
    const uint32_t t = tile + lane / 2;
    if (t >= last_tile) return p;
    const uint32_t piece = t * (kTileTokens / kPiece) + 2 * wave + (lane & 1);
    const uint32_t per_block = a.block_tokens / kPiece;
    uint32_t place = piece / per_block;
    const uint32_t inside = (piece - place * per_block) * kPiece;
    if (picked != nullptr) {
        if (place >= a.keep) return p;
        place = (uint32_t)picked[place];
    }
    if (place >= a.row_blocks) return p;
    const uint64_t token = (uint64_t)place * a.block_tokens + inside;
    if (token >= len) return p;
    const uint32_t block = (uint32_t)row[place];
    if (block >= a.blocks) return p;
    const uint64_t valid = len - token < kPiece ? len - token : kPiece;
    p.block = block;
    p.inside = inside | (uint32_t)valid << 16;
    return p;
}

template <class H, uint32_t kDim, bool kExact>
__global__ __launch_bounds__(kThreads, kDim == 256 ? 1 : 2) void attend_kernel(AttendArgs a) {
    typedef Walk<H, kDim, kExact> W;
    __shared__ AttendShared<kDim> shared;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t g = lane / 16, i = lane % 16;
    const uint32_t per_request = a.kv_heads * a.group_tiles;

    // The tiles of all items, in the order of requests and heads, in equal spans: this workgroup's is [from, to).
    uint32_t all = 0, tiles = 0, upto = 0;   // those of up to 64 requests, and of all before and with them
    for (uint32_t b0 = 0; b0 < a.requests; b0 += 64) {
        const uint32_t b = b0 + lane;
        tiles = b < a.requests ? tiles_of(a, b) : 0;
        upto = all + scan(tiles);
        all = __builtin_amdgcn_readlane(upto, 63);
        // requests without tokens are answered here
        uint64_t empty = __ballot(b < a.requests && tiles == 0 && b % gridDim.x == blockIdx.x);
        for (; empty != 0; empty &= empty - 1) {
            const uint32_t e = b0 + __builtin_ctzll(empty), heads = a.kv_heads * a.group;
            for (uint32_t x = threadIdx.x; x < heads * a.head_dim; x += kThreads)
                *(uint16_t*)(a.out + e * a.out_request + x / a.head_dim * a.out_head + 2 * (x % a.head_dim)) = 0;
            for (uint32_t h = threadIdx.x; h < heads; h += kThreads) {
                if (a.lse != nullptr) a.lse[(size_t)e * heads + h] = -INFINITY;
                if (a.piece_lse != nullptr) a.head_lse[(size_t)e * heads + h] = -INFINITY;
            }
        }
    }
    all *= per_request;
    if (all == 0) return;
    const uint32_t least = (all + kMinTiles - 1) / kMinTiles;
    const uint32_t groups = gridDim.x < least ? gridDim.x : least;
    if (blockIdx.x >= groups) return;
    auto start_of = [&](uint32_t w) { return (uint32_t)((uint64_t)w * all / groups); };
    auto owner_of = [&](uint32_t tile) { return (uint32_t)((((uint64_t)tile + 1) * groups - 1) / all); };
    const uint32_t from = start_of(blockIdx.x), to = start_of(blockIdx.x + 1);

    // the request that the span begins in, and its first tile
    uint32_t request = 0, before = 0;
    for (uint32_t b0 = 0, sum = 0; b0 < a.requests; b0 += 64) {
        if (a.requests > 64) {
            const uint32_t b = b0 + lane;
            tiles = b < a.requests ? tiles_of(a, b) : 0;
            upto = sum + scan(tiles);
        }
        const uint64_t past = __ballot(upto * per_request > from);
        if (past != 0) {
            const uint32_t at = __builtin_ctzll(past);
            request = b0 + at;
            before = __builtin_amdgcn_readlane(upto - tiles, at) * per_request;
            break;
        }
        sum = __builtin_amdgcn_readlane(upto, 63);
    }
    request = __builtin_amdgcn_readfirstlane(request);
    before = __builtin_amdgcn_readfirstlane(before);

    W walk;
    for (uint32_t at = from; at < to;) {
        uint32_t tiles = tiles_of(a, request);
        while (at >= before + tiles * per_request) {
            before += tiles * per_request;
            tiles = tiles_of(a, ++request);
        }
        const uint32_t len = clamped_len(a, a.lens[request]);
        const uint32_t item = (at - before) / tiles;
        const uint32_t item_from = before + item * tiles, item_to = item_from + tiles;
        const uint32_t head = item / a.group_tiles, head0 = item % a.group_tiles * 16;  // kv head; first of its group
        const uint32_t heads = a.group - head0 < 16 ? a.group - head0 : 16;
        const uint32_t first_head = head * a.group + head0;
        uint32_t tile = at - item_from;
        const uint32_t tile_to = (to < item_to ? to : item_to) - item_from;
        const int32_t* row = a.tables + request * a.table_row;
        const int32_t* picked =
            a.selected == nullptr ? nullptr : a.selected + ((size_t)request * a.kv_heads + head) * a.keep;
        const uint8_t *k0 = a.k + head * a.k_head, *v0 = a.v + head * a.v_head;

        walk.begin(a, a.q + request * a.q_request + (first_head + (i < heads ? i : 0)) * a.q_head, i < heads, g);

        Pieces pieces;
        uint32_t b0, b1, in0, in1;   // of the tile in hand
        auto take = [&](uint32_t j) {
            b0 = __builtin_amdgcn_readlane(pieces.block, 2 * j), b1 = __builtin_amdgcn_readlane(pieces.block, 2 * j + 1);
            in0 = __builtin_amdgcn_readlane(pieces.inside, 2 * j), in1 = __builtin_amdgcn_readlane(pieces.inside, 2 * j + 1);
        };
        // A masked piece of a tile that is not masked as a whole reads the other one's rows, which are there.
        auto load_keys = [&](uint32_t x0, uint32_t x1, uint32_t n0, uint32_t n1) {
            const bool one0 = x0 != ~0u, one1 = x1 != ~0u;
            const uint32_t y0 = one0 ? x0 : x1, y1 = one1 ? x1 : x0;
            const uint32_t o0 = (one0 ? n0 : n1) & 0xFFFF, o1 = (one1 ? n1 : n0) & 0xFFFF;
            walk.load_k(a, 0, k0 + y0 * a.k_block + (o0 + i) * a.k_token, g);
            walk.load_k(a, 1, k0 + y1 * a.k_block + (o1 + i) * a.k_token, g);
        };
        auto load_values = [&](uint32_t x0, uint32_t x1, uint32_t n0, uint32_t n1) {
            const bool one0 = x0 != ~0u, one1 = x1 != ~0u;
            const uint32_t y0 = one0 ? x0 : x1, y1 = one1 ? x1 : x0;
            const uint32_t o0 = (one0 ? n0 : n1) & 0xFFFF, o1 = (one1 ? n1 : n0) & 0xFFFF;
            walk.load_v(a, 0, v0 + y0 * a.v_block + (o0 + 4 * g) * a.v_token, i);
            walk.load_v(a, 1, v0 + y1 * a.v_block + (o1 + 4 * g) * a.v_token, i);
        };
        // the next tile, from `tile` on, that is not masked as a whole; tile_to if none is
        uint32_t looked = tile;      // pieces holds those of [looked, looked + 32)
        auto seek = [&]() {
            while (tile < tile_to) {
                if (tile == looked) pieces = find_pieces(a, row, picked, len, tile, tile_to, wave, lane);
                const uint64_t live = __ballot(pieces.block != ~0u);
                const uint32_t past = tile - looked;      // < 32
                const uint64_t rest = live >> (2 * past);
                if (rest != 0) {
                    const uint32_t skip = __builtin_ctzll(rest) / 2;
                    tile += skip;
                    take(past + skip);
                    return;
                }
                looked += 32;
                tile = looked < tile_to ? looked : tile_to;
            }
        };
        seek();
        if (tile < tile_to) {
            load_keys(b0, b1, in0, in1);
            load_values(b0, b1, in0, in1);
        }
        while (tile < tile_to) {
            const uint32_t valid0 = b0 == ~0u ? 0 : in0 >> 16, valid1 = b1 == ~0u ? 0 : in1 >> 16;
            const uint32_t this_tile = tile;
            float s[8];
            walk.scores(s, a.scale, valid0, valid1, g);
            if (++tile == looked + 32) looked += 32;
            seek();
            if (tile < tile_to) load_keys(b0, b1, in0, in1);   // under way while the weights are made
            walk.weigh(s);
            if (a.piece_lse != nullptr) {
                const float w0 = over_rows_sum((s[0] + s[1]) + (s[2] + s[3]));
                const float w1 = over_rows_sum((s[4] + s[5]) + (s[6] + s[7]));
                if (g == 0 && i < heads) {
                    const uint32_t per_row = a.row_blocks * (a.block_tokens / kPiece);
                    float* to_row = a.piece_lse + ((size_t)request * a.kv_heads * a.group + first_head + i) * per_row +
                                    this_tile * (kTileTokens / kPiece) + 2 * wave;
                    // (a row's last tile may be cut by its end)
                    if (valid0 != 0) to_row[0] = walk.top + __builtin_amdgcn_logf(w0);
                    if (valid1 != 0) to_row[1] = walk.top + __builtin_amdgcn_logf(w1);
                }
            }
            if (valid0 < kPiece || valid1 < kPiece) {
                walk.drop_v(0, valid0, g);
                walk.drop_v(1, valid1, g);
            }
            walk.add_v(s);
            if (tile < tile_to) load_values(b0, b1, in0, in1);
        }

        // The wavefronts' results as one.  A lane holds, of head i, channels kRun (4 g + r) + t.
        walk.total = over_rows_sum(walk.total);
        __syncthreads();
        if (i < heads) {
#pragma unroll
            for (uint32_t p = 0; p < W::kParts; ++p)
#pragma unroll
                for (uint32_t r = 0; r < 4; ++r)
#pragma unroll
                    for (uint32_t t = 0; t < W::kRun; t += 4)
                        *(float4*)&shared.sum[wave][i][128 * p + W::kRun * (4 * g + r) + t] =
                            make_float4(walk.sum[p][t][r], walk.sum[p][t + 1][r], walk.sum[p][t + 2][r], walk.sum[p][t + 3][r]);
            if (g == 0) {
                shared.top[wave][i] = walk.top;
                shared.total[wave][i] = walk.total;
            }
        }
        __syncthreads();

        auto finish = [&](uint32_t h, uint32_t d, float4 x, float top, float total) {
            const float by = total == 0.f ? 0.f : 1.f / total;   // (a NaN stays one)
            const uint32_t out_head = first_head + h;
            if (d < a.head_dim) {
                typename H::one y[4] = {(typename H::one)(x.x * by), (typename H::one)(x.y * by),
                                        (typename H::one)(x.z * by), (typename H::one)(x.w * by)};
                uint2 words;
                __builtin_memcpy(&words, y, 8);
                *(uint2*)(a.out + request * a.out_request + out_head * a.out_head + 2 * d) = words;
            }
            if (d == 0) {
                const float of_head = total == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(total);
                const size_t n = (size_t)request * a.kv_heads * a.group + out_head;
                if (a.lse != nullptr) a.lse[n] = of_head * 0.693147180559945f;
                if (a.piece_lse != nullptr) a.head_lse[n] = of_head;
            }
        };

        const uint32_t first_part = owner_of(item_from), parts = owner_of(item_to - 1) - first_part + 1;
        constexpr uint32_t kQuads = kDim / 4;
        const size_t part_floats = 16 * kDim + 32;
        auto slot_of = [&](uint32_t w) {   // a workgroup's first item, or its last
            return a.partials + (2 * (size_t)w + (item_from > start_of(w) ? 1 : 0)) * part_floats;
        };
        for (uint32_t x = threadIdx.x; x < heads * kQuads; x += kThreads) {
            const uint32_t h = x / kQuads, d = x % kQuads * 4;
            float top = shared.top[0][h];
#pragma unroll
            for (uint32_t w = 1; w < kWaves; ++w) top = fmaxf(top, shared.top[w][h]);
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            float total = 0.f;
#pragma unroll
            for (uint32_t w = 0; w < kWaves; ++w) {
                const float by = exp2_from(shared.top[w][h], top);
                const float4 y = *(const float4*)&shared.sum[w][h][d];
                total += shared.total[w][h] * by;
                sum.x += y.x * by, sum.y += y.y * by, sum.z += y.z * by, sum.w += y.w * by;
            }
            if (parts == 1) {
                finish(h, d, sum, top, total);
            } else {
                float* slot = slot_of(blockIdx.x);
                uint64_t* to_sum = (uint64_t*)(slot + h * kDim + d);
                put_shared(to_sum, __builtin_bit_cast(uint64_t, make_float2(sum.x, sum.y)));
                put_shared(to_sum + 1, __builtin_bit_cast(uint64_t, make_float2(sum.z, sum.w)));
                if (d == 0) put_shared((uint64_t*)(slot + 16 * kDim) + h, __builtin_bit_cast(uint64_t, make_float2(top, total)));
            }
        }
        if (parts > 1 && last_to_arrive(a.counters + request * per_request + item, parts, &shared.last)) {
            // the parts' results as one, 64 parts at a step
            constexpr uint32_t kMine = (16 * kQuads + kThreads - 1) / kThreads;
            float4 sum[kMine];
            float top[kMine], total[kMine];
#pragma unroll
            for (uint32_t n = 0; n < kMine; ++n) sum[n] = make_float4(0.f, 0.f, 0.f, 0.f), top[n] = -INFINITY, total[n] = 0.f;
            for (uint32_t p0 = 0; p0 < parts; p0 += 64) {
                const uint32_t some = parts - p0 < 64 ? parts - p0 : 64;
                __syncthreads();
                for (uint32_t x = threadIdx.x; x < some * heads; x += kThreads) {
                    const uint32_t p = x / heads, h = x - p * heads;
                    const float2 y = __builtin_bit_cast(
                        float2, get_shared((const uint64_t*)(slot_of(first_part + p0 + p) + 16 * kDim) + h));
                    shared.part_top[p][h] = y.x;
                    shared.part_total[p][h] = y.y;
                }
                __syncthreads();
#pragma unroll
                for (uint32_t n = 0; n < kMine; ++n) {
                    const uint32_t x = threadIdx.x + n * kThreads;
                    if (x >= heads * kQuads) break;
                    const uint32_t h = x / kQuads, d = x % kQuads * 4;
                    float now = top[n];
                    for (uint32_t p = 0; p < some; ++p) now = fmaxf(now, shared.part_top[p][h]);
                    const float keep = exp2_from(top[n], now);
                    top[n] = now;
                    total[n] *= keep;
                    sum[n].x *= keep, sum[n].y *= keep, sum[n].z *= keep, sum[n].w *= keep;
#pragma unroll 8
                    for (uint32_t p = 0; p < some; ++p) {
                        const uint64_t* at_sum = (const uint64_t*)(slot_of(first_part + p0 + p) + h * kDim + d);
                        const float2 y = __builtin_bit_cast(float2, get_shared(at_sum));
                        const float2 z = __builtin_bit_cast(float2, get_shared(at_sum + 1));
                        const float by = exp2_from(shared.part_top[p][h], now);
                        total[n] += shared.part_total[p][h] * by;
                        sum[n].x += y.x * by, sum[n].y += y.y * by, sum[n].z += z.x * by, sum[n].w += z.y * by;
                    }
                }
            }
#pragma unroll
            for (uint32_t n = 0; n < kMine; ++n) {
                const uint32_t x = threadIdx.x + n * kThreads;
                if (x < heads * kQuads) finish(x / kQuads, x % kQuads * 4, sum[n], top[n], total[n]);
            }
        }
        at = item_from + tile_to;
    }
}

// weights[b][j] = decay kept[b][j] + sum over heads and pieces of 2^(piece - head): 64 blocks a workgroup, a quarter of
// the heads each wavefront, added up in their order
__global__ __launch_bounds__(kThreads) void weights_kernel(AttendArgs a, const float* kept, float* weights, float decay) {
    __shared__ float quarter[kWaves][64];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, request = blockIdx.y;
    const uint32_t j = blockIdx.x * 64 + lane, heads = a.kv_heads * a.group, per_block = a.block_tokens / kPiece;
    const uint32_t len = clamped_len(a, a.lens[request]);
    float sum = 0.f;
    if (j < a.row_blocks && (uint64_t)j * a.block_tokens < len && (uint32_t)a.tables[request * a.table_row + j] < a.blocks) {
        const uint32_t tokens = len - j * a.block_tokens < a.block_tokens ? len - j * a.block_tokens : a.block_tokens;
        const uint32_t pieces = (tokens + kPiece - 1) / kPiece, per_row = a.row_blocks * per_block;
        const float* at = a.piece_lse + (size_t)request * heads * per_row + j * per_block;
        const float* of = a.head_lse + (size_t)request * heads;
        const uint32_t to = heads * (wave + 1) / kWaves;
        for (uint32_t p = 0; p < pieces; ++p)
            for (uint32_t h = heads * wave / kWaves; h < to; h += 8) {   // eight heads' loads under way together
                float x[8], y[8];
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) {
                    x[e] = h + e < to ? at[(size_t)(h + e) * per_row + p] : -INFINITY;
                    y[e] = h + e < to ? of[h + e] : 0.f;
                }
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) sum += exp2_from(x[e], y[e]);
            }
    }
    quarter[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && j < a.row_blocks) {
        const size_t n = (size_t)request * a.row_blocks + j;
        sum = (quarter[0][lane] + quarter[1][lane]) + (quarter[2][lane] + quarter[3][lane]);
        weights[n] = kept == nullptr ? sum : decay * kept[n] + sum;
    }
}

template <class H>
void launch(const AttendArgs& a, uint32_t groups, hipStream_t stream) {
    const uint32_t d = a.head_dim;
    if (d == 64) attend_kernel<H, 64, true><<<groups, kThreads, 0, stream>>>(a);
    else if (d < 64) attend_kernel<H, 64, false><<<groups, kThreads, 0, stream>>>(a);
    else if (d == 128) attend_kernel<H, 128, true><<<groups, kThreads, 0, stream>>>(a);
    else if (d < 128) attend_kernel<H, 128, false><<<groups, kThreads, 0, stream>>>(a);
    else if (d == 256) attend_kernel<H, 256, true><<<groups, kThreads, 0, stream>>>(a);
    else attend_kernel<H, 256, false><<<groups, kThreads, 0, stream>>>(a);
}

}  // namespace
}  // namespace pgcm_kv_impl

using namespace pgcm_kv_impl;
using pgcm::hip_noted;

extern "C" {
#pragma GCC visibility push(default)

int pgcm_kv_attend(pgcm_kv_t* kv, const pgcm_kv_cache* cache, const pgcm_kv_attend_args* args, void* hip_stream) {
    if (kv == nullptr || args == nullptr) return PGCM_ERR_ARG;
    if (const int rc = check_cache(cache)) return rc;
    if (args->requests == 0) return PGCM_OK;
    if (args->q == nullptr || args->out == nullptr || args->lens == nullptr || !std::isfinite(args->scale) ||
        (args->tables == nullptr && args->row_blocks != 0) || (args->selected != nullptr && args->weights != nullptr) ||
        (args->kept != nullptr && args->weights == nullptr) || args->requests > 65535)
        return PGCM_ERR_ARG;
    if (const int rc = check_sizes(args->requests, args->heads, cache->kv_heads, cache->head_dim, cache->block_tokens,
                                   args->selected != nullptr && args->keep > args->row_blocks ? args->keep : args->row_blocks))
        return rc;
    if (!aligned(args->q, args->q_request, args->q_head) || !aligned(args->out, args->out_request, args->out_head))
        return PGCM_ERR_ALIGN;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const bool weigh = args->weights != nullptr;
    const uint64_t row_pieces = (uint64_t)args->row_blocks * (cache->block_tokens / kPiece);
    const Room room = attend_room(args->requests, args->heads, cache->kv_heads, cache->head_dim, weigh ? row_pieces : 0);
    if (const int rc = kv_ensure(kv, room.counters, room.scratch, stream)) return rc;

    AttendArgs a{};
    a.k = (const uint8_t*)cache->k, a.v = (const uint8_t*)cache->v, a.q = (const uint8_t*)args->q;
    a.out = (uint8_t*)args->out;
    a.tables = args->tables, a.lens = args->lens, a.selected = args->selected, a.lse = args->lse;
    a.counters = (uint32_t*)kv->counters.at;
    uint8_t* at = kv->scratch.at;
    a.partials = (float*)at;
    at += whole_lines(4 * partial_floats(cache->head_dim) * 2 * kAttendGroups);
    a.head_lse = (float*)at;
    at += whole_lines(4 * (size_t)args->requests * args->heads);
    a.piece_lse = weigh ? (float*)at : nullptr;
    a.k_block = 2 * cache->k_block, a.k_token = 2 * cache->k_token, a.k_head = 2 * cache->k_head;
    a.v_block = 2 * cache->v_block, a.v_token = 2 * cache->v_token, a.v_head = 2 * cache->v_head;
    a.q_request = 2 * args->q_request, a.q_head = 2 * args->q_head;
    a.out_request = 2 * args->out_request, a.out_head = 2 * args->out_head;
    a.table_row = args->table_row;
    a.requests = args->requests, a.kv_heads = cache->kv_heads, a.group = args->heads / cache->kv_heads;
    a.group_tiles = (a.group + 15) / 16;
    a.head_dim = cache->head_dim, a.block_tokens = cache->block_tokens;
    a.row_blocks = args->row_blocks, a.blocks = cache->blocks, a.keep = args->selected != nullptr ? args->keep : 0;
    a.scale = (float)((double)args->scale * 1.4426950408889634);

    // no more workgroups than the longest lengths could use
    const uint64_t walk_blocks = args->selected != nullptr ? args->keep : args->row_blocks;
    const uint64_t tiles = (walk_blocks * cache->block_tokens + kTileTokens - 1) / kTileTokens;
    const uint64_t most = (tiles * a.requests * a.kv_heads * a.group_tiles + kMinTiles - 1) / kMinTiles;
    const uint32_t groups = most > kAttendGroups ? kAttendGroups : most > 1 ? (uint32_t)most : 1;
    if (cache->half == PGCM_KV_F16) launch<F16>(a, groups, stream);
    else launch<Bf16>(a, groups, stream);
    if (hip_noted(hipGetLastError())) return PGCM_ERR_HIP;
    if (weigh && args->row_blocks != 0) {
        weights_kernel<<<dim3((args->row_blocks + 63) / 64, args->requests), kThreads, 0, stream>>>(a, args->kept, args->weights,
                                                                                                  args->decay);
        if (hip_noted(hipGetLastError())) return PGCM_ERR_HIP;
    }
    return PGCM_OK;
}

#pragma GCC visibility pop
}  // extern "C"
