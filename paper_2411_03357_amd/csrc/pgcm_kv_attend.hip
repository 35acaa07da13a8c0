// Attention of one new token of each request over its KV blocks (include/pgcm_kv.h), on the matrix cores.
//
// Per request, kv head and group of up to sixteen of its query heads (an "item"):
//   s[t][h] = scale k_t . q_h,   m = max s,   out = sum 2^(s - m) v_t / sum 2^(s - m)     (s in units of log 2)
// with running m and sums, one pass over K and V.  What bounds it is memory: at sixteen heads an item, 16 flops a byte.
// Two requests of 131 059 tokens, 8 kv heads of 128 (1.07 GB): 200 us, 5.4 TB/s, each byte read once; a kernel that only reads
// the same rows takes 183 to 230, by the order of its loads.  32 of up to 2048 tokens, 40 heads of 128 (396 MB): 86 us, 4.6
// TB/s.  One of 33 tokens, 40 heads: 4.7 us, the launch and trips to memory one after the other (table, rows).
//
// The tiles of all items, 128 tokens each, are cut into equal spans, one for each workgroup, so that neither lengths nor their
// number matter (short items are left whole); an item of several workgroups is joined by the last of them, in two levels if they
// are many.  A workgroup's four wavefronts take 32 tokens of a tile each and are joined through LDS at an item's end; the next
// tile's rows, the next item's among them, are on their way to LDS then.
#include "pgcm_kv_common.h"

#include <cmath>

namespace pgcm_kv_impl {
namespace {

constexpr uint32_t kWaves = 4;
constexpr uint32_t kThreads = kWaves * 64;
constexpr int64_t kMostTokenStride = 1 << 25;
constexpr uint32_t kCus = 256;
// Which workgroups there are.  One for each item, if none is longer than kWholeTiles, or than kWholeTilesOfMany where there are
// kManyItems: joining parts costs more than a few tiles do (80 items of 4 tiles: 10.3 us, in parts 12.0; 504 of up to 4, 14.7 and
// 19.6; 248 of up to 5, 17.0 and 17.6; but 8 items of 8 tiles 12.8 and 9.6).  Else, by the tiles of an item on average:
//   up to kShortItem: one for each tile, if that fills no more than the chip; above, for two: joining more parts costs more than
//   a tile does (one request of 4096 tokens, 8 kv heads: 14.1 us with two tiles each, 17.4 with one)
//   from kLongItem on, if there are kManyTiles for each compute unit: one for each, whose four wavefronts have 64 KiB under way;
//   with two, memory serves no more and in a worse order (1 GiB in 16 items, 64 tiles each: 201 us with one, 208 with two; 8
//   items, 4 tiles each: 21.8 and 22.5).  With fewer tiles or shorter items one would be alone with each item's end (24 items,
//   3.6 tiles each: 24.7 and 21.7; 1280 items of 1 to 16 tiles: 115 and 95).
constexpr uint32_t kWholeTiles = 4, kWholeTilesOfMany = 8, kManyItems = 64;
constexpr uint32_t kShortItem = 8, kLongItem = 16, kManyTiles = 4;
// Parts of an item that are joined in one go, by what a thread reads of each; more are joined in groups, and the groups then: of
// 128 channels and 4 heads, 16 parts 14.1 us in one go and 15.2 in two, 32 parts 19.5 and 17.7; 128 parts of 16 heads 79 and 35.
constexpr uint32_t kJoinedAtOnce = 24;
static_assert(kJoinedAtOnce * kJoinedAtOnce >= kAttendGroups, "two levels are enough");
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

// A request's length, which nothing writes to while the kernel runs: so it may come through the scalar cache.
__device__ __forceinline__ int32_t len_of(const AttendArgs& a, uint32_t request) {
    return ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)a.lens)[request];
}
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
    return (walked(a, len_of(a, request)) + kTileTokens - 1) / kTileTokens;
}

__device__ __forceinline__ float exp2_from(float x, float top) {  // 0 for x = -inf, whatever the top
    return __builtin_amdgcn_exp2f(x - (top == -INFINITY ? 0.f : top));
}

// How channels and tokens lie in a wavefront of lanes (g = lane / 16, i = lane % 16), for a tile of 32 tokens:
//   K as the left operand, piece by piece: lane has token i, channels 32 c + 8 g ... + 7 in step c
//   S comes out with head i, tokens 4 g + r: already the right operand of the second product, which takes
//     tokens 4 g + r of the first piece and of the second as its eight of lane (g, i)
//   V: lane loads, of its eight tokens, the kRun channels from kRun i (+ 128); row i of the left operand of product
//     t is channel kRun i + t, so that the lane has all of its operands' words and only swaps halves of registers
template <uint32_t kDim>
struct Layout {
    static constexpr uint32_t kSteps = kDim / 32;               // of the first product
    static constexpr uint32_t kRun = kDim == 64 ? 4 : 8;        // channels of V that a lane loads at once
    static constexpr uint32_t kParts = kDim == 256 ? 2 : 1;     // ... so many times
    static constexpr uint32_t kWords = kRun / 2;                // 32-bit words of that
    };

constexpr uint32_t kMergedHeads = 4;   // at a time
template <uint32_t kDim>
struct AttendShared {
    __align__(4096) uint8_t rows[kWaves][4 * 16 * 2 * kDim];
    union {
        float sum[kWaves][kMergedHeads][kDim + 4];
        struct {
            float top[kJoinedAtOnce][16], total[kJoinedAtOnce][16];
        } part;
    };
    float top[kWaves][16], total[kWaves][16];
    uint32_t last;
};

// A wavefront's tile, 32 rows of K and of V, goes to LDS as it comes, without a register: lanes ask for whole rows, sixteen
// for 256 bytes.  (Asked for in the layout of the first product, sixteen lanes would ask for sixteen rows of K, and the cache
// serve each by itself: 64 accesses an instruction instead of 16, 42 million for 1 GiB of cache instead of 17.)  Sixteen
// bytes p of row r of K are kept at place p ^ swap(r), so that those of sixteen rows lie in different banks.
template <uint32_t kDim>
struct Rows : Layout<kDim> {
    typedef Layout<kDim> L;
    static constexpr uint32_t kPlaces = kDim / 8;               // of a row
    static constexpr uint32_t kRowsAtOnce = 64 / kPlaces;       // that an instruction asks for
    static constexpr uint32_t kAsked = 16 / kRowsAtOnce;        // instructions a piece
    static constexpr uint32_t kPieceBytes = 16 * 2 * kDim, kBytes = 4 * kPieceBytes;

    uint32_t k_at[kAsked], v_at;   // where the lane's bytes lie from an instruction's first row on

    static __device__ __forceinline__ uint32_t swap(uint32_t row) { return kDim == 64 ? row / 2 % 8 : row % 16; }

    __device__ __forceinline__ Rows(const AttendArgs& a, uint32_t lane) {
        const uint32_t row = lane / kPlaces, there = a.head_dim / 8;   // (beyond the channels: anything that is there)
#pragma unroll
        for (uint32_t n = 0; n < kAsked; ++n) {
            const uint32_t p = (lane % kPlaces) ^ swap(n * kRowsAtOnce + row);
            k_at[n] = row * (uint32_t)a.k_token + 16 * (p < there ? p : 0);
        }
        v_at = row * (uint32_t)a.v_token + 16 * (lane % kPlaces < there ? lane % kPlaces : 0);
    }
    // Sixteen rows from `row` on, to `to`.  An instruction's constant offset counts on both sides, so that the place in LDS
    // is set for up to four of them at once.
    template <class At>
    static __device__ __forceinline__ void ask(uint64_t row, int64_t stride, uint8_t* to, At at) {
        const int64_t step = (int64_t)kRowsAtOnce * stride - 1024;
#pragma unroll
        for (uint32_t n = 0; n < kAsked; ++n) {
            asked<kAsked>(row + at(n), to + n / 4 * 4096, n % 4);
            row += n % 4 == 3 ? step + 4096 : step;
        }
    }
    template <uint32_t>
    static __device__ __forceinline__ void asked(uint64_t from, uint8_t* to, uint32_t n) {
        typedef const __attribute__((address_space(1))) void* Global;
        typedef __attribute__((address_space(3))) void* Lds;
        if (n == 0) __builtin_amdgcn_global_load_lds((Global)from, (Lds)to, 16, 0, 0);
        if (n == 1) __builtin_amdgcn_global_load_lds((Global)from, (Lds)to, 16, 1 * 1024, 0);
        if (n == 2) __builtin_amdgcn_global_load_lds((Global)from, (Lds)to, 16, 2 * 1024, 0);
        if (n == 3) __builtin_amdgcn_global_load_lds((Global)from, (Lds)to, 16, 3 * 1024, 0);
    }
    // k, v: addresses of the rows of the piece's first token; lds: K of both pieces, then V of both
    __device__ __forceinline__ void ask_piece(const AttendArgs& a, uint8_t* lds, uint32_t which, uint64_t k, uint64_t v) const {
        ask(k, a.k_token, lds + which * kPieceBytes, [&](uint32_t n) { return k_at[n]; });
        ask(v, a.v_token, lds + (2 + which) * kPieceBytes, [&](uint32_t) { return v_at; });
    }
};

// What a wavefront holds of a tile: K as the operand of the first product, V as rows.
template <class H, uint32_t kDim, bool kExact>
struct Held : Layout<kDim> {
    typedef Layout<kDim> L;
    uint4 k[2][L::kSteps];
    uint32_t v[L::kParts][8][L::kWords];

    __device__ __forceinline__ void take(const AttendArgs& a, const uint8_t* lds, uint32_t g, uint32_t i) {
#pragma unroll
        for (uint32_t c = 0; c < L::kSteps; ++c)
#pragma unroll
            for (uint32_t which = 0; which < 2; ++which) {
                k[which][c] = *(const uint4*)(lds + which * Rows<kDim>::kPieceBytes + i * 2 * kDim +
                                              ((4 * c + g) ^ Rows<kDim>::swap(i)) * 16);
                if (!kExact && 32 * c + 8 * g >= a.head_dim) k[which][c] = make_uint4(0, 0, 0, 0);
            }
#pragma unroll
        for (uint32_t p = 0; p < L::kParts; ++p)
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
                const uint8_t* at = lds + (2 + j / 4) * Rows<kDim>::kPieceBytes + (4 * g + j % 4) * 2 * kDim + 256 * p + 2 * L::kRun * i;
                if constexpr (L::kWords == 4) {
                    const uint4 x = *(const uint4*)at;
                    v[p][j][0] = x.x, v[p][j][1] = x.y, v[p][j][2] = x.z, v[p][j][3] = x.w;
                } else {
                    const uint2 x = *(const uint2*)at;
                    v[p][j][0] = x.x, v[p][j][1] = x.y;
                }
            }
    }
    // Finite, or in some lane not if any of the wavefront's values is not: their products with whatever is at hand, as the matrix
    // cores make them beside those of the scores, which wait for each other.  Rows that are not there, queries that are not
    // finite and sums beyond the range of binary32 may make it infinite or NaN, which costs time alone.  (12 requests of up to
    // 1000 tokens, 8 kv heads of 256: 19.9 us, by dot products with zero 20.6, without 19.1; two of 131 059 tokens equal.)
    __device__ __forceinline__ float probe(typename H::eight by) const {
        f32x4 sums[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (uint32_t p = 0; p < L::kParts; ++p)
#pragma unroll
            for (uint32_t j = 0; j < 8; j += 4 / L::kWords) {   // (as they came from LDS: no register moves)
                const uint32_t n = j / (4 / L::kWords) % 2;
                const uint4 x = L::kWords == 4 ? make_uint4(v[p][j][0], v[p][j][1], v[p][j][L::kWords - 2], v[p][j][L::kWords - 1])
                                               : make_uint4(v[p][j][0], v[p][j][1], v[p][j + 1 & 7][0], v[p][j + 1 & 7][1]);
                sums[n] = H::product(as_eight<H>(x), by, sums[n]);
            }
        sums[0] += sums[1];
        return (sums[0][0] + sums[0][1]) + (sums[0][2] + sums[0][3]);
    }
    // rows of tokens that are not there count as zero, whatever they hold
    __device__ __forceinline__ void drop_v(uint32_t which, uint32_t valid, uint32_t g) {
#pragma unroll
        for (uint32_t p = 0; p < L::kParts; ++p)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r)
#pragma unroll
                for (uint32_t w = 0; w < L::kWords; ++w)
                    v[p][4 * which + r][w] = 4 * g + r < valid ? v[p][4 * which + r][w] : 0u;
    }
};

template <class H, uint32_t kDim, bool kExact>
struct Walk : Layout<kDim> {
    typedef Layout<kDim> L;
    f32x4 sum[L::kParts][L::kRun];
    float top, total;
    uint4 q[L::kSteps];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (uint32_t p = 0; p < L::kParts; ++p)
#pragma unroll
            for (uint32_t t = 0; t < L::kRun; ++t) sum[p][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        top = -INFINITY;
        total = 0.f;
    }
    __device__ __forceinline__ void load_q(const AttendArgs& a, const uint8_t* row, bool there, uint32_t g) {
#pragma unroll
        for (uint32_t c = 0; c < L::kSteps; ++c) {
            const uint32_t d = 32 * c + 8 * g;
            q[c] = make_uint4(0, 0, 0, 0);
            if (there && (kExact || d < a.head_dim)) q[c] = *(const uint4*)(row + 2 * d);
        }
    }
    // ... and the values' probe, in the products' shadow
    __device__ __forceinline__ float scores(float (&s)[8], const Held<H, kDim, kExact>& held, float scale, uint32_t valid0,
                                            uint32_t valid1, uint32_t g) const {
        f32x4 s0{0.f, 0.f, 0.f, 0.f}, s1{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (uint32_t c = 0; c < L::kSteps; ++c) {
            s0 = H::product(as_eight<H>(held.k[0][c]), as_eight<H>(q[c]), s0);
            s1 = H::product(as_eight<H>(held.k[1][c]), as_eight<H>(q[c]), s1);
        }
        float probe = held.probe(as_eight<H>(q[0]));
        asm volatile("" : "+v"(probe));   // (it would be made where it is looked at)
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) s[r] = s0[r] * scale, s[4 + r] = s1[r] * scale;
        if (valid0 < kPiece || valid1 < kPiece) {
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                s[r] = 4 * g + r < valid0 ? s[r] : -INFINITY;
                s[4 + r] = 4 * g + r < valid1 ? s[4 + r] : -INFINITY;
            }
        }
        return probe;
    }
    // Sums are kept relative to 2^top, which makes the largest weight so far 2^H::kLargest when they were last brought up to
    // it, and at most 2^H::kOverflows before the next time: a new maximum rarely takes that.  The scores become weights.
    __device__ __forceinline__ void weigh(float (&s)[8]) {
        float most = s[0];
#pragma unroll
        for (uint32_t j = 1; j < 8; ++j) most = fmaxf(most, s[j]);
        most = over_rows_max(most);
        if (__any(most > top + H::kOverflows || (top == -INFINITY && most > top))) {
            const float now = fmaxf(most - H::kLargest, top), keep = exp2_from(top, now);
            top = now;
            total *= keep;
#pragma unroll
            for (uint32_t p = 0; p < L::kParts; ++p)
#pragma unroll
                for (uint32_t t = 0; t < L::kRun; ++t) sum[p][t] *= keep;
        }
        const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            s[j] = __builtin_amdgcn_exp2f(s[j] - from);
            total += s[j];
        }
    }
    // Eight rows' words of two channels as the left operand of one of them
    static __device__ __forceinline__ typename H::eight channel(const uint32_t (&rows)[8], uint32_t second) {
        const uint32_t pick = second ? 0x07060302u : 0x05040100u;
        return as_eight<H>(make_uint4(__builtin_amdgcn_perm(rows[1], rows[0], pick), __builtin_amdgcn_perm(rows[3], rows[2], pick),
                                      __builtin_amdgcn_perm(rows[5], rows[4], pick), __builtin_amdgcn_perm(rows[7], rows[6], pick)));
    }
    // Values that are not finite are added with a weight of 1, if theirs is not 0, and leave the rows: a half of a weight may be
    // 0 where the weight is not, and 0 times infinity is no number.
    __device__ __forceinline__ void add_odd(const float (&s)[8], Held<H, kDim, kExact>& held) {
        typename H::eight any;
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) any[j] = (typename H::one)(s[j] != 0.f ? 1.f : 0.f);
        constexpr uint32_t kInf = H::kInfinity;
#pragma unroll
        for (uint32_t p = 0; p < L::kParts; ++p)
#pragma unroll
            for (uint32_t w = 0; w < L::kWords; ++w) {
                uint32_t odd[8];
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) {
                    const uint32_t word = held.v[p][j][w];
                    const uint32_t of = ((word & kInf) == kInf ? 0xFFFFu : 0u) |
                                        ((word & kInf << 16) == kInf << 16 ? 0xFFFF0000u : 0u);
                    odd[j] = word & of;
                    held.v[p][j][w] = word & ~of;
                }
                sum[p][2 * w] = H::product(channel(odd, 0), any, sum[p][2 * w]);
                sum[p][2 * w + 1] = H::product(channel(odd, 1), any, sum[p][2 * w + 1]);
            }
    }
    __device__ __forceinline__ void add_v(const float (&s)[8], Held<H, kDim, kExact>& held, float probe) {
        if (__builtin_expect(__any(!(fabsf(probe) < INFINITY)), false)) add_odd(s, held);
        // A weight goes to the matrix cores in halves, each of what the ones before leave: in bfloat16 all of its 24 bits, in
        // float16 at least 22.  (Two of 8 bits each were off by up to 2^-17 of a sum's size where values cancel, and three cost
        // little beside memory: two requests of 131 059 tokens 200.3 us, with two 199.2.)
        typename H::eight halves[H::kHalves];
        H::split(s, halves);
        typename H::eight x[L::kParts][L::kRun];
#pragma unroll
        for (uint32_t p = 0; p < L::kParts; ++p)
#pragma unroll
            for (uint32_t t = 0; t < L::kRun; ++t) {
                const uint32_t rows[8] = {held.v[p][0][t / 2], held.v[p][1][t / 2], held.v[p][2][t / 2], held.v[p][3][t / 2],
                                          held.v[p][4][t / 2], held.v[p][5][t / 2], held.v[p][6][t / 2], held.v[p][7][t / 2]};
                x[p][t] = channel(rows, t % 2);
                sum[p][t] = H::product(x[p][t], halves[0], sum[p][t]);
            }
#pragma unroll
        for (uint32_t n = 1; n < H::kHalves; ++n)
#pragma unroll
            for (uint32_t p = 0; p < L::kParts; ++p)
#pragma unroll
                for (uint32_t t = 0; t < L::kRun; ++t) sum[p][t] = H::product(x[p][t], halves[n], sum[p][t]);
    }
};

// What a workgroup walks over at a time: up to 32 tiles of an item.
struct Segment {
    uint32_t request, before, tiles;  // the request's first tile of all, and the tiles of each of its items
    uint32_t item, tile, tile_to;     // of the request; of the item
};

// Where a wavefront's pieces of a segment lie: lane l has its l-th, two of each tile.
struct Pieces {
    uint32_t block;          // number; anything out of the pool, e.g. ~0: masked
    uint32_t inside, valid;  // token of the block; how many of its sixteen are there
};
template <bool kShort>
__device__ __forceinline__ Pieces find_pieces(const AttendArgs& a, const Segment& s, uint32_t wave, uint32_t lane) {
    Pieces p{~0u, 0u, 0u};
    const uint32_t t = s.tile + lane / 2;
    if (t >= s.tile_to) return p;
    const uint32_t piece = t * (kTileTokens / kPiece) + 2 * wave + (lane & 1);
    const uint32_t per_block = a.block_tokens / kPiece;
    uint32_t place = piece / per_block;
    const uint32_t inside = (piece - place * per_block) * kPiece;
    if (a.selected != nullptr) {
        if (place >= a.keep) return p;
        place = (uint32_t)a.selected[((size_t)s.request * a.kv_heads + s.item / a.group_tiles) * a.keep + place];
    }
    if (place >= a.row_blocks) return p;
    uint32_t block = 0;
    if constexpr (kShort) block = (uint32_t)a.tables[s.request * a.table_row + place];   // on its way with the length
    const uint32_t len = clamped_len(a, len_of(a, s.request));
    const uint64_t token = (uint64_t)place * a.block_tokens + inside;
    if (token >= len) return p;
    p.valid = len - token < kPiece ? (uint32_t)(len - token) : kPiece;
    p.inside = inside;
    if constexpr (!kShort) block = (uint32_t)a.tables[s.request * a.table_row + place];
    p.block = block;   // (looked at when it is used)
    return p;
}

// kShort: a workgroup for each item of all requests, also of those without tokens, whose rows have room for at most 32 tiles.
template <class H, uint32_t kDim, bool kExact, bool kShort>
__global__ __launch_bounds__(kThreads, kDim == 256 ? 1 : 2) void attend_kernel(AttendArgs a) {
    typedef Walk<H, kDim, kExact> W;
    __shared__ AttendShared<kDim> shared;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t g = lane / 16, i = lane % 16;
    const uint32_t per_request = a.kv_heads * a.group_tiles;

    // The tiles of all items
    // requests with any; all tiles; the most of a request; those of request `lane`, or of the last 64
    uint32_t some = 0, all = 0, longest = 0, tiles = 0;
    uint32_t groups = 1;
    bool whole = false;
    if constexpr (!kShort) {
        for (uint32_t b0 = 0; b0 < a.requests; b0 += 64) {
            const uint32_t b = b0 + lane;
            tiles = b < a.requests ? tiles_of(a, b) : 0;
            all += __builtin_amdgcn_readlane(scan(tiles), 63);
            some += __builtin_popcountll(__ballot(tiles != 0));
            longest = tiles > longest ? tiles : longest;
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
        some *= per_request;
        if (all == 0) return;
        longest = over_wave(longest, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
        whole = longest <= (some >= kManyItems ? kWholeTilesOfMany : kWholeTiles) && some <= gridDim.x;
        // ... in the order of requests and heads, are cut into equal spans (of one tile more or less), or at the items' ends: this
        // workgroup's is [from, to).
        const uint32_t by_tiles = all / some <= kShortItem ? all : (all + 1) / 2, useful = by_tiles > some ? by_tiles : some;
        // (of 256 channels, two workgroups have no room on a compute unit)
        const bool alone = kDim == 256 || (all / some >= kLongItem && all >= kManyTiles * kCus);
        groups = alone && gridDim.x > kCus ? kCus : gridDim.x;
        if (groups > useful) groups = useful;
        if (whole) groups = some;
        if (blockIdx.x >= groups) return;
    }
    const uint32_t share = all / groups, longer = all - share * groups;   // the first `longer` spans have one tile more
    auto start_of = [&](uint32_t w) { return w * share + (w < longer ? w : longer); };
    auto owner_of = [&](uint32_t tile) {
        const uint32_t in_longer = longer * (share + 1), x = tile - longer;   // (x: less what the longer ones have more)
        return tile < in_longer ? tile / (share + 1) : x / share;
    };
    uint32_t from = start_of(blockIdx.x), to = start_of(blockIdx.x + 1);
    uint32_t request = 0, before = 0;
    if constexpr (!kShort) {
        // the request that the span begins in, and its first tile
        for (uint32_t b0 = 0, sum = 0, there = 0; b0 < a.requests; b0 += 64) {
            if (a.requests > 64) tiles = b0 + lane < a.requests ? tiles_of(a, b0 + lane) : 0;
            const uint32_t upto = sum + scan(tiles);
            const uint64_t any = __ballot(tiles != 0);
            const uint32_t nth = there + __builtin_popcountll(any & (2ull << lane) - 1);   // of those with any
            const uint64_t past = __ballot(whole ? nth * per_request > blockIdx.x : upto * per_request > from);
            if (past != 0) {
                const uint32_t at = __builtin_ctzll(past);
                request = b0 + at;
                before = __builtin_amdgcn_readlane(upto - tiles, at) * per_request;
                if (whole) {
                    const uint32_t its = __builtin_amdgcn_readlane(tiles, at), n = __builtin_amdgcn_readlane(nth, at) - 1;
                    from = before + (blockIdx.x - n * per_request) * its;
                    to = from + its;
                }
                break;
            }
            sum = __builtin_amdgcn_readlane(upto, 63);
            there += __builtin_popcountll(any);
        }
        request = __builtin_amdgcn_readfirstlane(request);
        before = __builtin_amdgcn_readfirstlane(before);
        from = __builtin_amdgcn_readfirstlane(from);
        to = __builtin_amdgcn_readfirstlane(to);
    }

    // the segment that begins at a tile
    auto segment_at = [&](uint32_t at, uint32_t request, uint32_t before) {
        Segment s{request, before, tiles_of(a, request), 0, 0, 0};
        while (at >= s.before + s.tiles * per_request) {
            s.before += s.tiles * per_request;
            s.tiles = tiles_of(a, ++s.request);
        }
        s.item = (at - s.before) / s.tiles;
        const uint32_t item_from = s.before + s.item * s.tiles;
        s.tile = at - item_from;
        const uint32_t item_to = item_from + s.tiles, end = to < item_to ? to : item_to;
        s.tile_to = end - at < 32 ? end - item_from : s.tile + 32;
        return s;
    };

    W walk;
    const Rows<kDim> rows(a, lane);
    // of the segment's pieces, lane by lane: how many tokens are there (none: masked), and where their rows lie
    uint32_t piece_valid;
    uint64_t piece_k, piece_v;
    uint64_t live;                  // those that are not masked, from the tile in hand on
    uint32_t valid0, valid1, in_segment;   // the next tile
    uint64_t k0, k1, v0, v1;
    auto lane_of = [](uint64_t x, uint32_t j) {
        const uint32_t low = __builtin_amdgcn_readlane((uint32_t)x, j), high = __builtin_amdgcn_readlane((uint32_t)(x >> 32), j);
        return (uint64_t)high << 32 | low;   // (what comes from a lane is an int)
    };
    // the next tile that is not masked as a whole, if there is one
    auto seek = [&]() {
        if (live == 0) return false;
        const uint32_t j = __builtin_ctzll(live) & ~1u;
        in_segment = j / 2;
        live &= ~(3ull << j);
        valid0 = __builtin_amdgcn_readlane(piece_valid, j), valid1 = __builtin_amdgcn_readlane(piece_valid, j + 1);
        k0 = lane_of(piece_k, j), k1 = lane_of(piece_k, j + 1), v0 = lane_of(piece_v, j), v1 = lane_of(piece_v, j + 1);
        return true;
    };
    auto use_pieces = [&](const Pieces& p, const Segment& s) {
        const uint32_t head = s.item / a.group_tiles;
        const bool there = p.block < a.blocks;
        piece_valid = there ? p.valid : 0;
        live = __ballot(there);
        piece_k = (uint64_t)(uintptr_t)a.k + head * a.k_head + p.block * a.k_block + p.inside * a.k_token;
        piece_v = (uint64_t)(uintptr_t)a.v + head * a.v_head + p.block * a.v_block + p.inside * a.v_token;
        // A masked piece of a tile that is not masked as a whole has the other one's rows, which are there.
        const uint64_t other_k = __shfl_xor(piece_k, 1), other_v = __shfl_xor(piece_v, 1);
        piece_k = there ? piece_k : other_k;
        piece_v = there ? piece_v : other_v;
    };
    uint8_t* const lds = shared.rows[wave];
    auto ask = [&]() {
        rows.ask_piece(a, lds, 0, k0, v0);
        rows.ask_piece(a, lds, 1, k1, v1);
    };
    auto load_query = [&](const Segment& s) {
        const uint32_t head0 = s.item % a.group_tiles * 16, first = s.item / a.group_tiles * a.group + head0;
        const bool there = i < a.group - head0;
        walk.load_q(a, a.q + s.request * a.q_request + (first + (there ? i : 0)) * a.q_head, there, g);
    };

    uint32_t at = from;
    Segment now;
    if constexpr (kShort) {
        const uint32_t most = ((a.selected == nullptr ? a.row_blocks : a.keep) * a.block_tokens + kTileTokens - 1) / kTileTokens;
        request = blockIdx.x / per_request;
        now = Segment{request, 0, most, blockIdx.x - request * per_request, 0, most};
    } else {
        now = segment_at(at, request, before);
    }
    use_pieces(find_pieces<kShort>(a, now, wave, lane), now);
    bool some_left = seek();
    walk.clear();
    load_query(now);
    if (some_left) ask();
    while (true) {
        at += now.tile_to - now.tile;
        const bool more = !kShort && at < to;
        Segment next = now;
        Pieces next_pieces{~0u, 0u, 0u};
        if (more) {         // where the next segment's pieces lie is asked for while this one is walked over
            next = segment_at(at, now.request, now.before);
            next_pieces = find_pieces<kShort>(a, next, wave, lane);
        }
        const uint32_t head0 = now.item % a.group_tiles * 16, first_head = now.item / a.group_tiles * a.group + head0;
        const uint32_t heads = a.group - head0 < 16 ? a.group - head0 : 16;
        bool ahead = false, turned = false;    // the next segment's first tile is asked for; its pieces are in use
        while (some_left) {
            const uint32_t here0 = valid0, here1 = valid1;
            const uint32_t piece0 = (now.tile + in_segment) * (kTileTokens / kPiece) + 2 * wave;
            Held<H, kDim, kExact> held;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the tile's rows are in LDS
            held.take(a, lds, g, i);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // ... and have left it
            // all rows of the next tile are asked for at once, and are under way while this one is worked on
            some_left = seek();
            if (!some_left && more) {
                turned = true;
                use_pieces(next_pieces, next);
                ahead = seek();
            }
            if (some_left || ahead) ask();
            float s[8];
            const float probe = walk.scores(s, held, a.scale, here0, here1, g);
            walk.weigh(s);
            if (a.piece_lse != nullptr) {
                const float w0 = over_rows_sum((s[0] + s[1]) + (s[2] + s[3]));
                const float w1 = over_rows_sum((s[4] + s[5]) + (s[6] + s[7]));
                if (g == 0 && i < heads) {
                    const uint32_t per_row = a.row_blocks * (a.block_tokens / kPiece);
                    float* to_row = a.piece_lse + ((size_t)now.request * a.kv_heads * a.group + first_head + i) * per_row + piece0;
                    // (a row's last tile may be cut by its end)
                    if (here0 != 0) to_row[0] = walk.top + __builtin_amdgcn_logf(w0);
                    if (here1 != 0) to_row[1] = walk.top + __builtin_amdgcn_logf(w1);
                }
            }
            if (here0 < kPiece || here1 < kPiece) {
                held.drop_v(0, here0, g);
                held.drop_v(1, here1, g);
            }
            walk.add_v(s, held, probe);
        }
        if (more && !turned) {
            use_pieces(next_pieces, next);
            ahead = seek();
            if (ahead) ask();
        }
        some_left = ahead;
        const bool same = more && next.request == now.request && next.item == now.item;
        if (more && !same) load_query(next);   // under way while this item is finished
        if (same) {
            now = next;
            continue;
        }

        // The wavefronts' results as one.  A lane holds, of head i, channels kRun (4 g + r) + t.
        walk.total = over_rows_sum(walk.total);
        if (g == 0 && i < heads) {
            shared.top[wave][i] = walk.top;
            shared.total[wave][i] = walk.total;
        }

        auto finish = [&](uint32_t h, uint32_t d, float4 x, float top, float total) {
            const float by = total == 0.f ? 0.f : 1.f / total;   // (a NaN stays one)
            const uint32_t out_head = first_head + h;
            if (d < a.head_dim) {
                typename H::one y[4] = {(typename H::one)(x.x * by), (typename H::one)(x.y * by),
                                        (typename H::one)(x.z * by), (typename H::one)(x.w * by)};
                uint2 words;
                __builtin_memcpy(&words, y, 8);
                *(uint2*)(a.out + now.request * a.out_request + out_head * a.out_head + 2 * d) = words;
            }
            if (d == 0) {
                const float of_head = total == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(total);
                const size_t n = (size_t)now.request * a.kv_heads * a.group + out_head;
                if (a.lse != nullptr) a.lse[n] = of_head * 0.693147180559945f;
                if (a.piece_lse != nullptr) a.head_lse[n] = of_head;
            }
        };

        const uint32_t item_from = now.before + now.item * now.tiles, item_to = item_from + now.tiles;
        uint32_t first_part = blockIdx.x, parts = 1;
        if (!kShort && (item_from < from || item_to > to)) {
            first_part = owner_of(item_from);
            parts = owner_of(item_to - 1) - first_part + 1;
        }
        constexpr uint32_t kQuads = kDim / 4;
        const uint32_t rows_kept = a.group < 16 ? a.group : 16;
        const size_t part_floats = (size_t)rows_kept * (kDim + 2);   // sums, then tops and totals
        // (a workgroup's first item and its last one are the two of several parts)
        auto slot_of = [&](uint32_t w) { return 2 * w + (item_from > start_of(w) ? 1 : 0); };
        auto part_at = [&](uint32_t w) { return a.partials + slot_of(w) * part_floats; };
        float* slot = part_at(blockIdx.x);
        auto put_part = [&](float* part, uint32_t h, uint32_t d, float4 sum, float top, float total) {
            uint64_t* to_sum = (uint64_t*)(part + h * kDim + d);
            put_shared(to_sum, __builtin_bit_cast(uint64_t, make_float2(sum.x, sum.y)));
            put_shared(to_sum + 1, __builtin_bit_cast(uint64_t, make_float2(sum.z, sum.w)));
            if (d == 0)
                put_shared((uint64_t*)(part + rows_kept * kDim) + h, __builtin_bit_cast(uint64_t, make_float2(top, total)));
        };
        for (uint32_t h0 = 0; h0 < heads; h0 += kMergedHeads) {
            const uint32_t these = heads - h0 < kMergedHeads ? heads - h0 : kMergedHeads;
            __syncthreads();
            if (i - h0 < these) {
#pragma unroll
                for (uint32_t p = 0; p < W::kParts; ++p)
#pragma unroll
                    for (uint32_t r = 0; r < 4; ++r)
#pragma unroll
                        for (uint32_t t = 0; t < W::kRun; t += 4)
                            *(float4*)&shared.sum[wave][i - h0][128 * p + W::kRun * (4 * g + r) + t] = make_float4(
                                walk.sum[p][t][r], walk.sum[p][t + 1][r], walk.sum[p][t + 2][r], walk.sum[p][t + 3][r]);
            }
            __syncthreads();
            for (uint32_t x = threadIdx.x; x < these * kQuads; x += kThreads) {
                const uint32_t h = x / kQuads, d = x % kQuads * 4;
                float top = shared.top[0][h0 + h];
#pragma unroll
                for (uint32_t w = 1; w < kWaves; ++w) top = fmaxf(top, shared.top[w][h0 + h]);
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
                float total = 0.f;
#pragma unroll
                for (uint32_t w = 0; w < kWaves; ++w) {
                    const float by = exp2_from(shared.top[w][h0 + h], top);
                    const float4 y = *(const float4*)&shared.sum[w][h][d];
                    total += shared.total[w][h0 + h] * by;
                    sum.x += y.x * by, sum.y += y.y * by, sum.z += y.z * by, sum.w += y.w * by;
                }
                if (parts == 1) {
                    finish(h0 + h, d, sum, top, total);
                } else {
                    put_part(slot, h0 + h, d, sum, top, total);
                }
            }
        }
        // The parts' results as one: those of workgroups first, first + apart, ..., to the outputs or to the first's place.
        // (Loads of eight words under way together: sixteen take registers from the walk, 22.2 us and 19.7 for 480 items of 64
        // channels; four 36.6 and 34.9 for two items of 16 heads.)
        constexpr uint32_t kMine = (16 * kQuads + kThreads - 1) / kThreads, kTogether = 8 / kMine;
        auto join = [&](uint32_t first, uint32_t apart, uint32_t count, bool last) {
            for (uint32_t x = threadIdx.x; x < count * heads; x += kThreads) {
                const uint32_t p = x / heads, h = x - p * heads;
                const float2 y = __builtin_bit_cast(
                    float2, get_shared((const uint64_t*)(part_at(first + p * apart) + rows_kept * kDim) + h));
                shared.part.top[p][h] = y.x;
                shared.part.total[p][h] = y.y;
            }
            __syncthreads();
            float4 sum[kMine];
            float top[kMine], total[kMine];
#pragma unroll
            for (uint32_t n = 0; n < kMine; ++n) {
                const uint32_t x = threadIdx.x + n * kThreads, h = x / kQuads;
                sum[n] = make_float4(0.f, 0.f, 0.f, 0.f), top[n] = -INFINITY, total[n] = 0.f;
                if (x < heads * kQuads)
                    for (uint32_t p = 0; p < count; ++p) top[n] = fmaxf(top[n], shared.part.top[p][h]);
            }
            for (uint32_t p0 = 0; p0 < count; p0 += kTogether) {
                uint64_t y[kTogether][kMine][2];   // under way together
#pragma unroll
                for (uint32_t e = 0; e < kTogether; ++e) {
                    const uint32_t p = p0 + e < count ? p0 + e : p0;
                    const float* from = part_at(first + p * apart);
#pragma unroll
                    for (uint32_t n = 0; n < kMine; ++n) {
                        const uint32_t x = threadIdx.x + n * kThreads;
                        const uint64_t* at_sum = (const uint64_t*)(from + 4 * (x < heads * kQuads ? x : 0));
                        y[e][n][0] = get_shared(at_sum), y[e][n][1] = get_shared(at_sum + 1);
                    }
                }
#pragma unroll
                for (uint32_t n = 0; n < kMine; ++n) {
                    const uint32_t x = threadIdx.x + n * kThreads, h = x / kQuads;
                    if (x >= heads * kQuads) continue;
#pragma unroll
                    for (uint32_t e = 0; e < kTogether; ++e) {
                        if (p0 + e >= count) break;
                        const float2 u = __builtin_bit_cast(float2, y[e][n][0]), v = __builtin_bit_cast(float2, y[e][n][1]);
                        const float by = exp2_from(shared.part.top[p0 + e][h], top[n]);
                        total[n] += shared.part.total[p0 + e][h] * by;
                        sum[n].x += u.x * by, sum[n].y += u.y * by, sum[n].z += v.x * by, sum[n].w += v.y * by;
                    }
                }
            }
            float* to_part = part_at(first);
#pragma unroll
            for (uint32_t n = 0; n < kMine; ++n) {
                const uint32_t x = threadIdx.x + n * kThreads, h = x / kQuads, d = x % kQuads * 4;
                if (x >= heads * kQuads) continue;
                if (last) finish(h, d, sum[n], top[n], total[n]);
                else put_part(to_part, h, d, sum[n], top[n], total[n]);
            }
        };
        if (parts > 1) {
            // in one go, or in groups of as many as there are groups
            uint32_t fan = parts;
            if (parts * ((heads * kQuads + kThreads - 1) / kThreads) > kJoinedAtOnce)
                for (fan = 4; fan * fan < parts;) ++fan;
            const uint32_t mine = (blockIdx.x - first_part) / fan * fan, count = parts - mine < fan ? parts - mine : fan;
            bool last = last_to_arrive(a.counters + slot_of(first_part + mine), count, &shared.last);
            if (last) {
                join(first_part + mine, 1, count, fan == parts);
                const uint32_t groups_of = (parts + fan - 1) / fan;
                if (fan < parts && last_to_arrive(a.counters + 2 * kAttendGroups + slot_of(first_part), groups_of, &shared.last))
                    join(first_part, fan, groups_of, true);
            }
        }
        if (!more) return;
        __syncthreads();   // (what is in LDS of this item has been read)
        walk.clear();
        now = next;
    }
}

// weights[b][j] = decay kept[b][j] + sum over heads and pieces of 2^(piece - head): 64 blocks a workgroup, a quarter of
// the heads each wavefront, added up in their order.  Few bytes, so the trips to memory bound it: 32 requests of up to 128
// blocks, 40 heads: 5.6 us, with one head's load at a time 11.3.
__global__ __launch_bounds__(kThreads) void weights_kernel(AttendArgs a, const float* kept, float* weights, float decay) {
    __shared__ float quarter[kWaves][64];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, request = blockIdx.y;
    const uint32_t j = blockIdx.x * 64 + lane, heads = a.kv_heads * a.group, per_block = a.block_tokens / kPiece;
    const uint32_t len = clamped_len(a, len_of(a, request));
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

template <class H, bool kShort>
void launch(const AttendArgs& a, uint32_t groups, hipStream_t stream) {
    const uint32_t d = a.head_dim;
    if (d == 64) attend_kernel<H, 64, true, kShort><<<groups, kThreads, 0, stream>>>(a);
    else if (d < 64) attend_kernel<H, 64, false, kShort><<<groups, kThreads, 0, stream>>>(a);
    else if (d == 128) attend_kernel<H, 128, true, kShort><<<groups, kThreads, 0, stream>>>(a);
    else if (d < 128) attend_kernel<H, 128, false, kShort><<<groups, kThreads, 0, stream>>>(a);
    else if (d == 256) attend_kernel<H, 256, true, kShort><<<groups, kThreads, 0, stream>>>(a);
    else attend_kernel<H, 256, false, kShort><<<groups, kThreads, 0, stream>>>(a);
}
template <class H>
void launch(const AttendArgs& a, uint32_t groups, bool by_item, hipStream_t stream) {
    if (by_item) launch<H, true>(a, groups, stream);
    else launch<H, false>(a, groups, stream);
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
    // (lanes' places within sixteen rows are counted in 32 bits)
    if (cache->k_token < 0 || cache->k_token > kMostTokenStride || cache->v_token < 0 || cache->v_token > kMostTokenStride)
        return PGCM_ERR_ARG;
    if (!aligned(args->q, args->q_request, args->q_head) || !aligned(args->out, args->out_request, args->out_head))
        return PGCM_ERR_ALIGN;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const bool weigh = args->weights != nullptr;
    const uint64_t row_pieces = (uint64_t)args->row_blocks * (cache->block_tokens / kPiece);
    const Room room = attend_room(args->requests, args->heads, cache->kv_heads, cache->head_dim, weigh ? row_pieces : 0);
    const std::lock_guard<std::mutex> held(kv->enqueue);
    if (const int rc = kv_ensure(kv, room.counters, room.scratch, stream)) return rc;

    AttendArgs a{};
    a.k = (const uint8_t*)cache->k, a.v = (const uint8_t*)cache->v, a.q = (const uint8_t*)args->q;
    a.out = (uint8_t*)args->out;
    a.tables = args->tables, a.lens = args->lens, a.selected = args->selected, a.lse = args->lse;
    a.counters = (uint32_t*)kv->counters.at;
    uint8_t* at = kv->scratch.at;
    a.partials = (float*)at;
    at += whole_lines(4 * partial_floats(cache->head_dim, args->heads / cache->kv_heads) * 2 * kAttendGroups);
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
    const uint64_t items = (uint64_t)a.requests * a.kv_heads * a.group_tiles, most = tiles * items;
    const uint64_t useful = most > items ? most : items;
    // Room for few tiles only: a workgroup for each item, which looks at no lengths but its own request's and cuts and joins
    // nothing.  Microseconds of that and of the general kernel, for rows that are full and "ragged" ones (down to a sixteenth):
    //   one request of 33 tokens, 40 heads of 128: 4.3 and 6.4
    //   128 channels  8 items, 6 tiles 9.7 and 9.6, 8 tiles 11.6 and 9.7; 32, 6 tiles 10.2 and 10.5, ragged 9.6 and 10.4, 8 tiles
    //                 12.1 and 11.6, ragged 11.5 and 10.6; 96, 8 tiles 12.7 and 15.3, ragged 12.1 and 15.1, 10 tiles 14.5 and
    //                 17.9, ragged 14.0 and 13.3, 12 tiles 16.4 and 19.8, ragged 15.8 and 13.8; 64, 16 tiles 20.0 and 17.9,
    //                 ragged 19.8 and 14.4; 160, 12 tiles 27.6 and 30.4, ragged 16.4 and 18.6; 256, 16 tiles 51.7 and 53.7,
    //                 ragged 22.8 and 24.2, but 512 99.6 and 97.9, 46.4 and 45.9
    //   256 channels  96 items, 8 tiles 27.4 and 30.7, ragged 20.4 and 25.4, 10 tiles 34.6 and 35.8, ragged 23.8 and 21.7; 160,
    //                 12 tiles 50.3 and 56.3, ragged 30.6 and 29.6
    // Lists of a selection are as good as full, and worth more tiles: 64 items, 12 tiles 16.3 and 16.6, 16 tiles 20.1 and 18.2;
    // 96, 14 tiles 20.1 and 24.0, 16 tiles 24.5 and 24.6, 18 tiles 28.5 and 26.4; 128, 16 tiles 30.6 and 30.6; 256, 16 tiles 46
    // and 54; of 256 channels 64 items, 12 tiles 33.7 and 24.8, 128, 12 tiles 43.1 and 44.9.
    const bool wide = a.head_dim > 128, many = items >= kCus / 2;
    const uint32_t whole_tiles = items < kManyItems          ? 6
                                 : args->selected == nullptr ? (many ? 12 : wide ? 8 : 10)
                                                             : (many || (items >= 96 && !wide) ? 16 : wide ? 10 : 12);
    const bool by_item = items < 1 << 24 && tiles <= whole_tiles;   // (threads of a grid are counted in 32 bits)
    const uint32_t groups = by_item ? (uint32_t)items : useful > kAttendGroups ? kAttendGroups : (uint32_t)useful;
    if (cache->half == PGCM_KV_F16) launch<F16>(a, groups, by_item, stream);
    else launch<Bf16>(a, groups, by_item, stream);
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
