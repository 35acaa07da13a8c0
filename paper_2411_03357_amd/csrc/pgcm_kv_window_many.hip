// Attention of many new tokens of each request over KV blocks of halves, with a window (include/pgcm_kv8.h), on the matrix cores.
//
// New tokens and the query heads of a kv head make its rows, token by token; 128 of them (an "item") walk over what they see in
// tiles of 64 tokens, each of a workgroup's four wavefronts with 32 rows:
//   S' = K Q',  P' = 2^(S' - m),  O' = V' P'     (transposed, so that P' comes out as the right operand that it goes in as)
// with running m and sums.  Where there are few items, each is cut into parts, whose results a second kernel puts together.
// Weights are sums of two halves, so the second product is made twice (see there).  What bounds it are the matrix cores, busy 60 % of
// the cycles, and vector instructions, under way in 49 %: the two wavefronts of a SIMD hide little more of one behind the other, at
// a clock that falls to 1.8 GHz.  (LDS: 50 % of the cycles by the bytes, 4 % of all waits.)  Four prompts of up to 16384 tokens, 32
// heads of 128, window 4096 (1.12 TFLOP): 1.52 to 1.54 ms, 727 to 738 TFLOP/s, where a library's product of 8192^3 reaches 1247; 512
// tokens behind 65536, window 16384 (0.14 TFLOP, 512 parts): 207 to 240 us.
//
// K and V go to LDS without registers, two tiles by turns, and the lanes read them from there without conflicts of banks, V across
// its rows (ds_read_b64_tr_b16), as the left operand of the second product has tokens side by side.  A wavefront has 32 rows: two
// workgroups a compute unit, one of which multiplies while the other weighs.  (A tile in two halves, the products of one beside the
// exponentials of the other in the same wavefront: 3 % slower.)
#include "pgcm_kv_window.h"

namespace pgcm_kv_impl {
namespace {

constexpr uint32_t kWaves = 4, kThreads = kWaves * 64, kRows = 32 * kWaves;
constexpr uint32_t kTile = 64, kTilePieces = kTile / kPiece;
constexpr uint32_t kManyGroups = 512;    // workgroups that the chip holds at once
constexpr uint32_t kLeastTiles = 8;      // of a part
constexpr uint32_t kMostParts = 1024;    // of all items, where they are cut
static_assert(kTilePieces == kWaves, "a wavefront asks for a piece of a tile");

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class H>
struct Wide;
template <>
struct Wide<F16> {
    static __device__ __forceinline__ f32x16 product(uint4 a, uint4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(as_eight<F16>(a), as_eight<F16>(b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ void split(const float (&x)[8], uint4 (&halves)[2]) {   // all but 2^-22
        F16::eight y[2];
        F16::split(x, y);
        halves[0] = as_words<F16>(y[0]), halves[1] = as_words<F16>(y[1]);
    }
};
template <>
struct Wide<Bf16> {
    static __device__ __forceinline__ f32x16 product(uint4 a, uint4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_eight<Bf16>(a), as_eight<Bf16>(b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ void split(const float (&x)[8], uint4 (&halves)[2]) {   // all but 2^-16
        uint32_t first[4], left[4];
#pragma unroll
        for (uint32_t e = 0; e < 8; e += 2) {   // (the upper half of a float is its bfloat16 towards zero)
            const uint32_t a = __builtin_bit_cast(uint32_t, x[e]), b = __builtin_bit_cast(uint32_t, x[e + 1]);
            first[e / 2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            typedef __bf16 two __attribute__((ext_vector_type(2)));   // (converted in pairs: the prompts in 1.52 ms, by one 1.58)
            left[e / 2] = __builtin_bit_cast(uint32_t, two{(__bf16)(x[e] - __builtin_bit_cast(float, a & 0xFFFF0000u)),
                                                           (__bf16)(x[e + 1] - __builtin_bit_cast(float, b & 0xFFFF0000u))});
        }
        halves[0] = make_uint4(first[0], first[1], first[2], first[3]), halves[1] = make_uint4(left[0], left[1], left[2], left[3]);
    }
};

// A request's rows from `first` on, kRows at most
struct Item {
    uint32_t request, from, count;   // its first row of q; its new tokens
    uint32_t first, rows, len, kv_head;
    bool there;
    // one more than the place of new token j, 0 before the request's first
    __device__ __forceinline__ uint32_t end_of(uint32_t j) const {
        const uint32_t behind = count - 1 - j;
        return len > behind ? len - behind : 0;
    }
};
// items in the order of kv heads first, then from the last rows of the last request back, as those see the most
__device__ __forceinline__ Item item_of(const WindowArgs& a, uint32_t item, uint32_t ranks) {
    const uint32_t lane = threadIdx.x % 64, turn = item / a.kv_heads, rank = ranks - 1 - turn;
    Item x{};
    x.kv_head = item - turn * a.kv_heads;
    uint32_t before = 0;
    for (uint32_t b0 = 0; b0 < a.requests; b0 += 64) {
        const uint32_t b = b0 + lane;
        uint32_t from = 0, count = 0;
        if (b < a.requests) {
            from = clamped(a.starts[b], a.tokens);
            const uint32_t to = clamped(a.starts[b + 1], a.tokens);
            count = to <= from ? 0 : to - from < a.most ? to - from : a.most;
        }
        const uint32_t its = (uint32_t)(((uint64_t)count * a.group + kRows - 1) / kRows), upto = before + scan(its);
        const uint64_t past = __ballot(upto > rank);
        if (past != 0) {
            const uint32_t at = __builtin_ctzll(past);
            x.there = true;
            x.request = b0 + at;
            x.from = __builtin_amdgcn_readlane(from, at), x.count = __builtin_amdgcn_readlane(count, at);
            x.first = (rank - (uint32_t)__builtin_amdgcn_readlane(upto - its, at)) * kRows;
            const uint32_t left = x.count * a.group - x.first;
            x.rows = left < kRows ? left : kRows;
            x.len = clamped(constant(a.lens, x.request), a.row_blocks * a.block_tokens);
            return x;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return x;
}
struct Parts {
    Seen seen;
    uint32_t pieces, tiles, parts;
};
__device__ __forceinline__ Parts parts_of(const WindowArgs& a, const Item& x, uint32_t most_parts) {
    Parts p;
    const uint32_t first_end = x.end_of(x.first / a.group), last_end = x.end_of((x.first + x.rows - 1) / a.group);
    p.seen = last_end == 0 ? Seen{0, 0, 0} : seen_of(a, first_end, last_end);
    p.pieces = p.seen.pieces();
    p.tiles = (p.pieces + kTilePieces - 1) / kTilePieces;
    const uint32_t useful = (p.tiles + kLeastTiles - 1) / kLeastTiles;
    p.parts = useful < 1 ? 1 : useful < most_parts ? useful : most_parts;
    return p;
}

// How rows of K and V lie in LDS: sixteen bytes p of row t of K at place p ^ of_k(t), of V at p ^ of_v(t), so that the sixteen
// rows that an instruction reads of K, and the four of V, lie in different banks.
template <uint32_t kDim>
struct Rows {
    static constexpr uint32_t kBytes = 2 * kDim, kPlaces = kDim / 8, kRowsAtOnce = 64 / kPlaces, kAsked = 16 / kRowsAtOnce;
    static __device__ __forceinline__ uint32_t of_k(uint32_t t) { return kDim == 64 ? t / 2 % 8 : t % 16; }
    static __device__ __forceinline__ uint32_t of_v(uint32_t t) { return kDim == 64 ? t / 2 % 2 * 4 : t % 4 * 4; }
};

// Sixteen bytes a lane from base + at to LDS, without a register.  As an instruction of its own, since of the compiler's it waits
// for all that are under way before it reads anything from LDS; who reads what it brings waits for it.
// (m0 is reserved: the compiler sees that it changes here, and warns that it will not restore it, which nothing needs.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void to_lds(const uint8_t* base, uint32_t at, uint32_t place) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(place), "v"(at), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

template <uint32_t kDim>
struct ManyShared {
    __align__(1024) uint8_t rows[2][2][kTile * 2 * kDim];   // by turns; K, V
    // of values that are not finite: a bit for each channel of a token, and which pieces have any
    uint32_t odd[2][kTile][kDim / 32];
    uint32_t any[2][kTilePieces];
};

template <class H, uint32_t kDim, bool kExact, bool kCut>
__global__ __launch_bounds__(kThreads, kDim == 256 ? 1 : 2) void many_kernel(WindowArgs a, uint32_t ranks, uint32_t most_parts) {
    typedef Rows<kDim> R;
    typedef Wide<H> W;
    constexpr uint32_t kSteps = kDim / 16, kOut = kDim / 32;
    __shared__ ManyShared<kDim> shared;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t hh = lane / 32, col = lane % 32;

    const uint32_t item = kCut ? blockIdx.x / most_parts : blockIdx.x, part = kCut ? blockIdx.x - item * most_parts : 0;
    const Item x = item_of(a, item, ranks);
    if (!x.there) return;
    const Parts split = parts_of(a, x, kCut ? most_parts : 1);
    if (part >= split.parts) return;
    const Seen seen = split.seen;
    // (`longer` parts have one tile more; a product of tiles and parts would pass 32 bits)
    const uint32_t even = split.tiles / split.parts, longer = split.tiles - even * split.parts;
    const uint32_t from = even * part + (part < longer ? part : longer), to = from + even + (part < longer ? 1 : 0);

    // the wavefront's rows, and the lane's
    const uint32_t row0 = 32 * wave, mine = x.rows <= row0 ? 0 : x.rows - row0 < 32 ? x.rows - row0 : 32;
    const uint32_t first_token = (x.first + row0) / a.group, last_token = mine == 0 ? first_token : (x.first + row0 + mine - 1) / a.group;
    const uint32_t least_end = mine == 0 ? 0 : x.end_of(first_token), most_end = mine == 0 ? 0 : x.end_of(last_token);
    const uint32_t least_low = low_of(a, least_end), most_low = low_of(a, most_end);
    const uint32_t row = x.first + row0 + (col < mine ? col : 0), token = row / a.group;
    const uint32_t head = x.kv_head * a.group + row - token * a.group;
    const uint32_t end = mine == 0 ? 0 : x.end_of(token), low = low_of(a, end);

    uint4 q[kSteps];
    {
        const uint8_t* at = a.q + (x.from + token) * a.q_token + head * a.q_head;
#pragma unroll
        for (uint32_t c = 0; c < kSteps; ++c) {
            const uint32_t d = 16 * c + 8 * hh;
            q[c] = make_uint4(0, 0, 0, 0);
            if (mine != 0 && (kExact || d < a.head_dim)) q[c] = *(const uint4*)(at + 2 * d);
            // (a factor below zero turns the signs of q, one of zero makes it zero, or NaN: the factor left is more than zero)
            if (a.scale <= 0.f) {
                auto with = [&](uint32_t w) {
                    constexpr uint32_t kInf = H::kInfinity;
                    if (a.scale != 0.f) return w ^ 0x80008000u;
                    return ((w & kInf) == kInf ? 0x7FFFu : 0u) | ((w & kInf << 16) == kInf << 16 ? 0x7FFF0000u : 0u);
                };
                q[c] = make_uint4(with(q[c].x), with(q[c].y), with(q[c].z), with(q[c].w));
            }
        }
    }
    const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale);
    f32x16 sum[kOut];
#pragma unroll
    for (uint32_t n = 0; n < kOut; ++n) sum[n] = f32x16{};
    float top = -INFINITY, total = 0.f;

    // where the lane's bytes lie from an instruction's first row on
    uint32_t k_at[R::kAsked], v_at[R::kAsked];
#pragma unroll
    for (uint32_t n = 0; n < R::kAsked; ++n) {
        const uint32_t t = lane / R::kPlaces, there = a.head_dim / 8;   // (beyond the channels: anything that is there)
        const uint32_t pk = (lane % R::kPlaces) ^ R::of_k(n * R::kRowsAtOnce + t), pv = (lane % R::kPlaces) ^ R::of_v(n * R::kRowsAtOnce + t);
        k_at[n] = (n * R::kRowsAtOnce + t) * (uint32_t)a.k_token + 16 * (pk < there ? pk : 0);
        v_at[n] = (n * R::kRowsAtOnce + t) * (uint32_t)a.v_token + 16 * (pv < there ? pv : 0);
    }
    // Sixteen tiles' pieces at a time, lane by lane: where they lie, and, as bits, which of them are on the device, which do not all
    // of the item's or of the wavefront's rows see whole, and which does any of the wavefront's see.
    constexpr uint32_t kBatch = 64 / kTilePieces;
    auto token_of = [&](uint32_t tile) { return seen.piece(tile * kTilePieces + lane) * kPiece; };
    auto find = [&](uint32_t tile) {
        if (tile + lane / kTilePieces >= to || tile * kTilePieces + lane >= split.pieces) return ~0u;
        return (uint32_t)a.tables[x.request * a.table_row + token_of(tile) / a.block_tokens];
    };
    const uint32_t all_end = x.end_of(x.first / a.group), all_low = low_of(a, x.end_of((x.first + x.rows - 1) / a.group));
    uint32_t ahead = from, next = find(ahead), piece_at = 0;
    uint64_t live = 0, hidden_all = 0, hidden_mine = 0, seen_mine = 0, piece_k = 0, piece_v = 0;
    auto use = [&]() {
        piece_at = token_of(ahead);
        const bool there = next < a.blocks;
        const uint32_t block = there ? next : 0, inside = there ? piece_at % a.block_tokens : 0;   // (else any that is there)
        piece_k = (uint64_t)(uintptr_t)a.k + x.kv_head * a.k_head + block * a.k_block + inside * a.k_token;
        piece_v = (uint64_t)(uintptr_t)a.v + x.kv_head * a.v_head + block * a.v_block + inside * a.v_token;
        const uint32_t piece_end = piece_at + kPiece;
        live = __ballot(there);
        hidden_all = __ballot(!there || piece_end > all_end || (piece_at < all_low && piece_end > a.sinks));
        hidden_mine = __ballot(!there || piece_end > least_end || (piece_at < most_low && piece_end > a.sinks));
        seen_mine = __ballot(there && piece_at < most_end && (piece_end > least_low || piece_at < a.sinks));
        ahead += kBatch;
        next = find(ahead);
    };
    auto lane_of = [](uint64_t x, uint32_t j) {
        const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, j), hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), j);
        return (const uint8_t*)(uintptr_t)((uint64_t)hi << 32 | lo);   // (what comes from a lane is an int)
    };
    struct Tile {
        uint32_t here, hidden_all, hidden_mine, seen_mine;   // bits of its four pieces
        uint32_t at[kTilePieces];                            // their first tokens, where any is hidden
    };
    // where the wavefront's piece goes in LDS
    const uint32_t rows_at = __builtin_amdgcn_readfirstlane(
        (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&shared.rows[0][0][0] + wave * 16 * R::kBytes);
    // the next tile of which any piece is there; its rows are asked for
    auto ask = [&](Tile& t, uint32_t turn) {
        while (live == 0) {
            if (ahead >= to) return false;
            use();
        }
        const uint32_t n = __builtin_ctzll(live) / kTilePieces * kTilePieces;
        t.here = (uint32_t)(live >> n) & 15;
        t.hidden_all = (uint32_t)(hidden_all >> n) & 15;
        t.hidden_mine = (uint32_t)(hidden_mine >> n) & 15;
        t.seen_mine = (uint32_t)(seen_mine >> n) & 15;
        live &= ~(15ull << n);
        if (t.hidden_all != 0)
#pragma unroll
            for (uint32_t p = 0; p < kTilePieces; ++p) t.at[p] = __builtin_amdgcn_readlane(piece_at, n + p);
        const uint8_t* const k = lane_of(piece_k, n + wave);
        const uint8_t* const v = lane_of(piece_v, n + wave);
#pragma unroll
        for (uint32_t i = 0; i < R::kAsked; ++i) to_lds(k, k_at[i], rows_at + turn * 2 * kTile * R::kBytes + i * 1024);
#pragma unroll
        for (uint32_t i = 0; i < R::kAsked; ++i) to_lds(v, v_at[i], rows_at + (turn * 2 + 1) * kTile * R::kBytes + i * 1024);
        return true;
    };

    // K as the left operand: the lane has token col (and 32 on), channels 16 c + 8 hh ... + 7 in step c
    const uint32_t k_row = col * R::kBytes, k_place = hh ^ R::of_k(col);
    // V as the left operand: lanes read four tokens' rows of sixteen channels across; a lane gets, of channel 32 n + col, tokens
    // 8 e + 4 hh ... + 3 of a step's sixteen
    const uint32_t v_token = 4 * hh + lane % 16 / 4;
    auto v_place = [&](uint32_t n) { return (4 * n + 2 * (lane / 16 % 2) + lane % 4 / 2) ^ R::of_v(v_token); };
    uint32_t v_from[kOut];
#pragma unroll
    for (uint32_t n = 0; n < kOut; ++n) v_from[n] = v_token * R::kBytes + 16 * v_place(n) + 8 * (lane % 2);

    // Tokens that a row does not see have a weight of zero, and zero times what is no number is none.  So where there are such
    // tokens, the wavefront that asked for a piece of V takes what is not finite out of it, and writes down where that was.
    auto clean = [&](uint32_t turn) {
        uint8_t* const rows = shared.rows[turn][1] + wave * 16 * R::kBytes;
        uint4 x[R::kAsked];
        uint32_t odd = 0;
#pragma unroll
        for (uint32_t i = 0; i < R::kAsked; ++i) {
            x[i] = *(const uint4*)(rows + i * 1024 + 16 * lane);
            const uint32_t words[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                constexpr uint32_t kInf = H::kInfinity;
                odd |= (words[j] & kInf) == kInf || (words[j] & kInf << 16) == kInf << 16;
            }
        }
        const bool any = __any(odd);
        if (any) {
#pragma unroll
            for (uint32_t i = 0; i < R::kAsked; ++i) {
                uint32_t words[4] = {x[i].x, x[i].y, x[i].z, x[i].w}, bits = 0;
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) {
                    constexpr uint32_t kInf = H::kInfinity;
                    if ((words[j] & kInf) == kInf) words[j] &= 0xFFFF0000u, bits |= 1u << 2 * j;
                    if ((words[j] & kInf << 16) == kInf << 16) words[j] &= 0xFFFFu, bits |= 2u << 2 * j;
                }
                *(uint4*)(rows + i * 1024 + 16 * lane) = make_uint4(words[0], words[1], words[2], words[3]);
                const uint32_t t = i * R::kRowsAtOnce + lane / R::kPlaces, place = (lane % R::kPlaces) ^ R::of_v(t);
                ((uint8_t*)shared.odd[turn][16 * wave + t])[place] = (uint8_t)bits;
            }
        }
        if (lane == 0) shared.any[turn][wave] = any;
    };
    uint32_t spoilt[kOut] = {};   // of the lane's row: the channels that saw such a value, bit 8 i + 4 hh + r (as in a row of odd)

    auto work = [&](const Tile& t, uint32_t turn) {
        if (t.seen_mine == 0) return;
        const uint8_t* const k_rows = shared.rows[turn][0];
        const uint8_t* const v_rows = shared.rows[turn][1];
        f32x16 w[2];
#pragma unroll
        for (uint32_t b = 0; b < 2; ++b) {
            w[b] = f32x16{};
#pragma unroll
            for (uint32_t c = 0; c < kSteps; ++c) {
                if (!kExact && 16 * c >= a.head_dim) break;
                uint4 k = *(const uint4*)(k_rows + 32 * b * R::kBytes + k_row + 16 * (k_place ^ 2 * c));
                if (!kExact && 16 * c + 8 * hh >= a.head_dim) k = make_uint4(0, 0, 0, 0);   // (infinity times zero is no number)
                w[b] = W::product(k, q[c], w[b]);
                if (kDim == 256 && c % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (reads made far ahead have no registers)
            }
        }
        if (t.hidden_all != 0 && (t.hidden_mine != 0 || (shared.any[turn][0] | shared.any[turn][1] | shared.any[turn][2] | shared.any[turn][3]) != 0)) {
            // bit 16 b + r: whether the lane's row sees the token of w[b][r]
            uint32_t sees = 0;
#pragma unroll
            for (uint32_t p = 0; p < kTilePieces; ++p) {
                const uint32_t at = t.at[p];
                auto below = [&](uint32_t x) {   // tokens of the piece before x
                    return x <= at ? 0u : x - at < kPiece ? (1u << (x - at)) - 1 : 0xFFFFu;
                };
                const uint32_t of = t.here >> p & 1 ? below(end) & (~below(low) | below(a.sinks)) : 0u, its = of >> 4 * hh;
                sees |= ((its & 0xF) | (its >> 4 & 0xF0)) << 8 * p;
                if (shared.any[turn][p] != 0)   // (hardly ever)
#pragma unroll 1
                    for (uint32_t j = 0; j < kPiece; ++j)
#pragma unroll
                        for (uint32_t n = 0; n < kOut; ++n) spoilt[n] |= of >> j & 1 ? shared.odd[turn][16 * p + j][n] : 0u;
            }
#pragma unroll
            for (uint32_t b = 0; b < 2; ++b)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) w[b][r] = sees >> (16 * b + r) & 1 ? w[b][r] : -INFINITY;
        }
        float most = -INFINITY;
#pragma unroll
        for (uint32_t b = 0; b < 2; ++b)
#pragma unroll
            for (uint32_t r = 0; r < 16; ++r) most = fmaxf(most, w[b][r]);
        const Two both = of_halves(most);
        most = fmaxf(both.a, both.b) * scale;
        // Sums are kept relative to 2^top, which makes the largest weight so far 2^H::kLargest when they were last brought up to
        // it, and at most 2^H::kOverflows before the next time: a new maximum rarely takes that.
        const bool over = most > top + H::kOverflows || (top == -INFINITY && most > top);
        if (__any(over)) {   // (what other rows need changes nothing in a row)
            const float now = over ? fmaxf(most - H::kLargest, top) : top, keep = exp2_from(top, now);
            top = now;
            total *= keep;
#pragma unroll
            for (uint32_t n = 0; n < kOut; ++n) sum[n] *= keep;
        }
        const float down = top == -INFINITY ? 0.f : -top;
        __builtin_amdgcn_s_setprio(1);
        typedef __attribute__((address_space(3))) s16x4* Lds;
#pragma unroll
        for (uint32_t b = 0; b < 2; ++b)
#pragma unroll
            for (uint32_t e = 0; e < 2; ++e) {
                // Weights as the right operand, sixteen tokens a step, as sums of two halves.  Rounded to one each, they cost more
                // than the outputs' own rounding: the prompts' were off by 0.0022 (2-norm, relative, bfloat16) instead of 0.0017, the
                // chunk's by 0.00025 instead of 0.00021 (binary16), and a token's results were others than alone.  With one: 1.19
                // ms and 166 us instead of 1.52 and 207.
                float z[8];
#pragma unroll
                for (uint32_t r = 0; r < 8; ++r) {
                    z[r] = __builtin_amdgcn_exp2f(fmaf(w[b][8 * e + r], scale, down));
                    total += z[r];
                }
                uint4 p[2];
                W::split(z, p);
#pragma unroll
                for (uint32_t n = 0; n < kOut; ++n) {
                    if (!kExact && 32 * n >= a.head_dim) break;
                    const uint8_t* from_row = v_rows + (32 * b + 16 * e) * R::kBytes + v_from[n];
                    const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)from_row));
                    const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(from_row + 8 * R::kBytes)));
                    const uint4 v = make_uint4(x.x, x.y, y.x, y.y);
                    sum[n] = W::product(v, p[1], W::product(v, p[0], sum[n]));
                }
                if (kDim == 256) __builtin_amdgcn_sched_barrier(0);
            }
        __builtin_amdgcn_s_setprio(0);
    };

    {
        Tile now{}, after{};
        uint32_t turn = 0;
        bool more = ask(now, 0);
        while (more) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the wavefront's rows are in LDS
            if (now.hidden_all != 0) clean(turn);
            __syncthreads();                                   // ... and the others', and all have left the tile before
            more = ask(after, turn ^ 1);
            work(now, turn);
            now = after;
            turn ^= 1;
        }
    }
#pragma unroll
    for (uint32_t n = 0; n < kOut; ++n)
        if (__any(spoilt[n] != 0))
#pragma unroll
            for (uint32_t r = 0; r < 16; ++r) sum[n][r] = spoilt[n] >> (r / 4 * 8 + 4 * hh + r % 4) & 1 ? NAN : sum[n][r];

    // The lane holds, of row col, channels 32 n + 8 i + 4 hh ... + 3 in sum[n][4 i] on.
    const Two both = of_halves(total);
    total = both.a + both.b;
    if (col >= mine) return;
    if (kCut && split.parts > 1) {
        float* const to_part = a.partials + (size_t)blockIdx.x * kRows * (kDim + 2);
#pragma unroll
        for (uint32_t n = 0; n < kOut; ++n)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                *(float4*)(to_part + (row0 + col) * kDim + 32 * n + 8 * i + 4 * hh) =
                    make_float4(sum[n][4 * i], sum[n][4 * i + 1], sum[n][4 * i + 2], sum[n][4 * i + 3]);
        if (hh == 0) *(float2*)(to_part + kRows * kDim + 2 * (row0 + col)) = make_float2(top, total);
        return;
    }
    const float by = total == 0.f ? 0.f : 1.f / total;   // (a NaN stays one)
    uint8_t* const out = a.out + (x.from + token) * a.out_token + head * a.out_head;
#pragma unroll
    for (uint32_t n = 0; n < kOut; ++n)
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t d = 32 * n + 8 * i + 4 * hh;
            if (!kExact && d >= a.head_dim) continue;
            typename H::one y[4];
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) y[r] = (typename H::one)(sum[n][4 * i + r] * by);
            uint2 words;
            __builtin_memcpy(&words, y, 8);
            *(uint2*)(out + 2 * d) = words;
        }
    if (hh == 0 && a.lse != nullptr)
        a.lse[(size_t)(x.from + token) * a.kv_heads * a.group + head] =
            total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * 0.693147180559945f;
}

// The parts of an item as one: blockIdx.y takes a sixteenth of its rows, a thread four channels of one at a time.
constexpr uint32_t kJoins = 16, kTogether = 8;   // parts whose loads are under way together
template <class H, uint32_t kDim>
__global__ __launch_bounds__(kThreads) void join_kernel(WindowArgs a, uint32_t ranks, uint32_t most_parts) {
    const uint32_t item = blockIdx.x;
    const Item x = item_of(a, item, ranks);
    if (!x.there) return;
    const uint32_t parts = parts_of(a, x, most_parts).parts;
    if (parts == 1) return;
    constexpr uint32_t kQuads = kDim / 4;
    constexpr size_t kPart = (size_t)kRows * (kDim + 2);
    const float* const first = a.partials + (size_t)item * most_parts * kPart;
    for (uint32_t n = threadIdx.x; n < kRows / kJoins * kQuads; n += kThreads) {
        const uint32_t r = blockIdx.y * (kRows / kJoins) + n / kQuads, d = n % kQuads * 4;
        if (r >= x.rows) return;
        // (sums to the largest top so far, as in the walk)
        float most = -INFINITY, total = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (uint32_t p0 = 0; p0 < parts; p0 += kTogether) {
            float2 of[kTogether];
            float4 y[kTogether];
#pragma unroll
            for (uint32_t e = 0; e < kTogether; ++e) {
                const float* const part = first + (p0 + e < parts ? p0 + e : p0) * kPart;
                of[e] = *(const float2*)(part + kRows * kDim + 2 * r);
                y[e] = *(const float4*)(part + r * kDim + d);
            }
            float now = most;
#pragma unroll
            for (uint32_t e = 0; e < kTogether; ++e) now = fmaxf(now, of[e].x);
            const float keep = exp2_from(most, now);
            most = now;
            total *= keep;
            sum.x *= keep, sum.y *= keep, sum.z *= keep, sum.w *= keep;
#pragma unroll
            for (uint32_t e = 0; e < kTogether; ++e) {
                if (p0 + e >= parts) break;
                const float by = exp2_from(of[e].x, most);
                total += of[e].y * by;
                sum.x += y[e].x * by, sum.y += y[e].y * by, sum.z += y[e].z * by, sum.w += y[e].w * by;
            }
        }
        const uint32_t row = x.first + r, token = row / a.group, head = x.kv_head * a.group + row - token * a.group;
        const float by = total == 0.f ? 0.f : 1.f / total;   // (a NaN stays one)
        if (d < a.head_dim) {
            typename H::one y[4] = {(typename H::one)(sum.x * by), (typename H::one)(sum.y * by), (typename H::one)(sum.z * by),
                                    (typename H::one)(sum.w * by)};
            uint2 words;
            __builtin_memcpy(&words, y, 8);
            *(uint2*)(a.out + (x.from + token) * a.out_token + head * a.out_head + 2 * d) = words;
        }
        if (d == 0 && a.lse != nullptr)
            a.lse[(size_t)(x.from + token) * a.kv_heads * a.group + head] =
                total == 0.f ? -INFINITY : (most + __builtin_amdgcn_logf(total)) * 0.693147180559945f;
    }
}

template <class H, uint32_t kDim, bool kExact>
void launch(const WindowArgs& a, uint32_t items, uint32_t ranks, uint32_t parts, hipStream_t stream) {
    if (parts == 1) {
        many_kernel<H, kDim, kExact, false><<<items, kThreads, 0, stream>>>(a, ranks, 1);
        return;
    }
    many_kernel<H, kDim, kExact, true><<<items * parts, kThreads, 0, stream>>>(a, ranks, parts);
    join_kernel<H, kDim><<<dim3(items, kJoins), kThreads, 0, stream>>>(a, ranks, parts);
}
template <class H>
void launch(const WindowArgs& a, uint32_t items, uint32_t ranks, uint32_t parts, hipStream_t stream) {
    const uint32_t d = a.head_dim;
    if (d == 64) launch<H, 64, true>(a, items, ranks, parts, stream);
    else if (d < 64) launch<H, 64, false>(a, items, ranks, parts, stream);
    else if (d == 128) launch<H, 128, true>(a, items, ranks, parts, stream);
    else if (d < 128) launch<H, 128, false>(a, items, ranks, parts, stream);
    else if (d == 256) launch<H, 256, true>(a, items, ranks, parts, stream);
    else launch<H, 256, false>(a, items, ranks, parts, stream);
}
size_t part_bytes(uint32_t head_dim) { return 4 * (size_t)kRows * ((head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256) + 2); }

}  // namespace

// (of any call; one takes as much as it has parts)
Room window_many_room(uint32_t head_dim) { return Room{0, part_bytes(head_dim) * kMostParts}; }

int window_many(pgcm_kv* kv, WindowArgs& a, uint32_t half, hipStream_t stream) {
    // runs of kRows rows, at most: each request's last one may be short of that
    const uint64_t some = a.requests < a.tokens ? a.requests : a.tokens;
    const uint64_t ranks = ((uint64_t)a.tokens * a.group + some * (kRows - 1)) / kRows, items = ranks * a.kv_heads;
    if (!launchable(items, kThreads) || items > 0x7FFFFFFFull) return PGCM_ERR_ARG;
    uint64_t walked = (uint64_t)a.row_blocks * a.block_tokens;
    const uint64_t seen = (uint64_t)a.window + a.sinks + kRows / a.group + 4 * kPiece;
    if (a.window != 0 && walked > seen) walked = seen;
    const uint64_t tiles = (walked + kTile - 1) / kTile, useful = (tiles + kLeastTiles - 1) / kLeastTiles;
    // (512 tokens, 128 items: 4 parts 236 us, 3 262, 8 253; 1200, 304 items: 3 parts 530, 1 619; 8 tokens, 8 items: 33 parts 37, 16 48)
    // As many parts as take the least time, in tiles: rounds of as many workgroups as the chip holds, two tiles' time at a part's
    // start and end each, and the join's.
    const uint64_t at_once = a.head_dim > 128 ? kManyGroups / 2 : kManyGroups;
    uint64_t parts = 1;
    double least = 0;
    for (uint64_t p = 1; p == 1 || (p <= useful && items * p <= kMostParts); ++p) {
        const double time = (double)((items * p + at_once - 1) / at_once) * ((double)tiles / (double)p + 2) +
                            (p == 1 ? 0 : 1.5 + 0.007 * (double)(items * p));
        if (p == 1 || time < least) least = time, parts = p;
    }
    if (parts > 1) {
        if (const int rc = kv_ensure(kv, 0, part_bytes(a.head_dim) * items * parts, stream)) return rc;
        a.partials = (float*)kv->scratch.at;
    }
    if (half == PGCM_KV_F16) launch<F16>(a, (uint32_t)items, (uint32_t)ranks, (uint32_t)parts, stream);
    else launch<Bf16>(a, (uint32_t)items, (uint32_t)ranks, (uint32_t)parts, stream);
    return pgcm::hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

}  // namespace pgcm_kv_impl
