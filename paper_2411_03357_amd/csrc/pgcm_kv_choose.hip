// The best blocks of a request for attention, and the least of them for eviction (include/pgcm_kv.h): so many largest
// of a row of keys, equal ones from the front.
#include "pgcm_kv_common.h"

namespace pgcm_kv_impl {
namespace {

constexpr uint32_t kMostThreads = 1024;
// Keys that a lane holds in registers, kHeld; rows that are too long for kMostHeld are read from memory at each look.  All loops
// over them are laid out in full, so that of a kernel with room for more keys than the row has much code is fetched and passed
// over: 256 rows of up to 8192 keys take 11.5 us with room for 8 keys a lane, 13.0 with room for 16.
constexpr uint32_t kFewHeld = 2, kSomeHeld = 8, kMostHeld = 16;
constexpr uint32_t kBinBits = 10, kBins = 1u << kBinBits;
constexpr uint32_t kNever = 0, kAlways = 0xFFFFFFFFu;  // keys of what cannot be chosen, and of what is chosen before all others

// Whole numbers in the order of numbers; those of -inf and inf are not kNever and kAlways.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);  // (-0 as 0)
    return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

// A row of n keys: each wavefront has an equal part of it, 64 keys a step.  each(f): f(i, key of i, step) step by step
// for all lanes together, kNever beyond the row.
template <uint32_t kThreads>
struct Part {
    uint32_t first, steps;
    __device__ __forceinline__ explicit Part(uint32_t n) {
        steps = (n + kThreads - 1) / kThreads;
        first = threadIdx.x / 64 * 64 * steps + threadIdx.x % 64;
    }
};
template <uint32_t kThreads, uint32_t kHeld>
struct HeldKeys {
    Part<kThreads> part;
    uint32_t key[kHeld];
    __device__ __forceinline__ explicit HeldKeys(uint32_t n) : part(n) {}
    static bool __device__ __forceinline__ holds(uint32_t n) { return n <= kHeld * kThreads; }
    template <class F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (uint32_t s = 0; s < kHeld; ++s)
            if (s < part.steps) f(part.first + 64 * s, key[s], s);
    }
};
template <uint32_t kThreads, class Read>
struct ReadKeys {
    Part<kThreads> part;
    uint32_t n;
    Read read;
    __device__ __forceinline__ ReadKeys(uint32_t n, Read read) : part(n), n(n), read(read) {}
    template <class F>
    __device__ __forceinline__ void each(F f) const {
        for (uint32_t s = 0; s < part.steps; ++s) {
            const uint32_t i = part.first + 64 * s;
            f(i, i < n ? read(i) : kNever, s);
        }
    }
};

struct ChooseShared {
    __align__(16) uint32_t bins[3][kBins];   // of a look and of the next one; those of the one before may still be read
    uint32_t able[kMostThreads / 64], always[kMostThreads / 64], least[kMostThreads / 64], most[kMostThreads / 64];
    uint32_t above[kMostThreads / 64], equal[kMostThreads / 64];
};

// What is chosen: the keys above `above`, and of those equal to `equal` the first `of_equal`; `count` in all.
struct Chosen {
    uint32_t above, equal, of_equal, count;
};

// The sum of the figures of the wavefronts before this one.
__device__ __forceinline__ uint32_t of_waves_before(const uint32_t* figures) {
    const uint32_t lane = threadIdx.x % 64;
    return over_wave(lane < threadIdx.x / 64 ? figures[lane] : 0u, [](uint32_t a, uint32_t b) { return a + b; });
}

// The `want` largest keys.  All threads call it.  Keys are whole numbers, so that counts say exactly where the last one chosen
// lies, and no order of threads shows.  What bounds it are looks at the keys, each with its counts in LDS and a barrier: 256 rows
// of up to 8192, 64 chosen, 11.3 us with keys in registers, 18 with keys read from memory at each look.
template <uint32_t kThreads, class Keys>
__device__ __forceinline__ Chosen choose(const Keys& keys, uint32_t want, ChooseShared& shared) {
    constexpr uint32_t kWaves = kThreads / 64;
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const auto less = [](uint32_t a, uint32_t b) { return a < b ? a : b; };
    const auto more = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    uint32_t able = 0, always = 0, least = kAlways, most = 0;
    keys.each([&](uint32_t, uint32_t k, uint32_t) {
        able += __builtin_popcountll(__ballot(k != kNever));
        always += __builtin_popcountll(__ballot(k == kAlways));
        const bool between = k != kNever && k != kAlways;
        least = less(least, between ? k : kAlways);
        most = more(most, between ? k : 0u);
    });
    least = over_wave(least, less);
    most = over_wave(most, more);
    for (uint32_t b = threadIdx.x; b < kBins; b += kThreads) shared.bins[0][b] = 0;
    if (lane == 0) shared.able[wave] = able, shared.always[wave] = always, shared.least[wave] = least, shared.most[wave] = most;
    __syncthreads();
    // (a wavefront's figures in a lane each: sixteen wavefronts that read all of them one by one keep LDS busy for 0.5 us)
    const bool has = lane < kWaves;
    const auto plus = [](uint32_t a, uint32_t b) { return a + b; };
    able = over_wave(has ? shared.able[lane] : 0u, plus), always = over_wave(has ? shared.always[lane] : 0u, plus);
    least = over_wave(has ? shared.least[lane] : kAlways, less), most = over_wave(has ? shared.most[lane] : 0u, more);
    if (able <= want) return Chosen{kNever, kNever, 0, able};
    if (want == 0) return Chosen{kAlways, kNever, 0, 0};
    if (always >= want) return Chosen{kAlways, kAlways, want, want};

    // The place of the last one chosen, within [least, most]: counts of equal pieces of that range, from the top, then
    // the piece that it is in; as a rule one or two looks, at most four.  Each wavefront adds up all counts by itself, which
    // takes less than a barrier.
    uint32_t need = want - always;
    for (uint32_t look = 0;; ++look) {
        const uint32_t width = most - least;
        const uint32_t bits = width == 0 ? 0 : 32 - __builtin_clz(width);
        const uint32_t shift = bits > kBinBits ? bits - kBinBits : 0;
        uint32_t* bins = shared.bins[look % 3];
        keys.each([&](uint32_t, uint32_t k, uint32_t) {
            if (k >= least && k <= most) atomicAdd(&bins[(k - least) >> shift], 1u);
        });
        for (uint32_t b = threadIdx.x; b < kBins; b += kThreads) shared.bins[(look + 1) % 3][b] = 0;
        __syncthreads();
        // lane l adds up the l-th of 64 runs of bins from the top
        constexpr uint32_t kRun = kBins / 64;
        uint32_t sum = 0;
#pragma unroll
        for (uint32_t e = 0; e < kRun; e += 4) {
            const uint4 x = *(const uint4*)&bins[(63 - lane) * kRun + (e + 4 * lane) % kRun];   // (in turn, for LDS's banks)
            sum += (x.x + x.y) + (x.z + x.w);
        }
        uint32_t upto = scan(sum);
        const uint32_t run = __builtin_ctzll(__ballot(upto >= need));
        const uint32_t before_run = __builtin_amdgcn_readlane(upto - sum, run);
        // ... and the run's bins, one a lane
        const uint32_t top = (64 - run) * kRun - 1;
        sum = lane < kRun ? bins[top - lane] : 0;
        upto = before_run + scan(sum);
        const uint32_t at = __builtin_ctzll(__ballot(upto >= need));
        const uint32_t in_bin = __builtin_amdgcn_readlane(sum, at);
        need -= (uint32_t)__builtin_amdgcn_readlane(upto - sum, at);
        least += (top - at) << shift;
        if (need == in_bin) return Chosen{least - 1, kNever, 0, want};   // (least is no key of kNever: at least 1)
        if (shift == 0) return Chosen{least, least, need, want};
        most = less(most, least + ((1u << shift) - 1));
    }
}

// put(i, place, step) for each chosen i, with the places in the order of i.
template <uint32_t kThreads, class Keys, class Put>
__device__ __forceinline__ void put_in_order(const Keys& keys, const Chosen& c, ChooseShared& shared, Put put) {
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t above = 0, equal = 0;
    keys.each([&](uint32_t, uint32_t k, uint32_t) {
        above += __builtin_popcountll(__ballot(k > c.above));
        equal += __builtin_popcountll(__ballot(k == c.equal && c.of_equal != 0));
    });
    const bool any = (above | equal) != 0;
    if (lane == 0) shared.above[wave] = above, shared.equal[wave] = equal;
    __syncthreads();
    if (!any) return;
    above = of_waves_before(shared.above), equal = of_waves_before(shared.equal);
    const uint64_t before_me = (1ull << lane) - 1;
    keys.each([&](uint32_t i, uint32_t k, uint32_t s) {
        const uint64_t is_above = __ballot(k > c.above), is_equal = __ballot(k == c.equal && c.of_equal != 0);
        if ((is_above | is_equal) == 0) return;
        const uint32_t rank = equal + __builtin_popcountll(is_equal & before_me);
        const bool chosen = k > c.above || ((is_equal >> lane & 1) && rank < c.of_equal);
        const uint32_t place = above + __builtin_popcountll(is_above & before_me) + (rank < c.of_equal ? rank : c.of_equal);
        if (chosen) put(i, place, s);
        above += __builtin_popcountll(is_above);
        equal += __builtin_popcountll(is_equal);
    });
}

// ---------------------------------------------------------------------------------------------
struct EvictArgs {
    const float* weights;
    const int32_t *tables, *lens, *evict;
    int32_t *victims, *victim_blocks, *tables_out;
    int64_t table_row, table_out_row;
    uint32_t row_blocks, block_tokens, blocks, most, first, last;
};

// A row a workgroup: the least weights are the largest of what ~ makes of them.  One row of 128 blocks 3.2 us, the launch and
// its steps one after the other; 256 rows of up to 8192 blocks, 64 leaving (9 MB): 11.3 us, a compute unit each.
template <uint32_t kThreads, uint32_t kHeld>
__global__ __launch_bounds__(kThreads) void evict_kernel(EvictArgs a) {
    __shared__ ChooseShared shared;
    const uint32_t request = blockIdx.x;
    const int32_t len = a.lens[request], asked = a.evict[request];
    const float* weights = a.weights + (size_t)request * a.row_blocks;
    const int32_t* row = a.tables + request * a.table_row;
    int32_t* row_out = a.tables_out == nullptr ? nullptr : a.tables_out + request * a.table_out_row;
    int32_t* victims = a.victims + (size_t)request * a.most;
    int32_t* victim_blocks = a.victim_blocks == nullptr ? nullptr : a.victim_blocks + (size_t)request * a.most;
    const bool copied = row_out != nullptr && row_out != row;
    uint32_t want = asked <= 0 ? 0u : (uint32_t)asked;
    if (want > a.most) want = a.most;
    auto candidates = [&]() {   // below this place: the last ones stay
        uint32_t blocks = len <= 0 ? 0u : ((uint32_t)len - 1) / a.block_tokens + 1;
        if (blocks > a.row_blocks) blocks = a.row_blocks;
        return blocks > a.last ? blocks - a.last : 0u;
    };
    auto made = [&](uint32_t i, int32_t block, float w) {
        return i < a.first || (uint32_t)block >= a.blocks ? kNever : w == w ? ~ordered(w) : 1u;
    };
    auto run = [&](const auto& keys, auto block_of) {
        const Chosen c = choose<kThreads>(keys, want, shared);   // (its barriers are between the row's copy and the holes)
        put_in_order<kThreads>(keys, c, shared, [&](uint32_t i, uint32_t place, uint32_t s) {
            victims[place] = (int32_t)i;
            if (victim_blocks != nullptr) victim_blocks[place] = block_of(i, s);
            if (row_out != nullptr) row_out[i] = -1;   // (a table that is changed in place: the last look at it)
        });
        for (uint32_t i = c.count + threadIdx.x; i < a.most; i += kThreads) {
            victims[i] = -1;
            if (victim_blocks != nullptr) victim_blocks[i] = -1;
        }
    };
    if (HeldKeys<kThreads, kHeld>::holds(a.row_blocks)) {
        // (parts of the whole row, so that its copy takes no look of its own; all loads are under way together)
        HeldKeys<kThreads, kHeld> keys(a.row_blocks);
        int32_t block[kHeld];
        float w[kHeld];
#pragma unroll
        for (uint32_t s = 0; s < kHeld; ++s) {
            const uint32_t i = keys.part.first + 64 * s;
            block[s] = s < keys.part.steps && i < a.row_blocks ? row[i] : -1;
        }
        const uint32_t n = candidates();
#pragma unroll
        for (uint32_t s = 0; s < kHeld; ++s) {
            const uint32_t i = keys.part.first + 64 * s;
            w[s] = s < keys.part.steps && i < n ? weights[i] : 0.f;
        }
#pragma unroll
        for (uint32_t s = 0; s < kHeld; ++s) {
            const uint32_t i = keys.part.first + 64 * s;
            keys.key[s] = i < n ? made(i, block[s], w[s]) : kNever;
            if (copied && s < keys.part.steps && i < a.row_blocks) row_out[i] = block[s];
        }
        run(keys, [&](uint32_t, uint32_t s) { return block[s]; });
    } else {
        const uint32_t n = candidates();
        if (copied)
            for (uint32_t i = threadIdx.x; i < a.row_blocks; i += kThreads) row_out[i] = row[i];
        auto read = [&](uint32_t i) { return made(i, row[i], weights[i]); };
        run(ReadKeys<kThreads, decltype(read)>(n, read), [&](uint32_t i, uint32_t) { return row[i]; });
    }
}

// ---------------------------------------------------------------------------------------------
struct SelectArgs {
    const uint8_t* q;
    const int32_t *tables, *lens;
    const int8_t* bounds;
    const float* scales;
    int32_t *selected, *counts;
    uint32_t* keys;
    int64_t q_request, q_head;  // bytes
    int64_t table_row;
    uint32_t requests, kv_heads, group, head_dim, block_tokens, row_blocks, entry_count, keep, first, last;
    uint32_t parts;  // of a row: workgroups that score it
};

__device__ __forceinline__ uint32_t blocks_of(const SelectArgs& a, uint32_t request) {
    const int32_t len = a.lens[request];
    const uint32_t blocks = len <= 0 ? 0u : ((uint32_t)len - 1) / a.block_tokens + 1;
    return blocks < a.row_blocks ? blocks : a.row_blocks;
}

template <uint32_t kThreads, class Keys>
__device__ __forceinline__ void choose_list(const SelectArgs& a, uint32_t list, const Keys& keys, ChooseShared& shared) {
    int32_t* selected = a.selected + (size_t)list * a.keep;
    const Chosen c = choose<kThreads>(keys, a.keep, shared);
    put_in_order<kThreads>(keys, c, shared, [&](uint32_t j, uint32_t place, uint32_t) { selected[place] = (int32_t)j; });
    for (uint32_t n = c.count + threadIdx.x; n < a.keep; n += kThreads) selected[n] = -1;
    if (threadIdx.x == 0 && a.counts != nullptr) a.counts[list] = (int32_t)c.count;
}

constexpr uint32_t kScoreThreads = 256, kScoreWaves = kScoreThreads / 64;
// A wavefront scores 16 kSteps blocks at a time, a part of a row so many times its wavefronts: four steps, or one where four
// would leave half of the compute units without a part (8 lists of 1250 blocks, 256 channels: 14 us with one, 20 with four; 256
// lists of up to 2048 blocks, 128 channels: 28 and 22).
constexpr uint32_t kMostSteps = 4, kFewParts = 128;
__host__ __device__ constexpr uint32_t part_blocks(uint32_t steps) { return kScoreWaves * 16 * steps; }
// Rows scored and chosen from in one launch, a workgroup each: of up to kShortBlocks (one request with 8 lists: of 100 blocks
// 7.3 us, of 250 8.3, of 500 10.7, in two launches 9.9, 10.2 and 10.2), and of up to kWholeBlocks where there are lists for all
// compute units (of 1000 blocks: 32 requests 21.0 us and 22.1, one 15.2 and 10.4).
constexpr uint32_t kShortBlocks = 384, kWholeBlocks = 1024, kListsToFill = 256;

// Keys of the blocks [from, to) of a request for one kv head, at key_of(j).  The scores are products on the matrix cores,
// of 2 head_dim whole numbers: for each of sixteen query heads, its negative channels (for the least values) and its
// positive ones, with the bounds of sixteen blocks.  All threads call it; q8 and q_scale are theirs.
template <class H, uint32_t kChunks, uint32_t kSteps, class KeyOf>   // kChunks pieces of 64 numbers
__device__ __forceinline__ void score(const SelectArgs& a, uint32_t request, uint32_t head, uint32_t from, uint32_t to,
                                      uint32_t blocks, int8_t (&q8)[16][64 * kChunks + 16], float (&q_scale)[16], KeyOf key_of) {
    // what the registers hold of bounds: steps, and pieces of each
    constexpr uint32_t kTogether = kSteps == 1 ? 1 : kChunks == 4 ? 2 : 4, kAtOnce = kChunks < 4 || kSteps == 1 ? kChunks : 4;
    constexpr uint32_t kWaveBlocks = 16 * kSteps;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / 16, i = lane % 16;
    const uint32_t numbers = 2 * a.head_dim;
    const uint64_t entry_bytes = (uint64_t)a.kv_heads * numbers;
    const int8_t* of_head = a.bounds + (uint64_t)head * numbers;
    const int32_t* row = a.tables + request * a.table_row;

    for (uint32_t head0 = 0; head0 < a.group; head0 += 16) {
        const uint32_t heads = a.group - head0 < 16 ? a.group - head0 : 16;
        // queries in 8 bits: four heads a wavefront
        float y[4][kChunks / 2];
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n) {
            const uint32_t h = 4 * wave + n;
            const uint8_t* at = a.q + request * a.q_request + (head * a.group + head0 + (h < heads ? h : 0)) * a.q_head;
#pragma unroll
            for (uint32_t c = 0; c < kChunks / 2; ++c) {
                const uint32_t d = 64 * c + lane;
                y[n][c] = h < heads && d < a.head_dim ? (float)*(const typename H::one*)(at + 2 * d) : 0.f;
            }
        }
        i32x4 x[kTogether][kAtOnce];          // bounds of some steps, or of half of each
        uint32_t known;                       // entries of the wavefront's blocks; 0 for those that cannot be chosen
        uint64_t able;
        float scale;
        auto load = [&](uint32_t t0, uint32_t first) {
#pragma unroll
            for (uint32_t t = 0; t < kTogether; ++t) {
                const int8_t* at = of_head + __shfl(known, 16 * (t0 + t) + i) * entry_bytes;
#pragma unroll
                for (uint32_t c = 0; c < kAtOnce; ++c) {   // (beyond the numbers anything that is there: the query has zeros)
                    const uint32_t d = 64 * (first + c) + 16 * g;
                    x[t][c] = *(const i32x4*)(at + (d < numbers ? d : 0));
                }
            }
        };
        auto begin = [&](uint32_t j0) {
            const uint32_t entry = lane < kWaveBlocks && j0 + lane < to ? (uint32_t)row[j0 + lane] : ~0u;
            able = __ballot(entry < a.entry_count);
            known = entry < a.entry_count ? entry : 0;
            scale = a.scales[(uint64_t)known * a.kv_heads + head];
            load(0, 0);
        };
        uint32_t j0 = from + kWaveBlocks * wave;
        if (j0 < to) begin(j0);               // under way while the queries are made whole numbers
        __syncthreads();
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n) {
            const uint32_t h = 4 * wave + n;
            float most = 0.f;
#pragma unroll
            for (uint32_t c = 0; c < kChunks / 2; ++c) {
                if (!(fabsf(y[n][c]) < INFINITY)) y[n][c] = 0.f;
                most = fmaxf(most, fabsf(y[n][c]));
            }
            most = over_rows_max(row_max(most));
            const bool small = !(most >= 1e-30f);
            const float by = small ? 0.f : 127.f / most;
#pragma unroll
            for (uint32_t c = 0; c < kChunks / 2; ++c) {
                const uint32_t d = 64 * c + lane;
                const int32_t whole = small ? 0 : (int32_t)rintf(y[n][c] * by);
                if (d < a.head_dim) {
                    q8[h][d] = (int8_t)(whole < 0 ? whole : 0);
                    q8[h][a.head_dim + d] = (int8_t)(whole > 0 ? whole : 0);
                }
            }
            for (uint32_t d = numbers + lane; d < 64 * kChunks; d += 64) q8[h][d] = 0;
            if (lane == 0) q_scale[h] = small ? 0.f : most / 127.f;
        }
        __syncthreads();
        i32x4 q[kChunks];
#pragma unroll
        for (uint32_t c = 0; c < kChunks; ++c) q[c] = *(const i32x4*)&q8[i][64 * c + 16 * g];
        float qs[4];
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) qs[r] = q_scale[4 * g + r];

        while (j0 < to) {
#pragma unroll
            for (uint32_t t0 = 0; t0 < kSteps; t0 += kTogether) {
                i32x4 sum[kTogether];
#pragma unroll
                for (uint32_t first = 0; first < kChunks; first += kAtOnce) {
#pragma unroll
                    for (uint32_t t = 0; t < kTogether; ++t)
#pragma unroll
                        for (uint32_t c = 0; c < kAtOnce; ++c)
                            sum[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[first + c], x[t][c],
                                                                           first + c == 0 ? i32x4{0, 0, 0, 0} : sum[t], 0, 0, 0);
                    if (first + kAtOnce < kChunks) load(t0, first + kAtOnce);
                    else if (t0 + kTogether < kSteps) load(t0 + kTogether, 0);
                }
#pragma unroll
                for (uint32_t t = 0; t < kTogether; ++t) {
                    const float of_block = __shfl(scale, 16 * (t0 + t) + i);
                    float most = -INFINITY;      // of block i: heads 4 g + r, then those of all rows of lanes
#pragma unroll
                    for (uint32_t r = 0; r < 4; ++r)
                        if (4 * g + r < heads) most = fmaxf(most, (float)sum[t][r] * of_block * qs[r]);
                    most = over_rows_max(most);
                    const uint32_t j = j0 + 16 * (t0 + t) + i;
                    if (g == 0 && j < to) {
                        uint32_t key = ordered(most);
                        if (head0 != 0 && *key_of(j) > key) key = *key_of(j);
                        if (j < a.first || blocks - j <= a.last) key = kAlways;
                        *key_of(j) = able >> (16 * (t0 + t) + i) & 1 ? key : kNever;
                    }
                }
            }
            j0 += part_blocks(kSteps);
            if (j0 < to) begin(j0);
        }
    }
}

// Rows of any length, part by part.  What bounds it is memory: 32 requests of up to 2048 blocks, 8 kv heads of 128 (45 MB) take
// 14.9 us, 3.0 TB/s, some 4 of them the launch's; 1 of 8192 (17 MB) 8.6.  The heads of a part, whose entries and scales share
// lines, run on one XCD; parts go to the XCDs in turn.
template <class H, uint32_t kChunks, uint32_t kSteps>
__global__ __launch_bounds__(kScoreThreads, kChunks == 8 ? 2 : 4) void score_kernel(SelectArgs a) {
    __shared__ __align__(16) int8_t q8[16][64 * kChunks + 16];
    __shared__ float q_scale[16];
    const uint32_t in_xcd = blockIdx.x / kXcds, head = in_xcd % a.kv_heads;
    const uint32_t part = in_xcd / a.kv_heads * kXcds + blockIdx.x % kXcds;
    // (each row begins with another of its parts: those that every row has would otherwise all go to one XCD)
    const uint32_t request = part / a.parts, from = (part + request) % a.parts * part_blocks(kSteps);
    if (request >= a.requests) return;
    const uint32_t blocks = blocks_of(a, request);
    if (from >= blocks) return;
    const uint32_t to = blocks - from < part_blocks(kSteps) ? blocks : from + part_blocks(kSteps);
    uint32_t* keys = a.keys + ((size_t)request * a.kv_heads + head) * a.row_blocks;
    score<H, kChunks, kSteps>(a, request, head, from, to, blocks, q8, q_scale, [&](uint32_t j) { return keys + j; });
}

// ... and chosen from: 256 rows of up to 2048 keys 6.0 us, 8 of 8192 8.5.
template <uint32_t kHeld>
__global__ __launch_bounds__(kMostThreads) void choose_kernel(SelectArgs a) {
    __shared__ ChooseShared shared;
    const uint32_t list = blockIdx.x, blocks = blocks_of(a, list / a.kv_heads);
    const uint32_t* row_keys = a.keys + (size_t)list * a.row_blocks;
    if (HeldKeys<kMostThreads, kHeld>::holds(blocks)) {
        HeldKeys<kMostThreads, kHeld> keys(blocks);
#pragma unroll
        for (uint32_t s = 0; s < kHeld; ++s) {
            const uint32_t j = keys.part.first + 64 * s;
            keys.key[s] = s < keys.part.steps && j < blocks ? row_keys[j] : kNever;
        }
        choose_list<kMostThreads>(a, list, keys, shared);
    } else {
        auto read = [&](uint32_t j) { return row_keys[j]; };
        choose_list<kMostThreads>(a, list, ReadKeys<kMostThreads, decltype(read)>(blocks, read), shared);
    }
}

// Short rows, a workgroup each, whose keys stay in LDS: 8 lists of 100 blocks 7.3 us, 256 of 500 14.5.
template <class H, uint32_t kChunks, uint32_t kHeld>
__global__ __launch_bounds__(kScoreThreads, kChunks == 8 ? 2 : 4) void select_kernel(SelectArgs a) {
    __shared__ ChooseShared shared;
    __shared__ uint32_t row_keys[kScoreThreads * kHeld];
    __shared__ __align__(16) int8_t q8[16][64 * kChunks + 16];
    __shared__ float q_scale[16];
    const uint32_t list = blockIdx.x, request = list / a.kv_heads, blocks = blocks_of(a, request);
    score<H, kChunks, kMostSteps>(a, request, list % a.kv_heads, 0, blocks, blocks, q8, q_scale, [&](uint32_t j) { return row_keys + j; });
    __syncthreads();
    HeldKeys<kScoreThreads, kHeld> keys(blocks);
#pragma unroll
    for (uint32_t s = 0; s < kHeld; ++s) {
        const uint32_t j = keys.part.first + 64 * s;
        keys.key[s] = s < keys.part.steps && j < blocks ? row_keys[j] : kNever;
    }
    choose_list<kScoreThreads>(a, list, keys, shared);
}

template <class H, uint32_t kChunks, uint32_t kSteps>
void launch_score(SelectArgs& a, hipStream_t stream) {
    a.parts = (a.row_blocks + part_blocks(kSteps) - 1) / part_blocks(kSteps);
    const uint32_t parts = (a.requests * a.parts + kXcds - 1) / kXcds * kXcds;
    score_kernel<H, kChunks, kSteps><<<parts * a.kv_heads, kScoreThreads, 0, stream>>>(a);
}
template <class H, uint32_t kChunks>
void launch(SelectArgs& a, hipStream_t stream) {
    const uint32_t lists = a.requests * a.kv_heads;
    static_assert(kShortBlocks <= kScoreThreads * kFewHeld && kWholeBlocks <= kScoreThreads * kSomeHeld, "rows fit");
    if (a.row_blocks <= kShortBlocks) {
        select_kernel<H, kChunks, kFewHeld><<<lists, kScoreThreads, 0, stream>>>(a);
        return;
    }
    if (a.row_blocks <= kWholeBlocks && lists >= kListsToFill) {
        select_kernel<H, kChunks, kSomeHeld><<<lists, kScoreThreads, 0, stream>>>(a);
        return;
    }
    const uint64_t parts = (uint64_t)lists * ((a.row_blocks + part_blocks(kMostSteps) - 1) / part_blocks(kMostSteps));
    if (parts > kFewParts) launch_score<H, kChunks, kMostSteps>(a, stream);
    else launch_score<H, kChunks, 1>(a, stream);
    if (a.row_blocks <= kMostThreads * kFewHeld) choose_kernel<kFewHeld><<<lists, kMostThreads, 0, stream>>>(a);
    else if (a.row_blocks <= kMostThreads * kSomeHeld) choose_kernel<kSomeHeld><<<lists, kMostThreads, 0, stream>>>(a);
    else choose_kernel<kMostHeld><<<lists, kMostThreads, 0, stream>>>(a);
}
template <class H>
void launch(SelectArgs& a, hipStream_t stream) {
    if (a.head_dim <= 64) launch<H, 2>(a, stream);
    else if (a.head_dim <= 128) launch<H, 4>(a, stream);
    else launch<H, 8>(a, stream);
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
        !launchable((uint64_t)args->requests * args->kv_heads, kScoreThreads))
        return PGCM_ERR_ARG;   // (longer rows, that take more threads, are fewer by check_sizes)
    if (!aligned(args->q, args->q_request, args->q_head) || !aligned(args->bounds)) return PGCM_ERR_ALIGN;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const size_t room = select_room(args->requests, args->kv_heads, args->row_blocks);
    const std::lock_guard<std::mutex> held(kv->enqueue);
    if (const int rc = kv_ensure(kv, 0, room, stream)) return rc;
    SelectArgs a{};
    a.q = (const uint8_t*)args->q;
    a.tables = args->tables, a.lens = args->lens, a.bounds = args->bounds, a.scales = args->scales;
    a.selected = args->selected, a.counts = args->counts;
    a.keys = (uint32_t*)kv->scratch.at;
    a.q_request = 2 * args->q_request, a.q_head = 2 * args->q_head, a.table_row = args->table_row;
    a.requests = args->requests, a.kv_heads = args->kv_heads, a.group = args->heads / args->kv_heads;
    a.head_dim = args->head_dim, a.block_tokens = args->block_tokens, a.row_blocks = args->row_blocks;
    a.entry_count = args->entry_count, a.keep = args->keep, a.first = args->first, a.last = args->last;
    if (args->half == PGCM_KV_F16) launch<F16>(a, stream);
    else launch<Bf16>(a, stream);
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
    // four wavefronts a row, or sixteen for longer ones (8 rows of 2000 blocks: 7.7 us and 8.2; of 4000 9.3 and 9.1)
    constexpr uint32_t kFew = 256;
    const hipStream_t stream = (hipStream_t)hip_stream;
    if (!launchable(args->requests, a.row_blocks <= kFew * kSomeHeld ? kFew : kMostThreads)) return PGCM_ERR_ARG;
    if (a.row_blocks <= kFew * kFewHeld) evict_kernel<kFew, kFewHeld><<<args->requests, kFew, 0, stream>>>(a);
    else if (a.row_blocks <= kFew * kSomeHeld) evict_kernel<kFew, kSomeHeld><<<args->requests, kFew, 0, stream>>>(a);
    else if (a.row_blocks <= kMostThreads * kSomeHeld) evict_kernel<kMostThreads, kSomeHeld><<<args->requests, kMostThreads, 0, stream>>>(a);
    else evict_kernel<kMostThreads, kMostHeld><<<args->requests, kMostThreads, 0, stream>>>(a);
    return hip_noted(hipGetLastError()) ? PGCM_ERR_HIP : PGCM_OK;
}

#pragma GCC visibility pop
}  // extern "C"
