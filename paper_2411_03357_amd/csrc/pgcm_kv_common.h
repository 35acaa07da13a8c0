// What the operators on KV blocks share: the two 16-bit types, argument checks and the workspace.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <mutex>
#include <vector>

#include "../../include/pgcm.h"
#include "../../include/pgcm_kv.h"

namespace pgcm {
// for pgcm_last_hip_error; true if e is an error
bool hip_noted(hipError_t e);
}  // namespace pgcm

// A workspace: counters, zero between calls, and scratch that means nothing between calls.
struct pgcm_kv {
    struct Memory {
        uint8_t* at = nullptr;
        size_t bytes = 0;
    };
    int device = 0;
    std::mutex enqueue;  // held while a call's launches are enqueued, which leave to each other what lies in scratch
    Memory counters, scratch;
    std::vector<void*> outgrown;  // a captured graph may still name them
};

namespace pgcm_kv_impl {

constexpr uint32_t kPiece = 16;  // tokens of a matrix-core tile: a block is a whole number of pieces
constexpr uint32_t kMaxHeadDim = 256;
constexpr uint32_t kMaxHeads = 65535;
constexpr uint32_t kXcds = 8;
constexpr uint32_t kTileTokens = 128;  // tokens that a workgroup of attention takes at a step

// At least so many bytes of zeroed counters and of scratch; kv->enqueue is held.
int kv_ensure(pgcm_kv* kv, size_t counters, size_t scratch, hipStream_t stream);

inline bool aligned(const void* p, const int64_t a = 0, const int64_t b = 0, const int64_t c = 0) {
    return ((uintptr_t)p & 15) == 0 && ((a | b | c) & 7) == 0;
}

inline int check_shape(uint32_t kv_heads, uint32_t head_dim, uint32_t block_tokens) {
    if (kv_heads == 0 || kv_heads > kMaxHeads || head_dim == 0 || head_dim % 8 != 0 || head_dim > kMaxHeadDim ||
        block_tokens == 0 || block_tokens % kPiece != 0 || block_tokens > 4096)
        return PGCM_ERR_ARG;
    return PGCM_OK;
}

// Sizes of a call on a batch of requests.  What kernels count in 32 bits stays below 2^31: blocks of all rows,
// and tiles of attention for each head.
inline int check_sizes(uint32_t requests, uint32_t heads, uint32_t kv_heads, uint32_t head_dim, uint32_t block_tokens,
                       uint32_t row_blocks) {
    if (const int rc = check_shape(kv_heads, head_dim, block_tokens)) return rc;
    if (heads == 0 || heads > kMaxHeads || heads % kv_heads != 0) return PGCM_ERR_ARG;
    if ((uint64_t)row_blocks * block_tokens > 0x7FFFFFFFull) return PGCM_ERR_ARG;
    const uint64_t groups = kv_heads * (uint64_t)((heads / kv_heads + kPiece - 1) / kPiece);
    const uint64_t tiles = ((uint64_t)row_blocks * block_tokens + kTileTokens - 1) / kTileTokens;
    if (requests != 0 && (groups * requests > 0x7FFFFFFFull || tiles * groups > 0x7FFFFFFFull / requests ||
                          (uint64_t)row_blocks * kv_heads > 0x7FFFFFFFull / requests))
        return PGCM_ERR_ARG;
    return PGCM_OK;
}

inline int check_cache(const pgcm_kv_cache* c) {
    if (c == nullptr || c->k == nullptr || c->v == nullptr || c->half > PGCM_KV_BF16 || c->reserved != 0 ||
        c->blocks == 0 || c->blocks > 0x7FFFFFFFu)
        return PGCM_ERR_ARG;
    if (const int rc = check_shape(c->kv_heads, c->head_dim, c->block_tokens)) return rc;
    if (!aligned(c->k, c->k_block, c->k_token, c->k_head) || !aligned(c->v, c->v_block, c->v_token, c->v_head))
        return PGCM_ERR_ALIGN;
    return PGCM_OK;
}

// Threads of a launch are counted in 32 bits, in each dimension of the grid.
inline bool launchable(uint64_t groups, uint32_t threads) { return groups * threads <= 0xFFFFFFFFull; }

// ---- workspace
struct Room {
    size_t counters, scratch;
};
inline size_t whole_lines(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Attention: two partial results for each workgroup, and for each of these two counters; and, for weights, log-sums of heads
// and of each piece of a row.
constexpr uint32_t kAttendGroups = 512;  // workgroups of a launch, at most
inline size_t partial_floats(uint32_t head_dim, uint32_t group) {
    return (size_t)(group < 16 ? group : 16) * ((head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256) + 2);
}
inline Room attend_room(uint32_t requests, uint32_t heads, uint32_t kv_heads, uint32_t head_dim, uint64_t row_pieces) {
    return Room{4 * 2 * 2 * kAttendGroups, whole_lines(4 * partial_floats(head_dim, heads / kv_heads) * 2 * kAttendGroups) +
                               whole_lines(4 * (size_t)requests * heads) + 4 * (size_t)requests * heads * row_pieces};
}

// Selection: a key for each block of a request and kv head.
inline size_t select_room(uint32_t requests, uint32_t kv_heads, uint32_t row_blocks) {
    return 4 * (size_t)requests * kv_heads * row_blocks;
}

// ---- device side
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct F16 {
    typedef _Float16 one;
    typedef f16x8 eight;
    static constexpr uint32_t kInfinity = 0x7C00;
    // Weights of attention, as powers of 2: the largest ones near the end of the range, since the least that a half can tell
    // apart, 2^-24, is then 2^-37 of them; beside a weight of 1, 2^-21 would keep three bits.
    static constexpr float kLargest = 13.f, kOverflows = 15.f;
    static __device__ __forceinline__ f32x4 product(eight a, eight b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    // x as the sum of halves of 11 bits, the first towards zero: all but 2^-22 of it
    static constexpr uint32_t kHalves = 2;
    static __device__ __forceinline__ void split(const float (&x)[8], eight (&halves)[kHalves]) {
#pragma unroll
        for (uint32_t e = 0; e < 8; e += 2) {
            const auto h = __builtin_amdgcn_cvt_pkrtz(x[e], x[e + 1]);
            halves[0][e] = (one)h[0], halves[0][e + 1] = (one)h[1];
        }
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) halves[1][e] = (one)(x[e] - (float)halves[0][e]);
    }
};
struct Bf16 {
    typedef __bf16 one;
    typedef bf16x8 eight;
    static constexpr uint32_t kInfinity = 0x7F80;
    static constexpr float kLargest = 0.f, kOverflows = 8.f;   // (the range is that of a float)
    static __device__ __forceinline__ f32x4 product(eight a, eight b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    // x as the sum of halves of 8 bits, towards zero: all of it
    static constexpr uint32_t kHalves = 3;
    static __device__ __forceinline__ void split(const float (&x)[8], eight (&halves)[kHalves]) {
        float left[8];
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) left[e] = x[e];
#pragma unroll
        for (uint32_t n = 0; n < kHalves; ++n) {
            uint32_t words[4];
#pragma unroll
            for (uint32_t e = 0; e < 8; e += 2) {   // (the upper half of a float is its bfloat16 towards zero)
                const uint32_t a = __builtin_bit_cast(uint32_t, left[e]), b = __builtin_bit_cast(uint32_t, left[e + 1]);
                words[e / 2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
                left[e] -= __builtin_bit_cast(float, a & 0xFFFF0000u);
                left[e + 1] -= __builtin_bit_cast(float, b & 0xFFFF0000u);
            }
            halves[n] = __builtin_bit_cast(eight, words);
        }
    }
};

template <class H>
__device__ __forceinline__ typename H::eight as_eight(uint4 x) {
    return __builtin_bit_cast(typename H::eight, x);
}
template <class H>
__device__ __forceinline__ uint4 as_words(typename H::eight x) {
    return __builtin_bit_cast(uint4, x);
}

// Over the sixteen lanes of a row, and over the four rows: each lane gets the result.
template <uint32_t kPattern>
__device__ __forceinline__ float from_lane(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kPattern, 0xF, 0xF, true));
}
constexpr uint32_t kPairs = 0xB1, kQuads = 0x4E, kMirrorEight = 0x141, kMirrorRow = 0x140;  // DPP: lanes 1, 2 apart; mirrored
__device__ __forceinline__ float row_max(float x) {
    x = fmaxf(x, from_lane<kPairs>(x));
    x = fmaxf(x, from_lane<kQuads>(x));
    x = fmaxf(x, from_lane<kMirrorEight>(x));
    return fmaxf(x, from_lane<kMirrorRow>(x));
}
struct Two {
    float a, b;
};
// of rows 0 and 1, 2 and 3: the first, the second of the pair; of both pairs of rows: the first, the second
__device__ __forceinline__ Two of_row_pairs(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto y = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a = y[0], b = y[1];   // (of an element of a vector, the cast below takes the vector's first)
    return Two{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ __forceinline__ Two of_halves(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto y = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = y[0], b = y[1];   // (of an element of a vector, the cast below takes the vector's first)
    return Two{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ __forceinline__ float over_rows_max(float x) {
    const Two p = of_row_pairs(x), h = of_halves(fmaxf(p.a, p.b));
    return fmaxf(h.a, h.b);
}
__device__ __forceinline__ float over_rows_sum(float x) {
    const Two p = of_row_pairs(x), h = of_halves(p.a + p.b);
    return h.a + h.b;
}
// the least or largest whole number of the wavefront
template <class Of>
__device__ __forceinline__ uint32_t over_wave(uint32_t x, Of of) {
    x = of(x, (uint32_t)__builtin_amdgcn_update_dpp(0, x, kPairs, 0xF, 0xF, true));
    x = of(x, (uint32_t)__builtin_amdgcn_update_dpp(0, x, kQuads, 0xF, 0xF, true));
    x = of(x, (uint32_t)__builtin_amdgcn_update_dpp(0, x, kMirrorEight, 0xF, 0xF, true));
    x = of(x, (uint32_t)__builtin_amdgcn_update_dpp(0, x, kMirrorRow, 0xF, 0xF, true));
    const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = of(p[0], p[1]);
    const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return of(h[0], h[1]);
}
// inclusive sums over the wavefront: in rows, then the rows before
__device__ __forceinline__ uint32_t scan(uint32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);  // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // row_bcast:31 into rows 2 and 3
    return x;
}

// Four-byte and eight-byte words that other workgroups of the launch read: written through to where every XCD
// sees them, and read from there.  (A device-scope fence would write back or drop a whole L2.)
template <class T>
__device__ __forceinline__ void put_shared(T* at, T v) {
    __hip_atomic_store(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class T>
__device__ __forceinline__ T get_shared(const T* at) {
    return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// All of this wavefront's stores have arrived there.
__device__ __forceinline__ void stores_arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Whether the calling workgroup is the last of `of` to arrive; the counter is left zero then.  What the others put
// before arriving can be got afterwards.  All threads call it; *word is in LDS.
__device__ __forceinline__ bool last_to_arrive(uint32_t* counter, uint32_t of, uint32_t* word) {
    stores_arrived();
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before + 1 == of) put_shared(counter, 0u);
        *word = before + 1 == of;
    }
    __syncthreads();
    return *word != 0;
}

}  // namespace pgcm_kv_impl
