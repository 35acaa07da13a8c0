// What the kernels of attention with a window share (include/pgcm_kv8.h): their arguments, which tokens a row sees, and how a
// call's results are put together.
#pragma once
#include "pgcm_kv8_common.h"

namespace pgcm_kv_impl {

struct WindowArgs {
    const uint8_t *k, *v, *q;
    uint8_t* out;
    const float *k_scales, *v_scales;   // of codes
    const int32_t *tables, *lens, *starts;
    float *lse, *partials;
    uint32_t* counters;
    int64_t k_block, k_token, k_head, v_block, v_token, v_head, q_token, q_head, out_token, out_head;  // bytes
    int64_t k_scale_block, k_scale_head, v_scale_block, v_scale_head;
    int64_t table_row;
    uint32_t requests, tokens, most, kv_heads, group, head_dim, block_tokens, row_blocks, blocks, window, sinks;
    float scale;  // times log2 e
};

// ---- device side

__device__ __forceinline__ uint32_t clamped(int32_t x, uint32_t most) {
    return x <= 0 ? 0u : (uint32_t)x < most ? (uint32_t)x : most;
}
__device__ __forceinline__ float exp2_from(float x, float top) {  // 0 for x = -inf, whatever the top
    return __builtin_amdgcn_exp2f(x - (top == -INFINITY ? 0.f : top));
}

// The tokens that a run of rows, of places first ... last of a request, may see: below `lead` pieces of sixteen from the start,
// and pieces [from, to).
struct Seen {
    uint32_t lead, from, to;
    __device__ __forceinline__ uint32_t pieces() const { return lead + to - from; }
    __device__ __forceinline__ uint32_t piece(uint32_t x) const { return x < lead ? x : x - lead + from; }
};
// the first token of the window of a row that sees tokens below `end`
__device__ __forceinline__ uint32_t low_of(const WindowArgs& a, uint32_t end) {
    return a.window == 0 || end <= a.window ? 0 : end - a.window;
}
// ends: one more than the places of the first row and of the last; 0 for a row before its request's first token
__device__ __forceinline__ Seen seen_of(const WindowArgs& a, uint32_t first_end, uint32_t last_end) {
    Seen s;
    s.from = low_of(a, first_end) / kPiece;
    s.to = (last_end + kPiece - 1) / kPiece;
    if (s.from > s.to) s.from = s.to;
    const uint32_t sinks = a.sinks < last_end ? a.sinks : last_end, of_sinks = (sinks + kPiece - 1) / kPiece;
    s.lead = of_sinks < s.from ? of_sinks : s.from;
    return s;
}

}  // namespace pgcm_kv_impl

namespace pgcm_kv_impl {
// Launches of the two kinds of kernels; args are checked.  code: pgcm_kv8_code, or ~0: blocks of halves.
int window_few(pgcm_kv* kv, WindowArgs& a, uint32_t half, uint32_t code, hipStream_t stream);
int window_many(pgcm_kv* kv, WindowArgs& a, uint32_t half, hipStream_t stream);
Room window_few_room(uint32_t heads, uint32_t kv_heads, uint32_t head_dim);
Room window_many_room(uint32_t head_dim);
}  // namespace pgcm_kv_impl
