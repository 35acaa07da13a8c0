/*
 * pgcm_kv: what a serving runtime does, between two swaps, with the KV blocks that this library encrypts and
 * decrypts (paper section 2.1 on what is swapped, section 5.1 on when): new keys and values are appended to a
 * layer's blocks, one new token of each request attends over them in place, and which blocks are read next or
 * swapped out next is decided from the blocks themselves.
 *
 *   pgcm_kv_append     norms of queries and keys per head, rotation by position, keys and values into their slots
 *   pgcm_kv_attend     attention of one new token of each request over its blocks; blocks that are swapped out are
 *                      masked; optionally the attention weight that each block has gathered
 *   pgcm_kv_summarize  bounds of a block's keys, in 8 bits
 *   pgcm_kv_select     by those bounds, the best blocks of a request for each kv head
 *   pgcm_kv_evict      the blocks with the least gathered weight: to be swapped out
 *
 * A cache (pgcm_kv_cache) is one layer's view of a pool of blocks: element (block, token, head, channel) of the keys
 * is k[block * k_block + token * k_token + head * k_head + channel], the values likewise.  A block of
 * [K, V][token][head][channel] is one chunk for pgcm_encrypt_batch.  A request has a row of block numbers: block j
 * holds its tokens j * block_tokens and on.  A number outside [0, blocks) says that the block is not on the device.
 * A length beyond the row's blocks is cut to them, one below zero is zero.
 *
 * Conventions are those of pgcm.h: DEVICE and HOST pointers, work enqueued on `hip_stream` without synchronising, errors as
 * return codes with nothing enqueued after an argument error.  "half" below is the cache's type, IEEE binary16 or
 * bfloat16; sums, softmax statistics and norms are held in binary32, and each output is rounded once.  Rows of halves
 * are read in pieces of 16 bytes: their pointers are 16-byte aligned and their strides multiples of 8 elements
 * (otherwise PGCM_ERR_ALIGN); head_dim is a multiple of 8 up to 256, block_tokens a multiple of 16 up to 4096.
 * A call for which a launch would need 2^32 threads is refused: some 2^24 tokens, blocks' heads, lists or rows, 2^22 rows of
 * more than 2048 blocks to evict from.  Results do not depend on the order in which workgroups run.
 */
#ifndef PGCM_KV_H
#define PGCM_KV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PGCM_KV_F16 = 0, PGCM_KV_BF16 = 1 } pgcm_kv_half;

typedef struct {
    void *k, *v;           /* DEVICE */
    uint32_t half;         /* pgcm_kv_half */
    uint32_t blocks;       /* of the pool, at least 1 */
    uint32_t block_tokens;
    uint32_t kv_heads;
    uint32_t head_dim;
    uint32_t reserved;     /* 0 */
    int64_t k_block, k_token, k_head; /* strides in elements; those of tokens in [0, 2^25] for pgcm_kv_attend */
    int64_t v_block, v_token, v_head;
} pgcm_kv_cache;

/*
 * Workspace of pgcm_kv_attend and pgcm_kv_select on the current device.  Calls that use one object go on one stream,
 * or are ordered by the caller; any number of threads may make them.  It grows when a call needs more (that call
 * allocates; on a stream that is being captured it fails with PGCM_ERR_CAPACITY instead) and never shrinks; what it
 * outgrew lives until it is destroyed, so a captured graph may be replayed until then, in the order of the object's
 * other calls.
 */
typedef struct pgcm_kv pgcm_kv_t;
int pgcm_kv_create(pgcm_kv_t **out);
void pgcm_kv_destroy(pgcm_kv_t *kv); /* NULL is allowed; the caller has synchronised the streams that use it */
/* Room for calls of at most these sizes: requests, query heads and kv heads, tokens of a block, blocks of a row. */
int pgcm_kv_reserve(pgcm_kv_t *kv, uint32_t requests, uint32_t heads, uint32_t kv_heads, uint32_t head_dim,
                    uint32_t block_tokens, uint32_t row_blocks, void *hip_stream);

typedef struct {
    uint32_t tokens, heads;            /* heads: query heads, a multiple of kv_heads; 0 with q == NULL */
    const void *q, *k, *v;             /* DEVICE halves: q [tokens][heads][head_dim], k and v [tokens][kv_heads][head_dim] */
    int64_t q_token, q_head, k_token, k_head, v_token, v_head;
    const int32_t *positions;          /* DEVICE [tokens]; NULL if rope is */
    const int64_t *slots;              /* DEVICE [tokens]: block * block_tokens + token in it; a slot outside the pool
                                          is not written.  Two tokens of a call do not share a slot */
    const void *q_weight, *k_weight;   /* DEVICE halves [head_dim], or NULL: that norm is left out */
    float eps;
    uint32_t adjacent;                 /* pairs of the rotation: (d, d + rope_dim / 2), or, not 0, (2 d, 2 d + 1) */
    const float *rope;                 /* DEVICE [rope_positions][rope_dim]: cosines, then sines, of the rope_dim / 2 pairs; or NULL */
    uint32_t rope_positions, rope_dim; /* rope_dim: a multiple of 16 up to head_dim; channels beyond it are not rotated */
    void *q_out;                       /* DEVICE halves [tokens][heads][head_dim]; may be q */
    int64_t q_out_token, q_out_head;
} pgcm_kv_append_args;
/*
 * For each token and head x of q and k: x <- x / sqrt(mean(x^2) + eps) * weight, rounded nowhere in between, then its
 * pairs (a, b) turned: (a cos - b sin, b cos + a sin).  A position outside the table makes the head's rotated channels NaN.
 */
int pgcm_kv_append(const pgcm_kv_cache *cache, const pgcm_kv_append_args *args, void *hip_stream);

typedef struct {
    uint32_t requests, heads;          /* heads: query heads, a multiple of kv_heads: head h reads kv head h / (heads / kv_heads) */
    const void *q;                     /* DEVICE halves [requests][heads][head_dim] */
    int64_t q_request, q_head;
    const int32_t *tables;             /* DEVICE [requests][row_blocks], rows table_row elements apart */
    int64_t table_row;
    uint32_t row_blocks;
    float scale;                       /* of q . k; finite */
    const int32_t *lens;               /* DEVICE [requests]: tokens of each */
    const int32_t *selected;           /* DEVICE [requests][kv_heads][keep], or NULL: places in the request's row that this kv
                                          head reads, each at most once; what lies outside the request's blocks is passed over */
    uint32_t keep;                     /* 0: nothing is read */
    float decay;
    void *out;                         /* DEVICE halves [requests][heads][head_dim] */
    int64_t out_request, out_head;
    float *lse;                        /* DEVICE [requests][heads], or NULL: log of the sum of exp(scale q . k) */
    const float *kept;                 /* DEVICE [requests][row_blocks], or NULL: zeros */
    float *weights;                    /* DEVICE [requests][row_blocks], or NULL; not with `selected`; may be kept */
} pgcm_kv_attend_args;
/*
 * out = sum over the request's tokens that are on the device of softmax(scale q . k) v; a request without any gives zeros and
 * a lse of minus infinity.  What lies in the pool beyond a request's tokens is not used, whatever it holds.
 * A score that is NaN or plus infinity makes its head's results NaN, one of minus infinity has no weight.
 * A value that is not finite makes its channel so: infinite, or NaN if infinities of both signs meet.  (Where its weight is
 * less than 2^-100 of the head's largest, infinite or NaN.)
 * weights[b][j] = decay * kept[b][j] + the weights of block j's tokens, summed over the heads.
 * Softmax weights are multiplied with v as sums of halves, and added up in binary32: three (bfloat16) leave nothing out, two
 * (binary16) 2^-22 of a weight at most, or 2^-38 of the head's largest where that is more.  In bfloat16 sums of values
 * beyond 2^88 may leave the range of binary32.
 */
int pgcm_kv_attend(pgcm_kv_t *kv, const pgcm_kv_cache *cache, const pgcm_kv_attend_args *args, void *hip_stream);

/*
 * Bounds of n blocks' keys.  blocks: DEVICE [n], counts: DEVICE [n], tokens of each that are there (cut to
 * [0, block_tokens]); entries: DEVICE [n], where the results go, or NULL: at the blocks' numbers.  A block or an entry
 * outside its pool is passed over.  For each head, with a = the largest |k| of the block (below 1e-30, or without tokens: 0):
 *   bounds: DEVICE [entry_count][kv_heads][2][head_dim], 16-byte aligned: the least and the largest value of each channel
 *           times 127 / a, to the nearest whole number (ties to even)
 *   scales: DEVICE [entry_count][kv_heads]: a / 127
 * Both quotients are rounded to binary32.  Infinities and NaN count as zero.
 */
int pgcm_kv_summarize(const pgcm_kv_cache *cache, uint32_t n, const int32_t *blocks, const int32_t *counts,
                      const int32_t *entries, uint32_t entry_count, int8_t *bounds, float *scales, void *hip_stream);

typedef struct {
    uint32_t requests, heads, kv_heads, head_dim;
    uint32_t half;                     /* of q */
    uint32_t block_tokens;
    const void *q;                     /* DEVICE halves [requests][heads][head_dim] */
    int64_t q_request, q_head;
    const int32_t *tables;             /* DEVICE [requests][row_blocks]: the entry of each block's bounds; a block whose
                                          number lies outside [0, entry_count) cannot be selected */
    int64_t table_row;
    uint32_t row_blocks;
    uint32_t entry_count;
    const int32_t *lens;               /* DEVICE [requests] */
    const int8_t *bounds;              /* as pgcm_kv_summarize leaves them */
    const float *scales;
    uint32_t keep;                     /* blocks of each list, at least 1 */
    uint32_t first, last;              /* so many blocks at a request's ends go before all others */
    int32_t *selected;                 /* DEVICE [requests][kv_heads][keep]: places in the row, ascending, then -1 */
    int32_t *counts;                   /* DEVICE [requests][kv_heads], or NULL: how many */
} pgcm_kv_select_args;
/*
 * The score of a block estimates the largest that q . k may be for keys within its bounds: with c = round(q * (127 / a)) of
 * each head, a its largest |q|, and s = a / 127 (as for the bounds),  max over the group's heads of
 * (sum_d max(c low, c high) * scale) * s.  The sum is exact, the products are rounded to binary32 in this order.  It is not a
 * bound itself, as c, low and high are rounded to nearest: q . k is at most
 * (sum_d (max(c low, c high) + (|c| + max(|low|, |high|)) / 2 + 1/4)) * scale * s.
 * The largest scores win, among equal ones the first; and among the blocks at the ends, where keep is less than those, the
 * first.
 */
int pgcm_kv_select(pgcm_kv_t *kv, const pgcm_kv_select_args *args, void *hip_stream);

typedef struct {
    uint32_t requests, row_blocks, block_tokens;
    uint32_t blocks;                   /* of the pool */
    const float *weights;              /* DEVICE [requests][row_blocks] */
    const int32_t *tables;             /* DEVICE [requests][row_blocks], rows table_row elements apart */
    int64_t table_row;
    const int32_t *lens;               /* DEVICE [requests] */
    const int32_t *evict;              /* DEVICE [requests]: how many of each */
    uint32_t most;                     /* ... and at most */
    uint32_t first, last;              /* so many blocks at a request's ends stay */
    int32_t *victims;                  /* DEVICE [requests][most]: places in the row, ascending, then -1 */
    int32_t *victim_blocks;            /* DEVICE [requests][most], or NULL: their block numbers, then -1 */
    int32_t *tables_out;               /* DEVICE [requests][row_blocks], rows table_out_row apart, or NULL: tables with -1
                                          in the victims' places; may be tables */
    int64_t table_out_row;
} pgcm_kv_evict_args;
/* The blocks on the device with the least weights, among equal ones the first; NaN is more than any number. */
int pgcm_kv_evict(const pgcm_kv_evict_args *args, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PGCM_KV_H */
