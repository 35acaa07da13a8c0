/*
 * pgcm_kv8: KV blocks in 8 bits, and attention with a window.  What a block's encryption, its way over the bus and its
 * reading cost goes by its bytes (paper section 2.1 on what is swapped); in 8 bits they are half as many.
 *
 *   pgcm_kv8_append   norms of queries and keys per head, rotation, keys and values into their slots in 8 bits
 *   pgcm_kv8_store    blocks of halves (pgcm_kv.h) to blocks in 8 bits
 *   pgcm_kv8_load     ... and back
 *   pgcm_kv8_attend   attention of new tokens of each request over blocks in 8 bits
 *   pgcm_kv_window    ... over blocks of halves, one or many new tokens of each request; both with a sliding window and a few
 *                     first tokens that stay visible
 *
 * A cache in 8 bits (pgcm_kv8_cache) has codes where pgcm_kv_cache has halves, and for each block and kv head a scale of its
 * keys and one of its values: a value is its code times the scale.  For codes and scales in one piece, as one chunk for
 * pgcm_encrypt_batch takes them, the scales' strides may step over the codes.
 *
 * Codes are whole numbers from -127 to 127 (PGCM_KV8_INT8) or numbers of 4 bits of exponent and 3 of fraction, up to 448
 * (PGCM_KV8_E4M3).  Scales that this library writes are powers of two, 2^e with the least e from -100 on for which 2^e times
 * 127 or 448 reaches the largest |x| of the block's tokens and of the head; a code is x / 2^e, rounded once, to nearest, ties to even.
 * So reading back is exact in binary32, and in halves but for the ends of their range; and a scale that has to grow while a
 * block fills doubles, so that the codes that are there are rounded again at most once for each doubling, which adds up to
 * less than one step of the last scale in int8, and in e4m3 changes only codes that fall below its least normal number.
 * A cache may hold other scales above zero; append keeps the larger of what is there and what its values need, and 0 for none.
 * If a value is infinite or NaN the head's scale of that block is NaN, and the codes that come with it are zero: nothing that is
 * read from there is taken for a number.
 *
 * Conventions are those of pgcm.h and pgcm_kv.h, workspaces and alignment among them: rows of codes are 16-byte aligned, with
 * strides that are multiples of 16, head_dim is a multiple of 16 here.  Results do not depend on the order in which workgroups run.
 */
#ifndef PGCM_KV8_H
#define PGCM_KV8_H

#include "pgcm_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PGCM_KV8_INT8 = 0, PGCM_KV8_E4M3 = 1 } pgcm_kv8_code;

typedef struct {
    void *k, *v;                 /* DEVICE codes */
    float *k_scales, *v_scales;  /* DEVICE */
    uint32_t code;               /* pgcm_kv8_code */
    uint32_t half;               /* pgcm_kv_half: of queries, keys and values that go in and of what comes out */
    uint32_t blocks;             /* of the pool, at least 1 */
    uint32_t block_tokens;
    uint32_t kv_heads;
    uint32_t head_dim;           /* a multiple of 16 up to 256 */
    int64_t k_block, k_token, k_head; /* strides in codes; those of tokens in [0, 2^25] for pgcm_kv8_attend (and, in halves,
                                         for pgcm_kv_window) */
    int64_t v_block, v_token, v_head;
    int64_t k_scale_block, k_scale_head, v_scale_block, v_scale_head; /* in floats */
} pgcm_kv8_cache;

/*
 * As pgcm_kv_append, with k and v rounded once, to their codes.  Tokens of the call whose slots lie in one block follow each other
 * in `slots`, each slot one more than the one before; a call names each block in one such run.  A run that begins with its
 * block's first token starts the block anew; any other raises the block's scales, where its values need that, from what they
 * are (never lowers them), and then the codes of the tokens before the run are rounded to the new scale.  What the block holds
 * behind the run no longer counts.  A slot outside the pool is not written.  Strides of tokens of k, v and of the cache are in
 * [0, 2^23].
 */
int pgcm_kv8_append(const pgcm_kv8_cache *cache, const pgcm_kv_append_args *args, void *hip_stream);

/*
 * n blocks' first tokens, from `from` (block from_blocks[i], or blocks[i] if NULL) to `to` (block blocks[i]).  counts: DEVICE
 * [n], tokens of each (cut to [0, block_tokens]), or NULL: all.  Both caches have the same sizes but for the number of blocks, and
 * one `half`.  A block outside its pool is passed over; no block of `to` is named twice.  Store starts each block anew, with the
 * scales of those tokens; places behind them are left as they are, in both directions.  Load rounds once to a half; a finite
 * product beyond its range becomes its largest number, however far beyond it is.  Of blocks that store made, only what rounding
 * to a code has put there is (2^16 in binary16).  Append rounds values of 32 bits to codes, and scales of others may be any: such
 * a value of a binary16 cache may be far beyond 65504.  pgcm_kv8_attend takes it as it is, load makes it 65504, where
 * pgcm_kv_append would have made it infinite.
 */
int pgcm_kv8_store(const pgcm_kv8_cache *to, const pgcm_kv_cache *from, uint32_t n, const int32_t *blocks, const int32_t *counts,
                   const int32_t *from_blocks, void *hip_stream);
int pgcm_kv8_load(const pgcm_kv8_cache *from, const pgcm_kv_cache *to, uint32_t n, const int32_t *blocks, const int32_t *counts,
                  const int32_t *to_blocks, void *hip_stream);

typedef struct {
    uint32_t requests, heads;          /* heads: query heads, a multiple of kv_heads: head h reads kv head h / (heads / kv_heads) */
    uint32_t tokens;                   /* rows of q and out; `requests` if starts is NULL */
    uint32_t most;                     /* no request has more new tokens; 1 if starts is NULL */
    const int32_t *starts;             /* DEVICE [requests + 1], ascending: request b's new tokens are rows starts[b] up to
                                          starts[b + 1] (cut to [0, tokens], and to `most` rows); NULL: row b */
    const void *q;                     /* DEVICE halves [tokens][heads][head_dim] */
    int64_t q_token, q_head;
    const int32_t *tables;             /* DEVICE [requests][row_blocks], rows table_row elements apart */
    int64_t table_row;
    uint32_t row_blocks;
    float scale;                       /* of q . k; finite */
    const int32_t *lens;               /* DEVICE [requests]: tokens of each, the new ones, its last ones, among them */
    uint32_t window;                   /* how many tokens a token sees, itself among them; 0: all */
    uint32_t sinks;                    /* ... and so many first tokens of its request */
    void *out;                         /* DEVICE halves [tokens][heads][head_dim]; not q */
    int64_t out_token, out_head;
    float *lse;                        /* DEVICE [tokens][heads], or NULL: log of the sum of exp(scale q . k) */
} pgcm_kv_window_args;
/*
 * The new token at place p of its request (the last one's place is its length - 1) attends to the tokens t <= p that are on the
 * device and for which t > p - window or t < sinks: out = sum softmax(scale q . k) v.  A token that sees none gives zeros and a
 * lse of minus infinity.  Rows of q that no request has are not read, and those of out and lse left as they are.
 * What lies in the pool beyond what a token sees has no part in its results, whatever it holds.
 * A score that is NaN or plus infinity makes its row's results NaN, one of minus infinity has no weight.  A value that is not finite
 * makes its channel infinite or NaN in the rows that see it.
 * Softmax weights are multiplied with values as sums of halves, and added up as they are.  One new token of each request, and
 * always in pgcm_kv8_attend: they leave nothing out over bfloat16 blocks of halves, else 2^-22 of a weight at most, or 2^-38 of the
 * row's largest where that is more.  More of them over blocks of halves: 2^-16 of a weight at most in bfloat16, in binary16 as much
 * as one does.
 * In pgcm_kv8_attend a query is multiplied as a power of two times binary16 numbers, its largest channel near 2^14: what of a
 * bfloat16 channel lies below 2^-38 of that one is rounded away, and a row whose largest is below 2^-126 counts as zero.  One with
 * a channel that is not finite makes its results NaN where it sees a token that is on the device, whatever its scores are.
 * Sums of values are held in binary32 times 2^15 and less: values beyond 2^88 may leave its range.
 * One new token of each request without a window is also what pgcm_kv_attend does, which takes 3 % less time in large batches, 30 %
 * less in small ones of some 1000 tokens, and 5 to 25 % more for one request of some 4000 tokens or a few of 100000.
 */
int pgcm_kv8_attend(pgcm_kv_t *kv, const pgcm_kv8_cache *cache, const pgcm_kv_window_args *args, void *hip_stream);
int pgcm_kv_window(pgcm_kv_t *kv, const pgcm_kv_cache *cache, const pgcm_kv_window_args *args, void *hip_stream);
/* Room of a workspace for any calls of both with at most these sizes: what many new tokens may take, 35 MB with up to 64 channels,
 * 68 with up to 128, 135 with more, and half as much again.  A call by itself asks for what it takes, single tokens for a quarter of
 * that at most (1 MB for each query head of a kv head, with 128 channels). */
int pgcm_kv_window_reserve(pgcm_kv_t *kv, uint32_t heads, uint32_t kv_heads, uint32_t head_dim, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PGCM_KV8_H */
