/*
 * isjl_kv.h -- C ABI of a decode step over a paged KV cache.
 *
 * The simulator (isjl_sim.h) decides which requests run in a step, and charges
 * the step c + tau * |S| * max r.  This part of the library is that step on the
 * machine below the schedule: every running request gets one token, whose key
 * and value need a place in the KV memory that the schedule reserves, and whose
 * query attends to what the request has there.  A step is
 *
 *   isjl_kv_assign   block tables and slot maps from request lengths
 *   isjl_kv_append   norms and position rotation of the new queries and keys,
 *                    keys and values written to their slots
 *   isjl_kv_attend   attention of each query over its request's tokens: all of
 *                    them, or a sliding window and a few first tokens; with or
 *                    without a prefix that all requests share
 *
 * The cache.  Key and value caches hold n_blocks blocks of block_size tokens;
 * element [b][s][h][d] lies at b * stride[0] + s * stride[1] + h * stride[2] + d
 * (strides in elements).  Slot number b * block_size + s.  Row i of a block table
 * names the blocks that hold request i's own tokens in order; tokens of a shared
 * prefix lie in blocks of their own, named once for the whole batch, and come
 * before every request's own tokens.
 *
 * Conventions are those of isjl_sim.h: device pointers unless said otherwise
 * (numbers at multiples of their size, what holds heads at multiples of 16 bytes),
 * stream is a cudaStream_t passed as void*, calls are asynchronous on it and
 * allocate nothing (they can be captured into a graph), no entry point throws,
 * traps or aborts, errors are isjl_status codes.  What only the device can see is
 * reported by isjl_kv_status and skipped: tokens in a block whose number is outside
 * the cache read as 0, a request whose length is beyond its table's width is
 * inactive, a token with a slot or position out of range is padding, a token that
 * assign finds a block number outside the cache for gets slot -1.  A handle holds the workspace of its calls: they must not
 * overlap on the GPU, and a handle is not thread safe.  It belongs to the device that was current when it was created:
 * with another one current its calls are refused (INVALID_ARG), the report too; it can be destroyed.
 */
#ifndef ISJL_KV_H
#define ISJL_KV_H

#include <stdint.h>

#include "isjl_sim.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    ISJL_KV_BF16 = 0,
    ISJL_KV_FP16 = 1
} isjl_kv_type;

#define ISJL_KV_MAX_ROWS 4096   /* most queries of one isjl_kv_attend call */

typedef struct {
    int32_t n_blocks;     /* blocks of the cache, >= 1 */
    int32_t block_size;   /* tokens of a block: 8, 16, 32, 64, 128 or 256 */
    int32_t n_q_heads;    /* a multiple of n_kv_heads, at most 1024 */
    int32_t n_kv_heads;   /* >= 1; query head h reads key head h / (n_q_heads / n_kv_heads) */
    int32_t head_dim;     /* 64, 128 or 256 */
    int32_t type;         /* isjl_kv_type of queries, keys, values and outputs */
    int32_t max_rows;     /* most rows of isjl_kv_assign; most queries of isjl_kv_attend (there also
                             at most ISJL_KV_MAX_ROWS) */
} isjl_kv_config;

/* Device memory of the two caches, 16-byte aligned; strides of block, slot and
 * head in elements, each a positive multiple of 8. */
typedef struct {
    void *k;
    void *v;
    int64_t k_stride[3];
    int64_t v_stride[3];
} isjl_kv_cache;

/* One step's new tokens.  Row i holds lens[i] own tokens and asks for
 * new_tokens[i] more; a negative number ends it.
 *
 * Rows that end push their blocks on the free list, rows ascending, their blocks
 * in order.  Then rows are served in order: a row gets all it asks for or
 * nothing.  It gets it if the blocks asked for by it and all rows before it do
 * not exceed those free (a row that needs no new block passes), and the tokens
 * asked for by it and all rows before it do not exceed max_tokens.  A row that
 * asks for more than its table row can hold gets nothing and asks for nothing.
 * New blocks come from the top of the free list, one after another.
 *
 * The outputs of rows that end: granted 0, lens_out 0; their table entries stay.
 * lens_out may be lens and n_free_out may be n_free (a step in place); otherwise
 * inputs and outputs must not overlap.  The same inputs give the same outputs. */
typedef struct {
    int32_t n_rows;              /* 0..max_rows */
    int32_t table_width;         /* blocks of a table row, >= 1; table_width * block_size < 2^31 */
    int32_t max_tokens;          /* entries of the maps, >= 1 */
    int32_t prefix_len;          /* tokens before every row's own, >= 0: added to positions */
    const int32_t *lens;         /* [n_rows] own tokens held */
    const int32_t *new_tokens;   /* [n_rows] */
    int32_t *table;              /* [n_rows][table_width], entries of new blocks are written */
    int32_t *free_list;          /* [n_blocks], the first n_free are free */
    const int32_t *n_free;       /* [1] */
    int32_t *lens_out;           /* [n_rows] */
    int32_t *n_free_out;         /* [1] */
    int32_t *granted;            /* [n_rows] tokens granted */
    int32_t *starts;             /* [n_rows + 1] first entry of each row in the maps, and their total */
    int64_t *slots;              /* [max_tokens] slot of each new token, -1 beyond the total */
    int32_t *positions;          /* [max_tokens] prefix_len + place among the own tokens, 0 beyond */
    int32_t *rows;               /* [max_tokens] its row, -1 beyond */
    int32_t *visible;            /* [max_tokens] own tokens that it attends to, itself among them, 0 beyond */
} isjl_kv_assign_args;

/* For each token: q, k and v heads lie one after another in a row of qkv.  q and
 * k heads are normed, y = x / sqrt(mean(x^2) + eps) * weight (a NULL weight: not
 * normed), and the first rot of their head_dim values are rotated by the angles
 * of the token's position: pairs (a, b) become (a cos - b sin, b cos + a sin),
 * where a pair is values j and j + rot / 2, or 2 j and 2 j + 1 with
 * interleaved.  q goes to q_out, k and v to their slot.  A token with a
 * negative slot is padding: its q_out is 0 and nothing else is written.  Two
 * tokens must not have the same slot.  q_out may be qkv itself (its stride then
 * qkv's). */
typedef struct {
    int32_t n_tokens;            /* >= 0 */
    int32_t n_positions;         /* rows of rope */
    int32_t rot;                 /* 0 or a multiple of 16, at most head_dim */
    int32_t interleaved;         /* 0 or 1 */
    float eps;                   /* >= 0 */
    const void *qkv;             /* [n_tokens][n_q_heads + 2 n_kv_heads][head_dim] */
    int64_t qkv_stride;          /* elements between tokens, a multiple of 8 */
    void *q_out;                 /* [n_tokens][n_q_heads][head_dim] */
    int64_t q_out_stride;        /* elements between tokens, a multiple of 8 */
    const void *q_weight;        /* [head_dim] of the cache's type, or NULL */
    const void *k_weight;
    const float *rope;           /* [n_positions][rot]: rot / 2 cosines, then rot / 2 sines */
    const int32_t *positions;    /* [n_tokens], 0..n_positions - 1 where the slot is not negative */
    const int64_t *slots;        /* [n_tokens] */
} isjl_kv_append_args;

/* For query t with request i = rows[t] and x = lens[t] visible own tokens: its
 * tokens are the prefix's P = n_prefix_blocks * block_size, then the x own ones;
 * the query is the last of them.  Of the P + x it sees the last `window` (all if
 * window is 0) and the first `sinks`.  With s = scale * q . k over those,
 * out = sum exp(s) v / sum exp(s) and lse = log(sum exp(s)).  A query with
 * lens[t] <= 0 or rows[t] < 0 sees nothing: out 0, lse -infinity. */
typedef struct {
    int32_t n;                   /* queries, 0..max_rows */
    int32_t n_table_rows;
    int32_t table_width;         /* table_width * block_size + prefix <= 2^31 - 256, and n times that < 2^36 */
    int32_t n_prefix_blocks;     /* >= 0 */
    int32_t window;              /* >= 0 */
    int32_t sinks;               /* >= 0, used with a window */
    float scale;                 /* > 0, finite */
    const void *q;               /* [n][n_q_heads][head_dim], 16-byte aligned */
    int64_t q_stride[2];         /* elements between queries and between heads, multiples of 8 */
    void *out;
    int64_t out_stride[2];
    float *lse;                  /* [n][n_q_heads] or NULL */
    const int32_t *lens;         /* [n] */
    const int32_t *rows;         /* [n], or NULL: query t is request t's */
    const int32_t *table;        /* [n_table_rows][table_width] */
    const int32_t *prefix;       /* [n_prefix_blocks], NULL if there are none */
} isjl_kv_attend_args;

typedef struct isjl_kv isjl_kv;

/* Create a handle for one cache and head shape on the current CUDA device, with
 * the workspace of its calls (about 80 MB of device memory, and where a prefix can
 * be done apart, n_q_heads / n_kv_heads <= 128 and head_dim <= 128, 20 MB and three
 * times max_rows * n_q_heads * head_dim * 4 bytes more).  Errors: INVALID_ARG (null pointer, a value outside
 * the ranges above), OOM, CUDA.  On error *out is NULL. */
isjl_status isjl_kv_create(const isjl_kv_config *cfg, isjl_kv **out);

/* Free the workspace.  Synchronizes the device first.  NULL is ignored. */
void isjl_kv_destroy(isjl_kv *kv);

/* The three parts of a step.  Errors: INVALID_ARG (null pointers, values outside
 * the ranges above, misaligned pointers or strides), CUDA (launch failure).
 * The cache argument's memory must hold n_blocks blocks. */
isjl_status isjl_kv_assign(isjl_kv *kv, const isjl_kv_assign_args *args, void *stream);
isjl_status isjl_kv_append(isjl_kv *kv, const isjl_kv_append_args *args, const isjl_kv_cache *cache, void *stream);
isjl_status isjl_kv_attend(isjl_kv *kv, const isjl_kv_attend_args *args, const isjl_kv_cache *cache, void *stream);

/* Wait for the device's work (calls may have been replayed from graphs on any
 * stream); INVALID_ARG if any call since the last report met an invalid value on
 * the device (see above), INTERNAL if a kernel gave up a wait (a library bug: the
 * call's outputs are not valid), else OK.  Resets the report.  CUDA on a failed
 * sync.  Not inside a capture. */
isjl_status isjl_kv_status(isjl_kv *kv);

#ifdef __cplusplus
}
#endif

#endif /* ISJL_KV_H */
