/*
 * us_kv.h - an 8-bit key/value cache and the attention over it, for MI355X (gfx950).
 *
 * The projections of a decoder layer (us.h) end in FP32 after the dequant
 * epilogue; these calls take them from there to the attention's output: new
 * keys and values are quantised into a paged cache, queries attend over it,
 * and a sequence's cache can be cut to its recent and most attended tokens.
 * Attention and caches are not part of the paper.
 *
 * Conventions are those of us.h: arguments are checked before any work, device
 * pointers belong to the caller, every call is asynchronous on its stream,
 * allocates nothing, never synchronises, and can be captured in a HIP graph.
 * Calls that touch the same blocks are ordered by their stream; on several
 * streams the caller orders them.
 *
 * The cache. A block holds US_KV_BLOCK tokens of one head: codes c in
 * [-127, 127], stored as bytes c + 128, and one float32 scale s for the keys
 * and one for the values of each (block, head); a value is c s. The pool has
 * n_blocks x heads such blocks of US_KV_BLOCK * us_kv_row(head_dim) bytes for
 * keys and as many for values. Within a block, with R = us_kv_row(head_dim):
 *   key   (token t, value d) is byte
 *         2048 (d / 32) + 1024 (t / 32) + 64 (t % 16) + 16 ((d / 8) % 4) + 8 ((t / 16) % 2) + d % 8
 *   value (token t, value d) is byte
 *         64 d + 16 ((t / 4) % 4) + 4 (t / 16) + t % 4
 * which is the order in which the matrix cores take them: 64 lanes with 16
 * bytes each read 1 KB without a gap. Bytes that no token was stored to may
 * hold anything. Scales are not negative.
 *
 * What the GPU reads from the caller's tables is bounded there: block numbers
 * outside [0, n_blocks) are blocks that are not there (nothing is stored to
 * them, they read as zero, no query sees them), lengths are cut to the table,
 * and token ranges to the arrays they index.
 */
#ifndef UNIONSPARSE_US_KV_H
#define UNIONSPARSE_US_KV_H

#include <stddef.h>
#include <stdint.h>

#include "us.h"

#ifdef __cplusplus
extern "C" {
#endif

#define US_KV_BLOCK 64         /* tokens of a block                           */
#define US_KV_HEAD_DIM_MAX 256 /* widest head                                 */
#define US_KV_WIDTH_MAX (1 << 22) /* most blocks of a sequence                */
#define US_KV_NEW_MAX (1 << 25)   /* most new tokens, or query rows of a cache
                                     head, of a sequence in one call          */

typedef enum { US_F32 = 0, US_BF16 = 1, US_F16 = 2 } us_dtype;

/* A pool of blocks. k and v 16-byte aligned; scales n_blocks x heads. */
typedef struct {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    int32_t n_blocks, heads, head_dim;
} us_kv_cache;

/*
 * The sequences of a call. Sequence b's token j is in block
 * blocks[b * stride + j / US_KV_BLOCK], and it has lens[b] tokens, those that
 * the call is about included. These are its last starts[b + 1] - starts[b]
 * tokens, at most max_new of them, in order rows starts[b] .. of the arrays
 * of tokens; starts = NULL is one token per sequence (row b; max_new = 1).
 */
typedef struct {
    const int32_t *blocks;  /* device, batch x stride                          */
    int64_t stride;         /* >= width                                        */
    int32_t width;          /* blocks of a sequence at most, to US_KV_WIDTH_MAX */
    int32_t batch;          /* 1 .. 65535                                      */
    const int32_t *lens;    /* device, batch                                   */
    const int32_t *starts;  /* device, batch + 1, or NULL                      */
    int32_t max_new;
} us_kv_seqs;

/* An array of token rows: value d of head h of row t is element
 * t * token_stride + h * head_stride + d. Rows from `tokens` on are not
 * touched. Any alignment that the type itself has will do. */
typedef struct {
    void *data;
    int64_t token_stride, head_stride; /* elements                            */
    int32_t tokens;
    int32_t dtype;                     /* us_dtype                            */
} us_rows;

/* Bytes of a head's key (or value) per token: head_dim rounded up to 64, 96,
 * 128, 192 or 256; 0 for a head_dim outside [1, US_KV_HEAD_DIM_MAX]. */
int32_t us_kv_row(int32_t head_dim);

/*
 * us_kv_append - quantise new tokens into the cache.
 * The scale of a block that the call stores to becomes
 *   s' = max(s, amax / 127)
 * with amax the largest magnitude of the block's new values and s its scale
 * where it holds earlier tokens of the sequence (else 0). New codes are
 * rint(x / s'), halves to even; where s' > s the earlier codes c become
 * rint(c (s / s')). Infinities and NaN do not count for amax; an infinity is
 * stored as +-127, a NaN as 0. All in float32; a block of zeros has scale 0.
 * A code is off by half a step when stored, and by half a step of the new scale
 * each time that the block's scale grows afterwards.
 * k, v: rows of heads x head_dim, of one type. A block that a call stores to
 * belongs to one of its sequences.
 */
us_status us_kv_append(const us_kv_cache *cache, const us_kv_seqs *seqs, const us_rows *k, const us_rows *v,
                       void *stream);

/*
 * us_kv_read - the inverse: the last tokens of every sequence as dense rows,
 * c s rounded once to the rows' type. Rows of positions that the sequence does
 * not have (more rows than tokens) become zero.
 */
us_status us_kv_read(const us_kv_cache *cache, const us_kv_seqs *seqs, const us_rows *k, const us_rows *v,
                     void *stream);

typedef struct {
    float scale;            /* of q k; 0 = 1 / sqrt(head_dim)                  */
    int32_t causal;         /* 1: a query sees the keys up to its own position;
                               0: all keys of its sequence (an encoder's states,
                               then lens counts those and not the queries)     */
    int32_t window;         /* 0, or (causal only) a query sees the last
                               `window` positions, its own included            */
    int32_t max_len;        /* no sequence is longer; 0 = width * US_KV_BLOCK  */
    float *weights;         /* NULL, or device, batch x heads x weights_stride:
                               weights[b, h, j] += the probabilities that the
                               queries of the call gave token j, summed over
                               the call's queries and the query heads of h     */
    int64_t weights_stride; /* >= max_len                                      */
} us_kv_attend_opts;

/*
 * us_kv_attend - softmax attention of the sequences' last tokens over the
 * cache: for query row t and head h of `q_heads` (a multiple of the cache's
 * heads; head h reads cache head h / (q_heads / heads)),
 *   out = sum_j p_j v_j,  p = softmax over the visible j of scale (q . k_j).
 * A query that sees no key gets zeros. Query i of a sequence's n is at
 * position lens - n + i. q and out have one type. Scores, their maximum, sums
 * and results are in float32. A probability meets the values as float16 where
 * the rows are bfloat16 or float16 (off by at most 2^-12 of itself, less than
 * their own rounding), as two float16 parts where they are float32 (2^-22); one
 * below 2^-27 (2^-16) of the row's largest, in calls of many rows both times
 * their blocks' value scales, keeps fewer bits. Sums are held with probabilities times
 * up to 2^15: values times keys have to stay below 2^113. A query with an
 * infinity or a NaN gives a NaN row, also in the weights of the keys it sees.
 * ws: us_kv_attend_workspace_size bytes, 16-byte aligned, zero-filled before
 * its first use and left so that any later call can use it again; calls that
 * may overlap need workspaces of their own. The size for a call without a
 * window (or without the causal mask) serves the same call with one. Calls of
 * few rows with weights keep their scores there: batch x q_heads x max_new x
 * max_len floats, without a limit up to 16 rows of a cache head, up to 64 MB past
 * that.
 * opts = NULL: causal, the rest 0. US_ERR_SHAPE also for more than 2^25 query
 * rows of a cache head (max_new x q_heads / heads), and for calls of many rows
 * if batch x heads x rows / 256 (128 for head_dim above 128) passes 2^22.
 */
us_status us_kv_attend_workspace_size(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads,
                                      int32_t tokens, const us_kv_attend_opts *opts, size_t *bytes);
us_status us_kv_attend(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads, const us_rows *q,
                       const us_rows *out, const us_kv_attend_opts *opts, void *ws, size_t ws_bytes, void *stream);

typedef struct {
    int32_t prompt;      /* 0: the kernel for few rows of a cache head, 1: for many */
    int32_t tile_rows;   /* rows of a workgroup                                     */
    int32_t split_keys;  /* parts that the longest sequence's keys may be cut into  */
    int32_t part_blocks; /* blocks of such a part                                   */
} us_kv_attend_route_info;

/*
 * us_kv_attend_route - what us_kv_attend launches for these sizes and this
 * type of rows on the current device (256 CUs when no device is visible).
 * Host only; for reporting and tests. Refusals as the workspace's size.
 */
us_status us_kv_attend_route(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads, int32_t tokens,
                             int32_t dtype, const us_kv_attend_opts *opts, us_kv_attend_route_info *out);

/* Where an eviction leaves what it keeps; none of it overlaps what the call reads. */
typedef struct {
    const int32_t *blocks;  /* device, batch x stride: blocks of the same pool,
                               none of them one of the sequences' own          */
    int64_t stride;
    int32_t width;          /* width * US_KV_BLOCK >= keep, or >= every length;
                               to US_KV_WIDTH_MAX                              */
    int32_t *lens;          /* device, batch: min(length, keep)                */
    float *weights;         /* device, batch x heads x weights_stride, or NULL:
                               of the kept tokens in order, then zeros for the
                               tokens that the blocks have room for            */
    int64_t weights_stride; /* >= min(keep, width * US_KV_BLOCK)               */
    int32_t *index;         /* device, batch x heads x keep: the kept positions,
                               ascending, then -1                              */
} us_kv_kept;

/*
 * us_kv_evict - keep at most `keep` tokens of every sequence, per head: its
 * last `recent` ones and, of the others, those of largest weight (equal
 * weights: the earlier token; a NaN counts as the smallest). The kept tokens
 * go, in order, to the blocks of `to`, with their weights. The scale of such a
 * block is the largest of the scales its tokens had, s', and their codes
 * become rint(c (s / s')). Afterwards the caller uses to's blocks and lengths.
 * weights: as us_kv_attend adds them up; 1 <= keep, 0 <= recent <= keep.
 * max_len: no sequence is longer; 0 = width * US_KV_BLOCK.
 */
us_status us_kv_evict(const us_kv_cache *cache, const us_kv_seqs *seqs, const float *weights, int64_t weights_stride,
                      int32_t max_len, int32_t keep, int32_t recent, const us_kv_kept *to, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* UNIONSPARSE_US_KV_H */
