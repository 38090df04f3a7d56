/*
 * us_kv.h - an 8-bit key/value cache and the attention over it, for MI355X (gfx950).
 *
 * The projections of a decoder layer (us.h) end in FP32 after the dequant
 * epilogue; these calls take them from there to the attention's output: new
 * keys and values are quantised into a paged cache, queries attend over it,
 * and a sequence's cache can be cut to its recent and most attended tokens.
 * Attention and caches are not part of the paper.
 *
 * Around the cache: queries and keys are normed and rotated by their positions
 * on the way there (us_kv_rotate); sequences continue others without copying what
 * they have in common (us_kv_fork), which attention then reads once for all of
 * them (us_kv_attend_shared); and a long cache is attended to in the blocks alone
 * whose keys can matter to a query (us_kv_summarise, us_kv_choose,
 * us_kv_attend_chosen).
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
#define US_KV_AXES_MAX 4       /* position axes of a rotation                 */
#define US_KV_CHOSEN_MAX (1 << 16) /* most blocks that a query chooses        */
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

/* How us_kv_rotate turns a row. */
typedef struct {
    const float *freq;         /* device, axes x pairs, contiguous              */
    int32_t pairs;             /* 0 .. head_dim / 2; 0: no rotation             */
    int32_t axes;              /* 1 .. US_KV_AXES_MAX                           */
    const int32_t *positions;  /* device, axes x positions_stride: of every row */
    int64_t positions_stride;  /* >= tokens                                     */
    int32_t offset;            /* added to every position (lengths are the positions
                                  of the newest tokens with an offset of -1)    */
    int32_t adjacent;          /* pair i is values (2 i, 2 i + 1), not (i, pairs + i) */
    int32_t norm;              /* 1: rows are normed first                      */
    float eps;                 /* with norm: > 0                                */
    const float *q_weight, *k_weight; /* with norm: device, head_dim, or NULL (ones) */
} us_kv_rotation;

/*
 * us_kv_rotate - norms of query and key heads and their rotation, in one pass.
 * A row x (a token's head) becomes, where `norm`,
 *   n = x w / sqrt(mean(x^2) + eps),
 * then pair i of its first 2 pairs values (n1, n2) becomes
 *   (n1 cos a_i - n2 sin a_i, n2 cos a_i + n1 sin a_i),
 *   a_i = sum over the axes of (positions[axis, row] + offset) freq[axis, i],
 * and the rest stays. (An axis that does not turn a pair has frequency 0 there.)
 * Angles are taken in 64 bits, the rest in float32, rounded once. q_out may be q
 * and k_out may be k, with the same strides (others, US_ERR_ARG); otherwise they
 * overlap nothing, and no rows of an output share memory (US_ERR_ARG): a head that
 * is there once for several is turned into an output of its own. All
 * rows have one type and number. k = k_out = NULL with k_heads = 0: queries alone.
 * US_ERR_SHAPE for more than 2^23 times as many rows as a workgroup takes together
 * (one, at least).
 */
us_status us_kv_rotate(int32_t q_heads, int32_t k_heads, int32_t head_dim, const us_rows *q, const us_rows *q_out,
                       const us_rows *k, const us_rows *k_out, const us_kv_rotation *how, void *stream);

/* The sequences that a fork makes; none of it overlaps what the call reads (old
 * and new tables that do, US_ERR_ARG; in one tensor, rows of one stride beside
 * each other). */
typedef struct {
    int32_t *blocks;        /* device, batch x stride                           */
    int64_t stride;
    int32_t width;          /* >= that of the old table, to US_KV_WIDTH_MAX     */
    int32_t batch;          /* 1 .. 65535                                       */
    int32_t *lens;          /* device, batch                                    */
} us_kv_forked;

/*
 * us_kv_fork - sequences that continue others, in tables of their own. New
 * sequence b has the tokens of the old one parents[b] (NULL: b; a number outside
 * the old ones: none) and blocks for room[b] more (NULL or below 0: none), as far
 * as the table is wide. refs[i] is how often the tables name block i; 0 is a free
 * block. Full blocks are shared by all children of a sequence. The block that a
 * sequence's next token goes to, and those behind it that its room reaches, stay
 * with its first child (the lowest b) if refs is 1; any other child is given a
 * block for each of them, a copy of the started one. Blocks that are given are the free ones of
 * lowest number, in the order of sequences and of their tables. Then the old
 * tables count for nothing any more, over their whole width: entries without a
 * block have to be outside [0, n_blocks). So a call frees what no child
 * continues, and gives a growing sequence its next block.
 * Where there are too few free blocks, missing (device, one number) is how many
 * are lacking, the new sequences are empty, and the old tables, refs and blocks
 * stay as they are and count on; else missing is 0.
 * A started block that is not there stays so. Only the blocks of seqs count:
 * its starts and max_new are not looked at.
 * ws: us_kv_fork_workspace_size bytes, 16-byte aligned, zero-filled before its
 * first use; not one that other calls use, nor calls that may overlap.
 * A call changes the tables and references of one pool: layers that have pools of
 * their own have tables, references and a call each.
 * US_ERR_SHAPE for more than 32767 heads.
 */
us_status us_kv_fork_workspace_size(const us_kv_cache *cache, int32_t batch, int32_t to_batch, size_t *bytes);
us_status us_kv_fork(const us_kv_cache *cache, int32_t *refs, const us_kv_seqs *seqs, const int32_t *parents,
                     const int32_t *room, const us_kv_forked *to, int32_t *missing, void *ws, size_t ws_bytes, void *stream);

/* Groups of sequences that have their first blocks in common: group g is
 * sequences starts[g] .. starts[g + 1] - 1, which have shared[g] blocks in
 * common. Sequences of no group have none. */
typedef struct {
    const int32_t *starts;  /* device, groups + 1, ascending                    */
    const int32_t *shared;  /* device, groups                                   */
    int32_t groups;         /* 1 .. 65535                                       */
    int32_t max_group;      /* no group has more sequences; 1 .. 65535          */
    int32_t max_shared;     /* nor more blocks in common; 0 = the table's width */
} us_kv_groups;

/*
 * us_kv_attend_shared - us_kv_attend for sequences with their first blocks in
 * common, which are read once for a group: those of its first sequence. (Where
 * another sequence's table differs there, its own blocks are not looked at.)
 * Queries see what us_kv_attend shows them, also if a sequence is shorter than
 * the common blocks, and results are off by as much. Sequences past max_group
 * in a group count as sequences of none. Where the sequences' token rows are not in
 * order, or one of them has more than max_new, rows of its group may miss common
 * keys. What pays depends on the sizes. With 32 heads over 8 of 128 a call takes less
 * than us_kv_attend on 16384 common tokens from 2 sequences on (1.2 times as fast; 2.7
 * with 64); on 4096 it does with 8 (1.2) and from 32 on, not with 4 or 16; on 1024 it
 * is 0.8 to 1.1 times as fast. It takes longer with one cache head, and for
 * sequences with whole prompts of their own. max_group and max_shared bound the
 * workspace and choose the kernel: as low as they are known. opts->window has to be 0
 * and opts->weights NULL. ws: us_kv_attend_shared_workspace_size bytes, as
 * us_kv_attend's, and one workspace serves both in turn. US_ERR_SHAPE as
 * us_kv_attend, for groups as for sequences (for more than 2^25 query rows of a
 * group and cache head), for more than 2^25 rows of a sequence and all heads, and
 * for more than 2^22 workgroups over the common keys or the others.
 */
us_status us_kv_attend_shared_workspace_size(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads,
                                             int32_t tokens, const us_kv_groups *groups, const us_kv_attend_opts *opts,
                                             size_t *bytes);
us_status us_kv_attend_shared(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads, const us_rows *q,
                              const us_rows *out, const us_kv_groups *groups, const us_kv_attend_opts *opts, void *ws,
                              size_t ws_bytes, void *stream);

/*
 * us_kv_summarise - the extremes of keys, for us_kv_choose. For every block that
 * holds some of the sequences' last tokens (those of starts and max_new),
 * summary (n_blocks x heads x 2 x us_kv_row(head_dim) bytes, 16-byte aligned)
 * gets the smallest byte of each value over the sequence's tokens in the block,
 * then the largest. Called after the append of these tokens, also because that
 * may change a block's scale and with it older codes; after us_kv_evict for all
 * tokens that are left. us_kv_fork copies no summary: a started block that it
 * copies has one after the next append to it, or a call for its tokens.
 */
us_status us_kv_summarise(const us_kv_cache *cache, const us_kv_seqs *seqs, uint8_t *summary, void *stream);

typedef struct {
    float *scores;          /* device, tokens x heads x scores_stride           */
    int64_t scores_stride;  /* >= the blocks of max_len tokens                  */
    int32_t *chosen;        /* device, tokens x heads x top                     */
    int32_t top;            /* 1 .. US_KV_CHOSEN_MAX                            */
    int32_t sinks, recent;  /* blocks taken in any case; together at most top   */
    int32_t max_len;        /* no sequence is longer; 0 = width * US_KV_BLOCK   */
} us_kv_choice;

/*
 * us_kv_choose - for every query row and cache head, the blocks of its sequence
 * whose keys can have the largest score. With lo and hi the codes of a block's
 * summary and s its keys' scale, its score is
 *   s max over the query heads of sum_d max(q_d, 0) hi_d + min(q_d, 0) lo_d,
 * no less than any q . k_j of it: exact for q held to 2^-30 of its largest
 * value, rounded once to float32. A query head with an infinity or a NaN does
 * not count; -infinity if none is left.
 * Row i of a sequence's n is at position p = lens - n + i and looks at the
 * blocks up to that of p. chosen gets, ascending, then -1, `top` of them: the
 * first `sinks` and the last `recent` ones, then those of largest score (equal
 * scores: the earlier one; a NaN counts as the smallest). Blocks that are not
 * there are not chosen. scores gets the scores of the blocks that a row looks
 * at (-infinity for one that is not there). Rows that are none of the sequences'
 * are left as they were. ws: us_kv_choose_workspace_size bytes, zero-filled
 * before its first use and left so; not one that other calls use.
 * US_ERR_SHAPE for more than 65535 rows.
 */
us_status us_kv_choose_workspace_size(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t tokens, int32_t top,
                                      size_t *bytes);
us_status us_kv_choose(const us_kv_cache *cache, const us_kv_seqs *seqs, const uint8_t *summary, int32_t q_heads,
                       const us_rows *q, const us_kv_choice *choice, void *ws, size_t ws_bytes, void *stream);

/*
 * us_kv_attend_chosen - us_kv_attend (causal) over the chosen blocks alone:
 * row t and head h of cache head k sees the keys up to its position in blocks
 * chosen[t, k, :] (tokens x heads x top). Numbers outside the sequence's blocks
 * up to that position count for nothing, a number that is there twice counts
 * twice. Rows without any key get zeros. For single tokens and a few drafted
 * ones: a row's blocks are read for it alone. With the summaries and the choice it
 * takes less than us_kv_attend from about 64 K tokens of one sequence on, or 8 K of
 * 16 (32 heads over 8 of 128, 48 blocks). opts: causal, without window and
 * weights. ws: us_kv_attend_chosen_workspace_size bytes, as us_kv_attend's, and
 * one workspace serves both in turn. US_ERR_SHAPE for more than 65535 rows.
 */
us_status us_kv_attend_chosen_workspace_size(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads,
                                             int32_t tokens, int32_t top, size_t *bytes);
us_status us_kv_attend_chosen(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads, const us_rows *q,
                              const us_rows *out, const int32_t *chosen, int32_t top, const us_kv_attend_opts *opts, void *ws,
                              size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* UNIONSPARSE_US_KV_H */
