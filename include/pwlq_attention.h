/*
 * pwlq_attention.h - what a transformer block has between its projections: a
 * paged cache of keys and values, in 16 bits or in 8-bit rows, new rows that
 * enter it with their position's rotation on the way, and attention over it for
 * single tokens, trees of drafted tokens and prompts.
 *
 * Conventions: those of pwlq.h (device pointers owned by the caller, work
 * enqueued on `stream`, nothing allocated, pwlq_last_error), and
 *   - A cache is `pages` pages of keys and as many of values, each
 *     [heads, page, D]: `page` rows, a power of two from 16 to 65536, of each
 *     of `heads` heads of D channels, D a multiple of 16 up to 256.  type is
 *     PWLQ_BF16, PWLQ_F16, or PWLQ_I8: codes with a binary32 step for each row
 *     of a head, [pages, heads, page], value = code * step, as pwlq_pack_rows
 *     (pwlq_block.h) defines codes and steps.  The arrays are 16-byte aligned.
 *   - A batch is S sequences.  Sequence s holds lengths[s] rows, those of this
 *     call included; its row `slot` is row slot % page of page
 *     table[s * table_stride + slot / page].  Lengths beyond table_pages * page
 *     (which is at most 2^30) count as that.  Entries that no row needs are not
 *     read.  Rows on a page outside [0, pages) do not exist: nothing is written
 *     there, they read as zeros, and attention does not see them.  Sequences may
 *     share pages that no row of the call is written to.
 *   - The T rows of a call are the last ones of their sequences: sequence s has
 *     rows starts[s] to starts[s+1] - 1 (starts: S+1 values in rising order,
 *     from 0 to at most T), row starts[s] + j at slot lengths[s] - n + j, n the
 *     sequence's rows.  starts NULL: T = S, one row for each.  Rows from
 *     starts[S] on belong to no sequence: nothing is done with them.  A row
 *     whose slot is negative is not in the cache: append skips it (its query is
 *     still written), read gives zeros, attention gives zeros.
 *   - Rows of heads are given as a pwlq_heads: `stride` elements from one row to
 *     the next, `head_stride` from one head to the next, channels next to each
 *     other, so columns of a projection's output can be passed as they stand.
 *     Outputs must not overlap inputs or each other.
 *   - All tensors of a call but the codes of a cache have one type, PWLQ_BF16
 *     or PWLQ_F16.  T and S are at most 2^20, heads of queries at most 1024 and
 *     a multiple of the cache's.
 */
#ifndef PWLQ_ATTENTION_H
#define PWLQ_ATTENTION_H

#include <stddef.h>
#include <stdint.h>

#include "pwlq_block.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    void *keys, *values;
    float *key_step, *value_step;    /* with PWLQ_I8, else NULL */
    int64_t pages;
    int heads, page, D, type;
} pwlq_cache;

typedef struct {
    int64_t S, T;
    const int32_t *table;
    int64_t table_stride, table_pages;
    const int32_t *lengths, *starts;
} pwlq_batch;

typedef struct {
    void *data;
    int64_t stride, head_stride;
    int type;
} pwlq_heads;

/*
 * New rows into the cache: k and v are [T, heads, D], q [T, q_heads, D] or left
 * out (data NULL, q_heads 0).  The first `rotated` channels of each head of q and
 * k turn by the row's position: for i < rotated/2, with angle positions[t] *
 * frequencies[i], formed in binary64,
 *     a' = a cos - b sin,  b' = b cos + a sin
 * (a, b) being channels (i, i + rotated/2), or (2i, 2i+1) where `interleaved`.
 * positions: T values, or NULL for each row's slot.  rotated: a multiple of 16
 * up to D, 0 for none (frequencies NULL).  The rotated queries go to q_out;
 * keys and values to the cache, rounded once, to its type.
 */
typedef struct {
    pwlq_cache cache;
    pwlq_batch batch;
    pwlq_heads q, k, v, q_out;
    int q_heads, rotated, interleaved;
    const int32_t *positions;
    const float *frequencies;
} pwlq_append_args;

int pwlq_append(const pwlq_append_args *args, void *stream);

/* The values of the call's rows in the cache, to k and v [T, heads, D] (either
 * may be left out). */
typedef struct {
    pwlq_cache cache;
    pwlq_batch batch;
    pwlq_heads k, v;
} pwlq_read_args;

int pwlq_read(const pwlq_read_args *args, void *stream);

/*
 * Attention of q [T, q_heads, D] over the cache; head h reads head
 * h / (q_heads / heads) of the cache.  For a row at `own` and a key at `slot`:
 *     s   = scale * (q . k)                            |scale| at most 2^60
 *     s   = cap * tanh(s / cap)                        unless cap is 0; 2^-60 to 2^60
 *     s   = s - slopes[h] * |own - slot|               where slopes are given
 *     out = sum_slot softmax(s)[slot] v[slot]          over the slots it sees
 * A row sees slot < lengths[s], if
 *     slot <= own and (window = 0 or own - slot < window),  or  slot < prefix[s]
 * or, where `tree` is given, slots before its sequence's rows of this call, and
 * row j' of those rows if bit j' % 64 of tree[t * tree_words + j' / 64] is set
 * (j' >= 64 * tree_words: not).  A tree goes without slopes, window and prefix.
 * Scores are formed in binary32: one beyond its range is infinite, and the softmax of a row that sees plus infinity is NaN.
 * What a row does not see does not touch it, infinities and NaN included.  A row
 * that sees nothing (or only scores of minus infinity) is zeros.  An infinite
 * value that it sees makes its output infinite, or NaN where the weight is next
 * to nothing.
 * Roundings: a weight is rounded to the elements' type for its product with the
 * values (with PWLQ_I8 and bfloat16 together with the value's step; with
 * binary16 the value is, which must be within its range), the output once.
 * With a prefix a window saves no time: keys between the two are gone through.
 * longest: the most rows of a sequence, as far as the caller knows (0: T); it
 * decides which kernel runs and nothing else.
 * Workspace: device, 256-byte aligned, pwlq_attend_workspace_bytes(args) bytes,
 * which read nothing that args points to.  Calls that may run at the
 * same time need workspaces of their own.
 */
typedef struct {
    pwlq_cache cache;
    pwlq_batch batch;
    pwlq_heads q, out;
    int q_heads;
    float scale, cap;
    const float *slopes;
    int64_t window;
    const int32_t *prefix;
    const uint64_t *tree;
    int64_t tree_words;
    int64_t longest;
} pwlq_attend_args;

size_t pwlq_attend_workspace_bytes(const pwlq_attend_args *args);
int pwlq_attend(const pwlq_attend_args *args, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PWLQ_ATTENTION_H */
