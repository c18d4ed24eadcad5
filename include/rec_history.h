/*
 * rec_history.h - user histories: a compressed cache of keys and values, and
 * attention over it, on one MI355X (gfx950).
 *
 * Models that weigh a user's past events (the attention rows of Table I) turn
 * each event into a key and a value per head and let queries - the next event, or
 * candidate items - attend to them.  A server keeps those between requests:
 *
 *   rec_rotate_heads()     its queries and keys are normalised and rotated by position
 *   rec_window_attend()    a whole new history attends to itself
 *   rec_history_write()    its keys and values enter the cache, 4 or 8 bits a number
 *   rec_history_attend()   later queries attend to what the cache holds
 *   rec_history_summarise(), _select(), _attend_selected()
 *                          or, of a long history, to the pages that score highest only
 *   rec_history_attend_shared()
 *                          or to what many histories begin with and each one's own
 *   rec_history_read()     stored keys and values are read back
 *
 * What a query sees.  The query at position p (counted from 0 in its history) sees
 * the key at position j iff
 *
 *   0 <= j <= p   and   (window == 0  or  p - j < window  or  j < sinks)
 *
 *   out = sum_j w_j v_j,   w = softmax over the seen j of  scale * <q, k_j>
 *
 * A query that sees nothing gets zeros.  A key or value that it does not see has no
 * part in its result, whatever it holds, NaN and infinity included.
 *
 * The cache.  Elements of 32 neighbouring columns (a block) of one token and head
 * share a scale 2^e, stored as the byte e + 127.
 *   REC_MX4   elements E2M1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives
 *   REC_MX8   elements E4M3: largest 448, smallest 2^-9
 * e is the smallest that keeps every element of the block within half a step of the
 * largest element's neighbours: floor(log2 amax) - 2 (REC_MX8: - 8), one more where
 * amax is over 1.75 (1.8125) times its power of two; at least -110 and at most 125
 * (119), so that whatever is read back is a finite fp32.  Elements are rounded to
 * nearest, ties to even, and saturate.  A block with a NaN or an infinity has the
 * byte 255, reads back as NaN and is reported.  Nothing else is written; what a query
 * gets from a place that was never written, where it sees one, may be anything.
 *
 * Pages: [num_pages][kv_heads][page_tokens / 16] groups.  A group holds 16 tokens of
 * one head, D = head_dim:
 *   REC_MX4   K codes [16][D/2]    element 2 c in the low half of byte c, 2 c + 1 in the high
 *             V codes [D/2][16]    row 16 i + c: element 32 i + c low, 32 i + c + 16 high
 *   REC_MX8   K codes [16][D],  V codes [D/2][16][2] (the same two elements a row)
 *   then      K scales [16][D/32],  V scales [D/32][16]
 * Values lie along the tokens because that is the axis their product sums over.
 *
 * Conventions are those of rec.h: dev_* is device memory of the caller, nothing is
 * allocated, calls only enqueue kernels on `stream` (so they can be captured), and
 * host-checkable faults return at once with nothing enqueued.  Faults only the
 * device can see never stop a call, touch nothing outside the buffers, and go into
 * the record dev_fault where there is one.  Arrays of 32-bit and 64-bit words lie on 4
 * and 8 bytes (REC_ERR_ARG).
 */
#ifndef REC_HISTORY_H
#define REC_HISTORY_H

#include <stddef.h>
#include <stdint.h>
#include "rec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A type of the calls below beside rec_dtype's two. */
enum { REC_BF16 = 2 };

enum { REC_MX4 = 0, REC_MX8 = 1 };

/* Words of a fault record: smallest positions, all ones where there is no fault.
 * The caller sets all bytes to 255 once (or calls rec_history_check(), which does);
 * calls that find faults only lower the words. */
enum {
    REC_FAULT_LENGTH = 0,  /* history with a negative or too large length, or bad offsets     */
    REC_FAULT_SLOT = 1,    /* position in dev_slots of a slot outside the cache, or in dev_chosen of a page
                              that the history does not have                                  */
    REC_FAULT_PAGE = 2,    /* history * table_width + column (or position in dev_which) of a page outside
                              the cache                                                       */
    REC_FAULT_VALUE = 3,   /* position in dev_slots of a row with a NaN or an infinity         */
    REC_FAULT_WORDS = 4
};

/*
 * A cache.  The caller owns the pages; nothing in them needs setting beforehand.
 *   dev_pages     16-byte aligned, rec_history_bytes()
 *   num_pages     >= 1; num_pages * page_tokens < 2^40
 *   page_tokens   16, 32, 64, 128 or 256
 *   kv_heads      1 .. 1024
 *   head_dim      32, 64 or 128
 *   format        REC_MX4 or REC_MX8
 *   dev_fault     uint64 [REC_FAULT_WORDS], may be null
 */
typedef struct {
    void *dev_pages;
    int64_t num_pages;
    int32_t page_tokens;
    int32_t kv_heads;
    int32_t head_dim;
    int32_t format;
    uint64_t *dev_fault;
} rec_history;

/* Bytes of the pages; 0 where the shape is not allowed (dev_pages is not looked at). */
REC_API size_t rec_history_bytes(const rec_history *h);

/* Rows [tokens][heads][head_dim] of a caller's tensor: strides in elements, both
 * multiples of 16 bytes, and the elements of a row adjacent. */
typedef struct {
    const void *dev;
    int64_t token_stride;
    int64_t head_stride;
} rec_rows;

/*
 * Quantises `tokens` keys and values into the cache, row i into slot dev_slots[i] =
 * page * page_tokens + place in the page.  Slot -1: the row is left out (padding).
 *   k, v     [tokens][kv_heads][head_dim] of dtype (REC_F32, REC_F16, REC_BF16)
 * Device faults: REC_FAULT_SLOT (the row is left out), REC_FAULT_VALUE.
 * A slot that is named twice in one call holds one of its rows or a mixture.
 * REC_ERR_ARG: null, misaligned, bad enum, tokens < 0; REC_ERR_SHAPE: a shape that
 * rec_history_bytes() refuses; REC_ERR_OVERFLOW: 2^30 tokens, or
 * ceil(tokens / 16) * kv_heads > 2^26 - 4 (more threads than a launch can have).
 */
REC_API rec_status rec_history_write(const rec_history *h, const rec_rows *k, const rec_rows *v,
                                     int32_t dtype, const int64_t *dev_slots, int64_t tokens, void *stream);

/* Reads the rows of dev_slots back: dev_k and dev_v are [tokens][kv_heads][head_dim]
 * of dtype, contiguous, 16-byte aligned.  Slot -1, and one outside the cache (which is
 * reported), give zeros.  Values are exact in fp32 and bf16; in fp16 they are rounded, to
 * infinity beyond its range.  Errors as above. */
REC_API rec_status rec_history_read(const rec_history *h, const int64_t *dev_slots, int64_t tokens,
                                    int32_t dtype, void *dev_k, void *dev_v, void *stream);

/*
 * Queries over cached histories.
 *   dev_q          [batch][queries][heads][head_dim] of dtype; strides in elements,
 *                  multiples of 16 bytes
 *   dev_out        the same shape, contiguous, 16-byte aligned
 *   dtype          REC_F16 or REC_BF16
 *   heads          a multiple of kv_heads; head n reads kv head n / (heads / kv_heads)
 *   dev_pages_of   int32 [batch][table_width], rows table_stride apart: the pages of each
 *                  history in order.  Entries behind its last token are not read.
 *   dev_lengths    int32 [batch]: tokens of each history, those of the queries included
 *   candidates     0: query i of history b is its token dev_lengths[b] - queries + i.
 *                  1: every query stands at the last token and sees what that sees.
 *   window, sinks  see above; 0 each for none
 * Device faults: REC_FAULT_LENGTH (a negative length counts as 0, one over
 * table_width * page_tokens as that), REC_FAULT_PAGE (its tokens are not seen).
 */
typedef struct {
    const void *dev_q;
    void *dev_out;
    int64_t batch_stride, query_stride, head_stride;
    int32_t dtype;
    int32_t batch, queries, heads;
    const int32_t *dev_pages_of;
    int64_t table_stride;
    int32_t table_width;
    const int32_t *dev_lengths;
    float scale;
    int32_t window, sinks;
    int32_t candidates;
} rec_query;

/* Bytes of workspace of rec_history_attend() with this query (long histories are
 * divided among workgroups, and their parts meet there): 0 where it needs none or the
 * query is refused.  Only shapes matter, not pointers. */
REC_API size_t rec_history_attend_workspace_bytes(const rec_history *h, const rec_query *q);

/* Enqueues the attention.  dev_workspace: 16-byte aligned, as many bytes as said above,
 * free for other use once the call's work is done; what it holds before does not matter.
 * REC_ERR_ARG: null, misaligned, bad enum, negative counts, a workspace too small;
 * REC_ERR_SHAPE: heads no multiple of kv_heads, or a shape that rec_history_bytes()
 * refuses; REC_ERR_OVERFLOW: batch * queries * heads >= 2^31, or table_width * page_tokens
 * > 2^31 - 1024, or more threads than a launch can have (2^32). */
REC_API rec_status rec_history_attend(const rec_history *h, const rec_query *q, void *dev_workspace,
                                      size_t workspace_bytes, void *stream);

/*
 * Chosen pages.  Of a long history a query need not see all: each page has a mean key, and each query attends,
 * for each kv head, to the pages whose means score highest with it.
 *
 * rec_history_summarise() writes the mean keys of `pages` pages, bf16 [kv_heads][head_dim] each, into
 * dev_means [num_pages][kv_heads][head_dim] (16-byte aligned): those of a page dev_which[i] (int32; -1: left out) at that
 * page.  All page_tokens places count, so a page has its turn once it is full; NaN where a key is NaN.  A page that is
 * named twice is written twice, alike.
 * Device faults: REC_FAULT_PAGE (position in dev_which; nothing is written for it).
 * REC_ERR_ARG: null, misaligned, pages < 0; REC_ERR_SHAPE as above; REC_ERR_OVERFLOW: more threads than a launch can have.
 */
REC_API rec_status rec_history_summarise(const rec_history *h, const int32_t *dev_which, int32_t pages, void *dev_means, void *stream);

/*
 * rec_history_select() chooses `count` pages for each query and kv head, of those up to the one that the query
 * stands in: the first `first` of the history and the last `last` always (of which the query's own is one), and
 * between them those with the highest scores
 *
 *   score = max over the heads n of the kv head of  <q_n, mean>
 *
 * in 64 bits; of equal ones the earlier.  A product that is NaN counts for nothing; a page outside the cache, or
 * without a product that counts, scores -infinity.  dev_chosen [batch][queries][kv_heads][count], int32, gets the pages'
 * numbers in their history, ascending, -1 behind them where there are fewer.  The means of the last `last` pages are not
 * looked at, so a page that is not full yet needs none.
 *   q              as for rec_history_attend(); dev_out and scale are not looked at, window and sinks are 0
 *   count          >= first + last, first >= 0, last >= 1
 * Device faults: REC_FAULT_LENGTH, REC_FAULT_PAGE as there.
 * REC_ERR_ARG: null, misaligned, bad counts, a workspace too small; REC_ERR_SHAPE, REC_ERR_OVERFLOW as there, and
 * REC_ERR_OVERFLOW: count > 2^31 - 1024.
 */
REC_API size_t rec_history_select_workspace_bytes(const rec_history *h, const rec_query *q, int32_t count);
REC_API rec_status rec_history_select(const rec_history *h, const rec_query *q, const void *dev_means, int32_t count, int32_t first,
                                      int32_t last, int32_t *dev_chosen, void *dev_workspace, size_t workspace_bytes, void *stream);

/*
 * rec_history_attend_selected(): rec_history_attend() where each query and kv head sees, of what its position allows, only
 * the pages in dev_chosen, int32 [batch][queries][kv_heads][count], in any order.  An entry of -1 is none; a page that
 * is named twice counts twice.  window and sinks are 0.
 * Device faults: REC_FAULT_LENGTH, REC_FAULT_PAGE as there, and REC_FAULT_SLOT: position in dev_chosen of an entry that is
 * neither -1 nor under table_width (it is not seen).  Errors as there; REC_ERR_ARG: count < 1; REC_ERR_OVERFLOW: count * page_tokens
 * > 2^31 - 1024.
 */
REC_API size_t rec_history_attend_selected_workspace_bytes(const rec_history *h, const rec_query *q, int32_t count);
REC_API rec_status rec_history_attend_selected(const rec_history *h, const rec_query *q, const int32_t *dev_chosen, int32_t count,
                                               void *dev_workspace, size_t workspace_bytes, void *stream);

/*
 * Histories that begin alike.  rec_history_attend_shared(): rec_history_attend() where the histories of a batch all begin with the
 * same tokens, *dev_prefix_length (int32, on the device) of them in the pages dev_prefix_pages, int32 [prefix_width]; q describes what
 * each has behind them, its pages, its length and its queries.  A query sees the whole prefix and, of its own history, what it
 * would see by itself; one that stands before its own history's first token sees nothing, but for candidates, which then see
 * the prefix.  Where there is much to read, the prefix is read once for
 * many queries.  window and sinks are 0.
 * Device faults: as there; of the prefix REC_FAULT_LENGTH with position batch, REC_FAULT_PAGE with position
 * batch * table_width + column.  Errors as there; REC_ERR_ARG: prefix_width < 0, dev_prefix_pages (where prefix_width > 0) or
 * dev_prefix_length null or misaligned; REC_ERR_OVERFLOW: prefix_width * page_tokens > 2^31 - 1024.
 */
REC_API size_t rec_history_attend_shared_workspace_bytes(const rec_history *h, const rec_query *q, int32_t prefix_width);
REC_API rec_status rec_history_attend_shared(const rec_history *h, const rec_query *q, const int32_t *dev_prefix_pages, int32_t prefix_width,
                                             const int32_t *dev_prefix_length, void *dev_workspace, size_t workspace_bytes, void *stream);

/*
 * Whole histories attend to themselves, without a cache.
 *   q             [tokens][heads][head_dim], k and v [tokens][kv_heads][head_dim], of
 *                 dtype (REC_F16 or REC_BF16): histories one after the other
 *   dev_out       [tokens][heads][head_dim], contiguous, 16-byte aligned
 *   dev_offsets   int32 [batch + 1], non-decreasing from 0 to tokens: history b is rows
 *                 dev_offsets[b] .. dev_offsets[b + 1] - 1, the first at position 0
 *   head_dim      32, 64 or 128; heads a multiple of kv_heads
 *   dev_fault     as in rec_history; may be null
 * Device faults: REC_FAULT_LENGTH (offsets that decrease, or do not run from 0 to tokens,
 * are brought into that range; rows of no history are not written).
 * Rows near a value that is not finite are computed a second time, several times as slowly.
 * REC_ERR_ARG, REC_ERR_SHAPE as above; REC_ERR_OVERFLOW: tokens * heads >= 2^31, more
 * than 2^24 workgroups (tokens * heads / 128 + batch * kv_heads), a token stride of k or v that is
 * negative or >= 2^23 elements.
 */
typedef struct {
    rec_rows q, k, v;
    void *dev_out;
    int32_t dtype;
    int32_t batch;
    int64_t tokens;
    int32_t heads, kv_heads, head_dim;
    const int32_t *dev_offsets;
    float scale;
    int32_t window, sinks;
    uint64_t *dev_fault;
} rec_window;

REC_API rec_status rec_window_attend(const rec_window *w, void *stream);

/*
 * Queries and keys of events, normalised per head and rotated by their position, in one pass.
 *
 *   y = x / sqrt(mean(x^2) + eps) * w         a row of head_dim columns; y = x without a weight w
 *   (y_a, y_b) -> (y_a cos t - y_b sin t,  y_a sin t + y_b cos t)     t = position * dev_frequencies[i]
 *
 * for the pairs i = 0 .. pairs - 1 of the first 2 * pairs columns: (a, b) = (i, i + pairs), or, interleaved,
 * (2 i, 2 i + 1).  Columns behind those are not rotated; pairs = 0 rotates none.
 *
 *   q, k           [tokens][heads][head_dim], [tokens][kv_heads][head_dim] of dtype (REC_F32, REC_F16, REC_BF16);
 *                  one of heads and kv_heads may be 0, and its rows and weight null
 *   q_out, k_out   the same shapes and type, rows that do not overlap; they may be q and k themselves
 *                  (the same address and strides) and may not overlap them, or each other, otherwise.  Rows that lie between
 *                  another argument's have its token stride, or one row for all tokens (stride 0)
 *   head_dim       32, 64 or 128
 *   dev_positions  int32 or, wide = 1, int64 [tokens], of either sign
 *   dev_frequencies  double [pairs], radians a position; pairs a multiple of 8, at most head_dim / 2
 *   dev_q_weight, dev_k_weight   float [head_dim], 16-byte aligned, or null: those rows are not normalised
 *   eps            >= 0
 * Squares are summed in fp32, or in 64 bits where that would overflow or vanish; angles are worked out in 64 bits.
 * REC_ERR_ARG: null, misaligned, bad enum, negative counts or eps, rows of q_out or k_out that overlap each other or q and k;
 * REC_ERR_SHAPE: head_dim or pairs; REC_ERR_OVERFLOW: more than 2^20 heads, or more threads
 * than a launch can have (2^32; a wave has 4 to 32 rows).
 */
typedef struct {
    rec_rows q, k, q_out, k_out;
    int32_t dtype;
    int32_t heads, kv_heads, head_dim;
    int64_t tokens;
    const void *dev_positions;
    int32_t wide;
    int32_t pairs;
    const double *dev_frequencies;
    int32_t interleaved;
    float eps;
    const float *dev_q_weight, *dev_k_weight;
} rec_turn;

REC_API rec_status rec_rotate_heads(const rec_turn *t, void *stream);

/* Waits for `stream`, reads a fault record and clears what it read: faults that work on other
 * streams adds meanwhile stay for the next check.  REC_OK, REC_ERR_LENGTHS
 * (REC_FAULT_LENGTH), REC_ERR_INDEX_RANGE (REC_FAULT_SLOT or REC_FAULT_PAGE) or
 * REC_ERR_VALUE (REC_FAULT_VALUE), the first of these that applies, with its position
 * in *first_bad_pos (may be null; -1 without a fault) and its word in *word (may be null). */
REC_API rec_status rec_history_check(uint64_t *dev_fault, void *stream, int64_t *first_bad_pos, int32_t *word);

#ifdef __cplusplus
}
#endif
#endif /* REC_HISTORY_H */
