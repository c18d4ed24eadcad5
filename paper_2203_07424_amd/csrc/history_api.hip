// Host side of include/rec_history.h: checks, and nothing else.
#include <algorithm>
#include <utility>

#include "history.h"
#include "rec_probe.h"

namespace {

using rec::hist::Cache;

// Of a history: the kernels count a little past the last one in 32 bits.
constexpr int64_t MOST_TOKENS = (1ll << 31) - 1024;

// What a launch counts its threads in.
constexpr int64_t MOST_THREADS = (1ll << 32) - 1;

bool head_dim_fits(int d) { return d == 32 || d == 64 || d == 128; }

bool shape_fits(const rec_history *h)
{
    const int p = h->page_tokens;
    return h->num_pages >= 1 && p >= 16 && p <= 256 && (p & (p - 1)) == 0 && h->num_pages < (1ll << 40) / p &&
           h->kv_heads >= 1 && h->kv_heads <= 1024 && head_dim_fits(h->head_dim) &&
           (h->format == REC_MX4 || h->format == REC_MX8);
}

bool aligned(const void *p) { return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Words of `size` bytes, where there are any, on their own alignment.
bool words_fit(const void *p, unsigned size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) == 0; }

// Strides whose rows all start on 16 bytes.
bool stride_fits(int64_t stride, int size) { return stride * size % 16 == 0; }

Cache cache_of(const rec_history *h)
{
    Cache c;
    c.pages = static_cast<unsigned char *>(h->dev_pages);
    c.num_pages = h->num_pages;
    c.page_shift = __builtin_ctz((unsigned)h->page_tokens);
    c.kv_heads = h->kv_heads;
    c.fault = reinterpret_cast<unsigned long long *>(h->dev_fault);
    return c;
}

// What a call on the cache's rows needs; REC_OK if it can go on.
rec_status check_rows(const rec_history *h, int32_t dtype, const int64_t *dev_slots, int64_t tokens)
{
    if (!h) return REC_ERR_ARG;
    if (!shape_fits(h)) return REC_ERR_SHAPE;
    if (!aligned(h->dev_pages) || (dtype != REC_F32 && dtype != REC_F16 && dtype != REC_BF16) || tokens < 0) return REC_ERR_ARG;
    if (!words_fit(h->dev_fault, 8) || (tokens && (!dev_slots || !words_fit(dev_slots, 8)))) return REC_ERR_ARG;
    if (tokens >= 1ll << 30 || rec::hist::rows_threads(cache_of(h), tokens) > MOST_THREADS) return REC_ERR_OVERFLOW;
    return REC_OK;
}

// Shapes and counts of a query, whatever reads it.
rec_status check_counts(const rec_history *h, const rec_query *q)
{
    if (!h || !q) return REC_ERR_ARG;
    if (!shape_fits(h)) return REC_ERR_SHAPE;
    if ((q->dtype != REC_F16 && q->dtype != REC_BF16) || q->batch < 0 || q->queries < 0 || q->heads < 1 || q->table_width < 0 ||
        q->window < 0 || q->sinks < 0 || (q->candidates != 0 && q->candidates != 1))
        return REC_ERR_ARG;
    if (q->heads % h->kv_heads) return REC_ERR_SHAPE;
    if ((int64_t)q->table_width * h->page_tokens > MOST_TOKENS || (int64_t)q->queries * q->heads >= 1ll << 31 ||
        (int64_t)q->queries * q->heads * q->batch >= 1ll << 31)
        return REC_ERR_OVERFLOW;
    return REC_OK;
}

rec_status check_query(const rec_history *h, const rec_query *q)
{
    const rec_status st = check_counts(h, q);
    if (st != REC_OK) return st;
    return rec::hist::attend_threads(cache_of(h), h->format, h->head_dim, *q) > MOST_THREADS ? REC_ERR_OVERFLOW : REC_OK;
}

// Calls in which all that stands before a query may be seen.
rec_status check_unmasked(const rec_history *h, const rec_query *q)
{
    const rec_status st = check_counts(h, q);
    return st == REC_OK && (q->window || q->sinks) ? REC_ERR_ARG : st;
}

rec_status check_select(const rec_history *h, const rec_query *q, int32_t count)
{
    const rec_status st = check_unmasked(h, q);
    if (st != REC_OK) return st;
    if (count < 1) return REC_ERR_ARG;
    if (count > MOST_TOKENS) return REC_ERR_OVERFLOW;  // entries are counted a block of up to 1024 threads past the last one
    return rec::hist::select_threads(cache_of(h), h->head_dim, *q) > MOST_THREADS ? REC_ERR_OVERFLOW : REC_OK;
}

rec_status check_chosen(const rec_history *h, const rec_query *q, int32_t count)
{
    const rec_status st = check_unmasked(h, q);
    if (st != REC_OK) return st;
    if (count < 1) return REC_ERR_ARG;
    if ((int64_t)count * h->page_tokens > MOST_TOKENS) return REC_ERR_OVERFLOW;
    return rec::hist::chosen_threads(cache_of(h), h->format, h->head_dim, *q, count) > MOST_THREADS ? REC_ERR_OVERFLOW : REC_OK;
}

rec_status check_shared(const rec_history *h, const rec_query *q, int32_t prefix_width)
{
    const rec_status st = check_unmasked(h, q);
    if (st != REC_OK) return st;
    if (prefix_width < 0) return REC_ERR_ARG;
    if ((int64_t)prefix_width * h->page_tokens > MOST_TOKENS) return REC_ERR_OVERFLOW;
    const Cache c = cache_of(h);
    return std::max(rec::hist::attend_threads(c, h->format, h->head_dim, *q), rec::hist::shared_threads(c, h->format, h->head_dim, *q, prefix_width)) >
                   MOST_THREADS
               ? REC_ERR_OVERFLOW
               : REC_OK;
}

// What a query that has something to do points to, but for its results.
bool query_fits(const rec_query *q)
{
    return aligned(q->dev_q) && stride_fits(q->batch_stride, 2) && stride_fits(q->query_stride, 2) && stride_fits(q->head_stride, 2) &&
           q->dev_lengths && words_fit(q->dev_lengths, 4) && (q->table_width == 0 || q->dev_pages_of) && words_fit(q->dev_pages_of, 4);
}

bool workspace_fits(size_t need, const void *dev, size_t bytes) { return !need || (aligned(dev) && bytes >= need); }

bool rows_fit(const rec_rows &r, int size)
{
    return aligned(r.dev) && stride_fits(r.token_stride, size) && stride_fits(r.head_stride, size);
}

// Tiles of 64 rows are addressed from their first one in 31 bits.
bool tiles_fit(const rec_rows &r) { return r.token_stride >= 0 && r.token_stride < 1ll << 23; }

// Rows [tokens][heads][d] that have no element in common.
bool rows_apart(const rec_rows &r, int64_t tokens, int64_t heads, int64_t d)
{
    int64_t near = r.head_stride < 0 ? -r.head_stride : r.head_stride, far = r.token_stride < 0 ? -r.token_stride : r.token_stride;
    int64_t n_near = heads, n_far = tokens;
    if (near > far) {
        std::swap(near, far);
        std::swap(n_near, n_far);
    }
    // Bounds as quotients: products of strides and counts may not fit 64 bits.
    return (n_near == 1 || near >= d) && (n_far == 1 || (far >= d && (n_near == 1 || (far - d) / near >= n_near - 1)));
}

// Rows [tokens][heads][d] of `size` bytes an element.
struct Place {
    const rec_rows *r;
    int64_t heads;
};

// Whether the rows x of a result and those of another argument have no element in common.  `own`: y is what x is made of, so that they may be the
// same rows: each is read before it is written.  Rows between each other's of several tokens that are as many, but not as far apart, count as overlapping; so do
// more than 2^20 pairs of heads that lie between each other.
bool places_apart(const Place &x, const Place &y, bool own, int64_t tokens, int64_t d, int size)
{
    typedef __int128 wide;  // products of strides and counts
    struct Span {
        wide from, to;
    };
    const auto span_of = [&](const Place &p, int64_t n) {  // of n tokens, in bytes
        const wide t = (wide)p.r->token_stride * (n - 1), h = (wide)p.r->head_stride * (p.heads - 1);
        const wide from = reinterpret_cast<uintptr_t>(p.r->dev);
        return Span{from + ((t < 0 ? t : 0) + (h < 0 ? h : 0)) * size, from + ((t > 0 ? t : 0) + (h > 0 ? h : 0) + d) * size};
    };
    const Span a = span_of(x, tokens), b = span_of(y, tokens);
    if (a.to <= b.from || b.to <= a.from) return true;
    const bool same_tokens = tokens == 1 || x.r->token_stride == y.r->token_stride;
    if (own && same_tokens && x.r->dev == y.r->dev && (x.heads == 1 || x.r->head_stride == y.r->head_stride)) return true;
    // One row for all tokens or heads: y's only, as a result's would overlap (rows_apart()).
    const int64_t y_tokens = y.r->token_stride == 0 ? 1 : tokens, y_heads = y.r->head_stride == 0 ? 1 : y.heads;
    if (!same_tokens && y_tokens > 1) return false;
    const wide by_token = (wide)x.r->token_stride * size, step = by_token < 0 ? -by_token : by_token;  // not 0, of several tokens
    if (tokens > 1) {
        // What x and y have of a token, repeated a step further each time.
        const Span p = span_of(x, 1), q = span_of(y, 1);
        const wide ahead = ((q.from - p.from) % step + step) % step;
        if (p.to - p.from <= ahead && ahead + (q.to - q.from) <= step) return true;
    }
    const wide bytes = (wide)d * size;
    // Whether a row of y, `at` bytes behind one of x in their first tokens, meets it in others: with y's n tokens behind x's.
    const auto meet = [&](wide at) {
        if (tokens > 1) {
            const wide last = tokens - 1, least = by_token < 0 ? -last : 1 - (wide)y_tokens, most = by_token < 0 ? (wide)y_tokens - 1 : last;
            at -= std::clamp<wide>((at < 0 ? at - step / 2 : at + step / 2) / step, least, most) * step;
        }
        return at < bytes && -at < bytes;
    };
    const wide off = (wide) reinterpret_cast<uintptr_t>(y.r->dev) - (wide) reinterpret_cast<uintptr_t>(x.r->dev);
    const wide x_head = (wide)x.r->head_stride * size, y_head = (wide)y.r->head_stride * size;
    if (x.heads == 1 || y_heads == 1 || x_head == y_head) {  // the same for heads as far apart
        for (int64_t i = 1 - x.heads; i < y_heads; ++i)
            if (meet(off + i * (x.heads == 1 ? y_head : x_head))) return false;
        return true;
    }
    if (x.heads * y_heads > 1 << 20) return false;
    for (int64_t i = 0; i < x.heads; ++i)
        for (int64_t j = 0; j < y_heads; ++j)
            if (meet(off + j * y_head - i * x_head)) return false;
    return true;
}

rec_status status_of(hipError_t e) { return e == hipSuccess ? REC_OK : REC_ERR_DEVICE; }

}  // namespace

extern "C" {

size_t rec_history_bytes(const rec_history *h)
{
    if (!h || !shape_fits(h)) return 0;
    const size_t group = h->format == REC_MX4 ? rec::hist::group_bytes<REC_MX4>(h->head_dim)
                                              : rec::hist::group_bytes<REC_MX8>(h->head_dim);
    return (size_t)h->num_pages * h->kv_heads * (h->page_tokens / 16) * group;
}

rec_status rec_history_write(const rec_history *h, const rec_rows *k, const rec_rows *v, int32_t dtype,
                             const int64_t *dev_slots, int64_t tokens, void *stream)
{
    const rec_status st = check_rows(h, dtype, dev_slots, tokens);
    if (st != REC_OK) return st;
    if (!k || !v) return REC_ERR_ARG;
    if (tokens == 0) return REC_OK;
    const int size = dtype == REC_F32 ? 4 : 2;
    if (!rows_fit(*k, size) || !rows_fit(*v, size)) return REC_ERR_ARG;
    return status_of(rec::hist::launch_write(cache_of(h), h->format, h->head_dim, *k, *v, dtype, dev_slots, tokens,
                                             static_cast<hipStream_t>(stream)));
}

rec_status rec_history_read(const rec_history *h, const int64_t *dev_slots, int64_t tokens, int32_t dtype, void *dev_k,
                            void *dev_v, void *stream)
{
    const rec_status st = check_rows(h, dtype, dev_slots, tokens);
    if (st != REC_OK) return st;
    if (tokens == 0) return REC_OK;
    if (!aligned(dev_k) || !aligned(dev_v)) return REC_ERR_ARG;
    return status_of(rec::hist::launch_read(cache_of(h), h->format, h->head_dim, dev_slots, tokens, dtype, dev_k, dev_v,
                                            static_cast<hipStream_t>(stream)));
}

size_t rec_history_attend_workspace_bytes(const rec_history *h, const rec_query *q)
{
    if (check_query(h, q) != REC_OK) return 0;
    return rec::hist::attend_workspace(cache_of(h), h->format, h->head_dim, *q);
}

rec_status rec_history_attend(const rec_history *h, const rec_query *q, void *dev_workspace, size_t workspace_bytes, void *stream)
{
    const rec_status st = check_query(h, q);
    if (st != REC_OK) return st;
    if (!aligned(h->dev_pages) || !words_fit(h->dev_fault, 8)) return REC_ERR_ARG;
    if (q->batch == 0 || q->queries == 0) return REC_OK;
    if (!query_fits(q) || !aligned(q->dev_out)) return REC_ERR_ARG;
    if (!workspace_fits(rec::hist::attend_workspace(cache_of(h), h->format, h->head_dim, *q), dev_workspace, workspace_bytes)) return REC_ERR_ARG;
    return status_of(rec::hist::launch_attend(cache_of(h), h->format, h->head_dim, *q, dev_workspace,
                                              static_cast<hipStream_t>(stream)));
}

rec_status rec_history_summarise(const rec_history *h, const int32_t *dev_which, int32_t pages, void *dev_means, void *stream)
{
    if (!h) return REC_ERR_ARG;
    if (!shape_fits(h)) return REC_ERR_SHAPE;
    if (!aligned(h->dev_pages) || !words_fit(h->dev_fault, 8) || pages < 0) return REC_ERR_ARG;
    if (pages && (!dev_which || !words_fit(dev_which, 4) || !aligned(dev_means))) return REC_ERR_ARG;
    const Cache c = cache_of(h);
    if (rec::hist::means_threads(c, h->head_dim, pages) > MOST_THREADS) return REC_ERR_OVERFLOW;
    if (pages == 0) return REC_OK;
    return status_of(rec::hist::launch_means(c, h->format, h->head_dim, dev_which, pages, dev_means, static_cast<hipStream_t>(stream)));
}

size_t rec_history_select_workspace_bytes(const rec_history *h, const rec_query *q, int32_t count)
{
    return check_select(h, q, count) != REC_OK ? 0 : rec::hist::select_workspace(cache_of(h), h->head_dim, *q, count);
}

rec_status rec_history_select(const rec_history *h, const rec_query *q, const void *dev_means, int32_t count, int32_t first,
                              int32_t last, int32_t *dev_chosen, void *dev_workspace, size_t workspace_bytes, void *stream)
{
    const rec_status st = check_select(h, q, count);
    if (st != REC_OK) return st;
    if (first < 0 || last < 1 || (int64_t)first + last > count || !words_fit(h->dev_fault, 8)) return REC_ERR_ARG;
    if (q->batch == 0 || q->queries == 0) return REC_OK;
    if (!query_fits(q) || !aligned(dev_means) || !dev_chosen || !words_fit(dev_chosen, 4)) return REC_ERR_ARG;
    const Cache c = cache_of(h);
    if (!workspace_fits(rec::hist::select_workspace(c, h->head_dim, *q, count), dev_workspace, workspace_bytes)) return REC_ERR_ARG;
    const rec::hist::Select sel = {dev_means, count, first, last, dev_chosen, static_cast<unsigned long long *>(dev_workspace)};
    return status_of(rec::hist::launch_select(c, h->head_dim, *q, sel, static_cast<hipStream_t>(stream)));
}

size_t rec_history_attend_selected_workspace_bytes(const rec_history *h, const rec_query *q, int32_t count)
{
    return check_chosen(h, q, count) != REC_OK ? 0 : rec::hist::chosen_workspace(cache_of(h), h->format, h->head_dim, *q, count);
}

rec_status rec_history_attend_selected(const rec_history *h, const rec_query *q, const int32_t *dev_chosen, int32_t count,
                                       void *dev_workspace, size_t workspace_bytes, void *stream)
{
    const rec_status st = check_chosen(h, q, count);
    if (st != REC_OK) return st;
    if (!aligned(h->dev_pages) || !words_fit(h->dev_fault, 8)) return REC_ERR_ARG;
    if (q->batch == 0 || q->queries == 0) return REC_OK;
    if (!query_fits(q) || !aligned(q->dev_out) || !dev_chosen || !words_fit(dev_chosen, 4)) return REC_ERR_ARG;
    const Cache c = cache_of(h);
    if (!workspace_fits(rec::hist::chosen_workspace(c, h->format, h->head_dim, *q, count), dev_workspace, workspace_bytes)) return REC_ERR_ARG;
    return status_of(rec::hist::launch_chosen(c, h->format, h->head_dim, *q, dev_chosen, count, dev_workspace, static_cast<hipStream_t>(stream)));
}

size_t rec_history_attend_shared_workspace_bytes(const rec_history *h, const rec_query *q, int32_t prefix_width)
{
    return check_shared(h, q, prefix_width) != REC_OK ? 0 : rec::hist::shared_workspace(cache_of(h), h->format, h->head_dim, *q, prefix_width);
}

rec_status rec_history_attend_shared(const rec_history *h, const rec_query *q, const int32_t *dev_prefix_pages, int32_t prefix_width,
                                     const int32_t *dev_prefix_length, void *dev_workspace, size_t workspace_bytes, void *stream)
{
    const rec_status st = check_shared(h, q, prefix_width);
    if (st != REC_OK) return st;
    if (!aligned(h->dev_pages) || !words_fit(h->dev_fault, 8)) return REC_ERR_ARG;
    if (q->batch == 0 || q->queries == 0) return REC_OK;
    if (!query_fits(q) || !aligned(q->dev_out) || (prefix_width && !dev_prefix_pages) || !words_fit(dev_prefix_pages, 4) || !dev_prefix_length ||
        !words_fit(dev_prefix_length, 4))
        return REC_ERR_ARG;
    const Cache c = cache_of(h);
    if (!workspace_fits(rec::hist::shared_workspace(c, h->format, h->head_dim, *q, prefix_width), dev_workspace, workspace_bytes)) return REC_ERR_ARG;
    const rec::hist::Prefix prefix = {dev_prefix_pages, prefix_width, dev_prefix_length};
    return status_of(rec::hist::launch_shared(c, h->format, h->head_dim, *q, prefix, dev_workspace, static_cast<hipStream_t>(stream)));
}

rec_status rec_window_attend(const rec_window *w, void *stream)
{
    if (!w || (w->dtype != REC_F16 && w->dtype != REC_BF16) || w->batch < 0 || w->tokens < 0 || w->heads < 1 || w->kv_heads < 1 ||
        w->window < 0 || w->sinks < 0)
        return REC_ERR_ARG;
    if (!head_dim_fits(w->head_dim) || w->heads % w->kv_heads) return REC_ERR_SHAPE;
    if (w->tokens > MOST_TOKENS || w->tokens * w->heads >= 1ll << 31) return REC_ERR_OVERFLOW;
    if (rec::hist::window_blocks(*w) > MOST_THREADS / 256 || !tiles_fit(w->k) || !tiles_fit(w->v)) return REC_ERR_OVERFLOW;
    if (w->tokens == 0 || w->batch == 0) return REC_OK;
    if (!rows_fit(w->q, 2) || !rows_fit(w->k, 2) || !rows_fit(w->v, 2) || !aligned(w->dev_out) || !w->dev_offsets ||
        !words_fit(w->dev_offsets, 4) || !words_fit(w->dev_fault, 8))
        return REC_ERR_ARG;
    return status_of(rec::hist::launch_window(*w, static_cast<hipStream_t>(stream)));
}

rec_status rec_rotate_heads(const rec_turn *t, void *stream)
{
    if (!t || (t->dtype != REC_F32 && t->dtype != REC_F16 && t->dtype != REC_BF16) || t->tokens < 0 || t->heads < 0 || t->kv_heads < 0 ||
        (t->wide != 0 && t->wide != 1) || (t->interleaved != 0 && t->interleaved != 1) || !(t->eps >= 0.0f))
        return REC_ERR_ARG;
    if (!head_dim_fits(t->head_dim) || t->pairs < 0 || t->pairs % 8 || t->pairs > t->head_dim / 2) return REC_ERR_SHAPE;
    const int64_t all = (int64_t)t->heads + t->kv_heads;
    if (all > 1 << 20) return REC_ERR_OVERFLOW;
    if (t->tokens == 0 || all == 0) return REC_OK;
    if (t->tokens > MOST_TOKENS || rec::hist::rotate_threads(*t) > MOST_THREADS) return REC_ERR_OVERFLOW;
    const int size = t->dtype == REC_F32 ? 4 : 2;
    if (t->heads && (!rows_fit(t->q, size) || !rows_fit(t->q_out, size) || !rows_apart(t->q_out, t->tokens, t->heads, t->head_dim))) return REC_ERR_ARG;
    if (t->kv_heads && (!rows_fit(t->k, size) || !rows_fit(t->k_out, size) || !rows_apart(t->k_out, t->tokens, t->kv_heads, t->head_dim))) return REC_ERR_ARG;
    const Place q = {&t->q, t->heads}, k = {&t->k, t->kv_heads}, q_out = {&t->q_out, t->heads}, k_out = {&t->k_out, t->kv_heads};
    const auto apart = [&](const Place &x, const Place &y, bool own) {
        return !x.heads || !y.heads || places_apart(x, y, own, t->tokens, t->head_dim, size);
    };
    if (!apart(q_out, q, true) || !apart(k_out, k, true) || !apart(q_out, k, false) || !apart(k_out, q, false) || !apart(q_out, k_out, false)) return REC_ERR_ARG;
    if (t->pairs && (!t->dev_positions || !words_fit(t->dev_positions, t->wide ? 8 : 4) || !t->dev_frequencies || !words_fit(t->dev_frequencies, 8)))
        return REC_ERR_ARG;
    if ((t->dev_q_weight && !aligned(t->dev_q_weight)) || (t->dev_k_weight && !aligned(t->dev_k_weight))) return REC_ERR_ARG;
    return status_of(rec::hist::launch_rotate(*t, static_cast<hipStream_t>(stream)));
}

rec_status rec_history_check(uint64_t *dev_fault, void *stream, int64_t *first_bad_pos, int32_t *word)
{
    if (!dev_fault || !words_fit(dev_fault, 8)) return REC_ERR_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    rec::hist::Faults read;
    const auto &f = read.word;
    if (hipStreamSynchronize(s) != hipSuccess) return REC_ERR_DEVICE;
    if (hipMemcpy(&read, dev_fault, sizeof(read), hipMemcpyDeviceToHost) != hipSuccess) return REC_ERR_DEVICE;
    if (rec::hist::launch_clear_faults(reinterpret_cast<unsigned long long *>(dev_fault), read, s) != hipSuccess) return REC_ERR_DEVICE;
    if (hipStreamSynchronize(s) != hipSuccess) return REC_ERR_DEVICE;
    for (int i = 0; i < REC_FAULT_WORDS; ++i) {
        if (f[i] == ~0ull) continue;
        if (first_bad_pos) *first_bad_pos = (int64_t)f[i];
        if (word) *word = i;
        return i == REC_FAULT_LENGTH ? REC_ERR_LENGTHS : i == REC_FAULT_VALUE ? REC_ERR_VALUE : REC_ERR_INDEX_RANGE;
    }
    if (first_bad_pos) *first_bad_pos = -1;
    if (word) *word = -1;
    return REC_OK;
}

rec_status rec_probe_history_form(const rec_history *h, const rec_query *q, int32_t *form)
{
    if (!form) return REC_ERR_ARG;
    const rec_status st = check_query(h, q);
    if (st != REC_OK) return st;
    int32_t f[3];
    rec::hist::attend_form(cache_of(h), h->format, h->head_dim, *q, f);
    for (int i = 0; i < 3; ++i) form[i] = f[i];
    return REC_OK;
}

rec_status rec_probe_select_form(const rec_history *h, const rec_query *q, int32_t count, int32_t *form)
{
    if (!form) return REC_ERR_ARG;
    const rec_status st = check_select(h, q, count);
    if (st != REC_OK) return st;
    int32_t f[3];
    rec::hist::select_form(cache_of(h), h->head_dim, *q, count, f);
    for (int i = 0; i < 3; ++i) form[i] = f[i];
    return REC_OK;
}

rec_status rec_probe_shared_form(const rec_history *h, const rec_query *q, int32_t prefix_width, int32_t *form)
{
    if (!form) return REC_ERR_ARG;
    const rec_status st = check_shared(h, q, prefix_width);
    if (st != REC_OK) return st;
    int32_t f[3];
    rec::hist::shared_form(cache_of(h), h->format, h->head_dim, *q, prefix_width, f);
    for (int i = 0; i < 3; ++i) form[i] = f[i];
    return REC_OK;
}

rec_status rec_probe_clear_faults(uint64_t *dev_fault, const uint64_t *seen, void *stream)
{
    if (!dev_fault || !words_fit(dev_fault, 8) || !seen) return REC_ERR_ARG;
    rec::hist::Faults read;
    for (int i = 0; i < REC_FAULT_WORDS; ++i) read.word[i] = seen[i];
    return status_of(rec::hist::launch_clear_faults(reinterpret_cast<unsigned long long *>(dev_fault), read, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
