// Host side of include/rec_history.h: checks, and nothing else.
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

rec_status check_query(const rec_history *h, const rec_query *q)
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
    return rec::hist::attend_threads(cache_of(h), h->format, h->head_dim, *q) > MOST_THREADS ? REC_ERR_OVERFLOW : REC_OK;
}

bool rows_fit(const rec_rows &r, int size)
{
    return aligned(r.dev) && stride_fits(r.token_stride, size) && stride_fits(r.head_stride, size);
}

// Tiles of 64 rows are addressed from their first one in 31 bits.
bool tiles_fit(const rec_rows &r) { return r.token_stride >= 0 && r.token_stride < 1ll << 23; }

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
    if (!aligned(q->dev_q) || !aligned(q->dev_out) || !stride_fits(q->batch_stride, 2) || !stride_fits(q->query_stride, 2) ||
        !stride_fits(q->head_stride, 2) || !q->dev_lengths || !words_fit(q->dev_lengths, 4) || (q->table_width > 0 && !q->dev_pages_of) ||
        !words_fit(q->dev_pages_of, 4))
        return REC_ERR_ARG;
    const size_t need = rec::hist::attend_workspace(cache_of(h), h->format, h->head_dim, *q);
    if (need && (!aligned(dev_workspace) || workspace_bytes < need)) return REC_ERR_ARG;
    return status_of(rec::hist::launch_attend(cache_of(h), h->format, h->head_dim, *q, dev_workspace,
                                              static_cast<hipStream_t>(stream)));
}

rec_status rec_window_attend(const rec_window *w, void *stream)
{
    if (!w || (w->dtype != REC_F16 && w->dtype != REC_BF16) || w->batch < 0 || w->tokens < 0 || w->heads < 1 || w->kv_heads < 1 ||
        w->window < 0 || w->sinks < 0)
        return REC_ERR_ARG;
    if (!head_dim_fits(w->head_dim) || w->heads % w->kv_heads) return REC_ERR_SHAPE;
    if (w->tokens > MOST_TOKENS || w->tokens * w->heads >= 1ll << 31) return REC_ERR_OVERFLOW;
    if (rec::hist::window_blocks(*w) * 256 > MOST_THREADS || !tiles_fit(w->k) || !tiles_fit(w->v)) return REC_ERR_OVERFLOW;
    if (w->tokens == 0 || w->batch == 0) return REC_OK;
    if (!rows_fit(w->q, 2) || !rows_fit(w->k, 2) || !rows_fit(w->v, 2) || !aligned(w->dev_out) || !w->dev_offsets ||
        !words_fit(w->dev_offsets, 4) || !words_fit(w->dev_fault, 8))
        return REC_ERR_ARG;
    return status_of(rec::hist::launch_window(*w, static_cast<hipStream_t>(stream)));
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

rec_status rec_probe_clear_faults(uint64_t *dev_fault, const uint64_t *seen, void *stream)
{
    if (!dev_fault || !words_fit(dev_fault, 8) || !seen) return REC_ERR_ARG;
    rec::hist::Faults read;
    for (int i = 0; i < REC_FAULT_WORDS; ++i) read.word[i] = seen[i];
    return status_of(rec::hist::launch_clear_faults(reinterpret_cast<unsigned long long *>(dev_fault), read, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
