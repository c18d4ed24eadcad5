// Attention over cached histories.
//
// A wave has 16 query rows of one kv head (its heads of every query, one after the
// other) and walks over 64 keys at a time.  Scores come transposed, S^T = K Q^T, on
// the block-scaled matrix instructions (16 x 16 x 128): they take the cache's codes and
// scale bytes as they lie in memory, so keys cost no vector instruction at all.  A
// query enters as two (fp16: three) E4M3 terms, each the rounding of what the terms before
// left: exact for elements of at least 2^-13 (2^-14) of the largest of their 32, others are off
// by less than 2^-21 (2^-25) of that, which in a score is what sums in fp32 are off by.  For head_dim
// 32 and 64 the terms share an instruction's 128 columns and the keys are repeated.
//
// Key 4 r + x of a tile is row r of its x-th product, so that a lane's scores (column c =
// query row, lane group g) are those of the 16 neighbouring tokens 16 g ..., which is
// what it also loads of the values: one row of a group, 16 tokens of two columns.
// Weights therefore go from scores straight into the operand of O^T += V^T P^T
// (16 x 16 x 32 bf16), with no exchange between lanes.  Values become bf16 exactly: the
// scaled conversions look at a scale's exponent bits only, so one shift puts a scale
// byte in place.  A product with ones sums the weights as they were rounded.  A weight of a bf16 result
// is rounded once, by no more than the result is (2^-8 of itself), and an fp16 result's has what that left beside
// it.  Errors against 64 bits, of the outputs' size, 32 x 32768: 0.0023, with weights in fp32 0.0017; a second term
// would make 44 matrix instructions of a tile's 26 (head_dim 128).
//
// The running maximum moves only when a tile's exceeds it by 2^8: weights stay within 2^8 of it,
// and the accumulators are rescaled a few times a history instead of every tile.
//
// Few pairs of history and head are divided: among the waves of a block, which meet in
// LDS, and, where that leaves compute units idle, among blocks, whose parts
// combine_kernel joins.
//
// Long histories are bound by the cache's bytes (32 of 32768 events, 8 kv heads of 128, mx4: 200 us, 5.7 TB/s), many
// short ones by a chain of length, page and tile and the exponentials behind it (4096 of about 80 events, 2 kv heads
// of 32, mx8, fp16: 18 us, 2.5 TB/s), candidates by the keys that several row tiles read (64 x 50 over up to 1004
// events: 22 to 23 us), and so are many causal queries (32 x 64 over 4000 events, 4 kv heads of 64, mx4: 50 us).
#include <algorithm>

#include "history_attend_body.h"

namespace rec {
namespace hist {
namespace {

constexpr int CUS = 256;

// What a launch attends to: histories, histories behind the sums of a prefix, or a prefix and histories one behind the other.
enum { WHOLE, BEHIND, JOINED };

// Waves that a SIMD holds at once; the compiler gives a wave at most its share of registers.
__host__ __device__ constexpr int waves_of(int format, int d, bool bf, int heads, int kind = WHOLE)
{
    if (kind != WHOLE && d == 32 && format == REC_MX8 && heads == 1) return 3;  // a row's parts, or a prefix, besides
    if (heads > 1) return d == 32 && format == REC_MX4 ? 3 : 2;
    return d == 128 ? (format == REC_MX4 && bf ? 3 : 2) : d == 64 ? (format == REC_MX4 && bf ? 4 : 3) : 4;
}

struct AttendArgs {
    Cache c;
    rec_query q;
    int per;        // query heads of a kv head
    Divider by_per;
    int rows;       // queries * per
    int row_tiles;  // of ROWS
    int splits;
    Divider inner, heads;  // by splits * row_tiles, by the waves that have a history's kv heads
    float *part_o;   // [splits][batch * queries * heads][D]
    f32x2 *part_ml;  // [splits][batch * queries * heads]
    bool parted;     // the results are parts, even of one split
    // Histories behind a prefix: their rows' sums over it, which results include.
    int before;            // parts of it
    const float *before_o;
    const f32x2 *before_ml;
    Prefix prefix;
};

// Joins a row's sums x, of some columns, its weights' sum l and its maximum's exponent m with those of `parts` parts, in their order.
// part: of the first part's same columns, `stride` elements apart; ml: of its maximum and sum.
template <int N>
__device__ inline void add_parts(f32x4 (&x)[N], float &l, float &m, const float *part, int stride, const f32x2 *ml, int parts, long long all_rows, int d)
{
    const auto weight = [](f32x2 ml, float most) { return ml[0] == neg_inf() ? (ml[1] == 0.0f ? 0.0f : ml[1]) : __builtin_amdgcn_exp2f(ml[0] - most); };
    float most = m;
#pragma unroll 4
    for (int i = 0; i < parts; ++i) most = fmaxf(most, ml[i * all_rows][0]);
    const float mine = weight(f32x2{m, l}, most);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= mine;
    l *= mine;
#pragma unroll 4
    for (int i = 0; i < parts; ++i) {
        const f32x2 its = ml[i * all_rows];
        const float by = weight(its, most);
        l += its[1] * by;
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] += *reinterpret_cast<const f32x4 *>(part + i * all_rows * d + stride * j) * by;
    }
    m = most;
}

// Where a wave's row goes.
__device__ inline long long out_row(const AttendArgs &a, int b, int kv, int row)
{
    const int i = a.by_per.of(row);
    return ((long long)b * a.q.queries + i) * a.q.heads + kv * a.per + (row - i * a.per);
}

template <int FMT, int D, bool BF, int W, int HEADS, int KIND>
__global__ __launch_bounds__(64 * W, waves_of(FMT, D, BF, HEADS, KIND)) void attend_kernel(AttendArgs a)
{
    static_assert(HEADS == 1 || W == 1, "several heads a wave: only where there are waves enough");
    constexpr int SLOT = ROWS / HEADS;  // rows of a kv head
    using T = std::conditional_t<BF, __bf16, _Float16>;
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int slot = c / SLOT, r = c % SLOT;  // which of the wave's kv heads, and its row
    // Parts of a history's head next to each other, then its heads, whose groups share a page.
    const int pair = a.inner.of((int)blockIdx.x), part = (int)blockIdx.x - pair * a.splits * a.row_tiles;
    const int b = a.heads.of(pair), first_kv = pair * HEADS - b * a.c.kv_heads, kv = first_kv + slot;
    const int row_tile = a.splits == 1 ? part : part / a.splits, split = part - row_tile * a.splits;

    const int shift = a.c.page_shift, most_tokens = a.q.table_width << shift;
    int len = a.q.dev_lengths[b];
    if (len < 0 || len > most_tokens) {
        if (threadIdx.x == 0 && first_kv == 0) report(a.c.fault, REC_FAULT_LENGTH, (unsigned long long)b);
        len = len < 0 ? 0 : most_tokens;
    }
    // Tokens of the prefix, and where a history's first one stands behind it: at the next group of 16, as a group is in one page.
    int prefix = 0, own = 0;
    if constexpr (KIND == JOINED) {
        const int most = a.prefix.width << shift;
        prefix = *a.prefix.length;
        if (prefix < 0 || prefix > most) {
            if (blockIdx.x == 0 && threadIdx.x == 0) report(a.c.fault, REC_FAULT_LENGTH, (unsigned long long)a.q.batch);
            prefix = prefix < 0 ? 0 : most;
        }
        own = (prefix + GROUP - 1) & -GROUP;
    }
    // Positions of this wave's rows: of its first, its last, and this lane's; -1 sees nothing.
    const int first_row = row_tile * ROWS, last_row = min(first_row + SLOT, a.rows) - 1, row = min(first_row + r, last_row);
    const bool real = first_row + r <= last_row;
    const bool together = a.q.candidates != 0;
    auto position = [&](int row) {
        const int p = together ? len - 1 : max(len - a.q.queries + a.by_per.of(row), -1);
        return KIND == JOINED && (p >= 0 || together) ? own + p : p;
    };
    const int p_lo = position(first_row), p_hi = position(last_row), pos = position(row);
    const int window = a.q.window == 0 ? 0x7fffffff : a.q.window, sinks = a.q.sinks;

    // Tiles that some row sees something of: [0, n_sink) and [n_from, n_to).
    int n_from = 0, n_sink = 0, n_to = 0;
    if (p_hi >= 0) {
        n_to = p_hi / TILE + 1;
        n_from = max(p_lo - window + 1, 0) / TILE;
        n_sink = min((min(sinks, p_hi + 1) + TILE - 1) / TILE, n_from);
    }
    const int tiles = n_sink + n_to - n_from, each = (tiles + a.splits - 1) / a.splits;
    const int begin = min(split * each, tiles), end = min(begin + each, tiles);

    Sums<D, HEADS> sum;
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int i = 0; i < D / 16; ++i) sum.o[h][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    sum.l = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    sum.m = neg_inf();
    unsigned saw = 0;  // not 0: this lane's row has seen a key

    if (begin + wave < end) {
        const int query = a.by_per.of(row), head = kv * a.per + row - query * a.per;
        const long long row_bytes = 2 * (b * a.q.batch_stride + query * a.q.query_stride + head * a.q.head_stride);
        // Positive, so that masked scores stay at -inf.
        const float factor = a.q.scale == 0.0f ? 1.0f : __builtin_fabsf(a.q.scale) * 1.44269504088896341f;
        const int32_t *table = a.q.dev_pages_of + b * a.q.table_stride;
        const int groups = 1 << (shift - 4);
        const int head_bytes = groups * group_bytes<FMT>(D);
        const unsigned char *first_page = a.c.pages + (long long)first_kv * head_bytes;
        const unsigned page_bytes = (unsigned)(a.c.kv_heads * head_bytes);
        const unsigned pages = (unsigned)min(a.c.num_pages, 1ll << 31);

        // Tile n of the walk starts at this key.
        auto key_of = [&](int n) { return (n < n_sink ? n : n_from + n - n_sink) * TILE; };
        // The page of a group's first token, or -1.
        auto page_of = [&](int token) {
            int page = -1;
            if (KIND == JOINED && token < own) page = a.prefix.pages[token >> shift];
            else if (token - own < len) page = table[(token - own) >> shift];
            return page;
        };
        auto group_at = [&](int page, int token) {
            const bool ok = (unsigned)page < pages;  // else some group that is there: its tokens count for nothing
            if (KIND == JOINED && token >= own) token -= own;
            const unsigned in_page = ok ? (unsigned)((token >> 4) & (groups - 1)) * group_bytes<FMT>(D) : 0u;
            return first_page + ((unsigned long long)(ok ? (unsigned)page : 0u) * page_bytes + in_page);
        };

        int n = begin + wave, key = key_of(n);
        int k_page = page_of(key + 16 * (c >> 2)), v_page = page_of(key + 16 * g);
        Query<D, BF> q;
        q.fetch(real ? static_cast<const char *>(a.q.dev_q) + row_bytes : nullptr, g);
        Tile<FMT, D> tile[HEADS];
        auto load_keys = [&](int h, int key) { tile[h].load_keys(group_at(k_page, key + 16 * (c >> 2)) + h * head_bytes, c, g); };
        auto load_values = [&](int h, int page, int key) { tile[h].load_values(group_at(page, key + 16 * g) + h * head_bytes, c); };
#pragma unroll
        for (int h = 0; h < HEADS; ++h) load_keys(h, key);
#pragma unroll
        for (int h = 0; h < HEADS; ++h) load_values(h, v_page, key);
        k_page = n + W < end ? page_of(key_of(n + W) + 16 * (c >> 2)) : -1;
        int v_next = n + W < end ? page_of(key_of(n + W) + 16 * g) : -1;
        q.convert(a.q.scale < 0.0f ? -1.0f : a.q.scale == 0.0f ? 0.0f : 1.0f, g);  // while the first tile is on its way
        for (;; n += W) {
            const bool more = n + W < end;
            const int key_next = more ? key_of(n + W) : 0;
            f32x4 s[4];
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
                const f32x4 mine[4] = {scores<FMT, D, BF, 0>(tile[h], q, g), scores<FMT, D, BF, 1>(tile[h], q, g),
                                       scores<FMT, D, BF, 2>(tile[h], q, g), scores<FMT, D, BF, 3>(tile[h], q, g)};
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[x][i] = h == 0 || slot == h ? mine[x][i] : s[x][i];
                // The next tile's keys and values take the place of this one's as soon as that is used.
                if (more) load_keys(h, key_next);
            }

            // Groups come with their page or not at all.
            const bool there = (unsigned)v_page < pages;
            const bool whole = key + TILE - 1 <= p_lo && (key > p_hi - window || key + TILE <= sinks) && __all(there) &&
                               !(KIND == JOINED && key < own && key + TILE > prefix);
            unsigned nan = 0;  // bit 4 h + b: row c sees a NaN in block b of head h's values
            if (!whole) {
                // Bit t: row c sees token t of group g; some row does.
                const int first = key + 16 * g;
                auto upto = [&](int at) { return below(max(at - first, -1) + 1); };
                auto before = [&](int at) { return below(max(at - first, -1) - window + 1); };
                unsigned seen = upto(pos) & (~before(pos) | below(sinks - first));
                unsigned used = upto(p_hi) & (~before(p_lo) | below(sinks - first));
                if (KIND == JOINED && first < own) {  // nothing stands between the prefix's end and the history
                    seen &= below(prefix - first);
                    used &= below(prefix - first);
                }
                if (!there) {
                    if (used && c == 0)
                        report(a.c.fault, REC_FAULT_PAGE, (unsigned long long)(KIND == JOINED && first < own ? a.q.batch : b) * (unsigned)a.q.table_width +
                                                              (unsigned)((KIND == JOINED && first >= own ? first - own : first) >> shift));
                    seen = used = 0;
                }
                saw |= seen;
#pragma unroll
                for (int h = 0; h < HEADS; ++h) {
                    nan |= clear_values<FMT, D>(tile[h], used, seen) << (4 * h);
                    if constexpr (FMT == REC_MX8)
                        if (p_lo != p_hi) clear_nan_codes<D>(tile[h], seen, sum.o[h]);
                }
#pragma unroll
                for (int t = 0; t < 16; ++t) s[t & 3][t >> 2] = unless_hidden(s[t & 3][t >> 2], ~seen, t);
            } else {
                saw = 1;
            }

            float most = neg_inf();
#pragma unroll
            for (int t = 0; t < 16; ++t) most = fmaxf(most, s[t & 3][t >> 2]);
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            most = most == neg_inf() ? most : most * factor;
            if (__any(most > sum.m + (SLACK - ROOM))) {
                const float m = fmaxf(sum.m, most + ROOM);
                if (__any(sum.m != neg_inf())) {  // not the first tile
                    const float down = sum.m == m ? 1.0f : __builtin_amdgcn_exp2f(sum.m - m);
#pragma unroll
                    for (int h = 0; h < HEADS; ++h)
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) sum.o[h][i] *= down;
                    sum.l *= down;
                }
                sum.m = m;
            }
            const float by = sum.m == neg_inf() ? 0.0f : sum.m;  // a row that sees nothing yet has weights of 2^(-inf)
            float p[16];
#pragma unroll
            for (int t = 0; t < 16; ++t) p[t] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t & 3][t >> 2], factor, -by));

            // Weights as bf16, for fp16 results with what that rounding left out beside them.
            constexpr int TERMS = BF ? 1 : 2;
            u32x4 w[TERMS][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[0][h][i] = pack(p[8 * h + 2 * i], p[8 * h + 2 * i + 1]);
                    if constexpr (TERMS == 2) {
                        const unsigned word = w[0][h][i];
                        w[1][h][i] = pack(p[8 * h + 2 * i] - __builtin_bit_cast(float, word << 16),
                                          p[8 * h + 2 * i + 1] - __builtin_bit_cast(float, word & 0xffff0000u));
                    }
                }
            const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
            for (int k = 0; k < TERMS; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) sum.l = product(ones, w[k][h], sum.l);
#pragma unroll
            for (int h = 0; h < HEADS; ++h)
#pragma unroll
                for (int i = 0; i < D / BLOCK; ++i) {
                    f32x4 &x = sum.o[h][2 * i], &y = sum.o[h][2 * i + 1];
                    u32x4 lo, hi;
                    value_operands<FMT, D, 0>(tile[h], i, lo, hi);
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) {
                        x = product(lo, w[k][0], x);
                        y = product(hi, w[k][0], y);
                    }
                    value_operands<FMT, D, 1>(tile[h], i, lo, hi);
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) {
                        x = product(lo, w[k][1], x);
                        y = product(hi, w[k][1], y);
                    }
                }
            if (nan)
#pragma unroll
                for (int h = 0; h < HEADS; ++h)
#pragma unroll
                    for (int i = 0; i < D / 16; ++i)
                        if (nan >> (4 * h + i / 2) & 1u) sum.o[h][i] += __builtin_nanf("");
            if (!more) break;
#pragma unroll
            for (int h = 0; h < HEADS; ++h) load_values(h, v_next, key_next);
            key = key_next;
            v_page = v_next;
            if (n + 2 * W < end) {
                k_page = page_of(key_of(n + 2 * W) + 16 * (c >> 2));
                v_next = page_of(key_of(n + 2 * W) + 16 * g);
            }
        }
    }

    // All of a row's scores may be -inf, which is not the same as having none: the maximum tells.
    saw |= (unsigned)__shfl_xor((int)saw, 16);
    saw |= (unsigned)__shfl_xor((int)saw, 32);
    if (saw && sum.m == neg_inf() && sum.l[0] == 0.0f) sum.m = LOWEST;

    f32x4 o[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        o[i] = sum.o[0][i];
#pragma unroll
        for (int h = 1; h < HEADS; ++h) o[i] = slot == h ? sum.o[h][i] : o[i];
    }
    const long long out = out_row(a, b, kv, row);
    const long long all_rows = (long long)a.q.batch * a.q.queries * a.q.heads;
    if constexpr (W == 1) {
        const float l = sum.l[0];
        if (a.parted) {
            if (real && g == 0) a.part_ml[split * all_rows + out] = f32x2{sum.m, l};
            if (real)
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                    *reinterpret_cast<f32x4 *>(a.part_o + (split * all_rows + out) * D + 16 * i + 4 * g) = o[i];
        } else if (real) {
            float m = sum.m, total = l;
            if constexpr (KIND == BEHIND)
                add_parts(o, total, m, a.before_o + out * D + 4 * g, 16, a.before_ml + out, a.before, all_rows, D);
            const float by = inverse(total, m);
            typedef T tx4 __attribute__((ext_vector_type(4)));
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                *reinterpret_cast<tx4 *>(static_cast<T *>(a.q.dev_out) + out * D + 16 * i + 4 * g) = __builtin_convertvector(o[i] * by, tx4);
        }
    } else {
        // Rows of all waves in LDS; a thread then joins eight columns of a row.
        constexpr int LD = D + 4;
        __shared__ float o_of[W][ROWS][LD];
        __shared__ f32x2 ml_of[W][ROWS];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4 *>(&o_of[wave][c][16 * i + 4 * g]) = o[i];
        if (g == 0) ml_of[wave][c] = f32x2{sum.m, sum.l[0]};
        __syncthreads();
        for (int i = threadIdx.x; i < ROWS * D / 8; i += 64 * W) {
            const int r = i / (D / 8), col = i % (D / 8) * 8;
            if (first_row + r > last_row) break;
            float m = neg_inf();
#pragma unroll
            for (int w = 0; w < W; ++w) m = fmaxf(m, ml_of[w][r][0]);
            float l = 0.0f;
            f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = x;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const f32x2 ml = ml_of[w][r];
                const float by = ml[0] == neg_inf() ? (ml[1] == 0.0f ? 0.0f : ml[1]) : __builtin_amdgcn_exp2f(ml[0] - m);
                l += ml[1] * by;
                x += *reinterpret_cast<const f32x4 *>(&o_of[w][r][col]) * by;
                y += *reinterpret_cast<const f32x4 *>(&o_of[w][r][col + 4]) * by;
            }
            const long long to = out_row(a, b, kv, first_row + r);
            if (a.parted) {
                float *p = a.part_o + (split * all_rows + to) * D + col;
                *reinterpret_cast<f32x4 *>(p) = x;
                *reinterpret_cast<f32x4 *>(p + 4) = y;
                if (col == 0) a.part_ml[split * all_rows + to] = f32x2{m, l};
            } else {
                typedef T tx8 __attribute__((ext_vector_type(8)));
                if constexpr (KIND == BEHIND) {
                    f32x4 both[2] = {x, y};
                    add_parts(both, l, m, a.before_o + to * D + col, 4, a.before_ml + to, a.before, all_rows, D);
                    x = both[0];
                    y = both[1];
                }
                const float by = inverse(l, m);
                x *= by;
                y *= by;
                const f32x8 z = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                *reinterpret_cast<tx8 *>(static_cast<T *>(a.q.dev_out) + to * D + col) = __builtin_convertvector(z, tx8);
            }
        }
    }
}

struct Plan {
    int waves, splits, row_tiles, per;
    int heads;       // kv heads of a wave
    long long rows;  // of the whole call
    bool join = true;  // parts become results
};

// `most` is of parts.
Plan plan_of(const Cache &c, int format, int d, const rec_query &q, int kind = WHOLE, int most = MOST_PARTS)
{
    Plan p;
    p.per = q.heads / c.kv_heads;
    p.rows = (long long)q.batch * q.queries * q.heads;
    const long long rows = (long long)q.queries * p.per;
    p.row_tiles = (int)((rows + ROWS - 1) / ROWS);
    const long long pairs = (long long)q.batch * c.kv_heads * p.row_tiles;
    p.waves = p.splits = p.heads = 1;
    if (pairs == 0) return p;
    // Most tiles that a wave's rows can see something of.
    long long tiles = (((long long)q.table_width << c.page_shift) + TILE - 1) / TILE;
    if (q.window) {
        const long long apart = q.candidates ? 0 : std::min<long long>(q.queries - 1, (ROWS - 1) / p.per + 1);
        tiles = std::min(tiles, (q.window + apart + TILE - 2) / TILE + 1 + ((long long)q.sinks + TILE - 1) / TILE);
    }
    // Several waves for a history where there are few pairs, and where the longest may be much longer than most:
    // a wave that has it alone works on when all others are done.  64-wide mx4, 4 kv heads, lengths up to 2000,
    // log-uniform or all alike, four waves against one or two: 1600 pairs 72 -> 51 us or 174 -> 171 (up to 8000), 4096 pairs
    // 53 -> 34 us, 8192 pairs 80 -> 65 us or 111 -> 122.  (80 events: 14.0 us with one wave, 15.0 with four.)
    p.waves = (tiles >= 4 && pairs < 4 * CUS) || (tiles >= 16 && pairs <= 32 * CUS) ? 4 : tiles >= 2 && pairs < 8 * CUS ? 2 : 1;
    // A wave has room for the rows of several kv heads: masks, exponentials and the rows' terms
    // then cost it no more than for one.
    if (d <= 64 && p.waves == 1 && pairs >= 16 * CUS) p.heads = rows <= ROWS / 2 && c.kv_heads % 2 == 0 ? 2 : 1;
    // Long histories of few pairs: as many parts as are all at work at once (a part too many waits
    // for a place and then reads alone: 4 parts of 256 pairs in 3 places 221 us, 3 parts 199; 400 pairs of 1000 tokens behind 4000, of 32 columns in
    // mx8, two parts 21.2, one 19.7), of two tiles a wave at least.
    // Where pairs alone take all places, parts of eight tiles a wave, up to four, for the longest of ragged
    // histories (1600 pairs up to 8000 long 51 -> 43 us; all alike 171 -> 178).
    const long long room = 4ll * waves_of(format, d, q.dtype == REC_BF16, 1, kind) * CUS / (pairs * p.waves);
    const long long parts = room > 1 ? std::min({room, tiles / (2 * p.waves), (long long)most}) : p.waves == 4 ? std::min(tiles / (8 * p.waves), 4ll) : 1;
    p.splits = (int)std::max(1ll, parts);
    return p;
}

template <int FMT, int D, bool BF, int KIND>
hipError_t attend_as(const AttendArgs &a, const Plan &p, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)a.q.batch * a.c.kv_heads / p.heads * p.row_tiles * p.splits));
    if constexpr (D <= 64 && KIND != JOINED)
        if (p.heads == 2) {
            hipLaunchKernelGGL((attend_kernel<FMT, D, BF, 1, 2, KIND>), grid, dim3(64), 0, s, a);
            return hipGetLastError();
        }
    if (p.waves == 4) hipLaunchKernelGGL((attend_kernel<FMT, D, BF, 4, 1, KIND>), grid, dim3(256), 0, s, a);
    else if (p.waves == 2) hipLaunchKernelGGL((attend_kernel<FMT, D, BF, 2, 1, KIND>), grid, dim3(128), 0, s, a);
    else hipLaunchKernelGGL((attend_kernel<FMT, D, BF, 1, 1, KIND>), grid, dim3(64), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1 || !p.join) return e;
    hipLaunchKernelGGL((combine_kernel<D, BF>), dim3((unsigned)p.rows), dim3(256), 0, s, a.part_o, a.part_ml, p.splits, p.rows, a.q.dev_out);
    return hipGetLastError();
}

template <int FMT, int D>
hipError_t attend_of(const AttendArgs &a, const Plan &p, hipStream_t s)
{
    const bool bf = a.q.dtype == REC_BF16;
    if (a.prefix.length) return bf ? attend_as<FMT, D, true, JOINED>(a, p, s) : attend_as<FMT, D, false, JOINED>(a, p, s);
    if (a.before) return bf ? attend_as<FMT, D, true, BEHIND>(a, p, s) : attend_as<FMT, D, false, BEHIND>(a, p, s);
    return bf ? attend_as<FMT, D, true, WHOLE>(a, p, s) : attend_as<FMT, D, false, WHOLE>(a, p, s);
}

hipError_t attend_any(const AttendArgs &a, const Plan &p, int format, int d, hipStream_t s)
{
    if (format == REC_MX4)
        return d == 32 ? attend_of<REC_MX4, 32>(a, p, s) : d == 64 ? attend_of<REC_MX4, 64>(a, p, s) : attend_of<REC_MX4, 128>(a, p, s);
    return d == 32 ? attend_of<REC_MX8, 32>(a, p, s) : d == 64 ? attend_of<REC_MX8, 64>(a, p, s) : attend_of<REC_MX8, 128>(a, p, s);
}

AttendArgs args_of(const Cache &c, int d, const rec_query &q, const Plan &p, void *workspace)
{
    AttendArgs a;
    a.c = c;
    a.q = q;
    a.per = p.per;
    a.by_per = Divider(p.per);
    a.inner = Divider(p.splits * p.row_tiles);
    a.heads = Divider(c.kv_heads / p.heads);
    a.rows = (int)((long long)q.queries * p.per);
    a.row_tiles = p.row_tiles;
    a.splits = p.splits;
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<f32x2 *>(a.part_o + (p.splits > 1 ? p.splits * p.rows * d : 0));
    a.parted = p.splits > 1;
    a.before = 0;
    a.prefix = {nullptr, 0, nullptr};
    return a;
}

size_t workspace_of(const Plan &p, int d) { return p.splits == 1 ? 0 : (size_t)p.splits * (size_t)p.rows * ((size_t)d * sizeof(float) + sizeof(f32x2)); }

long long threads_of(const Cache &c, const rec_query &q, const Plan &p) { return (long long)q.batch * c.kv_heads * p.row_tiles * p.splits * 64 * p.waves; }

}  // namespace

// A call whose histories have the prefix's pages before their own, for plans only.
rec_query joined_query(const rec_query &q, int prefix_width)
{
    rec_query j = q;
    j.table_width += prefix_width + 1;
    return j;
}

long long joined_work(const Cache &c, const rec_query &q, int prefix_width)
{
    const long long rows = (long long)q.queries * (q.heads / c.kv_heads);
    return q.batch * (long long)c.kv_heads * ((rows + ROWS - 1) / ROWS) * ((((long long)q.table_width + prefix_width + 1) << c.page_shift) / TILE + 1);
}

Plan joined_plan(const Cache &c, int format, int d, const rec_query &q, int prefix_width)
{
    Plan p = plan_of(c, format, d, joined_query(q, prefix_width), JOINED);
    p.heads = 1;
    return p;
}

long long joined_threads(const Cache &c, int format, int d, const rec_query &q, int prefix_width)
{
    return threads_of(c, q, joined_plan(c, format, d, q, prefix_width));
}

size_t joined_workspace(const Cache &c, int format, int d, const rec_query &q, int prefix_width)
{
    return workspace_of(joined_plan(c, format, d, q, prefix_width), d);
}

int joined_parts(const Cache &c, int format, int d, const rec_query &q, int prefix_width) { return joined_plan(c, format, d, q, prefix_width).splits; }

hipError_t launch_joined(const Cache &c, int format, int d, const rec_query &q, const Prefix &prefix, void *workspace, hipStream_t s)
{
    const Plan p = joined_plan(c, format, d, q, prefix.width);
    AttendArgs a = args_of(c, d, q, p, workspace);
    a.prefix = prefix;
    return attend_any(a, p, format, d, s);
}

int own_parts(const Cache &c, int format, int d, const rec_query &q) { return plan_of(c, format, d, q, BEHIND, MOST_PARTS - MOST_BEFORE).splits; }

hipError_t launch_behind(const Cache &c, int format, int d, const rec_query &q, const Parts &parts, int before, hipStream_t s)
{
    Plan p = plan_of(c, format, d, q, BEHIND, MOST_PARTS - MOST_BEFORE);
    p.join = false;
    const long long at = before * p.rows;
    AttendArgs a = args_of(c, d, q, p, parts.o + at * d);
    a.part_ml = reinterpret_cast<f32x2 *>(parts.ml) + at;
    a.before = p.splits > 1 ? 0 : before;
    a.before_o = parts.o;
    a.before_ml = reinterpret_cast<const f32x2 *>(parts.ml);
    return attend_any(a, p, format, d, s);
}

long long attend_threads(const Cache &c, int format, int d, const rec_query &q) { return threads_of(c, q, plan_of(c, format, d, q)); }

void attend_form(const Cache &c, int format, int d, const rec_query &q, int32_t (&form)[3])
{
    const Plan p = plan_of(c, format, d, q);
    form[0] = p.waves;
    form[1] = p.splits;
    form[2] = p.heads;
}

size_t attend_workspace(const Cache &c, int format, int d, const rec_query &q)
{
    return q.batch == 0 || q.queries == 0 ? 0 : workspace_of(plan_of(c, format, d, q), d);
}

hipError_t launch_attend(const Cache &c, int format, int d, const rec_query &q, void *workspace, hipStream_t s)
{
    const Plan p = plan_of(c, format, d, q);
    return attend_any(args_of(c, d, q, p, workspace), p, format, d, s);
}

}  // namespace hist
}  // namespace rec
