// Attention over chosen pages of cached histories: each query and kv head has a list of its own.
//
// The products are those of history_attend.hip: a wave has 16 rows, here the heads of one query and kv head, and walks over 64 of the
// chosen tokens at a time.  Where a page lies takes two trips to memory, so a wave looks up 64 pages at once, one a lane, and asks
// lanes for them.  Two tiles are on their way in registers: lists are short, and with one a tile took a trip to memory.
// All rows stand at one position, so that a tile's tokens are seen by all or none.
//
// 1024 queries, 2 kv heads of 64 with 4 rows each, mx8, up to 768 tokens: 22.6 us, bound by the longest lists: a wave has one list, of 5 tiles
// on average, a quarter of them of 12, which it walks over one behind the other (350 vector instructions a tile are 6 us of a SIMD in all).
// 16 histories of 2048 chosen tokens, 8 kv heads of 128, mx4: 35.7 MB in 14 us, 2.5 TB/s: 128 blocks of eight waves, on half of the compute units.
#include <algorithm>

#include "history_attend_body.h"

namespace rec {
namespace hist {
namespace {

constexpr int CUS = 256;

// Tiles on their way, as many as registers hold, and waves that a SIMD holds then.
__host__ __device__ constexpr int depth_of(int format, int d) { return format == REC_MX8 && d == 128 ? 1 : 2; }
__host__ __device__ constexpr int waves_of(int format, int d, bool bf) { return d == 128 ? 2 : (d == 64 ? 2 : 3) + (format == REC_MX4 && bf ? 1 : 0); }

struct ChosenArgs {
    Cache c;
    rec_query q;
    const int32_t *chosen;  // [batch][queries][kv_heads][width]
    int width, per, row_tiles, splits;
    Divider inner, by_heads, by_queries;  // by splits * row_tiles
    float *part_o;
    f32x2 *part_ml;
};

template <int FMT, int D, bool BF, int W>
__global__ __launch_bounds__(64 * W, waves_of(FMT, D, BF)) void chosen_kernel(ChosenArgs a)
{
    constexpr int DEPTH = depth_of(FMT, D);
    using T = std::conditional_t<BF, __bf16, _Float16>;
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    // Queries of one history may have chosen the same pages: neighbours run on one XCD, of which blocks take turns.
    const int all = (int)gridDim.x, xcd = (int)blockIdx.x & 7, block = xcd * (all >> 3) + min(xcd, all & 7) + ((int)blockIdx.x >> 3);
    const int pair = a.inner.of(block), part = block - pair * a.splits * a.row_tiles;
    const int at = a.by_heads.of(pair), kv = pair - at * a.c.kv_heads;  // query of all, kv head
    const int b = a.by_queries.of(at), query = at - b * a.q.queries;
    const int row_tile = a.splits == 1 ? part : part / a.splits, split = part - row_tile * a.splits;

    const int first_row = row_tile * ROWS, last_row = min(first_row + ROWS, a.per) - 1, row = min(first_row + c, last_row);
    const bool real = first_row + c <= last_row;
    const long long out = (long long)at * a.q.heads + kv * a.per + row, all_rows = (long long)a.q.batch * a.q.queries * a.q.heads;
    Query<D, BF> q;
    q.fetch(real ? static_cast<const char *>(a.q.dev_q) + 2 * (b * a.q.batch_stride + query * a.q.query_stride + (kv * a.per + row) * a.q.head_stride) : nullptr, g);

    const int shift = a.c.page_shift, most_tokens = a.q.table_width << shift;
    int len = a.q.dev_lengths[b];
    if (len < 0 || len > most_tokens) {
        if (threadIdx.x == 0 && kv == 0) report(a.c.fault, REC_FAULT_LENGTH, (unsigned long long)b);
        len = len < 0 ? 0 : most_tokens;
    }
    const int position = a.q.candidates ? len - 1 : len - a.q.queries + query;  // negative: sees nothing

    // Lane i has the i-th of 64 chosen pages: its number in the history and its page, or -1.  A tile's pages are all in one window.
    const int32_t *const table = a.q.dev_pages_of + b * a.q.table_stride;
    const int32_t *const chosen = a.chosen + (long long)pair * a.width;
    int window = -1, numbers = -1, pages_of = -1;
    auto look_up = [&](int at) {
        window = at;
        const int i = 64 * at + lane;
        numbers = i < a.width ? chosen[i] : -1;
        pages_of = -1;
        if ((unsigned)numbers < (unsigned)a.q.table_width && numbers << shift <= position) pages_of = table[numbers];
    };
    int tiles = 0;
    if (position >= 0) {
        look_up(0);
        int last = a.width;  // entries up to the last that is one, where that is known
        if (a.width <= 64) last = 64 - __builtin_clzll(__ballot(numbers != -1) | 1ull);
        tiles = (int)((((long long)last << shift) + TILE - 1) / TILE);
    }
    const int each = (tiles + a.splits - 1) / a.splits, begin = min(split * each, tiles), end = min(begin + each, tiles);

    f32x4 o[D / 16], l = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float m = neg_inf();
    unsigned saw = 0;  // not 0: a key has been seen

    if (begin + wave < end) {
        // Positive, so that masked scores stay at -inf.
        const float factor = a.q.scale == 0.0f ? 1.0f : __builtin_fabsf(a.q.scale) * 1.44269504088896341f;
        const int groups = 1 << (shift - 4), head_bytes = groups * group_bytes<FMT>(D);
        const unsigned char *first_page = a.c.pages + (long long)kv * head_bytes;
        const unsigned page_bytes = (unsigned)(a.c.kv_heads * head_bytes);
        const unsigned pages = (unsigned)min(a.c.num_pages, 1ll << 31);
        auto group_at = [&](int page, int token) {
            const bool ok = (unsigned)page < pages;  // else some group that is there: its tokens count for nothing
            const unsigned in_page = ok ? (unsigned)((token >> 4) & (groups - 1)) * group_bytes<FMT>(D) : 0u;
            return first_page + ((unsigned long long)(ok ? (unsigned)page : 0u) * page_bytes + in_page);
        };
        struct Slot {
            Tile<FMT, D> tile;
            int page, number;  // of this lane's group of values
        } slot[DEPTH];
        int page_next = -1, number_next = -1;
        auto load_keys = [&](Slot &s, int n) {  // and look up where its values are
            if (n >> shift != window) look_up(n >> shift);
            const int k_token = n * TILE + 16 * (c >> 2), v_token = n * TILE + 16 * g;
            s.tile.load_keys(group_at(__shfl(pages_of, k_token >> shift), k_token), c, g);
            page_next = __shfl(pages_of, v_token >> shift);
            number_next = __shfl(numbers, v_token >> shift);
        };
        auto load_values = [&](Slot &s, int n) {
            s.page = page_next;
            s.number = number_next;
            s.tile.load_values(group_at(s.page, n * TILE + 16 * g), c);
        };
        int n = begin + wave;
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (n + d * W < end) {
                load_keys(slot[d], n + d * W);
                load_values(slot[d], n + d * W);
            }
        q.convert(a.q.scale < 0.0f ? -1.0f : a.q.scale == 0.0f ? 0.0f : 1.0f, g);  // while the first tiles are on their way

        auto turn = [&](Slot &t, int n) {
            f32x4 s[4] = {scores<FMT, D, BF, 0>(t.tile, q, g), scores<FMT, D, BF, 1>(t.tile, q, g), scores<FMT, D, BF, 2>(t.tile, q, g), scores<FMT, D, BF, 3>(t.tile, q, g)};
            // Another tile's keys and values take the place of this one's as soon as that is used.
            const bool more = n + DEPTH * W < end;
            const bool there = (unsigned)t.page < pages;
            const int number = t.number, first = (number << shift) + ((n * TILE + 16 * g) & ((1 << shift) - 1));  // where the group's tokens stand
            if (more) load_keys(t, n + DEPTH * W);
            const bool whole = __all(there && first + 15 <= position);
            unsigned nan = 0;  // bit b: a NaN in block b of the values
            if (!whole) {
                unsigned seen = there ? below(position - first + 1) : 0u;
                if (!there && c == 0) {
                    if ((unsigned)number >= (unsigned)a.q.table_width) {
                        if (number != -1) report(a.c.fault, REC_FAULT_SLOT, (unsigned long long)(chosen - a.chosen + ((n * TILE + 16 * g) >> shift)));
                    } else if (number << shift <= position) {
                        report(a.c.fault, REC_FAULT_PAGE, (unsigned long long)b * (unsigned)a.q.table_width + (unsigned)number);
                    }
                }
                saw |= seen;
                nan = clear_values<FMT, D>(t.tile, seen, seen);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i & 3][i >> 2] = unless_hidden(s[i & 3][i >> 2], ~seen, i);
            } else {
                saw = 1;
            }
            // A lane's own scores tell whether some row's maximum has to move.
            float most = neg_inf();
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s[i & 3][i >> 2]);
            if (__any(most != neg_inf() && most * factor > m + (SLACK - ROOM))) {
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                most = most == neg_inf() ? most : most * factor;
                const float up = most > m + (SLACK - ROOM) ? fmaxf(m, most + ROOM) : m;
                const float down = m == up ? 1.0f : m == neg_inf() ? 0.0f : __builtin_amdgcn_exp2f(m - up);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) o[i] *= down;
                l *= down;
                m = up;
            }
            const float by = m == neg_inf() ? 0.0f : m;  // a row that sees nothing yet has weights of 2^(-inf)
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i & 3][i >> 2], factor, -by));

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
                for (int h = 0; h < 2; ++h) l = product(ones, w[k][h], l);
#pragma unroll
            for (int i = 0; i < D / BLOCK; ++i) {
                auto half = [&](auto at) {
                    u32x4 lo, hi;
                    value_operands<FMT, D, at()>(t.tile, i, lo, hi);
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) {
                        o[2 * i] = product(lo, w[k][at()], o[2 * i]);
                        o[2 * i + 1] = product(hi, w[k][at()], o[2 * i + 1]);
                    }
                };
                half(std::integral_constant<int, 0>());
                half(std::integral_constant<int, 1>());
            }
            if (nan)
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                    if (nan >> (i / 2) & 1u) o[i] += __builtin_nanf("");
            if (more) load_values(t, n + DEPTH * W);
        };
        for (; n < end; n += DEPTH * W) {
            turn(slot[0], n);
            if constexpr (DEPTH == 2)
                if (n + W < end) turn(slot[1], n + W);
        }
    }
    // All of a row's scores may be -inf, which is not the same as having none: the maximum tells.
    saw |= (unsigned)__shfl_xor((int)saw, 16);
    saw |= (unsigned)__shfl_xor((int)saw, 32);
    if (saw && m == neg_inf() && l[0] == 0.0f) m = LOWEST;

    if constexpr (W == 1) {
        if (!real) return;
        if (a.splits > 1) {
            if (g == 0) a.part_ml[split * all_rows + out] = f32x2{m, l[0]};
#pragma unroll
            for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4 *>(a.part_o + (split * all_rows + out) * D + 16 * i + 4 * g) = o[i];
            return;
        }
        const float by = inverse(l[0], m);
        typedef T tx4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
            *reinterpret_cast<tx4 *>(static_cast<T *>(a.q.dev_out) + out * D + 16 * i + 4 * g) = __builtin_convertvector(o[i] * by, tx4);
    } else {
        // Rows of all waves in LDS; a thread then joins eight columns of a row.
        constexpr int LD = D + 4;
        __shared__ float o_of[W][ROWS][LD];
        __shared__ f32x2 ml_of[W][ROWS];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4 *>(&o_of[wave][c][16 * i + 4 * g]) = o[i];
        if (g == 0) ml_of[wave][c] = f32x2{m, l[0]};
        __syncthreads();
        for (int i = threadIdx.x; i < ROWS * D / 8; i += 64 * W) {
            const int r = i / (D / 8), col = i % (D / 8) * 8;
            if (first_row + r > last_row) break;
            float most, sum;
            f32x4 x, y;
            join_waves(o_of, ml_of, r, col, most, sum, x, y);
            const long long to = (long long)at * a.q.heads + kv * a.per + first_row + r;
            if (a.splits > 1) {
                float *p = a.part_o + (split * all_rows + to) * D + col;
                *reinterpret_cast<f32x4 *>(p) = x;
                *reinterpret_cast<f32x4 *>(p + 4) = y;
                if (col == 0) a.part_ml[split * all_rows + to] = f32x2{most, sum};
            } else {
                typedef T tx8 __attribute__((ext_vector_type(8)));
                const float by = inverse(sum, most);
                x *= by;
                y *= by;
                const f32x8 z = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                *reinterpret_cast<tx8 *>(static_cast<T *>(a.q.dev_out) + to * D + col) = __builtin_convertvector(z, tx8);
            }
        }
    }
}

struct Plan {
    int per, row_tiles, waves, splits;
    long long pairs;  // of queries and kv heads
    long long rows;
};

Plan plan_of(const Cache &c, int format, int d, const rec_query &q, int count)
{
    Plan p;
    p.per = q.heads / c.kv_heads;
    p.row_tiles = (p.per + ROWS - 1) / ROWS;
    p.pairs = (long long)q.batch * q.queries * c.kv_heads;
    p.rows = (long long)q.batch * q.queries * q.heads;
    p.waves = p.splits = 1;
    const long long blocks = p.pairs * p.row_tiles, tiles = (((long long)count << c.page_shift) + TILE - 1) / TILE, room = 4ll * CUS * waves_of(format, d, q.dtype == REC_BF16);
    if (blocks == 0) return p;
    // As many waves of a block as are all at work at once (8 pairs of query and kv head with 256 tokens: 4.2 us with four
    // waves, 5.8 with one; 2560 pairs with 384: 15.7 with one, 16.5 with two, which take turns), then parts in blocks of their own, of two tiles a
    // wave at least (2 pairs with 8192 tokens: 10.2 us in 8 parts, 24.9 in one; 64 with 4096: 10.4 and 15.3).
    while (p.waves < 8 && 2 * p.waves <= tiles && 2 * p.waves * blocks <= room) p.waves *= 2;
    // Two parts take as long as one, and a launch and a workspace more (16 histories of 2048 tokens, 8 kv heads of 128: 13.8 us).
    const long long parts = std::min({room / (blocks * p.waves), tiles / (2 * p.waves), 64ll});
    p.splits = parts > 2 ? (int)parts : 1;
    return p;
}

template <int FMT, int D, bool BF>
hipError_t chosen_as(const ChosenArgs &a, const Plan &p, hipStream_t s)
{
    const dim3 grid((unsigned)(p.pairs * p.row_tiles * p.splits));
    if (p.waves == 8) hipLaunchKernelGGL((chosen_kernel<FMT, D, BF, 8>), grid, dim3(512), 0, s, a);
    else if (p.waves == 4) hipLaunchKernelGGL((chosen_kernel<FMT, D, BF, 4>), grid, dim3(256), 0, s, a);
    else if (p.waves == 2) hipLaunchKernelGGL((chosen_kernel<FMT, D, BF, 2>), grid, dim3(128), 0, s, a);
    else hipLaunchKernelGGL((chosen_kernel<FMT, D, BF, 1>), grid, dim3(64), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL((combine_kernel<D, BF>), dim3((unsigned)p.rows), dim3(256), 0, s, a.part_o, a.part_ml, p.splits, p.rows, a.q.dev_out);
    return hipGetLastError();
}

template <int FMT, int D>
hipError_t chosen_of(const ChosenArgs &a, const Plan &p, hipStream_t s)
{
    return a.q.dtype == REC_BF16 ? chosen_as<FMT, D, true>(a, p, s) : chosen_as<FMT, D, false>(a, p, s);
}

}  // namespace

long long chosen_threads(const Cache &c, int format, int d, const rec_query &q, int count)
{
    const Plan p = plan_of(c, format, d, q, count);
    return p.pairs * p.row_tiles * p.splits * 64 * p.waves;
}

size_t chosen_workspace(const Cache &c, int format, int d, const rec_query &q, int count)
{
    const Plan p = plan_of(c, format, d, q, count);
    return p.splits == 1 ? 0 : (size_t)p.splits * (size_t)p.rows * ((size_t)d * sizeof(float) + sizeof(f32x2));
}

hipError_t launch_chosen(const Cache &c, int format, int d, const rec_query &q, const int32_t *chosen, int count, void *workspace, hipStream_t s)
{
    const Plan p = plan_of(c, format, d, q, count);
    ChosenArgs a;
    a.c = c;
    a.q = q;
    a.chosen = chosen;
    a.width = count;
    a.per = p.per;
    a.row_tiles = p.row_tiles;
    a.splits = p.splits;
    a.inner = Divider(p.splits * p.row_tiles);
    a.by_heads = Divider(c.kv_heads);
    a.by_queries = Divider(q.queries);
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<f32x2 *>(a.part_o + (p.splits > 1 ? p.splits * p.rows * d : 0));
    if (format == REC_MX4)
        return d == 32 ? chosen_of<REC_MX4, 32>(a, p, s) : d == 64 ? chosen_of<REC_MX4, 64>(a, p, s) : chosen_of<REC_MX4, 128>(a, p, s);
    return d == 32 ? chosen_of<REC_MX8, 32>(a, p, s) : d == 64 ? chosen_of<REC_MX8, 64>(a, p, s) : chosen_of<REC_MX8, 128>(a, p, s);
}

}  // namespace hist
}  // namespace rec
