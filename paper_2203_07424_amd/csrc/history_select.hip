// Which pages of a long history a query attends to: mean keys of pages, their scores, and the highest of them.
//
// means_kernel: a lane has 32 columns of a token at a time, one scale's, and adds up its tokens'; lanes of different rows of 16 meet by
// swaps, which leave each a half of its columns, those of a row by rotations.  Bound by the keys' bytes: 8192 pages of 64 tokens,
// 8 heads of 128, mx4 62 us, 4.9 TB/s, with columns halved by shuffles, through the caches and with a page looked up a lane 79; mx8 124 us, 4.6 TB/s.
//
// score_pages(): products of queries and means, in 64 bits on the matrix instructions (16 x 16 x 4): which of two pages
// comes first must not hang on the order of a sum.  Operands are bf16 or fp16 numbers, so that their products are exact.
// A wave has 16 rows (the heads of as many queries as fit) and walks over tiles of 16 pages, whose numbers in 64 bits take as long as
// the products (a matrix instruction of 32 cycles for each four columns, with four rows or fewer one of 16).
//
// choose(): a score becomes a whole number of the same order; the one that `count` pages reach is found by halving the range of
// numbers it lies in and counting over all lanes.
//
// In one launch, 16 histories of 512 pages, 8 kv heads of 128 with 4 rows each: 14 us, of which 1.5 are the length and the pages one behind the
// other, 7 the scores (two waves of a SIMD, 4 tiles each, on half of the compute units: 128 blocks), 3.5 the choice (8 counts of 470 cycles); 256 x 4
// queries of 47 pages: 8.5 us.  In two launches, 16 histories of 4096 pages as above: 134 MB of means in 48 us, 2.8 TB/s.
#include <algorithm>

#include "history.h"

namespace rec {
namespace hist {
namespace {

typedef double f64;
typedef f64 f64x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned long long u64;

constexpr int THREADS = 256;

// ------------------------------------------------------------------ mean keys
// Lanes of a page's head.
__host__ __device__ inline int lanes_of(int page_shift, int d) { return (d / BLOCK) << page_shift < 64 ? (d / BLOCK) << page_shift : 64; }

template <int FMT, int D, int LANES>
__global__ __launch_bounds__(THREADS) void means_kernel(Cache c, const int32_t *which, int pages, Divider by_heads, u32x4 *means)
{
    constexpr int BLOCKS = D / BLOCK, CB = code_bytes<FMT>(D), WORDS = FMT == REC_MX4 ? 4 : 8, step = LANES / BLOCKS;
    const int lane = threadIdx.x & 63, in_item = lane % LANES, block = in_item % BLOCKS, first = in_item / BLOCKS;
    const int wave = (int)blockIdx.x * (THREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int item = wave * (64 / LANES) + (LANES == 64 ? 0 : lane / LANES);  // below 2^28, as the launch has fewer than 2^32 threads
    const int entry = by_heads.of(item), head = item - entry * c.kv_heads;
    long long page = -1;
    if (entry < pages) {
        page = which[entry];
        if (page < 0 || page >= c.num_pages) {
            if (page != -1 && head == 0 && in_item == 0) report(c.fault, REC_FAULT_PAGE, (u64)entry);
            page = -1;
        }
    }
    float sum[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) sum[i] = 0.0f;
    if (page >= 0) {
        const unsigned char *from = group_of<FMT>(c, D, page, 0, head);
        const int tokens = 1 << c.page_shift;
        const float share = __builtin_bit_cast(float, (unsigned)(127 - c.page_shift) << 23);  // means of the largest numbers do not overflow
#pragma unroll 4
        for (int t = first; t < tokens; t += step) {
            const unsigned char *group = from + (t >> 4) * group_bytes<FMT>(D);
            const unsigned char *codes = group + (t & 15) * CB + block * (CB / BLOCKS);
            const float scale = scale_of(group[2 * GROUP * CB + (t & 15) * BLOCKS + block]) * share;
            u32x4 w[WORDS / 4];
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(codes + 16 * i));
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                const unsigned word = w[i / 4][i % 4];
                auto add = [&](int column, f32x2 x) {
                    sum[column] = __builtin_fmaf(x[0], scale, sum[column]);
                    sum[column + 1] = __builtin_fmaf(x[1], scale, sum[column + 1]);
                };
                if constexpr (FMT == REC_MX4) {
                    add(8 * i, two_values<FMT, 0>(word));
                    add(8 * i + 2, two_values<FMT, 1>(word));
                    add(8 * i + 4, two_values<FMT, 2>(word));
                    add(8 * i + 6, two_values<FMT, 3>(word));
                } else {
                    add(4 * i, two_values<FMT, 0>(word));
                    add(4 * i + 2, two_values<FMT, 1>(word));
                }
            }
        }
    }
    // Sums of two columns: of one in even rows of 16 lanes, or in the lower half, of the other in odd ones or in the upper.
    auto two = [](float x, float y, auto half) {
        const unsigned a = __builtin_bit_cast(unsigned, x), b = __builtin_bit_cast(unsigned, y);
        if constexpr (half()) {
            const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
            return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
        } else {
            const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
            return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
        }
    };
    constexpr int AFTER_32 = LANES == 64 ? 16 : 32, COLUMNS = LANES == 16 ? 32 : AFTER_32 / 2;  // of a lane
    int column = 0;
    if constexpr (LANES == 64) {
        column += lane & 32 ? 16 : 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] = two(sum[i], sum[i + 16], std::true_type());
    }
    if constexpr (LANES >= 32) {
        column += lane & 16 ? COLUMNS : 0;
#pragma unroll
        for (int i = 0; i < COLUMNS; ++i) sum[i] = two(sum[i], sum[i + COLUMNS], std::false_type());
    }
    auto rotated = [](float x, auto by) {
        return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x120 + by(), 0xf, 0xf, false));
    };
#pragma unroll
    for (int i = 0; i < COLUMNS; ++i) {
        sum[i] = rotated(sum[i], std::integral_constant<int, 8>());
        sum[i] = rotated(sum[i], std::integral_constant<int, 4>());
        if constexpr (BLOCKS <= 2) sum[i] = rotated(sum[i], std::integral_constant<int, 2>());
        if constexpr (BLOCKS == 1) sum[i] = rotated(sum[i], std::integral_constant<int, 1>());
    }
    if (page >= 0 && lane % 16 < BLOCKS) {
        u32x4 *to = means + ((page * c.kv_heads + head) * D + block * BLOCK + column) / 8;
#pragma unroll
        for (int i = 0; i < COLUMNS; i += 8) {
            u32x4 w;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const bf16x2 mean = {(__bf16)sum[i + 2 * k], (__bf16)sum[i + 2 * k + 1]};
                w[k] = __builtin_bit_cast(unsigned, mean);
            }
            to[i / 8] = w;
        }
    }
}

// --------------------------------------------------------------------- scores
struct SelectArgs {
    Cache c;
    rec_query q;
    Select sel;
    int per;            // query heads of a kv head
    int at_once;        // queries of a wave
    int query_tiles;
    int walks, each;    // waves that share a row's pages, and tiles of 16 of each
    Divider by_walks, by_query_tiles, by_heads;
};

constexpr int PAGES = 16;  // of a tile

// Whole numbers of the same order; 0 is none's.
__device__ inline u64 key_of(f64 x)
{
    const u64 u = __builtin_bit_cast(u64, x + 0.0);  // one zero
    return u >> 63 ? ~u : u | 1ull << 63;
}

// What a key was made of.
__device__ inline f64 number_of(u64 key) { return __builtin_bit_cast(f64, key >> 63 ? key & ~(1ull << 63) : ~key); }

// A history's length, brought into its range.
__device__ inline int length_of(const SelectArgs &a, int b, bool tell)
{
    const int most = a.q.table_width << a.c.page_shift;
    int len = a.q.dev_lengths[b];
    if (len < 0 || len > most) {
        if (tell) report(a.c.fault, REC_FAULT_LENGTH, (u64)b);
        len = len < 0 ? 0 : most;
    }
    return len;
}

// Pages up to that of query i.
__device__ inline int pages_up_to(const SelectArgs &a, int len, int i)
{
    const int p = a.q.candidates ? len - 1 : len - a.q.queries + i;
    return p < 0 ? 0 : (p >> a.c.page_shift) + 1;
}

// What lane l + SHIFT of a row of 16 has (beyond it: 0).
template <int SHIFT>
__device__ inline f64 later_lane(f64 x)
{
    const u64 u = __builtin_bit_cast(u64, x);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, 0x100 + SHIFT, 0xf, 0xf, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), 0x100 + SHIFT, 0xf, 0xf, false);
    return __builtin_bit_cast(f64, (u64)hi << 32 | lo);
}

// Sums of lanes up to each.
__device__ inline unsigned sums_up_to(unsigned x)
{
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);  // by 1, 2, 4 and 8 lanes of a row of 16
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);  // a row's last to the next row
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);  // lane 31's to the upper half
    return x;
}

// f over all lanes, in each of them, without a trip through LDS or the scalar unit: what a wave that works by itself waits for most.
template <class F>
__device__ inline unsigned over_lanes(unsigned x, const F &f)
{
    x = f(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));   // lanes l ^ 1
    x = f(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));   // l ^ 2
    x = f(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, false));  // the other four of eight
    x = f(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, false));  // the other eight of a row
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = f((unsigned)r[0], (unsigned)r[1]);
    const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return f((unsigned)h[0], (unsigned)h[1]);
}
__device__ inline unsigned total(unsigned x)
{
    return over_lanes(x, [](unsigned a, unsigned b) { return a + b; });
}
__device__ inline unsigned largest(unsigned x)
{
    return over_lanes(x, [](unsigned a, unsigned b) { return max(a, b); });
}

// Tiles n, n + step ... before `end` of pages [from, to).
struct Walk {
    int from, to, n, step, end;
};

// Scores of a wave's 16 rows: the heads of `queries` queries from first_query on, of history b and kv head kv, over the pages of
// walk(), which is asked once the rows are on their way.  store(query - first_query, page, key).  FEW: at most four rows, on 4 x 4 x 4,
// which has four products of as many pages and takes half the time (the case above: 22 -> 14 us).
// Means are loaded a row after the other (a lane of the operand has a page of its own, and 16 lines at once for 16 lanes
// were what bounded this) and get to their lanes through `lds`, 16 rows of this wave's own, whose pieces are exchanged by the row's number.
template <int D, bool BF, bool FEW, class W, class F>
__device__ inline void score_pages(const SelectArgs &a, int b, int kv, int first_query, int queries, u32x4 *lds, const W &walk, const F &store)
{
    constexpr int N = D / 4;  // columns of a lane: pieces of eight, g, g + 4 ...
    constexpr int CH = D / 8, AT_ONCE = 64 / CH;  // pieces of a row, rows of a load
    constexpr int PER_LANE = FEW ? 1 : 4;  // results
    const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4, column = FEW ? lane & 3 : j;
    const int heads = min(a.per, 16), rows = queries * heads, row_tiles = (a.per + 15) / 16;
    const int row = min(column, rows - 1), query = row / heads;
    const char *mine = static_cast<const char *>(a.q.dev_q) + 2 * (b * a.q.batch_stride + (first_query + query) * a.q.query_stride + 8 * g);
    auto element = [](u32x4 w, int k, bool bf) -> f64 {
        if (bf) return (f64) __builtin_bit_cast(float, k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
        return (f64) __builtin_bit_cast(f16x8, w)[k];
    };
    u32x4 x[N / 8];
    auto load_rows = [&](int t) {
        const char *q = mine + 2 * (kv * a.per + min(16 * t + row - query * heads, a.per - 1)) * a.q.head_stride;
#pragma unroll
        for (int i = 0; i < N / 8; ++i) x[i] = *reinterpret_cast<const u32x4 *>(q + 64 * i);
    };
    load_rows(0);
    // Rows in 64 bits once, where registers for that do not cost a block its place (16 histories of 512 pages, 4 rows of 128 columns:
    // 15.7 -> 14.1 us; 2048 blocks of 16 rows of 64: 45 -> 51): a tile's conversions take as long as its products.
    constexpr bool ONCE = D == 32 || FEW;
    f64 y[N];
    auto convert_rows = [&]() {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            y[i] = element(x[i / 8], i % 8, BF);
            asm volatile("" : "+v"(y[i]));  // else it is converted where it is used
        }
    };

    const Walk w = walk();
    const int32_t *table = a.q.dev_pages_of + b * a.q.table_stride;
    const u32x4 *means = static_cast<const u32x4 *>(a.sel.means);
    // Four tiles at a time: lane group g has the pages of the g-th, and the means of all are on their way together.
    constexpr int BATCH = 4;
    auto look_up = [&](int n) {
        const int tile = n + g * w.step, number = tile * PAGES + j;
        int page = -1;
        if (tile < w.end && number >= w.from && number < w.to) {
            page = table[number];
            if (page < 0 || (long long)page >= a.c.num_pages) {
                report(a.c.fault, REC_FAULT_PAGE, (u64)b * (unsigned)a.q.table_width + (unsigned)number);
                page = -1;
            }
        }
        return page;
    };
    u32x4 loaded[BATCH][N / 8];
    auto load_means = [&](int pages) {
#pragma unroll
        for (int t = 0; t < BATCH; ++t)
#pragma unroll
            for (int i = 0; i < N / 8; ++i) {
                const int page = __shfl(pages, 16 * t + i * AT_ONCE + lane / CH);
                loaded[t][i] = u32x4{0u, 0u, 0u, 0u};
                if (page >= 0) loaded[t][i] = means[((long long)page * a.c.kv_heads + kv) * CH + lane % CH];
            }
    };
    auto exchange = [&](const u32x4 (&loaded)[N / 8], u32x4 (&raw)[N / 8]) {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const int row = i * AT_ONCE + lane / CH;
            lds[row * CH + (lane % CH ^ row % CH)] = loaded[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < N / 8; ++i) raw[i] = lds[j * CH + ((4 * i + g) ^ j % CH)];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    // known: bit i, page i of the tile is one.
    auto score = [&](const u32x4 (&raw)[N / 8], int n, unsigned known) {
        f64 best[PER_LANE];
#pragma unroll
        for (int r = 0; r < PER_LANE; ++r) best[r] = -__builtin_inf();
        for (int t = 0; t < row_tiles; ++t) {
            if (row_tiles > 1) {
                load_rows(t);
                if constexpr (ONCE) convert_rows();
            }
            // Two sums, which do not wait for each other.
            std::conditional_t<FEW, f64, f64x4> even = {}, odd = {};
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                u32x4 p = raw[i / 8], q = x[i / 8];
                if constexpr (D == 128) {  // converted where they are used: all at once they would take 128 registers
                    if (i % 8 == 0) __builtin_amdgcn_sched_barrier(0);
                    if constexpr (ONCE) asm volatile("" : "+v"(p));
                    else asm volatile("" : "+v"(p), "+v"(q));
                }
                const f64 m = element(p, i % 8, true), m1 = element(p, i % 8 + 1, true);
                if constexpr (FEW) {
                    even = __builtin_amdgcn_mfma_f64_4x4x4f64(m, ONCE ? y[i] : element(q, i % 8, BF), even, 0, 0, 0);
                    odd = __builtin_amdgcn_mfma_f64_4x4x4f64(m1, ONCE ? y[i + 1] : element(q, i % 8 + 1, BF), odd, 0, 0, 0);
                } else {
                    even = __builtin_amdgcn_mfma_f64_16x16x4f64(m, ONCE ? y[i] : element(q, i % 8, BF), even, 0, 0, 0);
                    odd = __builtin_amdgcn_mfma_f64_16x16x4f64(m1, ONCE ? y[i + 1] : element(q, i % 8 + 1, BF), odd, 0, 0, 0);
                }
            }
            // A product that is NaN counts for nothing.
            if constexpr (FEW) {
                best[0] = even + odd > best[0] ? even + odd : best[0];
            } else {
                even += odd;
#pragma unroll
                for (int r = 0; r < 4; ++r) best[r] = even[r] > best[r] ? even[r] : best[r];
            }
        }
#pragma unroll
        for (int r = 0; r < PER_LANE; ++r) {
            // The largest of `heads` neighbours from a query's first lane on: of twice as many each time, then of two such sets that overlap.
            f64 most = best[r];
            auto with = [&](f64 other) { most = other > most ? other : most; };
            if (heads > 1) with(later_lane<1>(most));
            if (heads > 3) with(later_lane<2>(most));
            if (heads > 7) with(later_lane<4>(most));
            if (heads > 15) with(later_lane<8>(most));
            if (heads & (heads - 1)) with(__shfl(most, lane + heads - (1 << (31 - __builtin_clz(heads)))));
            // Row r of a lane's four: page 4 r + g; of four products: page g of the lane's own.
            const int in_tile = FEW ? (lane >> 2 & 3) * 4 + g : 4 * r + g, number = n * PAGES + in_tile;
            if (column == query * heads && column < rows && number >= w.from && number < w.to) store(query, number, key_of(known >> in_tile & 1 ? most : -__builtin_inf()));
        }
    };
    int pages = look_up(w.n);
    if constexpr (ONCE) convert_rows();
    for (int n = w.n; n < w.end; n += BATCH * w.step) {
        load_means(pages);
        const u64 known = __ballot(pages >= 0);
        pages = look_up(n + BATCH * w.step);
#pragma unroll
        for (int t = 0; t < BATCH; ++t) {
            if (n + t * w.step >= w.end) break;
            u32x4 raw[N / 8];
            exchange(loaded[t], raw);
            score(raw, n + t * w.step, (unsigned)(known >> (16 * t)) & 0xffffu);
        }
    }
}

// Pages that some of a tile's queries may choose between those that all have.
__device__ inline Walk between(const SelectArgs &a, int there, int n, int step, int most)
{
    const int to = there - a.sel.last, from = a.sel.first;
    return {from, to, from / PAGES + n, step, min((to + PAGES - 1) / PAGES, most)};
}

template <int D, bool BF, bool FEW>
__global__ __launch_bounds__(THREADS) void score_kernel(SelectArgs a)
{
    const int wave = (int)(blockIdx.x * (THREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    const int rest = a.by_walks.of(wave), walk = wave - rest * a.walks;
    const int pair = a.by_query_tiles.of(rest), tile = rest - pair * a.query_tiles;
    const int b = a.by_heads.of(pair), kv = pair - b * a.c.kv_heads;
    if (b >= a.q.batch) return;
    const int first_query = tile * a.at_once, queries = min(a.at_once, a.q.queries - first_query);
    u64 *keys = a.sel.keys + (((long long)b * a.q.queries + first_query) * a.c.kv_heads + kv) * a.q.table_width;
    __shared__ u32x4 rows[THREADS / 64][PAGES * D / 8];
    score_pages<D, BF, FEW>(
        a, b, kv, first_query, queries, rows[threadIdx.x >> 6],
        [&]() {
            Walk w = between(a, pages_up_to(a, length_of(a, b, false), first_query + queries - 1), 0, 1, (walk + 1) * a.each);
            w.n = max(w.n, walk * a.each);
            return w;
        },
        [&](int query, int page, u64 key) { keys[(long long)query * a.c.kv_heads * a.q.table_width + page] = key; });
}

// --------------------------------------------------------------------- choice
// What the waves of a row tell each other.
template <int W>
struct Meeting {
    unsigned words[2][2][W];
};
template <>
struct Meeting<1> {};

// The choice of one row, by W waves with KEYS of its scores in each lane at a time: of the pages up to `there`, whose scores are keys[page - first].
// ONE: all scores are in lanes at once.
template <int W, int KEYS, bool ONE>
__device__ inline void choose_between(const SelectArgs &a, const u64 *keys, int n, int32_t *out, Meeting<W> &m)
{
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), thread = 64 * wave + lane;
    const int first = a.sel.first, want = a.sel.count - first - a.sel.last;
    constexpr int CHUNK = 64 * W * KEYS;
    u64 key[KEYS];  // neighbouring pages'; 0 behind the last
    auto load = [&](int from) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const int k = from + thread * KEYS + i;
            key[i] = 0;
            if (k < n) key[i] = keys[k];
        }
    };
    auto each_chunk = [&](auto f) {
        if constexpr (ONE) f(0);
        else
            for (int from = 0; from < n; from += CHUNK) {
                load(from);
                f(from);
            }
    };
    if constexpr (ONE) load(0);
    int turn = 0;
    // Two words of each wave to all.
    auto meet = [&](unsigned x, unsigned y, auto f) {
        if constexpr (W == 1) {
            f(0, x, y);
        } else {
            if (lane == 0) {
                m.words[turn][0][wave] = x;
                m.words[turn][1][wave] = y;
            }
            __syncthreads();
#pragma unroll
            for (int w = 0; w < W; ++w) f(w, m.words[turn][0][w], m.words[turn][1][w]);
            turn ^= 1;
        }
    };
    auto count = [&](auto is) {
        unsigned c = 0, all = 0;
        each_chunk([&](int) {
#pragma unroll
            for (int i = 0; i < KEYS; ++i) c += is(key[i]) ? 1u : 0u;
        });
        meet(total(c), 0, [&](int, unsigned x, unsigned) { all += x; });
        return (int)all;
    };

    // The score that `want` pages reach lies in [low, high].  Half way between as numbers, by their upper halves, which takes as many
    // counts as the scores nearest to it are apart; then, where that does not end, bit by bit.
    unsigned highest = 0, lowest = 0;  // the latter's complement
    each_chunk([&](int) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const unsigned top = (unsigned)(key[i] >> 32);
            highest = max(highest, top);
            lowest = max(lowest, top ? ~top : 0u);
        }
    });
    unsigned low = ~0u, high = 0;
    meet(largest(highest), largest(lowest), [&](int, unsigned x, unsigned y) {
        high = max(high, x);
        low = min(low, ~y);
    });
    int c = 0;
    for (int i = 0; i < 16; ++i) {
        asm("" : "+v"(low), "+v"(high));  // all the same, but kept from the scalar unit, which a vector instruction waits for
        // Of the numbers that these halves begin, the mean's; not a number, or none between them: half way as they are.
        const f64 mean = 0.5 * number_of((u64)low << 32) + 0.5 * number_of((u64)high << 32);
        unsigned middle = (unsigned)(key_of(mean) >> 32);
        if (!(middle > low && middle <= high)) middle = low + (high - low + 1) / 2;
        c = count([&](u64 k) { return (unsigned)(k >> 32) >= middle; });
        const bool enough = c >= want;
        low = enough ? middle : low;
        high = enough ? high : middle - 1;
        if (__any(c == want || high <= low)) break;
    }
    u64 bar = (u64)low << 32;
    if (__any(c != want)) {
        const u64 top = (u64)high << 32 | 0xffffffffu, differ = bar ^ top;
        int bit = 63 - __builtin_clzll(differ);
        bar &= bit == 63 ? 0ull : ~0ull << (bit + 1);
        for (; bit >= 0; --bit) {
            asm("" : "+v"(bar), "+v"(bit));
            const u64 higher = bar | 1ull << bit;
            c = count([&](u64 k) { return k >= higher; });
            bar = c >= want ? higher : bar;
            if (__any(c == want)) break;
        }
    }
    const int ties = want - count([&](u64 k) { return k > bar; });

    // In order: those above the bar, and of those at it the first.
    int taken = 0, tied = 0;  // before this chunk
    each_chunk([&](int from) {
        unsigned gt = 0, eq = 0;
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            gt += key[i] > bar ? 1u : 0u;
            eq += key[i] == bar ? 1u : 0u;
        }
        const unsigned gt_sum = sums_up_to(gt), eq_sum = sums_up_to(eq);
        int mine = taken + (int)(gt_sum - gt), mine_tied = tied + (int)(eq_sum - eq);
        if (!ONE || W > 1)
            meet((unsigned)__builtin_amdgcn_readlane((int)gt_sum, 63), (unsigned)__builtin_amdgcn_readlane((int)eq_sum, 63), [&](int w, unsigned x, unsigned y) {
                taken += (int)x;
                tied += (int)y;
                if (W > 1 && w < wave) {
                    mine += (int)x;
                    mine_tied += (int)y;
                }
            });
        if (gt + eq == 0) return;
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const bool over = key[i] > bar, at = key[i] == bar;
            if (over || (at && mine_tied < ties)) out[first + mine + min(mine_tied, ties)] = first + from + thread * KEYS + i;
            mine += over;
            mine_tied += at;
        }
    });
}

template <int W, int KEYS>
__device__ inline void choose(const SelectArgs &a, const u64 *keys, int there, int32_t *out, Meeting<W> &m)
{
    const int thread = W == 1 ? threadIdx.x & 63 : threadIdx.x, first = a.sel.first, last = a.sel.last;
    if (there <= a.sel.count) {  // all of them
        for (int i = thread; i < a.sel.count; i += 64 * W) out[i] = i < there ? i : -1;
        return;
    }
    for (int i = thread; i < first; i += 64 * W) out[i] = i;
    for (int i = thread; i < last; i += 64 * W) out[a.sel.count - last + i] = there - last + i;
    if (a.sel.count == first + last) return;
    const int n = there - first - last;
    if (W == 1 || n <= 64 * W * KEYS) choose_between<W, KEYS, true>(a, keys, n, out, m);
    else if constexpr (W > 1) choose_between<W, KEYS, false>(a, keys, n, out, m);
}

template <int W, int KEYS>
__global__ __launch_bounds__(64 * W) void choose_kernel(SelectArgs a)
{
    __shared__ Meeting<W> m;
    const long long row = blockIdx.x;
    const int at = a.by_heads.of((int)row), kv = (int)row - at * a.c.kv_heads;
    const int b = a.by_query_tiles.of(at), query = at - b * a.q.queries;
    const int len = length_of(a, b, threadIdx.x == 0 && kv == 0 && query == 0);
    choose<W, KEYS>(a, a.sel.keys + row * a.q.table_width + a.sel.first, pages_up_to(a, len, query), a.sel.chosen + row * a.sel.count, m);
}

// Keys that a block has in LDS beside its waves' rows, and that a wave has in its lanes.
constexpr int MOST_KEYS = 4096, WAVE_KEYS = 512;

// Both in one launch, where the scores of a block's queries fit LDS: all waves score, then each chooses for a query.
template <int D, bool BF, bool FEW, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void select_kernel(SelectArgs a)
{
    extern __shared__ u64 keys[];  // [at_once][table_width]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pair = a.by_query_tiles.of((int)blockIdx.x), tile = (int)blockIdx.x - pair * a.query_tiles;
    const int b = a.by_heads.of(pair), kv = pair - b * a.c.kv_heads;
    const int first_query = tile * a.at_once, queries = min(a.at_once, a.q.queries - first_query);
    int len = 0;
    __shared__ u32x4 rows[WAVES][PAGES * D / 8];
    score_pages<D, BF, FEW>(
        a, b, kv, first_query, queries, rows[wave],
        [&]() {
            len = length_of(a, b, threadIdx.x == 0 && kv == 0 && tile == 0);
            const int there = pages_up_to(a, len, first_query + queries - 1);
            return there > a.sel.count ? between(a, there, wave, WAVES, a.q.table_width) : Walk{0, 0, 0, 1, 0};  // else all are chosen
        },
        [&](int query, int page, u64 key) { keys[query * a.q.table_width + page] = key; });
    __syncthreads();
    Meeting<1> none;
    for (int i = wave; i < queries; i += WAVES) {
        const long long row = ((long long)b * a.q.queries + first_query + i) * a.c.kv_heads + kv;
        choose<1, WAVE_KEYS / 64>(a, keys + i * a.q.table_width + a.sel.first, pages_up_to(a, len, first_query + i), a.sel.chosen + row * a.sel.count, none);
    }
}

// Waves of a block that does both, by the tiles of a row: 512 pages (as above) 13.7 us with eight waves, 16.3 with four; 1024 queries of 47 pages
// 10.9 and 10.3.
int select_waves(const rec_query &q) { return q.table_width > 4 * PAGES ? 8 : 4; }

SelectArgs args_of(const Cache &c, int d, const rec_query &q)
{
    SelectArgs a;
    a.c = c;
    a.q = q;
    a.per = q.heads / c.kv_heads;
    const int tiles = (q.table_width + PAGES - 1) / PAGES;
    const auto with = [&](int at_once) {
        a.at_once = std::max(std::min({at_once, a.per >= 16 ? 1 : 16 / a.per, std::max(q.queries, 1)}), 1);
        a.query_tiles = (q.queries + a.at_once - 1) / a.at_once;
        return (long long)q.batch * c.kv_heads * a.query_tiles;  // blocks, or rows of waves
    };
    a.walks = 0;
    a.each = 0;
    // In one launch where a wave has all of a row's keys in its lanes and the block's tiles do not take longer than a second launch (4 histories,
    // 2 kv heads of 64, 4 rows: 512 pages 8.7 us in one, 9.2 in two, 1024 pages 19 and 10; 8 rows of 128: 256 pages 14.4 and 12.8, 512 pages
    // 22 and 12.7; 256 such histories: 256 pages 27 and 32, 512 pages 47 and 48.  8 kv heads of 128: 4 histories of 4 rows, 300 pages 10.8 and 11.4, 512
    // 14.9 and 14.4, 16 histories 11.4 and 16.2, 14.0 and 18.1, 64 histories 21 and 25, 26 and 34; 16 of 8 rows, 256 pages 15.6 and 15.8, 384 19.0 and 16.7,
    // 64 of them 26 and 32, 34 and 37).
    if (q.table_width <= WAVE_KEYS) {
        with(MOST_KEYS / std::max(q.table_width, 1));
        if (tiles * (d / 32) * (a.at_once * a.per <= 4 ? 1 : 2) <= 128) {
            a.by_walks = Divider(1);
            a.by_query_tiles = Divider(std::max(a.query_tiles, 1));
            a.by_heads = Divider(c.kv_heads);
            return a;
        }
    }
    const long long rows = with(16);
    // A tile a wave where there are few rows; several where that would be more waves than work at once, and all of a row's at most.
    a.each = (int)std::clamp((rows * tiles + 8191) / 8192, 1ll, std::max((long long)tiles, 1ll));
    a.walks = std::max((tiles + a.each - 1) / a.each, 1);
    a.by_walks = Divider(a.walks);
    a.by_query_tiles = Divider(std::max(a.query_tiles, 1));
    a.by_heads = Divider(c.kv_heads);
    return a;
}

// Waves that choose for a row, so that all of its keys are in lanes, up to 16384: 1500 pages 10.7 us with 4 waves of 8 keys a lane, 11.8 with 8, 18.0 with
// 16 of 16; 4096 pages 44 (read again for each count), 17.6 and 24.8; 16384 pages 104, 98 and 29.7.
int choose_waves(const rec_query &q) { return q.table_width <= 4 * 8 * 64 ? 4 : q.table_width <= 8 * 8 * 64 ? 8 : 16; }

long long score_blocks(const SelectArgs &a)
{
    return ((long long)a.q.batch * a.c.kv_heads * a.query_tiles * a.walks + THREADS / 64 - 1) / (THREADS / 64);  // none in one launch
}

long long means_blocks(const Cache &c, int d, int pages)
{
    const int per_block = THREADS / lanes_of(c.page_shift, d);
    return ((long long)pages * c.kv_heads + per_block - 1) / per_block;
}

template <int FMT, int D>
hipError_t means_as(const Cache &c, const int32_t *which, int pages, void *means, hipStream_t s)
{
    const dim3 grid((unsigned)means_blocks(c, D, pages)), block(THREADS);
    u32x4 *to = static_cast<u32x4 *>(means);
    const int lanes = lanes_of(c.page_shift, D);
    const Divider by_heads(c.kv_heads);
    if constexpr (D == 32)
        if (lanes == 16) {
            hipLaunchKernelGGL((means_kernel<FMT, D, 16>), grid, block, 0, s, c, which, pages, by_heads, to);
            return hipGetLastError();
        }
    if constexpr (D <= 64)
        if (lanes == 32) {
            hipLaunchKernelGGL((means_kernel<FMT, D, 32>), grid, block, 0, s, c, which, pages, by_heads, to);
            return hipGetLastError();
        }
    hipLaunchKernelGGL((means_kernel<FMT, D, 64>), grid, block, 0, s, c, which, pages, by_heads, to);
    return hipGetLastError();
}

template <int FMT>
hipError_t means_of(const Cache &c, int d, const int32_t *which, int pages, void *means, hipStream_t s)
{
    return d == 32 ? means_as<FMT, 32>(c, which, pages, means, s) : d == 64 ? means_as<FMT, 64>(c, which, pages, means, s) : means_as<FMT, 128>(c, which, pages, means, s);
}

template <int D, bool BF, bool FEW>
hipError_t scored_as(const SelectArgs &a, hipStream_t s)
{
    if (a.walks == 0) {
        const dim3 grid((unsigned)((long long)a.q.batch * a.c.kv_heads * a.query_tiles));
        const size_t lds = sizeof(u64) * a.at_once * std::max(a.q.table_width, 1);
        if (select_waves(a.q) == 8) hipLaunchKernelGGL((select_kernel<D, BF, FEW, 8>), grid, dim3(512), lds, s, a);
        else hipLaunchKernelGGL((select_kernel<D, BF, FEW, 4>), grid, dim3(256), lds, s, a);
    } else {
        hipLaunchKernelGGL((score_kernel<D, BF, FEW>), dim3((unsigned)score_blocks(a)), dim3(THREADS), 0, s, a);
    }
    return hipGetLastError();
}

// Scores, and in one launch the choice too.
template <int D>
hipError_t scored_of(const SelectArgs &a, hipStream_t s)
{
    const bool few = a.at_once * a.per <= 4;
    if (a.q.dtype == REC_BF16) return few ? scored_as<D, true, true>(a, s) : scored_as<D, true, false>(a, s);
    return few ? scored_as<D, false, true>(a, s) : scored_as<D, false, false>(a, s);
}

}  // namespace

long long means_threads(const Cache &c, int d, int pages) { return means_blocks(c, d, pages) * THREADS; }

hipError_t launch_means(const Cache &c, int format, int d, const int32_t *which, int pages, void *means, hipStream_t s)
{
    return format == REC_MX4 ? means_of<REC_MX4>(c, d, which, pages, means, s) : means_of<REC_MX8>(c, d, which, pages, means, s);
}

long long select_threads(const Cache &c, int d, const rec_query &q)
{
    const SelectArgs a = args_of(c, d, q);
    return a.walks ? std::max(score_blocks(a) * THREADS, (long long)q.batch * q.queries * c.kv_heads * 64 * choose_waves(q))
                   : (long long)q.batch * c.kv_heads * a.query_tiles * 64 * select_waves(q);
}

size_t select_workspace(const Cache &c, int d, const rec_query &q, int count)
{
    if (q.table_width <= count || args_of(c, d, q).walks == 0) return 0;
    return (size_t)q.batch * q.queries * c.kv_heads * (size_t)q.table_width * sizeof(u64);
}

void select_form(const Cache &c, int d, const rec_query &q, int count, int32_t (&form)[3])
{
    const SelectArgs a = args_of(c, d, q);
    form[0] = a.walks == 0 || q.table_width <= count ? 1 : 2;
    form[1] = a.at_once * std::min(a.per, 16);
    form[2] = a.walks == 0 ? 1 : choose_waves(q);
}

hipError_t launch_select(const Cache &c, int d, const rec_query &q, const Select &sel, hipStream_t s)
{
    SelectArgs a = args_of(c, d, q);
    a.sel = sel;
    if (a.walks == 0 || (q.table_width > sel.count && sel.count > sel.first + sel.last)) {
        const hipError_t e = d == 32 ? scored_of<32>(a, s) : d == 64 ? scored_of<64>(a, s) : scored_of<128>(a, s);
        if (e != hipSuccess || a.walks == 0) return e;
    }
    a.by_query_tiles = Divider(q.queries);
    const dim3 grid((unsigned)((long long)q.batch * q.queries * c.kv_heads));
    const int waves = choose_waves(q);
    if (waves == 4) hipLaunchKernelGGL((choose_kernel<4, 8>), grid, dim3(256), 0, s, a);
    else if (waves == 8) hipLaunchKernelGGL((choose_kernel<8, 8>), grid, dim3(512), 0, s, a);
    else hipLaunchKernelGGL((choose_kernel<16, 16>), grid, dim3(1024), 0, s, a);
    return hipGetLastError();
}

}  // namespace hist
}  // namespace rec
