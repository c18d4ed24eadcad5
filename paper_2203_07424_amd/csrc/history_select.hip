// Which pages of a long history a query attends to: mean keys of pages, their scores, and the highest of them.
//
// means_kernel: a lane has 32 columns of a token at a time, one scale's, and adds up its tokens'; lanes meet by
// exchanges that halve the columns of each.  Bound by the keys' bytes.
//
// score_kernel: products of queries and means, in 64 bits on the matrix instructions (16 x 16 x 4): which of two pages
// comes first must not hang on the order of a sum.  Operands are bf16 or fp16 numbers, so that their products are exact.
// A wave has 16 rows (the heads of as many queries as fit) and walks over tiles of 16 pages.
//
// choose_kernel: a score becomes a whole number of the same order; the one that `count` pages reach is found bit
// by bit, from the first in which the scores differ, by counting over a wave's ballots, and mostly long before the last bit.
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

template <int FMT, int D>
__global__ __launch_bounds__(THREADS) void means_kernel(Cache c, const int32_t *which, int pages, unsigned *means)
{
    constexpr int BLOCKS = D / BLOCK, CB = code_bytes<FMT>(D), WORDS = FMT == REC_MX4 ? 4 : 8;
    const int lane = threadIdx.x & 63, lanes = lanes_of(c.page_shift, D), in_item = lane & (lanes - 1);
    const int block = in_item % BLOCKS, first = in_item / BLOCKS, step = lanes / BLOCKS;
    const long long item = ((long long)blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6)) * (64 / lanes) + lane / lanes;
    const long long entry = item / c.kv_heads;
    const int head = (int)(item - entry * c.kv_heads);
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
            for (int i = 0; i < WORDS / 4; ++i) w[i] = *reinterpret_cast<const u32x4 *>(codes + 16 * i);
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
    // Lanes of the same columns, BLOCKS apart: with each exchange a lane keeps half of its columns, down to two.
    int column = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int half = 16 >> k;
        const bool upper = first >> k & 1;
        column += upper ? half : 0;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float keep = upper ? sum[half + i] : sum[i], give = upper ? sum[i] : sum[half + i];
            sum[i] = keep + __shfl_xor(give, BLOCKS << k);
        }
    }
#pragma unroll
    for (int k = 4; k < 6; ++k)
        if (BLOCKS << k < lanes) {
            const float x = __shfl_xor(sum[0], BLOCKS << k), y = __shfl_xor(sum[1], BLOCKS << k);
            sum[0] += x;
            sum[1] += y;
        }
    if (page >= 0 && first < 16) {
        const bf16x2 mean = {(__bf16)sum[0], (__bf16)sum[1]};
        means[((page * c.kv_heads + head) * D + block * BLOCK + column) / 2] = __builtin_bit_cast(unsigned, mean);
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

template <int D, bool BF>
__global__ __launch_bounds__(THREADS) void score_kernel(SelectArgs a)
{
    constexpr int N = D / 4;  // columns of a lane: group g has N g ...
    const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const int wave = (int)(blockIdx.x * (THREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    const int rest = a.by_walks.of(wave), walk = wave - rest * a.walks;
    const int pair = a.by_query_tiles.of(rest), tile = rest - pair * a.query_tiles;
    const int b = a.by_heads.of(pair), kv = pair - b * a.c.kv_heads;
    if (b >= a.q.batch) return;
    const int len = length_of(a, b, false);
    const int first_query = tile * a.at_once, queries = min(a.at_once, a.q.queries - first_query);
    // Pages that some of the queries may choose.
    const int to = pages_up_to(a, len, first_query + queries - 1) - a.sel.last, from = a.sel.first;
    int n = max(from / PAGES, walk * a.each);
    const int end = min((to + PAGES - 1) / PAGES, (walk + 1) * a.each);
    if (n >= end) return;

    const int32_t *table = a.q.dev_pages_of + b * a.q.table_stride;
    const u32x4 *means = static_cast<const u32x4 *>(a.sel.means);
    auto page_of = [&](int n) {
        const int number = n * PAGES + j;
        int page = -1;
        if (number >= from && number < to) {
            page = table[number];
            if ((long long)page >= a.c.num_pages || page < 0) {
                if (g == 0) report(a.c.fault, REC_FAULT_PAGE, (u64)b * (unsigned)a.q.table_width + (unsigned)number);
                page = -1;
            }
        }
        return page;
    };
    const int rows = a.per > 16 ? 16 : queries * a.per, row_tiles = (a.per + 15) / 16;
    for (; n < end; ++n) {
        const int page = page_of(n);
        u32x4 raw[N / 8];
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            raw[i] = u32x4{0u, 0u, 0u, 0u};
            if (page >= 0) raw[i] = means[(((long long)page * a.c.kv_heads + kv) * D + N * g) / 8 + i];
        }
        const unsigned there = (unsigned)__ballot(page >= 0) & 0xffffu;
        f64 best[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) best[r] = -__builtin_inf();
        for (int t = 0; t < row_tiles; ++t) {
            const int row = min(j, rows - 1), query = a.per > 16 ? 0 : row / a.per, head = min(a.per > 16 ? 16 * t + row : row - query * a.per, a.per - 1);
            const char *q = static_cast<const char *>(a.q.dev_q) + 2 * (b * a.q.batch_stride + (first_query + query) * a.q.query_stride + (kv * a.per + head) * a.q.head_stride + N * g);
            f64x4 s = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
            for (int i = 0; i < N / 8; ++i) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(q + 16 * i);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float m = __builtin_bit_cast(float, k & 1 ? raw[i][k / 2] & 0xffff0000u : raw[i][k / 2] << 16);
                    const float x = BF ? __builtin_bit_cast(float, k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16) : (float)__builtin_bit_cast(f16x8, w)[k];
                    s = __builtin_amdgcn_mfma_f64_16x16x4f64((f64)m, (f64)x, s, 0, 0, 0);
                }
            }
            // Row r of a lane's four: page 4 r + g.  A product that is NaN counts for nothing.
#pragma unroll
            for (int r = 0; r < 4; ++r) best[r] = s[r] > best[r] ? s[r] : best[r];
        }
        const int heads = min(a.per, 16);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            f64 most = best[r];
            for (int d = 1; d < heads; ++d) {
                const f64 other = __shfl(best[r], lane + d);
                most = other > most ? other : most;
            }
            const int in_tile = 4 * r + g, number = n * PAGES + in_tile;
            const int query = j / heads;
            if (j == query * heads && query < queries && number >= from && number < to)
                a.sel.keys[(((long long)b * a.q.queries + first_query + query) * a.c.kv_heads + kv) * a.q.table_width + number] =
                    key_of(there >> in_tile & 1 ? most : -__builtin_inf());
        }
    }
}

// --------------------------------------------------------------------- choice
// W waves a row, KEYS of its scores in each lane at a time.
template <int W, int KEYS>
__global__ __launch_bounds__(64 * W) void choose_kernel(SelectArgs a)
{
    __shared__ u64 ends[2][W];
    __shared__ unsigned counts[2][W];
    __shared__ unsigned before[2][KEYS][W];
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long row = blockIdx.x;
    const int at = a.by_heads.of((int)row), kv = (int)row - at * a.c.kv_heads;
    const int b = a.by_query_tiles.of(at), query = at - b * a.q.queries;
    const int len = length_of(a, b, threadIdx.x == 0 && kv == 0 && query == 0), there = pages_up_to(a, len, query);
    int32_t *out = a.sel.chosen + row * a.sel.count;
    if (there <= a.sel.count) {  // all of them
        for (int i = threadIdx.x; i < a.sel.count; i += 64 * W) out[i] = i < there ? i : -1;
        return;
    }
    const int first = a.sel.first, last = a.sel.last, want = a.sel.count - first - last, n = there - first - last;
    for (int i = threadIdx.x; i < first; i += 64 * W) out[i] = i;
    for (int i = threadIdx.x; i < last; i += 64 * W) out[a.sel.count - last + i] = there - last + i;
    if (want == 0) return;

    const u64 *keys = a.sel.keys + row * a.q.table_width + first;
    constexpr int CHUNK = 64 * W * KEYS;
    const bool one_chunk = n <= CHUNK;
    u64 key[KEYS];
    auto load = [&](int from) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const int k = from + (i * W + wave) * 64 + lane;
            key[i] = k < n ? keys[k] : 0;
        }
    };
    auto each_chunk = [&](auto f) {
        for (int from = 0; from < n; from += CHUNK) {
            if (!one_chunk) load(from);
            f(from);
        }
    };
    load(0);
    int turn = 0;
    auto sum = [&](unsigned x) {  // over the waves
        if constexpr (W == 1) return x;
        if (lane == 0) counts[turn][wave] = x;
        __syncthreads();
        unsigned s = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) s += counts[turn][w];
        turn ^= 1;
        return s;
    };
    auto count = [&](auto is) {
        unsigned c = 0;
        each_chunk([&](int) {
#pragma unroll
            for (int i = 0; i < KEYS; ++i) c += (unsigned)__popcll(__ballot(is(key[i])));
        });
        return sum(c);
    };

    // The bits that all scores begin with.
    u64 all = ~0ull, any = 0;
    each_chunk([&](int) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i)
            if (key[i]) {
                all &= key[i];
                any |= key[i];
            }
    });
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        all &= (u64)__shfl_xor((long long)all, d);
        any |= (u64)__shfl_xor((long long)any, d);
    }
    if constexpr (W > 1) {
        if (lane == 0) {
            ends[0][wave] = all;
            ends[1][wave] = any;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) {
            all &= ends[0][w];
            any |= ends[1][w];
        }
    }
    const u64 differ = all ^ any;
    u64 bar = all;  // the score that `want` pages reach
    if (differ) {
        int bit = 63 - __builtin_clzll(differ);
        bar &= bit == 63 ? 0ull : ~0ull << (bit + 1);
        for (; bit >= 0; --bit) {
            const u64 higher = bar | 1ull << bit;
            const unsigned c = count([&](u64 k) { return k >= higher; });
            if (c >= (unsigned)want) bar = higher;
            if (c == (unsigned)want) break;
        }
    }
    const int above = (int)count([&](u64 k) { return k > bar; }), ties = want - above;

    // In order: those above the bar, and of those at it the first.
    int taken = 0, tied = 0;  // before this chunk
    each_chunk([&](int from) {
        if constexpr (W > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
                const unsigned gt = (unsigned)__popcll(__ballot(key[i] > bar)), eq = (unsigned)__popcll(__ballot(key[i] == bar));
                if (lane == 0) {
                    before[0][i][wave] = gt;
                    before[1][i][wave] = eq;
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const u64 gt = __ballot(key[i] > bar), eq = __ballot(key[i] == bar);
            int mine_gt = taken, mine_eq = tied;
            if constexpr (W > 1) {
                for (int w = 0; w < wave; ++w) {
                    mine_gt += (int)before[0][i][w];
                    mine_eq += (int)before[1][i][w];
                }
                for (int w = 0; w < W; ++w) {
                    taken += (int)before[0][i][w];
                    tied += (int)before[1][i][w];
                }
            } else {
                taken += __popcll(gt);
                tied += __popcll(eq);
            }
            const u64 lower = (1ull << lane) - 1;
            const int eq_rank = mine_eq + __popcll(eq & lower);
            const bool tie = key[i] == bar && eq_rank < ties;
            if (key[i] > bar || tie) out[first + mine_gt + __popcll(gt & lower) + min(eq_rank, ties)] = first + from + (i * W + wave) * 64 + lane;
        }
    });
}

SelectArgs args_of(const Cache &c, const rec_query &q)
{
    SelectArgs a;
    a.c = c;
    a.q = q;
    a.per = q.heads / c.kv_heads;
    a.at_once = a.per >= 16 ? 1 : 16 / a.per;
    a.query_tiles = (q.queries + a.at_once - 1) / a.at_once;
    const long long rows = (long long)q.batch * c.kv_heads * a.query_tiles;
    const int tiles = (q.table_width + PAGES - 1) / PAGES;
    // A tile a wave where there are few rows; more where that would be more waves than work at once.
    a.each = (int)((rows * tiles + 8191) / 8192);
    a.each = a.each < 1 ? 1 : a.each;
    a.walks = (tiles + a.each - 1) / a.each;
    a.walks = a.walks < 1 ? 1 : a.walks;
    a.by_walks = Divider(a.walks);
    a.by_query_tiles = Divider(std::max(a.query_tiles, 1));
    a.by_heads = Divider(c.kv_heads);
    return a;
}

long long score_blocks(const SelectArgs &a)
{
    return ((long long)a.q.batch * a.c.kv_heads * a.query_tiles * a.walks + THREADS / 64 - 1) / (THREADS / 64);
}

long long means_blocks(const Cache &c, int d, int pages)
{
    const int per_block = THREADS / lanes_of(c.page_shift, d);
    return ((long long)pages * c.kv_heads + per_block - 1) / per_block;
}

template <int FMT>
hipError_t means_of(const Cache &c, int d, const int32_t *which, int pages, void *means, hipStream_t s)
{
    const dim3 grid((unsigned)means_blocks(c, d, pages)), block(THREADS);
    unsigned *to = static_cast<unsigned *>(means);
    if (d == 32) hipLaunchKernelGGL((means_kernel<FMT, 32>), grid, block, 0, s, c, which, pages, to);
    else if (d == 64) hipLaunchKernelGGL((means_kernel<FMT, 64>), grid, block, 0, s, c, which, pages, to);
    else hipLaunchKernelGGL((means_kernel<FMT, 128>), grid, block, 0, s, c, which, pages, to);
    return hipGetLastError();
}

template <int D>
hipError_t score_of(const SelectArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)score_blocks(a));
    if (a.q.dtype == REC_BF16) hipLaunchKernelGGL((score_kernel<D, true>), grid, dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((score_kernel<D, false>), grid, dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

}  // namespace

long long means_threads(const Cache &c, int d, int pages) { return means_blocks(c, d, pages) * THREADS; }

hipError_t launch_means(const Cache &c, int format, int d, const int32_t *which, int pages, void *means, hipStream_t s)
{
    return format == REC_MX4 ? means_of<REC_MX4>(c, d, which, pages, means, s) : means_of<REC_MX8>(c, d, which, pages, means, s);
}

long long select_threads(const Cache &c, const rec_query &q)
{
    return std::max(score_blocks(args_of(c, q)) * THREADS, (long long)q.batch * q.queries * c.kv_heads * 256);
}

size_t select_workspace(const Cache &c, const rec_query &q, int count)
{
    if (q.table_width <= count) return 0;  // all pages are chosen
    return (size_t)q.batch * q.queries * c.kv_heads * (size_t)q.table_width * sizeof(u64);
}

hipError_t launch_select(const Cache &c, int d, const rec_query &q, const Select &sel, hipStream_t s)
{
    SelectArgs a = args_of(c, q);
    a.sel = sel;
    if (q.table_width > sel.count && sel.count > sel.first + sel.last) {
        const hipError_t e = d == 32 ? score_of<32>(a, s) : d == 64 ? score_of<64>(a, s) : score_of<128>(a, s);
        if (e != hipSuccess) return e;
    }
    a.by_query_tiles = Divider(q.queries);
    const dim3 grid((unsigned)((long long)q.batch * q.queries * c.kv_heads));
    if (q.table_width <= 512) hipLaunchKernelGGL((choose_kernel<1, 8>), grid, dim3(64), 0, s, a);
    else hipLaunchKernelGGL((choose_kernel<4, 8>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace hist
}  // namespace rec
