// Attention of many histories that begin with the same tokens.
//
// prefix_kernel: the rows of all histories' queries against the shared tokens.  A wave has RT tiles of 16 rows of a kv
// head, so that a tile of 64 keys and values is loaded, and its values made into bf16, once for all of them; its four
// neighbours in the block have the same rows and other keys, and meet it in LDS.  The products are those of history_attend.hip.
// attend_kernel has what each history holds of its own, as parts, and combine_kernel joins both.
#include <algorithm>

#include "history_attend_body.h"

namespace rec {
namespace hist {
namespace {

constexpr int WAVES = 4;
constexpr int CUS = 256;
constexpr int MOST_PARTS = 64;  // of a row, of which half may be the prefix's

// Row tiles of a wave, and waves that a SIMD holds at once: as many as its registers hold.
__host__ __device__ constexpr int row_tiles_of(int d, bool bf) { return d == 128 ? 2 : d == 64 ? (bf ? 3 : 2) : 4; }
__host__ __device__ constexpr int waves_of(int format, int d, bool bf) { return d == 128 && !(format == REC_MX4 && bf) ? 1 : 2; }

struct SharedArgs {
    Cache c;
    rec_query q;
    Prefix prefix;
    int per;
    Divider by_per, by_queries, by_heads, by_splits;
    int rows;     // of a kv head: batch * queries * per
    int splits;
    float *part_o;
    f32x2 *part_ml;
};

template <int FMT, int D, bool BF>
__global__ __launch_bounds__(64 * WAVES, waves_of(FMT, D, BF)) void prefix_kernel(SharedArgs a)
{
    constexpr int RT = row_tiles_of(D, BF), W = WAVES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    // Blocks of one kv head are kv_heads apart: they have its keys and values in one L2 where that divides the XCDs.
    const int rest = a.by_heads.of((int)blockIdx.x), kv = (int)blockIdx.x - rest * a.c.kv_heads;
    const int row_block = a.by_splits.of(rest), split = rest - row_block * a.splits;
    const int first_row = row_block * RT * ROWS;

    const int shift = a.c.page_shift, most_tokens = a.prefix.width << shift;
    int len = *a.prefix.length;
    if (len < 0 || len > most_tokens) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report(a.c.fault, REC_FAULT_LENGTH, (unsigned long long)a.q.batch);
        len = len < 0 ? 0 : most_tokens;
    }
    const int tiles = (len + TILE - 1) / TILE, each = (tiles + a.splits - 1) / a.splits;
    const int begin = min(split * each, tiles), end = min(begin + each, tiles);

    f32x4 o[RT][D / 16], l[RT];
    float m[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[t][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        l[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        m[t] = neg_inf();
    }
    unsigned saw = 0;  // not 0: this wave's rows have seen a key

    if (begin + wave < end) {
        // Positive, so that masked scores stay at -inf.
        const float factor = a.q.scale == 0.0f ? 1.0f : __builtin_fabsf(a.q.scale) * 1.44269504088896341f;
        const float sign = a.q.scale < 0.0f ? -1.0f : a.q.scale == 0.0f ? 0.0f : 1.0f;
        const int groups = 1 << (shift - 4), head_bytes = groups * group_bytes<FMT>(D);
        const unsigned char *first_page = a.c.pages + (long long)kv * head_bytes;
        const unsigned page_bytes = (unsigned)(a.c.kv_heads * head_bytes);
        const unsigned pages = (unsigned)min(a.c.num_pages, 1ll << 31);
        auto page_of = [&](int token) {
            int page = -1;
            if (token < len) page = a.prefix.pages[token >> shift];
            return page;
        };
        auto group_at = [&](int page, int token) {
            const bool ok = (unsigned)page < pages;  // else some group that is there: its tokens count for nothing
            const unsigned in_page = ok ? (unsigned)((token >> 4) & (groups - 1)) * group_bytes<FMT>(D) : 0u;
            return first_page + ((unsigned long long)(ok ? (unsigned)page : 0u) * page_bytes + in_page);
        };
        int n = begin + wave;
        Tile<FMT, D> tile;
        int k_page = page_of(n * TILE + 16 * (c >> 2)), v_page = page_of(n * TILE + 16 * g);
        tile.load_keys(group_at(k_page, n * TILE + 16 * (c >> 2)), c, g);
        tile.load_values(group_at(v_page, n * TILE + 16 * g), c);
        Query<D, BF> q[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int row = first_row + t * ROWS + c;
            const char *from = nullptr;
            if (row < a.rows) {
                const int at = a.by_per.of(row), b = a.by_queries.of(at);
                from = static_cast<const char *>(a.q.dev_q) + 2 * (b * a.q.batch_stride + (at - b * a.q.queries) * a.q.query_stride + (kv * a.per + row - at * a.per) * a.q.head_stride);
            }
            q[t].fetch(from, g);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) q[t].convert(sign, g);
        k_page = page_of((n + W) * TILE + 16 * (c >> 2));
        int v_next = page_of((n + W) * TILE + 16 * g);
        for (;; n += W) {
            const bool more = n + W < end;
            const int key = n * TILE, key_next = (n + W) * TILE;
            const bool there = (unsigned)v_page < pages;
            const bool whole = key + TILE <= len && __all(there);
            unsigned seen = 0xffffu, nan = 0;
            if (!whole) {
                seen = below(len - key - 16 * g);
                if (!there) {
                    if (seen && c == 0)
                        report(a.c.fault, REC_FAULT_PAGE, (unsigned long long)a.q.batch * (unsigned)a.q.table_width + (unsigned)((key + 16 * g) >> shift));
                    seen = 0;
                }
                nan = clear_values<FMT, D>(tile, seen, seen);
            }
            saw |= seen;

            constexpr int TERMS = BF ? 1 : 2;
            u32x4 w[RT][TERMS][2];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                f32x4 s[4] = {scores<FMT, D, BF, 0>(tile, q[t], g), scores<FMT, D, BF, 1>(tile, q[t], g),
                              scores<FMT, D, BF, 2>(tile, q[t], g), scores<FMT, D, BF, 3>(tile, q[t], g)};
                if (!whole)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i & 3][i >> 2] = unless_hidden(s[i & 3][i >> 2], ~seen, i);
                float most = neg_inf();
#pragma unroll
                for (int i = 0; i < 16; ++i) most = fmaxf(most, s[i & 3][i >> 2]);
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                most = most == neg_inf() ? most : most * factor;
                if (__any(most > m[t] + (SLACK - ROOM))) {
                    const float up = fmaxf(m[t], most + ROOM);
                    if (__any(m[t] != neg_inf())) {
                        const float down = m[t] == up ? 1.0f : __builtin_amdgcn_exp2f(m[t] - up);
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) o[t][i] *= down;
                        l[t] *= down;
                    }
                    m[t] = up;
                }
                const float by = m[t] == neg_inf() ? 0.0f : m[t];
                float p[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i & 3][i >> 2], factor, -by));
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w[t][0][h][i] = pack(p[8 * h + 2 * i], p[8 * h + 2 * i + 1]);
                        if constexpr (TERMS == 2) {
                            const unsigned word = w[t][0][h][i];
                            w[t][1][h][i] = pack(p[8 * h + 2 * i] - __builtin_bit_cast(float, word << 16),
                                                 p[8 * h + 2 * i + 1] - __builtin_bit_cast(float, word & 0xffff0000u));
                        }
                    }
                const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
                for (int k = 0; k < TERMS; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h) l[t] = product(ones, w[t][k][h], l[t]);
            }
            if (more) tile.load_keys(group_at(k_page, key_next + 16 * (c >> 2)), c, g);
#pragma unroll
            for (int i = 0; i < D / BLOCK; ++i) {
                auto half = [&](auto at) {
                    u32x4 lo, hi;
                    value_operands<FMT, D, at()>(tile, i, lo, hi);
#pragma unroll
                    for (int t = 0; t < RT; ++t)
#pragma unroll
                        for (int k = 0; k < TERMS; ++k) {
                            o[t][2 * i] = product(lo, w[t][k][at()], o[t][2 * i]);
                            o[t][2 * i + 1] = product(hi, w[t][k][at()], o[t][2 * i + 1]);
                        }
                };
                half(std::integral_constant<int, 0>());
                half(std::integral_constant<int, 1>());
            }
            if (nan)
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int i = 0; i < D / 16; ++i)
                        if (nan >> (i / 2) & 1u) o[t][i] += __builtin_nanf("");
            if (!more) break;
            tile.load_values(group_at(v_next, key_next + 16 * g), c);
            v_page = v_next;
            if (n + 2 * W < end) {
                k_page = page_of(key_next + W * TILE + 16 * (c >> 2));
                v_next = page_of(key_next + W * TILE + 16 * g);
            }
        }
    }
    // All scores may be -inf, which is not the same as having none: the maximum tells.
    saw |= (unsigned)__shfl_xor((int)saw, 16);
    saw |= (unsigned)__shfl_xor((int)saw, 32);

    // Rows of all waves in LDS; a thread then joins eight columns of a row.
    constexpr int LD = D + 4;
    __shared__ float o_of[W][RT * ROWS][LD];
    __shared__ f32x2 ml_of[W][RT * ROWS];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if (saw && m[t] == neg_inf() && l[t][0] == 0.0f) m[t] = LOWEST;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4 *>(&o_of[wave][t * ROWS + c][16 * i + 4 * g]) = o[t][i];
        if (g == 0) ml_of[wave][t * ROWS + c] = f32x2{m[t], l[t][0]};
    }
    __syncthreads();
    for (int i = threadIdx.x; i < RT * ROWS * D / 8; i += 64 * W) {
        const int r = i / (D / 8), col = i % (D / 8) * 8, row = first_row + r;
        if (row >= a.rows) break;
        const int at = a.by_per.of(row), b = a.by_queries.of(at);
        // A query before its history's first token sees nothing.
        const bool sees = a.q.candidates || min(max(a.q.dev_lengths[b], 0), a.q.table_width << shift) - a.q.queries + at - b * a.q.queries >= 0;
        float most = neg_inf();
#pragma unroll
        for (int w = 0; w < W; ++w) most = fmaxf(most, ml_of[w][r][0]);
        float sum = 0.0f;
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = x;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const f32x2 ml = ml_of[w][r];
            const float by = ml[0] == neg_inf() ? (ml[1] == 0.0f ? 0.0f : ml[1]) : __builtin_amdgcn_exp2f(ml[0] - most);
            sum += ml[1] * by;
            x += *reinterpret_cast<const f32x4 *>(&o_of[w][r][col]) * by;
            y += *reinterpret_cast<const f32x4 *>(&o_of[w][r][col + 4]) * by;
        }
        if (!sees) {
            most = neg_inf();
            sum = 0.0f;
            x = y = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const long long all_rows = (long long)a.q.batch * a.q.queries * a.q.heads;
        const long long to = split * all_rows + (long long)at * a.q.heads + kv * a.per + (row - at * a.per);
        *reinterpret_cast<f32x4 *>(a.part_o + to * D + col) = x;
        *reinterpret_cast<f32x4 *>(a.part_o + to * D + col + 4) = y;
        if (col == 0) a.part_ml[to] = f32x2{most, sum};
    }
}

struct Plan {
    long long rows;  // of the whole call
    int blocks;      // of rows and kv heads
    int splits, own;
};

Plan plan_of(const Cache &c, int format, int d, const rec_query &q, int prefix_width)
{
    Plan p;
    p.rows = (long long)q.batch * q.queries * q.heads;
    const long long of_head = p.rows / c.kv_heads, rows = row_tiles_of(d, q.dtype == REC_BF16) * ROWS;
    p.blocks = (int)((of_head + rows - 1) / rows * c.kv_heads);
    p.own = own_parts(c, format, d, q, MOST_PARTS / 2);
    const long long tiles = (((long long)prefix_width << c.page_shift) + TILE - 1) / TILE;
    // As many parts of the prefix as are all at work at once, of two tiles a wave at least.
    p.splits = (int)std::max(1ll, std::min({(long long)waves_of(format, d, q.dtype == REC_BF16) * CUS / std::max(p.blocks, 1), tiles / (2 * WAVES), (long long)MOST_PARTS / 2}));
    return p;
}

template <int FMT, int D, bool BF>
hipError_t shared_as(const SharedArgs &a, const Plan &p, int format, hipStream_t s)
{
    hipLaunchKernelGGL((prefix_kernel<FMT, D, BF>), dim3((unsigned)(p.blocks * p.splits)), dim3(64 * WAVES), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const Parts own = {a.part_o + p.splits * p.rows * D, reinterpret_cast<float *>(a.part_ml + p.splits * p.rows)};
    e = launch_own_parts(a.c, format, D, a.q, MOST_PARTS / 2, own, s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((combine_kernel<D, BF>), dim3((unsigned)p.rows), dim3(256), 0, s, a.part_o, a.part_ml, p.splits + p.own, p.rows, a.q.dev_out);
    return hipGetLastError();
}

template <int FMT, int D>
hipError_t shared_of(const SharedArgs &a, const Plan &p, int format, hipStream_t s)
{
    return a.q.dtype == REC_BF16 ? shared_as<FMT, D, true>(a, p, format, s) : shared_as<FMT, D, false>(a, p, format, s);
}

}  // namespace

long long shared_threads(const Cache &c, int format, int d, const rec_query &q, int prefix_width)
{
    const Plan p = plan_of(c, format, d, q, prefix_width);
    return std::max((long long)p.blocks * p.splits * 64 * WAVES, p.rows * 256);
}

size_t shared_workspace(const Cache &c, int format, int d, const rec_query &q, int prefix_width)
{
    if (q.batch == 0 || q.queries == 0) return 0;
    const Plan p = plan_of(c, format, d, q, prefix_width);
    return (size_t)(p.splits + p.own) * (size_t)p.rows * ((size_t)d * sizeof(float) + sizeof(f32x2));
}

hipError_t launch_shared(const Cache &c, int format, int d, const rec_query &q, const Prefix &prefix, void *workspace, hipStream_t s)
{
    const Plan p = plan_of(c, format, d, q, prefix.width);
    SharedArgs a;
    a.c = c;
    a.q = q;
    a.prefix = prefix;
    a.per = q.heads / c.kv_heads;
    a.by_per = Divider(a.per);
    a.by_queries = Divider(q.queries);
    a.by_heads = Divider(c.kv_heads);
    a.by_splits = Divider(p.splits);
    a.rows = (int)(p.rows / c.kv_heads);
    a.splits = p.splits;
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<f32x2 *>(a.part_o + (p.splits + p.own) * p.rows * d);
    if (format == REC_MX4)
        return d == 32 ? shared_of<REC_MX4, 32>(a, p, format, s) : d == 64 ? shared_of<REC_MX4, 64>(a, p, format, s) : shared_of<REC_MX4, 128>(a, p, format, s);
    return d == 32 ? shared_of<REC_MX8, 32>(a, p, format, s) : d == 64 ? shared_of<REC_MX8, 64>(a, p, format, s) : shared_of<REC_MX8, 128>(a, p, format, s);
}

}  // namespace hist
}  // namespace rec
