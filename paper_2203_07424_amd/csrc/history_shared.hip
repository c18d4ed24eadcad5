// Attention of many histories that begin with the same tokens.
//
// The rows of all histories' queries against the shared tokens are large products, those of history_attend.hip.
// wide_kernel: a block has 128 rows of a kv head or more, four waves of RT tiles of 16, and two such groups of waves, which
// have every other tile of keys and meet in LDS in the end.  The four waves of a group share a tile's values: each makes a
// quarter of them into bf16, in the order of the operands, in LDS, while the tile before is multiplied.  Keys go into the products as they are stored.
// Bound by matrix instructions and exponentials, which the two groups' halves of a turn overlap in part: 1024 rows of each of 8 kv heads of 128, mx4, before
// 8192 tokens 46 us, 750 TFLOP/s of the plain products.  (With the launch behind it 59 us in bf16, mx8 too, and 79 in fp16, 81 in mx8: twice the weights' products, half
// as many row tiles.)
// narrow_kernel: one tile of 16 rows, whose keys four waves share.
//
// What that leaves are parts of the rows' sums; attend_kernel joins them with what each history holds of its own.  Where there is little to
// read, attend_kernel walks over the prefix and the history by itself.
#include <algorithm>

#include "history_attend_body.h"
#include "rec_probe.h"

namespace rec {
namespace hist {
namespace {

constexpr int CUS = 256;

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
__global__ __launch_bounds__(256) void narrow_kernel(SharedArgs a)
{
    constexpr int RT = 1, W = 4;
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
        float most, sum;
        f32x4 x, y;
        join_waves(o_of, ml_of, r, col, most, sum, x, y);
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

// Row tiles of a wave: as many as 256 registers hold.
__host__ __device__ constexpr int row_tiles_of(int d, bool bf)
{
    return d == 32 ? (bf ? 4 : 3) : d == 64 ? (bf ? 3 : 2) : bf ? 2 : 1;
}
constexpr int ROW_WAVES = 4, GROUPS = 2;  // of a block

// The block of 32 columns of which wave w of a group makes half h of a tile's values, or -1: each is made once.
__host__ __device__ constexpr int block_made(int d, int w, int h) { return d == 128 ? w : (w & 1) == h && w / 2 < d / BLOCK ? w / 2 : -1; }
constexpr bool each_made_once(int d)
{
    for (int i = 0; i < d / BLOCK; ++i)
        for (int h = 0; h < 2; ++h) {
            int by = 0;
            for (int w = 0; w < ROW_WAVES; ++w) by += block_made(d, w, h) == i ? 1 : 0;
            if (by != 1) return false;
        }
    return true;
}
static_assert(each_made_once(32) && each_made_once(64) && each_made_once(128), "two waves would store to one place");

// This lane's codes and scales of one block of 32 columns of a tile's values.
template <int FMT, int D>
__device__ inline void load_block(Tile<FMT, 32> &t, const unsigned char *vg, int b, int c)
{
    constexpr int CB = code_bytes<FMT>(D), WIDE = Tile<FMT, 32>::WIDE;
    const unsigned char *vp = vg + GROUP * CB + (b * GROUP + c) * GROUP * WIDE;
#pragma unroll
    for (int w = 0; w < WIDE; ++w) t.v[0][w] = *reinterpret_cast<const u32x4 *>(vp + 16 * w);
    t.vs[0] = *reinterpret_cast<const u32x4 *>(vg + 2 * GROUP * CB + GROUP * (D / BLOCK) + b * GROUP);
}

// Tokens that are not `seen` become zeros, whatever their bytes are.
template <int FMT>
__device__ inline void hide(Tile<FMT, 32> &t, unsigned seen)
{
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const unsigned keep = bytes_of(seen >> (4 * x) & 15u);
        t.vs[0][x] &= keep;
        if constexpr (FMT == REC_MX8) {
            t.v[0][x >> 1][2 * (x & 1)] &= __builtin_amdgcn_perm(keep, keep, 0x01010000u);
            t.v[0][x >> 1][2 * (x & 1) + 1] &= __builtin_amdgcn_perm(keep, keep, 0x03030202u);
        }
    }
}

// Pieces of 16 bytes of a key's codes.  A lane has one or two of each of its four keys: the one that it begins with.
template <int FMT, int D>
constexpr int PIECES = code_bytes<FMT>(D) / 16;
template <int FMT, int D>
__device__ inline int piece_of(int g) { return PIECES<FMT, D> == 1 ? 0 : PIECES<FMT, D> == 2 ? g & 1 : g; }

// Step i of the x-th product of scores(), of a key's pieces and its scales `ks`, so that steps which wait for each other can be apart.
template <int FMT, int D, bool BF, int X>
__device__ inline void add_scores(f32x4 &r, const u32x4 (&k)[PIECES<FMT, D> == 8 ? 2 : 1], const unsigned (&ks)[D / BLOCK], const Query<D, BF> &q, int i, int g)
{
    constexpr int SW = D / BLOCK, AT = D == 32 ? X : D == 64 ? 2 * (X & 1) : 0;
    i32x8 a;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        a[j] = (int)k[0][j];
        a[4 + j] = (int)k[PIECES<FMT, D> == 8 ? 1 : 0][j];
    }
    const int s = (int)(D == 32 ? ks[0] : D == 64 ? ks[(X >> 1) % SW] >> (8 * (g & 1)) : ks[X % SW] >> (8 * g));
    if (i == 0) r = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    r = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.b[i], r, FMT == REC_MX4 ? 4 : 0, 0, AT, s, 0, q.scale[i]);
}

template <int FMT, int D, bool BF>
__global__ __launch_bounds__(64 * ROW_WAVES * GROUPS, 2) void wide_kernel(SharedArgs a)
{
    constexpr int RT = row_tiles_of(D, BF), TERMS = BF ? 1 : 2;
    constexpr int VALUES = D * TILE / 8, SUMS = ROW_WAVES * RT * (D / 16) * 64;  // 16 bytes each: a tile's values, a group's sums
    __shared__ u32x4 lds[GROUPS * 2 * VALUES > SUMS ? GROUPS * 2 * VALUES : SUMS];
    __shared__ u32x4 keys_of[GROUPS][PIECES<FMT, D>][4][16];  // a tile's keys: piece, product, lane % 16
    __shared__ f32x2 ml_of[ROW_WAVES][RT][ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int part_of_rows = wave % ROW_WAVES, group = wave / ROW_WAVES;
    // Blocks of one kv head are kv_heads apart: they have its keys and values in one L2 where that divides the XCDs.
    const int rest = a.by_heads.of((int)blockIdx.x), kv = (int)blockIdx.x - rest * a.c.kv_heads;
    const int row_block = a.by_splits.of(rest), split = rest - row_block * a.splits;
    const int first_row = (row_block * ROW_WAVES + part_of_rows) * RT * ROWS;

    // The rows' queries, on their way while the prefix is looked up, and which of them see it: a query before its history's first
    // token sees nothing.
    const int shift = a.c.page_shift;
    Query<D, BF> q[RT];
    unsigned sees = 0;
    long long to[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int row = first_row + t * ROWS + c;
        const char *from = nullptr;
        to[t] = -1;
        if (row < a.rows) {
            const int at = a.by_per.of(row), b = a.by_queries.of(at), i = at - b * a.q.queries, head = kv * a.per + row - at * a.per;
            from = static_cast<const char *>(a.q.dev_q) + 2 * (b * a.q.batch_stride + i * a.q.query_stride + head * a.q.head_stride);
            to[t] = (long long)at * a.q.heads + head;
            sees |= a.q.candidates || min(max(a.q.dev_lengths[b], 0), a.q.table_width << shift) - a.q.queries + i >= 0 ? 1u << t : 0u;
        }
        q[t].fetch(from, g);
    }
    const int most_tokens = a.prefix.width << shift;
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

    // Positive, so that masked scores stay at -inf.
    const float factor = a.q.scale == 0.0f ? 1.0f : __builtin_fabsf(a.q.scale) * 1.44269504088896341f;
    const int groups = 1 << (shift - 4), head_bytes = groups * group_bytes<FMT>(D);
    const unsigned char *first_page = a.c.pages + (long long)kv * head_bytes;
    const unsigned page_bytes = (unsigned)(a.c.kv_heads * head_bytes);
    const unsigned pages = (unsigned)min(a.c.num_pages, 1ll << 31);
    auto page_of = [&](int n, int in_tile) {
        int page = -1;
        if (n < end && n * TILE + in_tile < len) page = a.prefix.pages[(n * TILE + in_tile) >> shift];
        return page;
    };
    auto group_at = [&](int page, int token) {
        const bool ok = (unsigned)page < pages;  // else some group that is there: its tokens count for nothing
        const unsigned in_page = ok ? (unsigned)((token >> 4) & (groups - 1)) * group_bytes<FMT>(D) : 0u;
        return first_page + ((unsigned long long)(ok ? (unsigned)page : 0u) * page_bytes + in_page);
    };
    // Bit t: token t of this lane's group of tile n is seen.
    auto seen_of = [&](int n, int page) { return (unsigned)page < pages ? below(len - n * TILE - 16 * g) : 0u; };

    // What this wave makes of a tile's values: both halves of a block of 32 columns, one of them, or (of one block) nothing.
    const int first_half = block_made(D, part_of_rows, 0), second_half = block_made(D, part_of_rows, 1), block = max(first_half, second_half);
    u32x4 *const values = lds + group * 2 * VALUES;
    Tile<FMT, 32> made;
    auto load_made = [&](int n, int page) {
        if (block >= 0) load_block<FMT, D>(made, group_at(page, n * TILE + 16 * g), block, c);
    };
    auto make = [&](unsigned seen, bool whole, int buffer) {
        if (block < 0) return;
        if (!whole) hide<FMT>(made, seen);
        u32x4 *to = values + buffer * VALUES + block * 4 * 64 + lane;
        auto half = [&](auto h) {
            u32x4 lo, hi;
            value_operands<FMT, 32, h()>(made, 0, lo, hi);
            to[(2 * h()) * 64] = lo;
            to[(2 * h() + 1) * 64] = hi;
        };
        if (first_half >= 0) half(std::integral_constant<int, 0>());
        if (second_half >= 0) half(std::integral_constant<int, 1>());
    };

    int n = begin + group;
    int page = page_of(n, 16 * g), page_next = page_of(n + GROUPS, 16 * g);
    int k_page = page_of(n, 16 * (c >> 2)), k_next = page_of(n + GROUPS, 16 * (c >> 2));
    // Keys' codes go to LDS as the products take them, once for the group; their scales are each wave's own.
    unsigned ks[D / BLOCK];
    auto load_keys = [&](int n, int page) {
        constexpr int CB = code_bytes<FMT>(D), SW = D / BLOCK;
        const unsigned char *from = group_at(page, n * TILE + 16 * (c >> 2));
        const unsigned char *row = from + (4 * (c & 3) + g) * CB;  // lane group g brings the g-th product's
#pragma unroll
        for (int i = 0; i < (PIECES<FMT, D> + ROW_WAVES - 1) / ROW_WAVES; ++i) {
            const int piece = i * ROW_WAVES + part_of_rows;
            if (PIECES<FMT, D> % ROW_WAVES == 0 || piece < PIECES<FMT, D>)
                __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void *)(row + 16 * piece),
                                                 (__attribute__((address_space(3))) void *)&keys_of[group][piece][0][0], 16, 0, 0);
        }
        const unsigned char *scales = from + 2 * GROUP * CB + 4 * (c & 3) * SW;
        if constexpr (SW == 1) {
            ks[0] = *reinterpret_cast<const unsigned *>(scales);
        } else if constexpr (SW == 2) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(scales);
            ks[0] = x[0];
            ks[1] = x[1];
        } else {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(scales);
#pragma unroll
            for (int j = 0; j < 4; ++j) ks[j] = x[j];
        }
    };
    load_made(n, page);
    load_keys(n, k_page);
#pragma unroll
    for (int t = 0; t < RT; ++t) q[t].convert(a.q.scale < 0.0f ? -1.0f : a.q.scale == 0.0f ? 0.0f : 1.0f, g);
    // The weights of the tile before, and its values: none yet.
    u32x4 w[RT][TERMS][2];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int k = 0; k < TERMS; ++k) w[t][k][0] = w[t][k][1] = u32x4{0u, 0u, 0u, 0u};
    for (int i = part_of_rows * 64 + lane; i < VALUES; i += 64 * ROW_WAVES) values[VALUES + i] = u32x4{0u, 0u, 0u, 0u};
    // Loads that go to LDS are not among those that a barrier waits for.
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();

    // o += values of a buffer times w, and l the weights.  A block's operands are on their way while the one before is multiplied.
    u32x4 operand[2][4];
    auto fetch = [&](int buffer, int i) {
#pragma unroll
        for (int x = 0; x < 4; ++x) operand[i & 1][x] = values[buffer * VALUES + (4 * i + x) * 64 + lane];
    };
    auto multiply = [&](int buffer) {  // block 0 is fetched
        const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
        for (int i = 0; i < D / BLOCK; ++i) {
            if (i + 1 < D / BLOCK) fetch(buffer, i + 1);
            __builtin_amdgcn_sched_barrier(0);
            if (i == 0)
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int k = 0; k < TERMS; ++k)
#pragma unroll
                        for (int h = 0; h < 2; ++h) l[t] = product(ones, w[t][k][h], l[t]);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int k = 0; k < TERMS; ++k)
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        o[t][2 * i] = product(operand[i & 1][2 * h], w[t][k][h], o[t][2 * i]);
                        o[t][2 * i + 1] = product(operand[i & 1][2 * h + 1], w[t][k][h], o[t][2 * i + 1]);
                    }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // A turn has two halves.  In the first a group scores its next tile and multiplies the one before it, whose weights are
    // ready, with all matrix instructions one after the other; in the second it makes weights of the scores.  The two groups, of each of
    // which a SIMD has a wave, are half a turn apart, so that one's matrix instructions run beside the other's exponentials.
    const int turns = (end - begin + GROUPS - 1) / GROUPS;
    fetch(1, 0);
    if (group == 1) __syncthreads();
    for (int turn = 0; turn < turns; ++turn, n += GROUPS) {
        const unsigned seen = seen_of(n, page);
        const bool whole = __all(seen == 0xffffu);
        saw |= seen;
        __builtin_amdgcn_s_setprio(1);  // before the other group's exponentials
        u32x4 k[4][PIECES<FMT, D> == 8 ? 2 : 1];
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int j = 0; j < (PIECES<FMT, D> == 8 ? 2 : 1); ++j) k[x][j] = keys_of[group][piece_of<FMT, D>(g) + 4 * j][x][c];
        multiply((turn + 1) & 1);
        f32x4 s[RT][4];
#pragma unroll
        for (int i = 0; i < Query<D, BF>::STEPS; ++i)
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                add_scores<FMT, D, BF, 0>(s[t][0], k[0], ks, q[t], i, g);
                add_scores<FMT, D, BF, 1>(s[t][1], k[1], ks, q[t], i, g);
                add_scores<FMT, D, BF, 2>(s[t][2], k[2], ks, q[t], i, g);
                add_scores<FMT, D, BF, 3>(s[t][3], k[3], ks, q[t], i, g);
            }
        make(seen, whole, turn & 1);
#pragma unroll
        for (int t = 0; t < RT; ++t) asm volatile("" : "+v"(s[t][0]), "+v"(s[t][1]), "+v"(s[t][2]), "+v"(s[t][3]));  // else they are worked out where they are used
        __builtin_amdgcn_s_setprio(0);
        __syncthreads();

        // The next tile's codes, and where the one's behind it are.
        load_keys(n + GROUPS, k_next);
        load_made(n + GROUPS, page_next);
        const int page_now = page;
        page = page_next;
        page_next = page_of(n + 2 * GROUPS, 16 * g);
        k_next = page_of(n + 2 * GROUPS, 16 * (c >> 2));
        if (!whole) {
            if ((unsigned)page_now >= pages && n < end && n * TILE + 16 * g < len && c == 0)
                report(a.c.fault, REC_FAULT_PAGE, (unsigned long long)a.q.batch * (unsigned)a.q.table_width + (unsigned)((n * TILE + 16 * g) >> shift));
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[t][i & 3][i >> 2] = unless_hidden(s[t][i & 3][i >> 2], ~seen, i);
        }
        // A lane's own scores tell whether some row's maximum has to move.
        float most[RT];
        bool moves = false;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            most[t] = neg_inf();
#pragma unroll
            for (int i = 0; i < 16; ++i) most[t] = fmaxf(most[t], s[t][i & 3][i >> 2]);
            moves |= most[t] != neg_inf() && most[t] * factor > m[t] + (SLACK - ROOM);
        }
        if (__any(moves))
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                float x = fmaxf(most[t], __shfl_xor(most[t], 16));
                x = fmaxf(x, __shfl_xor(x, 32));
                x = x == neg_inf() ? x : x * factor;
                const float up = x > m[t] + (SLACK - ROOM) ? fmaxf(m[t], x + ROOM) : m[t];
                const float down = m[t] == up ? 1.0f : m[t] == neg_inf() ? 0.0f : __builtin_amdgcn_exp2f(m[t] - up);
                m[t] = up;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) o[t][i] *= down;
                l[t] *= down;
            }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const float by = m[t] == neg_inf() ? 0.0f : m[t];
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i & 3][i >> 2], factor, -by));
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
        }
        fetch(turn & 1, 0);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    multiply((turns + 1) & 1);
    if (group == 0) __syncthreads();
    __syncthreads();
    // All scores may be -inf, which is not the same as having none: the maximum tells.
    saw |= (unsigned)__shfl_xor((int)saw, 16);
    saw |= (unsigned)__shfl_xor((int)saw, 32);
#pragma unroll
    for (int t = 0; t < RT; ++t)
        if (saw && m[t] == neg_inf() && l[t][0] == 0.0f) m[t] = LOWEST;

    // The second group's sums join the first's.
    f32x4 *const sums = reinterpret_cast<f32x4 *>(lds) + part_of_rows * RT * (D / 16) * 64 + lane;
    if (group == 1) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) sums[(t * (D / 16) + i) * 64] = o[t][i];
            if (g == 0) ml_of[part_of_rows][t][c] = f32x2{m[t], l[t][0]};
        }
    }
    __syncthreads();
    if (group == 1) return;
    const long long all_rows = (long long)a.q.batch * a.q.queries * a.q.heads;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if (to[t] < 0) break;
        const bool see = sees >> t & 1u;
        const f32x2 ml = ml_of[part_of_rows][t][c];
        const float most = fmaxf(m[t], ml[0]);
        const float mine = m[t] == neg_inf() ? (l[t][0] == 0.0f ? 0.0f : l[t][0]) : __builtin_amdgcn_exp2f(m[t] - most);
        const float its = ml[0] == neg_inf() ? (ml[1] == 0.0f ? 0.0f : ml[1]) : __builtin_amdgcn_exp2f(ml[0] - most);
        const long long row = split * all_rows + to[t];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            const f32x4 x = o[t][i] * mine + sums[(t * (D / 16) + i) * 64] * its;
            *reinterpret_cast<f32x4 *>(a.part_o + row * D + 16 * i + 4 * g) = see ? x : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        if (g == 0) a.part_ml[row] = see ? f32x2{most, l[t][0] * mine + ml[1] * its} : f32x2{neg_inf(), 0.0f};
    }
}

struct Plan {
    long long rows;  // of the whole call
    bool wide;
    int blocks;      // of rows and kv heads
    int splits, own;
};

Plan plan_of(const Cache &c, int format, int d, const rec_query &q, int prefix_width)
{
    Plan p;
    p.rows = (long long)q.batch * q.queries * q.heads;
    const bool bf = q.dtype == REC_BF16;
    const long long of_head = p.rows / c.kv_heads;
    const long long tiles = (((long long)prefix_width << c.page_shift) + TILE - 1) / TILE;
    // A wide block has a row's tile done in 0.08 to 0.13 us of a compute unit (head_dim 32 to 128), a narrow one in 0.17 to 0.25, but takes 7 us more
    // to start and end.  Rows of two heads of 64, mx4: 1024 before 16000 tokens 37 us narrow, 38 wide, 2048 65 and 49; 4096 before 2000
    // 27 and 30, 8192 48 and 45; 8192 before 300 29 and 33, 16384 50 and 47.
    p.wide = (of_head + ROWS - 1) / ROWS * c.kv_heads * (tiles + 12) > 30000;
    const int per_block = p.wide ? row_tiles_of(d, bf) * ROW_WAVES * ROWS : ROWS;
    p.blocks = (int)((of_head + per_block - 1) / per_block * c.kv_heads);
    p.own = own_parts(c, format, d, q);
    // Parts of the prefix: as many as end soonest, at what a block's start and end cost beside its tiles, where so many
    // blocks work at once (two narrow ones of a compute unit: of 128 columns a SIMD's registers hold two waves; planned for four, 1024 rows of 2 heads
    // of 128 before 2000 tokens take 28 us, so 20).
    const long long waves = p.wide ? GROUPS : 4, at_once = p.wide ? CUS : 2 * CUS;
    long long best = 0;
    p.splits = 1;
    for (int s = 1; s <= std::clamp<long long>(tiles, 1, MOST_BEFORE); ++s) {
        const long long each = (tiles + s - 1) / s, turns = (each + waves - 1) / waves, cost = (p.blocks * (long long)s + at_once - 1) / at_once * (turns + 6);
        if (s == 1 || cost < best) {
            best = cost;
            p.splits = s;
        }
    }
    return p;
}

template <int FMT, int D, bool BF>
hipError_t shared_as(const SharedArgs &a, const Plan &p, int format, hipStream_t s)
{
    const dim3 grid((unsigned)(p.blocks * p.splits));
    if (p.wide) hipLaunchKernelGGL((wide_kernel<FMT, D, BF>), grid, dim3(64 * ROW_WAVES * GROUPS), 0, s, a);
    else hipLaunchKernelGGL((narrow_kernel<FMT, D, BF>), grid, dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    e = launch_behind(a.c, format, D, a.q, {a.part_o, reinterpret_cast<float *>(a.part_ml)}, p.splits, s);
    if (e != hipSuccess || p.own == 1) return e;
    hipLaunchKernelGGL((combine_kernel<D, BF>), dim3((unsigned)p.rows), dim3(256), 0, s, a.part_o, a.part_ml, p.splits + p.own, p.rows, a.q.dev_out);
    return hipGetLastError();
}

template <int FMT, int D>
hipError_t shared_of(const SharedArgs &a, const Plan &p, int format, hipStream_t s)
{
    return a.q.dtype == REC_BF16 ? shared_as<FMT, D, true>(a, p, format, s) : shared_as<FMT, D, false>(a, p, format, s);
}

}  // namespace

// Few tiles in all: each history reads the prefix for itself, in one launch.  4 kv heads of 64, mx8, fp16, 20 events behind a prefix: 8 histories
// behind 400 tokens 6.5 us so, 10.5 in two launches, 128 (4096 tiles) 8.6 and 11.4, 32 behind 4000 (8192 tiles) 16.0 and 13.2, 128 behind 1000
// (8704) 14.4 and 11.4.  4 kv heads of 32, mx4, bf16: 128 behind 300 (3584 tiles) 6.8 and 9.5, 500 (5120) 7.5 and 9.6, 1000 (9216) 12.9 and 9.6; 32 behind
// 2000 (4352) 10.1 both ways; of 128, mx8, fp16: 12.3 and 13.6, 14.0 and 14.7, 20.1 and 15.0, 16.1 and 15.8; of 128, mx4, bf16: 9.9 and 12.5, 11.1 and 13.0,
// 15.6 and 13.9, 13.4 and 15.6.
bool joined(const Cache &c, const rec_query &q, int prefix_width) { return joined_work(c, q, prefix_width) <= 4096; }

long long shared_threads(const Cache &c, int format, int d, const rec_query &q, int prefix_width)
{
    if (joined(c, q, prefix_width)) return joined_threads(c, format, d, q, prefix_width);
    const Plan p = plan_of(c, format, d, q, prefix_width);
    return std::max((long long)p.blocks * p.splits * 64 * ROW_WAVES * GROUPS, p.own == 1 ? 0 : p.rows * 256);
}

size_t shared_workspace(const Cache &c, int format, int d, const rec_query &q, int prefix_width)
{
    if (q.batch == 0 || q.queries == 0) return 0;
    if (joined(c, q, prefix_width)) return joined_workspace(c, format, d, q, prefix_width);
    const Plan p = plan_of(c, format, d, q, prefix_width);
    return (size_t)(p.splits + (p.own == 1 ? 0 : p.own)) * (size_t)p.rows * ((size_t)d * sizeof(float) + sizeof(f32x2));
}

void shared_form(const Cache &c, int format, int d, const rec_query &q, int prefix_width, int32_t (&form)[3])
{
    if (q.batch == 0 || q.queries == 0 || joined(c, q, prefix_width)) {
        form[0] = REC_SHARED_JOINED;
        form[1] = 0;
        form[2] = joined_parts(c, format, d, q, prefix_width);
        return;
    }
    const Plan p = plan_of(c, format, d, q, prefix_width);
    form[0] = p.wide ? REC_SHARED_WIDE : REC_SHARED_NARROW;
    form[1] = p.splits;
    form[2] = p.own;
}

hipError_t launch_shared(const Cache &c, int format, int d, const rec_query &q, const Prefix &prefix, void *workspace, hipStream_t s)
{
    if (joined(c, q, prefix.width)) return launch_joined(c, format, d, q, prefix, workspace, s);
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
    a.part_ml = reinterpret_cast<f32x2 *>(a.part_o + (p.splits + (p.own == 1 ? 0 : p.own)) * p.rows * d);
    if (format == REC_MX4)
        return d == 32 ? shared_of<REC_MX4, 32>(a, p, format, s) : d == 64 ? shared_of<REC_MX4, 64>(a, p, format, s) : shared_of<REC_MX4, 128>(a, p, format, s);
    return d == 32 ? shared_of<REC_MX8, 32>(a, p, format, s) : d == 64 ? shared_of<REC_MX8, 64>(a, p, format, s) : shared_of<REC_MX8, 128>(a, p, format, s);
}

}  // namespace hist
}  // namespace rec
