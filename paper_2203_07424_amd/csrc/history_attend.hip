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

#include "history.h"

namespace rec {
namespace hist {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

constexpr int ROWS = 16;       // query rows of a wave
constexpr int TILE = 64;       // keys
// A row's largest weight lies between 2^-ROOM and 2^(SLACK - ROOM): sums over 2^31 tokens of values up to fp32's largest
// stay in its range, and weights are rounded to bf16 of themselves down to 2^-86 of the largest.
constexpr float SLACK = 8.0f, ROOM = 40.0f;
constexpr float LOWEST = -3.4e38f;  // the maximum of a row that has seen nothing but scores of -inf
constexpr int CUS = 256;

// Waves that a SIMD holds at once; the compiler gives a wave at most its share of registers.
__host__ __device__ constexpr int waves_of(int format, int d, bool bf, int heads)
{
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
};

__device__ inline float neg_inf() { return -__builtin_inff(); }

// What a row's sums are multiplied by in the end, from its weights' sum and their maximum's exponent.
__device__ inline float inverse(float l, float m) { return l == 0.0f && m == neg_inf() ? 0.0f : 1.0f / l; }

// Terms of eight query elements x in units of `scale`; x becomes what is left.
__device__ inline u32x2 term_of(float (&x)[8], float scale)
{
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        s16x2 w = {0, 0};
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[4 * i], x[4 * i + 1], scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[4 * i + 2], x[4 * i + 3], scale, true);
        const unsigned bits = __builtin_bit_cast(unsigned, w);
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bits, scale, false);
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bits, scale, true);
        x[4 * i] -= a[0];
        x[4 * i + 1] -= a[1];
        x[4 * i + 2] -= b[0];
        x[4 * i + 3] -= b[1];
        r[i] = bits;
    }
    return r;
}

// A wave's query rows as operands.  Column k of a product is byte k % 16 of half k / 64 of
// lane group k / 16 % 4; its scale is byte 0 of lane group k / 32.
template <int D, bool BF>
struct Query {
    static constexpr int TERMS = BF ? 2 : 3;
    static constexpr int STEPS = D == 128 ? TERMS : D == 64 && TERMS == 3 ? 2 : 1;
    i32x8 b[STEPS];
    int scale[STEPS];

    static constexpr int PARTS = D == 128 ? 2 : 1;  // 16 elements of this lane each
    u32x4 raw[PARTS][2];

    // `row`: this lane's row (lane % 16) or null.
    __device__ inline void fetch(const void *row, int g)
    {
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                raw[p][h] = u32x4{0u, 0u, 0u, 0u};
                if (row) raw[p][h] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(row) + 2 * (64 * p + 16 * (D == 32 ? g & 1 : g) + 8 * h));
            }
    }

    // What was fetched, times `sign`, as terms.
    __device__ inline void convert(float sign, int g)
    {
        using T = std::conditional_t<BF, __bf16, _Float16>;
        typedef T tx8 __attribute__((ext_vector_type(8)));
        float x[PARTS][2][8];
        unsigned most[PARTS];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            most[p] = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const tx8 v = __builtin_bit_cast(tx8, raw[p][h]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float f = (float)v[i];
                    x[p][h][i] = f;
                    most[p] = max(most[p], __builtin_bit_cast(unsigned, f) & 0x7fffffffu);
                }
            }
            most[p] = max(most[p], (unsigned)__shfl_xor((int)most[p], 16));  // 32 elements: lane groups 2 j and 2 j + 1
        }
        unsigned byte[PARTS];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            // So that the largest is at most 448, and no term overflows; 255 where the query is not finite.
            const int e = max((int)(most[p] >> 23) - 127 - 8 + ((most[p] & 0x7fffffu) > 0x600000u ? 1 : 0), -110);
            byte[p] = most[p] >= 0x7f800000u ? 255u : (unsigned)(e + 127);
            const float unit = sign * __builtin_bit_cast(float, (unsigned)(127 - e) << 23);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[p][h][i] *= unit;
        }
        u32x4 term[TERMS][PARTS];
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                const float s = t == 0 ? 1.0f : t == 1 ? 0x1p-4f : 0x1p-8f;
                const u32x2 lo = term_of(x[p][0], s), hi = term_of(x[p][1], s);
                term[t][p] = u32x4{lo[0], lo[1], hi[0], hi[1]};
            }
        // The scale of block j of 32 elements is with lane groups 2 j and 2 j + 1 of its part.
        const int lane = threadIdx.x & 63;
        if constexpr (D == 128) {
            const unsigned a = (unsigned)__shfl((int)byte[0], (g & 1) * 32 + (lane & 15)), z = (unsigned)__shfl((int)byte[1], (g & 1) * 32 + (lane & 15));
            const unsigned mine = g < 2 ? a : z;
#pragma unroll
            for (int t = 0; t < TERMS; ++t) {
                set(t, term[t][0], term[t][1]);
                scale[t] = mine == 255u ? 255 : (int)(mine - 4 * t);
            }
        } else if constexpr (D == 64) {
            const unsigned mine = (unsigned)__shfl((int)byte[0], (g & 1) * 32 + (lane & 15));
            set(0, term[0][0], term[1][0]);
            scale[0] = mine == 255u ? 255 : (int)(mine - 4 * (g >> 1));
            if constexpr (TERMS == 3) {
                set(1, term[2][0], u32x4{0u, 0u, 0u, 0u});
                scale[1] = mine == 255u ? 255 : (int)(mine - 8);
            }
        } else {
            const u32x4 none = {0u, 0u, 0u, 0u};
            set(0, g < 2 ? term[0][0] : term[1][0], TERMS == 3 && g < 2 ? term[TERMS - 1][0] : none);
            scale[0] = byte[0] == 255u ? 255 : (int)(byte[0] - 4 * min(g, TERMS - 1));
        }
    }
    __device__ inline void set(int s, u32x4 lo, u32x4 hi)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            b[s][i] = (int)lo[i];
            b[s][4 + i] = (int)hi[i];
        }
    }
};

// Codes and scales of 64 keys and values, as this lane needs them.
template <int FMT, int D>
struct Tile {
    static constexpr int WIDE = FMT == REC_MX8 ? 2 : 1;
    static constexpr int KW = FMT == REC_MX8 && D == 128 ? 2 : 1;
    static constexpr int SW = D / BLOCK;
    u32x4 k[4][KW];
    unsigned ks[SW];
    u32x4 v[D / BLOCK][WIDE], vs[D / BLOCK];

    // kg: the group of this lane's keys.
    __device__ inline void load_keys(const unsigned char *kg, int c, int g)
    {
        constexpr int CB = code_bytes<FMT>(D);
        const int part = FMT == REC_MX4 ? (D == 32 ? 0 : D == 64 ? 16 * (g & 1) : 16 * g) : (D == 32 ? 16 * (g & 1) : 16 * g);
        const unsigned char *kp = kg + 4 * (c & 3) * CB + part;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int w = 0; w < KW; ++w) k[x][w] = *reinterpret_cast<const u32x4 *>(kp + x * CB + 64 * w);
        const unsigned char *sp = kg + 2 * GROUP * CB + 4 * (c & 3) * SW;
        if constexpr (SW == 1) {
            ks[0] = *reinterpret_cast<const unsigned *>(sp);
        } else if constexpr (SW == 2) {
            const u32x2 s = *reinterpret_cast<const u32x2 *>(sp);
            ks[0] = s[0];
            ks[1] = s[1];
        } else {
            const u32x4 s = *reinterpret_cast<const u32x4 *>(sp);
#pragma unroll
            for (int x = 0; x < 4; ++x) ks[x] = s[x];
        }
    }
    // vg: the group of its values.
    __device__ inline void load_values(const unsigned char *vg, int c)
    {
        constexpr int CB = code_bytes<FMT>(D);
        const unsigned char *vp = vg + GROUP * CB + c * GROUP * WIDE, *vsp = vg + 2 * GROUP * CB + GROUP * SW;
#pragma unroll
        for (int b = 0; b < D / BLOCK; ++b) {
#pragma unroll
            for (int w = 0; w < WIDE; ++w) v[b][w] = *reinterpret_cast<const u32x4 *>(vp + b * GROUP * GROUP * WIDE + 16 * w);
            vs[b] = *reinterpret_cast<const u32x4 *>(vsp + b * GROUP);
        }
    }
};

// Scores of the x-th product.
template <int FMT, int D, bool BF, int X>
__device__ inline f32x4 scores(const Tile<FMT, D> &t, const Query<D, BF> &q, int g)
{
    i32x8 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = (int)t.k[X][0][i];
        a[4 + i] = (int)t.k[X][Tile<FMT, D>::KW - 1][i];
    }
    // Byte of the scale word; the block's byte moves there where it depends on the lane.
    constexpr int AT = D == 32 ? X : D == 64 ? 2 * (X & 1) : 0;
    const int s = (int)(D == 32 ? t.ks[0] : D == 64 ? t.ks[(X >> 1) % Tile<FMT, D>::SW] >> (8 * (g & 1)) : t.ks[X % Tile<FMT, D>::SW] >> (8 * g));
    f32x4 r = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < Query<D, BF>::STEPS; ++i)
        r = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.b[i], r, FMT == REC_MX4 ? 4 : 0, 0, AT, s, 0, q.scale[i]);
    return r;
}

// The values of token T of a lane's 16 in columns j and j + 16 of block b, in bf16.
template <int FMT, int D, int T>
__device__ inline unsigned value_pair(const Tile<FMT, D> &t, int b)
{
    constexpr int at = 8 * (T & 3);
    const unsigned word = t.vs[b][T >> 2];
    const float s = __builtin_bit_cast(float, at < 23 ? word << (23 - at) : word >> (at - 23));
    bf16x2 r;
    if constexpr (FMT == REC_MX4) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.v[b][0][T >> 2], s, T & 3);
    else r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(t.v[b][T >> 3][(T >> 1) & 3], s, (T & 1) != 0);
    return __builtin_bit_cast(unsigned, r);
}

// Operands of eight tokens, 8 H ..., for the two column tiles of block b.
template <int FMT, int D, int H>
__device__ inline void value_operands(const Tile<FMT, D> &t, int b, u32x4 &lo, u32x4 &hi)
{
    const unsigned a[8] = {value_pair<FMT, D, 8 * H>(t, b),     value_pair<FMT, D, 8 * H + 1>(t, b), value_pair<FMT, D, 8 * H + 2>(t, b),
                           value_pair<FMT, D, 8 * H + 3>(t, b), value_pair<FMT, D, 8 * H + 4>(t, b), value_pair<FMT, D, 8 * H + 5>(t, b),
                           value_pair<FMT, D, 8 * H + 6>(t, b), value_pair<FMT, D, 8 * H + 7>(t, b)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lo[i] = __builtin_amdgcn_perm(a[2 * i + 1], a[2 * i], 0x05040100u);
        hi[i] = __builtin_amdgcn_perm(a[2 * i + 1], a[2 * i], 0x07060302u);
    }
}

__device__ inline f32x4 product(u32x4 a, u32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ inline unsigned pack(float a, float b)
{
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(unsigned, r);
}

// What a wave carries: for query row lane % 16, columns 16 i + 4 (lane / 16) ... + 3.  With several
// kv heads a wave, o[h] holds the products with head h's values, of which only its own rows count.
template <int D, int HEADS>
struct Sums {
    f32x4 o[HEADS][D / 16], l;
    float m;  // exponent of weight 1, ROOM above the largest score's
};

// Bytes of 255 where the bits of a nibble are set.
__device__ inline unsigned bytes_of(unsigned nibble)
{
    const unsigned ones = nibble * 0x204081u & 0x01010101u;
    return (ones << 8) - ones;
}

// Tokens of a lane's 16 that count as zero whatever their bytes are: 0 * NaN would reach the
// rows that do not see a value.  Those are the ones that no row sees (bit t of `used` clear) and,
// a block at a time, those whose block is NaN, or under a scale that no write makes, which could be
// infinite; a scale of 2^-127 does it, and for the former no code that is NaN itself.  Returns the
// blocks (bit b) of which row c, which sees the tokens in `seen`, sees one of those.
template <int FMT, int D>
__device__ inline unsigned clear_values(Tile<FMT, D> &t, unsigned used, unsigned seen)
{
    constexpr unsigned NO_SCALE = FMT == REC_MX4 ? 253u : 247u;
    unsigned nan = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const unsigned keep = bytes_of(used >> (4 * x) & 15u), mine = bytes_of(seen >> (4 * x) & 15u);
#pragma unroll
        for (int b = 0; b < D / BLOCK; ++b) {
            const unsigned s = t.vs[b][x], top = ((s & 0x7f7f7f7fu) + (256u - NO_SCALE) * 0x01010101u) & s & 0x80808080u;  // bytes from NO_SCALE on
            nan |= (top & mine) != 0 ? 1u << b : 0u;
            t.vs[b][x] = s & keep & ~((top << 1) - (top >> 7));
            if constexpr (FMT == REC_MX8) {
                t.v[b][x >> 1][2 * (x & 1)] &= __builtin_amdgcn_perm(keep, keep, 0x01010000u);
                t.v[b][x >> 1][2 * (x & 1) + 1] &= __builtin_amdgcn_perm(keep, keep, 0x03030202u);
            }
        }
    }
    nan |= (unsigned)__shfl_xor((int)nan, 16);
    return nan | (unsigned)__shfl_xor((int)nan, 32);
}

// Codes that are NaN under any scale (E4M3 has two; write_kernel makes neither, but a place that was never written may
// hold them) count as zero too, and rows that see one get NaN in its column: a product of ones, where such a code is and where a
// row sees its token, tells which.  Only where rows of a wave see different tokens; else clear_values() left none but
// what all of them see.
template <int D>
__device__ inline void clear_nan_codes(Tile<REC_MX8, D> &t, unsigned seen, f32x4 (&o)[D / 16])
{
    auto nan_bytes = [](unsigned codes) { return ((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };  // their top bits
    unsigned found = 0;
#pragma unroll
    for (int b = 0; b < D / BLOCK; ++b)
#pragma unroll
        for (int i = 0; i < 8; ++i) found |= nan_bytes(t.v[b][i >> 2][i & 3]);
    if (!__any(found != 0)) return;
#pragma unroll
    for (int b = 0; b < D / BLOCK; ++b) {
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = x;
        auto half = [&](auto h) {  // eight tokens
            constexpr int H = h();
            Tile<REC_MX8, D> ones;
            u32x4 sees, lo, hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unsigned codes = t.v[b][H][i];
                asm("" : "+v"(codes));  // looked at again: what was found above would take a register a word
                const unsigned top = nan_bytes(codes);
                ones.v[b][H][i] = (top >> 7) * 0x38u;
                t.v[b][H][i] = codes & ~((top << 1) - (top >> 7));
                sees[i] = (seen >> (8 * H + 2 * i) & 1u) * 0x3f80u | (seen >> (8 * H + 2 * i + 1) & 1u) * 0x3f800000u;
            }
            ones.vs[b] = u32x4{0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
            value_operands<REC_MX8, D, H>(ones, b, lo, hi);
            x = product(lo, sees, x);
            y = product(hi, sees, y);
            __builtin_amdgcn_sched_barrier(0);  // in these registers, then the next half
        };
        half(std::integral_constant<int, 0>());
        half(std::integral_constant<int, 1>());
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[2 * b][i] = x[i] != 0.0f ? __builtin_nanf("") : o[2 * b][i];
            o[2 * b + 1][i] = y[i] != 0.0f ? __builtin_nanf("") : o[2 * b + 1][i];
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Bits [0, n) of a lane's 16 tokens, for any n.
__device__ inline unsigned below(int n) { return (1u << min(max(n, 0), 16)) - 1u; }

// Where a wave's row goes.
__device__ inline long long out_row(const AttendArgs &a, int b, int kv, int row)
{
    const int i = a.by_per.of(row);
    return ((long long)b * a.q.queries + i) * a.q.heads + kv * a.per + (row - i * a.per);
}

template <int FMT, int D, bool BF, int W, int HEADS>
__global__ __launch_bounds__(64 * W, waves_of(FMT, D, BF, HEADS)) void attend_kernel(AttendArgs a)
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
    // Positions of this wave's rows: of its first, its last, and this lane's; -1 sees nothing.
    const int first_row = row_tile * ROWS, last_row = min(first_row + SLOT, a.rows) - 1, row = min(first_row + r, last_row);
    const bool real = first_row + r <= last_row;
    const bool together = a.q.candidates != 0;
    auto position = [&](int row) { return together ? len - 1 : max(len - a.q.queries + a.by_per.of(row), -1); };
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
            if (token < len) page = table[token >> shift];
            return page;
        };
        auto group_at = [&](int page, int token) {
            const bool ok = (unsigned)page < pages;  // else some group that is there: its tokens count for nothing
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
            const bool whole = key + TILE - 1 <= p_lo && (key > p_hi - window || key + TILE <= sinks) && __all(there);
            unsigned nan = 0;  // bit 4 h + b: row c sees a NaN in block b of head h's values
            if (!whole) {
                // Bit t: row c sees token t of group g; some row does.
                const int first = key + 16 * g;
                auto upto = [&](int at) { return below(max(at - first, -1) + 1); };
                auto before = [&](int at) { return below(max(at - first, -1) - window + 1); };
                unsigned seen = upto(pos) & (~before(pos) | below(sinks - first));
                unsigned used = upto(p_hi) & (~before(p_lo) | below(sinks - first));
                if (!there) {
                    if (used && c == 0)
                        report(a.c.fault, REC_FAULT_PAGE, (unsigned long long)b * (unsigned)a.q.table_width + (unsigned)(first >> shift));
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
        if (a.splits > 1) {
            if (real && g == 0) a.part_ml[split * all_rows + out] = f32x2{sum.m, l};
            if (real)
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                    *reinterpret_cast<f32x4 *>(a.part_o + (split * all_rows + out) * D + 16 * i + 4 * g) = o[i];
        } else if (real) {
            const float by = inverse(l, sum.m);
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
            if (a.splits > 1) {
                float *p = a.part_o + (split * all_rows + to) * D + col;
                *reinterpret_cast<f32x4 *>(p) = x;
                *reinterpret_cast<f32x4 *>(p + 4) = y;
                if (col == 0) a.part_ml[split * all_rows + to] = f32x2{m, l};
            } else {
                typedef T tx8 __attribute__((ext_vector_type(8)));
                const float by = inverse(l, m);
                x *= by;
                y *= by;
                const f32x8 z = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                *reinterpret_cast<tx8 *>(static_cast<T *>(a.q.dev_out) + to * D + col) = __builtin_convertvector(z, tx8);
            }
        }
    }
}

// Joins the at most 64 parts of a row by a block: a lane looks up a part's weight, then groups
// of D / 4 threads add up a share of the parts' sums, all loaded at once, and meet in LDS.  Always in the same order.  (A thread for all parts of its columns took 20 us for 64.)
template <int D, bool BF>
__global__ __launch_bounds__(256) void combine_kernel(const float *part_o, const f32x2 *part_ml, int splits, long long rows, void *out)
{
    using T = std::conditional_t<BF, __bf16, _Float16>;
    typedef T tx4 __attribute__((ext_vector_type(4)));
    constexpr int LANES = D / 4, GROUPS = 256 / LANES;
    __shared__ float weight[64];
    __shared__ f32x4 sums[GROUPS][LANES];
    const long long row = blockIdx.x;
    const int col = threadIdx.x % LANES, group = threadIdx.x / LANES, lane = threadIdx.x & 63;
    f32x2 ml = {neg_inf(), 0.0f};
    if (lane < splits) ml = part_ml[lane * rows + row];
    // The parts' sums are on their way while their weights are worked out.
    f32x4 part[64 / GROUPS];
#pragma unroll
    for (int i = 0; i < 64 / GROUPS; ++i) {
        part[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (group + i * GROUPS < splits) part[i] = *reinterpret_cast<const f32x4 *>(part_o + ((group + i * GROUPS) * rows + row) * D + 4 * col);
    }
    float m = ml[0];
#pragma unroll
    for (int i = 32; i; i >>= 1) m = fmaxf(m, __shfl_xor(m, i));
    const float by = ml[0] == neg_inf() ? (ml[1] == 0.0f ? 0.0f : ml[1]) : __builtin_amdgcn_exp2f(ml[0] - m);
    float l = ml[1] * by;
#pragma unroll
    for (int i = 32; i; i >>= 1) l += __shfl_xor(l, i);
    if (threadIdx.x < 64) weight[lane] = by;
    __syncthreads();
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 64 / GROUPS; ++i)
        if (group + i * GROUPS < splits) x += part[i] * weight[group + i * GROUPS];
    sums[group][col] = x;
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) x += sums[i][col];
    x *= inverse(l, m);
    *reinterpret_cast<tx4 *>(static_cast<T *>(out) + row * D + 4 * col) = __builtin_convertvector(x, tx4);
}

struct Plan {
    int waves, splits, row_tiles, per;
    int heads;       // kv heads of a wave
    long long rows;  // of the whole call
};

Plan plan_of(const Cache &c, int format, int d, const rec_query &q)
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
        tiles = std::min(tiles, (q.window + apart + TILE - 2) / TILE + 1 + (q.sinks + TILE - 1ll) / TILE);
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
    // for a place and then reads alone: 4 parts of 256 pairs in 3 places 221 us, 3 parts 199), of two tiles a wave at least.
    // Where pairs alone take all places, parts of eight tiles a wave, up to four, for the longest of ragged
    // histories (1600 pairs up to 8000 long 51 -> 43 us; all alike 171 -> 178).
    const long long room = 4ll * waves_of(format, d, q.dtype == REC_BF16, 1) * CUS / (pairs * p.waves);
    const long long parts = room > 1 ? std::min({room, tiles / (2 * p.waves), 64ll}) : p.waves == 4 ? std::min(tiles / (8 * p.waves), 4ll) : 1;
    p.splits = (int)std::max(1ll, parts);
    return p;
}

template <int FMT, int D, bool BF>
hipError_t attend_as(const AttendArgs &a, const Plan &p, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)a.q.batch * a.c.kv_heads / p.heads * p.row_tiles * p.splits));
    if constexpr (D <= 64)
        if (p.heads == 2) {
            hipLaunchKernelGGL((attend_kernel<FMT, D, BF, 1, 2>), grid, dim3(64), 0, s, a);
            return hipGetLastError();
        }
    if (p.waves == 4) hipLaunchKernelGGL((attend_kernel<FMT, D, BF, 4, 1>), grid, dim3(256), 0, s, a);
    else if (p.waves == 2) hipLaunchKernelGGL((attend_kernel<FMT, D, BF, 2, 1>), grid, dim3(128), 0, s, a);
    else hipLaunchKernelGGL((attend_kernel<FMT, D, BF, 1, 1>), grid, dim3(64), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL((combine_kernel<D, BF>), dim3((unsigned)p.rows), dim3(256), 0, s, a.part_o, a.part_ml, p.splits, p.rows, a.q.dev_out);
    return hipGetLastError();
}

template <int FMT, int D>
hipError_t attend_of(const AttendArgs &a, const Plan &p, hipStream_t s)
{
    return a.q.dtype == REC_BF16 ? attend_as<FMT, D, true>(a, p, s) : attend_as<FMT, D, false>(a, p, s);
}

}  // namespace

long long attend_threads(const Cache &c, int format, int d, const rec_query &q)
{
    const Plan p = plan_of(c, format, d, q);
    return (long long)q.batch * c.kv_heads * p.row_tiles * p.splits * 64 * p.waves;
}

void attend_form(const Cache &c, int format, int d, const rec_query &q, int32_t (&form)[3])
{
    const Plan p = plan_of(c, format, d, q);
    form[0] = p.waves;
    form[1] = p.splits;
    form[2] = p.heads;
}

size_t attend_workspace(const Cache &c, int format, int d, const rec_query &q)
{
    if (q.batch == 0 || q.queries == 0) return 0;
    const Plan p = plan_of(c, format, d, q);
    return p.splits == 1 ? 0 : (size_t)p.splits * (size_t)p.rows * ((size_t)d * sizeof(float) + sizeof(f32x2));
}

hipError_t launch_attend(const Cache &c, int format, int d, const rec_query &q, void *workspace, hipStream_t s)
{
    const Plan p = plan_of(c, format, d, q);
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
    if (format == REC_MX4)
        return d == 32 ? attend_of<REC_MX4, 32>(a, p, s) : d == 64 ? attend_of<REC_MX4, 64>(a, p, s) : attend_of<REC_MX4, 128>(a, p, s);
    return d == 32 ? attend_of<REC_MX8, 32>(a, p, s) : d == 64 ? attend_of<REC_MX8, 64>(a, p, s) : attend_of<REC_MX8, 128>(a, p, s);
}

}  // namespace hist
}  // namespace rec
