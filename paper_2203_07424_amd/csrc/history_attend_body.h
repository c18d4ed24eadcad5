// What the kernels that attend to the cache share: queries as terms, tiles of 64 keys and values, the products
// over them, what masks leave out, and the joining of parts (csrc/history_attend.hip has the description).
#ifndef REC_HISTORY_ATTEND_BODY_H
#define REC_HISTORY_ATTEND_BODY_H
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

// Eight columns of a row from the W waves that have a share of its keys: sums x and y, the weights' sum l and the maximum's exponent m.
template <int W, int LD, int N>
__device__ inline void join_waves(const float (&o_of)[W][N][LD], const f32x2 (&ml_of)[W][N], int r, int col, float &m, float &l, f32x4 &x, f32x4 &y)
{
    m = neg_inf();
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, ml_of[w][r][0]);
    l = 0.0f;
    x = y = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const f32x2 ml = ml_of[w][r];
        const float by = ml[0] == neg_inf() ? (ml[1] == 0.0f ? 0.0f : ml[1]) : __builtin_amdgcn_exp2f(ml[0] - m);
        l += ml[1] * by;
        x += *reinterpret_cast<const f32x4 *>(&o_of[w][r][col]) * by;
        y += *reinterpret_cast<const f32x4 *>(&o_of[w][r][col + 4]) * by;
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
    static_assert(MOST_PARTS == 64, "a wave has a lane for each part's weight");
    __shared__ float weight[MOST_PARTS];
    __shared__ f32x4 sums[GROUPS][LANES];
    const long long row = blockIdx.x;
    const int col = threadIdx.x % LANES, group = threadIdx.x / LANES, lane = threadIdx.x & 63;
    f32x2 ml = {neg_inf(), 0.0f};
    if (lane < splits) ml = part_ml[lane * rows + row];
    // The parts' sums are on their way while their weights are worked out.
    f32x4 part[MOST_PARTS / GROUPS];
#pragma unroll
    for (int i = 0; i < MOST_PARTS / GROUPS; ++i) {
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
    for (int i = 0; i < MOST_PARTS / GROUPS; ++i)
        if (group + i * GROUPS < splits) x += part[i] * weight[group + i * GROUPS];
    sums[group][col] = x;
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) x += sums[i][col];
    x *= inverse(l, m);
    *reinterpret_cast<tx4 *>(static_cast<T *>(out) + row * D + 4 * col) = __builtin_convertvector(x, tx4);
}

}  // namespace
}  // namespace hist
}  // namespace rec
#endif
