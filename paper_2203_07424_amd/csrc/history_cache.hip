// Quantising keys and values into the paged cache, and reading them back.
//
// Four lanes have a block of 32 columns, eight each: the block's largest magnitude is
// two exchanges within four lanes away, the scale is its exponent (so scaling is exact and only
// the conversion rounds), and the hardware's scaled conversions make the codes from
// the type at hand.  Bound by the bytes of the uncompressed side, as long as whole groups are
// stored as such: values lie along the tokens, so a token by itself is a byte in each of D / 2
// rows.  A group passes through LDS, where the tokens of a lane meet as words.
//
// The uncompressed side is streamed: it passes once, and beside it what is used again keeps its place in
// the caches.  65536 rows of 8 heads of 128 bf16, inputs changing: write 88 -> 69 us (4.9 TB/s), read
// 60 -> 50 (6.8 TB/s; a copy of this size 5.5); 81920 rows of 4 heads of 32 fp32: write 24 us, read
// 23 (4.5 TB/s).  Rows of fp32 are loaded as usual: a lane's 32 bytes are two loads of the same
// lines, which streaming may fetch twice (27 us).  Several heads a wave with the next one's rows on
// their way were no faster (98 us at two or four), keys and values in one wave 0.8 us slower where
// calls are smallest.
#include "history.h"

namespace rec {
namespace hist {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int THREADS = 256;

// Eight neighbouring columns as they lie in memory.
template <int DT>
struct Eight {
    u32x4 w[DT == REC_F32 ? 2 : 1];

    __device__ inline void load(const void *p, long long i)
    {
        const char *from = static_cast<const char *>(p) + (DT == REC_F32 ? 4 : 2) * i;
        if constexpr (DT == REC_F32) {
            w[0] = *reinterpret_cast<const u32x4 *>(from);
            w[1] = *reinterpret_cast<const u32x4 *>(from + 16);
        } else {
            w[0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from));
        }
    }

    // Bits of the largest magnitude in fp32; as whole numbers magnitudes order like the numbers, NaN last.
    __device__ inline unsigned most() const
    {
        if constexpr (DT == REC_F32) {
            unsigned m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, w[i >> 2][i & 3] & 0x7fffffffu);
            return m;
        } else {
            u16x2 m = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[0][i] & 0x7fff7fffu));
            const unsigned short one = m[0] > m[1] ? m[0] : m[1];
            if constexpr (DT == REC_BF16) return (unsigned)one << 16;
            else return __builtin_bit_cast(unsigned, (float)__builtin_bit_cast(_Float16, one));
        }
    }

    // No magnitude above that of bits `top`.
    __device__ inline void limit(unsigned top)
    {
#pragma unroll
        for (int i = 0; i < (DT == REC_F32 ? 8 : 4); ++i) {
            const unsigned x = w[i >> 2][i & 3];
            if constexpr (DT == REC_F32) {
                w[i >> 2][i & 3] = (x & 0x80000000u) | min(x & 0x7fffffffu, top);
            } else {
                const unsigned hi = min(x & 0x7fff0000u, top), lo = min(x << 16 & 0x7fff0000u, top) >> 16;
                w[0][i] = (x & 0x80008000u) | hi | lo;
            }
        }
    }

    // Columns 2 I and 2 I + 1.
    template <int I>
    __device__ inline auto two() const
    {
        if constexpr (DT == REC_F16) return __builtin_bit_cast(f16x2, (unsigned)w[0][I]);
        else return __builtin_bit_cast(bf16x2, (unsigned)w[0][I]);
    }
    template <int I>
    __device__ inline float one() const { return __builtin_bit_cast(float, (unsigned)w[I >> 2][I & 3]); }
};

// A result's eight columns, streamed.
template <int DT>
__device__ inline void store8(void *p, long long i, f32x8 x)
{
    if constexpr (DT == REC_F32)
        __builtin_nontemporal_store(x, reinterpret_cast<f32x8 *>(static_cast<float *>(p) + i));
    else if constexpr (DT == REC_F16)
        __builtin_nontemporal_store(__builtin_convertvector(x, f16x8), reinterpret_cast<f16x8 *>(static_cast<_Float16 *>(p) + i));
    else
        __builtin_nontemporal_store(__builtin_convertvector(x, bf16x8), reinterpret_cast<bf16x8 *>(static_cast<__bf16 *>(p) + i));
}

// What lanes l ^ 1 and l ^ 2 have.
__device__ inline unsigned next_lane(unsigned x) { return (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true); }
__device__ inline unsigned next_pair(unsigned x) { return (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true); }

// The scale byte of a block from the bits of its largest magnitude.
template <int FMT>
__device__ inline unsigned scale_byte(unsigned bits)
{
    constexpr int top = FMT == REC_MX4 ? 2 : 8, cap = FMT == REC_MX4 ? 125 : 119;
    constexpr unsigned over = FMT == REC_MX4 ? 0x600000u : 0x680000u;  // 1.75, 1.8125
    const int byte = min(max((int)(bits >> 23) - top + ((bits & 0x7fffffu) > over ? 1 : 0), 127 - 110), 127 + cap);
    return bits >= 0x7f800000u ? 255u : (unsigned)byte;
}

// Two codes, the I-th eighth of r.  E2M1 has no infinity, so the conversion itself saturates.
template <int FMT, int DT, int I>
__device__ inline void convert_two(u32x2 &r, const Eight<DT> &x, float scale)
{
    if constexpr (FMT == REC_MX4) {
        if constexpr (DT == REC_F32) r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r[0], x.template one<2 * I>(), x.template one<2 * I + 1>(), scale, I);
        else if constexpr (DT == REC_F16) r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r[0], x.template two<I>(), scale, I);
        else r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r[0], x.template two<I>(), scale, I);
    } else {
        constexpr bool HIGH = I % 2 != 0;
        const unsigned before = r[I / 2];
        s16x2 w = __builtin_bit_cast(s16x2, before);
        if constexpr (DT == REC_F32) w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x.template one<2 * I>(), x.template one<2 * I + 1>(), scale, HIGH);
        else if constexpr (DT == REC_F16) w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, x.template two<I>(), scale, HIGH);
        else w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, x.template two<I>(), scale, HIGH);
        r[I / 2] = __builtin_bit_cast(unsigned, w);
    }
}

// Block scale and codes (mx4 in one word, mx8 in two) of a lane's eight columns; no codes where the
// block is not finite.
template <int FMT, int DT>
__device__ inline u32x2 quantise(Eight<DT> x, unsigned &byte)
{
    unsigned most = x.most();
    most = max(most, next_lane(most));
    most = max(most, next_pair(most));
    byte = scale_byte<FMT>(most);
    if constexpr (FMT == REC_MX8 && DT != REC_F16) {
        // The scale's own limit leaves up to 512 where E4M3 ends at 448: magnitudes from
        // 1.8125 x 2^127, which only fp32 and bf16 have.
        if (__any(most > 0x7f680000u)) x.limit(0x7f600000u);
    }
    const float scale = __builtin_bit_cast(float, byte << 23);
    u32x2 r = {0u, 0u};
    convert_two<FMT, DT, 0>(r, x, scale);
    convert_two<FMT, DT, 1>(r, x, scale);
    convert_two<FMT, DT, 2>(r, x, scale);
    convert_two<FMT, DT, 3>(r, x, scale);
    const unsigned keep = byte == 255u ? 0u : ~0u;
    return u32x2{r[0] & keep, r[1] & keep};
}

// What a wave does: 16 entries of the slot list for one head, keys or values.  Most lists are
// histories, whose slots count up: 16 entries that fill a group are stored as the group, from
// wherever in the list it starts (the wave of its first entry has it, so it looks 16 entries
// back and ahead).  All other entries are stored by themselves.
struct Share {
    long long slot;       // lane i: entry 16 unit - 16 + i, or -1
    int first;            // entry (of those 48) where a whole group starts that is this wave's, or -1
    unsigned rest;        // bit i: entry 16 + i is this wave's alone
};

__device__ inline Share share_of(const int64_t *slots, long long tokens, long long unit, const Cache &c, int lane, bool tell)
{
    Share s;
    const long long at = 16 * unit - 16 + lane;
    s.slot = -1;
    if (lane < 48 && at >= 0 && at < tokens) s.slot = slots[at];
    if (s.slot < 0 || s.slot >> c.page_shift >= c.num_pages) {
        if (s.slot != -1 && tell && lane >= 16 && lane < 32) report(c.fault, REC_FAULT_SLOT, (unsigned long long)at);
        s.slot = -1;
    }
    const long long before = __shfl_up(s.slot, 1);
    const bool goes_on = lane > 0 && s.slot >= 0 && s.slot == before + 1 && (s.slot & 15) != 0;
    // Entries from which 15 more go on.
    unsigned long long run = __ballot(goes_on) >> 1;
    run &= run >> 1;
    run &= run >> 2;
    run &= run >> 4;               // 8 in a row
    run &= run >> 7;               // 15
    const unsigned long long starts = run & __ballot(s.slot >= 0 && (s.slot & 15) == 0);
    const unsigned mine = (unsigned)(starts >> 16) & 0xffffu;
    s.first = mine ? 16 + __builtin_ctz(mine) : -1;
    unsigned long long in_group = starts;  // and the 15 entries behind each
    in_group |= in_group << 1;
    in_group |= in_group << 2;
    in_group |= in_group << 4;
    in_group |= in_group << 8;
    s.rest = (unsigned)((__ballot(s.slot >= 0) & ~in_group) >> 16) & 0xffffu;
    return s;
}

// The n-th set bit.
__device__ inline int nth_bit(unsigned bits, int n)
{
    for (; n > 0; --n) bits &= bits - 1;
    return bits ? __builtin_ctz(bits) : -1;
}

// Elements j and j + 16 of a block are one place of a V row: lanes 0 and 1 of four have the
// first of 8 such pairs each, lanes 2 and 3 the second.  After an exchange each lane has four
// places, first_pair() ...: mx4 a byte each, mx8 two.
__device__ inline int first_pair(int block, int quad) { return 16 * block + 8 * (quad & 1) + 4 * (quad >> 1); }
template <int FMT>
__device__ inline u32x2 pairs_of(u32x2 codes, int quad)
{
    if constexpr (FMT == REC_MX4) {
        const unsigned other = next_pair(codes[0]);
        // Four codes of element j in the low bytes' halves, four of j + 16 in the high ones.
        unsigned lo = quad < 2 ? codes[0] & 0xffffu : other >> 16, hi = quad < 2 ? other & 0xffffu : codes[0] >> 16;
        lo = (lo | lo << 8) & 0x00ff00ffu;
        hi = (hi | hi << 8) & 0x00ff00ffu;
        lo = (lo | lo << 4) & 0x0f0f0f0fu;
        hi = (hi | hi << 4) & 0x0f0f0f0fu;
        return u32x2{lo | hi << 4, 0u};
    } else {
        const unsigned other = next_pair(quad < 2 ? codes[1] : codes[0]);
        const unsigned lo = quad < 2 ? codes[0] : other, hi = quad < 2 ? other : codes[1];
        return u32x2{__builtin_amdgcn_perm(hi, lo, 0x05010400u), __builtin_amdgcn_perm(hi, lo, 0x07030602u)};
    }
}

// Place I of a lane's four in PASSES tokens, next to each other.
template <int FMT, int PASSES, int I>
__device__ inline unsigned long long place_of(const u32x2 (&pair)[PASSES])
{
    if constexpr (FMT == REC_MX4) {
        if constexpr (PASSES == 1) return pair[0][0] >> (8 * I);
        constexpr unsigned two = I < 2 ? 0x05010400u : 0x07030602u;
        const unsigned a = __builtin_amdgcn_perm(pair[1 % PASSES][0], pair[0][0], two);
        if constexpr (PASSES == 2) return a >> (16 * (I & 1));
        const unsigned b = __builtin_amdgcn_perm(pair[3 % PASSES][0], pair[2 % PASSES][0], two);
        return __builtin_amdgcn_perm(b, a, I & 1 ? 0x07060302u : 0x05040100u);
    } else {
        constexpr unsigned two = I & 1 ? 0x07060302u : 0x05040100u;
        if constexpr (PASSES == 1) return pair[0][I / 2] >> (16 * (I & 1));
        const unsigned a = __builtin_amdgcn_perm(pair[1 % PASSES][I / 2], pair[0][I / 2], two);
        if constexpr (PASSES == 2) return a;
        const unsigned b = __builtin_amdgcn_perm(pair[3 % PASSES][I / 2], pair[2 % PASSES][I / 2], two);
        return a | (unsigned long long)b << 32;
    }
}

template <int FMT, int D>
constexpr int part_bytes() { return GROUP * code_bytes<FMT>(D); }

// LDS copy of a group's codes and scales of one side, 16 bytes a lane.
template <int FMT, int D>
__device__ inline unsigned char *piece_of(unsigned char *group, bool is_v, int piece)
{
    constexpr int CODES = part_bytes<FMT, D>() / 16, SCALES = D / 2 / 16;
    if (piece < CODES) return group + (is_v ? part_bytes<FMT, D>() : 0) + 16 * piece;
    return group + 2 * part_bytes<FMT, D>() + (is_v ? 16 * SCALES : 0) + 16 * (piece - CODES);
}

// The type that BYTES bytes are stored as.
template <int BYTES>
using Word = std::conditional_t<BYTES == 8, unsigned long long,
                                std::conditional_t<BYTES == 4, unsigned, std::conditional_t<BYTES == 2, unsigned short, unsigned char>>>;

// A wave's 16 entries, one side of them after the other.
template <int FMT, int DT, int D>
struct Writer {
    static constexpr int LANES = D / 8, ROWS = 64 / LANES, PASSES = GROUP / ROWS;  // of a row; rows at once; for 16 rows
    static constexpr int CB = code_bytes<FMT>(D), PIECES = part_bytes<FMT, D>() / 16 + D / 32;
    const Cache &c;
    int lane, in_row, quad, block, r, head;

    // A whole group, from list entry `entry` on, through LDS.  A lane has PASSES neighbouring tokens, so
    // that their places in a V row are one word.
    template <bool V>
    __device__ inline void group(const Eight<DT> (&x)[PASSES], unsigned char *group, long long entry, u32x4 *lds) const
    {
        unsigned char *to = reinterpret_cast<unsigned char *>(lds);
        u32x2 codes[PASSES];
        unsigned byte[PASSES], worst = 0;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            codes[p] = quantise<FMT, DT>(x[p], byte[p]);
            worst = max(worst, byte[p]);
        }
        if constexpr (V) {
            u32x2 pair[PASSES];
            unsigned scales = 0;
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                pair[p] = pairs_of<FMT>(codes[p], quad);
                scales |= byte[p] << (8 * p);
            }
            constexpr int BYTES = PASSES * (FMT == REC_MX4 ? 1 : 2);
            unsigned char *row = to + first_pair(block, quad) * (FMT == REC_MX4 ? 16 : 32) + BYTES * r;
            constexpr int NEXT = FMT == REC_MX4 ? 16 : 32;
            *reinterpret_cast<Word<BYTES> *>(row) = (Word<BYTES>)place_of<FMT, PASSES, 0>(pair);
            *reinterpret_cast<Word<BYTES> *>(row + NEXT) = (Word<BYTES>)place_of<FMT, PASSES, 1>(pair);
            *reinterpret_cast<Word<BYTES> *>(row + 2 * NEXT) = (Word<BYTES>)place_of<FMT, PASSES, 2>(pair);
            *reinterpret_cast<Word<BYTES> *>(row + 3 * NEXT) = (Word<BYTES>)place_of<FMT, PASSES, 3>(pair);
            if (quad == 0) *reinterpret_cast<Word<PASSES> *>(to + part_bytes<FMT, D>() + block * GROUP + PASSES * r) = (Word<PASSES>)scales;
        } else {
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int t = PASSES * r + p;
                if constexpr (FMT == REC_MX4) *reinterpret_cast<unsigned *>(to + t * CB + 4 * in_row) = codes[p][0];
                else *reinterpret_cast<u32x2 *>(to + t * CB + 8 * in_row) = codes[p];
            }
            if (quad == 0)
#pragma unroll
                for (int p = 0; p < PASSES; ++p) to[part_bytes<FMT, D>() + (PASSES * r + p) * (D / BLOCK) + block] = (unsigned char)byte[p];
        }
        if (c.fault && __any(worst == 255u) && quad == 0)
#pragma unroll
            for (int p = 0; p < PASSES; ++p)
                if (byte[p] == 255u) report(c.fault, REC_FAULT_VALUE, (unsigned long long)(entry + PASSES * r + p));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < (PIECES + 63) / 64; ++i)
            if (64 * i + lane < PIECES) *reinterpret_cast<u32x4 *>(piece_of<FMT, D>(group, V, 64 * i + lane)) = lds[64 * i + lane];
    }

    // A row by itself, to `slot`, where `there`.
    template <bool V>
    __device__ inline void row(const Eight<DT> &x, bool there, long long slot, long long entry) const
    {
        unsigned byte;
        const u32x2 codes = quantise<FMT, DT>(x, byte);
        const u32x2 pair = V ? pairs_of<FMT>(codes, quad) : codes;
        if (!there) return;
        if (byte == 255u && quad == 0) report(c.fault, REC_FAULT_VALUE, (unsigned long long)entry);
        const int at = (int)(slot & ((1 << c.page_shift) - 1)), t = at & 15;
        unsigned char *group = group_of<FMT>(c, D, slot >> c.page_shift, at, head);
        unsigned char *scales = group + 2 * part_bytes<FMT, D>();
        if constexpr (V) {
            unsigned char *to = group + part_bytes<FMT, D>();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int place = (first_pair(block, quad) + i) * GROUP + t;
                if constexpr (FMT == REC_MX4) to[place] = (unsigned char)(pair[0] >> (8 * i));
                else *reinterpret_cast<unsigned short *>(to + 2 * place) = (unsigned short)(pair[i / 2] >> (16 * (i & 1)));
            }
            if (quad == 0) scales[GROUP * (D / BLOCK) + block * GROUP + t] = (unsigned char)byte;
        } else {
            if constexpr (FMT == REC_MX4) *reinterpret_cast<unsigned *>(group + t * CB + 4 * in_row) = codes[0];
            else *reinterpret_cast<u32x2 *>(group + t * CB + 8 * in_row) = codes;
            if (quad == 0) scales[t * (D / BLOCK) + block] = (unsigned char)byte;
        }
    }
};

template <int FMT, int DT, int D>
__global__ __launch_bounds__(THREADS) void write_kernel(Cache c, rec_rows k, rec_rows v, const int64_t *slots, long long tokens)
{
    using W = Writer<FMT, DT, D>;
    constexpr int PASSES = W::PASSES;
    __shared__ u32x4 lds[THREADS / 64][W::PIECES];
    const int lane = threadIdx.x & 63, in_row = lane & (W::LANES - 1);
    const unsigned work = blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6);
    const long long unit = work / (unsigned)c.kv_heads;
    const int head = (int)(work - (unsigned)unit * (unsigned)c.kv_heads);
    if (16 * unit >= tokens) return;
    const W w = {c, lane, in_row, in_row & 3, in_row >> 2, lane / W::LANES, head};
    const bool is_v = blockIdx.y != 0;
    const rec_rows &src = is_v ? v : k;
    const Share s = share_of(slots, tokens, unit, c, lane, head == 0 && !is_v);
    const long long base = 16 * unit - 16;  // entry of the list that lane 0 has
    const long long column = (long long)head * src.head_stride + 8 * in_row;

    if (s.first >= 0) {
        Eight<DT> x[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) x[p].load(src.dev, (base + s.first + PASSES * w.r + p) * src.token_stride + column);
        const long long slot = __shfl(s.slot, s.first);
        unsigned char *group = group_of<FMT>(c, D, slot >> c.page_shift, (int)(slot & ((1 << c.page_shift) - 1)), head);
        if (is_v) w.template group<true>(x, group, base + s.first, lds[threadIdx.x >> 6]);
        else w.template group<false>(x, group, base + s.first, lds[threadIdx.x >> 6]);
    }

    const int count = __popc(s.rest);
    for (int p = 0; p * W::ROWS < count; ++p) {
        const int bit = nth_bit(s.rest, p * W::ROWS + w.r), entry = 16 + max(bit, 0);
        const long long slot = __shfl(s.slot, entry);
        Eight<DT> x = {};
        if (bit >= 0) x.load(src.dev, (base + entry) * src.token_stride + column);
        if (is_v) w.template row<true>(x, bit >= 0, slot, base + entry);
        else w.template row<false>(x, bit >= 0, slot, base + entry);
    }
}

// Eight neighbouring columns of a token's keys.
template <int FMT>
__device__ inline f32x8 eight_keys(const unsigned char *from, float scale)
{
    f32x2 a, b, e, f;
    if constexpr (FMT == REC_MX4) {
        const unsigned w = *reinterpret_cast<const unsigned *>(from);
        a = two_values<FMT, 0>(w);
        b = two_values<FMT, 1>(w);
        e = two_values<FMT, 2>(w);
        f = two_values<FMT, 3>(w);
    } else {
        const u32x2 w = *reinterpret_cast<const u32x2 *>(from);
        a = two_values<FMT, 0>(w[0]);
        b = two_values<FMT, 1>(w[0]);
        e = two_values<FMT, 0>(w[1]);
        f = two_values<FMT, 1>(w[1]);
    }
    return f32x8{a[0], a[1], b[0], b[1], e[0], e[1], f[0], f[1]} * scale;
}

template <int FMT, int DT, int D>
__global__ __launch_bounds__(THREADS) void read_kernel(Cache c, const int64_t *slots, long long tokens, void *k, void *v)
{
    constexpr int LANES = D / 8, ROWS = 64 / LANES, PASSES = GROUP / ROWS;
    constexpr int CB = code_bytes<FMT>(D), PIECES = part_bytes<FMT, D>() / 16 + D / 32;
    __shared__ u32x4 lds[THREADS / 64][PIECES];
    const int lane = threadIdx.x & 63, in_row = lane & (LANES - 1), quad = in_row & 3, block = in_row >> 2, r = lane / LANES;
    const unsigned work = blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6);
    const long long unit = work / (unsigned)c.kv_heads;
    const int head = (int)(work - (unsigned)unit * (unsigned)c.kv_heads);
    if (16 * unit >= tokens) return;
    const bool is_v = blockIdx.y != 0;
    void *out = is_v ? v : k;
    const Share s = share_of(slots, tokens, unit, c, lane, head == 0 && !is_v);
    const long long base = 16 * unit - 16;
    auto store = [&](long long entry, f32x8 x) { store8<DT>(out, ((base + entry) * c.kv_heads + head) * D + 8 * in_row, x); };

    if (s.first >= 0) {
        const long long slot = __shfl(s.slot, s.first);
        unsigned char *group = group_of<FMT>(c, D, slot >> c.page_shift, (int)(slot & ((1 << c.page_shift) - 1)), head);
#pragma unroll
        for (int i = 0; i < (PIECES + 63) / 64; ++i)
            if (64 * i + lane < PIECES) lds[threadIdx.x >> 6][64 * i + lane] = *reinterpret_cast<const u32x4 *>(piece_of<FMT, D>(group, is_v, 64 * i + lane));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const unsigned char *from = reinterpret_cast<const unsigned char *>(lds[threadIdx.x >> 6]), *scales = from + part_bytes<FMT, D>();
        if (!is_v) {
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int t = PASSES * r + p;
                store(s.first + t, eight_keys<FMT>(from + t * CB + in_row * CB / LANES, scale_of(scales[t * (D / BLOCK) + block])));
            }
        } else {
            // A lane's PASSES tokens of its eight rows, one word a row; four lanes share them by halves.
            constexpr int BYTES = PASSES * (FMT == REC_MX4 ? 1 : 2);
            Word<BYTES> word[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                word[i] = *reinterpret_cast<const Word<BYTES> *>(from + (16 * block + 8 * (quad & 1) + i) * (FMT == REC_MX4 ? 16 : 32) + BYTES * r);
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int t = PASSES * r + p;
                const float scale = scale_of(scales[block * GROUP + t]);
                f32x8 x;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const unsigned w = (unsigned)(word[i] >> ((FMT == REC_MX4 ? 8 : 16) * p)) >> ((FMT == REC_MX4 ? 4 : 8) * (quad >> 1));
                    x[i] = two_values<FMT, 0>(w)[0] * scale;
                }
                store(s.first + t, x);
            }
        }
    }

    const unsigned here = (unsigned)min(tokens - 16 * unit, 16ll);  // entries of the list: those without a slot get zeros
    const unsigned none = (unsigned)((__ballot(s.slot < 0)) >> 16) & ((1u << here) - 1u), rest = s.rest | none;
    const int count = __popc(rest);
    for (int p = 0; p * ROWS < count; ++p) {
        const int bit = nth_bit(rest, p * ROWS + r), entry = 16 + max(bit, 0);
        const long long slot = __shfl(s.slot, entry);
        if (bit < 0) continue;
        f32x8 x = {};
        if (slot >= 0) {
            const int at = (int)(slot & ((1 << c.page_shift) - 1)), t = at & 15;
            const unsigned char *group = group_of<FMT>(c, D, slot >> c.page_shift, at, head), *scales = group + 2 * part_bytes<FMT, D>();
            if (!is_v) {
                x = eight_keys<FMT>(group + t * CB + in_row * CB / LANES, scale_of(scales[t * (D / BLOCK) + block]));
            } else {
                const float scale = scale_of(scales[GROUP * (D / BLOCK) + block * GROUP + t]);
                const unsigned char *from = group + part_bytes<FMT, D>();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int place = (16 * block + 8 * (quad & 1) + i) * GROUP + t;
                    const unsigned w = FMT == REC_MX4 ? from[place] : *reinterpret_cast<const unsigned short *>(from + 2 * place);
                    x[i] = two_values<FMT, 0>(w >> ((FMT == REC_MX4 ? 4 : 8) * (quad >> 1)))[0] * scale;
                }
            }
        }
        store(entry, x);
    }
}

// A word that has been lowered since it was read stays.
__global__ void clear_faults_kernel(unsigned long long *fault, Faults seen)
{
    if (threadIdx.x < REC_FAULT_WORDS) atomicCAS(fault + threadIdx.x, seen.word[threadIdx.x], ~0ull);
}

struct Rows {
    rec_rows k, v;
};

dim3 grid_of(const Cache &c, long long tokens) { return dim3((unsigned)(rows_threads(c, tokens) / THREADS), 2); }

template <int FMT, int DT, int D>
hipError_t write_as(const Cache &c, const Rows &in, const int64_t *slots, long long tokens, hipStream_t s)
{
    hipLaunchKernelGGL((write_kernel<FMT, DT, D>), grid_of(c, tokens), dim3(THREADS), 0, s, c, in.k, in.v, slots, tokens);
    return hipGetLastError();
}

template <int FMT, int DT, int D>
hipError_t read_as(const Cache &c, const int64_t *slots, long long tokens, void *k, void *v, hipStream_t s)
{
    hipLaunchKernelGGL((read_kernel<FMT, DT, D>), grid_of(c, tokens), dim3(THREADS), 0, s, c, slots, tokens, k, v);
    return hipGetLastError();
}

// f(format, type, head_dim) with each a constant.
template <int FMT, int DT, class F>
hipError_t with_dim(int d, const F &f)
{
    using std::integral_constant;
    const integral_constant<int, FMT> fmt;
    const integral_constant<int, DT> dt;
    return d == 32 ? f(fmt, dt, integral_constant<int, 32>()) : d == 64 ? f(fmt, dt, integral_constant<int, 64>()) : f(fmt, dt, integral_constant<int, 128>());
}
template <int FMT, class F>
hipError_t with_type(int dtype, int d, const F &f)
{
    return dtype == REC_F32 ? with_dim<FMT, REC_F32>(d, f) : dtype == REC_F16 ? with_dim<FMT, REC_F16>(d, f) : with_dim<FMT, REC_BF16>(d, f);
}
template <class F>
hipError_t with_all(int format, int dtype, int d, const F &f)
{
    return format == REC_MX4 ? with_type<REC_MX4>(dtype, d, f) : with_type<REC_MX8>(dtype, d, f);
}

}  // namespace

long long rows_threads(const Cache &c, long long tokens)
{
    const long long waves = (tokens + 15) / 16 * c.kv_heads;
    return (waves + THREADS / 64 - 1) / (THREADS / 64) * THREADS;
}

hipError_t launch_write(const Cache &c, int format, int d, const rec_rows &k, const rec_rows &v, int dtype,
                        const int64_t *slots, long long tokens, hipStream_t s)
{
    const Rows in = {k, v};
    return with_all(format, dtype, d, [&](auto fmt, auto dt, auto dim) { return write_as<fmt(), dt(), dim()>(c, in, slots, tokens, s); });
}

hipError_t launch_read(const Cache &c, int format, int d, const int64_t *slots, long long tokens, int dtype,
                       void *k, void *v, hipStream_t s)
{
    return with_all(format, dtype, d, [&](auto fmt, auto dt, auto dim) { return read_as<fmt(), dt(), dim()>(c, slots, tokens, k, v, s); });
}

hipError_t launch_clear_faults(unsigned long long *fault, const Faults &seen, hipStream_t s)
{
    hipLaunchKernelGGL(clear_faults_kernel, dim3(1), dim3(64), 0, s, fault, seen);
    return hipGetLastError();
}

}  // namespace hist
}  // namespace rec
