// Quantising keys and values into the paged cache, and reading them back.
//
// Four lanes have a block of 32 columns, eight each: the block's largest magnitude is
// two exchanges away, the scale is its exponent (so scaling is exact and only the
// conversion rounds), and the hardware's scaled conversions make the codes.  Bound by
// the bytes of the uncompressed side, as long as whole groups are stored as such: values
// lie along the tokens, so a token by itself is a byte in each of D / 2 rows.  A group passes
// through LDS, where the tokens of a lane meet as words.
#include "history.h"

namespace rec {
namespace hist {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

constexpr int THREADS = 256;

template <int DT>
__device__ inline f32x8 load8(const void *p, long long i)
{
    f32x8 r;
    if constexpr (DT == REC_F32) {
        r = *reinterpret_cast<const f32x8 *>(static_cast<const float *>(p) + i);
    } else if constexpr (DT == REC_F16) {
        const f16x8 x = *reinterpret_cast<const f16x8 *>(static_cast<const _Float16 *>(p) + i);
        r = __builtin_convertvector(x, f32x8);
    } else {
        const bf16x8 x = *reinterpret_cast<const bf16x8 *>(static_cast<const __bf16 *>(p) + i);
        r = __builtin_convertvector(x, f32x8);
    }
    return r;
}

template <int DT>
__device__ inline void store8(void *p, long long i, f32x8 x)
{
    if constexpr (DT == REC_F32)
        *reinterpret_cast<f32x8 *>(static_cast<float *>(p) + i) = x;
    else if constexpr (DT == REC_F16)
        *reinterpret_cast<f16x8 *>(static_cast<_Float16 *>(p) + i) = __builtin_convertvector(x, f16x8);
    else
        *reinterpret_cast<bf16x8 *>(static_cast<__bf16 *>(p) + i) = __builtin_convertvector(x, bf16x8);
}

// The scale byte of a block from the bits of its largest magnitude.
template <int FMT>
__device__ inline unsigned scale_byte(unsigned bits)
{
    constexpr int top = FMT == REC_MX4 ? 2 : 8, cap = FMT == REC_MX4 ? 125 : 119;
    constexpr unsigned over = FMT == REC_MX4 ? 0x600000u : 0x680000u;  // 1.75, 1.8125
    if (bits >= 0x7f800000u) return 255u;
    const int e = (int)(bits >> 23) - 127 - top + ((bits & 0x7fffffu) > over ? 1 : 0);
    return (unsigned)(min(max(e, -110), cap) + 127);
}

// Eight codes: mx4 in one word, mx8 in two.
template <int FMT>
__device__ inline u32x2 codes_of(f32x8 x, float scale)
{
    const float most = scale * (FMT == REC_MX4 ? 6.0f : 448.0f);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_fmed3f(x[i], -most, most);
    u32x2 r = {0u, 0u};
    if constexpr (FMT == REC_MX4) {
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r[0], x[0], x[1], scale, 0);
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r[0], x[2], x[3], scale, 1);
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r[0], x[4], x[5], scale, 2);
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r[0], x[6], x[7], scale, 3);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s16x2 w = {0, 0};
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[4 * i], x[4 * i + 1], scale, false);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[4 * i + 2], x[4 * i + 3], scale, true);
            r[i] = __builtin_bit_cast(unsigned, w);
        }
    }
    return r;
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

// Block scale and codes of a lane's eight columns.
template <int FMT>
__device__ inline u32x2 quantise(f32x8 x, unsigned &byte)
{
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float one = x[i];  // a vector's element is no lvalue to cast the bits of
        most = max(most, __builtin_bit_cast(unsigned, one) & 0x7fffffffu);
    }
    most = max(most, (unsigned)__shfl_xor((int)most, 1));
    most = max(most, (unsigned)__shfl_xor((int)most, 2));
    byte = scale_byte<FMT>(most);
    if (byte == 255u) return u32x2{0u, 0u};
    return codes_of<FMT>(x, scale_of(byte));
}

// Elements j and j + 16 of a block are one place of a V row: lanes 0 and 1 of four have the
// first of 8 such pairs each, lanes 2 and 3 the second.  After an exchange each lane has four
// places, first_pair() ...: mx4 a byte each, mx8 two.
__device__ inline int first_pair(int block, int quad) { return 16 * block + 8 * (quad & 1) + 4 * (quad >> 1); }
template <int FMT>
__device__ inline void pairs_of(u32x2 codes, int quad, unsigned (&pair)[4])
{
    if constexpr (FMT == REC_MX4) {
        const unsigned other = (unsigned)__shfl_xor((int)codes[0], 2);
        const unsigned lo = quad < 2 ? codes[0] : other >> 16, hi = quad < 2 ? other : codes[0] >> 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) pair[i] = (lo >> (4 * i) & 15u) | (hi >> (4 * i) & 15u) << 4;
    } else {
        const unsigned other = (unsigned)__shfl_xor((int)(quad < 2 ? codes[1] : codes[0]), 2);
        const unsigned lo = quad < 2 ? codes[0] : other, hi = quad < 2 ? other : codes[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) pair[i] = (lo >> (8 * i) & 255u) | (hi >> (8 * i) & 255u) << 8;
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

template <int FMT, int DT, int D>
__global__ __launch_bounds__(THREADS) void write_kernel(Cache c, rec_rows k, rec_rows v, const int64_t *slots, long long tokens)
{
    constexpr int LANES = D / 8, ROWS = 64 / LANES, PASSES = GROUP / ROWS;  // of a row; rows at once; for 16 rows
    constexpr int CB = code_bytes<FMT>(D), PIECES = part_bytes<FMT, D>() / 16 + D / 32;
    __shared__ u32x4 lds[THREADS / 64][PIECES];
    const int lane = threadIdx.x & 63, in_row = lane & (LANES - 1), quad = in_row & 3, block = in_row >> 2, r = lane / LANES;
    const unsigned work = blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6);
    const long long unit = work / (unsigned)c.kv_heads;
    const int head = (int)(work - (unsigned)unit * (unsigned)c.kv_heads);
    if (16 * unit >= tokens) return;
    const bool is_v = blockIdx.y != 0;
    const rec_rows &src = is_v ? v : k;
    const Share s = share_of(slots, tokens, unit, c, lane, head == 0 && !is_v);
    const long long base = 16 * unit - 16;  // entry of the list that lane 0 has
    const long long column = (long long)head * src.head_stride + 8 * in_row;

    if (s.first >= 0) {
        // A lane has PASSES neighbouring tokens, so that their places in a V row are one word.
        f32x8 x[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) x[p] = load8<DT>(src.dev, (base + s.first + PASSES * r + p) * src.token_stride + column);
        unsigned char *to = reinterpret_cast<unsigned char *>(lds[threadIdx.x >> 6]);
        unsigned long long word[4] = {0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int t = PASSES * r + p;
            unsigned byte;
            const u32x2 codes = quantise<FMT>(x[p], byte);
            if (byte == 255u && quad == 0) report(c.fault, REC_FAULT_VALUE, (unsigned long long)(base + s.first + t));
            if (quad == 0) to[part_bytes<FMT, D>() + (is_v ? block * GROUP + t : t * (D / BLOCK) + block)] = (unsigned char)byte;
            if (is_v) {
                unsigned pair[4];
                pairs_of<FMT>(codes, quad, pair);
#pragma unroll
                for (int i = 0; i < 4; ++i) word[i] |= (unsigned long long)pair[i] << ((FMT == REC_MX4 ? 8 : 16) * p);
            } else if constexpr (FMT == REC_MX4) {
                *reinterpret_cast<unsigned *>(to + t * CB + 4 * in_row) = codes[0];
            } else {
                *reinterpret_cast<u32x2 *>(to + t * CB + 8 * in_row) = codes;
            }
        }
        if (is_v) {
            constexpr int BYTES = PASSES * (FMT == REC_MX4 ? 1 : 2);
            using Word = std::conditional_t<BYTES == 8, unsigned long long,
                                            std::conditional_t<BYTES == 4, unsigned, std::conditional_t<BYTES == 2, unsigned short, unsigned char>>>;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<Word *>(to + (first_pair(block, quad) + i) * (FMT == REC_MX4 ? 16 : 32) + BYTES * r) = (Word)word[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const long long slot = __shfl(s.slot, s.first);
        unsigned char *group = group_of<FMT>(c, D, slot >> c.page_shift, (int)(slot & ((1 << c.page_shift) - 1)), head);
#pragma unroll
        for (int i = 0; i < (PIECES + 63) / 64; ++i)
            if (64 * i + lane < PIECES) *reinterpret_cast<u32x4 *>(piece_of<FMT, D>(group, is_v, 64 * i + lane)) = lds[threadIdx.x >> 6][64 * i + lane];
    }

    const int count = __popc(s.rest);
    for (int p = 0; p * ROWS < count; ++p) {
        const int bit = nth_bit(s.rest, p * ROWS + r), entry = 16 + max(bit, 0);
        const long long slot = __shfl(s.slot, entry);
        f32x8 x = {};
        if (bit >= 0) x = load8<DT>(src.dev, (base + entry) * src.token_stride + column);
        unsigned byte, pair[4];
        const u32x2 codes = quantise<FMT>(x, byte);
        pairs_of<FMT>(codes, quad, pair);
        if (bit < 0) continue;
        if (byte == 255u && quad == 0) report(c.fault, REC_FAULT_VALUE, (unsigned long long)(base + entry));
        const int at = (int)(slot & ((1 << c.page_shift) - 1)), t = at & 15;
        unsigned char *group = group_of<FMT>(c, D, slot >> c.page_shift, at, head);
        unsigned char *scales = group + 2 * part_bytes<FMT, D>();
        if (is_v) {
            unsigned char *to = group + part_bytes<FMT, D>();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int place = (first_pair(block, quad) + i) * GROUP + t;
                if constexpr (FMT == REC_MX4) to[place] = (unsigned char)pair[i];
                else *reinterpret_cast<unsigned short *>(to + 2 * place) = (unsigned short)pair[i];
            }
            if (quad == 0) scales[GROUP * (D / BLOCK) + block * GROUP + t] = (unsigned char)byte;
        } else {
            if constexpr (FMT == REC_MX4) *reinterpret_cast<unsigned *>(group + t * CB + 4 * in_row) = codes[0];
            else *reinterpret_cast<u32x2 *>(group + t * CB + 8 * in_row) = codes;
            if (quad == 0) scales[t * (D / BLOCK) + block] = (unsigned char)byte;
        }
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
            using Word = std::conditional_t<BYTES == 8, unsigned long long,
                                            std::conditional_t<BYTES == 4, unsigned, std::conditional_t<BYTES == 2, unsigned short, unsigned char>>>;
            Word word[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                word[i] = *reinterpret_cast<const Word *>(from + (16 * block + 8 * (quad & 1) + i) * (FMT == REC_MX4 ? 16 : 32) + BYTES * r);
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

__global__ void clear_faults_kernel(unsigned long long *fault)
{
    if (threadIdx.x < REC_FAULT_WORDS) fault[threadIdx.x] = ~0ull;
}

struct Rows {
    rec_rows k, v;
};

dim3 grid_of(const Cache &c, long long tokens)
{
    const long long waves = (tokens + 15) / 16 * c.kv_heads;
    return dim3((unsigned)((waves + THREADS / 64 - 1) / (THREADS / 64)), 2);
}

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

hipError_t launch_clear_faults(unsigned long long *fault, hipStream_t s)
{
    hipLaunchKernelGGL(clear_faults_kernel, dim3(1), dim3(64), 0, s, fault);
    return hipGetLastError();
}

}  // namespace hist
}  // namespace rec
