// Quantising keys and values into the paged cache, and reading them back.
//
// Four lanes have a block of 32 columns, eight each: the block's largest magnitude is
// two exchanges away, the scale is its exponent (so scaling is exact and only the
// conversion rounds), and the hardware's scaled conversions make the codes.  Bound by
// the bytes of the uncompressed side.
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

template <int FMT, int DT>
__global__ __launch_bounds__(THREADS) void write_kernel(Cache c, int d, rec_rows k, rec_rows v, const int64_t *slots,
                                                        unsigned rows)
{
    const int lanes = d / 8, in_row = threadIdx.x & (lanes - 1), quad = in_row & 3, block = in_row >> 2;
    const unsigned row = blockIdx.x * (THREADS / lanes) + threadIdx.x / lanes;
    if (row >= rows) return;
    const unsigned token = row / (unsigned)c.kv_heads;
    const int head = (int)(row - token * (unsigned)c.kv_heads);
    const bool is_v = blockIdx.y != 0;
    const long long slot = slots[token];
    if (slot < 0 || slot >> c.page_shift >= c.num_pages) {
        if (slot != -1 && head == 0 && in_row == 0) report(c.fault, REC_FAULT_SLOT, token);
        return;
    }
    const rec_rows &src = is_v ? v : k;
    f32x8 x = load8<DT>(src.dev, token * src.token_stride + head * src.head_stride + 8 * in_row);
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float one = x[i];  // a vector's element is no lvalue to cast the bits of
        most = max(most, __builtin_bit_cast(unsigned, one) & 0x7fffffffu);
    }
    most = max(most, (unsigned)__shfl_xor((int)most, 1));
    most = max(most, (unsigned)__shfl_xor((int)most, 2));
    const unsigned byte = scale_byte<FMT>(most);
    u32x2 codes = {0u, 0u};
    if (byte == 255u) {
        if (quad == 0) report(c.fault, REC_FAULT_VALUE, token);
    } else {
        codes = codes_of<FMT>(x, scale_of(byte));
    }
    const int at = (int)(slot & ((1 << c.page_shift) - 1)), t = at & 15;
    unsigned char *group = group_of<FMT>(c, d, slot >> c.page_shift, at, head);
    unsigned char *scales = group + 2 * GROUP * code_bytes<FMT>(d);
    if (!is_v) {
        unsigned char *to = group + t * code_bytes<FMT>(d) + in_row * (FMT == REC_MX4 ? 4 : 8);
        if constexpr (FMT == REC_MX4) *reinterpret_cast<unsigned *>(to) = codes[0];
        else *reinterpret_cast<u32x2 *>(to) = codes;
        if (quad == 0) scales[t * (d / BLOCK) + block] = (unsigned char)byte;
        return;
    }
    // Elements j and j + 16 of a block are one place of a V row: lanes 0 and 1 have the
    // first of 8 such pairs each, lanes 2 and 3 the second; each lane writes four.
    unsigned char *to = group + GROUP * code_bytes<FMT>(d);
    const int first = 16 * block + 8 * (quad & 1) + 4 * (quad >> 1);
    if constexpr (FMT == REC_MX4) {
        const unsigned other = (unsigned)__shfl_xor((int)codes[0], 2);
        const unsigned lo = quad < 2 ? codes[0] : other >> 16, hi = quad < 2 ? other : codes[0] >> 16;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            to[(first + i) * GROUP + t] = (unsigned char)((lo >> (4 * i) & 15u) | (hi >> (4 * i) & 15u) << 4);
    } else {
        const unsigned other = (unsigned)__shfl_xor((int)(quad < 2 ? codes[1] : codes[0]), 2);
        const unsigned lo = quad < 2 ? codes[0] : other, hi = quad < 2 ? other : codes[1];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<unsigned short *>(to + ((first + i) * GROUP + t) * 2) =
                (unsigned short)((lo >> (8 * i) & 255u) | (hi >> (8 * i) & 255u) << 8);
    }
    if (quad == 0) scales[GROUP * (d / BLOCK) + block * GROUP + t] = (unsigned char)byte;
}

template <int FMT, int DT>
__global__ __launch_bounds__(THREADS) void read_kernel(Cache c, int d, const int64_t *slots, unsigned rows, void *k, void *v)
{
    const int lanes = d / 8, in_row = threadIdx.x & (lanes - 1), quad = in_row & 3, block = in_row >> 2;
    const unsigned row = blockIdx.x * (THREADS / lanes) + threadIdx.x / lanes;
    if (row >= rows) return;
    const unsigned token = row / (unsigned)c.kv_heads;
    const int head = (int)(row - token * (unsigned)c.kv_heads);
    const bool is_v = blockIdx.y != 0;
    const long long slot = slots[token];
    f32x8 x = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (slot < 0 || slot >> c.page_shift >= c.num_pages) {
        if (slot != -1 && head == 0 && in_row == 0) report(c.fault, REC_FAULT_SLOT, token);
    } else {
        const int at = (int)(slot & ((1 << c.page_shift) - 1)), t = at & 15;
        const unsigned char *group = group_of<FMT>(c, d, slot >> c.page_shift, at, head);
        const unsigned char *scales = group + 2 * GROUP * code_bytes<FMT>(d);
        if (!is_v) {
            const float scale = scale_of(scales[t * (d / BLOCK) + block]);
            const unsigned char *from = group + t * code_bytes<FMT>(d) + in_row * (FMT == REC_MX4 ? 4 : 8);
            if constexpr (FMT == REC_MX4) {
                const unsigned w = *reinterpret_cast<const unsigned *>(from);
                const f32x2 a = two_values<FMT, 0>(w), b = two_values<FMT, 1>(w), e = two_values<FMT, 2>(w), f = two_values<FMT, 3>(w);
                x = f32x8{a[0], a[1], b[0], b[1], e[0], e[1], f[0], f[1]} * scale;
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(from);
                const f32x2 a = two_values<FMT, 0>(w[0]), b = two_values<FMT, 1>(w[0]), e = two_values<FMT, 0>(w[1]), f = two_values<FMT, 1>(w[1]);
                x = f32x8{a[0], a[1], b[0], b[1], e[0], e[1], f[0], f[1]} * scale;
            }
        } else {
            const float scale = scale_of(scales[GROUP * (d / BLOCK) + block * GROUP + t]);
            const unsigned char *from = group + GROUP * code_bytes<FMT>(d);
            const int first = 16 * block + 8 * (quad & 1), half = quad >> 1;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at_code = (first + i) * GROUP + t;
                const unsigned w = FMT == REC_MX4 ? from[at_code] : *reinterpret_cast<const unsigned short *>(from + 2 * at_code);
                const f32x2 a = two_values<FMT, 0>(w);
                x[i] = (half ? a[1] : a[0]) * scale;
            }
        }
    }
    store8<DT>(is_v ? v : k, (long long)row * d + 8 * in_row, x);
}

__global__ void clear_faults_kernel(unsigned long long *fault)
{
    if (threadIdx.x < REC_FAULT_WORDS) fault[threadIdx.x] = ~0ull;
}

template <int FMT, int DT>
hipError_t write_as(const Cache &c, int d, const rec_rows &k, const rec_rows &v, const int64_t *slots, unsigned rows, hipStream_t s)
{
    const unsigned per = (unsigned)(THREADS / (d / 8));
    hipLaunchKernelGGL((write_kernel<FMT, DT>), dim3((rows + per - 1) / per, 2), dim3(THREADS), 0, s, c, d, k, v, slots, rows);
    return hipGetLastError();
}

template <int FMT, int DT>
hipError_t read_as(const Cache &c, int d, const int64_t *slots, unsigned rows, void *k, void *v, hipStream_t s)
{
    const unsigned per = (unsigned)(THREADS / (d / 8));
    hipLaunchKernelGGL((read_kernel<FMT, DT>), dim3((rows + per - 1) / per, 2), dim3(THREADS), 0, s, c, d, slots, rows, k, v);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_write(const Cache &c, int format, int d, const rec_rows &k, const rec_rows &v, int dtype,
                        const int64_t *slots, long long tokens, hipStream_t s)
{
    const unsigned rows = (unsigned)(tokens * c.kv_heads);
    if (format == REC_MX4) {
        if (dtype == REC_F32) return write_as<REC_MX4, REC_F32>(c, d, k, v, slots, rows, s);
        if (dtype == REC_F16) return write_as<REC_MX4, REC_F16>(c, d, k, v, slots, rows, s);
        return write_as<REC_MX4, REC_BF16>(c, d, k, v, slots, rows, s);
    }
    if (dtype == REC_F32) return write_as<REC_MX8, REC_F32>(c, d, k, v, slots, rows, s);
    if (dtype == REC_F16) return write_as<REC_MX8, REC_F16>(c, d, k, v, slots, rows, s);
    return write_as<REC_MX8, REC_BF16>(c, d, k, v, slots, rows, s);
}

hipError_t launch_read(const Cache &c, int format, int d, const int64_t *slots, long long tokens, int dtype,
                       void *k, void *v, hipStream_t s)
{
    const unsigned rows = (unsigned)(tokens * c.kv_heads);
    if (format == REC_MX4) {
        if (dtype == REC_F32) return read_as<REC_MX4, REC_F32>(c, d, slots, rows, k, v, s);
        if (dtype == REC_F16) return read_as<REC_MX4, REC_F16>(c, d, slots, rows, k, v, s);
        return read_as<REC_MX4, REC_BF16>(c, d, slots, rows, k, v, s);
    }
    if (dtype == REC_F32) return read_as<REC_MX8, REC_F32>(c, d, slots, rows, k, v, s);
    if (dtype == REC_F16) return read_as<REC_MX8, REC_F16>(c, d, slots, rows, k, v, s);
    return read_as<REC_MX8, REC_BF16>(c, d, slots, rows, k, v, s);
}

hipError_t launch_clear_faults(unsigned long long *fault, hipStream_t s)
{
    hipLaunchKernelGGL(clear_faults_kernel, dim3(1), dim3(64), 0, s, fault);
    return hipGetLastError();
}

}  // namespace hist
}  // namespace rec
