// Shared by the kernels of include/rec_history.h: the cache's layout, its number
// formats, and which keys a query sees.
#ifndef REC_HISTORY_INTERNAL_H
#define REC_HISTORY_INTERNAL_H
#include "rec_history.h"
#include "rec_internal.h"

namespace rec {
namespace hist {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int GROUP = 16;  // tokens
constexpr int BLOCK = 32;  // columns of one scale

// Bytes of one token's codes in a K or V part, and of a group, by head_dim.
template <int FMT>
__host__ __device__ constexpr int code_bytes(int d) { return FMT == REC_MX4 ? d / 2 : d; }
template <int FMT>
__host__ __device__ constexpr int group_bytes(int d) { return 2 * GROUP * (code_bytes<FMT>(d) + d / BLOCK); }

// A cache as the kernels get it.
struct Cache {
    unsigned char *pages;
    long long num_pages;
    int page_shift;  // page_tokens = 1 << page_shift
    int kv_heads;
    unsigned long long *fault;
};

// A fault record's words, as they were read.
struct Faults {
    unsigned long long word[REC_FAULT_WORDS];
};

__device__ inline void report(unsigned long long *fault, int word, unsigned long long position)
{
    if (fault) atomicMin(fault + word, position);
}

// The group of `head` that holds place `at` of `page`.
template <int FMT>
__device__ inline unsigned char *group_of(const Cache &c, int d, long long page, int at, int head)
{
    return c.pages + ((((page * c.kv_heads + head) << (c.page_shift - 4)) + (at >> 4)) * (long long)group_bytes<FMT>(d));
}

// 2^(byte - 127), or NaN for 255.
__device__ inline float scale_of(unsigned byte)
{
    return byte == 255u ? __builtin_nanf("") : __builtin_bit_cast(float, byte << 23);
}

// Two codes as floats: mx4 the halves of a byte of `w`, mx8 two bytes of it.
template <int FMT, int AT>
__device__ inline f32x2 two_values(unsigned w)
{
    if constexpr (FMT == REC_MX4) return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, AT);
    else return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, 1.0f, AT != 0);
}

// -inf where bit `bit` of `unseen` is set, else x, in two instructions.  The compiler may not look through
// the bit: it would make a comparison and a selection of it (five a score).
__device__ inline float unless_hidden(float x, unsigned unseen, int bit)
{
    unsigned hide = (unsigned)__builtin_amdgcn_sbfe((int)unseen, bit, 1);
    asm("" : "+v"(hide));
    return __builtin_bit_cast(float, (hide & 0xff800000u) | (~hide & __builtin_bit_cast(unsigned, x)));
}

// Division by a number that the host knows: n / d = n * magic >> shift in 64 bits, for n below
// 2^31.  With d in (2^(k-1), 2^k], 2^(31+k) / d rounded up fits 32 bits and is off by less than
// 2^k / 2^(31+k) of itself.
struct Divider {
    unsigned magic = 0, shift = 0;
    Divider() = default;
    explicit Divider(int d)
    {
        shift = 31 + (d == 1 ? 0 : 32 - __builtin_clz((unsigned)d - 1));
        magic = (unsigned)(((1ull << shift) + d - 1) / d);
    }
    __device__ int of(int n) const { return (int)((unsigned long long)(unsigned)n * magic >> shift); }
};

long long rows_threads(const Cache &c, long long tokens);  // along x, for keys or values
hipError_t launch_write(const Cache &c, int format, int d, const rec_rows &k, const rec_rows &v, int dtype,
                        const int64_t *slots, long long tokens, hipStream_t s);
hipError_t launch_read(const Cache &c, int format, int d, const int64_t *slots, long long tokens, int dtype,
                       void *k, void *v, hipStream_t s);
long long attend_threads(const Cache &c, int format, int d, const rec_query &q);
void attend_form(const Cache &c, int format, int d, const rec_query &q, int32_t (&form)[3]);  // waves of a block, parts, kv heads of a wave
size_t attend_workspace(const Cache &c, int format, int d, const rec_query &q);
hipError_t launch_attend(const Cache &c, int format, int d, const rec_query &q, void *workspace, hipStream_t s);
long long chosen_threads(const Cache &c, int format, int d, const rec_query &q, int count);
size_t chosen_workspace(const Cache &c, int format, int d, const rec_query &q, int count);
hipError_t launch_chosen(const Cache &c, int format, int d, const rec_query &q, const int32_t *chosen, int count, void *workspace, hipStream_t s);
// Sums of rows in parts, [parts][rows][head_dim], and for each a maximum's exponent and the weights' sum, [parts][rows][2].
struct Parts {
    float *o, *ml;
};
struct Prefix {
    const int32_t *pages;
    int width;
    const int32_t *length;
};
// A prefix and histories one behind the other, in one launch: tiles that its waves walk over, and the call.
long long joined_work(const Cache &c, const rec_query &q, int prefix_width);
long long joined_threads(const Cache &c, int format, int d, const rec_query &q, int prefix_width);
size_t joined_workspace(const Cache &c, int format, int d, const rec_query &q, int prefix_width);
int joined_parts(const Cache &c, int format, int d, const rec_query &q, int prefix_width);
hipError_t launch_joined(const Cache &c, int format, int d, const rec_query &q, const Prefix &prefix, void *workspace, hipStream_t s);
// Of a row whose parts are joined; of those, parts of what stands before its history.
constexpr int MOST_PARTS = 64, MOST_BEFORE = 32;
int own_parts(const Cache &c, int format, int d, const rec_query &q);
// Histories behind `before` parts: results if own_parts() is 1, else that many parts more.
hipError_t launch_behind(const Cache &c, int format, int d, const rec_query &q, const Parts &parts, int before, hipStream_t s);
long long shared_threads(const Cache &c, int format, int d, const rec_query &q, int prefix_width);
size_t shared_workspace(const Cache &c, int format, int d, const rec_query &q, int prefix_width);
void shared_form(const Cache &c, int format, int d, const rec_query &q, int prefix_width, int32_t (&form)[3]);
hipError_t launch_shared(const Cache &c, int format, int d, const rec_query &q, const Prefix &prefix, void *workspace, hipStream_t s);
hipError_t launch_means(const Cache &c, int format, int d, const int32_t *which, int pages, void *means, hipStream_t s);
long long means_threads(const Cache &c, int d, int pages);
struct Select {
    const void *means;
    int count, first, last;
    int32_t *chosen;
    unsigned long long *keys;  // a score's, as whole numbers of the same order: [batch * queries * kv_heads][table_width]
};
long long select_threads(const Cache &c, int d, const rec_query &q);
size_t select_workspace(const Cache &c, int d, const rec_query &q, int count);
void select_form(const Cache &c, int d, const rec_query &q, int count, int32_t (&form)[3]);
hipError_t launch_select(const Cache &c, int d, const rec_query &q, const Select &sel, hipStream_t s);
long long window_blocks(const rec_window &w);  // of 256 threads
hipError_t launch_window(const rec_window &w, hipStream_t s);
long long rotate_threads(const rec_turn &t);
hipError_t launch_rotate(const rec_turn &t, hipStream_t s);
hipError_t launch_clear_faults(unsigned long long *fault, const Faults &seen, hipStream_t s);

}  // namespace hist
}  // namespace rec
#endif
