// Norms of queries and keys per head, and their rotation by position, in one pass.
//
// A lane has two pieces of 16 bytes of a row, those whose columns are pairs of each other, so that nothing but the
// sum of squares passes between lanes.  A wave has 64 / LANES rows at once: `tokens` of them, the others
// heads of the same token, whose sines and cosines a lane works out once.  Angles are reduced to turns in 64 bits, so
// that positions may be times in seconds.
//
// Bound by memory: every number is read once and written once, past the caches.  65536 events of 40 heads of 128, bf16: 231 us, 5.8 TB/s
// (weights in registers, one row of a lane at a time and through the caches: 331); 81920 of 8 heads of 32, fp32: 39 us, 4.3 TB/s; 256 events: 4.2 us.
#include "history.h"

namespace rec {
namespace hist {
namespace {

typedef double f64;

constexpr int THREADS = 256;
constexpr int CUS = 256;
constexpr int STEPS = 2;  // rows of a lane on their way at once

struct TurnArgs {
    rec_turn t;
    int all;        // heads + kv_heads
    int row_shift;  // rows of a token at once = 1 << row_shift
};

template <int DT>
constexpr int PIECE = DT == REC_F32 ? 4 : 8;  // columns of 16 bytes

template <int DT>
__device__ inline void widen(u32x4 w, float (&x)[PIECE<DT>])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned u = w[i];
        if constexpr (DT == REC_F32) {
            x[i] = __builtin_bit_cast(float, u);
        } else if constexpr (DT == REC_BF16) {
            x[2 * i] = __builtin_bit_cast(float, u << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
        } else {
            typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
            const f16x2 h = __builtin_bit_cast(f16x2, u);
            x[2 * i] = (float)h[0];
            x[2 * i + 1] = (float)h[1];
        }
    }
}

template <int DT>
__device__ inline u32x4 narrow(const float (&x)[PIECE<DT>])
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == REC_F32) {
            w[i] = __builtin_bit_cast(unsigned, x[i]);
        } else if constexpr (DT == REC_BF16) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const bf16x2 h = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
            w[i] = __builtin_bit_cast(unsigned, h);
        } else {
            typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
            const f16x2 h = {(_Float16)x[2 * i], (_Float16)x[2 * i + 1]};
            w[i] = __builtin_bit_cast(unsigned, h);
        }
    }
    return w;
}

template <int DT, int D, bool NEXT>
__global__ __launch_bounds__(THREADS) void rotate_kernel(TurnArgs a)
{
    constexpr int N = PIECE<DT>, LANES = D / (2 * N), ROWS = 64 / LANES, SIZE = DT == REC_F32 ? 4 : 2;
    const int lane = threadIdx.x & 63, j = lane % LANES, row = lane / LANES;
    const int at_once = 1 << a.row_shift, first_head = row & (at_once - 1);
    const long long wave = (long long)blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6);
    const long long token = wave * (ROWS >> a.row_shift) + (row >> a.row_shift);
    const bool there = token < a.t.tokens;
    const int pairs = a.t.pairs;
    const bool turns = N * j < pairs;
    // This lane's two pieces start at these columns.
    const int c0 = turns && !NEXT ? N * j : 2 * N * j, c1 = turns && !NEXT ? pairs + N * j : c0 + N;

    auto is_k = [&](int head) { return head >= a.t.heads; };
    auto row_of = [&](const rec_rows &q, const rec_rows &k, int head) {
        const rec_rows &r = is_k(head) ? k : q;
        return const_cast<char *>(static_cast<const char *>(r.dev)) +
               SIZE * (token * r.token_stride + (is_k(head) ? head - a.t.heads : head) * r.head_stride);
    };
    // Weights of queries and keys, ones where there are none, in LDS: in registers they would take as many as the rows on their way.
    __shared__ float weights[2][D];
    for (int i = threadIdx.x; i < 2 * D; i += THREADS) {
        const float *w = i < D ? a.t.dev_q_weight : a.t.dev_k_weight;
        weights[0][i] = w ? w[i % D] : 1.0f;
    }
    u32x4 raw[STEPS][2];
    auto load = [&](int from) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int head = from + s * at_once;
            if (there && head < a.all) {
                const char *p = row_of(a.t.q, a.t.k, head);
                raw[s][0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p + SIZE * c0));
                raw[s][1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p + SIZE * c1));
            }
        }
    };
    load(first_head);
    __syncthreads();

    float cosine[N], sine[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        cosine[i] = 1.0f;
        sine[i] = 0.0f;
    }
    if (there && turns) {
        const f64 p = a.t.wide ? (f64) static_cast<const int64_t *>(a.t.dev_positions)[token] : (f64) static_cast<const int32_t *>(a.t.dev_positions)[token];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            f64 turn = p * a.t.dev_frequencies[N * j + i] * 0.15915494309189533577;  // 1 / (2 pi)
            turn -= __builtin_rint(turn);
            sincospif(2.0f * (float)turn, &sine[i], &cosine[i]);
        }
    }
    for (int from = first_head;; from += STEPS * at_once) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int head = from + s * at_once;
            const bool mine = there && head < a.all;
            float x[2][N];
            widen<DT>(mine ? raw[s][0] : u32x4{0u, 0u, 0u, 0u}, x[0]);
            widen<DT>(mine ? raw[s][1] : u32x4{0u, 0u, 0u, 0u}, x[1]);
            const bool normed = (is_k(head) ? a.t.dev_k_weight : a.t.dev_q_weight) != nullptr;
            float sum = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < N; ++i) sum = __builtin_fmaf(x[h][i], x[h][i], sum);
#pragma unroll
            for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
            const float mean = sum * (1.0f / D) + a.t.eps;
            // Outside this range squares have overflowed, or may have vanished; NaN too.
            const bool fine = !normed || (mean > 1e-28f && mean < 1e36f);
            const float by = normed ? __builtin_amdgcn_rsqf(mean) : 1.0f;
            if (__any(mine && !fine)) {
                f64 wide = 0.0;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < N; ++i) wide = __builtin_fma((f64)x[h][i], (f64)x[h][i], wide);
#pragma unroll
                for (int d = 1; d < LANES; d *= 2) wide += __shfl_xor(wide, d);
                const f64 up = 1.0 / __builtin_sqrt(wide / D + (f64)a.t.eps);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < N; ++i) x[h][i] = fine ? x[h][i] * by : (float)((f64)x[h][i] * up);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < N; ++i) x[h][i] *= by;
            }
            float y[2][N];
            const float *w = weights[is_k(head) ? 1 : 0];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[0][i] *= w[c0 + i];
                x[1][i] *= w[c1 + i];
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (NEXT) {
                    // Pairs i of this lane: columns 2 i and 2 i + 1 of its 2 N.
                    const int h = 2 * i / N, c = 2 * i % N;
                    const float u = x[h][c], v = x[h][c + 1];
                    y[h][c] = turns ? u * cosine[i] - v * sine[i] : u;
                    y[h][c + 1] = turns ? u * sine[i] + v * cosine[i] : v;
                } else {
                    const float u = x[0][i], v = x[1][i];
                    y[0][i] = turns ? u * cosine[i] - v * sine[i] : u;
                    y[1][i] = turns ? u * sine[i] + v * cosine[i] : v;
                }
            }
            if (mine) {
                char *p = row_of(a.t.q_out, a.t.k_out, head);
                __builtin_nontemporal_store(narrow<DT>(y[0]), reinterpret_cast<u32x4 *>(p + SIZE * c0));
                __builtin_nontemporal_store(narrow<DT>(y[1]), reinterpret_cast<u32x4 *>(p + SIZE * c1));
            }
        }
        if (from - first_head + STEPS * at_once >= a.all) break;
        load(from + STEPS * at_once);
    }
}

// Rows of a wave, and how a launch deals them.
int rows_of(const rec_turn &t) { return 64 * 2 * (t.dtype == REC_F32 ? PIECE<REC_F32> : PIECE<REC_F16>) / t.head_dim; }

struct Deal {
    int shift;  // rows of a token beside each other, as a power of two
    long long blocks;
};

Deal deal_of(const rec_turn &t)
{
    // As few as leave no lane idle, as sines are then worked out least often, unless there are few waves: 4096 events of 10 heads of 64 5.6 us,
    // 7.5 with all rows of a token beside each other, 9.6 with one; 81920 of 8 of 32 29.6, 29.5 and 44.9.
    const int rows = rows_of(t), all = t.heads + t.kv_heads;
    const auto waves = [&](int shift) { return (t.tokens + (rows >> shift) - 1) / (rows >> shift); };
    int shift = 0;
    while ((1 << shift) < rows && (1 << shift) < all && ((all & (1 << shift)) == 0 || waves(shift) < 4 * CUS)) ++shift;
    return {shift, (waves(shift) + THREADS / 64 - 1) / (THREADS / 64)};
}

template <int DT, int D>
hipError_t rotate_as(const TurnArgs &a, long long blocks, hipStream_t s)
{
    if (a.t.interleaved) hipLaunchKernelGGL((rotate_kernel<DT, D, true>), dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((rotate_kernel<DT, D, false>), dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

template <int DT>
hipError_t rotate_of(const TurnArgs &a, long long blocks, hipStream_t s)
{
    return a.t.head_dim == 32 ? rotate_as<DT, 32>(a, blocks, s) : a.t.head_dim == 64 ? rotate_as<DT, 64>(a, blocks, s) : rotate_as<DT, 128>(a, blocks, s);
}

}  // namespace

long long rotate_threads(const rec_turn &t) { return deal_of(t).blocks * THREADS; }

hipError_t launch_rotate(const rec_turn &t, hipStream_t s)
{
    const Deal d = deal_of(t);
    const TurnArgs a = {t, t.heads + t.kv_heads, d.shift};
    return t.dtype == REC_F32 ? rotate_of<REC_F32>(a, d.blocks, s) : t.dtype == REC_F16 ? rotate_of<REC_F16>(a, d.blocks, s) : rotate_of<REC_BF16>(a, d.blocks, s);
}

}  // namespace hist
}  // namespace rec
