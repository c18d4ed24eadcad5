// Attention of whole, ragged histories to themselves, over a window and a few first events.
//
// A block has 128 query rows of one history and kv head (the heads that share it, token
// after token, so that a block spans few positions) and walks over tiles of 32 (head_dim 32: 64)
// keys that some of them sees.  Keys and values have two buffers in LDS: while a tile is computed the
// next one is on its way there.  A wave has 32 rows.
//
// Scores come transposed, S^T = K Q^T (32 x 32 x 16), so that a lane holds 16 scores of
// one row for each half of a tile, and those, exponentiated and narrowed, are the operand of
// O^T += V^T P^T as they stand: k of that product is a key in the order of the registers.
// V^T comes out of LDS by transposing reads (4 keys of a column each), which give just the
// four neighbouring keys that a lane's four neighbouring scores belong to.
//
// LDS rows have no padding; the 16-byte pieces of a row are exchanged by bits of its number
// instead, so that what 16 lanes (keys) or 32 (values) read at once lies in 256 different bytes of
// the 64 banks.
//
// The running maximum moves only when a tile's exceeds it by 2^8 (fp16: 2^4).  Masks are looked at in
// tiles that some row of the wave sees partly, and a masked weight is 0.  Since 0 * NaN is NaN,
// rows whose results are not finite are computed again, from what they see (again()).
//
// Weights are narrowed to the type of the values, by no more than the result is, and summed as narrowed (errors against
// 64 bits, of the outputs' size: 0.0021, with weights in fp32 0.0016).
//
// Bound by matrix instructions and the exponentials between them: 16 histories of 4096 events, 16 heads of 128 over
// 4 kv heads, window 1024 + 4: 557 to 572 us, 860 TFLOP/s, 71 % of a large product of the vendor's library (back to back; with the gaps
// of a trace between launches 587 to 635).  Of 256 ragged ones up to 1000
// events (8 heads of 64, window 200 + 4: 42 us) by masks and exponentials, and the last blocks.  A third
// tile on its way to LDS brought nothing (617 against 604 us in a trace).
#include <algorithm>

#include "history.h"

namespace rec {
namespace hist {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int WAVES = 4, THREADS = 64 * WAVES;
constexpr int WAVE_ROWS = 32, BLOCK_ROWS = WAVE_ROWS * WAVES;

// The largest weight of a row lies between 2^lift and 2^(lift + slack).  bf16 has fp32's exponents, so that a weight's rounding is
// of itself however small it is.  fp16 ends at 2^16 and, in steps of 2^-24, below: there a weight is off by at most 2^-36 of the largest,
// so that 2^25 tokens of least weight are off by no more than the type's own rounding.  (Weights of at most 1 lost what was below
// 2^-25 of the largest, and with it up to all of a result that thousands of small weights make.)
constexpr float lift_of(bool bf) { return bf ? 0.0f : 11.0f; }
constexpr float slack_of(bool bf) { return bf ? 8.0f : 4.0f; }

struct WindowArgs {
    rec_window w;
    int per;  // query heads of a kv head
    Divider by_per;
    int tiles;  // of BLOCK_ROWS, more than there can be
};

__device__ inline float neg_inf() { return -__builtin_inff(); }

template <bool BF>
__device__ inline f32x16 product(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <bool BF>
__device__ inline unsigned pack(float a, float b)
{
    if constexpr (BF) {
        const bf16x2 r = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(unsigned, r);
    } else {
        const f16x2 r = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(unsigned, r);
    }
}

// s + the two numbers of w times `by`.
template <bool BF>
__device__ inline float add_pair(unsigned w, float s, float by = 1.0f)
{
    if constexpr (BF) {
        const bf16x2 both = {(__bf16)by, (__bf16)by};
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), both, s, false);
    } else {
        const f16x2 both = {(_Float16)by, (_Float16)by};
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), both, s, false);
    }
}

// Where a 16-byte piece of a key's row is among the row's: 16 neighbouring rows are read at
// one piece.
template <int D>
__device__ inline int key_place(int row, int piece)
{
    return piece ^ (D == 32 ? (row >> 2) & 3 : D == 64 ? (row >> 1) & 7 : row & 15);
}
// Of a value's: four neighbouring rows (from a multiple of four) are read at four pieces (the same).
template <int D>
__device__ inline int value_place(int row, int piece)
{
    return piece ^ (D == 32 ? 0 : D == 64 ? (row & 2) << 1 : (row & 3) << 2);
}

// The larger of lanes l and l ^ 32.
__device__ inline float larger_half(float x)
{
    const unsigned bits = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}

// 1024 bytes of a buffer to LDS, 16 a lane from where each says.
__device__ inline void to_lds(__amdgpu_buffer_rsrc_t from, int offset, void *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void *)to, 16, offset, 0, 0, 0);
}

// Bits [0, n) of the 28 that a lane's scores of 32 keys take, for any n.
__device__ inline unsigned below(int n) { return (1u << min(max(n, 0), 28)) - 1u; }

// A history's share of the grid starts at this tile: every history has room for its rows'
// tiles between its own start and the next one's, whatever the lengths.  Rows and tiles of a call
// fit 31 bits (launch_window()'s callers see to that).
__device__ inline int first_tile(int offset, int per, int b) { return (int)((unsigned)offset * (unsigned)per / BLOCK_ROWS) + b; }

// A wave's rows once more, of which those in `rows` are stored: numbers of the values that are not finite count as zeros, and
// products of ones, where such a number is and where a row sees its key, tell whose results they are.  A slow path without barriers
// in few registers: 32 columns at a time, flags first, then sums; keys, queries and values straight from memory, values two bytes a
// lane.  Weights are such that no sum of finite numbers overflows, however large they are: at most 2^-40 in bf16, which goes on below.
// 4 histories of 4096 events (16 heads of 128 over 4), one with a NaN value in its first event, that all rows see: 0.33 -> 2.5 ms; 256 of
// 160 events (8 heads of 64) 37 -> 68 us.  (A wave that took a row at a time, key by key: 23 ms and 701 us.)
template <int D, bool BF, typename T>
__device__ inline void again(const WindowArgs &a, int start, int len, int kv, int wave_row, unsigned rows, int lane)
{
    constexpr unsigned TOP = BF ? 0x7f80u : 0x7c00u, ONE = BF ? 0x3f80u : 0x3c00u;
    constexpr float LIFT = BF ? -40.0f : lift_of(false);
    const rec_window &w = a.w;
    const int c = lane & 31, half = lane >> 5, all_rows = len * a.per;
    auto pos_of = [&](int row) { return a.by_per.of(min(row, all_rows - 1)); };
    const int w_lo = pos_of(wave_row), w_hi = pos_of(wave_row + WAVE_ROWS - 1), pos = pos_of(wave_row + c);
    const int head = kv * a.per + min(wave_row + c, all_rows - 1) - pos * a.per;
    const int window = w.window == 0 ? 0x7fffffff : w.window, sinks = w.sinks;
    const T *k_base = static_cast<const T *>(w.k.dev) + (long long)start * w.k.token_stride + (long long)kv * w.k.head_stride;
    const T *v_base = static_cast<const T *>(w.v.dev) + (long long)start * w.v.token_stride + (long long)kv * w.v.head_stride;
    const T *q_row = static_cast<const T *>(w.q.dev) + (long long)(start + pos) * w.q.token_stride + (long long)head * w.q.head_stride + 8 * half;
    T *out = static_cast<T *>(w.dev_out) + ((long long)(start + pos) * w.heads + head) * D + 4 * half;
    const int n_to = w_hi / 32 + 1, n_from = max(w_lo - window + 1, 0) / 32;
    const int n_sink = min((min(sinks, w_hi + 1) + 31) / 32, n_from), count = n_sink + n_to - n_from;
    auto key_of = [&](int n) { return (n < n_sink ? n : n_from + n - n_sink) * 32; };

    // Scores of 32 keys, in powers of two: s[r] is that of key 8 (r / 4) + r % 4 behind key + 4 half.  Bit r of `seen`: the row sees it.
    auto scores = [&](int key, unsigned &seen) {
        const T *k_row = k_base + key * w.k.token_stride + min(c, len - 1 - key) * (int)w.k.token_stride + 8 * half;
        f32x16 s = {};
#pragma unroll 1
        for (int i = 0; i < D; i += 16) s = product<BF>(*reinterpret_cast<const u32x4 *>(k_row + i), *reinterpret_cast<const u32x4 *>(q_row + i), s);
        const int first = key + 4 * half, ahead = max(pos - first, -1);
        const unsigned shown = below(ahead + 1) & (~below(ahead - window + 1) | below(sinks - first));
        seen = (shown & 0xfu) | (shown >> 4 & 0xf0u) | (shown >> 8 & 0xf00u) | (shown >> 12 & 0xf000u);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = unless_hidden(s[r] * (w.scale * 1.44269504088896341f), ~seen, r);
        return s;
    };
    // Numbers of this lane's column in the eight keys that s[8 t ...] belong to; f(finite, bits) of each.
    auto values = [&](int key, int column, int t, auto f) {
        const T *tile = v_base + key * w.v.token_stride + column;
        u32x4 r;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int row = min(16 * t + 8 * (e >> 2) + 4 * half + (e & 3), len - 1 - key);
            const unsigned x = __builtin_bit_cast(unsigned short, tile[row * (int)w.v.token_stride + c]), y = f((x & TOP) != TOP, x);
            r[e >> 1] = e & 1 ? r[e >> 1] | y << 16 : y;
        }
        return r;
    };

#pragma unroll 1
    for (int column = 0; column < D; column += 32) {
        // Bit r: the row sees NaN (or an infinity under a weight of 0), inf, -inf in the column of o[r].
        unsigned nan = 0, up = 0, down = 0;
#pragma unroll 1
        for (int n = 0; n < count; ++n) {
            const int key = key_of(n);
#pragma unroll 1
            for (int t = 0; t < 2; ++t) {
                const u32x4 odd = values(key, column, t, [](bool finite, unsigned x) { return finite ? 0u : x; });
                if (!__any((odd[0] | odd[1] | odd[2] | odd[3]) != 0)) continue;
                unsigned seen, lost = 0;
                {
                    const f32x16 s = scores(key, seen);
#pragma unroll
                    for (int r = 0; r < 16; ++r) lost |= s[r] == neg_inf() ? 1u << r : 0u;
                    lost &= seen;
                }
                // Bits r where a row that sees a key by `keys` sees a number of `which` in it.
                auto meet = [&](auto which, unsigned keys) {
                    u32x4 ones, sees;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        ones[j] = (which(odd[j] & 0xffffu) ? ONE : 0u) | (which(odd[j] >> 16) ? ONE << 16 : 0u);
                        sees[j] = (keys >> (8 * t + 2 * j) & 1u) * ONE | (keys >> (8 * t + 2 * j + 1) & 1u) * (ONE << 16);
                    }
                    const f32x16 met = product<BF>(ones, sees, f32x16{});
                    unsigned bits = 0;
#pragma unroll
                    for (int r = 0; r < 16; ++r) bits |= met[r] != 0.0f ? 1u << r : 0u;
                    __builtin_amdgcn_sched_barrier(0);
                    return bits;
                };
                nan |= meet([](unsigned x) { return (x & 0x7fffu) > TOP; }, seen);
                nan |= meet([](unsigned x) { return x != 0u; }, lost);
                up |= meet([](unsigned x) { return x == TOP; }, seen & ~lost);
                down |= meet([](unsigned x) { return x == (TOP | 0x8000u); }, seen & ~lost);
            }
        }
        nan |= up & down;

        f32x16 o = {};
        float m = neg_inf(), l = 0.0f;
#pragma unroll 1
        for (int n = 0; n < count; ++n) {
            const int key = key_of(n);
            unsigned seen;
            f32x16 s = scores(key, seen);
            float most = neg_inf();
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[r]);
            most = larger_half(most);
            const float next = fmaxf(m, !BF && __builtin_fabsf(most) >= 0x1p20f ? most : most - LIFT);
            const float by = next == neg_inf() ? 0.0f : next, less = m == next ? 1.0f : __builtin_amdgcn_exp2f(m - next);
            m = next;
            l *= less;
            o *= less;
            u32x4 p[2];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i >> 2][i & 3] = pack<BF>(__builtin_amdgcn_exp2f(s[2 * i] - by), __builtin_amdgcn_exp2f(s[2 * i + 1] - by));
                l = add_pair<BF>(p[i >> 2][i & 3], l);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                __builtin_amdgcn_sched_barrier(0);
                o = product<BF>(values(key, column, t, [](bool finite, unsigned x) { return finite ? x : 0u; }), p[t], o);
            }
        }

        l += __shfl_xor(l, 32);
        const float by = 1.0f / l;
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            f32x4 y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[j] = o[r + j] * by;
                if (up >> (r + j) & 1u) y[j] += __builtin_inff();  // NaN where all of the row is
                if (down >> (r + j) & 1u) y[j] -= __builtin_inff();
                if (nan >> (r + j) & 1u) y[j] = __builtin_nanf("");
            }
            if (rows >> c & 1u) *reinterpret_cast<u32x2 *>(out + column + 2 * r) = u32x2{pack<BF>(y[0], y[1]), pack<BF>(y[2], y[3])};
        }
    }
}

// Waves that a SIMD holds: three or five.  (At head_dim 64 the compiler takes 103 registers without the bound, for again();
// four waves instead of five cost 3 %, 43.7 -> 45.1 us.)
template <int D, bool BF>
__global__ __launch_bounds__(THREADS, D == 128 ? 3 : 5) void window_kernel(WindowArgs a)
{
    using T = std::conditional_t<BF, __bf16, _Float16>;
    constexpr int TILE = D == 32 ? 64 : 32, PARTS = TILE / 32;  // keys; every thread fetches 16 bytes of them at least
    constexpr int ROW_BYTES = 2 * D, PIECES = D / 8, LOADS = TILE * PIECES / THREADS;
    __shared__ __attribute__((aligned(16))) unsigned char lds[2][2][TILE * ROW_BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, half = lane >> 5;
    const rec_window &w = a.w;
    const int kv = (int)(blockIdx.x % (unsigned)w.kv_heads);
    // Late rows see most: they start first.
    const int x = a.tiles - 1 - (int)(blockIdx.x / (unsigned)w.kv_heads);

    if (w.dev_fault && blockIdx.x == 0)
        for (int b = threadIdx.x; b < w.batch; b += THREADS)
            if (w.dev_offsets[b] > w.dev_offsets[b + 1] || (b == 0 && w.dev_offsets[0] != 0) || (b == w.batch - 1 && w.dev_offsets[b + 1] != w.tokens))
                report(reinterpret_cast<unsigned long long *>(w.dev_fault), REC_FAULT_LENGTH, (unsigned long long)b);

    // The last history whose tiles start at or before this one.  A lane looks at up to four
    // candidates a step, so that up to 252 histories take one trip to memory.
    const int tokens = (int)w.tokens;
    int b = 0, start = 0, stop = 0;
    for (int n = w.batch;;) {
        const int step = (n + 251) / 252;
        int mine[4] = {}, last = -1;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (64 * i * step <= n) mine[i] = min(max(w.dev_offsets[min(b + (64 * i + lane) * step, w.batch)], 0), tokens);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (64 * i * step < n) {
                const int at = (64 * i + lane) * step;
                last += __popcll(__ballot(at < n && first_tile(mine[i], a.per, b + at) <= x));
            }
        last = max(last, 0);
        b += last * step;
        if (step == 1) {  // the next candidate has where it ends
            auto of = [&](int i) { return __builtin_amdgcn_readlane(i < 64 ? mine[0] : i < 128 ? mine[1] : i < 192 ? mine[2] : mine[3], i & 63); };
            start = of(last);
            stop = of(last + 1);
            break;
        }
        n = min(step, n - last * step);
    }
    b = __builtin_amdgcn_readfirstlane(b);
    const int len = max(stop - start, 0);
    const int first_row = (x - first_tile(start, a.per, b)) * BLOCK_ROWS, all_rows = len * a.per;
    if (first_row < 0 || first_row >= all_rows) return;

    const int window = w.window == 0 ? 0x7fffffff : w.window, sinks = w.sinks;
    auto pos_of = [&](int row) { return a.by_per.of(min(row, all_rows - 1)); };
    const int p_lo = pos_of(first_row), p_hi = pos_of(first_row + BLOCK_ROWS - 1);
    const int wave_row = first_row + wave * WAVE_ROWS;
    const bool busy = wave_row < all_rows;
    const int w_lo = pos_of(wave_row), w_hi = pos_of(wave_row + WAVE_ROWS - 1), pos = pos_of(wave_row + c);
    const int my_head = kv * a.per + min(wave_row + c, all_rows - 1) - pos * a.per;
    const T *k_base = static_cast<const T *>(w.k.dev) + (long long)start * w.k.token_stride + (long long)kv * w.k.head_stride;
    const T *v_base = static_cast<const T *>(w.v.dev) + (long long)start * w.v.token_stride + (long long)kv * w.v.head_stride;
    const T *q_row = static_cast<const T *>(w.q.dev) + (long long)(start + pos) * w.q.token_stride + (long long)my_head * w.q.head_stride;

    u32x4 q[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        q[i] = *reinterpret_cast<const u32x4 *>(q_row + 16 * i + 8 * half);
        if (w.scale < 0.0f) q[i] ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
    }
    // Positive, so that masked scores stay at -inf.
    const float factor = w.scale == 0.0f ? 1.0f : __builtin_fabsf(w.scale) * 1.44269504088896341f;

    const int n_to = p_hi / TILE + 1, n_from = max(p_lo - window + 1, 0) / TILE;
    const int n_sink = min((min(sinks, p_hi + 1) + TILE - 1) / TILE, n_from), count = n_sink + n_to - n_from;
    auto key_of = [&](int n) { return (n < n_sink ? n : n_from + n - n_sink) * TILE; };

    // A tile goes straight to LDS, 1024 bytes an instruction in the order of the lanes: a lane
    // fetches the piece whose place is its own.  Rows behind the history's end come as zeros.
    int k_offset[LOADS], v_offset[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int n = i * THREADS + threadIdx.x, row = n / PIECES, at = n % PIECES;
        k_offset[i] = row * (int)w.k.token_stride * 2 + 16 * key_place<D>(row, at);
        v_offset[i] = row * (int)w.v.token_stride * 2 + 16 * value_place<D>(row, at);
    }
    auto fetch = [&](int key, int buffer) {
        const int rows = min(TILE, len - key);
        const auto rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(k_base + key * w.k.token_stride), 0,
                                                          (int)(2 * (rows - 1) * w.k.token_stride + ROW_BYTES), 0x00020000);
        const auto rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(v_base + key * w.v.token_stride), 0,
                                                          (int)(2 * (rows - 1) * w.v.token_stride + ROW_BYTES), 0x00020000);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int to = 16 * (i * THREADS + 64 * wave);
            to_lds(rk, k_offset[i], &lds[buffer][0][to]);
            to_lds(rv, v_offset[i], &lds[buffer][1][to]);
        }
    };

    f32x16 o[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.0f;
    constexpr float LIFT = lift_of(BF), SLACK = slack_of(BF);
    float m = neg_inf(), l = 0.0f;  // m: the exponent of weight 1, LIFT below the largest score's

    fetch(key_of(0), 0);
    if (w.scale == 0.0f)  // the query counts as zeros; where it is not finite there is no result (0 * inf)
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                l = add_pair<BF>(q[i][j], l, 0.0f);
                q[i][j] = 0u;
            }
    for (int n = 0; n < count; ++n) {
        const int key = key_of(n);
        // This wave's part of tile n has arrived and its reads of the other buffer are done; then
        // so are all waves'.
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (n + 1 < count) fetch(key_of(n + 1), (n + 1) & 1);
        // Something in it for this wave.
        if (busy && key <= w_hi && (key + TILE > w_lo - window + 1 || key < sinks)) {
            const unsigned char *kt = lds[n & 1][0], *vt = lds[n & 1][1];
            f32x16 s[PARTS];
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int u = 0; u < PARTS; ++u) {
                    const u32x4 kk = *reinterpret_cast<const u32x4 *>(kt + (32 * u + c) * ROW_BYTES + 16 * key_place<D>(c, 2 * i + half));
                    s[u] = product<BF>(kk, q[i], i == 0 ? f32x16{} : s[u]);
                }
            const bool whole = key + TILE - 1 <= w_lo && (key > w_hi - window || key + TILE <= sinks);
            if (!whole) {
                // Bit j of a part: this lane's row sees the part's key 4 half + j.
#pragma unroll
                for (int u = 0; u < PARTS; ++u) {
                    const int first = key + 32 * u + 4 * half, ahead = max(pos - first, -1);
                    const unsigned unseen = ~(below(ahead + 1) & (~below(ahead - window + 1) | below(sinks - first)));
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[u][r] = unless_hidden(s[u][r], unseen, 8 * (r >> 2) + (r & 3));
                }
            }
            float most = neg_inf();
#pragma unroll
            for (int u = 0; u < PARTS; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, s[u][r]);
            most = larger_half(most);
            most = most == neg_inf() ? most : most * factor;
            if (__any(most > m + (LIFT + SLACK))) {
                // Scores so large that LIFT would be lost in rounding do without it.
                const float next = fmaxf(m, __builtin_fabsf(most) < 0x1p20f ? most - LIFT : most);
                if (__any(m != neg_inf())) {  // not the first tile
                    const float down = m == next ? 1.0f : __builtin_amdgcn_exp2f(m - next);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) o[i] *= down;
                    l *= down;
                }
                m = next;
            }
            const float by = m == neg_inf() ? 0.0f : m;  // a row that sees nothing yet has weights of 2^(-inf)
#pragma unroll
            for (int u = 0; u < PARTS; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][r], factor, -by));
#pragma unroll
            for (int u = 0; u < PARTS; ++u)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    u32x4 p;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[i] = pack<BF>(s[u][8 * t + 2 * i], s[u][8 * t + 2 * i + 1]);
                        l = add_pair<BF>(p[i], l);
                    }
                    const int row = 32 * u + 16 * t + 4 * half + ((lane & 15) >> 2);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        const int piece = 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
                        const unsigned char *at = vt + row * ROW_BYTES + 16 * value_place<D>(row, piece) + 8 * (lane & 1);
                        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
                        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 8 * ROW_BYTES));
                        const u32x2 lo2 = __builtin_bit_cast(u32x2, lo), hi2 = __builtin_bit_cast(u32x2, hi);
                        o[i] = product<BF>(u32x4{lo2[0], lo2[1], hi2[0], hi2[1]}, p, o[i]);
                    }
                }
        }
    }
    if (!busy) return;

    l += __shfl_xor(l, 32);
    const float by = 1.0f / l;
    float zero = 0.0f;  // NaN once a result is not finite
    const bool real = wave_row + c < all_rows;
    T *out = static_cast<T *>(w.dev_out) + ((long long)(start + pos) * w.heads + my_head) * D;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 y = f32x4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]} * by;
            const u32x2 z = {pack<BF>(y[0], y[1]), pack<BF>(y[2], y[3])};
            zero = add_pair<BF>(z[1], add_pair<BF>(z[0], zero, 0.0f), 0.0f);
            if (real) *reinterpret_cast<u32x2 *>(out + 32 * i + 8 * (r >> 2) + 4 * half) = z;
        }
    unsigned long long odd = __ballot(zero != 0.0f && real);
    if (odd) again<D, BF, T>(a, start, len, kv, wave_row, (unsigned)(odd | odd >> 32), lane);
}

template <int D>
hipError_t window_as(const WindowArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)a.tiles * (unsigned)a.w.kv_heads);
    if (a.w.dtype == REC_BF16) hipLaunchKernelGGL((window_kernel<D, true>), grid, dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((window_kernel<D, false>), grid, dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

}  // namespace

long long window_blocks(const rec_window &w)
{
    return (w.tokens * (w.heads / w.kv_heads) / BLOCK_ROWS + w.batch) * w.kv_heads;
}

hipError_t launch_window(const rec_window &w, hipStream_t s)
{
    WindowArgs a;
    a.w = w;
    a.per = w.heads / w.kv_heads;
    a.tiles = (int)(window_blocks(w) / w.kv_heads);
    a.by_per = Divider(a.per);
    return w.head_dim == 32 ? window_as<32>(a, s) : w.head_dim == 64 ? window_as<64>(a, s) : window_as<128>(a, s);
}

}  // namespace hist
}  // namespace rec
