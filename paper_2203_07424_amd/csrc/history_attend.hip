// Attention over cached histories: a wave a query row, a lane a key.
#include "history.h"

namespace rec {
namespace hist {
namespace {

template <int FMT, int D, bool BF>
__global__ __launch_bounds__(64) void attend_kernel(Cache c, rec_query q)
{
    __shared__ float qs[D], ps[64];
    using T = std::conditional_t<BF, __bf16, _Float16>;
    const int lane = threadIdx.x;
    const unsigned row = blockIdx.x;
    const int head = (int)(row % (unsigned)q.heads), i = (int)(row / (unsigned)q.heads % (unsigned)q.queries);
    const int b = (int)(row / (unsigned)q.heads / (unsigned)q.queries), kv = head / (q.heads / c.kv_heads);
    const T *src = static_cast<const T *>(q.dev_q) + b * q.batch_stride + i * q.query_stride + head * q.head_stride;
    for (int x = lane; x < D; x += 64) qs[x] = (float)src[x];
    __syncthreads();
    int len = q.dev_lengths[b];
    const int most = q.table_width << c.page_shift;
    if (len < 0 || len > most) {
        if (lane == 0) report(c.fault, REC_FAULT_LENGTH, b);
        len = len < 0 ? 0 : most;
    }
    const int pos = q.candidates ? len - 1 : len - q.queries + i;
    float m = -__builtin_inff(), l = 0.0f, o[(D + 63) / 64] = {};
    bool any = false;
    for (int t0 = 0; t0 <= pos; t0 += 64) {
        const int j = t0 + lane;
        bool seen = j <= pos && (q.window == 0 || pos - j < q.window || j < q.sinks);
        long long page = -1;
        if (j < len) {
            const int col = j >> c.page_shift;
            page = q.dev_pages_of[b * q.table_stride + col];
            if (page < 0 || page >= c.num_pages) {
                if (seen) report(c.fault, REC_FAULT_PAGE, (unsigned long long)b * q.table_width + col);
                page = -1;
                seen = false;
            }
        }
        const int at = j & ((1 << c.page_shift) - 1), t = at & 15;
        float x = -__builtin_inff();
        if (seen) {
            const unsigned char *g = group_of<FMT>(c, D, page, at, kv);
            const unsigned char *sc = g + 2 * GROUP * code_bytes<FMT>(D) + t * (D / BLOCK);
            float sum = 0.0f;
            for (int blk = 0; blk < D / BLOCK; ++blk) {
                float part = 0.0f;
                for (int e = 0; e < BLOCK; e += 2) {
                    const int el = blk * BLOCK + e;
                    const unsigned w = FMT == REC_MX4 ? g[t * code_bytes<FMT>(D) + el / 2]
                                                      : *reinterpret_cast<const unsigned short *>(g + t * code_bytes<FMT>(D) + el);
                    const f32x2 two = two_values<FMT, 0>(w);
                    part += qs[el] * two[0] + qs[el + 1] * two[1];
                }
                sum += part * scale_of(sc[blk]);
            }
            x = sum * q.scale;
        }
        float mt = x;
        for (int s = 32; s; s >>= 1) mt = fmaxf(mt, __shfl_xor(mt, s));
        const float mn = fmaxf(m, mt), ref = mn == -__builtin_inff() ? 0.0f : mn;
        const float p = seen ? __expf(x - ref) : 0.0f, alpha = __expf(m - ref);
        m = mn;
        float sum = p;
        for (int s = 32; s; s >>= 1) sum += __shfl_xor(sum, s);
        l = l * alpha + sum;
        ps[lane] = p;
        const unsigned long long who = __ballot(seen);
        any |= who != 0;
        for (int x2 = 0; x2 < (D + 63) / 64; ++x2) {
            const int el = x2 * 64 + lane;
            float acc = o[x2] * alpha;
            for (int s = 0; s < 64; ++s) {
                if (!(who >> s & 1)) continue;
                const long long pg = __shfl(page, s);
                const int a2 = (t0 + s) & ((1 << c.page_shift) - 1), tt = a2 & 15;
                if (el < D) {
                    const unsigned char *g = group_of<FMT>(c, D, pg, a2, kv);
                    const int code = ((el >> 5) * 16 + (el & 15)) * GROUP + tt;
                    const unsigned char *vp = g + GROUP * code_bytes<FMT>(D);
                    const unsigned w = FMT == REC_MX4 ? vp[code] : *reinterpret_cast<const unsigned short *>(vp + 2 * code);
                    const f32x2 two = two_values<FMT, 0>(w);
                    const float sc = scale_of(g[2 * GROUP * code_bytes<FMT>(D) + GROUP * (D / BLOCK) + (el >> 5) * GROUP + tt]);
                    acc += ps[s] * (el & 16 ? two[1] : two[0]) * sc;
                }
            }
            o[x2] = acc;
        }
        __syncthreads();
    }
    T *out = static_cast<T *>(q.dev_out) + (long long)row * D;
    for (int x2 = 0; x2 < (D + 63) / 64; ++x2)
        if (x2 * 64 + lane < D) out[x2 * 64 + lane] = (T)(any ? o[x2] / l : 0.0f);
}

template <int FMT, int D>
hipError_t attend_as(const Cache &c, const rec_query &q, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)q.batch * q.queries * q.heads));
    if (q.dtype == REC_BF16) hipLaunchKernelGGL((attend_kernel<FMT, D, true>), grid, dim3(64), 0, s, c, q);
    else hipLaunchKernelGGL((attend_kernel<FMT, D, false>), grid, dim3(64), 0, s, c, q);
    return hipGetLastError();
}

}  // namespace

size_t attend_workspace(const Cache &, int, int, const rec_query &) { return 0; }

hipError_t launch_attend(const Cache &c, int format, int d, const rec_query &q, void *, hipStream_t s)
{
    if (format == REC_MX4)
        return d == 32 ? attend_as<REC_MX4, 32>(c, q, s) : d == 64 ? attend_as<REC_MX4, 64>(c, q, s) : attend_as<REC_MX4, 128>(c, q, s);
    return d == 32 ? attend_as<REC_MX8, 32>(c, q, s) : d == 64 ? attend_as<REC_MX8, 64>(c, q, s) : attend_as<REC_MX8, 128>(c, q, s);
}

}  // namespace hist
}  // namespace rec
