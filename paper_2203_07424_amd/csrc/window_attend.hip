// Attention of whole histories to themselves: a wave a query row, a lane a key.
#include "history.h"

namespace rec {
namespace hist {
namespace {

template <int D, bool BF>
__global__ __launch_bounds__(64) void window_kernel(rec_window w)
{
    __shared__ float qs[D], ps[64];
    using T = std::conditional_t<BF, __bf16, _Float16>;
    const int lane = threadIdx.x;
    const unsigned row = blockIdx.x;
    const int head = (int)(row % (unsigned)w.heads), token = (int)(row / (unsigned)w.heads), kv = head / (w.heads / w.kv_heads);
    int lo = 0, hi = w.batch;  // the last history that starts at or before the token
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (w.dev_offsets[mid] <= token) lo = mid;
        else hi = mid;
    }
    const int start = w.dev_offsets[lo], end = w.dev_offsets[lo + 1];
    if (start < 0 || start > token || end <= token) return;
    const int pos = token - start;
    const T *src = static_cast<const T *>(w.q.dev) + token * w.q.token_stride + head * w.q.head_stride;
    const T *k = static_cast<const T *>(w.k.dev) + start * w.k.token_stride + kv * w.k.head_stride;
    const T *v = static_cast<const T *>(w.v.dev) + start * w.v.token_stride + kv * w.v.head_stride;
    for (int x = lane; x < D; x += 64) qs[x] = (float)src[x];
    __syncthreads();
    float m = -__builtin_inff(), l = 0.0f, o[(D + 63) / 64] = {};
    for (int t0 = 0; t0 <= pos; t0 += 64) {
        const int j = t0 + lane;
        const bool seen = j <= pos && (w.window == 0 || pos - j < w.window || j < w.sinks);
        float x = -__builtin_inff();
        if (seen) {
            float sum = 0.0f;
            for (int e = 0; e < D; ++e) sum += qs[e] * (float)k[j * w.k.token_stride + e];
            x = sum * w.scale;
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
        for (int x2 = 0; x2 < (D + 63) / 64; ++x2) {
            const int el = x2 * 64 + lane;
            float acc = o[x2] * alpha;
            for (int s = 0; s < 64; ++s)
                if ((who >> s & 1) && el < D) acc += ps[s] * (float)v[(t0 + s) * w.v.token_stride + el];
            o[x2] = acc;
        }
        __syncthreads();
    }
    T *out = static_cast<T *>(w.dev_out) + (long long)row * D;
    for (int x2 = 0; x2 < (D + 63) / 64; ++x2)
        if (x2 * 64 + lane < D) out[x2 * 64 + lane] = (T)(o[x2] / l);
}

// Offsets run from 0 to tokens and never decrease.
__global__ __launch_bounds__(256) void check_offsets_kernel(const int32_t *offsets, int batch, long long tokens, unsigned long long *fault)
{
    for (long long b = (long long)blockIdx.x * 256 + threadIdx.x; b < batch; b += 256ll * gridDim.x)
        if (offsets[b] > offsets[b + 1] || (b == 0 && offsets[0] != 0) || (b == batch - 1 && offsets[batch] != tokens))
            report(fault, REC_FAULT_LENGTH, (unsigned long long)b);
}

template <int D>
hipError_t window_as(const rec_window &w, hipStream_t s)
{
    const dim3 grid((unsigned)(w.tokens * w.heads));
    if (w.dtype == REC_BF16) hipLaunchKernelGGL((window_kernel<D, true>), grid, dim3(64), 0, s, w);
    else hipLaunchKernelGGL((window_kernel<D, false>), grid, dim3(64), 0, s, w);
    if (w.dev_fault)
        hipLaunchKernelGGL(check_offsets_kernel, dim3(1), dim3(256), 0, s, w.dev_offsets, w.batch, (long long)w.tokens,
                           reinterpret_cast<unsigned long long *>(w.dev_fault));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_window(const rec_window &w, hipStream_t s)
{
    return w.head_dim == 32 ? window_as<32>(w, s) : w.head_dim == 64 ? window_as<64>(w, s) : window_as<128>(w, s);
}

}  // namespace hist
}  // namespace rec
