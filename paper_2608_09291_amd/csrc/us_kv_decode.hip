// us_kv_attend with few query rows: every key and value is read once, for at
// most 16 rows at a time (the query heads of a cache head, and a few tokens).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "us_kv_attend.h"
#include "us_kv_decode.h"

namespace us_kv {
namespace {

constexpr int kThreads = kDecodeThreads, kWaves = kDecodeWaves, kRows = kDecodeRows;

template <int NT, int DT>
__global__ __launch_bounds__(kDecodeThreads, NT > 4 ? 1 : 2) void us_kv_decode_kernel(Args a) {
    decode_rows<kWhole, NT, DT>(a, Others{});
}

// weights[b, hk, j] += sum over the rows of 2^(x_j - m) / l: four keys per thread, and a quarter of a
// tile's rows per wavefront where there are more than two.
__global__ __launch_bounds__(kThreads) void us_kv_weights_saved_kernel(Args a, float *weights, int64_t stride, int shared) {
    __shared__ f32x4 part[kWaves][64];
    const int hk = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int r0, n;
    a.s.rows(b, r0, n);
    const int len = a.s.len(b), total = n * a.G;
    const int j0 = 4 * (shared ? (int)blockIdx.x * 64 + (tid & 63) : (int)blockIdx.x * kThreads + tid);
    if (4 * (int)blockIdx.x * (shared ? 64 : kThreads) >= len) return;         // (the whole workgroup)
    const int64_t bh = (int64_t)b * a.heads + hk;
    f32x4 sum = {0, 0, 0, 0};
    const int first = shared ? 4 * wave : 0, each = shared ? 4 : kRows;
    for (int base = 0; base < total; base += kRows) {
        // (no tile has stored scores of blocks ahead of its first row's window or past its last row's)
        int lo, hi, x;
        a.mask.range(base / a.G, n, len, lo, x);
        a.mask.range((min(base + kRows, total) - 1) / a.G, n, len, x, hi);
        if (j0 < lo / kBlock * kBlock || j0 >= hi) continue;
        const float2 *row_ml = a.sp.ml + 32 * row_block(a, hk, b, r0, base) + base % 32;
        const float *s = a.sp.scores + (bh * a.sp.rows * a.sp.tiles + base) * a.sp.scores_stride + j0;
        const int end = min(first + each, total - base);
#pragma unroll 4
        for (int r = first; r < end; ++r) {
            const f32x4 y = *(const f32x4 *)(s + r * a.sp.scores_stride);
            const float2 ml = row_ml[r];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float e = fmaf(__builtin_amdgcn_exp2f(y[v] - ml.x), ml.y, sum[v]);
                sum[v] = y[v] == -INFINITY ? sum[v] : e;   // (a masked key, whatever the row's sum is)
            }
        }
    }
    if (shared) {
        part[wave][tid & 63] = sum;
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) sum += part[w][tid];
    }
    float *w = weights + bh * stride + j0;
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (j0 + v < len) w[v] += sum[v];
}

}  // namespace

hipError_t launch_decode(int dtype, const Args &a, int batch, hipStream_t stream) {
    return with_row(a.D, [&](auto nt) {
        return with_type(dtype, [&](auto dt) {
            hipLaunchKernelGGL((us_kv_decode_kernel<decltype(nt)::value, decltype(dt)::value>),
                               dim3(a.heads, batch, a.sp.splits * a.sp.tiles), dim3(kThreads), 0, stream, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_weights_saved(const Args &a, int batch, float *weights, int64_t stride, hipStream_t stream) {
    const int shared = (int64_t)a.s.max_new * a.G > 2, keys = 4 * (shared ? 64 : kThreads);
    hipLaunchKernelGGL(us_kv_weights_saved_kernel, dim3((unsigned)((a.s.max_len + keys - 1) / keys), a.heads, batch), dim3(kThreads), 0,
                       stream, a, weights, stride, shared);
    return hipGetLastError();
}

}  // namespace us_kv
