// us_kv_evict: which tokens stay, and their move to new blocks.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "us_kv_common.h"

namespace {

using namespace us_kv;

constexpr int kSelThreads = 1024, kMoveThreads = 256;

// Orders like the weights: a NaN first, both zeros alike.
__device__ inline uint32_t order_of(float w) {
    if (!(w == w)) return 0u;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

// Exclusive sum over the workgroup's threads, and the total.
__device__ inline int scan(int x, int *lds, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(sum, o, 64);
        if (lane >= o) sum += y;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = sum;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) {
        if (w < wave) before += lds[w];
        total += lds[w];
    }
    return before + sum - x;
}

// One workgroup per (head, sequence). The k-th largest weight by its bits, 8 at
// a time from the top: a histogram of the next 8 bits of the weights that agree
// with the bits found so far. Then the positions in order.
__global__ __launch_bounds__(kSelThreads) void us_kv_select_kernel(Seqs s, const float *weights, int64_t w_stride, int keep,
                                                                   int recent, int heads, int32_t *to_lens,
                                                                   float *to_weights, int64_t to_w_stride,
                                                                   int32_t *index) {
    __shared__ int hist[256], lds[16], found[2];
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int len = s.len(b), stay = min(len, keep), late = min(recent, stay), m = len - late, take = stay - late;
    const float *w = weights + ((int64_t)b * heads + h) * w_stride;
    int32_t *idx = index + ((int64_t)b * heads + h) * keep;
    float *ow = to_weights ? to_weights + ((int64_t)b * heads + h) * to_w_stride : nullptr;
    if (h == 0 && tid == 0) to_lens[b] = stay;

    uint32_t bits = 0;                                     // of the smallest weight that stays
    int equal = take;                                      // how many of that weight do
    if (take < m && take > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int i = tid; i < m; i += kSelThreads) {
                const uint32_t u = order_of(w[i]);
                if (shift == 24 || u >> (shift + 8) == bits >> (shift + 8)) atomicAdd(&hist[(u >> shift) & 255u], 1);
            }
            __syncthreads();
            // bin of the equal-th largest: the one before whose larger bins hold fewer
            const int mine = tid < 256 ? hist[255 - tid] : 0;
            int total;
            const int above = scan(mine, lds, total);
            if (mine > 0 && above < equal && above + mine >= equal) {
                found[0] = 255 - tid;
                found[1] = equal - above;
            }
            __syncthreads();
            bits |= (uint32_t)found[0] << shift;
            equal = found[1];
            __syncthreads();
        }
    }
    int put = 0, same = 0;                                 // kept so far; of the smallest weight so far
    for (int i0 = 0; i0 < m; i0 += kSelThreads) {
        const int i = i0 + tid;
        const uint32_t u = i < m && take > 0 ? order_of(w[i]) : 0u;
        const bool all = take == m, eq = i < m && !all && take > 0 && u == bits;
        int n_eq, n_put;
        const int before = scan(eq, lds, n_eq);
        const bool stays = i < m && take > 0 && (all || u > bits || (eq && same + before < equal));
        const int at = put + scan(stays, lds, n_put);
        if (stays) {
            idx[at] = i;
            if (ow) ow[at] = w[i];
        }
        put += n_put;
        same += n_eq;
    }
    for (int i = tid; i < late; i += kSelThreads) {
        idx[take + i] = m + i;
        if (ow) ow[take + i] = w[m + i];
    }
    for (int i = stay + tid; i < keep; i += kSelThreads) {
        idx[i] = -1;
    }
}

// One workgroup per (new block, head, sequence): the 64 tokens that the index names.
template <int NT>
__global__ __launch_bounds__(kMoveThreads) void us_kv_move_kernel(uint8_t *kp, uint8_t *vp, float *ksp, float *vsp, Seqs s,
                                                                  const int32_t *index, int keep, const int32_t *to,
                                                                  int64_t to_stride, int to_width) {
    constexpr int R = 32 * NT, kOct = R / 8;
    __shared__ int64_t from[kBlock];                       // (block, head) of a token, -1: none
    __shared__ int token[kBlock];
    __shared__ float ratio[2][kBlock], scale[2][kBlock];
    const int j = blockIdx.x, h = blockIdx.y, b = blockIdx.z, heads = gridDim.y, tid = threadIdx.x;
    const int id = to[b * to_stride + j];
    const int left = min(min(s.len(b), keep), to_width * kBlock) - j * kBlock;
    if (id < 0 || id >= s.n_blocks || left <= 0) return;
    if (tid < kBlock) {
        int p = tid < left ? index[((int64_t)b * heads + h) * keep + j * kBlock + tid] : -1;
        const int src = p >= 0 ? s.block(b, p / kBlock) : -1;
        const int64_t at = src >= 0 ? (int64_t)src * heads + h : -1;
        from[tid] = at;
        token[tid] = p & (kBlock - 1);
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const float s1 = at >= 0 ? (v ? vsp : ksp)[at] : 0.0f;
            float s2 = s1;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) s2 = fmaxf(s2, __shfl_xor(s2, o, 64));
            ratio[v][tid] = s2 > 0.0f ? s1 / s2 : 0.0f;
            scale[v][tid] = s2;
        }
    }
    __syncthreads();
    const int64_t dst = (int64_t)id * heads + h;
    if (tid == 0) {
        ksp[dst] = scale[0][0];
        vsp[dst] = scale[1][0];
    }
#pragma unroll
    for (int i0 = 0; i0 < NT; ++i0) {
        const int i = tid + kMoveThreads * i0, t = i / kOct, o = i % kOct;
        u32x2 w = {0x80808080u, 0x80808080u}, q = {0, 0};
        if (from[t] >= 0) w = *(const u32x2 *)(kp + from[t] * (kBlock * R) + key_octet(token[t], o));
        const float r = ratio[0][t];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            q[e >> 2] |= (uint32_t)(int)(rintf(code_of(w[e >> 2], e & 3) * r) + 128.0f) << (8 * (e & 3));
        *(u32x2 *)(kp + dst * (kBlock * R) + key_octet(t, o)) = q;
    }
    for (int i = tid; i < 4 * R; i += kMoveThreads) {
        const int d = i >> 2, g = i & 3;
        u32x4 q = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int t = (int)value_token(16 * g + e);
            const float c = from[t] >= 0 ? (float)vp[from[t] * (kBlock * R) + 64 * d + value_place(token[t])] - 128.0f : 0.0f;
            q[e >> 2] |= (uint32_t)(int)(rintf(c * ratio[1][t]) + 128.0f) << (8 * (e & 3));
        }
        *(u32x4 *)(vp + dst * (kBlock * R) + 16 * i) = q;
    }
}

}  // namespace

extern "C" us_status us_kv_evict(const us_kv_cache *cache, const us_kv_seqs *seqs, const float *weights,
                                 int64_t weights_stride, int32_t max_len, int32_t keep, int32_t recent,
                                 const us_kv_kept *to, void *stream) {
    us_status st = check_cache(cache);
    if (st == US_OK) st = check_seqs(seqs);
    if (st != US_OK) return st;
    if (!weights || (uintptr_t)weights % 4 || !to || !to->blocks || !to->lens || !to->index) return US_ERR_ARG;
    if ((uintptr_t)to->blocks % 4 || (uintptr_t)to->lens % 4 || (uintptr_t)to->weights % 4 || (uintptr_t)to->index % 4)
        return US_ERR_ARG;
    if (max_len < 0 || keep < 1 || recent < 0 || recent > keep) return US_ERR_SHAPE;
    const Seqs s = seqs_of(*cache, *seqs, max_len, 0);
    const int most = keep < s.max_len ? keep : s.max_len;
    if (to->width < 1 || to->stride < to->width || (int64_t)to->width * kBlock < most || weights_stride < s.max_len ||
        (to->weights && to->weights_stride < most))
        return US_ERR_SHAPE;
    const hipStream_t q = (hipStream_t)stream;
    hipLaunchKernelGGL(us_kv_select_kernel, dim3(cache->heads, seqs->batch), dim3(kSelThreads), 0, q, s, weights,
                       weights_stride, keep, recent, cache->heads, to->lens, to->weights, to->weights_stride, to->index);
    if (hipGetLastError() != hipSuccess) return US_ERR_DEVICE;
    const hipError_t e = with_row(cache->head_dim, [&](auto nt) {
        hipLaunchKernelGGL((us_kv_move_kernel<decltype(nt)::value>),
                           dim3((most + kBlock - 1) / kBlock, cache->heads, seqs->batch), dim3(kMoveThreads), 0, q, cache->k,
                           cache->v, cache->k_scale, cache->v_scale, s, to->index, keep, to->blocks, to->stride, to->width);
        return hipGetLastError();
    });
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}
