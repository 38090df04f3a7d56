// us_kv_attend: softmax attention over the 8-bit cache.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "us_kv_common.h"

namespace {

using namespace us_kv;

struct Mask {
    int32_t causal, window;
    // Keys [lo, hi) that query i of n of a sequence of len tokens sees.
    __device__ void range(int i, int n, int len, int &lo, int &hi) const {
        lo = 0;
        hi = len;
        if (causal) {
            const int at = len - n + i;
            hi = max(at + 1, 0);
            lo = window > 0 ? max(at - window + 1, 0) : 0;
        }
    }
};

// One wavefront per (query head, query row): 64 keys at a time, a lane per key
// for the scores, a lane per value for the sum.
template <int NT, int DT>
__global__ __launch_bounds__(64) void us_kv_attend_kernel(const uint8_t *kp, const uint8_t *vp, const float *ksp,
                                                          const float *vsp, int heads, int D, Seqs s, Rows qr, Rows outr,
                                                          int q_heads, Mask mask, float scale, float *lse) {
    using T = typename Type<DT>::T;
    constexpr int R = 32 * NT;
    __shared__ float q[R], p[64];
    const int h = blockIdx.x, b = blockIdx.z, lane = threadIdx.x, hk = h / (q_heads / heads);
    int r0, n;
    s.rows(b, r0, n);
    const int i = blockIdx.y;
    if (i >= n) return;
    const int len = s.len(b);
    const T *src = (const T *)qr.data + (int64_t)(r0 + i) * qr.token_stride + (int64_t)h * qr.head_stride;
    for (int d = lane; d < R; d += 64) q[d] = d < D ? Type<DT>::get(src[d]) : 0.0f;
    __syncthreads();
    int lo, hi;
    mask.range(i, n, len, lo, hi);
    float m = -INFINITY, l = 0.0f, o[R / 64 + 1] = {};
    for (int blk = lo / kBlock; blk * kBlock < hi; ++blk) {
        const int id = s.block(b, blk), j = blk * kBlock + lane;
        if (id < 0) continue;
        const int64_t at = (int64_t)id * heads + hk;
        const uint8_t *k = kp + at * (kBlock * R), *v = vp + at * (kBlock * R);
        float dot = 0.0f;
        for (int oct = 0; oct < R / 8; ++oct) {
            const u32x2 w = *(const u32x2 *)(k + key_octet(lane, oct));
#pragma unroll
            for (int e = 0; e < 8; ++e) dot += code_of(w[e >> 2], e & 3) * q[8 * oct + e];
        }
        const float x = j >= lo && j < hi ? dot * (ksp[at] * scale) : -INFINITY;
        float top = x;
#pragma unroll
        for (int w = 32; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor(top, w, 64));
        const float m2 = fmaxf(m, top);
        const float to = m2 == -INFINITY ? 0.0f : m2;      // (nothing seen yet, or NaN)
        const float a = exp2f(m - to), pj = exp2f(x - to);
        m = m2;
        l = l * a + pj;                                    // (this lane's keys)
        p[lane] = pj;
        __syncthreads();
        const float sv = vsp[at];
        for (int c = 0; c < (R + 63) / 64; ++c) {
            const int d = 64 * c + lane;
            float sum = 0.0f;
            if (d < R)
                for (int t = 0; t < 64; ++t) sum += p[t] * ((float)v[64 * d + value_place(t)] - 128.0f);
            o[c] = o[c] * a + sum * sv;
        }
        __syncthreads();
    }
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) l += __shfl_xor(l, w, 64);
    T *dst = (T *)outr.data + (int64_t)(r0 + i) * outr.token_stride + (int64_t)h * outr.head_stride;
    for (int c = 0; c < (R + 63) / 64; ++c) {
        const int d = 64 * c + lane;
        if (d < D) dst[d] = Type<DT>::put(l == 0.0f ? 0.0f : o[c] / l);
    }
    if (lse && lane == 0) lse[(int64_t)(r0 + i) * q_heads + h] = l == 0.0f ? INFINITY : (m == -INFINITY ? 0.0f : m) + log2f(l);
}

// One wavefront per (64 keys, head, sequence): the probabilities again, from
// the logarithms of their sums.
template <int NT, int DT>
__global__ __launch_bounds__(64) void us_kv_weights_kernel(const uint8_t *kp, const float *ksp, int heads, int D, Seqs s,
                                                           Rows qr, int q_heads, Mask mask, float scale, const float *lse,
                                                           float *weights, int64_t w_stride) {
    using T = typename Type<DT>::T;
    constexpr int R = 32 * NT;
    __shared__ float q[R];
    const int blk = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, lane = threadIdx.x, G = q_heads / heads;
    int r0, n;
    s.rows(b, r0, n);
    const int len = s.len(b), j = blk * kBlock + lane;
    if (blk * kBlock >= len) return;
    const int id = s.block(b, blk);
    if (id < 0) return;
    const int64_t at = (int64_t)id * heads + hk;
    const uint8_t *k = kp + at * (kBlock * R);
    float sum = 0.0f;
    for (int i = 0; i < n; ++i) {
        int lo, hi;
        mask.range(i, n, len, lo, hi);
        if (blk * kBlock >= hi || blk * kBlock + kBlock <= lo) continue;
        for (int g = 0; g < G; ++g) {
            const int h = hk * G + g;
            const T *src = (const T *)qr.data + (int64_t)(r0 + i) * qr.token_stride + (int64_t)h * qr.head_stride;
            __syncthreads();
            for (int d = lane; d < R; d += 64) q[d] = d < D ? Type<DT>::get(src[d]) : 0.0f;
            __syncthreads();
            float dot = 0.0f;
            for (int oct = 0; oct < R / 8; ++oct) {
                const u32x2 w = *(const u32x2 *)(k + key_octet(lane, oct));
#pragma unroll
                for (int e = 0; e < 8; ++e) dot += code_of(w[e >> 2], e & 3) * q[8 * oct + e];
            }
            if (j >= lo && j < hi) sum += exp2f(dot * (ksp[at] * scale) - lse[(int64_t)(r0 + i) * q_heads + h]);
        }
    }
    if (j < len) weights[((int64_t)b * heads + hk) * w_stride + j] += sum;
}

constexpr us_kv_attend_opts kDefault = {0.0f, 1, 0, 0, nullptr, 0};

us_status check_opts(const us_kv_cache *c, const us_kv_seqs *s, int q_heads, const us_kv_attend_opts &o) {
    us_status st = check_cache(c);
    if (st == US_OK) st = check_seqs(s);
    if (st != US_OK) return st;
    if (!(o.scale >= 0.0f && o.scale < INFINITY) || o.causal < 0 || o.causal > 1 || o.window < 0 || (o.window && !o.causal))
        return US_ERR_ARG;
    if ((uintptr_t)o.weights % 4) return US_ERR_ARG;
    if (q_heads < 1 || q_heads % c->heads || q_heads > 65535 || o.max_len < 0) return US_ERR_SHAPE;
    if (o.weights && o.weights_stride < seqs_of(*c, *s, o.max_len, 0).max_len) return US_ERR_SHAPE;
    return US_OK;
}

size_t bytes_needed(int q_heads, int tokens, const us_kv_attend_opts &o) {
    return o.weights ? (size_t)q_heads * (size_t)tokens * 4 : 0;
}

}  // namespace

extern "C" us_status us_kv_attend_workspace_size(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads,
                                                 int32_t tokens, const us_kv_attend_opts *opts, size_t *bytes) {
    const us_kv_attend_opts &o = opts ? *opts : kDefault;
    const us_status st = check_opts(cache, seqs, q_heads, o);
    if (st != US_OK) return st;
    if (!bytes) return US_ERR_ARG;
    if (tokens < 1) return US_ERR_SHAPE;
    *bytes = bytes_needed(q_heads, tokens, o);
    return US_OK;
}

extern "C" us_status us_kv_attend(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads, const us_rows *q,
                                  const us_rows *out, const us_kv_attend_opts *opts, void *ws, size_t ws_bytes,
                                  void *stream) {
    const us_kv_attend_opts &o = opts ? *opts : kDefault;
    us_status st = check_opts(cache, seqs, q_heads, o);
    if (st == US_OK) st = check_rows(q);
    if (st == US_OK) st = check_rows(out);
    if (st != US_OK) return st;
    if (q->dtype != out->dtype) return US_ERR_ARG;
    if (q->tokens != out->tokens) return US_ERR_SHAPE;
    const size_t need = bytes_needed(q_heads, q->tokens, o);
    if (need && (!ws || (uintptr_t)ws % 16 || ws_bytes < need)) return US_ERR_ARG;
    const Seqs s = seqs_of(*cache, *seqs, o.max_len, q->tokens);
    const Mask mask{o.causal, o.window};
    const float scale = (o.scale > 0.0f ? o.scale : 1.0f / sqrtf((float)cache->head_dim)) * 1.44269504f;
    const Rows qr{q->data, q->token_stride, q->head_stride}, outr{out->data, out->token_stride, out->head_stride};
    float *lse = need ? (float *)ws : nullptr;
    if (seqs->max_new > 65535) return US_ERR_SHAPE;
    const hipError_t e = with_row(cache->head_dim, [&](auto nt) {
        return with_type(q->dtype, [&](auto dt) {
            constexpr int NT = decltype(nt)::value, DT = decltype(dt)::value;
            hipLaunchKernelGGL((us_kv_attend_kernel<NT, DT>), dim3(q_heads, seqs->max_new, seqs->batch), dim3(64), 0,
                               (hipStream_t)stream, cache->k, cache->v, cache->k_scale, cache->v_scale, cache->heads,
                               cache->head_dim, s, qr, outr, q_heads, mask, scale, lse);
            hipError_t err = hipGetLastError();
            if (err != hipSuccess || !o.weights) return err;
            hipLaunchKernelGGL((us_kv_weights_kernel<NT, DT>),
                               dim3((s.max_len + kBlock - 1) / kBlock, cache->heads, seqs->batch), dim3(64), 0,
                               (hipStream_t)stream, cache->k, cache->k_scale, cache->heads, cache->head_dim, s, qr, q_heads,
                               mask, scale, lse, o.weights, o.weights_stride);
            return hipGetLastError();
        });
    });
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}
