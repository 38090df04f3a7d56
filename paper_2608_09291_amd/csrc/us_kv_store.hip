// us_kv_append and us_kv_read: between dense rows and the blocks of the cache.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "us_kv_common.h"

namespace {

using namespace us_kv;

constexpr int kThreads = 256;

// Blocks that n consecutive tokens can touch at most, wherever they start.
int touched(int n) { return (n + kBlock - 2) / kBlock + 1; }

__device__ float block_max(float x, float *lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
}

// The byte of rint(x / s), within the codes; an infinity at the end of them, a NaN at zero.
__device__ inline uint32_t byte_of(float x, float s) {
    float q = s > 0.0f ? rintf(x / s) : fabsf(x) == INFINITY ? x : 0.0f;
    q = q == q ? q : 0.0f;
    return (uint32_t)(int)(fminf(fmaxf(q, -127.0f), 127.0f) + 128.0f);
}

// One workgroup per (block that gets new tokens, head, sequence; keys or
// values). It holds the block's new values in registers, so that they are
// read once: their largest magnitude gives the scale, then they are rounded.
template <int NT, int DT, bool VEC>
__global__ __launch_bounds__(kThreads) void us_kv_append_kernel(uint8_t *kp, uint8_t *vp, float *ksp, float *vsp, int D,
                                                                Seqs s, Rows kr, Rows vr) {
    using T = typename Type<DT>::T;
    constexpr int R = 32 * NT, kOct = R / 8;
    __shared__ float red[4];
    __shared__ __attribute__((aligned(16))) uint8_t tile[kBlock * (R + 8)];
    const int b = blockIdx.z, h = blockIdx.y, heads = gridDim.y, tid = threadIdx.x;
    const bool values = blockIdx.x & 1;
    int r0, n;
    s.rows(b, r0, n);
    const int len = s.len(b), p0 = len - n, first = max(p0, 0) / kBlock + (blockIdx.x >> 1);
    const int t0 = max(p0 - first * kBlock, 0), t1 = min(len - first * kBlock, kBlock);
    if (n <= 0 || t1 <= t0) return;
    const int id = s.block(b, first);
    if (id < 0) return;
    const int64_t at = (int64_t)id * heads + h;
    const Rows &rows = values ? vr : kr;
    const T *src = (const T *)rows.data + (int64_t)h * rows.head_stride;

    float x[NT][8], amax = 0.0f;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int i = tid + kThreads * j, t = i / kOct, o = i % kOct;
        if (t >= t0 && t < t1) {
            load_octet<DT, VEC>(src + (int64_t)(r0 + first * kBlock + t - p0) * rows.token_stride, o, D, x[j]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[j][e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = fabsf(x[j][e]);
            amax = fmaxf(amax, a < INFINITY ? a : 0.0f);   // (false for a NaN)
        }
    }
    float *scale = (values ? vsp : ksp) + at;
    const float s1 = t0 > 0 ? *scale : 0.0f;
    amax = block_max(amax, red);
    const float s2 = fmaxf(s1, amax / 127.0f), ratio = s2 > 0.0f ? s1 / s2 : 0.0f;
    if (tid == 0) *scale = s2;
    const bool grown = t0 > 0 && s2 != s1;

    if (!values) {
        uint8_t *dst = kp + at * (kBlock * R);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int i = tid + kThreads * j, t = i / kOct, o = i % kOct;
            u32x2 *p = (u32x2 *)(dst + key_octet(t, o));
            u32x2 w = {0, 0};
            if (t >= t0 && t < t1) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e >> 2] |= byte_of(x[j][e], s2) << (8 * (e & 3));
                *p = w;
            } else if (t < t0 && grown) {
                const u32x2 old = *p;
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e >> 2] |= rescaled((old[e >> 2] >> (8 * (e & 3))) & 255u, ratio) << (8 * (e & 3));
                *p = w;
            }
        }
        return;
    }
    // Values lie across: tokens to LDS, then rows of 64 places out of it.
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int i = tid + kThreads * j, t = i / kOct, o = i % kOct;
        u32x2 w = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2] |= byte_of(x[j][e], s2) << (8 * (e & 3));
        *(u32x2 *)(tile + t * (R + 8) + 8 * o) = w;
    }
    __syncthreads();
    uint8_t *dst = vp + at * (kBlock * R);
    if (t0 > 0 && !grown && t1 - t0 <= 4) {                // a step's token: its bytes alone
        for (int i = tid; i < (t1 - t0) * R; i += kThreads) {
            const int t = t0 + i / R, d = i % R;
            dst[64 * d + value_place(t)] = tile[t * (R + 8) + d];
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < NT / 2 + NT % 2; ++j) {            // 4 R pieces of 16 bytes
        const int i = tid + kThreads * j, d = i >> 2, g = i & 3;
        if (d >= R) break;
        u32x4 *p = (u32x4 *)(dst + 16 * i);
        u32x4 w = {0, 0, 0, 0}, old = {0, 0, 0, 0};
        if (t0 > 0) old = *p;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int t = (int)value_token(16 * g + e);
            const uint32_t was = (old[e >> 2] >> (8 * (e & 3))) & 255u;
            const uint32_t now = t < t0 ? (grown ? rescaled(was, ratio) : was) : tile[t * (R + 8) + d];
            w[e >> 2] |= now << (8 * (e & 3));
        }
        *p = w;
    }
}

template <int NT, int DT, bool VEC>
__global__ __launch_bounds__(kThreads) void us_kv_read_kernel(const uint8_t *kp, const uint8_t *vp, const float *ksp,
                                                              const float *vsp, int D, Seqs s, Rows kr, Rows vr) {
    using T = typename Type<DT>::T;
    constexpr int R = 32 * NT, kOct = R / 8;
    __shared__ __attribute__((aligned(16))) uint8_t tile[kBlock * (R + 8)];
    const int b = blockIdx.z, h = blockIdx.y, heads = gridDim.y, tid = threadIdx.x;
    const bool values = blockIdx.x & 1;
    int r0, n;
    s.rows(b, r0, n);
    // (positions before the sequence's first count as a block of their own sort: they read as zero)
    const int len = s.len(b), p0 = len - n, lead = max(-p0, 0);
    const Rows &rows = values ? vr : kr;
    T *out = (T *)rows.data + (int64_t)h * rows.head_stride;
    if (blockIdx.x < 2) {
        const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int i = tid; i < lead * kOct; i += kThreads)
            store_octet<DT, VEC>(out + (int64_t)(r0 + i / kOct) * rows.token_stride, i % kOct, D, zero);
    }
    const int first = max(p0, 0) / kBlock + (blockIdx.x >> 1);
    const int t0 = max(p0 - first * kBlock, 0), t1 = min(len - first * kBlock, kBlock);
    if (n <= 0 || t1 <= t0) return;
    const int id = s.block(b, first);
    const int64_t at = (int64_t)max(id, 0) * heads + h;
    const float scale = id < 0 ? 0.0f : (values ? vsp : ksp)[at];
    if (values && id >= 0) {
        const u32x4 *src = (const u32x4 *)(vp + at * (kBlock * R));
        for (int i = tid; i < 4 * R; i += kThreads) {
            const u32x4 w = src[i];
            const int d = i >> 2, g = i & 3;
#pragma unroll
            for (int e = 0; e < 16; ++e) tile[value_token(16 * g + e) * (R + 8) + d] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int i = tid + kThreads * j, t = i / kOct, o = i % kOct;
        if (t < t0 || t >= t1) continue;
        u32x2 w = {0x80808080u, 0x80808080u};
        if (id >= 0) w = values ? *(const u32x2 *)(tile + t * (R + 8) + 8 * o) : *(const u32x2 *)(kp + at * (kBlock * R) + key_octet(t, o));
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = code_of(w[e >> 2], e & 3) * scale;
        store_octet<DT, VEC>(out + (int64_t)(r0 + first * kBlock + t - p0) * rows.token_stride, o, D, x);
    }
}

us_status check(const us_kv_cache *c, const us_kv_seqs *s, const us_rows *k, const us_rows *v) {
    us_status st = check_cache(c);
    if (st == US_OK) st = check_seqs(s);
    if (st == US_OK) st = check_rows(k);
    if (st == US_OK) st = check_rows(v);
    if (st != US_OK) return st;
    if (k->dtype != v->dtype) return US_ERR_ARG;
    return k->tokens == v->tokens ? US_OK : US_ERR_SHAPE;
}

}  // namespace

extern "C" int32_t us_kv_row(int32_t head_dim) { return us_kv::row_of(head_dim); }

#define US_KV_STORE(KERNEL)                                                                                            \
    const us_status st = check(cache, seqs, k, v);                                                                     \
    if (st != US_OK) return st;                                                                                        \
    const Seqs s = seqs_of(*cache, *seqs, 0, k->tokens);                                                               \
    const dim3 grid(2 * touched(seqs->max_new), cache->heads, seqs->batch);                                            \
    const Rows kr{k->data, k->token_stride, k->head_stride}, vr{v->data, v->token_stride, v->head_stride};             \
    const bool vec = octets_aligned(*k, cache->head_dim) && octets_aligned(*v, cache->head_dim);                       \
    const hipError_t e = with_row(cache->head_dim, [&](auto nt) {                                                      \
        return with_type(k->dtype, [&](auto dt) {                                                                      \
            const auto go = [&](auto kern) {                                                                           \
                hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, (hipStream_t)stream, cache->k, cache->v,             \
                                   cache->k_scale, cache->v_scale, cache->head_dim, s, kr, vr);                        \
                return hipGetLastError();                                                                              \
            };                                                                                                         \
            return vec ? go(KERNEL<decltype(nt)::value, decltype(dt)::value, true>)                                    \
                       : go(KERNEL<decltype(nt)::value, decltype(dt)::value, false>);                                  \
        });                                                                                                            \
    });                                                                                                                \
    return e == hipSuccess ? US_OK : US_ERR_DEVICE

extern "C" us_status us_kv_append(const us_kv_cache *cache, const us_kv_seqs *seqs, const us_rows *k, const us_rows *v,
                                  void *stream) {
    US_KV_STORE(us_kv_append_kernel);
}

extern "C" us_status us_kv_read(const us_kv_cache *cache, const us_kv_seqs *seqs, const us_rows *k, const us_rows *v,
                                void *stream) {
    US_KV_STORE(us_kv_read_kernel);
}
