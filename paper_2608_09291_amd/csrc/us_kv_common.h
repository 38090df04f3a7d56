// What the kernels of the 8-bit key/value cache share: the layout of a block
// (us_kv.h), the caller's tables with their bounds, and rows of three types.
#ifndef UNIONSPARSE_US_KV_COMMON_H
#define UNIONSPARSE_US_KV_COMMON_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "us_kv.h"

namespace us_kv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = US_KV_BLOCK;

inline int row_of(int head_dim) {
    if (head_dim < 1 || head_dim > US_KV_HEAD_DIM_MAX) return 0;
    return head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : head_dim <= 128 ? 128 : head_dim <= 192 ? 192 : 256;
}

// Calls f with std::integral_constant<int, row / 32> for a row of row_of().
template <class F>
inline hipError_t with_row(int head_dim, F f) {
    switch (row_of(head_dim)) {
        case 64: return f(std::integral_constant<int, 2>());
        case 96: return f(std::integral_constant<int, 3>());
        case 128: return f(std::integral_constant<int, 4>());
        case 192: return f(std::integral_constant<int, 6>());
        case 256: return f(std::integral_constant<int, 8>());
    }
    return hipErrorInvalidValue;
}

// First byte of the 8 values 8 o .. 8 o + 7 of token t in a key block.
__device__ inline uint32_t key_octet(uint32_t t, uint32_t o) {
    return 2048u * (o >> 2) + 1024u * (t >> 5) + 64u * (t & 15u) + 16u * (o & 3u) + 8u * ((t >> 4) & 1u);
}
// Place of token t in a value block's row of 64, and the token at place p.
__device__ inline uint32_t value_place(uint32_t t) { return 16u * ((t >> 2) & 3u) + 4u * (t >> 4) + (t & 3u); }
__device__ inline uint32_t value_token(uint32_t p) { return 16u * ((p >> 2) & 3u) + 4u * (p >> 4) + (p & 3u); }

struct Seqs {
    const int32_t *blocks;
    int64_t stride;
    const int32_t *lens, *starts;
    int32_t max_len;  // tokens that a row of the table covers, or the caller's bound if lower
    int32_t max_new, tokens, n_blocks;

    __device__ int len(int b) const { return min(max(lens[b], 0), max_len); }
    // First row and number of rows of sequence b, within the arrays.
    __device__ void rows(int b, int &r0, int &n) const {
        r0 = b;
        n = 1;
        if (starts) {
            r0 = starts[b];
            n = starts[b + 1] - r0;
        }
        // (64 bits: the table may hold anything)
        n = r0 < 0 || r0 >= tokens ? 0 : (int)min((int64_t)max(min(n, max_new), 0), (int64_t)tokens - r0);
    }
    // The block that holds block `i` of sequence b, or -1. i < max_len / 64, rounded up.
    __device__ int valid(int id) const { return id >= 0 && id < n_blocks ? id : -1; }
    __device__ int block(int b, int i) const { return valid(blocks[b * stride + i]); }
};

struct Rows {
    void *data;
    int64_t token_stride, head_stride;
};

// --- values of a row type ----------------------------------------------------

template <int DT>
struct Type;
template <>
struct Type<US_F32> {
    typedef float T;
    static __device__ float get(float x) { return x; }
    static __device__ float put(float x) { return x; }
};
template <>
struct Type<US_BF16> {
    typedef uint16_t T;
    static __device__ float get(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    // round to nearest, halves to even; a NaN stays one
    static __device__ uint16_t put(float x) {
        const __bf16 h = (__bf16)x;
        return __builtin_bit_cast(uint16_t, h);
    }
};
template <>
struct Type<US_F16> {
    typedef uint16_t T;
    static __device__ float get(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ uint16_t put(float x) {
        const _Float16 h = (_Float16)x;
        return __builtin_bit_cast(uint16_t, h);
    }
};

// Calls f with std::integral_constant<int, dtype>.
template <class F>
inline hipError_t with_type(int dtype, F f) {
    if (dtype == US_F32) return f(std::integral_constant<int, US_F32>());
    if (dtype == US_BF16) return f(std::integral_constant<int, US_BF16>());
    return f(std::integral_constant<int, US_F16>());
}

// Whether rows can be moved 8 values (16 or 32 bytes) at a time: whole octets
// and 16-byte alignment of every one.
inline bool octets_aligned(const us_rows &r, int head_dim) {
    const int es = r.dtype == US_F32 ? 4 : 2, m = 16 / es;
    return head_dim % 8 == 0 && (uintptr_t)r.data % 16 == 0 && r.token_stride % m == 0 && r.head_stride % m == 0;
}

// Values 8 o .. 8 o + 7 of a row of D at p, zeros past D.
template <int DT, bool VEC>
__device__ inline void load_octet(const typename Type<DT>::T *p, int o, int D, float (&x)[8]) {
    if constexpr (VEC) {
        if (8 * o >= D) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.0f;
            return;
        }
        if constexpr (DT == US_F32) {
            const float4 a = *(const float4 *)(p + 8 * o), b = *(const float4 *)(p + 8 * o + 4);
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
        } else {
            const u32x4 a = *(const u32x4 *)(p + 8 * o);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = Type<DT>::get((uint16_t)(a[e >> 1] >> (16 * (e & 1))));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 8 * o + e < D ? Type<DT>::get(p[8 * o + e]) : 0.0f;
    }
}

template <int DT, bool VEC>
__device__ inline void store_octet(typename Type<DT>::T *p, int o, int D, const float (&x)[8]) {
    if constexpr (VEC) {
        if (8 * o >= D) return;
        if constexpr (DT == US_F32) {
            *(float4 *)(p + 8 * o) = make_float4(x[0], x[1], x[2], x[3]);
            *(float4 *)(p + 8 * o + 4) = make_float4(x[4], x[5], x[6], x[7]);
        } else {
            u32x4 a;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                a[e] = (uint32_t)Type<DT>::put(x[2 * e]) | (uint32_t)Type<DT>::put(x[2 * e + 1]) << 16;
            *(u32x4 *)(p + 8 * o) = a;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (8 * o + e < D) p[8 * o + e] = Type<DT>::put(x[e]);
    }
}

__device__ inline float code_of(uint32_t word, int byte) { return (float)((word >> (8 * byte)) & 255u) - 128.0f; }

// The byte of rint(c r), rounded once before it, for the code c of a byte; 0 <= r <= 1. Adding
// 1.5 x 2^23 rounds to a whole number, halves to even, and leaves it in the lowest bits.
__device__ inline uint32_t rescaled(uint32_t byte, float r) {
#pragma clang fp contract(off)
    const float x = ((float)byte - 128.0f) * r;
    return (__float_as_uint(x + 12582912.0f) + 128u) & 255u;
}

// --- argument checks ----------------------------------------------------------

inline us_status check_cache(const us_kv_cache *c) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return US_ERR_ARG;
    if ((uintptr_t)c->k % 16 || (uintptr_t)c->v % 16 || (uintptr_t)c->k_scale % 4 || (uintptr_t)c->v_scale % 4)
        return US_ERR_ARG;
    if (c->n_blocks < 1 || c->heads < 1 || c->heads > 65535 || !row_of(c->head_dim)) return US_ERR_SHAPE;
    return US_OK;
}

inline us_status check_seqs(const us_kv_seqs *s) {
    if (!s || !s->blocks || !s->lens || (uintptr_t)s->blocks % 4 || (uintptr_t)s->lens % 4 || (uintptr_t)s->starts % 4)
        return US_ERR_ARG;
    // (so that every grid has fewer than 2^32 threads)
    if (s->batch < 1 || s->batch > 65535 || s->width < 1 || s->width > US_KV_WIDTH_MAX || s->stride < s->width ||
        s->max_new < 1 || s->max_new > US_KV_NEW_MAX || (!s->starts && s->max_new != 1))
        return US_ERR_SHAPE;
    return US_OK;
}

inline us_status check_rows(const us_rows *r) {
    if (!r || !r->data || r->dtype < US_F32 || r->dtype > US_F16) return US_ERR_ARG;
    if ((uintptr_t)r->data % (r->dtype == US_F32 ? 4 : 2)) return US_ERR_ARG;
    if (r->tokens < 1 || r->token_stride < 0 || r->head_stride < 0) return US_ERR_SHAPE;
    return US_OK;
}

inline Seqs seqs_of(const us_kv_cache &c, const us_kv_seqs &s, int max_len, int tokens) {
    const int most = s.width * kBlock;
    return Seqs{s.blocks, s.stride, s.lens, s.starts, max_len > 0 && max_len < most ? max_len : most, s.max_new, tokens,
                c.n_blocks};
}

}  // namespace us_kv

#endif  // UNIONSPARSE_US_KV_COMMON_H
