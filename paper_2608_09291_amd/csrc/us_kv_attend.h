// What the attention kernels share: masks, fragments of codes and queries, the
// softmax's conventions, and the joining of a split row.
//
// Mathematics. With query q, key codes c_j and scales s, the score in base 2 is
// x_j = f (q . c_j), f = scale log2(e) s / n, where n is a power of two that
// brings the largest magnitude of q's row to [2^8, 2^9): its float16 form keeps
// 11 bits of every value that matters, whatever the row's range. Codes are
// whole numbers up to 127, exact in float16. The running maximum m, the
// probabilities p_j = 2^(x_j - m + 13) and their sum l are float32; p goes to
// the second product as float16 (the 13 keeps small ones normal), off by 2^-13
// of each on average, below the rounding of a bfloat16 or float16 result.
// Float32 rows carry the rounded-off part of q and p in a second product each,
// which leaves 2^-22. In prompts p is held times the value scale of its block,
// over the row's largest such product (us_kv_prompt.hip): beside it a smaller one
// keeps these bits down to 2^-27 of it, and adds at most 127 2^-38 of it below.
#ifndef UNIONSPARSE_US_KV_ATTEND_H
#define UNIONSPARSE_US_KV_ATTEND_H

#include "us_kv_common.h"
#include "us_kv_rules.h"

namespace us_kv {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLift = 13.0f;                             // log2 of a probability's form at m
constexpr float kLarge = 1024.0f;                          // scores past which the lift is not added to the maximum
constexpr float kSlack = 2.0f;                             // what m may lag behind the maximum: 2^15 at most

// How a launch splits a row's keys, and what it leaves in the workspace: per
// unit (sequence, cache head, row tile) and split, `rows` partial rows of R
// floats, then their (m, l) pairs.
struct Split {
    int32_t chunk, splits, tiles, rows;
    int32_t mix;      // of prompts: units of an XCD whose tiles run side by side; divides their number
    float *part;      // the rows of a split, then their (m, l): rows (R + 2) floats, to a multiple of 4
    int32_t *tickets;
    // For the weights, by cache head and row_block(), 32 rows each; else NULL.
    float2 *ml;       // m and 2^13 / l, apart: the logarithm of l would lose its bits in m; zeros for a row without keys
    int64_t row_blocks;                                    // of a head
    // of prompts: the rows' float16 form by (part, octet, row), and f without the key scale
    f16x8 *qn;
    float *qf;
    // of decode: x_j by (sequence, head, row, key)
    float *scores;
    int64_t scores_stride;
};

// Splits of a tile whose rows see keys [lo, hi).
__device__ inline int splits_of(int lo, int hi, int chunk) {
    return max(((hi + kBlock - 1) / kBlock - lo / kBlock + chunk - 1) / chunk, 1);
}

struct Args {
    const uint8_t *k, *v;
    const float *ks, *vs;
    int32_t heads, D, G, vec;
    float scale;      // log2(e) included
    Seqs s;
    Rows q, out;
    Mask mask;
    Split sp;
};

// 8 codes of two words as float16: byte u beside 0x64 is 1024 + u, and u = c + 128.
__device__ inline f16x8 halves_of(uint32_t w0, uint32_t w1) {
    const uint32_t a[4] = {__builtin_amdgcn_perm(0x64646464u, w0, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, w0, 0x04030402u),
                           __builtin_amdgcn_perm(0x64646464u, w1, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, w1, 0x04030402u)};
    const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    f16x8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f16x2 h = __builtin_bit_cast(f16x2, a[i]) - bias;
        r[2 * i] = h.x;
        r[2 * i + 1] = h.y;
    }
    return r;
}

// x as float16 and, where wanted, what that leaves of it.
template <bool SPLIT>
__device__ inline void halve(const float (&x)[8], f16x8 &hi, f16x8 &lo) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        hi[e] = (_Float16)x[e];
        if constexpr (SPLIT) lo[e] = (_Float16)(x[e] - (float)hi[e]);
    }
}

// The power of two that brings a row whose largest magnitude is mx to
// [2^8, 2^9), and its inverse; NaN for a row that is not finite, as its result
// is to be, and the largest for one of tiny values.
__device__ inline float row_norm(float mx, float &inverse) {
    uint32_t e = __float_as_uint(mx) >> 23;
    const bool finite = e < 255u;
    e = e < 9u ? 9u : e;
    inverse = __uint_as_float((e - 8u) << 23);
    return finite ? __uint_as_float((262u - e) << 23) : __uint_as_float(0x7FC00000u);
}

// Largest magnitude with infinities and NaN as an infinity.
__device__ inline float magnitude(const float (&x)[8], float mx) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float a = fabsf(x[e]);
        mx = a < INFINITY ? fmaxf(mx, a) : INFINITY;
    }
    return mx;
}

// Octets first, first + step, ... of a row as they lie in memory: all loads
// leave before the first is waited for. Past D the row's last values are read
// again, and octet() takes zeros for them.
template <int DT, int N>
struct RowPart {
    typename Type<DT>::T raw[N][8] __attribute__((aligned(16)));
    __device__ void load(const typename Type<DT>::T *p, int first, int step, int D, bool vec) {
        constexpr int ES = sizeof(raw[0][0]);
        if (vec) {
#pragma unroll
            for (int t = 0; t < N; ++t) {
                const typename Type<DT>::T *s = p + min(8 * (first + step * t), D - 8);
                u32x4 w[ES / 2];
#pragma unroll
                for (int z = 0; z < ES / 2; ++z) w[z] = ((const u32x4 *)s)[z];
                __builtin_memcpy(raw[t], w, 8 * ES);
            }
        } else {
#pragma unroll
            for (int t = 0; t < N; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) raw[t][e] = p[min(8 * (first + step * t) + e, D - 1)];
        }
    }
    // Octet o, the t-th that was loaded; `whole`: the row has no values past D.
    __device__ void octet(int t, int o, int D, bool whole, float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = Type<DT>::get(raw[t][e]);
        if (whole) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 8 * o + e < D ? x[e] : 0.0f;
    }
};
template <int DT>
__device__ inline void store_octet_any(typename Type<DT>::T *p, int o, int D, bool vec, const float (&x)[8]) {
    if (vec) store_octet<DT, true>(p, o, D, x);
    else store_octet<DT, false>(p, o, D, x);
}

// What is subtracted of a score: the maximum, or 0 where there is none yet.
__device__ inline float base_of(float m) { return m == -INFINITY ? 0.0f : m; }

// Stores finished values of a row, x / l: an octet, a quad.
template <int DT>
__device__ inline void put_octet(const Args &a, int row, int head, int oct, const float (&x)[8], float l) {
    using T = typename Type<DT>::T;
    float y[8];
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;         // a row without keys gives zeros
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = x[e] * inv;
    store_octet_any<DT>((T *)a.out.data + (int64_t)row * a.out.token_stride + (int64_t)head * a.out.head_stride, oct, a.D, a.vec, y);
}

template <int DT>
__device__ inline void put_quad(const Args &a, int row, int head, int quad, f32x4 x, float l) {
    using T = typename Type<DT>::T;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    T y[4] __attribute__((aligned(4 * sizeof(T))));
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = Type<DT>::put(x[e] * inv);
    T *dst = (T *)a.out.data + (int64_t)row * a.out.token_stride + (int64_t)head * a.out.head_stride + 4 * quad;
    if (a.vec) {
        if (4 * quad < a.D) __builtin_memcpy(__builtin_assume_aligned(dst, 4 * sizeof(T)), y, sizeof(y));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (4 * quad + e < a.D) dst[e] = y[e];
    }
}

__device__ inline float2 ml_of(float m, float l) { return make_float2(base_of(m), l == 0.0f ? 0.0f : 8192.0f / l); }

// Partial results pass from one workgroup to another, on another XCD with an L2
// of its own: they are stored through to memory and loaded past the L2 (sc1, the
// agent's scope). A fence instead writes the whole L2 back and empties it, for
// every workgroup that takes part: 64 sequences of up to 8192 tokens took 442 us
// with fences.
constexpr int kAgent = 16;                                 // the sc1 bit
struct Shared {
    __amdgpu_buffer_rsrc_t r;
    __device__ explicit Shared(float *p) : r(__builtin_amdgcn_make_buffer_rsrc(p, 0, 0x7FFFFFFF, 0x00020000)) {}
    __device__ void put(uint32_t at, f32x4 x) const {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), r, 4 * at, 0, kAgent);
    }
    __device__ f32x4 get(uint32_t at) const {
        return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, 4 * at, 0, kAgent));
    }
    __device__ void put2(uint32_t at, float x, float y) const {
        __builtin_amdgcn_raw_buffer_store_b64((u32x2){__float_as_uint(x), __float_as_uint(y)}, r, 4 * at, 0, kAgent);
    }
    __device__ void get2(uint32_t at, float &x, float &y) const {
        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(r, 4 * at, 0, kAgent);
        x = __uint_as_float(w[0]);
        y = __uint_as_float(w[1]);
    }
};

// Whether this workgroup is the last of `n` to arrive at `ticket`, which the
// last one resets. Every wavefront waits for its stores (to memory, see above)
// before the barrier, and the ticket is drawn after it: the last workgroup's
// loads, after its own second barrier, find what all others stored. Called by
// every thread.
__device__ inline bool last_of(int32_t *ticket, int n, int *lds) {
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const int t = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *lds = t == n - 1;
        if (t == n - 1) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    __asm__ volatile("" ::: "memory");
    return *lds != 0;
}

// Wavefronts of a prompt workgroup, 32 query rows each. Eight share the
// conversion of a block among twice the rows (us, four and eight: 8192 causal
// rows, 32 heads of 128, 639 and 611; 4096 float32 rows, heads of 64, 290 and
// 187, of 128 362 and 310); wider rows take the registers of four.
constexpr int prompt_waves(int row) { return row <= 128 ? 8 : 4; }

// The block of 32 rows that holds row `row` of sequence b, whose first token row is r0 and
// which has a.G rows to a token: every sequence begins a block of its own.
__device__ inline int64_t row_block(const Args &a, int hk, int b, int r0, int row) {
    return hk * a.sp.row_blocks + (int64_t)r0 * a.G / 32 + b + row / 32;
}

// The tickets, which have to be zero between calls, have a place of their own at
// a workspace's start, that no other part of any attention call takes.
constexpr int64_t kTickets = 16384;

// What an attention call launches, and where its parts of the workspace lie (bytes).
struct Plan {
    bool decode;
    int chunk, splits, tiles, rows, mix;
    int64_t scores_stride;
    int64_t row_blocks;
    size_t part, ml, qf, qn, scores, total;
};

__host__ __device__ inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

us_status check_opts(const us_kv_cache *c, const us_kv_seqs *s, int q_heads, const us_kv_attend_opts &o);
us_status plan_of(const us_kv_cache &c, const us_kv_seqs &s, int q_heads, int tokens, bool f32, const us_kv_attend_opts &o,
                  Plan &p);

hipError_t launch_decode(int dtype, const Args &a, int batch, hipStream_t stream);
hipError_t launch_prompt(int dtype, const Args &a, int batch, hipStream_t stream);
// Adds the probabilities up: from the scores that decode left, or by the scores' product again.
hipError_t launch_weights_saved(const Args &a, int batch, float *weights, int64_t stride, hipStream_t stream);
hipError_t launch_weights(int dtype, const Args &a, int batch, float *weights, int64_t stride, hipStream_t stream);

}  // namespace us_kv

#endif  // UNIONSPARSE_US_KV_ATTEND_H
