// us_kv_rotate: norms of query and key heads and their rotation by positions.
//
// A row (a token's head) of D values x becomes n = x w / sqrt(mean x^2 + eps),
// then its pairs (n1, n2) become (n1 cos - n2 sin, n2 cos + n1 sin) of the angle
// sum over the axes of position times frequency. The angle is taken in 64 bits:
// in 32, a position of a million would be off by up to a 32nd of a radian. What is
// left of it after whole quarters of a turn is at most pi / 4, and in float32
// there off by 2^-26 at most.
//
// Bound by memory: every value is read and written once, some ten operations
// each. us on the GPU: 8192 tokens, 64 + 8 heads of 128, normed, bfloat16, 48.8;
// 5007 tokens, 16 + 16 heads of 80, three axes, 14.6; one token of 64 heads 2.9,
// below what a launch takes the host.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "us_device.h"
#include "us_kv_common.h"

namespace {

using namespace us_kv;

constexpr int kThreads = 256;
constexpr int kAngles = 1024;                              // of a workgroup's tokens, at most

struct RotateArgs {
    Rows q, q_out, k, k_out;
    int32_t q_heads, rows, D, tokens;                      // rows of a token: its query and key heads
    const float *freq;
    const int32_t *positions;
    int64_t positions_stride;
    int32_t pairs, axes, offset, norm;
    int32_t group, part;                                   // tokens, and rows of each, that a workgroup takes together
    float eps;
    const float *qw, *kw;
};

// sin and cos by their series, on [-pi/4, pi/4]: the first terms left out are 2e-9 and 1e-10.
__device__ inline float2 turn(double angle) {
    const double turns = angle * 0.15915494309189535;      // 1 / (2 pi)
    const double quarters = rint(4.0 * turns);
    const float x = (float)((turns - 0.25 * quarters) * 6.283185307179586), y = x * x;
    const int q = (int)(quarters - 4.0 * floor(0.25 * quarters));
    const float s = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), 1.0f);
    const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
    const float a = q & 1 ? s : c, b = q & 1 ? c : s;
    return make_float2(q == 1 || q == 2 ? -a : a, q >= 2 ? -b : b);
}

// A lane has 16 values of a row, in two octets: 8 pairs, first members in u and second ones in v, or 16 of
// the values behind the pairs. Slot z's first value and its octets' places:
struct Slot {
    int a, b;                                              // first values of the octets
    int na, nb;                                            // how many of them there are
    __device__ Slot(int z, int D, int P, bool adjacent) {
        const int turned = (P + 7) / 8, rest = 2 * P + 16 * (z - turned);
        const bool pairs = z < turned;
        a = !pairs ? rest : adjacent ? 16 * z : 8 * z;
        b = pairs && !adjacent ? P + a : a + 8;
        const int end = !pairs ? D : adjacent ? 2 * P : P; // of octet a; b's is one further where pairs lie apart
        na = min(max(end - a, 0), 8);
        nb = pairs && !adjacent ? na : min(max(end - b, 0), 8);
    }
};

// An octet as it lies in memory, zeros past its n values.
template <int DT, bool VEC>
struct Octet {
    typename Type<DT>::T raw[8] __attribute__((aligned(16)));
    __device__ void load(const typename Type<DT>::T *p, int n) {
        if constexpr (VEC) {                               // (n is 0 or 8)
            constexpr int N = sizeof(raw) / 16;
            u32x4 w[N];
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = n ? ((const u32x4 *)p)[i] : (u32x4){0, 0, 0, 0};
            __builtin_memcpy(raw, w, sizeof(raw));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) raw[e] = e < n ? p[e] : (typename Type<DT>::T)0;
        }
    }
    __device__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = Type<DT>::get(raw[e]);
    }
    __device__ void put(const float (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) raw[e] = Type<DT>::put(x[e]);
    }
    __device__ void store(typename Type<DT>::T *p, int n) const {
        if constexpr (VEC) {
            constexpr int N = sizeof(raw) / 16;
            u32x4 w[N];
            __builtin_memcpy(w, raw, sizeof(raw));
            // (past the caches: 8192 tokens of 72 heads of 128 take 48.8 us on the GPU, 62 without)
            if (n)
#pragma unroll
                for (int i = 0; i < N; ++i) __builtin_nontemporal_store(w[i], (u32x4 *)p + i);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) p[e] = raw[e];
        }
    }
};

// n weights from w + at on, ones where there are none; n is 0 or 8 if VEC (they may lie at any float's place).
template <bool VEC>
__device__ inline void weights(const float *w, int at, int n, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 1.0f;
    if (!w) return;
    if constexpr (VEC) {
        if (n) __builtin_memcpy(x, w + at, sizeof(x));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) x[e] = w[at + e];
    }
}

// LANES lanes hold a row. A workgroup takes `part` rows of each of `group` tokens: it computes their angles
// together, a thread each, then passes over the rows, as many at a time as it has lanes for; the next pass's
// rows are asked for ahead of this one's arithmetic.
template <int DT, int LANES, bool VEC, bool ADJ>
__global__ __launch_bounds__(kThreads) void us_kv_rotate_kernel(RotateArgs a) {
    using T = typename Type<DT>::T;
    constexpr int kAtOnce = kThreads / LANES;
    __shared__ __attribute__((aligned(16))) float2 angle[kAngles];
    const int tid = threadIdx.x, z = tid % LANES, mine = tid / LANES;
    const int first = blockIdx.y * a.part, part = min(a.part, a.rows - first), P = a.pairs;
    const Slot slot(z, a.D, P, ADJ);
    const bool turns = 8 * z < P;
    // Tokens that a pass takes side by side, and passes over the rows of one.
    const int side = max(kAtOnce / part, 1), passes = (part + kAtOnce - 1) / kAtOnce;
    const int my_token = passes > 1 ? 0 : mine / part, my_row = passes > 1 ? mine : mine - my_token * part;
    const int t0 = blockIdx.x * a.group, n = my_token < side ? min(a.group, a.tokens - t0) : 0;
    const int times = (min(a.group, a.tokens - t0) + side - 1) / side;       // tokens of a pass, one after the other
    Octet<DT, VEC> ra, rb;
    const auto at = [&](const Rows &q, const Rows &k, int t, int row) {
        const int r = first + row;
        const bool key = r >= a.q_heads;
        // (fields selected one by one: a selected struct would be looked up in memory)
        T *data = (T *)(key ? k.data : q.data);
        const int64_t tokens = key ? k.token_stride : q.token_stride, heads = key ? k.head_stride : q.head_stride;
        return data + (int64_t)(t0 + t) * tokens + (int64_t)(key ? r - a.q_heads : r) * heads;
    };
    const auto fetch = [&](int t, int row) {
        if (t >= n || row >= part) return;
        const T *src = at(a.q, a.k, t, row);
        ra.load(src + slot.a, slot.na);
        rb.load(src + slot.b, slot.nb);
    };
    fetch(my_token, my_row);
    float w[2][8];
    const auto get_weights = [&](int row) {
        const float *src = first + row >= a.q_heads ? a.kw : a.qw;
        weights<VEC>(src, slot.a, slot.na, w[0]);
        weights<VEC>(src, slot.b, slot.nb, w[1]);
    };
    if (a.norm) get_weights(my_row);
    for (int i = tid; i < min(a.group, a.tokens - t0) * P; i += kThreads) {
        const int t = i / P, p = i - t * P;
        double sum = 0.0;
        for (int x = 0; x < a.axes; ++x)
            sum += ((double)a.positions[x * a.positions_stride + t0 + t] + a.offset) * (double)a.freq[x * P + p];
        angle[i] = turn(sum);
    }
    __syncthreads();
    for (int i = 0; i < passes * times; ++i) {
        const int pass = i / times, t = (i - pass * times) * side + my_token, row = my_row + pass * kAtOnce;
        float x[2][8];
        ra.get(x[0]);
        rb.get(x[1]);
        const bool last = t + side - my_token >= times * side;               // of its pass
        if (i + 1 < passes * times) fetch(last ? my_token : t + side, last ? row + kAtOnce : row);
        // (the rows of a pass are of queries or keys for all tokens)
        if (a.norm && i > 0 && t == my_token && (first + row >= a.q_heads) != (first + row - kAtOnce >= a.q_heads)) get_weights(row);
        if (t >= n || row >= part) continue;               // (the lanes of a row go together)
        float2 cs[8];
        if (turns) {
#pragma unroll
            for (int e = 0; e < 8; ++e) cs[e] = angle[t * P + min(8 * z + e, P - 1)];
        }
        if (a.norm) {
            float sum = 0.0f;
            const auto add = [&](float unit) {
                sum = 0.0f;
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum = fmaf(x[y][e] * unit, x[y][e] * unit, sum);
#pragma unroll
                for (int w = LANES / 2; w > 0; w >>= 1) sum += __shfl_xor(sum, w, 64);
            };
            add(1.0f);
            float scale = 1.0f / sqrtf(sum / (float)a.D + a.eps);
            if (sum == INFINITY) {                         // of values past 2^63: the same of 2^-64 x
                add(0x1p-64f);
                scale = 0x1p-64f / sqrtf(sum / (float)a.D);
            }
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[y][e] = x[y][e] * scale * w[y][e];
        }
        if (turns) {
            // pair 8 z + e: values e of both octets, or 2 e and 2 e + 1 of the sixteen; values behind the last stay
            // zero, and are not stored
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float &u = ADJ ? x[e >> 2][2 * (e & 3)] : x[0][e], &v = ADJ ? x[e >> 2][2 * (e & 3) + 1] : x[1][e];
                const float n1 = u, n2 = v;
                u = fmaf(n1, cs[e].x, -n2 * cs[e].y);
                v = fmaf(n2, cs[e].x, n1 * cs[e].y);
            }
        }
        T *dst = at(a.q_out, a.k_out, t, row);
        Octet<DT, VEC> out;
        out.put(x[0]);
        out.store(dst + slot.a, slot.na);
        out.put(x[1]);
        out.store(dst + slot.b, slot.nb);
    }
}

us_status check_pair(const us_rows *in, const us_rows *out, int tokens, int dtype) {
    us_status st = check_rows(in);
    if (st == US_OK) st = check_rows(out);
    if (st != US_OK) return st;
    if (in->dtype != dtype || out->dtype != dtype) return US_ERR_ARG;
    return in->tokens == tokens && out->tokens == tokens ? US_OK : US_ERR_SHAPE;
}

// Whether some of an output's rows share memory.
bool rows_meet(const us_rows &r, int heads, int D) {
    const int64_t t = r.token_stride, h = r.head_stride;
    if ((r.tokens > 1 && t < D) || (heads > 1 && h < D)) return true;
    if (r.tokens == 1 || heads == 1) return false;
    const __int128 most = (__int128)t * (r.tokens - 1);    // first value of the last token
    if (t - D >= (__int128)h * (heads - 1) || h - D >= most) return false;
    for (int j = 1; j < heads; ++j) {                      // (head j of a token and the first of the tokens next to it)
        const __int128 at = (__int128)h * j, below = at - at % t, above = below + t;
        if (at - D >= most) return false;
        if ((below > 0 && below <= most && at - below < D) || (above <= most && above - at < D)) return true;
    }
    return false;
}

// Whether an output is its input, and other rows of it.
bool other_rows(const us_rows &in, const us_rows &out, int heads) {
    return in.data == out.data && ((in.tokens > 1 && in.token_stride != out.token_stride) || (heads > 1 && in.head_stride != out.head_stride));
}

}  // namespace

extern "C" us_status us_kv_rotate(int32_t q_heads, int32_t k_heads, int32_t head_dim, const us_rows *q, const us_rows *q_out,
                                  const us_rows *k, const us_rows *k_out, const us_kv_rotation *how, void *stream) {
    if (!how || !q || !q_out || !k != !k_out) return US_ERR_ARG;
    us_status st = check_pair(q, q_out, q->tokens, q->dtype);
    if (st == US_OK && k) st = check_pair(k, k_out, q->tokens, q->dtype);
    if (st != US_OK) return st;
    if (!row_of(head_dim) || q_heads < 1 || q_heads > 65535 || k_heads < 0 || k_heads > 65535 || (k_heads > 0) != (k != nullptr))
        return US_ERR_SHAPE;
    // (such rows would be turned more than once, or while others read them)
    if (rows_meet(*q_out, q_heads, head_dim) || other_rows(*q, *q_out, q_heads)) return US_ERR_ARG;
    if (k && (rows_meet(*k_out, k_heads, head_dim) || other_rows(*k, *k_out, k_heads))) return US_ERR_ARG;
    if (how->pairs < 0 || how->pairs > head_dim / 2 || (how->pairs && (how->axes < 1 || how->axes > US_KV_AXES_MAX)))
        return US_ERR_SHAPE;
    if (how->pairs && how->positions_stride < q->tokens && how->axes > 1) return US_ERR_SHAPE;
    if (how->adjacent < 0 || how->adjacent > 1 || how->norm < 0 || how->norm > 1) return US_ERR_ARG;
    if (how->pairs && (!how->freq || !how->positions || (uintptr_t)how->freq % 4 || (uintptr_t)how->positions % 4)) return US_ERR_ARG;
    if (how->norm ? !(how->eps > 0.0f && how->eps < INFINITY) : how->q_weight || how->k_weight) return US_ERR_ARG;
    if ((uintptr_t)how->q_weight % 4 || (uintptr_t)how->k_weight % 4) return US_ERR_ARG;
    if (!how->norm && !how->pairs) return US_ERR_ARG;      // (nothing to do: a copy is not this call's work)
    RotateArgs a;
    const auto rows_of = [](const us_rows *r) { return r ? Rows{r->data, r->token_stride, r->head_stride} : Rows{nullptr, 0, 0}; };
    a.q = rows_of(q), a.q_out = rows_of(q_out), a.k = rows_of(k), a.k_out = rows_of(k_out);
    a.q_heads = q_heads, a.rows = q_heads + k_heads, a.D = head_dim, a.tokens = q->tokens;
    a.freq = how->freq, a.positions = how->positions, a.positions_stride = how->positions_stride;
    a.pairs = how->pairs, a.axes = how->axes, a.offset = how->offset, a.norm = how->norm;
    a.eps = how->eps, a.qw = how->q_weight, a.kw = how->k_weight;
    const int P = a.pairs, slots = (P + 7) / 8 + (head_dim - 2 * P + 15) / 16;
    const int lanes = slots <= 4 ? 4 : slots <= 8 ? 8 : slots <= 16 ? 16 : 32, at_once = kThreads / lanes;
    // A workgroup's tokens: such that a thread has about six items, which one computing of angles and one
    // loading of weights serve, but fewer where there would be less than four workgroups per CU, down to a
    // pass of one token's rows. us for 8192 tokens of 64 + 8 heads of 128, bfloat16, one, two and four
    // tokens: 61, 60 and 65; 5007 of 16 + 16 of 80, one, three and four: 20, 15.5 and 14.5.
    const int64_t some = 4 * us_device::compute_units();
    const int passes = (a.rows + at_once - 1) / at_once, side = at_once / a.rows;
    int group = (passes < 6 ? 6 / passes : 1) * (side > 1 ? side : 1);
    if (P && group > kAngles / P) group = kAngles / P;
    if (group > a.tokens / some) group = (int)(a.tokens / some);
    if (group < 1) group = 1;
    a.group = group;
    const int64_t groups = ((int64_t)a.tokens + group - 1) / group;
    a.part = groups >= some || a.rows <= at_once ? a.rows : at_once;
    // (a grid's dimension has fewer than 2^32 threads)
    if (groups > (1 << 23)) return US_ERR_SHAPE;
    const dim3 grid((unsigned)groups, (a.rows + a.part - 1) / a.part);
    // Octets move whole where every one begins at a multiple of 16 bytes and none is cut.
    const bool vec = octets_aligned(*q, head_dim) && octets_aligned(*q_out, head_dim) && (how->adjacent ? 2 * P : P) % 8 == 0 &&
                     (!k || (octets_aligned(*k, head_dim) && octets_aligned(*k_out, head_dim)));
    const hipError_t e = with_type(q->dtype, [&](auto dt) {
        const auto go = [&](auto kern) {
            hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
            return hipGetLastError();
        };
        const auto width = [&](auto n) {
            constexpr int DT = decltype(dt)::value, N = decltype(n)::value;
            if (how->adjacent) return vec ? go(us_kv_rotate_kernel<DT, N, true, true>) : go(us_kv_rotate_kernel<DT, N, false, true>);
            return vec ? go(us_kv_rotate_kernel<DT, N, true, false>) : go(us_kv_rotate_kernel<DT, N, false, false>);
        };
        switch (lanes) {
            case 4: return width(std::integral_constant<int, 4>());
            case 8: return width(std::integral_constant<int, 8>());
            case 16: return width(std::integral_constant<int, 16>());
        }
        return width(std::integral_constant<int, 32>());
    });
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}
