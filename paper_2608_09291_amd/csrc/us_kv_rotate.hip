// us_kv_rotate: norms of query and key heads and their rotation by positions.
//
// A row (a token's head) of D values x becomes n = x w / sqrt(mean x^2 + eps),
// then its pairs (n1, n2) become (n1 cos - n2 sin, n2 cos + n1 sin) of the angle
// sum over the axes of position times frequency. The angle is taken in 64 bits:
// in 32, a position of a million would be off by a sixteenth of a radian. What is
// left of it after whole quarters of a turn is at most pi / 4, and in float32
// there off by 2^-26 at most.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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
    int32_t pairs, axes, offset, adjacent, norm;
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

// LANES lanes hold a row, an octet each; the rows of `group` tokens pass through
// the workgroup together, which has their angles in LDS.
template <int DT, int LANES, bool VEC>
__global__ __launch_bounds__(kThreads) void us_kv_rotate_kernel(RotateArgs a) {
    using T = typename Type<DT>::T;
    constexpr int kAtOnce = kThreads / LANES;
    __shared__ float2 angle[kAngles];
    const int tid = threadIdx.x, o = tid % LANES;
    const int first = blockIdx.y * a.part, part = min(a.part, a.rows - first), P = a.pairs;
    // This lane's weights, and those of the values that it rotates with.
    int other[8], pair[8];
    bool turns[8];
    float wq[8], wk[8], vq[8], vk[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = 8 * o + e;
        turns[e] = d < 2 * P;
        other[e] = !turns[e] ? min(d, a.D - 1) : a.adjacent ? d ^ 1 : d < P ? d + P : d - P;
        pair[e] = !turns[e] ? 0 : a.adjacent ? d >> 1 : d < P ? d : d - P;
        const int at = min(d, a.D - 1);
        wq[e] = a.qw ? a.qw[at] : 1.0f;
        vq[e] = a.qw ? a.qw[other[e]] : 1.0f;
        wk[e] = a.kw ? a.kw[at] : 1.0f;
        vk[e] = a.kw ? a.kw[other[e]] : 1.0f;
    }
    const bool whole = VEC && !a.adjacent && P % 8 == 0;   // an octet's others are one octet
    const int step = gridDim.x;
    const int groups = (a.tokens + a.group - 1) / a.group;
    for (int g = blockIdx.x; g < groups; g += step) {
        const int t0 = g * a.group, n = min(a.group, a.tokens - t0);
        for (int i = tid; i < n * P; i += kThreads) {
            const int t = i / P, p = i - t * P;
            double sum = 0.0;
            for (int x = 0; x < a.axes; ++x)
                sum += ((double)a.positions[x * a.positions_stride + t0 + t] + a.offset) * (double)a.freq[x * P + p];
            angle[i] = turn(sum);
        }
        __syncthreads();
        for (int r = tid / LANES; r < n * part; r += kAtOnce) {
            const int t = r / part, row = first + r - t * part;
            const bool key = row >= a.q_heads;
            const Rows &in = key ? a.k : a.q, &out = key ? a.k_out : a.q_out;
            const int head = key ? row - a.q_heads : row;
            const T *src = (const T *)in.data + (int64_t)(t0 + t) * in.token_stride + (int64_t)head * in.head_stride;
            T *dst = (T *)out.data + (int64_t)(t0 + t) * out.token_stride + (int64_t)head * out.head_stride;
            float x[8], y[8];
            load_octet<DT, VEC>(src, o, a.D, x);
            if (8 * o >= 2 * P) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = 0.0f;
            } else if (whole) {
                load_octet<DT, true>(src, 8 * o < P ? o + P / 8 : o - P / 8, a.D, y);
            } else if (a.adjacent) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = turns[e] ? Type<DT>::get(src[other[e]]) : 0.0f;
            }
            float scale = 1.0f;
            if (a.norm) {
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
                for (int z = LANES / 2; z > 0; z >>= 1) sum += __shfl_xor(sum, z, 64);
                scale = 1.0f / sqrtf(sum / (float)a.D + a.eps);
                if (sum == INFINITY) {                     // of values past 2^63: the same of 2^-64 x
                    sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum = fmaf(x[e] * 0x1p-64f, x[e] * 0x1p-64f, sum);
#pragma unroll
                    for (int z = LANES / 2; z > 0; z >>= 1) sum += __shfl_xor(sum, z, 64);
                    scale = 0x1p-64f / sqrtf(sum / (float)a.D);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (a.norm) {
                    x[e] = x[e] * scale * (key ? wk[e] : wq[e]);
                    y[e] = y[e] * scale * (key ? vk[e] : vq[e]);
                }
                if (turns[e]) {
                    const float2 cs = angle[t * P + pair[e]];
                    const bool low = a.adjacent ? !(e & 1) : 8 * o + e < P;
                    x[e] = fmaf(x[e], cs.x, low ? -y[e] * cs.y : y[e] * cs.y);
                }
            }
            store_octet<DT, VEC>(dst, o, a.D, x);
        }
        __syncthreads();
    }
}

us_status check_pair(const us_rows *in, const us_rows *out, int tokens, int dtype) {
    us_status st = check_rows(in);
    if (st == US_OK) st = check_rows(out);
    if (st != US_OK) return st;
    if (in->dtype != dtype || out->dtype != dtype) return US_ERR_ARG;
    return in->tokens == tokens && out->tokens == tokens ? US_OK : US_ERR_SHAPE;
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
    a.pairs = how->pairs, a.axes = how->axes, a.offset = how->offset, a.adjacent = how->adjacent, a.norm = how->norm;
    a.eps = how->eps, a.qw = how->q_weight, a.kw = how->k_weight;
    const int lanes = head_dim <= 64 ? 8 : head_dim <= 128 ? 16 : 32, at_once = kThreads / lanes;
    // Few rows to a token: several tokens, as many as fill a pass. Few tokens: a workgroup takes a pass of
    // their rows alone, so that the rest runs beside it.
    int group = at_once / a.rows;
    group = group < 1 ? 1 : group;
    if (a.pairs && group * a.pairs > kAngles) group = kAngles / a.pairs;
    a.group = group;
    const int groups = (a.tokens + group - 1) / group;
    a.part = groups >= 2048 || a.rows <= at_once ? a.rows : at_once;
    const dim3 grid(groups < (1 << 22) ? groups : 1 << 22, (a.rows + a.part - 1) / a.part);
    const bool vec = octets_aligned(*q, head_dim) && octets_aligned(*q_out, head_dim) &&
                     (!k || (octets_aligned(*k, head_dim) && octets_aligned(*k_out, head_dim)));
    const hipError_t e = with_type(q->dtype, [&](auto dt) {
        const auto go = [&](auto kern) {
            hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
            return hipGetLastError();
        };
        const auto width = [&](auto n) {
            return vec ? go(us_kv_rotate_kernel<decltype(dt)::value, decltype(n)::value, true>)
                       : go(us_kv_rotate_kernel<decltype(dt)::value, decltype(n)::value, false>);
        };
        return lanes == 8 ? width(std::integral_constant<int, 8>())
                          : lanes == 16 ? width(std::integral_constant<int, 16>()) : width(std::integral_constant<int, 32>());
    });
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}
