// us_kv_attend with many query rows: prompts and chunks of them.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "us_kv_attend.h"
#include "us_kv_prompt.h"

namespace us_kv {
namespace {

constexpr int weights_blocks(int row, bool f32) { return row <= 192 || !f32 ? 2 : 1; }     // three stages of at most 160 KB

template <int NT, int DT, int W>
__global__ __launch_bounds__(64 * W, NT > 4 ? 1 : 2) void us_kv_prompt_kernel(Args a) {
    prompt_rows<kWhole, NT, DT, W>(a, Others{});
}

// Joins the splits of a row: a thread per quad of its values. (The last workgroup of a tile
// joining it alone, as in decode, took 400 us for 118 splits of 256 rows.)
template <int NT, int DT>
__global__ __launch_bounds__(256) void us_kv_join_kernel(Args a) {
    constexpr int R = 32 * NT, kRows = 32 * prompt_waves(R), kEach = 256 / (R / 4);
    const int hk = blockIdx.y, b = blockIdx.z, quad = threadIdx.x % (R / 4);
    const int row = blockIdx.x * kEach + threadIdx.x / (R / 4);
    int r0, n;
    a.s.rows(b, r0, n);
    const int len = a.s.len(b), total = n * a.G;
    if ((int)threadIdx.x >= kEach * (R / 4) || row >= total) return;
    const int tile = row / kRows, base = tile * kRows, last_row = min(base + kRows, total) - 1;
    int lo0, hi1, unused;
    a.mask.range(base / a.G, n, len, lo0, unused);
    a.mask.range(last_row / a.G, n, len, unused, hi1);
    const int ns = splits_of(lo0, hi1, a.sp.chunk);
    if (ns == 1) return;
    constexpr int kOne = kRows * (R + 2);
    const float *src = a.sp.part + (((int64_t)b * a.heads + hk) * a.sp.tiles + tile) * a.sp.splits * kOne;
    const int ml = kRows * R + 2 * (row - base), at = (row - base) * R + 4 * quad;
    float m = -INFINITY, l = 0.0f;
#pragma unroll 8
    for (int z = 0; z < ns; ++z) m = fmaxf(m, src[(int64_t)z * kOne + ml]);
    const float bm = base_of(m);
    f32x4 x = {0, 0, 0, 0};
#pragma unroll 8
    for (int z = 0; z < ns; ++z) {
        const float w = __builtin_amdgcn_exp2f(src[(int64_t)z * kOne + ml] - bm);
        const f32x4 y = *(const f32x4 *)(src + (int64_t)z * kOne + at);
        l = fmaf(src[(int64_t)z * kOne + ml + 1], w, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(y[e], w, x[e]);
    }
    put_quad<DT>(a, r0 + row / a.G, hk * a.G + row % a.G, quad, x, l);
    if (a.sp.ml && quad == 0) a.sp.ml[32 * row_block(a, hk, b, r0, row) + row % 32] = ml_of(m, l);
}

// The probabilities' sums over the query rows, from the rows' maxima and sums:
// the first product again, the other way about. A wavefront keeps a block
// of keys in registers; the rows, in the form that the first pass left them,
// pass through LDS, in three stages. Scores are computed 32 rows ahead of their
// exponentials, so that the matrix cores work under these. Chunks of 512 on
// 16000 keys, 64 heads over 8: 455 us without that and with a division per 32
// rows for the mask.
constexpr int kKeys = 256;                                 // of a workgroup
template <int NT, int DT>
__global__ __launch_bounds__(256, NT > 4 || (NT > 3 && DT == US_F32) ? 1 : 2) void us_kv_weights_kernel(Args a, float *weights, int64_t stride) {
    constexpr bool SPLIT = DT == US_F32;
    constexpr int R = 32 * NT, NS = R / 16, kParts = SPLIT ? 2 : 1;
    constexpr int kForm = kParts * R / 8 * 32;             // pieces of 32 rows
    constexpr int kBlocks = weights_blocks(R, SPLIT);      // blocks of 32 rows of a stage
    constexpr int kPieces = kBlocks * kForm / 256;
    static_assert(kBlocks * kForm % 256 == 0);
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    f16x8(*q)[kBlocks * kForm] = (f16x8(*)[kBlocks * kForm])lds;               // stage; row block, part, octet, row
    __shared__ float row_f[3][64];
    __shared__ float2 row_ml[3][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 31, h = lane >> 5, hk = blockIdx.y, b = blockIdx.z;
    int r0, n;
    a.s.rows(b, r0, n);
    const int len = a.s.len(b), j0 = blockIdx.x * kKeys;
    if (j0 >= len || n == 0) return;
    // Queries that see some of these keys.
    int i0 = 0, i1 = n;
    if (a.mask.causal) {
        i0 = max(j0 - (len - n), 0);
        if (a.mask.window > 0) i1 = (int)min((int64_t)n, (int64_t)j0 + kKeys - 1 + a.mask.window - (len - n));
    }
    if (i0 >= i1) return;
    const int total = n * a.G, first = i0 * a.G / 32, end = (i1 * a.G + 31) / 32;   // blocks of rows
    const int blk = 4 * (int)blockIdx.x + wave, k0 = blk * kBlock;
    // Rows [all0, all1) see all of this wavefront's keys.
    int all0 = 0, all1 = total;
    if (a.mask.causal) {
        all0 = (int)min((int64_t)total, (int64_t)max(k0 + kBlock - 1 - (len - n), 0) * a.G);
        if (a.mask.window > 0) all1 = (int)min((int64_t)total, max((int64_t)k0 + a.mask.window - (len - n), (int64_t)0) * a.G);
    } else if (k0 + kBlock > len) {
        all1 = 0;
    }
    const int id = k0 < len ? a.s.block(b, blk) : -1;
    const int64_t at = (int64_t)max(id, 0) * a.heads + hk;
    const float ks = id < 0 ? 0.0f : a.ks[at];
    const int64_t rb = row_block(a, hk, b, r0, 0);
    const f16x8 *src = a.sp.qn + rb * kForm;
    f16x8 piece[kPieces];
    float f_next = 0.0f;
    float2 ml_next = make_float2(0.0f, 0.0f);
    auto fetch = [&](int x) {                              // row blocks x .. (there is one past the last)
#pragma unroll
        for (int y = 0; y < kPieces; ++y) piece[y] = src[(int64_t)x * kForm + tid + 256 * y];
        if (tid < 32 * kBlocks) f_next = a.sp.qf[32 * (rb + x) + tid];
        if (lane < 32 * kBlocks) ml_next = a.sp.ml[32 * (rb + x) + lane];      // (by every wavefront, for put)
    };
    // Returns how many rows of these, from row block x on, have a maximum past kLarge.
    auto put = [&](int buf, int x) {
#pragma unroll
        for (int y = 0; y < kPieces; ++y) q[buf][tid + 256 * y] = piece[y];
        if (tid < 32 * kBlocks) {
            row_f[buf][tid] = f_next;
            row_ml[buf][tid] = ml_next;
        }
        // (rows past the last hold anything)
        return __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < 32 * kBlocks && 32 * x + lane < total && fabsf(ml_next.x) > kLarge));
    };
    fetch(first);
    f16x8 kf[2][NS];
    {
        // keys 32 u + c, octets 2 t + h
        const uint8_t *p = a.k + at * (kBlock * R) + 64 * (c & 15) + 8 * (c >> 4);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                const u32x2 w = *(const u32x2 *)(p + 1024 * u + 2048 * (t >> 1) + 16 * (2 * (t & 1) + h));
                kf[u][t] = halves_of(w[0], w[1]);
            }
    }
    f32x16 sum[2], sa[2], sb[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int v = 0; v < 16; ++v) sum[u][v] = 0.0f;
    auto scores = [&](int buf, int y, f32x16 (&s)[2]) {    // of row block y of a stage
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) s[u][v] = 0.0f;
#pragma unroll
        for (int t = 0; t < NS; ++t)
#pragma unroll
            for (int z = 0; z < kParts; ++z) {
                const f16x8 qf = q[buf][kForm * y + (z * (R / 8) + 2 * t + h) * 32 + c];
#pragma unroll
                for (int u = 0; u < 2; ++u) s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[u][t], qf, s[u], 0, 0, 0);
            }
    };
    auto add = [&](int x, float fk, float2 ml, int large, f32x16 (&s)[2]) {    // row block x
        const int base = 32 * x;
        // (ahead of the branches, so that they go beside the next scores' product: 6 % of the kernel)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) s[u][v] = fmaf(s[u][v], fk, -ml.x);
        if (__builtin_expect(large != 0, 0)) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int v = 0; v < 16; ++v) s[u][v] = above(s[u][v], ml.x);
        }
        if (base >= all0 && base + 32 <= all1) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int v = 0; v < 16; ++v) sum[u][v] = fmaf(__builtin_amdgcn_exp2f(s[u][v]), ml.y, sum[u][v]);
        } else {
            int from = 0, to = 0;
            if (base + c < total) a.mask.range((base + c) / a.G, n, len, from, to);
            from -= k0 + 4 * h;
            to -= k0 + 4 * h;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int j = 32 * u + 8 * (v >> 2) + (v & 3);
                    const float p = __builtin_amdgcn_exp2f(s[u][v]) * ml.y;
                    sum[u][v] += j >= from && j < to ? p : 0.0f;
                }
        }
    };
    // Stage i % 3 holds chunk i: while chunk i is added up and the first scores of
    // chunk i + 1 are taken, chunk i + 2 is put, and i + 3 is on its way.
    const int chunks = (end - first + kBlocks - 1) / kBlocks;
    int large = put(0, first), large1 = 0, large2 = 0;     // of this chunk and the next ones
    if (chunks > 1) {
        fetch(first + kBlocks);
        large1 = put(1, first + kBlocks);
    }
    if (chunks > 2) fetch(first + 2 * kBlocks);
    __syncthreads();
    scores(0, 0, sa);
    auto turn = [&](int i, int x, int y, f32x16 (&s)[2], f32x16 (&next)[2]) {  // row block y of chunk i, the x-th
        const int buf = i % 3;
        const float fk = row_f[buf][32 * y + c] * ks;
        const float2 ml = row_ml[buf][32 * y + c];
        if (y + 1 < kBlocks) scores(buf, y + 1, next);
        else scores((i + 1) % 3, 0, next);                 // (of no use after the last chunk)
        add(x, fk, ml, large, s);
    };
    for (int i = 0; i < chunks; ++i) {
        const int x = first + i * kBlocks;
        if constexpr (kBlocks == 2) {
            turn(i, x, 0, sa, sb);
            turn(i, x + 1, 1, sb, sa);
        } else {
            turn(i, x, 0, sa, sb);
#pragma unroll
            for (int u = 0; u < 2; ++u) sa[u] = sb[u];
        }
        if (i + 2 < chunks) large2 = put((i + 2) % 3, x + 2 * kBlocks);
        large = large1;
        large1 = large2;
        if (i + 3 < chunks) fetch(x + 3 * kBlocks);
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int v = 0; v < 16; ++v)
#pragma unroll
            for (int w = 16; w > 0; w >>= 1) sum[u][v] += __shfl_xor(sum[u][v], w, 64);
    if (c == 0 && id >= 0) {
        float *dst = weights + ((int64_t)b * a.heads + hk) * stride + k0 + 4 * h;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int j = 32 * u + 8 * (v >> 2) + (v & 3);
                if (k0 + 4 * h + j < len) dst[j] += sum[u][v];
            }
    }
}

}  // namespace

hipError_t launch_prompt(int dtype, const Args &a, int batch, hipStream_t stream) {
    return with_row(a.D, [&](auto nt) {
        return with_type(dtype, [&](auto dt) {
            constexpr int NT = decltype(nt)::value, R = 32 * NT;
            constexpr bool f32 = decltype(dt)::value == US_F32;
            constexpr int W = prompt_waves(R);
            constexpr int kLds = prompt_lds<R, f32>();
            auto kern = us_kv_prompt_kernel<NT, decltype(dt)::value, W>;
            if constexpr (kLds > 65536 - 1024) {
                static std::atomic<unsigned long long> set{0};
                const hipError_t e = allow_lds(kern, set);
                if (e != hipSuccess) return e;
            }
            hipLaunchKernelGGL(kern, dim3((unsigned)batch * a.heads * a.sp.tiles * a.sp.splits), dim3(64 * W), kLds, stream, a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess || a.sp.splits == 1) return e;
            constexpr int kEach = 256 / (8 * NT);
            const unsigned x = (unsigned)(((int64_t)a.s.max_new * a.G + kEach - 1) / kEach);
            hipLaunchKernelGGL((us_kv_join_kernel<NT, decltype(dt)::value>), dim3(x, a.heads, batch), dim3(256), 0, stream, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_weights(int dtype, const Args &a, int batch, float *weights, int64_t stride, hipStream_t stream) {
    return with_row(a.D, [&](auto nt) {
        return with_type(dtype, [&](auto dt) {
            constexpr int NT = decltype(nt)::value, DT = decltype(dt)::value;
            constexpr int kLds = 3 * (DT == US_F32 ? 2 : 1) * 32 * weights_blocks(32 * NT, DT == US_F32) * 32 * NT * 2;
            auto kern = us_kv_weights_kernel<NT, DT>;
            if constexpr (kLds > 65536 - 4096) {
                static std::atomic<unsigned long long> set{0};
                const hipError_t e = allow_lds(kern, set);
                if (e != hipSuccess) return e;
            }
            hipLaunchKernelGGL(kern, dim3((a.s.max_len + kKeys - 1) / kKeys, a.heads, batch), dim3(256), kLds, stream, a, weights, stride);
            return hipGetLastError();
        });
    });
}

}  // namespace us_kv
