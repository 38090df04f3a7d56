// us_kv_attend with few query rows: every key and value is read once, for at
// most 16 rows at a time (the query heads of a cache head, and a few tokens).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "us_kv_attend.h"

namespace us_kv {
namespace {

constexpr int kThreads = 256, kWaves = 4, kRows = 16;

template <int NT, int DT>
__global__ __launch_bounds__(kThreads, NT > 4 ? 1 : 2) void us_kv_decode_kernel(Args a) {
    using T = typename Type<DT>::T;
    constexpr bool SPLIT = DT == US_F32;
    constexpr int R = 32 * NT, NV = R / 16;
    constexpr int kCols = R > 128 ? R / 2 : R;             // columns joined at a time
    __shared__ __attribute__((aligned(16))) float sum[kWaves][kRows][kCols + 4];
    __shared__ float wm[kWaves][kRows], wl[kWaves][kRows];
    __shared__ float jm[16][kRows], jl[16][kRows];
    __shared__ int flag;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    // Workgroups go round the XCDs in order of blockIdx, x first: heads and
    // sequences spread over them, where splits, of which short sequences leave
    // the later ones empty, would load a few (64 ragged sequences to 8k: 100 us).
    const int tile = blockIdx.z % a.sp.tiles, split = blockIdx.z / a.sp.tiles, hk = blockIdx.x, b = blockIdx.y;
    // Without a window the first block to look up is known before the length is.
    const int guess = a.s.blocks[b * a.s.stride + min(split * a.sp.chunk + wave + kWaves * lane, (a.s.max_len - 1) / kBlock)];
    int r0, n;
    a.s.rows(b, r0, n);
    const int len = a.s.len(b), total = n * a.G, base = tile * kRows;
    if (base >= total) return;
    const int last_row = min(base + kRows, total) - 1;
    int lo0, hi0, lo1, hi1;                                // of the tile's first and last row
    a.mask.range(base / a.G, n, len, lo0, hi0);
    a.mask.range(last_row / a.G, n, len, lo1, hi1);
    const int first = lo0 / kBlock, end = (hi1 + kBlock - 1) / kBlock;
    const int ns = splits_of(lo0, hi1, a.sp.chunk);
    if (split >= ns) return;
    const int row = min(base + r, last_row), i = row / a.G, head = hk * a.G + row - i * a.G;
    int lo, hi;
    a.mask.range(i, n, len, lo, hi);

    // Queries: column r of the first product's right operand.
    RowPart<DT, NT> raw;
    raw.load((const T *)a.q.data + (int64_t)(r0 + i) * a.q.token_stride + (int64_t)head * a.q.head_stride, g, 4, a.D, a.vec);

    // This wavefront's blocks: start, start + 4, ... A lane looks one of them up.
    const int start = first + split * a.sp.chunk + wave, stop = min(first + (split + 1) * a.sp.chunk, end);
    const int count = start < stop ? (stop - start + kWaves - 1) / kWaves : 0;
    int my_id;
    float my_ks, my_vs;
    auto look_up = [&](int c) {                            // 64 of them, from the c-th on
        my_id = -1;
        my_ks = my_vs = 0.0f;
        if (c + lane < count) {
            my_id = c == 0 && first == 0 ? a.s.valid(guess) : a.s.block(b, start + kWaves * (c + lane));
            if (my_id >= 0) {
                my_ks = a.ks[(int64_t)my_id * a.heads + hk];
                my_vs = a.vs[(int64_t)my_id * a.heads + hk];
            }
        }
    };
    look_up(0);

    f16x8 qh[NT], ql[NT];
    float f;
    auto set_queries = [&]() {
        float x[NT][8], mx = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            raw.octet(t, 4 * t + g, a.D, a.D == R, x[t]);
            mx = magnitude(x[t], mx);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        float inv;
        const float norm = row_norm(mx, inv);
        f = inv * a.scale;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[t][e] *= norm;
            halve<SPLIT>(x[t], qh[t], ql[t]);
        }
    };

    const int64_t page = (int64_t)kBlock * R;
    auto at = [&](int c) {                                 // this wavefront's c-th block (block 0 where it is not there)
        const int id = __builtin_amdgcn_readlane(my_id, c & 63);
        return ((int64_t)max(id, 0) * a.heads + hk) * page;
    };
    u32x4 kr[NT][2], vr[NV];
    auto load_k = [&](int64_t off) {
        const uint8_t *p = a.k + off + 64 * r + 16 * g;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) kr[t][u] = __builtin_nontemporal_load((const u32x4 *)(p + 2048 * t + 1024 * u));
    };
    auto load_v = [&](int64_t off) {
        const uint8_t *p = a.v + off + 64 * r + 16 * g;
#pragma unroll
        for (int t = 0; t < NV; ++t) vr[t] = __builtin_nontemporal_load((const u32x4 *)(p + 1024 * t));
    };

    float m = -INFINITY, l = 0.0f;
    f32x4 o[NV];
#pragma unroll
    for (int t = 0; t < NV; ++t) o[t] = (f32x4){0, 0, 0, 0};
    if (count > 0) {
        load_k(at(0));
        load_v(at(0));
    }
    set_queries();
    for (int c = 0; c < count; ++c) {
        const int blk = start + kWaves * c;
        const bool there = __builtin_amdgcn_readlane(my_id, c & 63) >= 0;
        const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_ks), c & 63));
        const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_vs), c & 63));
        // Lane (r, g), element v of tile u: key 16 u + 4 g + v, row r.
        f32x4 s[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] = (f32x4){0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const f16x8 kh = halves_of(kr[t][u >> 1][2 * (u & 1)], kr[t][u >> 1][2 * (u & 1) + 1]);
                s[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, qh[t], s[u], 0, 0, 0);
                if constexpr (SPLIT) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, ql[t], s[u], 0, 0, 0);
            }
        if (c + 1 < count) {
            if (((c + 1) & 63) == 0) look_up(c + 1);
            load_k(at(c + 1));
        }
        const float fk = f * ks;
        const int j0 = blk * kBlock + 4 * g;
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] *= fk;
        if (!(there && blk * kBlock >= lo1 && blk * kBlock + kBlock <= hi0)) {
            int from = there ? lo - j0 : kBlock, to = hi - j0;
            __asm__ volatile("" : "+v"(from), "+v"(to));   // keeps the branch: most blocks have no masked keys
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) s[u][v] = 16 * u + v >= from && 16 * u + v < to ? s[u][v] : -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int v = 0; v < 4; ++v) top = fmaxf(top, s[u][v]);
        if (a.sp.scores && base + r <= last_row) {
            float *dst = a.sp.scores + (((int64_t)b * a.heads + hk) * a.sp.rows * a.sp.tiles + row) * a.sp.scores_stride + j0;
#pragma unroll
            for (int u = 0; u < 4; ++u) *(f32x4 *)(dst + 16 * u) = s[u];
        }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m2 = fmaxf(m, top), to = base_of(m2), alpha = __builtin_amdgcn_exp2f(m - to);
        m = m2;
        l *= alpha;
        f16x8 ph[2], pl[2];
        float sub = to - kLift;
        // (beside larger ones the lift would be rounded, past float16's range from 2^25 on)
        if (__builtin_amdgcn_ballot_w64(fabsf(to) > kLarge)) {
#pragma unroll
            for (int u = 0; u < 4; ++u) s[u] -= to;
            sub = -kLift;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(s[2 * u + (e >> 2)][e & 3] - sub);
                l += p[e];
            }
            halve<SPLIT>(p, ph[u], pl[u]);
        }
        // Lane (r, g) of the left operand: value 16 t + r of keys 16 u + 4 g + v.
#pragma unroll
        for (int t = 0; t < NV; ++t) {
            f32x4 pv = {0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const f16x8 vh = halves_of(vr[t][2 * u], vr[t][2 * u + 1]);
                pv = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, ph[u], pv, 0, 0, 0);
                if constexpr (SPLIT) pv = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, pl[u], pv, 0, 0, 0);
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) o[t][v] = fmaf(pv[v], vs, o[t][v] * alpha);
        }
        if (c + 1 < count) load_v(at(c + 1));
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);

    // Join the wavefronts; lane (r, g) holds values 16 t + 4 g + v of row r.
    if (g == 0) {
        wm[wave][r] = m;
        wl[wave][r] = l;
    }
    __syncthreads();
    float all = wm[0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) all = fmaxf(all, wm[w][r]);
    const float mine = __builtin_amdgcn_exp2f(m - base_of(all));
    const int64_t unit = ((int64_t)b * a.heads + hk) * a.sp.tiles + tile;
    const int rows_here = last_row - base + 1;
    const int one = (a.sp.rows * (R + 2) + 3) / 4 * 4;     // floats of a split
    const Shared mem(a.sp.part + unit * a.sp.splits * one);
#pragma unroll
    for (int c0 = 0; c0 < R; c0 += kCols) {
        if (c0) __syncthreads();
#pragma unroll
        for (int t = 0; t < kCols / 16; ++t) {
            f32x4 x = o[c0 / 16 + t];
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] *= mine;
            *(f32x4 *)&sum[wave][r][16 * t + 4 * g] = x;
        }
        __syncthreads();
        for (int q = tid; q < rows_here * (kCols / 8); q += kThreads) {
            const int rr = q / (kCols / 8), oc = q % (kCols / 8);
            float x[8], am = wm[0][rr], ll = 0.0f;
#pragma unroll
            for (int w = 1; w < kWaves; ++w) am = fmaxf(am, wm[w][rr]);
            const float bm = base_of(am);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) ll += wl[w][rr] * __builtin_amdgcn_exp2f(wm[w][rr] - bm);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] += sum[w][rr][8 * oc + e];
            const int gr = base + rr, ti = gr / a.G, hd = hk * a.G + gr - ti * a.G;
            if (ns == 1) {
                put_octet<DT>(a, r0 + ti, hd, c0 / 8 + oc, x, ll);
                if (a.sp.ml && c0 == 0 && oc == 0) a.sp.ml[32 * row_block(a, hk, b, r0, gr) + gr % 32] = ml_of(am, ll);
            } else {
                const uint32_t dst = split * one + rr * R + c0 + 8 * oc;
                mem.put(dst, (f32x4){x[0], x[1], x[2], x[3]});
                mem.put(dst + 4, (f32x4){x[4], x[5], x[6], x[7]});
                if (c0 == 0 && oc == 0) mem.put2(split * one + a.sp.rows * R + 2 * rr, am, ll);
            }
        }
    }
    if (ns == 1 || !last_of(a.sp.tickets + unit, ns, &flag)) return;
    // The last workgroup joins the splits, in an order that does not depend on
    // their arrival: first the rows' maxima and sums, 16 splits at a time, then
    // the rows by quads of values, the splits in as many runs as there are
    // threads for.
    {
        const int rr = tid & 15, z0 = tid >> 4;
        float mj = -INFINITY, lj = 0.0f;
        if (rr < rows_here)
#pragma unroll 4
            for (int z = z0; z < ns; z += 16) {
                float mz, lz;
                mem.get2(z * one + a.sp.rows * R + 2 * rr, mz, lz);
                const float m2 = fmaxf(mj, mz), to = base_of(m2);
                lj = lj * __builtin_amdgcn_exp2f(mj - to) + lz * __builtin_amdgcn_exp2f(mz - to);
                mj = m2;
            }
        jm[z0][rr] = mj;
        jl[z0][rr] = lj;
    }
    __syncthreads();
    const int items = rows_here * (R / 4), runs = items < kThreads ? kThreads / items : 1;
    const int per = (ns + runs - 1) / runs;
    f32x4 *joined = (f32x4 *)&sum[0][0][0];                // run, item
    float am, ll;
    auto part = [&](int it, int z0, int z1) {              // of splits z0 .. z1 - 1, times 2^-am
        const int rr = it / (R / 4), quad = it % (R / 4);
        am = -INFINITY, ll = 0.0f;
#pragma unroll
        for (int z = 0; z < 16; ++z) am = fmaxf(am, jm[z][rr]);
        const float bm = base_of(am);
#pragma unroll
        for (int z = 0; z < 16; ++z) ll += jl[z][rr] * __builtin_amdgcn_exp2f(jm[z][rr] - bm);
        f32x4 x = {0, 0, 0, 0};
#pragma unroll 8
        for (int z = z0; z < z1; ++z) {
            float mz, lz;
            mem.get2(z * one + a.sp.rows * R + 2 * rr, mz, lz);
            const f32x4 y = mem.get(z * one + rr * R + 4 * quad);
            const float w = __builtin_amdgcn_exp2f(mz - bm);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = fmaf(y[e], w, x[e]);
        }
        return x;
    };
    auto finish = [&](int it, f32x4 x) {
        const int gr = base + it / (R / 4), quad = it % (R / 4), ti = gr / a.G, hd = hk * a.G + gr - ti * a.G;
        put_quad<DT>(a, r0 + ti, hd, quad, x, ll);
        if (a.sp.ml && quad == 0) a.sp.ml[32 * row_block(a, hk, b, r0, gr) + gr % 32] = ml_of(am, ll);
    };
    if (runs > 1) {
        f32x4 x = {0, 0, 0, 0};
        const int run = tid / items, it = tid - run * items;
        if (run < runs) {
            x = part(it, run * per, min((run + 1) * per, ns));
            joined[tid] = x;
        }
        __syncthreads();
        if (run == 0) {
            for (int z = 1; z < runs; ++z) x += joined[z * items + it];
            finish(it, x);
        }
    } else {
        for (int it = tid; it < items; it += kThreads) finish(it, part(it, 0, ns));
    }
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
