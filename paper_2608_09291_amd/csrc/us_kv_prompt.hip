// us_kv_attend with many query rows: prompts and chunks of them.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "us_kv_attend.h"

namespace us_kv {
namespace {

constexpr int kThreads = 256, kWaves = 4, kRows = 128;     // 32 rows per wavefront

// A block's keys and values as float16 in LDS, in the order of the operands:
// 16 bytes (8 values of a key; 8 keys of a value) per lane.
template <int R>
struct Stage {
    f16x8 k[R / 8][kBlock];        // octet of values, key
    f16x8 v[8][R];                 // eight keys (2 j + h: 16 j + 4 h + {0..3, 8..11}), value
};

template <int NT, int DT>
__global__ __launch_bounds__(kThreads, NT > 4 || (NT > 2 && DT == US_F32) ? 1 : 2) void us_kv_prompt_kernel(Args a, int units) {
    using T = typename Type<DT>::T;
    constexpr bool SPLIT = DT == US_F32;
    constexpr int R = 32 * NT, NS = R / 16;                // NS: steps of the first product
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Stage<R> *stage = (Stage<R> *)lds;
    __shared__ int flag;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 31, h = lane >> 5;
    // The tiles of a unit (sequence, cache head) follow each other on one XCD,
    // whose L2 then serves their keys; the last tile, which sees the most, first.
    const int per = a.sp.tiles * a.sp.splits;
    int u = blockIdx.x / per, slot = blockIdx.x % per;
    if (units % 8 == 0) {
        u = (blockIdx.x >> 3) / per * 8 + (blockIdx.x & 7);
        slot = (blockIdx.x >> 3) % per;
    }
    const int tile = a.sp.tiles - 1 - slot / a.sp.splits, split = slot % a.sp.splits;
    const int b = u / a.heads, hk = u - b * a.heads;
    int r0, n;
    a.s.rows(b, r0, n);
    const int len = a.s.len(b), total = n * a.G, base = tile * kRows;
    if (base >= total) return;
    const int last_row = min(base + kRows, total) - 1;
    int lo0, hi0, lo1, hi1;
    a.mask.range(base / a.G, n, len, lo0, hi0);
    a.mask.range(last_row / a.G, n, len, lo1, hi1);
    const int first = lo0 / kBlock, end = (hi1 + kBlock - 1) / kBlock;
    const int ns = max((end - first + a.sp.chunk - 1) / a.sp.chunk, 1);
    if (split >= ns) return;
    const int start = first + split * a.sp.chunk, stop = min(start + a.sp.chunk, end);
    // This wavefront's rows, and this lane's; the range of keys that they see.
    const int w0 = min(base + 32 * wave, last_row), w1 = min(base + 32 * wave + 31, last_row);
    int wlo, whi, wlo1, whi0;
    a.mask.range(w0 / a.G, n, len, wlo, whi0);
    a.mask.range(w1 / a.G, n, len, wlo1, whi);
    const int row = min(base + 32 * wave + c, last_row), i = row / a.G, head = hk * a.G + row - i * a.G;
    const bool real = base + 32 * wave + c <= last_row;
    int lo, hi;
    a.mask.range(i, n, len, lo, hi);

    f16x8 qh[NS], ql[NS];
    float f;
    {
        RowPart<DT, NS> raw;
        raw.load((const T *)a.q.data + (int64_t)(r0 + i) * a.q.token_stride + (int64_t)head * a.q.head_stride, h, 2, a.D, a.vec);
        float mx = 0.0f;
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            float x[8];
            raw.octet(t, 2 * t + h, a.D, a.D == R, x);
            mx = magnitude(x, mx);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        float inv;
        const float norm = row_norm(mx, inv);
        f = inv * a.scale;
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            float x[8];
            raw.octet(t, 2 * t + h, a.D, a.D == R, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= norm;
            halve<SPLIT>(x, qh[t], ql[t]);
        }
    }

    // Blocks on their way: 16-byte pieces of the codes in registers.
    constexpr int kPieces = 4 * R / kThreads + (4 * R % kThreads ? 1 : 0);     // of the keys, per thread
    constexpr int kPairs = 2 * R / kThreads + (2 * R % kThreads ? 1 : 0);      // of the values, two pieces each
    u32x4 kr[kPieces], vr[kPairs][2];
    // A lane looks up one of 64 blocks, the next ones when those are used up.
    const int count = stop - start;
    int id_k, id_v;
    float sc_k, sc_v;                                      // of the 64 blocks whose keys (values) are in use
    auto look_up = [&](int c, int &id, float &sc, const float *scales) {
        id = -1;
        sc = -1.0f;
        if (c + lane < count) {
            id = a.s.block(b, start + c + lane);
            if (id >= 0) sc = scales[(int64_t)id * a.heads + hk];
        }
    };
    auto lane_of = [](float x, int c) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), c & 63)); };
    auto fetch_k = [&](int c) {
        const uint8_t *kp = a.k + ((int64_t)max(__builtin_amdgcn_readlane(id_k, c & 63), 0) * a.heads + hk) * (kBlock * R);
#pragma unroll
        for (int x = 0; x < kPieces; ++x) {
            // (64 lanes: 16 keys x 4 octets, one KB)
            const int q = tid + kThreads * x;
            if (4 * R % kThreads == 0 || q < 4 * R) kr[x] = *(const u32x4 *)(kp + 1024 * (q >> 6) + 64 * (q & 15) + 16 * ((q >> 4) & 3));
        }
    };
    auto fetch_v = [&](int c) {
        const uint8_t *vp = a.v + ((int64_t)max(__builtin_amdgcn_readlane(id_v, c & 63), 0) * a.heads + hk) * (kBlock * R);
#pragma unroll
        for (int x = 0; x < kPairs; ++x) {
            const int q = tid + kThreads * x;
            if (2 * R % kThreads == 0 || q < 2 * R) {
                vr[x][0] = *(const u32x4 *)(vp + 64 * (q >> 1) + 16 * (q & 1));
                vr[x][1] = *(const u32x4 *)(vp + 64 * (q >> 1) + 16 * (q & 1) + 32);
            }
        }
    };
    auto put_k = [&](int buf) {
#pragma unroll
        for (int x = 0; x < kPieces; ++x) {
            const int q = tid + kThreads * x;
            if (4 * R % kThreads == 0 || q < 4 * R) {
                const int oct = 4 * (q >> 7) + ((q >> 4) & 3), key = 32 * ((q >> 6) & 1) + (q & 15);
                stage[buf].k[oct][key] = halves_of(kr[x][0], kr[x][1]);
                stage[buf].k[oct][key + 16] = halves_of(kr[x][2], kr[x][3]);
            }
        }
    };
    auto put_v = [&](int buf) {
#pragma unroll
        for (int x = 0; x < kPairs; ++x) {
            const int q = tid + kThreads * x;
            if (2 * R % kThreads == 0 || q < 2 * R) {
#pragma unroll
                for (int j = 0; j < 4; ++j) stage[buf].v[2 * j + (q & 1)][q >> 1] = halves_of(vr[x][0][j], vr[x][1][j]);
            }
        }
    };

    // o is in units of vmax, the largest value scale so far: a block's
    // probabilities go to the second product times ratio = its scale / vmax,
    // which the exponent takes, so that the product adds up in place.
    float m = -INFINITY, l = 0.0f, vmax = 0.0f;
    f32x16 o[NT], s[2];                                    // s: scores of the block that is next in line
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[t][v] = 0.0f;
    // Lane (c, h), element v of s[y]: key 32 y + 8 (v / 4) + 4 h + v % 4, row c.
    auto scores = [&](int buf, f32x16 (&x)[2]) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
#pragma unroll
            for (int v = 0; v < 16; ++v) x[y][v] = 0.0f;
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                const f16x8 kf = stage[buf].k[2 * t + h][32 * y + c];
                x[y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qh[t], x[y], 0, 0, 0);
                if constexpr (SPLIT) x[y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, ql[t], x[y], 0, 0, 0);
            }
        }
    };
    auto hide = [&](int i, float ks, f32x16 (&x)[2]) {     // the masked keys of block i
        const int k0 = (start + i) * kBlock;
        if (k0 >= wlo1 && k0 + kBlock <= whi0 && ks >= 0.0f) return;
        int from = ks < 0.0f ? kBlock : lo - k0 - 4 * h, to = hi - k0 - 4 * h;
        __asm__ volatile("" : "+v"(from), "+v"(to));       // keeps the branch: most blocks have no masked keys
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int j = 32 * y + 8 * (v >> 2) + (v & 3);
                x[y][v] = j >= from && j < to ? x[y][v] : -INFINITY;
            }
    };
    auto largest = [&](const f32x16 (&x)[2]) {
        float top = -INFINITY;
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) top = fmaxf(top, x[y][v]);
        return fmaxf(top, __shfl_xor(top, 32, 64));
    };
    // A block's keys are staged two blocks ahead of their exponentials, its
    // values one; scores are computed one ahead. So the matrix cores work on
    // the next scores under a block's exponentials, and on its second product
    // under the staging of later blocks, in one wavefront.
    float ks = 0.0f, top = -INFINITY;
    if (count > 0) {
        look_up(0, id_k, sc_k, a.ks);
        look_up(0, id_v, sc_v, a.vs);
        fetch_k(0);
        fetch_v(0);
        put_k(0);
        put_v(0);
        if (count > 1) {
            fetch_k(1);
            fetch_v(1);
            put_k(1);
        }
        __syncthreads();
        ks = lane_of(sc_k, 0);
        scores(0, s);
        hide(0, ks, s);
        top = largest(s);
        __syncthreads();
        if (count > 2) fetch_k(2);
    }
    for (int i = 0; i < count; ++i) {
        const float vs = lane_of(sc_v, i), ks_next = lane_of(sc_k, min(i + 1, count - 1));
        // (above 0, so that a masked key's -inf stays one)
        const float fk = fmaxf(f * fabsf(ks), 1.17549435e-38f);
        // The maximum may lag behind by 2^kSlack before sums are brought to a new one.
        const float m2 = fmaxf(m, top * fk);
        float change = 1.0f;
        if (vs > vmax) {
            change = vmax * __builtin_amdgcn_rcpf(vs);
            vmax = vs;
        }
        if (m2 > m + kSlack || m == -INFINITY) {
            const float alpha = __builtin_amdgcn_exp2f(m - base_of(m2));
            m = m2;
            l *= alpha;
            change *= alpha;
        }
        if (__builtin_amdgcn_ballot_w64(change != 1.0f)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[t][v] *= change;
        }
        // (2^-60: below what any sum keeps; 1 as long as all scales are 0, where o does not count)
        const float ratio = vmax > 0.0f ? fmaxf(vs * __builtin_amdgcn_rcpf(vmax), 8.67361738e-19f) : 1.0f;
        const float sub = base_of(m) - kLift - __builtin_amdgcn_logf(ratio);
        float sum = 0.0f;
        f16x8 ph[4], pl[4];
        f32x16 next[2];
        scores((i + 1) & 1, next);                         // (of no use after the last block)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(fmaf(s[j >> 1][8 * (j & 1) + e], fk, -sub));
                sum += p[e];
            }
            halve<SPLIT>(p, ph[j], pl[j]);
        }
        l = fmaf(sum, __builtin_amdgcn_rcpf(ratio), l);
        // (keeps the exponentials here, beside the scores' product)
        __asm__ volatile("" : "+v"(ph[0]), "+v"(ph[1]), "+v"(ph[2]), "+v"(ph[3]), "+v"(l));
        if (i + 1 < count) hide(i + 1, ks_next, next);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f16x8 vf = stage[i & 1].v[2 * j + h][32 * t + c];
                o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, ph[j], o[t], 0, 0, 0);
                if constexpr (SPLIT) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pl[j], o[t], 0, 0, 0);
            }
        top = largest(next);
        ks = ks_next;
        // (past the last block: codes of an earlier one once more, which no product takes)
        put_k(i & 1);
        put_v((i + 1) & 1);
        if (i + 3 < count) {
            if (((i + 3) & 63) == 0) look_up(i + 3, id_k, sc_k, a.ks);
            fetch_k(i + 3);
        }
        if (i + 2 < count) {
            if (((i + 2) & 63) == 0) look_up(i + 2, id_v, sc_v, a.vs);
            fetch_v(i + 2);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) s[y] = next[y];
        __syncthreads();
    }
    l += __shfl_xor(l, 32, 64);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[t][v] *= vmax;

    // Lane (c, h), element 4 z + v of o[t]: value 32 t + 8 z + 4 h + v of row c.
    const int64_t unit = (int64_t)u * a.sp.tiles + tile;
    if (ns > 1) {
        constexpr int kOne = kRows * (R + 2);              // floats of a split
        const Shared mem(a.sp.part + unit * a.sp.splits * kOne);
        const int rr = 32 * wave + c;
        if (real) {
            const uint32_t dst = split * kOne + rr * R + 4 * h;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int z = 0; z < 4; ++z)
                    mem.put(dst + 32 * t + 8 * z, (f32x4){o[t][4 * z], o[t][4 * z + 1], o[t][4 * z + 2], o[t][4 * z + 3]});
            if (h == 0) mem.put2(split * kOne + kRows * R + 2 * rr, m, l);
        }
        if (!last_of(a.sp.tickets + unit, ns, &flag)) return;
        if (!real) return;
        m = -INFINITY;
        for (int z = 0; z < ns; ++z) {
            float mz, lz;
            mem.get2(z * kOne + kRows * R + 2 * rr, mz, lz);
            m = fmaxf(m, mz);
        }
        l = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[t][v] = 0.0f;
        for (int z = 0; z < ns; ++z) {
            float mz, lz;
            mem.get2(z * kOne + kRows * R + 2 * rr, mz, lz);
            const float w = __builtin_amdgcn_exp2f(mz - base_of(m));
            l += lz * w;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const f32x4 x = mem.get(z * kOne + rr * R + 4 * h + 32 * t + 8 * y);
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[t][4 * y + v] = fmaf(x[v], w, o[t][4 * y + v]);
                }
        }
    }
    if (!real) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;         // a row without keys gives zeros
    T *dst = (T *)a.out.data + (int64_t)(r0 + i) * a.out.token_stride + (int64_t)head * a.out.head_stride;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            const int d = 32 * t + 8 * z + 4 * h;
            T y[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) y[v] = Type<DT>::put(o[t][4 * z + v] * inv);
            if (a.vec) {
                if (d < a.D) __builtin_memcpy(__builtin_assume_aligned(dst + d, 4 * sizeof(T)), y, 4 * sizeof(T));
            } else {
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (d + v < a.D) dst[d + v] = y[v];
            }
        }
    if (a.sp.lse && h == 0) a.sp.lse[(int64_t)(r0 + i) * (a.heads * a.G) + head] = lse_of(m, l);
}

// The probabilities' sums over the query rows, from the logarithms of the rows'
// sums: the first product again, the other way about. A wavefront keeps 32 keys
// in registers; the rows pass through LDS, 64 at a time.
template <int NT, int DT>
__global__ __launch_bounds__(kThreads, NT > 4 ? 1 : 2) void us_kv_weights_kernel(Args a, float *weights, int64_t stride) {
    using T = typename Type<DT>::T;
    constexpr bool SPLIT = DT == US_F32;
    constexpr int R = 32 * NT, NS = R / 16, kParts = SPLIT ? 2 : 1;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    f16x8(*q)[R / 8][64] = (f16x8(*)[R / 8][64])lds;       // part, octet, row
    __shared__ float rf[64], rz[64];
    __shared__ int rlo[64], rhi[64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 31, h = lane >> 5, hk = blockIdx.y, b = blockIdx.z;
    int r0, n;
    a.s.rows(b, r0, n);
    const int len = a.s.len(b), j0 = blockIdx.x * 128;
    if (j0 >= len || n == 0) return;
    // Rows that see some of these keys.
    int i0 = 0, i1 = n;
    if (a.mask.causal) {
        i0 = max(j0 - (len - n), 0);
        if (a.mask.window > 0) i1 = (int)min((int64_t)n, (int64_t)j0 + 127 + a.mask.window - (len - n));
    }
    const int blk = 2 * (int)blockIdx.x + (wave >> 1);
    const int id = blk * kBlock < len ? a.s.block(b, blk) : -1;
    const int64_t at = (int64_t)max(id, 0) * a.heads + hk;
    const float ks = id < 0 ? 0.0f : a.ks[at];
    f16x8 kf[NS];
    {
        // key 32 (wave & 1) + c, octets 2 t + h
        const uint8_t *p = a.k + at * (kBlock * R) + 1024 * (wave & 1) + 64 * (c & 15) + 8 * (c >> 4);
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            const u32x2 w = *(const u32x2 *)(p + 2048 * (t >> 1) + 16 * (2 * (t & 1) + h));
            kf[t] = halves_of(w[0], w[1]);
        }
    }
    const int k0 = blk * kBlock + 32 * (wave & 1);
    f32x16 sum;
#pragma unroll
    for (int v = 0; v < 16; ++v) sum[v] = 0.0f;
    for (int base = i0 * a.G; base < i1 * a.G; base += 64) {
        __syncthreads();
        {
            const int rr = 16 * wave + (lane & 15), g = lane >> 4, row = base + rr;
            const bool real = row < i1 * a.G;
            const int i = real ? row / a.G : 0, head = hk * a.G + (real ? row - i * a.G : 0);
            RowPart<DT, NT> raw;
            raw.load((const T *)a.q.data + (int64_t)(r0 + i) * a.q.token_stride + (int64_t)head * a.q.head_stride, g, 4, a.D, a.vec);
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
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                f16x8 hi, lo;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[t][e] *= norm;
                halve<SPLIT>(x[t], hi, lo);
                q[0][4 * t + g][rr] = hi;
                if constexpr (SPLIT) q[1][4 * t + g][rr] = lo;
            }
            if (g == 0) {
                int lo = 0, hi = 0;
                if (real) a.mask.range(i, n, len, lo, hi);
                rf[rr] = inv * a.scale;
                rz[rr] = real ? a.sp.lse[(int64_t)(r0 + i) * (a.heads * a.G) + head] : INFINITY;
                rlo[rr] = lo;
                rhi[rr] = hi;
            }
        }
        __syncthreads();
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            f32x16 s;
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = 0.0f;
#pragma unroll
            for (int t = 0; t < NS; ++t)
#pragma unroll
                for (int z = 0; z < kParts; ++z)
                    s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[t], q[z][2 * t + h][32 * y + c], s, 0, 0, 0);
            const float fk = rf[32 * y + c] * ks, z = rz[32 * y + c];
            const int lo = rlo[32 * y + c], hi = rhi[32 * y + c];
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int j = k0 + 8 * (v >> 2) + 4 * h + (v & 3);
                const float p = __builtin_amdgcn_exp2f(fmaf(s[v], fk, -z));
                sum[v] += j >= lo && j < hi ? p : 0.0f;
            }
        }
    }
#pragma unroll
    for (int v = 0; v < 16; ++v)
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) sum[v] += __shfl_xor(sum[v], w, 64);
    if (c == 0 && id >= 0) {
        float *dst = weights + ((int64_t)b * a.heads + hk) * stride;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int j = k0 + 8 * (v >> 2) + 4 * h + (v & 3);
            if (j < len) dst[j] += sum[v];
        }
    }
}

// More than 64 KB of dynamic LDS: allowed once per kernel and device.
template <class K>
hipError_t allow_lds(K kern, std::atomic<unsigned long long> &set) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) dev = 0;
    const unsigned long long bit = 1ull << (dev & 63);
    if (set.load(std::memory_order_acquire) & bit) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 156 * 1024);
    if (e == hipSuccess) set.fetch_or(bit, std::memory_order_release);
    return e;
}

}  // namespace

hipError_t launch_prompt(int dtype, const Args &a, int batch, hipStream_t stream) {
    return with_row(a.D, [&](auto nt) {
        return with_type(dtype, [&](auto dt) {
            constexpr int NT = decltype(nt)::value, kLds = 2 * (int)sizeof(Stage<32 * NT>);
            auto kern = us_kv_prompt_kernel<NT, decltype(dt)::value>;
            if constexpr (kLds > 65536 - 1024) {
                static std::atomic<unsigned long long> set{0};
                const hipError_t e = allow_lds(kern, set);
                if (e != hipSuccess) return e;
            }
            const int units = batch * a.heads;
            hipLaunchKernelGGL(kern, dim3((unsigned)units * a.sp.tiles * a.sp.splits), dim3(kThreads), kLds, stream, a, units);
            return hipGetLastError();
        });
    });
}

hipError_t launch_weights(int dtype, const Args &a, int batch, float *weights, int64_t stride, hipStream_t stream) {
    return with_row(a.D, [&](auto nt) {
        return with_type(dtype, [&](auto dt) {
            constexpr int NT = decltype(nt)::value, DT = decltype(dt)::value;
            constexpr int kLds = (DT == US_F32 ? 2 : 1) * 64 * 32 * NT * 2;
            auto kern = us_kv_weights_kernel<NT, DT>;
            if constexpr (kLds > 65536 - 2048) {
                static std::atomic<unsigned long long> set{0};
                const hipError_t e = allow_lds(kern, set);
                if (e != hipSuccess) return e;
            }
            hipLaunchKernelGGL(kern, dim3((a.s.max_len + 127) / 128, a.heads, batch), dim3(kThreads), kLds, stream, a, weights, stride);
            return hipGetLastError();
        });
    });
}

}  // namespace us_kv
