// The body of the attention kernels with many query rows, of the kinds that
// us_kv_decode.h names (but for lists).
#ifndef UNIONSPARSE_US_KV_PROMPT_H
#define UNIONSPARSE_US_KV_PROMPT_H

#include <atomic>

#include "us_kv_attend.h"
#include "us_kv_others.h"

namespace us_kv {

// A block's keys and values as float16 in LDS, in the order of the operands:
// 16 bytes (8 values of a key; 8 keys of a value) per lane.
template <int R>
struct Stage {
    f16x8 k[R / 8][kBlock];        // octet of values, key
    f16x8 v[8][R];                 // eight keys (2 j + h: 16 j + 4 h + {0..3, 8..11}), value
};

// Stages of blocks, within 160 KB; beside them, of float32 rows above 64, the low parts of the queries.
constexpr bool prompt_low(int row, bool f32) { return f32 && row > 64 && row <= 128; }
constexpr int prompt_stages(int row, bool f32) { return row <= 128 && !prompt_low(row, f32) ? 4 : 2; }

template <int R, bool F32>
constexpr int prompt_lds() {
    return prompt_stages(R, F32) * (int)sizeof(Stage<R>) + (prompt_low(R, F32) ? prompt_waves(R) * R / 16 * 64 * 16 : 0);
}

// More than 64 KB of dynamic LDS: allowed once per kernel and device.
template <class K>
inline hipError_t allow_lds(K kern, std::atomic<unsigned long long> &set) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) dev = 0;
    const unsigned long long bit = 1ull << (dev & 63);
    if (set.load(std::memory_order_acquire) & bit) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 156 * 1024);
    if (e == hipSuccess) set.fetch_or(bit, std::memory_order_release);
    return e;
}

// A score's distance from m as that of its own float: x is the same before its rounding. Both
// passes take a large score's like this, so that the largest one's is 0.
__device__ inline float above(float x, float m) { return (x + m) - m; }

template <int KIND, int NT, int DT, int W>
__device__ __forceinline__ void prompt_rows(const Args a, const Others &more) {
    static_assert(KIND != kChosen);
    using T = typename Type<DT>::T;
    constexpr int kThreads = 64 * W, kRows = 32 * W;       // 32 rows per wavefront
    constexpr StageOrder kOrder{prompt_stages(32 * NT, DT == US_F32)};
    constexpr int kStages = kOrder.stages, kAhead = kOrder.ahead();
    constexpr bool SPLIT = DT == US_F32;
    constexpr int R = 32 * NT, NS = R / 16;                // NS: steps of the first product
    // Float32 rows above 64: the queries' low parts wait in LDS, and scores are not taken
    // ahead, so that two wavefronts fit a SIMD.
    constexpr bool kLow = prompt_low(R, SPLIT), kEarly = !kLow;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Stage<R> *stage = (Stage<R> *)lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 31, h = lane >> 5;
    // The tiles of a unit (sequence, cache head) run on one XCD, whose L2 then
    // serves their keys; of `mix` units together the last tiles, which see the most,
    // first, so that short ones fill the end.
    const int per = a.sp.tiles * a.sp.splits;
    int u = blockIdx.x / per, slot = blockIdx.x % per;
    if (a.heads % 8 == 0) {                                // (all XCDs then get parts of every sequence)
        const int s = blockIdx.x >> 3, turn = s / (per * a.sp.mix), in = s % (per * a.sp.mix);
        u = (turn * a.sp.mix + in % a.sp.mix) * 8 + (blockIdx.x & 7);
        slot = in / a.sp.mix;
    }
    const int tile = a.sp.tiles - 1 - slot / a.sp.splits, split = slot % a.sp.splits;
    int b = u / a.heads;                                   // the row of the table
    const int hk = u - b * a.heads;
    int r0, n, len = 0, cut = 0;
    Group group;
    if constexpr (KIND == kShared) {
        group = more.group(a.s, b);
        b = group.first;
        r0 = group.r0;
        n = group.n;
        cut = group.cut;
    } else {
        a.s.rows(b, r0, n);
        len = a.s.len(b);
        if constexpr (KIND == kRest) cut = more.group_of(a.s, b).cut;
    }
    const int total = n * a.G, base = tile * kRows;
    if (base >= total) return;
    const int last_row = min(base + kRows, total) - 1;
    int lo0 = 0, hi0, lo1, hi1 = cut;
    if constexpr (KIND != kShared) {
        a.mask.range(base / a.G, n, len, lo0, hi0);
        a.mask.range(last_row / a.G, n, len, lo1, hi1);
    }
    if constexpr (KIND == kRest) {
        lo0 = cut;
        hi1 = max(hi1, cut);
    }
    const int first = lo0 / kBlock, end = (hi1 + kBlock - 1) / kBlock;
    const int ns = splits_of(lo0, hi1, a.sp.chunk);
    if (split >= ns) return;
    const int start = first + split * a.sp.chunk, stop = min(start + a.sp.chunk, end);
    // This wavefront's first and last row: keys [all0, all1) are seen by both, and so by all between.
    // Then this lane's row and the keys that it sees.
    const int w0 = min(base + 32 * wave, last_row), w1 = min(base + 32 * wave + 31, last_row);
    int all0 = 0, all1, unused;
    if constexpr (KIND != kShared) {
        a.mask.range(w0 / a.G, n, len, unused, all1);
        a.mask.range(w1 / a.G, n, len, all0, unused);
    }
    const int row = min(base + 32 * wave + c, last_row), i = row / a.G, head = hk * a.G + row - i * a.G;
    const bool real = base + 32 * wave + c <= last_row;
    int lo = 0, hi;
    if constexpr (KIND != kShared) {
        a.mask.range(i, n, len, lo, hi);
        if constexpr (KIND == kRest) lo = all0 = cut;
    } else {                                               // every row has an end of its own
        hi = all1 = group.sees(a.s, a.mask, r0 + i);
#pragma unroll
        for (int z = 1; z < 32; z <<= 1) all1 = min(all1, __shfl_xor(all1, z, 64));
        all1 = __builtin_amdgcn_readfirstlane(all1);
    }

    f16x8 qh[NS], ql[kLow ? 1 : NS];
    f16x8 *low = (f16x8 *)(lds + kStages * sizeof(Stage<R>)) + wave * NS * 64 + lane;
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
            halve<SPLIT>(x, qh[t], ql[kLow ? 0 : t]);
            if constexpr (kLow) low[64 * t] = ql[0];       // (for this lane alone)
        }
    }

    if (KIND == kWhole && a.sp.qn && split == 0 && real) {
        const int64_t rb = row_block(a, hk, b, r0, row);
        constexpr int kParts = SPLIT ? 2 : 1;
        f16x8 *dst = a.sp.qn + rb * (kParts * R / 8 * 32) + h * 32 + c;
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            dst[64 * t] = qh[t];
            if constexpr (SPLIT) dst[64 * t + R / 8 * 32] = kLow ? low[64 * t] : ql[kLow ? 0 : t];
        }
        if (h == 0) a.sp.qf[32 * rb + c] = f;
    }

    // Blocks on their way: 16-byte pieces of the codes in registers.
    constexpr int kPieces = 4 * R / kThreads + (4 * R % kThreads ? 1 : 0);     // of the keys, per thread
    constexpr int kPairs = 2 * R / kThreads + (2 * R % kThreads ? 1 : 0);      // of the values, two pieces each
    u32x4 kr[kPieces], vr[kPairs][2];
    // A lane looks up one of 64 blocks, the next ones when those are used up.
    const int count = stop - start;
    int id_k, id_v;
    float sc_k, sc_v;
    auto look_up = [&](int c, int &id, float &sc, const float *scales) {
        id = -1;
        sc = -1.0f;
        if (c + lane < count) {
            id = a.s.block(b, start + c + lane);
            if (id >= 0) sc = scales[(int64_t)id * a.heads + hk];
        }
    };
    // Blocks on their way: their keys' (values') scales leave with them.
    auto lane_of = [](float x, int c) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), c & 63)); };
    auto fetch_k = [&](int c, float &scale) {
        if (c > 0 && (c & 63) == 0) look_up(c, id_k, sc_k, a.ks);
        scale = lane_of(sc_k, c);
        const uint8_t *kp = a.k + ((int64_t)max(__builtin_amdgcn_readlane(id_k, c & 63), 0) * a.heads + hk) * (kBlock * R);
#pragma unroll
        for (int x = 0; x < kPieces; ++x) {
            // (64 lanes: 16 keys x 4 octets, one KB)
            const int q = tid + kThreads * x;
            if (4 * R % kThreads == 0 || q < 4 * R) kr[x] = *(const u32x4 *)(kp + 1024 * (q >> 6) + 64 * (q & 15) + 16 * ((q >> 4) & 3));
        }
    };
    auto fetch_v = [&](int c, float &scale) {
        if (c > 0 && (c & 63) == 0) look_up(c, id_v, sc_v, a.vs);
        scale = lane_of(sc_v, c);
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
    auto put_k = [&](int blk) {
        const int buf = blk % kStages;
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
    auto put_v = [&](int blk) {
        const int buf = blk % kStages;
#pragma unroll
        for (int x = 0; x < kPairs; ++x) {
            const int q = tid + kThreads * x;
            if (2 * R % kThreads == 0 || q < 2 * R) {
#pragma unroll
                for (int j = 0; j < 4; ++j) stage[buf].v[2 * j + (q & 1)][q >> 1] = halves_of(vr[x][0][j], vr[x][1][j]);
            }
        }
    };

    // A block's value scale goes into its exponents, so that the second product
    // adds up in place: o is in units of 2^(m + mv), m + mv the largest score plus
    // log2 of its block's value scale that this row has seen. Neither a block that
    // is masked for the row nor one of large values and no weight moves it. mv is
    // kept apart from m, so that no score is large enough to take the scale's bits.
    float m = -INFINITY, l = 0.0f, mv = -INFINITY;
    f32x16 o[NT], sa[2], sb[2];                            // scores of a block and of the next one, in turn
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[t][v] = 0.0f;
    // Lane (c, h), element v of s[y]: key 32 y + 8 (v / 4) + 4 h + v % 4, row c.
    auto scores = [&](int blk, f32x16 (&x)[2]) {
        const int buf = blk % kStages;
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) x[y][v] = 0.0f;
        const auto product = [&](int y, int t, f16x8 lo) {
            const f16x8 kf = stage[buf].k[2 * t + h][32 * y + c];
            x[y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qh[t], x[y], 0, 0, 0);
            if constexpr (SPLIT) x[y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, lo, x[y], 0, 0, 0);
        };
        if constexpr (kLow) {
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                const f16x8 lo = low[64 * t];
                product(0, t, lo);
                product(1, t, lo);
            }
        } else {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int t = 0; t < NS; ++t) product(y, t, ql[kLow ? 0 : t]);
        }
    };
    auto hide = [&](int i, float ks, f32x16 (&x)[2]) {     // the masked keys of block i
        const int k0 = (start + i) * kBlock;
        if (k0 >= all0 && k0 + kBlock <= all1 && ks >= 0.0f) return;
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
    // Past kLarge the lift and the unit would be rounded off beside a score: there scores go down by m
    // first.
    auto hold_large = [&](f32x16 (&x)[2], float fk, float bm, float &fs, float &sub, float rest) {
        if (NT <= 4 && !__builtin_amdgcn_ballot_w64(fabsf(bm) > kLarge)) return;
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) x[y][v] = above(fmaf(x[y][v], fk, -bm), bm);
        fs = 1.0f;
        sub = rest;
    };
    // Scores are computed one block ahead of their exponentials, so that the
    // matrix cores work on the next scores under a block's exponentials, and on
    // its second product under the staging of later blocks, in one wavefront.
    // Keys are staged kAhead + 2 blocks ahead, values kAhead + 1: with four
    // stages a barrier serves two blocks.
    float top = -INFINITY;
    float ks[3 + kAhead] = {}, vs[2 + kAhead] = {};        // of block i and the next ones
    if (count > 0) {
        look_up(0, id_k, sc_k, a.ks);
        look_up(0, id_v, sc_v, a.vs);
#pragma unroll
        for (int z = 0; z < kOrder.first_keys(); ++z)
            if (z < count) {
                fetch_k(z, ks[z]);
                if (z < kOrder.first_values()) fetch_v(z, vs[z]);
                put_k(z);
                if (z < kOrder.first_values()) put_v(z);
            }
        if (2 + kAhead < count) fetch_k(2 + kAhead, ks[2 + kAhead]);
        if (1 + kAhead < count) fetch_v(1 + kAhead, vs[1 + kAhead]);
        __syncthreads();
        scores(0, sa);
        hide(0, ks[0], sa);
        top = largest(sa);
        if constexpr (kOrder.barrier_after_first()) __syncthreads();
    }
    auto step = [&](int i, auto odd, f32x16 (&s)[2], f32x16 (&next)[2]) {
        // (above 0, so that a masked key's -inf stays one)
        const float fk = fmaxf(f * fabsf(ks[0]), 1.17549435e-38f);
        // (-200: of a scale of 0, whose values count for nothing)
        const float lv = fmaxf(__builtin_amdgcn_logf(vs[0]), -200.0f);
        // The maxima may lag behind by 2^kSlack before sums are brought to new ones.
        const float t1 = top * fk;
        if (t1 - m > kSlack || m == -INFINITY) {
            const float m2 = fmaxf(m, t1), down = m - base_of(m2);
            l *= __builtin_amdgcn_exp2f(down);
            mv += down;                                    // (o as it is, in units of the new m)
            m = m2;
        }
        const float bm = base_of(m), t2 = t1 - bm + lv;
        float change = 1.0f;
        if (t2 > mv + kSlack || mv == -INFINITY) {
            const float m2 = fmaxf(mv, t2);
            change = __builtin_amdgcn_exp2f(mv - base_of(m2));
            mv = m2;
        }
        if (__builtin_amdgcn_ballot_w64(change != 1.0f)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[t][v] *= change;
        }
        // (60: values of less than 2^-60 of what o holds are lost in it, weights are not)
        const float unit = fminf(base_of(mv) - lv, 60.0f);                     // of p, over 2^m
        float fs = fk, sub = bm + (unit - kLift), sum = 0.0f;
        hold_large(s, fk, bm, fs, sub, unit - kLift);
        f16x8 ph[4], pl[4];
        if constexpr (kEarly) scores(i + 1, next);         // (of no use after the last block)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(fmaf(s[j >> 1][8 * (j & 1) + e], fs, -sub));
                sum += p[e];
            }
            halve<SPLIT>(p, ph[j], pl[j]);
        }
        l = fmaf(sum, __builtin_amdgcn_exp2f(unit), l);
        // (keeps the exponentials here, beside the scores' product)
        __asm__ volatile("" : "+v"(ph[0]), "+v"(ph[1]), "+v"(ph[2]), "+v"(ph[3]), "+v"(l));
        if (kEarly && i + 1 < count) hide(i + 1, ks[1], next);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f16x8 vf = stage[i % kStages].v[2 * j + h][32 * t + c];
                o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, ph[j], o[t], 0, 0, 0);
                if constexpr (SPLIT) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pl[j], o[t], 0, 0, 0);
            }
        if constexpr (!kEarly) {
            scores(i + 1, next);
            if (i + 1 < count) hide(i + 1, ks[1], next);
        }
        top = largest(next);
#pragma unroll
        for (int z = 0; z < 2 + kAhead; ++z) ks[z] = ks[z + 1];
#pragma unroll
        for (int z = 0; z < 1 + kAhead; ++z) vs[z] = vs[z + 1];
        // (past the last block: codes of an earlier one once more, which no product takes)
        put_k(kOrder.puts_keys(i));
        put_v(kOrder.puts_values(i));
        if (i + 3 + kAhead < count) fetch_k(i + 3 + kAhead, ks[2 + kAhead]);
        if (i + 2 + kAhead < count) fetch_v(i + 2 + kAhead, vs[1 + kAhead]);
        if constexpr (kOrder.barrier_after(decltype(odd)::value)) __syncthreads();
    };
    for (int i = 0; i < count; i += 2) {
        step(i, std::integral_constant<int, 0>(), sa, sb);
        if (i + 1 < count) step(i + 1, std::integral_constant<int, 1>(), sb, sa);
    }
    l += __shfl_xor(l, 32, 64);
    const float to_m = __builtin_amdgcn_exp2f(mv);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[t][v] *= to_m;

    // Lane (c, h), element 4 z + v of o[t]: value 32 t + 8 z + 4 h + v of row c.
    if (!real) return;
    if (ns > 1 || KIND != kWhole) {                        // left to the join
        float *dst = a.sp.part + (((int64_t)u * a.sp.tiles + tile) * a.sp.splits + split) * (kRows * (R + 2));
        const int rr = 32 * wave + c;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int z = 0; z < 4; ++z)
                *(f32x4 *)(dst + rr * R + 32 * t + 8 * z + 4 * h) = (f32x4){o[t][4 * z], o[t][4 * z + 1], o[t][4 * z + 2], o[t][4 * z + 3]};
        if (h == 0) {
            dst[kRows * R + 2 * rr] = m;
            dst[kRows * R + 2 * rr + 1] = l;
        }
        return;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int z = 0; z < 4; ++z)
            put_quad<DT>(a, r0 + i, head, 8 * t + 2 * z + h, (f32x4){o[t][4 * z], o[t][4 * z + 1], o[t][4 * z + 2], o[t][4 * z + 3]}, l);
    if (a.sp.ml && h == 0) a.sp.ml[32 * row_block(a, hk, b, r0, row) + row % 32] = ml_of(m, l);
}

}  // namespace us_kv

#endif  // UNIONSPARSE_US_KV_PROMPT_H
