// The body of the attention kernels with few query rows: every key and value is
// read once, for at most 16 rows at a time (the query heads of a cache head, and
// a few tokens). What a workgroup's rows and keys are differs by KIND:
//   kWhole   the rows of a sequence over all keys that they see;
//   kChosen  a token's rows over the blocks that a list of it names;
//   kPart    the rows of a group of sequences over the blocks that these have in common,
//            or those of a sequence over the keys behind (us_kv_shared.hip).
#ifndef UNIONSPARSE_US_KV_DECODE_H
#define UNIONSPARSE_US_KV_DECODE_H

#include "us_kv_attend.h"
#include "us_kv_others.h"

namespace us_kv {

constexpr int kDecodeThreads = 256, kDecodeWaves = 4, kDecodeRows = 16;

// Partial rows of other workgroups, as Shared reads them, at addresses that differ between lanes.
__device__ inline void get_pair(const float *p, float &x, float &y) {
    const uint64_t w = __hip_atomic_load((const uint64_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    x = __uint_as_float((uint32_t)w);
    y = __uint_as_float((uint32_t)(w >> 32));
}
__device__ inline f32x4 get_part(const float *p) {
    float a, b, c, d;
    get_pair(p, a, b);
    get_pair(p + 2, c, d);
    return (f32x4){a, b, c, d};
}

// The end of a kPart workgroup. A unit is a tile of a sequence's rows; it has partial rows over its own keys
// and, in one or two tiles of its group's rows, over the common ones. The last workgroup that leaves some of a
// unit's joins them, in an order that does not depend on who that is. A workgroup over common keys has rows of up
// to 16 units, and joins all that it is the last of together. (The tables may hold anything: both sorts of
// workgroups count a unit's parts from the same numbers.) r0, n, len: of a lane's sequence, the first of which is
// `seq`, up to `seqs`.
template <int NT, int DT>
__device__ inline void join_parts(const Args &a, const Others &more, bool rest, int seq, int seqs, int hk, int tile, const Group &group,
                                  int r0, int n, int len, float *lds) {
    constexpr int R = 32 * NT, kThreads = kDecodeThreads;
    struct Unit {
        int r0, base, rows;                                // of the sequence, and the tile's
        int own, pre;                                      // splits over the sequence's own keys, and over the common ones
        int at, unit;                                      // the first row's place among the group's; number of the unit
    };
    __shared__ Unit list[kDecodeRows];
    __shared__ int found;
    const int tid = threadIdx.x, end = group.n * a.G;
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (tid == 0) found = 0;
    __syncthreads();
    if (tid < 64) {
        const int row0 = tile * kDecodeRows;
#pragma unroll 1
        for (int b = seq + tid; b < seqs; b += 64) {
            int lo, hi;
            if (b != seq + tid) {
                a.s.rows(b, r0, n);
                len = a.s.len(b);
            }
            const int far = place_of(r0, group.r0, a.G, 0, end);               // of its first row
            const int total = n * a.G;
            if (total == 0) continue;                      // (no unit: no workgroup of its own would draw its ticket)
            const bool in = far >= 0 && group.cut > 0;
            const int at0 = in ? far : 0;
            if (!rest && (!in || at0 + total <= row0 || at0 >= row0 + kDecodeRows)) continue;
            const int t0 = rest ? tile : max(row0 - at0, 0) / kDecodeRows;
            const int t1 = rest ? tile : (min(total, row0 + kDecodeRows - at0) - 1) / kDecodeRows;
#pragma unroll 1
            for (int t = t0; t <= t1; ++t) {
                Unit x;
                x.r0 = r0;
                x.base = t * kDecodeRows;
                x.rows = min(total - x.base, kDecodeRows);
                a.mask.range((x.base + x.rows - 1) / a.G, n, len, lo, hi);
                x.own = splits_of(group.cut, max(hi, group.cut), more.own.chunk);
                x.at = at0 + x.base;
                x.pre = in && x.at < end ? splits_of(0, group.cut, a.sp.chunk) : 0;
                x.unit = (b * a.heads + hk) * more.own.tiles + t;
                const int first = x.at >> more.pre_shift, last = (min(x.at + x.rows, end) - 1) >> more.pre_shift;
                if (!rest && (!x.pre || tile < first || tile > last)) continue;
                const int parts = x.own + (more.pre_groups && x.pre ? x.pre * (last - first + 1) : 0);
                int32_t *ticket = more.own.tickets + x.unit;
                if (parts > 1) {
                    if (__hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != parts - 1) continue;
                    __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
                const int i = atomicAdd(&found, 1);
                if (i < kDecodeRows) list[i] = x;
            }
        }
    }
    __syncthreads();
    __asm__ volatile("" ::: "memory");
    const int count = __builtin_amdgcn_readfirstlane(min(found, kDecodeRows));
    if (count == 0) return;
    // The units' rows after each other.
    __shared__ int all_rows, where[kDecodeRows * kDecodeRows];
    if (tid < count) {
        int at = 0;
        for (int f = 0; f < tid; ++f) at += list[f].rows;
        for (int i = 0; i < list[tid].rows; ++i) where[at + i] = tid << 8 | i;
        if (tid == count - 1) all_rows = at + list[tid].rows;
    }
    __syncthreads();
    const int one = (more.own.rows * (R + 2) + 3) / 4 * 4, one_pre = (a.sp.rows * (R + 2) + 3) / 4 * 4;
    // A quad of a row's values per thread, or, where groups have few rows and parts are many, per `runs` of them,
    // which take every runs-th partial row: how many is the same for all workgroups of the call, and with it the
    // order of the sums. (A pass over the rows costs 2 us, eight partial rows more 1 us: 16 sequences of a row each
    // with 54 parts took 41 us with eight.)
    const int items = all_rows * (R / 4), tile_items = a.sp.rows * (R / 4);
    const int runs = a.sp.splits < 16 || tile_items > 64 ? 1 : tile_items > 32 ? 4 : 8;
    const int pass = kThreads / runs, run = tid / pass;
    const int64_t splits = (int64_t)a.sp.splits * one_pre;
    // Partial rows on their way. (us for 6 sequences on 1 K tokens, and 64 on 16 K: 4 13.6, 27.8; 6 12.8, 27.0; 8 13.2,
    // 27.9; 18 15.1, 27.6: more code is waited for.)
    constexpr int kAhead = 6;
#pragma unroll 1
    for (int base = 0; base < items; base += pass) {
        const int it = base + tid - run * pass;
        const bool here = it < items;
        const int place = where[here ? it / (R / 4) : 0], rr = place & 255, quad = it % (R / 4);
        const Unit x = list[place >> 8];
        float m = -INFINITY, l = 0.0f;
        f32x4 y = {0, 0, 0, 0};
        const auto add = [&](float mz, float lz, f32x4 part) {
            const float m2 = fmaxf(m, mz), to = base_of(m2);
            const float down = __builtin_amdgcn_exp2f(m - to), w = __builtin_amdgcn_exp2f(mz - to);
            m = m2;
            l = fmaf(l, down, lz * w);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = fmaf(y[e], down, part[e] * w);
        };
        if (here) {
            // Own parts, then the common ones: addresses of the quad and of (m, l), z-th of ns.
            const int at = x.at + rr, t = at >> more.pre_shift, pr = at - (t << more.pre_shift);
            const float *own = more.own.part + (int64_t)x.unit * more.own.splits * one;
            const float *pre = a.sp.part + (((int64_t)group.number * a.heads + hk) * a.sp.tiles + t) * splits;
            const int ns = x.own + (at < end ? x.pre : 0);
#pragma unroll 1
            for (int z0 = run; z0 < ns; z0 += kAhead * runs) {
                f32x4 part[kAhead];
                float mz[kAhead], lz[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {              // (past the last: it once more, for nothing)
                    const int z = min(z0 + i * runs, ns - 1);
                    const bool mine = z < x.own;
                    const float *src = mine ? own + (int64_t)z * one : pre + (int64_t)(z - x.own) * one_pre;
                    const int row = mine ? rr : pr, rows = mine ? more.own.rows : a.sp.rows;
                    part[i] = get_part(src + row * R + 4 * quad);
                    get_pair(src + rows * R + 2 * row, mz[i], lz[i]);
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (z0 + i * runs < ns) add(mz[i], lz[i], part[i]);
            }
        }
        if (runs > 1) {
            // thread's quad, then its (m, l)
            f32x4 *quads = (f32x4 *)lds;
            float2 *mls = (float2 *)(lds + 4 * kThreads);
            __syncthreads();
            quads[tid] = y;
            mls[tid] = make_float2(m, l);
            __syncthreads();
            if (run == 0 && here)
#pragma unroll 1
                for (int z = 1; z < runs; ++z) {
                    const float2 ml = mls[z * pass + tid];
                    add(ml.x, ml.y, quads[z * pass + tid]);
                }
        }
        if (run == 0 && here) {
            const int gr = x.base + rr, ti = gr / a.G;
            put_quad<DT>(a, x.r0 + ti, hk * a.G + gr - ti * a.G, quad, y, l);
        }
    }
}

template <int KIND, int NT, int DT>
__device__ __forceinline__ void decode_rows(const Args a, const Others &more) {
    constexpr int kThreads = kDecodeThreads, kWaves = kDecodeWaves, kRows = kDecodeRows;
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
    int tile, split, hk, u;
    bool rest = false;                                     // of kPart: the second sort
    if constexpr (KIND == kPart) {
        int x = blockIdx.x;
        rest = x >= more.pre_groups;
        const int units = rest ? more.batch : more.groups, tiles = rest ? more.own.tiles : a.sp.tiles;
        x -= rest ? more.pre_groups : 0;
        hk = x % a.heads;
        x /= a.heads;
        // (the tiles of a group's rows near each other, as they read the same keys: 2 groups of 5 to 16 sequences, 5
        // tokens, 40 heads over 8, 23.8 us; with the groups near each other 27.9)
        tile = x % tiles;
        x /= tiles;
        u = x % units;
        split = x / units;
    } else {
        tile = blockIdx.z % a.sp.tiles, split = blockIdx.z / a.sp.tiles, hk = blockIdx.x, u = blockIdx.y;
    }
    const int chunk = KIND == kPart && rest ? more.own.chunk : a.sp.chunk;
    const int tile_rows = KIND == kPart && rest ? more.own.rows : a.sp.rows;
    // Without a window the first block to look up is known before the length is.
    int guess = -1;
    if constexpr (KIND == kWhole)
        guess = a.s.blocks[u * a.s.stride + min(split * a.sp.chunk + wave + kWaves * lane, (a.s.max_len - 1) / kBlock)];
    // The rows, and the row of the table, b; with a list, the row's own keys end at list_end.
    int r0, n, b = u, len = 0, cut = 0, list_end = 0, unused;
    Group group;
    if constexpr (KIND == kWhole) {
        a.s.rows(b, r0, n);
        len = a.s.len(b);
    } else if constexpr (KIND == kChosen) {
        int at;
        if (!more.place(a.s, u, b, at)) return;
        list_end = at + 1;
        r0 = u;
        n = 1;
    } else if (rest) {
        a.s.rows(b, r0, n);
        len = a.s.len(b);
        group = more.group_of(a.s, b);
        cut = group.cut;
        if (more.inside && cut > 0) more.rows_of(a.s, group);                  // (for the join)
    } else {
        group = more.group(a.s, u);
        b = group.first;
        r0 = group.r0;
        n = group.n;
        cut = group.cut;
        if (cut == 0) return;
    }
    const int total = n * a.G, base = tile * kRows;
    if (base >= total) return;
    const int last_row = min(base + kRows, total) - 1;
    int lo0, hi0, lo1, hi1;                                // of the tile's first and last row
    if constexpr (KIND == kWhole) {
        a.mask.range(base / a.G, n, len, lo0, hi0);
        a.mask.range(last_row / a.G, n, len, lo1, hi1);
    } else if constexpr (KIND == kChosen) {
        lo0 = lo1 = 0;
        hi0 = hi1 = list_end;
    } else if (rest) {
        a.mask.range(base / a.G, n, len, unused, hi0);
        a.mask.range(last_row / a.G, n, len, unused, hi1);
        lo0 = lo1 = cut;
        hi1 = max(hi1, cut);
    } else {
        lo0 = lo1 = 0;
        hi1 = cut;
    }
    // (of a list, places in it)
    const int first = lo0 / kBlock, end = KIND == kChosen ? (list_end > 0 ? more.top : 0) : (hi1 + kBlock - 1) / kBlock;
    const int ns = KIND == kChosen ? (list_end > 0 ? a.sp.splits : 1) : splits_of(lo0, hi1, chunk);
    if (split >= ns) return;
    const int row = min(base + r, last_row), i = row / a.G, head = hk * a.G + row - i * a.G;
    int lo, hi;
    if constexpr (KIND == kWhole) {
        a.mask.range(i, n, len, lo, hi);
    } else if constexpr (KIND == kChosen) {
        lo = 0;
        hi = list_end;
    } else if (rest) {
        a.mask.range(i, n, len, unused, hi);
        lo = cut;
    } else {                                               // every row has an end of its own
        lo = 0;
        hi = hi0 = group.sees(a.s, a.mask, r0 + i);
#pragma unroll
        for (int z = 1; z < 16; z <<= 1) hi0 = min(hi0, __shfl_xor(hi0, z, 64));
        hi0 = __builtin_amdgcn_readfirstlane(hi0);
    }

    // Queries: column r of the first product's right operand.
    RowPart<DT, NT> raw;
    raw.load((const T *)a.q.data + (int64_t)(r0 + i) * a.q.token_stride + (int64_t)head * a.q.head_stride, g, 4, a.D, a.vec);

    // This wavefront's blocks: start, start + 4, ... A lane looks one of them up.
    const int start = first + split * chunk + wave, stop = min(first + (split + 1) * chunk, end);
    int count = start < stop ? (stop - start + kWaves - 1) / kWaves : 0;
    int my_id, my_at = 0;                                  // (my_at: with a list, the block's place in the sequence)
    float my_ks, my_vs;
    auto look_up = [&](int c) {                            // 64 of them, from the c-th on
        my_id = -1;
        my_ks = my_vs = 0.0f;
        if (c + lane < count) {
            const int place = start + kWaves * (c + lane);
            if constexpr (KIND == kWhole) {
                my_id = c == 0 && first == 0 ? a.s.valid(guess) : a.s.block(b, place);
            } else if constexpr (KIND == kChosen) {
                my_at = more.chosen[((int64_t)u * a.heads + hk) * more.top + place];
                if (my_at >= 0 && my_at <= (list_end - 1) / kBlock) my_id = a.s.block(b, my_at);
            } else {
                my_id = a.s.block(b, place);
            }
            if (my_id >= 0) {
                my_ks = a.ks[(int64_t)my_id * a.heads + hk];
                my_vs = a.vs[(int64_t)my_id * a.heads + hk];
            }
        }
    };
    look_up(0);
    if constexpr (KIND == kChosen) {                       // (a list ends in places without a block)
        const uint64_t some = __builtin_amdgcn_ballot_w64(my_id >= 0);
        if (count <= 64) count = some ? 64 - __builtin_clzll(some) : 0;
    }

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
        int blk = start + kWaves * c;
        if constexpr (KIND == kChosen) blk = __builtin_amdgcn_readlane(my_at, c & 63);
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
        if (KIND == kWhole && a.sp.scores && base + r <= last_row) {
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
    // (fields selected one by one: a selected struct would be looked up in memory)
    const int tiles = KIND == kPart && rest ? more.own.tiles : a.sp.tiles, splits = KIND == kPart && rest ? more.own.splits : a.sp.splits;
    float *parts = KIND == kPart && rest ? more.own.part : a.sp.part;
    const int64_t unit = ((int64_t)u * a.heads + hk) * tiles + tile;
    const int rows_here = last_row - base + 1;
    const int one = (tile_rows * (R + 2) + 3) / 4 * 4;     // floats of a split
    const Shared mem(parts + unit * splits * one);
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
            if (ns == 1 && KIND != kPart) {
                put_octet<DT>(a, r0 + ti, hd, c0 / 8 + oc, x, ll);
                if (KIND == kWhole && a.sp.ml && c0 == 0 && oc == 0) a.sp.ml[32 * row_block(a, hk, b, r0, gr) + gr % 32] = ml_of(am, ll);
            } else {
                const uint32_t dst = split * one + rr * R + c0 + 8 * oc;
                mem.put(dst, (f32x4){x[0], x[1], x[2], x[3]});
                mem.put(dst + 4, (f32x4){x[4], x[5], x[6], x[7]});
                if (c0 == 0 && oc == 0) mem.put2(split * one + tile_rows * R + 2 * rr, am, ll);
            }
        }
    }
    if constexpr (KIND == kPart) {
        if (more.inside) {
            __syncthreads();                               // (of the sums' place in LDS)
            join_parts<NT, DT>(a, more, rest, rest ? u : group.first, rest ? u + 1 : group.last, hk, tile, group,
                               rest ? r0 : group.my_r0, rest ? n : group.my_n, rest ? len : group.my_len, (float *)sum);
        }
        return;
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
        if (KIND == kWhole && a.sp.ml && quad == 0) a.sp.ml[32 * row_block(a, hk, b, r0, gr) + gr % 32] = ml_of(am, ll);
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

}  // namespace us_kv

#endif  // UNIONSPARSE_US_KV_DECODE_H
