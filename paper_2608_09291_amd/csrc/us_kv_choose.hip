// us_kv_summarise and us_kv_choose: the extremes of each block's keys, and the
// blocks of highest possible score for every query.
//
// With lo_d <= k_jd <= hi_d for all keys j of a block, q . k_j is at most
//   sum_d max(q_d, 0) hi_d + min(q_d, 0) lo_d,
// a product of 2 D whole codes with 2 D values, of which half are 0. A query is
// held as whole numbers below 2^30 times a power of two, each as four digits in
// [-128, 127] of base 256; the matrix cores multiply digits and codes exactly, in
// 32 bits, 16 blocks by the digits of four query heads at a time, and the digits'
// sums are joined in 64 bits. What a score is off by is the rounding of the
// query's small values (float32: below 2^-7 of its largest one, bfloat16: 2^-23,
// float16: 2^-20), 2^-30 of the largest at most each; two blocks change places
// only where their scores agree to about nine digits. (The same products in 64
// bit floating point: 23.5 us a call with summaries, in place of 16 at that time, for
// 8 sequences of 3000 to 9000, 32 heads.)
//
// A launch reads 2 D bytes of a block and cache head where the attention would
// read 64 times as much, so it is short, and bound by its chain of steps: the row's
// place, queries, digits, block numbers, summaries, products, a ticket, the scores
// again, three to five passes of the choice. us on the GPU (and its bytes' time):
// 131071 keys, 8 cache heads of 128, one query, 12.9 (0.9); 16 sequences of 9000 to
// 16384 and two queries of each, 9.8 (1.4); 8 of 3000 to 9000, 32 heads, 9.4 (1.3);
// with scores alone 6.2 to 8.6. Past 16 query heads to a cache head, lots of 16 after each other: one query on
// 16384 keys, 16 heads over 1 11.1, 32 over 1 19.6. Summaries are HBM's: 32700 keys of 8 heads, 9.0 us,
// 3.7 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "us_device.h"
#include "us_kv_others.h"

namespace {

using namespace us_kv;

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// --- summaries ----------------------------------------------------------------

__device__ inline u16x2 pair_of(uint32_t x) { return __builtin_bit_cast(u16x2, x); }
__device__ inline uint32_t bits_of(u16x2 x) { return __builtin_bit_cast(uint32_t, x); }

// A workgroup per (block, head, sequence), a wavefront per 32 values (the 2 KB of a block that hold these): lane
// (t % 16, octet) has those of 16 byte pieces, tokens t and t + 16.
template <int NT>
__global__ __launch_bounds__(256) void us_kv_summarise_kernel(const uint8_t *kp, uint8_t *summary, Seqs s) {
    constexpr int R = 32 * NT;
    const int b = blockIdx.z, h = blockIdx.y, heads = gridDim.y, tid = threadIdx.x, lane = tid & 63;
    int r0, n;
    s.rows(b, r0, n);
    const int len = s.len(b), p0 = len - n, blk = max(p0, 0) / kBlock + blockIdx.x;
    const int tokens = min(len - blk * kBlock, kBlock);
    if (n <= 0 || tokens <= 0) return;
    const int id = s.block(b, blk);
    if (id < 0) return;
    const int64_t at = (int64_t)id * heads + h;
    const int t0 = lane >> 2;
    for (int c = __builtin_amdgcn_readfirstlane(tid >> 6); c < NT; c += 4) {
        const u32x4 *src = (const u32x4 *)(kp + at * (kBlock * R) + 2048 * c) + lane;
        const u32x4 raw[2] = {src[0], src[64]};
        u16x2 lo[4], hi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) lo[i] = pair_of(0x00FF00FFu), hi[i] = pair_of(0);
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bool here = t0 + 16 * u + 32 * y < tokens;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t w = raw[y][2 * u + (i >> 1)];
                    const u16x2 x = pair_of(__builtin_amdgcn_perm(0, w, i & 1 ? 0x0C030C02u : 0x0C010C00u));
                    const u16x2 a = here ? x : pair_of(0x00FF00FFu), z = here ? x : pair_of(0);
                    lo[i] = __builtin_elementwise_min(lo[i], a);
                    hi[i] = __builtin_elementwise_max(hi[i], z);
                }
            }
#pragma unroll
        for (int z = 4; z < 64; z <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo[i] = __builtin_elementwise_min(lo[i], pair_of(__shfl_xor(bits_of(lo[i]), z, 64)));
                hi[i] = __builtin_elementwise_max(hi[i], pair_of(__shfl_xor(bits_of(hi[i]), z, 64)));
            }
        if (lane < 4) {
            u32x2 *dst = (u32x2 *)(summary + at * (2 * R) + 32 * c) + lane;
            dst[0] = (u32x2){__builtin_amdgcn_perm(bits_of(lo[1]), bits_of(lo[0]), 0x06040200u),
                             __builtin_amdgcn_perm(bits_of(lo[3]), bits_of(lo[2]), 0x06040200u)};
            dst[R / 8] = (u32x2){__builtin_amdgcn_perm(bits_of(hi[1]), bits_of(hi[0]), 0x06040200u),
                                 __builtin_amdgcn_perm(bits_of(hi[3]), bits_of(hi[2]), 0x06040200u)};
        }
    }
}

// --- scores and the choice ------------------------------------------------------

struct ChooseArgs {
    const uint8_t *summary;
    const float *ks;
    int32_t heads, D, G, vec;
    Seqs s;
    Rows q;
    Others more;
    float *scores;                                         // tokens x heads x stride
    int64_t stride;
    int32_t *chosen;                                       // tokens x heads x top
    int32_t top, sinks, recent;
    int32_t *tickets;                                      // tokens x heads
};

// A workgroup's wavefronts, and the keys that it holds in LDS. Where no sequence has more than kFew blocks, four:
// more workgroups fit a CU, and units are many rather than long (3 rows of 20 sequences of 58 blocks, 128 heads
// over 32: 37.7 us a call with eight, with the summaries).
constexpr int kFew = 128;
template <bool FEW>
struct Shape {
    static constexpr int kWaves = FEW ? 4 : 8, kThreads = 64 * kWaves, kHeld = FEW ? kFew : 4096;
    static constexpr int kChunk = 16 * kWaves;             // blocks scored at a time
};
// Chunks that one workgroup takes alone: its scores are keys in LDS at once, without a ticket and a second look at
// them. us of 8 float32 rows, 32 heads over 32, 47 to 141 blocks, alone and with two workgroups where there are two
// chunks: 9.4, 10.5; of 32 rows, 32 over 8, up to 256 blocks: 9.8, 11.7. For four and sixteen chunks, half as many
// workgroups take 1.4 and 1.5 us longer.
constexpr int kAlone = 2;
static_assert(kAlone * Shape<true>::kChunk >= kFew && kAlone * Shape<false>::kChunk >= kFew, "few blocks are one workgroup's");

// Scores in the order of whole numbers; a NaN below all of them, 0 for a block that is not there.
__device__ inline uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);          // (no -0)
    return x != x ? 1u : b >> 31 ? ~b : b | 0x80000000u;
}

// What of a row's scores the workgroup that chooses has in LDS.
template <bool FEW>
struct Pick : Shape<FEW> {
    using Shape<FEW>::kWaves, Shape<FEW>::kHeld;
    __attribute__((aligned(16))) uint32_t keys[kHeld];
    __attribute__((aligned(16))) int hist[FEW ? 1 : 4][256];                   // of the digits, the largest first
    u32x4 of_wave[kWaves];
    int counts[kWaves][2];
};

// The other lanes' x by data-parallel moves, a few cycles each where a permute through LDS takes a hundred.
template <int CTRL, int ROWS>
__device__ inline uint32_t moved(uint32_t none, uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, CTRL, ROWS, 0xF, false);
}
// Lane 63 gets f over all lanes, every lane that of the lanes up to its own; `none` is neutral to f.
template <class F>
__device__ inline uint32_t scan(uint32_t x, uint32_t none, F f) {
    x = f(x, moved<0x111, 0xF>(none, x));                  // from 1, 2, 4 and 8 lanes before, in rows of 16
    x = f(x, moved<0x112, 0xF>(none, x));
    x = f(x, moved<0x114, 0xF>(none, x));
    x = f(x, moved<0x118, 0xF>(none, x));
    x = f(x, moved<0x142, 0xA>(none, x));                  // a row's last lane to the next row, of two
    return f(x, moved<0x143, 0xC>(none, x));               // lane 31 to the upper half
}

// What is known of some keys: how many are there and fixed, the smallest and the largest of the others.
struct Seen {
    uint32_t there = 0, fixed = 0, low = ~0u, high = 0;
    __device__ void add(uint32_t k) {
        there += k != 0;
        fixed += k == ~0u;
        if (k != 0 && k != ~0u) low = min(low, k), high = max(high, k);
    }
};

// The places of the largest `top` of n keys to `out`, ascending, ties to the first. Keys of 0 count for
// nothing, those of ~0 are fixed: taken in any case (they are no more than `top`). The others are sought by 8
// bits of their distance from the smallest of them, shifted so that the largest distance fills 32 bits: the
// scores of a row have most of their first bits in common. Every wavefront follows the whole search, so that a
// step has one barrier. key(i) is asked for places up to the next multiple of kThreads past n, where it is 0.
template <class F>
__device__ inline void select(F key, Seen mine, int n, int top, int *out, Pick<false> &p) {
    constexpr int kWaves = Shape<false>::kWaves, kThreads = Shape<false>::kThreads;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const auto plus = [](uint32_t a, uint32_t b) { return a + b; };
    // A wavefront's places, 64 at a time.
    const int run = (n + kThreads - 1) / kThreads * 64, i0 = wave * run + lane, i1 = i0 + run;
    for (int i = tid; i < 1024; i += kThreads) (&p.hist[0][0])[i] = 0;
    mine.there = scan(mine.there, 0, plus);
    mine.fixed = scan(mine.fixed, 0, plus);
    mine.low = scan(mine.low, ~0u, [](uint32_t a, uint32_t b) { return min(a, b); });
    mine.high = scan(mine.high, 0, [](uint32_t a, uint32_t b) { return max(a, b); });
    if (lane == 63) p.of_wave[wave] = (u32x4){mine.there, mine.fixed, mine.low, mine.high};
    __syncthreads();
    uint32_t there = 0, fixed = 0, low = ~0u, high = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const u32x4 x = p.of_wave[w];
        there += x[0];
        fixed += x[1];
        low = min(low, x[2]);
        high = max(high, x[3]);
    }
    const int take = min(top, (int)there);
    int rest = take - (int)fixed;                          // of those that agree with `limit` in its first bits
    // A key is taken if it is fixed, above the limit, or among the first `rest` at it. Without a search: all that
    // are there, or the fixed ones alone.
    const bool none = take < (int)there && rest <= 0;
    uint32_t limit = 0;
    int shift = 32, up = 0;                                // bits of the limit that are not known yet
    if (take < (int)there && rest > 0) {
        up = high > low ? __builtin_clz(high - low) : 0;
#pragma unroll 1
        for (int step = 0; step < 4; ++step) {
            shift -= 8;
#pragma unroll 4
            for (int i = i0; i < i1; i += 64) {
                const uint32_t x = key(i), k = (x - low) << up;
                if (x != 0 && x != ~0u && (step == 0 || (k ^ limit) >> (shift + 8) == 0)) atomicAdd(&p.hist[step][255 - ((k >> shift) & 255)], 1);
            }
            __syncthreads();
            // lane z: the digits 255 - 4 z .. 252 - 4 z, from the largest on
            const u32x4 bin = *(const u32x4 *)&p.hist[step][4 * lane];
            const int some = (int)(bin[0] + bin[1] + bin[2] + bin[3]);
            int above = (int)scan((uint32_t)some, 0, plus) - some, digit = -1, left = 0, size = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (above < rest && above + (int)bin[i] >= rest) digit = 255 - 4 * lane - i, left = rest - above, size = (int)bin[i];
                above += (int)bin[i];
            }
            const int who = __builtin_ctzll(__builtin_amdgcn_ballot_w64(digit >= 0));          // (there is one: rest is no more than all)
            limit |= (uint32_t)__builtin_amdgcn_readlane(digit, who) << shift;
            rest = __builtin_amdgcn_readlane(left, who);
            if (rest == __builtin_amdgcn_readlane(size, who)) break;           // all that agree so far
        }
        limit >>= shift;
    }
    const auto masks = [&](int i, uint64_t &more, uint64_t &same) {
        const uint32_t x = key(i), k = shift < 32 ? ((x - low) << up) >> shift : 1;
        const bool other = x != 0 && x != ~0u && !none;
        more = __builtin_amdgcn_ballot_w64(x == ~0u || (other && k > limit));
        same = __builtin_amdgcn_ballot_w64(other && k == limit);
    };
    int m = 0, s = 0;
#pragma unroll 4
    for (int i = i0; i < i1; i += 64) {
        uint64_t more, same;
        masks(i, more, same);
        m += __builtin_popcountll(more);
        s += __builtin_popcountll(same);
    }
    if (lane == 0) p.counts[wave][0] = m, p.counts[wave][1] = s;
    __syncthreads();
    m = s = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (w < wave) m += p.counts[w][0], s += p.counts[w][1];
#pragma unroll 4
    for (int i = i0; i < i1; i += 64) {
        uint64_t more, same;
        masks(i, more, same);
        const int mm = m + __builtin_amdgcn_mbcnt_hi((uint32_t)(more >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)more, 0));
        const int ss = s + __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
        if ((more >> lane & 1) || ((same >> lane & 1) && ss < rest)) out[mm + min(ss, rest)] = i;
        m += __builtin_popcountll(more);
        s += __builtin_popcountll(same);
    }
    for (int i = take + tid; i < top; i += kThreads) out[i] = -1;
}

// Lanes that hold a row's octets together: a power of two.
constexpr int lanes_of(int row) { return row <= 64 ? 8 : row <= 128 ? 16 : 32; }

// The same of up to kFew keys in LDS, by counting for each how many come before it: up to a hundred or so,
// that takes less than the steps above.
template <bool FEW>
__device__ inline void select_few(int n, int top, int *out, Pick<FEW> &p) {
    constexpr int kThreads = Shape<FEW>::kThreads;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int before = 0;
    const uint32_t mine = tid < kFew ? p.keys[tid] : 0;
    if (tid < kFew) {
#pragma unroll 2
        for (int j = 0; j < n; j += 4) {
            const u32x4 k = *(const u32x4 *)&p.keys[j];
#pragma unroll
            for (int i = 0; i < 4; ++i) before += j + i < tid ? k[i] >= mine : k[i] > mine;
        }
    }
    const uint64_t taken = __builtin_amdgcn_ballot_w64(mine != 0 && before < top);
    if (lane == 0) p.counts[wave][0] = __builtin_popcountll(taken);
    __syncthreads();
    int first = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kFew / 64; ++w) {
        first += w < wave ? p.counts[w][0] : 0;
        all += p.counts[w][0];
    }
    if (taken >> lane & 1) out[first + __builtin_amdgcn_mbcnt_hi((uint32_t)(taken >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)taken, 0))] = tid;
    for (int i = all + tid; i < top; i += kThreads) out[i] = -1;
}

template <int NT, int DT, bool FEW>
__global__ __launch_bounds__(Shape<FEW>::kThreads) void us_kv_choose_kernel(ChooseArgs a) {
    constexpr int kThreads = Shape<FEW>::kThreads, kChunk = Shape<FEW>::kChunk, kHeld = Shape<FEW>::kHeld;
    using T = typename Type<DT>::T;
    constexpr int R = 32 * NT, kSteps = 2 * R / 64;        // of 64 values of a summary
    constexpr int kLanes = lanes_of(R), kHeads = kThreads / kLanes;            // query heads that are laid out at a time
    constexpr int kGroups = 4;                             // of four query heads, whose digits are columns together
    // The digits as the products' right operand: group, step, lane (column, piece of 16 values).
    __shared__ u32x4 digits[kGroups][kSteps][64];
    __shared__ double unit_of[4 * kGroups];                // a head's power of two; NaN for one that does not count
    __shared__ Pick<FEW> pick;
    __shared__ int flag;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, kk = lane >> 4, t = blockIdx.x, hk = blockIdx.y;
    const T *q = (const T *)a.q.data + (int64_t)t * a.q.token_stride + (int64_t)hk * a.G * a.q.head_stride;
    // This thread's octet of the first heads, on its way while the row's place is looked up.
    const int oct = tid % kLanes;
    RowPart<DT, 1> raw;
    raw.load(q + (int64_t)min(tid / kLanes, a.G - 1) * a.q.head_stride, min(oct, (a.D - 1) / 8), 0, a.D, a.vec);
    int b, at;
    if (!a.more.place(a.s, t, b, at)) return;
    const int64_t unit = (int64_t)t * a.heads + hk;
    const int blocks = at < 0 ? 0 : at / kBlock + 1, chunks = (blocks + kChunk - 1) / kChunk;
    const int parts = chunks <= kAlone ? 1 : min(chunks, (int)gridDim.z);
    if ((int)blockIdx.z >= parts) return;
    float *scores = a.scores + unit * a.stride;
    // Heads g0 .. g0 + 15 (zeros past the last). The first heads are in `raw` for the first chunk of blocks alone: with
    // more than 16, every chunk lays all of them out again, each over the ones before.
    const auto lay_out = [&](int g0, bool fetched) {
        for (int h0 = 0; h0 < min(4 * kGroups, (a.G - g0 + 3) / 4 * 4); h0 += kHeads) {
            const int h = h0 + tid / kLanes, o = oct, g = g0 + h;
            const bool here = h < 4 * kGroups && o < R / 8;
            if (!fetched || g0 + h0 > 0) raw.load(q + (int64_t)min(g, a.G - 1) * a.q.head_stride, min(o, (a.D - 1) / 8), 0, a.D, a.vec);
            float x[8], mx = 0.0f;
            raw.octet(0, o, a.D, false, x);                // (zeros past D)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = g < a.G ? x[e] : 0.0f;
            mx = magnitude(x, mx);
#pragma unroll
            for (int z = kLanes / 2; z > 0; z >>= 1) mx = fmaxf(mx, __shfl_xor(mx, z, 64));
            // 2^k that brings mx to [2^29, 2^30)
            int e2;
            frexpf(mx, &e2);                               // mx in [2^(e2 - 1), 2^e2)
            const int k = mx > 0.0f && mx < INFINITY ? 30 - e2 : 0;
            uint32_t lo[4][2] = {}, hi[4][2] = {};         // by digit, four values to a word
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // (two steps, so that neither power leaves float32's range; past them nothing is rounded but the value)
                const float y = ldexpf(ldexpf(x[e], k / 2), k - k / 2);
                int v = mx < INFINITY ? (int)rintf(y) : 0;
                const bool up = v > 0;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const int digit = (int)(int8_t)v;
                    v = (v - digit) >> 8;
                    const uint32_t byte = (uint32_t)(digit & 255) << (8 * (e & 3));
                    (up ? hi : lo)[d][e >> 2] |= byte;
                }
            }
            if (here) {
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const int col = 4 * (h & 3) + d, c = 8 * o;
                    u32x2 *l = (u32x2 *)&digits[h >> 2][c >> 6][((c >> 4) & 3) * 16 + col] + (o & 1);
                    const int c2 = R + c;
                    u32x2 *u = (u32x2 *)&digits[h >> 2][c2 >> 6][((c2 >> 4) & 3) * 16 + col] + (o & 1);
                    *l = (u32x2){lo[d][0], lo[d][1]};
                    *u = (u32x2){hi[d][0], hi[d][1]};
                }
                if (o == 0) unit_of[h] = g < a.G && mx < INFINITY ? ldexp(1.0, -k) : NAN;
            }
        }
        __syncthreads();
    };
    const auto key_of = [&](int i, bool there, float score) {
        return !there ? 0u : i < a.sinks || i >= blocks - a.recent ? ~0u : min(order_of(score), ~0u - 1);
    };
    // A wavefront's 16 blocks, of which a lane has the n-th; the first ones are on their way ahead of the queries' digits.
    u32x4 codes[kSteps];
    float ks;
    const auto look_up = [&](int c) {
        const int mine = kChunk * c + 16 * wave + n;
        return mine < blocks ? a.s.block(b, mine) : -1;
    };
    const auto fetch = [&](int id) {
        const int64_t where = (int64_t)max(id, 0) * a.heads + hk;
        const u32x4 *src = (const u32x4 *)(a.summary + where * (2 * R)) + kk;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) codes[j] = src[4 * j];
        ks = a.ks[where];
    };
    int id = look_up(blockIdx.z);
    fetch(id);
    if (a.G <= 4 * kGroups) lay_out(0, true);
    const bool alone = FEW || (parts == 1 && blocks <= kHeld);
    for (int c = blockIdx.z; c < chunks; c += parts) {
        const int m0 = kChunk * c + 16 * wave, next = look_up(c + parts);
#pragma unroll
        for (int j = 0; j < kSteps; ++j) codes[j] ^= 0x80808080u;              // bytes less 128
        double best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        for (int g0 = 0; g0 < a.G; g0 += 4 * kGroups) {
            if (a.G > 4 * kGroups) {
                __syncthreads();                           // (the heads before these)
                lay_out(g0, c == (int)blockIdx.z);
            }
            for (int g = 0; g < min(kGroups, (a.G - g0 + 3) / 4); ++g) {
                i32x4 x = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < kSteps; ++j)
                    x = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, codes[j]),
                                                              __builtin_bit_cast(i32x4, digits[g][j][lane]), x, 0, 0, 0);
                // Lane (n, kk), element v: block 4 kk + v, digit n % 4 of query head n / 4. Their sums are whole
                // numbers below 2^47, exact in 64 bits.
                const double weight = ldexp(unit_of[4 * g + (n >> 2)], 8 * (n & 3));
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    double y = (double)x[v] * weight;
                    y += __shfl_xor(y, 1, 64);
                    y += __shfl_xor(y, 2, 64);
                    best[v] = y > best[v] ? y : best[v];
                }
            }
        }
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int z = 4; z < 16; z <<= 1) {
                const double y = __shfl_xor(best[v], z, 64);
                best[v] = y > best[v] ? y : best[v];
            }
        double y = best[0];
#pragma unroll
        for (int v = 1; v < 4; ++v) y = n == v ? best[v] : y;
        const int m = 4 * kk + (n & 3);                    // of the 16, this lane's to store
        const float scale = __shfl(ks, m, 64);
        const bool there = __shfl(id, m, 64) >= 0;
        if (n < 4 && m0 + m < blocks) {
            // (without a finite query head y is -infinity, also times a scale of 0)
            const float score = there && y > -INFINITY ? (float)(y * (double)scale) : -INFINITY;
            __hip_atomic_store(scores + m0 + m, score, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (alone) pick.keys[m0 + m] = key_of(m0 + m, there, score);
        }
        id = next;
        if (c + parts < chunks) fetch(id);
    }
    // Keys past the last block, up to where the choice looks.
    if (alone)
        for (int i = blocks + tid; i < (blocks <= kFew ? kFew : (int)up(blocks, kThreads)); i += kThreads) pick.keys[i] = 0;
    if (!FEW && parts > 1) {
        if (!last_of(a.tickets + unit, parts, &flag)) return;
    } else {
        __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    const auto score_of = [&](int i) { return __hip_atomic_load(scores + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    int *out = a.chosen + unit * a.top;
    if (FEW || blocks <= kFew) {                           // (alone: the keys are there)
        select_few(blocks, a.top, out, pick);
        return;
    }
    if constexpr (!FEW) {
        Seen seen;
        const int per = (blocks + kThreads - 1) / kThreads;
        if (alone) {
            for (int e = 0; e < per; ++e) seen.add(pick.keys[tid + kThreads * e]);
        } else if (blocks <= kHeld) {
#pragma unroll 1
            for (int e0 = 0; e0 < per; e0 += 4) {          // (four on their way together)
                float score[4];
                int block[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = min(tid + kThreads * (e0 + e), blocks - 1);
                    score[e] = score_of(i);
                    block[e] = a.s.block(b, i);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = tid + kThreads * (e0 + e);
                    const uint32_t k = i < blocks ? key_of(i, block[e] >= 0, score[e]) : 0u;
                    if (i < kHeld) pick.keys[i] = k;
                    seen.add(k);
                }
            }
            __syncthreads();
        }
        if (blocks <= kHeld) {
            select([&](int i) { return pick.keys[i]; }, seen, blocks, a.top, out, pick);
        } else {
            const auto key = [&](int i) {
                const int j = min(i, blocks - 1);
                const uint32_t k = key_of(j, a.s.block(b, j) >= 0, score_of(j));
                return i < blocks ? k : 0u;
            };
            for (int e = 0; e < per; ++e) seen.add(key(tid + kThreads * e));
            select(key, seen, blocks, a.top, out, pick);
        }
    }
}

us_status check_summary(const us_kv_cache *c, const us_kv_seqs *s, const uint8_t *summary) {
    us_status st = check_cache(c);
    if (st == US_OK) st = check_seqs(s);
    if (st != US_OK) return st;
    return !summary || (uintptr_t)summary % 16 ? US_ERR_ARG : US_OK;
}

us_status check_units(const us_kv_cache &c, int tokens, int top) {
    return tokens < 1 || tokens > 65535 || top < 1 || top > US_KV_CHOSEN_MAX ? US_ERR_SHAPE : US_OK;
}

}  // namespace

extern "C" us_status us_kv_summarise(const us_kv_cache *cache, const us_kv_seqs *seqs, uint8_t *summary, void *stream) {
    const us_status st = check_summary(cache, seqs, summary);
    if (st != US_OK) return st;
    const Seqs s = seqs_of(*cache, *seqs, 0, INT32_MAX);
    const int most = seqs->max_new < seqs->width * kBlock ? seqs->max_new : seqs->width * kBlock;
    const dim3 grid((most + kBlock - 2) / kBlock + 1, cache->heads, seqs->batch);
    const hipError_t e = with_row(cache->head_dim, [&](auto nt) {
        hipLaunchKernelGGL(us_kv_summarise_kernel<decltype(nt)::value>, grid, dim3(256), 0, (hipStream_t)stream, cache->k, summary, s);
        return hipGetLastError();
    });
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}

extern "C" us_status us_kv_choose_workspace_size(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t tokens, int32_t top,
                                                 size_t *bytes) {
    us_status st = check_cache(cache);
    if (st == US_OK) st = check_seqs(seqs);
    if (st != US_OK) return st;
    if (!bytes) return US_ERR_ARG;
    st = check_units(*cache, tokens, top);
    if (st == US_OK) *bytes = (size_t)up((int64_t)tokens * cache->heads * 4, 16);
    return st;
}

extern "C" us_status us_kv_choose(const us_kv_cache *cache, const us_kv_seqs *seqs, const uint8_t *summary, int32_t q_heads,
                                  const us_rows *q, const us_kv_choice *choice, void *ws, size_t ws_bytes, void *stream) {
    us_status st = check_summary(cache, seqs, summary);
    if (st == US_OK) st = check_rows(q);
    if (st != US_OK) return st;
    if (!choice || !choice->scores || !choice->chosen || (uintptr_t)choice->scores % 4 || (uintptr_t)choice->chosen % 4) return US_ERR_ARG;
    st = check_units(*cache, q->tokens, choice->top);
    if (st != US_OK) return st;
    if (q_heads < 1 || q_heads % cache->heads || q_heads > 65535 || choice->max_len < 0) return US_ERR_SHAPE;
    if (choice->sinks < 0 || choice->recent < 0 || (int64_t)choice->sinks + choice->recent > choice->top) return US_ERR_SHAPE;
    ChooseArgs a;
    a.s = seqs_of(*cache, *seqs, choice->max_len, q->tokens);
    const int most = (int)(up(a.s.max_len, kBlock) / kBlock);
    if (choice->scores_stride < most) return US_ERR_SHAPE;
    const int64_t units = (int64_t)q->tokens * cache->heads;
    if (!ws || (uintptr_t)ws % 16 || ws_bytes < (size_t)up(units * 4, 16)) return US_ERR_ARG;
    a.summary = summary, a.ks = cache->k_scale, a.heads = cache->heads, a.D = cache->head_dim, a.G = q_heads / cache->heads;
    a.vec = octets_aligned(*q, cache->head_dim);
    a.q = Rows{q->data, q->token_stride, q->head_stride};
    a.more = Others{};
    a.more.batch = seqs->batch;
    a.scores = choice->scores, a.stride = choice->scores_stride, a.chosen = choice->chosen;
    a.top = choice->top, a.sinks = choice->sinks, a.recent = choice->recent, a.tickets = (int32_t *)ws;
    // Workgroups of a chunk of blocks, but no more of them than fill the GPU a few times: each has its queries to lay out.
    const bool few = most <= kFew;
    const int chunk = few ? Shape<true>::kChunk : Shape<false>::kChunk;
    const int64_t room = 8 * us_device::compute_units() / units;
    int64_t parts = (most + chunk - 1) / chunk;
    if (parts <= kAlone) parts = 1;
    if (parts > room) parts = room < 1 ? 1 : room;
    const dim3 grid(q->tokens, cache->heads, (unsigned)parts);
    const hipError_t e = with_row(cache->head_dim, [&](auto nt) {
        return with_type(q->dtype, [&](auto dt) {
            constexpr int NT = decltype(nt)::value, DT = decltype(dt)::value;
            const hipStream_t hs = (hipStream_t)stream;
            if (few) hipLaunchKernelGGL((us_kv_choose_kernel<NT, DT, true>), grid, dim3(Shape<true>::kThreads), 0, hs, a);
            else hipLaunchKernelGGL((us_kv_choose_kernel<NT, DT, false>), grid, dim3(Shape<false>::kThreads), 0, hs, a);
            return hipGetLastError();
        });
    });
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}
