// us_kv_evict: which tokens stay, and their move to new blocks.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "us_device.h"
#include "us_kv_common.h"

namespace {

using namespace us_kv;

constexpr int kMoveThreads = 256;

// Orders like the weights: a NaN first, both zeros alike.
__device__ inline uint32_t order_of(float w) {
    if (!(w == w)) return 0u;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

// Exclusive sum over the workgroup's threads, and the total.
__device__ inline int scan(int x, int *lds, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(sum, o, 64);
        if (lane >= o) sum += y;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = sum;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) {
        if (w < wave) before += lds[w];
        total += lds[w];
    }
    return before + sum - x;
}

// One workgroup per (head, sequence), a run of consecutive tokens per thread.
// The take-th largest weight by its bits, 8 at a time from the top: a histogram
// of the next 8 bits of the weights that agree with the bits found so far. Then
// the positions in order: one sum over the threads' counts places every run.
// Weights of up to kHeld tokens per thread stay in registers over the passes
// (16384 tokens, 128 rows: 57 us with the weights read again for every pass, 31
// so); the loops over them end where the longest run does (700-1100 tokens, 32
// rows: 11.6 us without, 9.0 so).
constexpr int kHeld = 32;
template <int kSelThreads>
__global__ __launch_bounds__(kSelThreads) void us_kv_select_kernel(Seqs s, const float *weights, int64_t w_stride, int keep,
                                                                   int recent, int heads, int32_t *to_lens,
                                                                   float *to_weights, int64_t to_w_stride, int to_w_end,
                                                                   int32_t *index) {
    __shared__ int hist[256], lds[16], found[2];
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int len = s.len(b), stay = min(len, keep), late = min(recent, stay), m = len - late, take = stay - late;
    const float *w = weights + ((int64_t)b * heads + h) * w_stride;
    int32_t *idx = index + ((int64_t)b * heads + h) * keep;
    float *ow = to_weights ? to_weights + ((int64_t)b * heads + h) * to_w_stride : nullptr;
    if (h == 0 && tid == 0) to_lens[b] = stay;
    for (int i = tid; i < late; i += kSelThreads) {
        idx[take + i] = m + i;
        if (ow) ow[take + i] = w[m + i];
    }
    for (uint32_t i = stay + tid; i < (uint32_t)keep; i += kSelThreads) idx[i] = -1;      // (keep goes up to 2^31 - 1)
    // (tokens still to come: us_kv_attend adds to what is there)
    if (ow)
        for (int i = stay + tid; i < to_w_end; i += kSelThreads) ow[i] = 0.0f;
    if (take == 0) return;
    if (take == m) {
        for (int i = tid; i < m; i += kSelThreads) {
            idx[i] = i;
            if (ow) ow[i] = w[i];
        }
        return;
    }

    const int run = __builtin_amdgcn_readfirstlane((m + kSelThreads - 1) / kSelThreads), i0 = min(tid * run, m), n = min(run, m - i0);
    uint32_t held[kHeld];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
        if (j >= run) break;                               // (of all threads at once)
        held[j] = j < n ? order_of(w[i0 + j]) : 0u;
    }
    // f(position, order) for this thread's tokens
    auto each = [&](auto f) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            if (j >= run) break;
            if (j < n) f(i0 + j, held[j]);
        }
        for (int j = kHeld; j < n; ++j) f(i0 + j, order_of(w[i0 + j]));
    };
    uint32_t bits = 0;                                     // of the smallest weight that stays
    int equal = take;                                      // how many of that weight do
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        each([&](int, uint32_t u) {
            if (shift == 24 || (u ^ bits) >> (shift + 8) == 0) atomicAdd(&hist[(u >> shift) & 255u], 1);
        });
        __syncthreads();
        if (tid < 64) {
            // bins from the largest down, four per lane; the one that holds the equal-th
            int c[4], sum = 0;
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                c[z] = hist[255 - 4 * tid - z];
                sum += c[z];
            }
            int above = sum;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int y = __shfl_up(above, o, 64);
                if (tid >= o) above += y;
            }
            above -= sum;
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                if (above < equal && above + c[z] >= equal) {
                    found[0] = 255 - 4 * tid - z;
                    found[1] = equal - above;
                }
                above += c[z];
            }
        }
        __syncthreads();
        bits |= (uint32_t)found[0] << shift;
        equal = found[1];
        __syncthreads();
    }
    int more = 0, same = 0, unused;
    each([&](int, uint32_t u) {
        more += u > bits;
        same += u == bits;
    });
    int left = equal - scan(same, lds, unused);            // of that weight, for this thread and the later ones
    int at = scan(more + min(max(left, 0), same), lds, unused);
    each([&](int i, uint32_t u) {
        if (u > bits || (u == bits && left-- > 0)) {
            idx[at] = i;
            if (ow) ow[at] = w[i];
            ++at;
        }
    });
}

// One workgroup per (new block, head, sequence) for values, per up to four new
// blocks for keys. The index, the block table and the scales of all its tokens
// are looked up together: each of these steps waits for the one before, and
// with one block of keys per workgroup the waits took most of the time. A key's
// octets are copied from where they are. Values lie across their block, so that
// any token of it touches all its lines: every block that has one passes
// through LDS whole. A wavefront does that for its quarter of the values alone,
// four source blocks on their way and no barrier (with the workgroup together,
// one block ahead: 4 sequences of 700-1100 tokens to 512, 8 heads of 128, 13 us
// and 7.7 so; 16 of 9000-16384 to 4096 120, 3 less, where the lines of values
// and keys that it has to touch, some 550 MB, bound it).
// What a wavefront's lanes have stored to LDS, its other lanes find after this.
__device__ inline void in_order() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int kPer = kMoveThreads / kBlock;                // most new blocks of a workgroup
template <int NT>
__global__ __launch_bounds__(kMoveThreads) void us_kv_move_kernel(uint8_t *kp, uint8_t *vp, float *ksp, float *vsp, Seqs s,
                                                                  const int32_t *index, int keep, const int32_t *to,
                                                                  int64_t to_stride, int to_width, int blocks, int key_blocks) {
    constexpr int R = 32 * NT, kOct = R / 8, kPitch = kBlock + 4;
    __shared__ int token[kMoveThreads], from[kMoveThreads], dst[kPer];         // place in its block; block, -1: none
    __shared__ float ratio[kMoveThreads];
    __shared__ __attribute__((aligned(16))) uint8_t in[R * kPitch], out[R * kPitch];
    __shared__ __attribute__((aligned(16))) uint32_t place[kMoveThreads / 64][kBlock];
    __shared__ __attribute__((aligned(16))) float part[kMoveThreads / 64][kBlock];
    const int h = blockIdx.y, b = blockIdx.z, heads = gridDim.y, tid = threadIdx.x;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int total = min(min(s.len(b), keep), to_width * kBlock);
    auto page = [&](int block) { return ((int64_t)block * heads + h) * (kBlock * R); };
    // Values first: a block each, as they take longest.
    if ((int)blockIdx.x < blocks) {
        const int j = blockIdx.x, n = min(total - j * kBlock, kBlock);
        if (n <= 0) return;
        // Every wavefront for itself: a lane per token, then the rows of R / 4 values.
        const int p = lane < n ? index[((int64_t)b * heads + h) * keep + j * kBlock + lane] : -1;
        const int from = p >= 0 ? s.block(b, p / kBlock) : -1, into = s.valid(to[b * to_stride + j]);
        const float s1 = from >= 0 ? vsp[(int64_t)from * heads + h] : 0.0f;    // (not waited for yet)
        place[wave][lane] = value_place(p & (kBlock - 1));
        const int before = __shfl_up(from, 1, 64);
        const uint64_t runs = __builtin_amdgcn_ballot_w64(lane == 0 || from != before);    // first tokens of runs of one source
        constexpr int kOwn = R / 4, kPieces = (4 * kOwn + 63) / 64, kStages = 4, kQuads = 64 / kOwn;
        u32x4 piece[kStages][kPieces];
        uint64_t ahead = runs, left = runs;
        auto fetch = [&](u32x4 (&w)[kPieces]) {            // of the next run, if there is one
            if (!ahead) return;
            const int block = __builtin_amdgcn_readlane(from, __builtin_ctzll(ahead));
            ahead &= ahead - 1;
            if (block < 0) return;
            const u32x4 *src = (const u32x4 *)(vp + page(block)) + 4 * kOwn * wave;
#pragma unroll
            for (int x = 0; x < kPieces; ++x)
                if (4 * kOwn % 64 == 0 || lane + 64 * x < 4 * kOwn) w[x] = src[lane + 64 * x];
        };
#pragma unroll
        for (int z = 0; z < kStages; ++z) fetch(piece[z]);
        float s2 = s1;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s2 = fmaxf(s2, __shfl_xor(s2, o, 64));
        // (a token without a block, or past the last: 0, which makes any byte a code of 0)
        part[wave][lane] = s2 > 0.0f ? s1 / s2 : 0.0f;
        if (into < 0) return;
        if (tid == 0) vsp[(int64_t)into * heads + h] = s2;
        uint8_t *mine_in = in + kOwn * kPitch * wave, *mine_out = out + kOwn * kPitch * wave;
        const int d = lane % kOwn, first = lane / kOwn;    // this lane's row, and which of kQuads quads at a time
        auto move = [&](const u32x4 (&w)[kPieces]) {
            const int t = __builtin_ctzll(left);
            left &= left - 1;
            const int end = left ? __builtin_ctzll(left) : kBlock;
            in_order();
#pragma unroll
            for (int x = 0; x < kPieces; ++x) {
                const int i = lane + 64 * x;
                if (4 * kOwn % 64 == 0 || i < 4 * kOwn) {
                    uint32_t *q = (uint32_t *)(mine_in + (i >> 2) * kPitch + 16 * (i & 3));
#pragma unroll
                    for (int z = 0; z < 4; ++z) q[z] = w[x][z];
                }
            }
            in_order();
            if (first >= kQuads) return;
            for (int quad = (t >> 2) + first; 4 * quad < end; quad += kQuads) {
                const u32x4 at = *(const u32x4 *)&place[wave][4 * quad];
                const float4 r = *(const float4 *)&part[wave][4 * quad];
                const float rv[4] = {r.x, r.y, r.z, r.w};
                uint8_t *q = mine_out + d * kPitch + value_place(4 * quad);
                uint32_t word = 0;
#pragma unroll
                for (int v = 0; v < 4; ++v) word |= rescaled(mine_in[d * kPitch + at[v]], rv[v]) << (8 * v);
                if (4 * quad >= t && 4 * quad + 4 <= end) {
                    *(uint32_t *)q = word;
                } else {
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (4 * quad + v >= t && 4 * quad + v < end) q[v] = (uint8_t)(word >> (8 * v));
                }
            }
        };
        while (left) {
#pragma unroll
            for (int z = 0; z < kStages; ++z)
                if (left) {
                    move(piece[z]);
                    fetch(piece[z]);
                }
        }
        in_order();
        u32x4 *dst = (u32x4 *)(vp + page(into)) + 4 * kOwn * wave;
#pragma unroll
        for (int x = 0; x < kPieces; ++x) {
            const int i = lane + 64 * x;
            if (4 * kOwn % 64 == 0 || i < 4 * kOwn) {
                const uint32_t *q = (const uint32_t *)(mine_out + (i >> 2) * kPitch + 16 * (i & 3));
                dst[i] = (u32x4){q[0], q[1], q[2], q[3]};
            }
        }
        return;
    }
    const int per = key_blocks, j0 = ((int)blockIdx.x - blocks) * per, n = min(total - j0 * kBlock, per * kBlock);
    if (n <= 0) return;
    float *scales = ksp;
    float s1 = 0.0f;
    if (tid < per * kBlock) {                              // a wavefront per new block
        const int p = tid < n ? index[((int64_t)b * heads + h) * keep + j0 * kBlock + tid] : -1;
        const int src = p >= 0 ? s.block(b, p / kBlock) : -1;
        token[tid] = p & (kBlock - 1);
        from[tid] = src;
        if (src >= 0) s1 = scales[(int64_t)src * heads + h];                   // (not waited for yet)
        if (lane == 0) dst[wave] = wave * kBlock < n ? s.valid(to[b * to_stride + j0 + wave]) : -1;
    }
    __syncthreads();
    auto set_ratios = [&]() {
        if (tid < per * kBlock) {
            float s2 = s1;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) s2 = fmaxf(s2, __shfl_xor(s2, o, 64));
            ratio[tid] = s2 > 0.0f ? s1 / s2 : 0.0f;
            if (lane == 0 && dst[wave] >= 0) scales[(int64_t)dst[wave] * heads + h] = s2;
        }
        __syncthreads();
    };
    u32x2 wa[NT], wb[NT];
    auto fetch = [&](int j, u32x2 (&w)[NT]) {
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            const int i = tid + kMoveThreads * x, t = j * kBlock + i / kOct, o = i % kOct;
            w[x] = (u32x2){0x80808080u, 0x80808080u};
            if (t < n && from[t] >= 0) w[x] = *(const u32x2 *)(kp + page(from[t]) + key_octet(token[t], o));
        }
    };
    auto put = [&](int j, const u32x2 (&w)[NT]) {
        if (dst[j] < 0) return;
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            const int i = tid + kMoveThreads * x, t = i / kOct, o = i % kOct;
            const float r = ratio[j * kBlock + t];
            u32x2 q = {0, 0};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                q[e >> 2] |= rescaled((w[x][e >> 2] >> (8 * (e & 3))) & 255u, r) << (8 * (e & 3));
            *(u32x2 *)(kp + page(dst[j]) + key_octet(t, o)) = q;
        }
    };
    const int count = (n + kBlock - 1) / kBlock;
    fetch(0, wa);
    set_ratios();
    for (int j = 0; j < count; j += 2) {
        if (j + 1 < count) fetch(j + 1, wb);
        put(j, wa);
        if (j + 2 < count) fetch(j + 2, wa);
        if (j + 1 < count) put(j + 1, wb);
    }
}

}  // namespace

extern "C" us_status us_kv_evict(const us_kv_cache *cache, const us_kv_seqs *seqs, const float *weights,
                                 int64_t weights_stride, int32_t max_len, int32_t keep, int32_t recent,
                                 const us_kv_kept *to, void *stream) {
    us_status st = check_cache(cache);
    if (st == US_OK) st = check_seqs(seqs);
    if (st != US_OK) return st;
    if (!weights || (uintptr_t)weights % 4 || !to || !to->blocks || !to->lens || !to->index) return US_ERR_ARG;
    if ((uintptr_t)to->blocks % 4 || (uintptr_t)to->lens % 4 || (uintptr_t)to->weights % 4 || (uintptr_t)to->index % 4)
        return US_ERR_ARG;
    if (max_len < 0 || keep < 1 || recent < 0 || recent > keep) return US_ERR_SHAPE;
    const Seqs s = seqs_of(*cache, *seqs, max_len, 0);
    const int most = keep < s.max_len ? keep : s.max_len;
    if (to->width < 1 || to->width > US_KV_WIDTH_MAX || to->stride < to->width || (int64_t)to->width * kBlock < most || weights_stride < s.max_len ||
        (to->weights && to->weights_stride < most))
        return US_ERR_SHAPE;
    // (some heads would be cut by the new length, some weights chosen by moved ones)
    if (to->lens == seqs->lens || to->weights == weights) return US_ERR_ARG;
    const hipStream_t q = (hipStream_t)stream;
    // Four wavefronts meet at a barrier sooner than sixteen: as long as they hold all weights.
    const int64_t to_tokens = (int64_t)to->width * kBlock < to->weights_stride ? (int64_t)to->width * kBlock : to->weights_stride;
    const int to_w_end = (int)to_tokens;                   // (at most 2^28: the widest table's)
    const auto select = [&](auto kern, int threads) {
        hipLaunchKernelGGL(kern, dim3(cache->heads, seqs->batch), dim3(threads), 0, q, s, weights, weights_stride, keep, recent,
                           cache->heads, to->lens, to->weights, to->weights_stride, to_w_end, to->index);
    };
    if (s.max_len <= 256 * kHeld) select(us_kv_select_kernel<256>, 256);
    else select(us_kv_select_kernel<1024>, 1024);
    if (hipGetLastError() != hipSuccess) return US_ERR_DEVICE;
    // (a block per workgroup as long as that leaves some CUs without one)
    const int blocks = (most + kBlock - 1) / kBlock;
    const int per = 2ll * blocks * cache->heads * seqs->batch > 4ll * us_device::compute_units() ? kPer : 1;
    const hipError_t e = with_row(cache->head_dim, [&](auto nt) {
        hipLaunchKernelGGL((us_kv_move_kernel<decltype(nt)::value>),
                           dim3(blocks + (blocks + per - 1) / per, cache->heads, seqs->batch), dim3(kMoveThreads), 0, q, cache->k,
                           cache->v, cache->k_scale, cache->v_scale, s, to->index, keep, to->blocks, to->stride, to->width, blocks, per);
        return hipGetLastError();
    });
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}
