// us_kv_fork: the block tables of sequences that continue others.
//
// Two launches. The first decides every new table entry: a workgroup per
// sequence, which counts the blocks it has to be given; the last workgroup to
// end numbers these over all sequences and finds as many free blocks, lowest
// first. The second writes them into the tables, updates the references and
// copies the started blocks, a workgroup per sequence, head and keys or values.
// The numbers do not depend on the order in which workgroups run: a reference
// count is only read in the first launch and only changed in the second.
//
// What is copied is read and written once, and the tables are small beside it, but
// what a call takes is mostly a chain of looks at memory, about 1 us each: parents,
// lengths, tables, references in the first launch (6.3 us for 8 sequences, 7.1 for
// 64), numbers, tables, blocks in the second (4.6 and 12.0 us; there 55 blocks of 40
// heads of 128 are copied, 36 MB).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "us_kv_attend.h"

namespace {

using namespace us_kv;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kEach = 4;                                  // references of a thread that are on their way together

struct ForkArgs {
    uint8_t *k, *v;
    float *ks, *vs;
    int32_t heads, n_blocks, size;                         // size: bytes of a block
    int32_t *refs;
    const int32_t *blocks, *lens, *parents, *room;
    int64_t stride, to_stride;
    int32_t width, batch, to_width, to_batch;
    int32_t *to_blocks, *to_lens, *missing;
    // The workspace: a ticket; of every old sequence its children and the first of them; of every new one
    // the blocks it is given, the first of these and the one that its started block is copied to (-1); whether
    // there are enough; the free blocks that are given, in order.
    int32_t *ticket, *children, *first_child, *wants, *copy, *short_of, *given;
    int64_t *base;

    __device__ int parent(int b) const {
        const int p = parents ? parents[b] : b;
        return p >= 0 && p < batch ? p : -1;
    }
    __device__ int len(int p) const { return min(max(lens[p], 0), width * kBlock); }
    __device__ int old_block(int p, int i) const {
        if (i >= width) return -1;
        const int id = blocks[p * stride + i];
        return id >= 0 && id < n_blocks ? id : -1;
    }
};

// Written by one workgroup of a launch for another.
__device__ inline void publish(int32_t *p, int32_t x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline int32_t published(const int32_t *p) {
    return __hip_atomic_load(const_cast<int32_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Sum of x over the threads before this one, and over all of them.
template <class T>
__device__ inline T before(T x, T *lds, T &all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T run = x;
#pragma unroll
    for (int z = 1; z < 64; z <<= 1) {
        const T y = __shfl_up(run, z, 64);
        if (lane >= z) run += y;
    }
    __syncthreads();                                       // (of an earlier call)
    if (lane == 63) lds[wave] = run;
    __syncthreads();
    T sum = run - x;
    all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) sum += lds[w];
        all += lds[w];
    }
    return sum;
}

__global__ __launch_bounds__(kThreads) void us_kv_fork_plan_kernel(ForkArgs a) {
    __shared__ int first, children, earlier, flag;
    __shared__ int sums[kWaves];
    __shared__ int64_t wide[kWaves];
    const int x = blockIdx.x, tid = threadIdx.x;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (tid == 0) first = a.to_batch, children = 0, earlier = 0;
    __syncthreads();
    const int p = x < a.to_batch ? a.parent(x) : -1;
    if (a.parents) {
        int n = 0, f = a.to_batch, e = 0;
        for (int j = tid; j < a.to_batch; j += kThreads) {
            const int pj = a.parent(j);
            if (pj == x) {
                ++n;
                f = min(f, j);
            }
            e |= pj >= 0 && pj == p && j < x;
        }
        if (n) {
            atomicAdd(&children, n);
            atomicMin(&first, f);
        }
        if (e) earlier = 1;
        __syncthreads();
    } else if (tid == 0 && x < a.to_batch) {
        first = x;
        children = 1;
    }
    if (x < a.batch && tid == 0) {
        a.children[x] = a.parents ? children : x < a.to_batch ? 1 : 0;
        a.first_child[x] = a.parents ? (children ? first : -1) : x < a.to_batch ? x : -1;
    }
    if (x < a.to_batch) {
        const int len = p < 0 ? 0 : a.len(p), full = len / kBlock, used = (len + kBlock - 1) / kBlock;
        const int64_t room = a.room ? max(a.room[x], 0) : 0;
        const int need = (int)min((len + room + kBlock - 1) / kBlock, (int64_t)a.to_width);
        const bool heir = !earlier;
        int count = 0;                                     // blocks to be given so far
        int32_t *to = a.to_blocks + x * a.to_stride;
        if (tid == 0 && full == a.to_width) a.copy[x] = -1;
        for (int i0 = 0; i0 < a.to_width; i0 += kThreads) {
            const int i = i0 + tid;
            int id = -1;
            bool given = false;
            if (i < need) {                                // (full <= need: the new table is no narrower than the old)
                id = p < 0 ? -1 : a.old_block(p, i);
                // What others hold too, or another child has taken, is not this sequence's to write to.
                if (i >= full && !(heir && id >= 0 && a.refs[id] == 1)) {
                    given = id >= 0 || i >= used;          // (a started block that is not there stays so)
                    if (!given) id = -1;
                }
            }
            int all;
            const int rank = count + before<int>(given, sums, all);
            count += all;
            if (i < a.to_width) to[i] = given ? -2 - rank : id;
            if (i == full && i < a.to_width) a.copy[x] = given && i < used ? rank : -1;
        }
        if (tid == 0) {
            a.to_lens[x] = len;
            publish(a.wants + x, count);
        }
    }
    if (!last_of(a.ticket, gridDim.x, &flag)) return;
    int64_t total = 0;
    for (int b0 = 0; b0 < a.to_batch; b0 += kThreads) {
        const int b = b0 + tid;
        const int64_t n = b < a.to_batch ? published(a.wants + b) : 0;
        int64_t all;
        const int64_t at = total + before<int64_t>(n, wide, all);
        if (b < a.to_batch) a.base[b] = at;
        total += all;
    }
    int64_t found = 0;
    // A wavefront's references, kEach times 64 after each other, 1 past the last; the next ones on their way. (us of
    // this launch for 64 sequences: 16 at a time 11.9, 8 8.8, 4 7.6, with the next on their way 7.0:
    // more code is waited for, and this workgroup does it alone. 100000 blocks of which the last ones alone are
    // free: 68 us a call.)
    int next[kEach];
    const auto look = [&](int64_t r0) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int64_t i = r0 + (wave * kEach + e) * 64 + lane;
            next[e] = i < a.n_blocks ? a.refs[i] : 1;
        }
    };
    look(0);
#pragma unroll 1
    for (int64_t r0 = 0; r0 < a.n_blocks && found < total; r0 += kThreads * kEach) {
        const int64_t at = r0 + wave * kEach * 64;
        int ref[kEach], free = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) ref[e] = next[e];
        look(r0 + kThreads * kEach);
#pragma unroll
        for (int e = 0; e < kEach; ++e) free += __builtin_popcountll(__builtin_amdgcn_ballot_w64(ref[e] == 0));
        __syncthreads();                                   // (of the chunk before)
        if (lane == 0) sums[wave] = free;
        __syncthreads();
        int64_t k = found;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            k += w < wave ? sums[w] : 0;
            found += sums[w];
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const uint64_t mask = __builtin_amdgcn_ballot_w64(ref[e] == 0);
            const int64_t mine = k + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
            if (ref[e] == 0 && mine < total) a.given[mine] = (int)(at + 64 * e + lane);
            k += __builtin_popcountll(mask);
        }
    }
    if (tid == 0) {
        const int64_t lack = total > found ? total - found : 0;
        *a.short_of = lack > 0;
        *a.missing = (int)min(lack, (int64_t)INT32_MAX);
    }
}

__global__ __launch_bounds__(kThreads) void us_kv_fork_apply_kernel(ForkArgs a) {
    const int x = blockIdx.x, tid = threadIdx.x;
    const bool enough = *a.short_of == 0;
    if (blockIdx.y == 0) {
        if (x < a.to_batch) {
            int32_t *to = a.to_blocks + x * a.to_stride;
            for (int i = tid; i < a.to_width; i += kThreads) {
                const int id = to[i];
                if (!enough) {
                    to[i] = -1;
                } else if (id < -1) {
                    const int got = a.given[a.base[x] + (-2 - id)];
                    to[i] = got;
                    atomicAdd(a.refs + got, 1);
                }
            }
            if (!enough && tid == 0) a.to_lens[x] = 0;
        }
        // What the old tables name: one reference less, and one more for every child that shares it. (A block
        // that the first child keeps is in its table; one that it is given instead is free, hence another.)
        if (x < a.batch && enough) {
            const int n = a.children[x], heir = a.first_child[x], full = a.len(x) / kBlock;
            for (int i = tid; i < a.width; i += kThreads) {
                const int id = a.old_block(x, i);
                if (id < 0) continue;
                const int change = i < full ? n - 1 : n && a.to_blocks[heir * a.to_stride + i] == id ? 0 : -1;
                if (change) atomicAdd(a.refs + id, change);
            }
        }
        return;
    }
    if (!enough || x >= a.to_batch || a.copy[x] < 0) return;
    const int head = (blockIdx.y - 1) >> 1, p = a.parent(x);
    const bool values = (blockIdx.y - 1) & 1;
    const int from = a.old_block(p, a.len(p) / kBlock), to = a.given[a.base[x] + a.copy[x]];
    const int64_t src = (int64_t)from * a.heads + head, dst = (int64_t)to * a.heads + head;
    uint8_t *pool = values ? a.v : a.k;
    const u32x4 *s = (const u32x4 *)(pool + src * a.size);
    u32x4 *d = (u32x4 *)(pool + dst * a.size);
#pragma unroll 4
    for (int i = tid; i < a.size / 16; i += kThreads) d[i] = s[i];
    float *scale = values ? a.vs : a.ks;
    if (tid == 0) scale[dst] = scale[src];
}

struct Places {
    int64_t children, first_child, wants, copy, short_of, base, given, total;     // bytes
};
Places places(int batch, int to_batch, int n_blocks) {
    Places p;
    p.children = 16;
    p.first_child = p.children + up(4LL * batch, 16);
    p.wants = p.first_child + up(4LL * batch, 16);
    p.copy = p.wants + up(4LL * to_batch, 16);
    p.short_of = p.copy + up(4LL * to_batch, 16);
    p.base = p.short_of + 16;
    p.given = p.base + up(8LL * to_batch, 16);
    p.total = p.given + up(4LL * n_blocks, 16);
    return p;
}

// Whether two tables share memory. (Where their extents meet, rows of one stride may lie beside each other.)
bool meet(const int32_t *a, int64_t a_stride, int a_width, int a_rows, const int32_t *b, int64_t b_stride, int b_width, int b_rows) {
    const int64_t a0 = (int64_t)((uintptr_t)a / 4), b0 = (int64_t)((uintptr_t)b / 4);
    const auto ends = [](int64_t at, int64_t stride, int width, int rows) { return (__int128)at + (__int128)stride * (rows - 1) + width; };
    if (ends(a0, a_stride, a_width, a_rows) <= b0 || ends(b0, b_stride, b_width, b_rows) <= a0) return false;
    if (a_rows == 1) a_stride = b_stride;
    if (b_rows == 1) b_stride = a_stride;
    if (a_stride != b_stride) return true;
    const int64_t past = ((b0 - a0) % a_stride + a_stride) % a_stride;       // of the start of a's row
    return past < a_width || past + b_width > a_stride;
}

us_status check_to(const us_kv_seqs *s, const us_kv_forked *to) {
    if (!to || !to->blocks || !to->lens || (uintptr_t)to->blocks % 4 || (uintptr_t)to->lens % 4) return US_ERR_ARG;
    if (to->batch < 1 || to->batch > 65535 || to->width < s->width || to->width > US_KV_WIDTH_MAX || to->stride < to->width)
        return US_ERR_SHAPE;
    if (meet(s->blocks, s->stride, s->width, s->batch, to->blocks, to->stride, to->width, to->batch) ||
        meet(s->lens, s->batch, s->batch, 1, to->lens, to->batch, to->batch, 1))
        return US_ERR_ARG;
    return US_OK;
}

}  // namespace

extern "C" us_status us_kv_fork_workspace_size(const us_kv_cache *cache, int32_t batch, int32_t to_batch, size_t *bytes) {
    const us_status st = check_cache(cache);
    if (st != US_OK) return st;
    if (!bytes) return US_ERR_ARG;
    if (batch < 1 || batch > 65535 || to_batch < 1 || to_batch > 65535) return US_ERR_SHAPE;
    *bytes = (size_t)places(batch, to_batch, cache->n_blocks).total;
    return US_OK;
}

extern "C" us_status us_kv_fork(const us_kv_cache *cache, int32_t *refs, const us_kv_seqs *seqs, const int32_t *parents,
                                const int32_t *room, const us_kv_forked *to, int32_t *missing, void *ws, size_t ws_bytes,
                                void *stream) {
    us_status st = check_cache(cache);
    if (st == US_OK) st = check_seqs(seqs);
    if (st == US_OK) st = check_to(seqs, to);
    if (st != US_OK) return st;
    if (!refs || (uintptr_t)refs % 4 || (uintptr_t)parents % 4 || (uintptr_t)room % 4 || !missing || (uintptr_t)missing % 4)
        return US_ERR_ARG;
    const Places p = places(seqs->batch, to->batch, cache->n_blocks);
    if (!ws || (uintptr_t)ws % 16 || ws_bytes < (size_t)p.total) return US_ERR_ARG;
    // (keys and values of every head beside the tables, in the grid's second dimension)
    if (2 * (int64_t)cache->heads + 1 > 65535) return US_ERR_SHAPE;
    uint8_t *w = (uint8_t *)ws;
    ForkArgs a;
    a.k = cache->k, a.v = cache->v, a.ks = cache->k_scale, a.vs = cache->v_scale;
    a.heads = cache->heads, a.n_blocks = cache->n_blocks, a.size = kBlock * row_of(cache->head_dim);
    a.refs = refs, a.blocks = seqs->blocks, a.lens = seqs->lens, a.parents = parents, a.room = room;
    a.stride = seqs->stride, a.to_stride = to->stride, a.width = seqs->width, a.batch = seqs->batch;
    a.to_width = to->width, a.to_batch = to->batch, a.to_blocks = to->blocks, a.to_lens = to->lens, a.missing = missing;
    a.ticket = (int32_t *)w, a.children = (int32_t *)(w + p.children), a.first_child = (int32_t *)(w + p.first_child);
    a.wants = (int32_t *)(w + p.wants), a.copy = (int32_t *)(w + p.copy), a.short_of = (int32_t *)(w + p.short_of);
    a.base = (int64_t *)(w + p.base), a.given = (int32_t *)(w + p.given);
    const int most = a.batch > a.to_batch ? a.batch : a.to_batch;
    hipLaunchKernelGGL(us_kv_fork_plan_kernel, dim3(most), dim3(kThreads), 0, (hipStream_t)stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return US_ERR_DEVICE;
    hipLaunchKernelGGL(us_kv_fork_apply_kernel, dim3(most, 1 + 2 * cache->heads), dim3(kThreads), 0, (hipStream_t)stream, a);
    e = hipGetLastError();
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}
