// us_kv_attend_shared: attention of sequences whose first blocks are the same.
//
// The softmax over all keys of a row is joined from two parts, each with its own
// maximum m, sum l of 2^(x - m) and sum o of these times the values:
//   m = max(m1, m2),  out = (o1 2^(m1 - m) + o2 2^(m2 - m)) / (l1 2^(m1 - m) + l2 2^(m2 - m)).
// The first part's rows are those of all sequences of a group, taken together,
// so that their common keys are read once for all of them; the second's are a
// sequence's over the keys behind. Both take the bodies of us_kv_attend's kernels
// (us_kv_decode.h, us_kv_prompt.h) and leave partial rows. Where both have few
// rows, one launch does it all: the last workgroup that leaves some of a unit's
// joins them. Common keys of many rows have a launch of their own ahead of it. Where
// the sequences themselves have many rows, or there are more units than tickets, a
// third one joins.
//
// Common keys with few rows are bound by memory, with many by the matrix and vector
// units as a prompt is; with the keys of its own, no sequence takes more than in
// us_kv_attend. us on the GPU: 6 sequences of 1 K common tokens 12.7 in one launch
// (about 6 of which every workgroup of this body takes, short as its keys are); 24 of
// 5 documents of 3000 to 12000, 3 tokens each, 98 to 102 (4 or 5 TB/s); 64 of 16 K
// common tokens 53.5 + 27.2, in which the first launch's products take 35 and its
// start, queries and partial rows (34 MB) the rest.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "us_kv_decode.h"
#include "us_kv_prompt.h"

namespace us_kv {
namespace {

template <int NT, int DT>
__global__ __launch_bounds__(kDecodeThreads, NT > 4 ? 1 : 2) void us_kv_shared_few_kernel(Args a, Others more) {
    decode_rows<kPart, NT, DT>(a, more);
}

template <int KIND, int NT, int DT, int W>
__global__ __launch_bounds__(64 * W, NT > 4 ? 1 : 2) void us_kv_shared_many_kernel(Args a, Others more) {
    prompt_rows<KIND, NT, DT, W>(a, more);
}

// What the join takes of either launch.
struct Parts {
    const float *part;
    int32_t chunk, splits, tiles, rows;
};

// A thread per quad of a row's values; a workgroup takes rows of one sequence.
template <int NT, int DT>
__global__ __launch_bounds__(256) void us_kv_shared_join_kernel(Args a, Others more, Parts pre, Parts own) {
    constexpr int R = 32 * NT, kEach = 256 / (R / 4);
    const int b = blockIdx.y, H = a.heads * a.G, quad = threadIdx.x % (R / 4);
    const int64_t place = (int64_t)blockIdx.x * kEach + threadIdx.x / (R / 4);
    int r0, n;
    a.s.rows(b, r0, n);
    Group group = more.group_of(a.s, b);
    if (group.cut > 0) more.rows_of(a.s, group);
    if ((int)threadIdx.x >= kEach * (R / 4) || place >= (int64_t)n * H) return;
    const int i = (int)(place / H), head = (int)(place - (int64_t)i * H), hk = head / a.G, hh = head - hk * a.G;
    float m = -INFINITY, l = 0.0f;
    f32x4 x = {0, 0, 0, 0};
    // Adds the partial rows of one launch: unit u, its row `row`, in ns splits.
    const auto add = [&](const Parts &p, int u, int row, int ns) {
        const int tile = row / p.rows, rr = row - tile * p.rows;
        const int64_t one = up((int64_t)p.rows * (R + 2), 4);
        const float *src = p.part + (((int64_t)u * a.heads + hk) * p.tiles + tile) * p.splits * one;
        float top = m;
#pragma unroll 8
        for (int z = 0; z < ns; ++z) top = fmaxf(top, src[z * one + p.rows * R + 2 * rr]);
        const float bm = base_of(top), down = __builtin_amdgcn_exp2f(m - bm);
        l *= down;
        x *= down;
        m = top;
#pragma unroll 8
        for (int z = 0; z < ns; ++z) {
            const float w = __builtin_amdgcn_exp2f(src[z * one + p.rows * R + 2 * rr] - bm);
            const f32x4 y = *(const f32x4 *)(src + z * one + rr * R + 4 * quad);
            l = fmaf(src[z * one + p.rows * R + 2 * rr + 1], w, l);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = fmaf(y[e], w, x[e]);
        }
    };
    const int row = i * a.G + hh, base = row / own.rows * own.rows;
    if (group.cut > 0) {
        const int at = place_of(r0, group.r0, a.G, row, group.n * a.G);
        if (at >= 0) add(pre, group.number, at, splits_of(0, group.cut, pre.chunk));
    }
    int lo, hi;
    a.mask.range((min(base + own.rows, n * a.G) - 1) / a.G, n, a.s.len(b), lo, hi);
    add(own, b, row, splits_of(group.cut, max(hi, group.cut), own.chunk));
    put_quad<DT>(a, r0 + i, head, quad, x, l);
}

struct SharedPlan {
    Plan pre, own;
    int64_t pre_groups, own_groups;                        // workgroups of either part
    bool inside;                                           // these join
    size_t pre_part, own_part, total;                      // bytes; the tickets lie at 0
};

constexpr int64_t kMost = 1 << 22;

size_t part_bytes(const Plan &p, int64_t pairs, int R) {
    return (size_t)(pairs * p.tiles * p.splits) * (size_t)up((int64_t)p.rows * (R + 2), 4) * 4;
}

constexpr us_kv_attend_opts kDefault = {0.0f, 1, 0, 0, nullptr, 0};

us_status check_shared(const us_kv_cache *c, const us_kv_seqs *s, int q_heads, int tokens, const us_kv_groups *g,
                       const us_kv_attend_opts &o) {
    const us_status st = check_opts(c, s, q_heads, o);
    if (st != US_OK) return st;
    if (!g || !g->starts || !g->shared || (uintptr_t)g->starts % 4 || (uintptr_t)g->shared % 4) return US_ERR_ARG;
    if (o.window || o.weights) return US_ERR_ARG;
    if (tokens < 1 || g->groups < 1 || g->groups > 65535 || g->max_group < 1 || g->max_group > 65535 || g->max_shared < 0 ||
        g->max_shared > s->width)
        return US_ERR_SHAPE;
    // (rows of a group; of a sequence with all heads, which the join has in one dimension of its grid)
    return (int64_t)g->max_group * s->max_new > US_KV_NEW_MAX || (int64_t)s->max_new * q_heads > US_KV_NEW_MAX ? US_ERR_SHAPE : US_OK;
}

// max_shared == 0: as wide as the table.
int most_shared(const us_kv_seqs &s, const us_kv_groups &g) { return g.max_shared ? g.max_shared : s.width; }

us_status shared_plan(const us_kv_cache &c, const us_kv_seqs &s, int q_heads, int tokens, bool f32, const us_kv_groups &g,
                      const us_kv_attend_opts &o, SharedPlan &p) {
    const int R = row_of(c.head_dim), max_len = seqs_of(c, s, o.max_len, tokens).max_len;
    us_kv_seqs all = s;
    all.batch = g.groups;
    all.max_new = g.max_group * s.max_new;
    us_kv_attend_opts first = o;
    first.causal = 0;
    const int64_t common = (int64_t)most_shared(s, g) * kBlock;
    first.max_len = (int)(common < max_len ? common : max_len);
    us_status st = plan_of(c, all, q_heads, tokens, f32, first, p.pre);
    if (st == US_OK) st = plan_of(c, s, q_heads, tokens, f32, o, p.own);
    if (st != US_OK) return st;
    // Of few rows at most 16 parts, as long as these stay below 64 blocks: a join passes over all of them. (One
    // group of 6 sequences, 4 heads over 1, 11456 common tokens, with 45 parts and 12: 27 and 22 us.)
    const int most = (first.max_len + kBlock - 1) / kBlock, chunk = (most + 15) / 16;
    if (p.pre.decode && p.own.decode && p.pre.chunk < chunk) {
        p.pre.chunk = chunk < 64 ? chunk : 64;
        p.pre.splits = (most + p.pre.chunk - 1) / p.pre.chunk;
    }
    const int64_t pre = (int64_t)g.groups * c.heads, own = (int64_t)s.batch * c.heads;
    p.pre_groups = pre * p.pre.tiles * p.pre.splits;
    p.own_groups = own * p.own.tiles * p.own.splits;
    // (in one dimension, of fewer than 2^32 threads)
    if (p.pre_groups > kMost || p.own_groups > kMost) return US_ERR_SHAPE;
    p.inside = p.own.decode && own * p.own.tiles <= kTickets;
    p.pre_part = 4 * kTickets;                             // (also where this call draws none)
    p.own_part = p.pre_part + part_bytes(p.pre, pre, R);
    p.total = p.own_part + part_bytes(p.own, own, R);
    return US_OK;
}

template <int NT, int DT>
hipError_t launch_few(const Args &a, const Others &more, int64_t groups, hipStream_t stream) {
    hipLaunchKernelGGL((us_kv_shared_few_kernel<NT, DT>), dim3((unsigned)groups), dim3(kDecodeThreads), 0, stream, a, more);
    return hipGetLastError();
}

template <int KIND, int NT, int DT>
hipError_t launch_many(const Args &a, const Others &more, int64_t groups, hipStream_t stream) {
    constexpr int R = 32 * NT, W = prompt_waves(R), kLds = prompt_lds<R, DT == US_F32>();
    auto kern = us_kv_shared_many_kernel<KIND, NT, DT, W>;
    if constexpr (kLds > 65536 - 1024) {
        static std::atomic<unsigned long long> set{0};
        const hipError_t e = allow_lds(kern, set);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(64 * W), kLds, stream, a, more);
    return hipGetLastError();
}

Split split_of(const Plan &p, float *part) {
    Split s = {};
    s.chunk = p.chunk, s.splits = p.splits, s.tiles = p.tiles, s.rows = p.rows, s.mix = p.mix, s.part = part;
    return s;
}

}  // namespace
}  // namespace us_kv

using namespace us_kv;

extern "C" us_status us_kv_attend_shared_workspace_size(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads,
                                                        int32_t tokens, const us_kv_groups *groups,
                                                        const us_kv_attend_opts *opts, size_t *bytes) {
    const us_kv_attend_opts &o = opts ? *opts : kDefault;
    us_status st = check_shared(cache, seqs, q_heads, tokens, groups, o);
    if (st != US_OK) return st;
    if (!bytes) return US_ERR_ARG;
    SharedPlan p, p32;                                     // (of either kind of rows)
    st = shared_plan(*cache, *seqs, q_heads, tokens, false, *groups, o, p);
    if (st == US_OK) st = shared_plan(*cache, *seqs, q_heads, tokens, true, *groups, o, p32);
    if (st == US_OK) *bytes = p.total > p32.total ? p.total : p32.total;
    return st;
}

extern "C" us_status us_kv_attend_shared(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads, const us_rows *q,
                                         const us_rows *out, const us_kv_groups *groups, const us_kv_attend_opts *opts, void *ws,
                                         size_t ws_bytes, void *stream) {
    const us_kv_attend_opts &o = opts ? *opts : kDefault;
    us_status st = check_rows(q);
    if (st == US_OK) st = check_rows(out);
    if (st == US_OK) st = check_shared(cache, seqs, q_heads, q->tokens, groups, o);
    if (st != US_OK) return st;
    if (q->dtype != out->dtype) return US_ERR_ARG;
    if (q->tokens != out->tokens) return US_ERR_SHAPE;
    SharedPlan p;
    st = shared_plan(*cache, *seqs, q_heads, q->tokens, q->dtype == US_F32, *groups, o, p);
    if (st != US_OK) return st;
    if (!ws || (uintptr_t)ws % 16 || ws_bytes < p.total) return US_ERR_ARG;
    uint8_t *w = (uint8_t *)ws;
    float *first = (float *)(w + p.pre_part), *second = (float *)(w + p.own_part);
    Args a = {};
    a.k = cache->k, a.v = cache->v, a.ks = cache->k_scale, a.vs = cache->v_scale;
    a.heads = cache->heads, a.D = cache->head_dim, a.G = q_heads / cache->heads;
    a.vec = octets_aligned(*q, cache->head_dim) && octets_aligned(*out, cache->head_dim);
    a.scale = (o.scale > 0.0f ? o.scale : 1.0f / sqrtf((float)cache->head_dim)) * 1.44269504f;
    a.s = seqs_of(*cache, *seqs, o.max_len, q->tokens);
    a.q = Rows{q->data, q->token_stride, q->head_stride};
    a.out = Rows{out->data, out->token_stride, out->head_stride};
    a.mask = Mask{o.causal, 0};
    Others more = {};
    more.batch = seqs->batch, more.group_starts = groups->starts, more.shared = groups->shared;
    more.groups = groups->groups, more.max_group = groups->max_group, more.max_shared = most_shared(*seqs, *groups);
    const hipStream_t hs = (hipStream_t)stream;
    const hipError_t e = with_row(cache->head_dim, [&](auto nt) {
        return with_type(q->dtype, [&](auto dt) {
            constexpr int NT = decltype(nt)::value, DT = decltype(dt)::value, kEach = 256 / (8 * NT);
            more.own = split_of(p.own, second);
            more.own.tickets = (int32_t *)w;
            a.sp = split_of(p.pre, first);
            // (a tile of fewer than 16 rows is the only one)
            more.pre_shift = p.pre.rows < kDecodeRows ? 30 : __builtin_ctz(p.pre.rows);
            hipError_t e = hipSuccess;
            if (!p.pre.decode) e = launch_many<kShared, NT, DT>(a, more, p.pre_groups, hs);
            if (e != hipSuccess) return e;
            more.inside = p.inside;
            more.pre_groups = p.pre.decode ? (int)p.pre_groups : 0;
            const int64_t few = more.pre_groups + (p.own.decode ? p.own_groups : 0);
            if (few) e = launch_few<NT, DT>(a, more, few, hs);
            if (e != hipSuccess || p.inside) return e;
            if (!p.own.decode) {
                a.sp = more.own;
                e = launch_many<kRest, NT, DT>(a, more, p.own_groups, hs);
                if (e != hipSuccess) return e;
            }
            const Parts pre{first, p.pre.chunk, p.pre.splits, p.pre.tiles, p.pre.rows};
            const Parts own{second, p.own.chunk, p.own.splits, p.own.tiles, p.own.rows};
            const unsigned x = (unsigned)(((int64_t)seqs->max_new * q_heads + kEach - 1) / kEach);
            hipLaunchKernelGGL((us_kv_shared_join_kernel<NT, DT>), dim3(x, seqs->batch), dim3(256), 0, hs, a, more, pre, own);
            return hipGetLastError();
        });
    });
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}
