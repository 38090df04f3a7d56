// us_kv_attend_chosen: the attention of single tokens over the blocks that a
// list of each names. The body is that of the attention with few query rows
// (us_kv_decode.h); a token and cache head is a unit, as its list is its own.
// Chosen blocks are 8 KB of keys and 8 KB of values each for heads of 128, read at
// the rate of whole sequences or more, as tokens of a sequence choose alike: 32
// tokens, 8 cache heads, 48 blocks each take 29.5 us, 6.8 TB/s. One token with 64
// takes 10.4 us for 8.4 MB: the start, the first loads, the join of its parts.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "us_device.h"
#include "us_kv_decode.h"

namespace us_kv {
namespace {

template <int NT, int DT>
__global__ __launch_bounds__(kDecodeThreads, NT > 4 ? 1 : 2) void us_kv_chosen_kernel(Args a, Others more) {
    decode_rows<kChosen, NT, DT>(a, more);
}

constexpr us_kv_attend_opts kDefault = {0.0f, 1, 0, 0, nullptr, 0};

struct ChosenPlan {
    int chunk, splits, tiles, rows;
    size_t part, total;
};

us_status chosen_plan(const us_kv_cache &c, int q_heads, int tokens, int top, ChosenPlan &p) {
    const int G = q_heads / c.heads, R = row_of(c.head_dim);
    p.tiles = (G + kDecodeRows - 1) / kDecodeRows;
    p.rows = G < kDecodeRows ? G : kDecodeRows;
    const int64_t units = (int64_t)tokens * c.heads * p.tiles;
    // Two workgroups per CU, of 4 to 64 blocks, as in us_kv_attend.
    int64_t chunk = up(units * top / (2 * us_device::compute_units()), 4);
    chunk = chunk < 4 ? 4 : chunk > 64 ? 64 : chunk;
    if (units > kTickets || top <= chunk) chunk = top;
    if ((top + chunk - 1) / chunk * p.tiles > 65535) chunk = (int64_t)top * p.tiles / 65535 + 1;
    p.chunk = (int)chunk;
    p.splits = (int)((top + chunk - 1) / chunk);
    const size_t one = (size_t)up((int64_t)p.rows * (R + 2), 4) * 4;
    p.part = 4 * kTickets;
    p.total = p.splits > 1 ? p.part + (size_t)(units * p.splits) * one : 0;
    return (int64_t)p.splits * p.tiles > 65535 ? US_ERR_SHAPE : US_OK;
}

us_status check_chosen(const us_kv_cache *c, const us_kv_seqs *s, int q_heads, int tokens, int top, const us_kv_attend_opts &o) {
    const us_status st = check_opts(c, s, q_heads, o);
    if (st != US_OK) return st;
    if (!o.causal || o.window || o.weights) return US_ERR_ARG;
    return tokens < 1 || tokens > 65535 || top < 1 || top > US_KV_CHOSEN_MAX ? US_ERR_SHAPE : US_OK;
}

}  // namespace
}  // namespace us_kv

using namespace us_kv;

extern "C" us_status us_kv_attend_chosen_workspace_size(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads,
                                                        int32_t tokens, int32_t top, size_t *bytes) {
    us_status st = check_chosen(cache, seqs, q_heads, tokens, top, kDefault);
    if (st != US_OK) return st;
    if (!bytes) return US_ERR_ARG;
    ChosenPlan p;
    st = chosen_plan(*cache, q_heads, tokens, top, p);
    if (st == US_OK) *bytes = p.total;
    return st;
}

extern "C" us_status us_kv_attend_chosen(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads, const us_rows *q,
                                         const us_rows *out, const int32_t *chosen, int32_t top,
                                         const us_kv_attend_opts *opts, void *ws, size_t ws_bytes, void *stream) {
    const us_kv_attend_opts &o = opts ? *opts : kDefault;
    us_status st = check_rows(q);
    if (st == US_OK) st = check_rows(out);
    if (st == US_OK) st = check_chosen(cache, seqs, q_heads, q->tokens, top, o);
    if (st != US_OK) return st;
    if (q->dtype != out->dtype || !chosen || (uintptr_t)chosen % 4) return US_ERR_ARG;
    if (q->tokens != out->tokens) return US_ERR_SHAPE;
    ChosenPlan p;
    st = chosen_plan(*cache, q_heads, q->tokens, top, p);
    if (st != US_OK) return st;
    if (p.total && (!ws || (uintptr_t)ws % 16 || ws_bytes < p.total)) return US_ERR_ARG;
    uint8_t *w = (uint8_t *)ws;
    Args a = {};
    a.k = cache->k, a.v = cache->v, a.ks = cache->k_scale, a.vs = cache->v_scale;
    a.heads = cache->heads, a.D = cache->head_dim, a.G = q_heads / cache->heads;
    a.vec = octets_aligned(*q, cache->head_dim) && octets_aligned(*out, cache->head_dim);
    a.scale = (o.scale > 0.0f ? o.scale : 1.0f / sqrtf((float)cache->head_dim)) * 1.44269504f;
    a.s = seqs_of(*cache, *seqs, o.max_len, q->tokens);
    a.q = Rows{q->data, q->token_stride, q->head_stride};
    a.out = Rows{out->data, out->token_stride, out->head_stride};
    a.mask = Mask{1, 0};
    a.sp.chunk = p.chunk, a.sp.splits = p.splits, a.sp.tiles = p.tiles, a.sp.rows = p.rows, a.sp.mix = 1;
    a.sp.part = (float *)(w + p.part), a.sp.tickets = (int32_t *)w;
    Others more = {};
    more.batch = seqs->batch, more.chosen = chosen, more.top = top;
    const dim3 grid(cache->heads, q->tokens, p.splits * p.tiles);
    const hipError_t e = with_row(cache->head_dim, [&](auto nt) {
        return with_type(q->dtype, [&](auto dt) {
            hipLaunchKernelGGL((us_kv_chosen_kernel<decltype(nt)::value, decltype(dt)::value>), grid, dim3(kDecodeThreads), 0,
                               (hipStream_t)stream, a, more);
            return hipGetLastError();
        });
    });
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}
