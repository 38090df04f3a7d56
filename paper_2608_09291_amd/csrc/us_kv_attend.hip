// us_kv_attend: checks, the choice of the kernel and of its split, launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "us_device.h"
#include "us_kv_attend.h"

namespace {

using namespace us_kv;

constexpr us_kv_attend_opts kDefault = {0.0f, 1, 0, 0, nullptr, 0};

// Workgroups of the prompt kernel, whose grid has one dimension of 512 threads each.
constexpr int64_t kMostPrompt = INT32_MAX / 512;

}  // namespace

namespace us_kv {

us_status check_opts(const us_kv_cache *c, const us_kv_seqs *s, int q_heads, const us_kv_attend_opts &o) {
    us_status st = check_cache(c);
    if (st == US_OK) st = check_seqs(s);
    if (st != US_OK) return st;
    if (!(o.scale >= 0.0f && o.scale < INFINITY) || o.causal < 0 || o.causal > 1 || o.window < 0 || (o.window && !o.causal))
        return US_ERR_ARG;
    if ((uintptr_t)o.weights % 4) return US_ERR_ARG;
    if (q_heads < 1 || q_heads % c->heads || q_heads > 65535 || o.max_len < 0) return US_ERR_SHAPE;
    if (o.weights && o.weights_stride < seqs_of(*c, *s, o.max_len, 0).max_len) return US_ERR_SHAPE;
    return US_OK;
}

us_status plan_of(const us_kv_cache &c, const us_kv_seqs &s, int q_heads, int tokens, bool f32, const us_kv_attend_opts &o,
                  Plan &p) {
    const int max_len = seqs_of(c, s, o.max_len, tokens).max_len, R = row_of(c.head_dim);
    const int64_t rows = (int64_t)s.max_new * (q_heads / c.heads), pairs = (int64_t)s.batch * c.heads;
    if (rows > US_KV_NEW_MAX) return US_ERR_SHAPE;
    const int cus = us_device::compute_units(), G = q_heads / c.heads;
    const int64_t all = up(max_len, kBlock) / kBlock;
    // Blocks that the rows of a tile see at most.
    const auto seen = [&](int tile) {
        const int64_t reach = (o.window + (int64_t)(tile + G - 1) / G) / kBlock + 2;
        return o.window && reach < all ? reach : all;
    };
    // Prompt: generations of workgroups, one per CU, times what one takes, in blocks: its own, and 10
    // for storing and joining its partial rows where there are several. (The tokens bound the tiles that
    // have rows where the sequences' numbers of them differ.) us per call, two workgroups per CU and a
    // join by the last of a tile before -> this: 64 queries on 30000 keys, 8 heads over 1, 567 -> 46;
    // 2048 causal, 32 heads, 115 -> 76; 512 on 16000, 64 heads over 8, 336 -> 285.
    const int wide = 32 * prompt_waves(R);
    const int64_t most_w = seen(wide), tiles_w = (rows + wide - 1) / wide;
    const int64_t filled = c.heads * ((int64_t)tokens * G / wide + s.batch);
    const int64_t work = filled < pairs * tiles_w ? filled : pairs * tiles_w;
    int64_t best = INT64_MAX, chunk_w = most_w;
    for (int64_t n = 1; n <= 128 && n <= most_w && (n == 1 || n * pairs * tiles_w <= kMostPrompt); ++n) {
        const int64_t chunk = (most_w + n - 1) / n, t = (work * n + cus - 1) / cus * (chunk + (n > 1 ? 10 : 0));
        if (t < best) {
            best = t;
            chunk_w = chunk;
        }
    }
    // Decode: two workgroups per CU, splits of 4 to 64 blocks.
    const int64_t most_n = seen(16), tiles_n = (rows + 15) / 16, units_n = pairs * tiles_n;
    int64_t chunk_n = up(units_n * most_n / (2 * cus), 4);
    chunk_n = chunk_n < 4 ? 4 : chunk_n > 64 ? 64 : chunk_n;
    // Which of the two, by what they take in us: the decode kernel reads the cache once per 16 rows,
    // from behind the L2s at 10 TB/s if the 256 MB there hold it and at 6 if not, a wavefront takes
    // 1 us for a block, a generation 4 at least; the prompt kernel takes 1.75 us for a block of the
    // above, 2.6 with float32 rows, 2.2 with four wavefronts. us per call, decode and prompt: 64 rows of
    // 4000 keys, 8 sequences of 8 heads of 128, 31 and 46; 128 rows, 16 sequences, 122 and 82; 500
    // causal rows, 32 heads, 17 and 26; 60 rows of 2000 keys, 32 sequences of 32 heads, 347 and 291; 328
    // rows of 43840 keys, 2 sequences of 8 heads, 311 and 192. Of 25 shapes the choice takes the faster
    // one 22 times, and else 1.1 (256 rows of 2000 keys, heads of 256), 1.3 (1000 causal float32 rows, 32
    // heads of 128) and 1.4 times its time (300 rows of 3000 keys, 2 sequences of 8 heads of 192).
    const double cached = (double)(pairs * all) * 128.0 * R, narrow_blocks = (double)units_n * (double)most_n;
    const double read = narrow_blocks * 128.0 * R / (cached <= 256e6 ? 1e7 : 6e6), math = narrow_blocks * R / (128.0 * 4 * cus);
    const double gens = 4.0 * (double)((units_n * ((most_n + chunk_n - 1) / chunk_n) + 2 * cus - 1) / (2 * cus));
    const double narrow = 5.0 + (read > math ? (read > gens ? read : gens) : (math > gens ? math : gens));
    const double broad = 8.0 + (wide < 256 ? 2.2 : f32 ? 2.6 : 1.75) * (double)best;
    // (the scores that weights need are kept up to 64 MB, for up to 16 rows however many there are)
    const bool keeps = !o.weights || rows <= 16 || (double)(pairs * tiles_n * 16) * (double)(all * kBlock) * 4.0 <= 64e6;
    p.decode = rows <= 16 || (narrow <= broad && keeps && tiles_n <= 4096);
    const int64_t most = p.decode ? most_n : most_w;
    const int tile = p.decode ? 16 : wide;
    p.tiles = (int)(p.decode ? tiles_n : tiles_w);
    p.rows = p.decode && rows < 16 ? (int)rows : tile;
    p.chunk = (int)(p.decode ? chunk_n : chunk_w);
    const int64_t units = pairs * p.tiles;
    // Heads of a sequence side by side on an XCD, up to 18 MB of cache. us per call, one by one and so:
    // 8192 causal rows, 32 heads, 655 and 619; 4096, 229 and 164; 2048, 4 sequences, 258 and 203; 16384,
    // 64 heads, 4527 and 4446. (Sequences differ in length: 4 of them side by side 1160 and 1376.)
    const int64_t share = c.heads % 8 == 0 ? c.heads / 8 : 1;
    int64_t mix = 18000000 / (all * 128 * R);
    mix = mix < 1 ? 1 : mix > share ? share : mix;
    while (share % mix) --mix;
    p.mix = (int)mix;
    // (a unit's partial rows lie within 2^31 bytes; decode calls of more units than there are tickets do not split)
    if (p.chunk < (most + 4095) / 4096) p.chunk = (int)((most + 4095) / 4096);
    if ((p.decode && units > kTickets) || most <= p.chunk) p.chunk = (int)most;
    if (p.decode && ((most + p.chunk - 1) / p.chunk) * p.tiles > 65535) p.chunk = (int)((most * p.tiles + 65534) / 65535) + 1;
    p.splits = (int)((most + p.chunk - 1) / p.chunk);
    if (!p.decode && units * p.splits > kMostPrompt) return US_ERR_SHAPE;
    p.scores_stride = up(max_len, kBlock);
    const size_t parts = p.splits > 1 ? (size_t)(units * p.splits) * (size_t)up((int64_t)p.rows * (R + 2), 4) * 4 : 0;
    p.part = parts || o.weights ? 4 * kTickets : 0;        // (also where this call draws none)
    p.ml = p.part + parts;
    // (one block past the last is read)
    p.row_blocks = (int64_t)tokens * (q_heads / c.heads) / 32 + s.batch + 2;
    const size_t rows32 = o.weights ? (size_t)(c.heads * p.row_blocks * 32) : 0;
    p.qf = p.ml + 8 * rows32;
    p.qn = p.qf + (p.decode ? 0 : 4 * rows32);
    p.scores = p.qn + (p.decode ? 0 : (f32 ? 4 : 2) * R * rows32);
    p.total = p.scores + (o.weights && p.decode ? (size_t)(pairs * p.tiles * p.rows * p.scores_stride) * 4 : 0);
    return US_OK;
}

}  // namespace us_kv

extern "C" us_status us_kv_attend_workspace_size(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads,
                                                 int32_t tokens, const us_kv_attend_opts *opts, size_t *bytes) {
    const us_kv_attend_opts &o = opts ? *opts : kDefault;
    us_status st = check_opts(cache, seqs, q_heads, o);
    if (st != US_OK) return st;
    if (!bytes) return US_ERR_ARG;
    if (tokens < 1) return US_ERR_SHAPE;
    // (of either kind of rows)
    Plan p, p32;
    st = plan_of(*cache, *seqs, q_heads, tokens, false, o, p);
    if (st == US_OK) st = plan_of(*cache, *seqs, q_heads, tokens, true, o, p32);
    if (st == US_OK) *bytes = p.total > p32.total ? p.total : p32.total;
    return st;
}

extern "C" us_status us_kv_attend_route(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads, int32_t tokens,
                                        int32_t dtype, const us_kv_attend_opts *opts, us_kv_attend_route_info *out) {
    const us_kv_attend_opts &o = opts ? *opts : kDefault;
    us_status st = check_opts(cache, seqs, q_heads, o);
    if (st != US_OK) return st;
    if (!out || dtype < US_F32 || dtype > US_F16) return US_ERR_ARG;
    if (tokens < 1) return US_ERR_SHAPE;
    Plan p;
    st = plan_of(*cache, *seqs, q_heads, tokens, dtype == US_F32, o, p);
    if (st == US_OK) *out = us_kv_attend_route_info{!p.decode, p.decode ? 16 : p.rows, p.splits, p.chunk};
    return st;
}

extern "C" us_status us_kv_attend(const us_kv_cache *cache, const us_kv_seqs *seqs, int32_t q_heads, const us_rows *q,
                                  const us_rows *out, const us_kv_attend_opts *opts, void *ws, size_t ws_bytes,
                                  void *stream) {
    const us_kv_attend_opts &o = opts ? *opts : kDefault;
    us_status st = check_opts(cache, seqs, q_heads, o);
    if (st == US_OK) st = check_rows(q);
    if (st == US_OK) st = check_rows(out);
    if (st != US_OK) return st;
    if (q->dtype != out->dtype) return US_ERR_ARG;
    if (q->tokens != out->tokens) return US_ERR_SHAPE;
    Plan p;
    st = plan_of(*cache, *seqs, q_heads, q->tokens, q->dtype == US_F32, o, p);
    if (st != US_OK) return st;
    if (o.window && p.total && (!ws || ws_bytes < p.total)) {
        // A workspace of the size for calls without a window (or with another one) serves as well: the
        // plan for all keys is right for any part of them, if with other splits.
        us_kv_attend_opts all = o;
        all.window = 0;
        Plan wide;
        st = plan_of(*cache, *seqs, q_heads, q->tokens, q->dtype == US_F32, all, wide);
        if (st != US_OK) return st;
        p = wide;
    }
    if (p.total && (!ws || (uintptr_t)ws % 16 || ws_bytes < p.total)) return US_ERR_ARG;
    uint8_t *w = (uint8_t *)ws;
    Args a;
    a.k = cache->k, a.v = cache->v, a.ks = cache->k_scale, a.vs = cache->v_scale;
    a.heads = cache->heads, a.D = cache->head_dim, a.G = q_heads / cache->heads;
    a.vec = octets_aligned(*q, cache->head_dim) && octets_aligned(*out, cache->head_dim);
    a.scale = (o.scale > 0.0f ? o.scale : 1.0f / sqrtf((float)cache->head_dim)) * 1.44269504f;
    a.s = seqs_of(*cache, *seqs, o.max_len, q->tokens);
    a.q = Rows{q->data, q->token_stride, q->head_stride};
    a.out = Rows{out->data, out->token_stride, out->head_stride};
    a.mask = Mask{o.causal, o.window};
    a.sp = Split{p.chunk, p.splits, p.tiles, p.rows, p.mix, (float *)(w + p.part), (int32_t *)w,
                 o.weights ? (float2 *)(w + p.ml) : nullptr, p.row_blocks,
                 o.weights && !p.decode ? (f16x8 *)(w + p.qn) : nullptr, (float *)(w + p.qf),
                 o.weights && p.decode ? (float *)(w + p.scores) : nullptr, p.scores_stride};
    const hipStream_t hs = (hipStream_t)stream;
    hipError_t e = p.decode ? launch_decode(q->dtype, a, seqs->batch, hs) : launch_prompt(q->dtype, a, seqs->batch, hs);
    if (e == hipSuccess && o.weights)
        e = p.decode ? launch_weights_saved(a, seqs->batch, o.weights, o.weights_stride, hs)
                     : launch_weights(q->dtype, a, seqs->batch, o.weights, o.weights_stride, hs);
    return e == hipSuccess ? US_OK : US_ERR_DEVICE;
}
