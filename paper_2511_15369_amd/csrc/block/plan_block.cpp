// Host-side validation and constants of the block operators, and their C entry points: everything is
// checked here, before anything is enqueued.
#include "../../../include/iptq.h"

#include <math.h>
#include <string.h>

#include "block.h"

using namespace iptq;

static int hip_rc(hipError_t e) { return e == hipSuccess ? IPTQ_OK : IPTQ_ERR_HIP; }

// whether [a, a + na) and [b, b + nb) share a byte
static bool overlap(const void *a, int64_t na, const void *b, int64_t nb)
{
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a && b && na > 0 && nb > 0 && a0 < b0 + (uintptr_t)nb && b0 < a0 + (uintptr_t)na;
}

static bool aligned(const void *p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

static int plan_attention(const iptq_attention_params_t *p, int32_t most_shift, AttentionDev *out)
{
    if (!p) return IPTQ_ERR_NULL;
    if (p->i0 < 16 || p->i0 > 1024 || p->score_shift < 0 || p->score_shift > most_shift) return IPTQ_ERR_PARAM;
    if (p->causal != 0 && p->causal != 1) return IPTQ_ERR_PARAM;
    if (p->n_shift < 0 || p->n_shift > 10) return IPTQ_ERR_PARAM;
    if (((int64_t)p->i0 << p->n_shift) > IPTQ_WEIGHT_MAX) return IPTQ_ERR_RANGE;
    int rc = check_dyadic(&p->post, 1);
    if (rc != IPTQ_OK) return rc;
    // the exponentials are the softmax's: its plan with a probability step that plays no part
    iptq_softmax_params_t s;
    memset(&s, 0, sizeof(s));
    s.variant = p->variant; s.i0 = p->i0; s.n_shift = p->n_shift;
    s.m_bits = 24; s.out_bits = 2;
    s.pre_m = 1;
    s.post.m = 1; s.post.qmax = 255;
    SoftmaxDev d;
    rc = plan_softmax(&s, 1, 1, 0, 0, &d);
    if (rc != IPTQ_OK) return rc;
    if (d.packed != 2) return IPTQ_ERR_RANGE;
    out->variant = p->variant; out->i0 = p->i0; out->i0n = d.i0n; out->n_shift = p->n_shift;
    out->d_clamp = d.d_clamp; out->div8 = d.div8; out->d2_magic = d.d2_magic; out->d2_sh = d.d2_sh;
    out->shift = p->score_shift; out->causal = p->causal;
    out->post_shift = shift_of(p->post.m, p->post.s, p->post.s >= 16);
    return plan_requant(&p->post, 1, &out->post);
}

static bool head_dim_served(int32_t dim) { return dim == 32 || dim == 64 || dim == 96 || dim == 128; }

static int check_heads(int32_t heads, int32_t kv_heads, int32_t dim)
{
    if (heads < 1 || kv_heads < 1 || heads > 4096 || heads % kv_heads != 0 || !head_dim_served(dim)) return IPTQ_ERR_SHAPE;
    return IPTQ_OK;
}

// bytes that `tokens` rows of `width` bytes, `stride` apart, reach over
static int64_t extent(int64_t tokens, int64_t stride, int64_t width) { return tokens > 0 ? (tokens - 1) * stride + width : 0; }

extern "C" int iptq_attention_i8(const int8_t *d_q, int64_t q_stride, const int8_t *d_k, int64_t k_stride, const int8_t *d_v,
                                 int64_t v_stride, const int32_t *d_q_offsets, const int32_t *d_k_offsets, int32_t n_seq,
                                 int32_t max_q, int64_t q_tokens, int64_t k_tokens, int32_t heads, int32_t kv_heads,
                                 int32_t head_dim, int8_t *d_out, int64_t out_stride, const iptq_attention_params_t *p,
                                 void *stream)
{
    AttentionCall c;
    int rc = plan_attention(p, IPTQ_SCORE_SHIFT_MAX, &c.P);
    if (rc != IPTQ_OK) return rc;
    rc = check_heads(heads, kv_heads, head_dim);
    if (rc != IPTQ_OK) return rc;
    const int64_t tokens_most = ((int64_t)1 << 31) - 256;        // (rows are counted past a tile's last in 32 bits)
    if (n_seq < 0 || max_q < 0 || q_tokens < 0 || k_tokens < 0 || q_tokens >= tokens_most || k_tokens >= tokens_most)
        return IPTQ_ERR_SHAPE;
    const int64_t qw = (int64_t)heads * head_dim, kw = (int64_t)kv_heads * head_dim, stride_most = (int64_t)1 << 31;
    if (q_stride < qw || out_stride < qw || k_stride < kw || v_stride < kw || q_stride >= stride_most ||
        out_stride >= stride_most || k_stride >= stride_most || v_stride >= stride_most)
        return IPTQ_ERR_SHAPE;
    if (!d_q_offsets != !d_k_offsets) return IPTQ_ERR_NULL;
    if (!d_q_offsets) {                                   // equal lengths
        if (n_seq > 0 && (q_tokens % n_seq != 0 || k_tokens % n_seq != 0 || k_tokens / n_seq > IPTQ_KEYS_MAX))
            return IPTQ_ERR_SHAPE;
        if (n_seq == 0 && (q_tokens != 0 || k_tokens != 0)) return IPTQ_ERR_SHAPE;
        if (n_seq > 0 && q_tokens / n_seq < max_q) max_q = (int32_t)(q_tokens / n_seq);
    }
    if (n_seq == 0 || max_q == 0 || q_tokens == 0) return IPTQ_OK;
    if (max_q > q_tokens) max_q = (int32_t)q_tokens;
    const int64_t tiles = ((int64_t)max_q + 31) / 32;
    if (tiles * n_seq * heads >= ((int64_t)1 << 31)) return IPTQ_ERR_SHAPE;
    if (!d_q || !d_out || (k_tokens > 0 && (!d_k || !d_v))) return IPTQ_ERR_NULL;
    if (!aligned(d_q_offsets, 4) || !aligned(d_k_offsets, 4)) return IPTQ_ERR_ALIGN;
    const int64_t out_bytes = extent(q_tokens, out_stride, qw);
    if (overlap(d_out, out_bytes, d_q, extent(q_tokens, q_stride, qw)) || overlap(d_out, out_bytes, d_k, extent(k_tokens, k_stride, kw)) ||
        overlap(d_out, out_bytes, d_v, extent(k_tokens, v_stride, kw)) ||
        overlap(d_out, out_bytes, d_q_offsets, ((int64_t)n_seq + 1) * 4) || overlap(d_out, out_bytes, d_k_offsets, ((int64_t)n_seq + 1) * 4))
        return IPTQ_ERR_PARAM;
    c.q = d_q; c.k = d_k; c.v = d_v; c.out = d_out;
    c.q_stride = q_stride; c.k_stride = k_stride; c.v_stride = v_stride; c.out_stride = out_stride;
    c.q_offsets = d_q_offsets; c.k_offsets = d_k_offsets;
    c.q_tokens = q_tokens; c.k_tokens = k_tokens;
    c.n_seq = n_seq; c.max_q = max_q; c.heads = heads; c.kv_heads = kv_heads; c.dim = head_dim;
    return hip_rc(attention_i8_dispatch(c, static_cast<hipStream_t>(stream)));
}

static int plan_cache(const iptq_cache_i4_t *cache, CacheDev *out)
{
    if (!cache) return IPTQ_ERR_NULL;
    if (!head_dim_served(cache->head_dim) || cache->kv_heads < 1 || cache->kv_heads > 4096 || cache->n_pages < 1) return IPTQ_ERR_SHAPE;
    const int32_t t = cache->page_tokens;
    if (t < 16 || t > 4096 || (t & (t - 1)) != 0) return IPTQ_ERR_SHAPE;
    if ((int64_t)cache->n_pages * t >= ((int64_t)1 << 31)) return IPTQ_ERR_SHAPE;
    if (!cache->d_k_codes || !cache->d_k_steps || !cache->d_v_codes || !cache->d_v_steps) return IPTQ_ERR_NULL;
    if (!aligned(cache->d_k_codes, 16) || !aligned(cache->d_k_steps, 16) || !aligned(cache->d_v_codes, 16) || !aligned(cache->d_v_steps, 16))
        return IPTQ_ERR_ALIGN;
    out->k_codes = cache->d_k_codes; out->k_steps = cache->d_k_steps;
    out->v_codes = cache->d_v_codes; out->v_steps = cache->d_v_steps;
    out->n_pages = cache->n_pages; out->page_tokens = t; out->kv_heads = cache->kv_heads; out->dim = cache->head_dim;
    out->page_log = 0;
    while ((1 << out->page_log) < t) ++out->page_log;
    return IPTQ_OK;
}

// whether [p, p + n) shares a byte with one of the cache's four arrays
static bool overlaps_cache(const void *p, int64_t n, const CacheDev &C)
{
    const int64_t rows = (int64_t)C.n_pages * C.kv_heads * C.page_tokens;
    const int64_t codes = rows * (C.dim / 2), steps = rows * ((C.dim + kGroup - 1) / kGroup);
    return overlap(p, n, C.k_codes, codes) || overlap(p, n, C.v_codes, codes) || overlap(p, n, C.k_steps, steps) ||
           overlap(p, n, C.v_steps, steps);
}

extern "C" int iptq_cache_store_i4(const iptq_cache_i4_t *cache, const int8_t *d_k, int64_t k_stride, const int8_t *d_v,
                                   int64_t v_stride, const int32_t *d_slots, int64_t tokens, void *stream)
{
    CacheStoreCall c;
    int rc = plan_cache(cache, &c.C);
    if (rc != IPTQ_OK) return rc;
    const int64_t kw = (int64_t)c.C.kv_heads * c.C.dim;
    if (tokens < 0 || tokens >= ((int64_t)1 << 31) || k_stride < kw || v_stride < kw || k_stride >= ((int64_t)1 << 31) ||
        v_stride >= ((int64_t)1 << 31) || (tokens + 15) / 16 * c.C.kv_heads >= ((int64_t)1 << 24))
        return IPTQ_ERR_SHAPE;
    if (tokens == 0) return IPTQ_OK;
    if (!d_k || !d_v || !d_slots) return IPTQ_ERR_NULL;
    if (!aligned(d_slots, 4)) return IPTQ_ERR_ALIGN;
    if (overlaps_cache(d_k, extent(tokens, k_stride, kw), c.C) || overlaps_cache(d_v, extent(tokens, v_stride, kw), c.C) ||
        overlaps_cache(d_slots, tokens * 4, c.C))
        return IPTQ_ERR_PARAM;
    c.k = d_k; c.v = d_v; c.k_stride = k_stride; c.v_stride = v_stride; c.slots = d_slots; c.tokens = tokens;
    return hip_rc(cache_store_i4_dispatch(c, static_cast<hipStream_t>(stream)));
}

static int plan_cache_attention(const iptq_cache_i4_t *cache, int32_t n_seq, int32_t q_tokens, int32_t heads, int32_t max_pages,
                                CacheAttentionCall *c)
{
    int rc = plan_cache(cache, &c->C);
    if (rc != IPTQ_OK) return rc;
    rc = check_heads(heads, c->C.kv_heads, c->C.dim);
    if (rc != IPTQ_OK) return rc;
    if (n_seq < 0 || q_tokens < 1 || q_tokens > IPTQ_CACHE_QUERIES_MAX || max_pages < 0 ||
        (int64_t)max_pages * c->C.page_tokens > IPTQ_CACHE_KEYS_MAX)
        return IPTQ_ERR_SHAPE;
    const int64_t rows = (int64_t)n_seq * heads * q_tokens, units = ((int64_t)max_pages * c->C.page_tokens + 1023) / 1024;
    if (rows >= ((int64_t)1 << 24) || rows * units >= ((int64_t)1 << 24)) return IPTQ_ERR_SHAPE;      // (a launch's threads are counted in 32 bits)
    c->n_seq = n_seq; c->q_tokens = q_tokens; c->heads = heads; c->max_pages = max_pages;
    return IPTQ_OK;
}

extern "C" int iptq_attention_cache_i4_workspace(const iptq_cache_i4_t *cache, int32_t n_seq, int32_t q_tokens, int32_t heads,
                                                 int32_t max_pages, int64_t *bytes)
{
    if (!bytes) return IPTQ_ERR_NULL;
    CacheAttentionCall c;
    int rc = plan_cache_attention(cache, n_seq, q_tokens, heads, max_pages, &c);
    if (rc != IPTQ_OK) return rc;
    *bytes = attention_cache_i4_workspace_bytes(c);
    return IPTQ_OK;
}

extern "C" int iptq_attention_cache_i4(const int8_t *d_q, int64_t q_stride, const iptq_cache_i4_t *cache, const int32_t *d_pages,
                                       int32_t max_pages, const int32_t *d_lengths, int32_t n_seq, int32_t q_tokens, int32_t heads,
                                       int8_t *d_out, int64_t out_stride, void *d_work, int64_t work_bytes,
                                       const iptq_attention_params_t *p, void *stream)
{
    CacheAttentionCall c;
    int rc = plan_attention(p, IPTQ_CACHE_SCORE_SHIFT_MAX, &c.P);
    if (rc != IPTQ_OK) return rc;
    rc = plan_cache_attention(cache, n_seq, q_tokens, heads, max_pages, &c);
    if (rc != IPTQ_OK) return rc;
    const int64_t qw = (int64_t)heads * c.C.dim, rows = (int64_t)n_seq * q_tokens;
    if (q_stride < qw || out_stride < qw || q_stride >= ((int64_t)1 << 31) || out_stride >= ((int64_t)1 << 31) || work_bytes < 0)
        return IPTQ_ERR_SHAPE;
    if (n_seq == 0) return IPTQ_OK;
    const int64_t need = attention_cache_i4_workspace_bytes(c);
    if (!d_q || !d_out || !d_lengths || (max_pages > 0 && !d_pages) || (need > 0 && !d_work)) return IPTQ_ERR_NULL;
    if (work_bytes < need) return IPTQ_ERR_WORKSPACE;
    if (!aligned(d_pages, 4) || !aligned(d_lengths, 4) || (need > 0 && !aligned(d_work, 16))) return IPTQ_ERR_ALIGN;
    const int64_t out_bytes = extent(rows, out_stride, qw), q_bytes = extent(rows, q_stride, qw);
    const int64_t table = (int64_t)n_seq * max_pages * 4, lens = (int64_t)n_seq * 4;
    if (overlap(d_out, out_bytes, d_q, q_bytes) || overlap(d_out, out_bytes, d_pages, table) || overlap(d_out, out_bytes, d_lengths, lens) ||
        overlaps_cache(d_out, out_bytes, c.C))
        return IPTQ_ERR_PARAM;
    if (need > 0 && (overlap(d_work, need, d_q, q_bytes) || overlap(d_work, need, d_out, out_bytes) || overlap(d_work, need, d_pages, table) ||
                     overlap(d_work, need, d_lengths, lens) || overlaps_cache(d_work, need, c.C)))
        return IPTQ_ERR_PARAM;
    c.q = d_q; c.out = d_out; c.q_stride = q_stride; c.out_stride = out_stride;
    c.pages = d_pages; c.lengths = d_lengths; c.work = d_work;
    return hip_rc(attention_cache_i4_dispatch(c, static_cast<hipStream_t>(stream)));
}

extern "C" int iptq_rmsnorm_i32(const int32_t *d_x, const int32_t *d_residual, const int16_t *d_gain, int32_t *d_residual_out,
                                int8_t *d_out, int32_t *d_row_scales, int64_t rows, int32_t cols, const iptq_rmsnorm_params_t *p,
                                void *stream)
{
    if (!p) return IPTQ_ERR_NULL;
    if (rows < 0 || rows >= ((int64_t)1 << 31) || cols < 1 || cols > IPTQ_NORM_COLS_MAX) return IPTQ_ERR_SHAPE;
    if (p->in_m <= -32768 || p->in_m >= 32768 || p->in_s < 0 || p->in_s > 62) return IPTQ_ERR_PARAM;
    if (p->eps < 0 || p->eps > ((int64_t)1 << 46)) return IPTQ_ERR_PARAM;
    RmsnormCall c;
    int rc = plan_requant(&p->post, 1, &c.post);
    if (rc != IPTQ_OK) return rc;
    if (rows == 0) return IPTQ_OK;
    if ((!d_x && !d_residual) || !d_gain || !d_out) return IPTQ_ERR_NULL;
    if (!aligned(d_x, 4) || !aligned(d_residual, 4) || !aligned(d_residual_out, 4) || !aligned(d_row_scales, 4) || !aligned(d_gain, 2))
        return IPTQ_ERR_ALIGN;
    const int64_t n = rows * cols;
    // a residual is updated in place or not at all; everything else lies apart
    if (d_residual_out != d_residual && overlap(d_residual_out, n * 4, d_residual, n * 4)) return IPTQ_ERR_PARAM;
    const struct { const void *p; int64_t n; } in[] = {{d_x, n * 4}, {d_residual, n * 4}, {d_gain, (int64_t)cols * 2}},
                                               outs[] = {{d_out, n}, {d_row_scales, rows * 4}, {d_residual_out, n * 4}};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 3; ++i)
            if (!(o == 2 && i == 1) && overlap(outs[o].p, outs[o].n, in[i].p, in[i].n)) return IPTQ_ERR_PARAM;
        for (int i = 0; i < o; ++i)
            if (overlap(outs[o].p, outs[o].n, outs[i].p, outs[i].n)) return IPTQ_ERR_PARAM;
    }
    c.x = d_x; c.residual = d_residual; c.residual_out = d_residual_out; c.gain = d_gain; c.out = d_out; c.row_scales = d_row_scales;
    c.rows = rows; c.cols = cols; c.in_m = p->in_m; c.in_s = p->in_s;
    c.eps_sum = p->eps * (int64_t)cols;                   // at most 2^61
    uint64_t root = 0;
    for (uint64_t bit = (uint64_t)1 << 24; bit != 0; bit >>= 1)
        if ((root + bit) * (root + bit) <= ((uint64_t)cols << 32)) root += bit;
    c.root_cols = (uint32_t)root;
    return hip_rc(rmsnorm_i32_dispatch(c, static_cast<hipStream_t>(stream)));
}

extern "C" int iptq_requant_rows(const int32_t *d_in, const int32_t *d_row_scales, int32_t row_shift, void *d_out, int64_t rows,
                                 int32_t cols, int32_t out_is_signed, const iptq_dyadic_t *p, void *stream)
{
    if (!p) return IPTQ_ERR_NULL;
    if (rows < 0 || rows >= ((int64_t)1 << 31) || cols < 1 || cols > IPTQ_ROW_COLS_MAX) return IPTQ_ERR_SHAPE;
    if (row_shift < 0 || row_shift > 62) return IPTQ_ERR_PARAM;
    DyadicDev dev;
    int rc = plan_requant(p, out_is_signed, &dev);
    if (rc != IPTQ_OK) return rc;
    if (rows == 0) return IPTQ_OK;
    if (!d_in || !d_row_scales || !d_out) return IPTQ_ERR_NULL;
    if (!aligned(d_in, 4) || !aligned(d_row_scales, 4)) return IPTQ_ERR_ALIGN;
    const int64_t n = rows * cols;
    if (overlap(d_in, n * 4, d_out, n) || overlap(d_row_scales, rows * 4, d_out, n)) return IPTQ_ERR_PARAM;
    return hip_rc(requant_rows_dispatch(d_in, d_row_scales, row_shift, d_out, rows, cols, dev, static_cast<hipStream_t>(stream)));
}

extern "C" int iptq_attention_prepare(double s_score, double s_v, double s_out, int32_t zp_out, int32_t variant, int32_t causal,
                                      int32_t of_cache, iptq_attention_params_t *out)
{
    if (!out) return IPTQ_ERR_NULL;
    if (!(s_score > 0.0) || !(s_v > 0.0) || !(s_out > 0.0) || isinf(s_score) || isinf(s_v) || isinf(s_out)) return IPTQ_ERR_PARAM;
    if (variant < 0 || variant > 2 || (causal != 0 && causal != 1) || (of_cache != 0 && of_cache != 1)) return IPTQ_ERR_PARAM;
    // a code of the cache stands for a seventh of its step
    const double s = of_cache ? s_score / 7.0 : s_score;
    const int most = of_cache ? IPTQ_CACHE_SCORE_SHIFT_MAX : IPTQ_SCORE_SHIFT_MAX;
    int shift = 0;
    while (shift < most && 1.0 / (s * ldexp(1.0, shift)) >= 1025.0) ++shift;
    const double inv = floor(1.0 / (s * ldexp(1.0, shift)));
    if (!(inv >= 16.0) || inv > 1024.0) return IPTQ_ERR_RANGE;
    memset(out, 0, sizeof(*out));
    out->variant = variant; out->i0 = (int32_t)inv; out->score_shift = shift; out->causal = causal;
    while (((int64_t)out->i0 << (out->n_shift + 1)) <= IPTQ_WEIGHT_MAX) ++out->n_shift;
    int rc = iptq_make_dyadic(s_v / ((of_cache ? 7.0 : 1.0) * 256.0 * s_out), &out->post.m, &out->post.s);
    if (rc != IPTQ_OK) return rc;
    out->post.zp = zp_out; out->post.qmin = -128; out->post.qmax = 127;
    return check_dyadic(&out->post, 1);
}
