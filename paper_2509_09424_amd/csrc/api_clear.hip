// C ABI of the decoder layer on clear activations: argument checks, handles; the kernels are in clear_*.hip.
#include <math.h>

#include <algorithm>
#include <new>

#include "api_util.h"
#include "clear.h"

#define CLEAR_MAX_HEADS 4096
#define CLEAR_MAX_NORM_ROWS (1 << 21)  // a grid has fewer than 2^32 threads, a row up to 1024 of them
#define CLEAR_MAX_SEQS 65535      // a grid's third dimension
#define CLEAR_MAX_NEW (1 << 20)   // its second one, in blocks of 16 tokens
#define CLEAR_MAX_CACHES 1024     // layers of one call

static int current_device(ensi_ctx *ctx) {
    int cur = -1;
    if (hipGetDevice(&cur) != hipSuccess || cur != ctx->device) ENSI_FAIL(ctx, ENSI_E_HIP, "the context's device is not current");
    return ENSI_OK;
}
// The workspace of the clear calls, made with the first cache, weights or sampling call of a context.
static int clear_workspace(ensi_ctx *ctx) {
    if (ctx->ws_clear) return ENSI_OK;
    hipError_t e = ctx->pool->alloc((void **)&ctx->ws_clear, CLEAR_WS_FLOATS * sizeof(float));
    if (e != hipSuccess) ENSI_FAIL(ctx, ENSI_E_NOMEM, "clear workspace: device allocation failed: %s", hipGetErrorString(e));
    return ENSI_OK;
}
static int type_size(int type) { return type == ENSI_T_F32 ? 4 : type == ENSI_T_BF16 || type == ENSI_T_F16 ? 2 : 0; }

// Rows of `width` elements, `stride` apart, as addresses.  Two arrays of one stride, slices of a wider one, meet where their columns do; of two strides where the ranges do.
struct Span {
    uintptr_t from, to;
    size_t step, row;  // in bytes; step 0: one row
    Span(const void *p, int64_t rows, int64_t stride, int64_t width, int size)
        : from((uintptr_t)p), to(p && rows > 0 ? from + (size_t)(((rows - 1) * stride + width) * size) : from), step(rows > 1 ? (size_t)stride * size : 0), row((size_t)width * size) {}
    bool meets(const Span &o) const {
        if (from >= o.to || o.from >= to) return false;
        if (step && o.step && step != o.step) return true;
        const size_t both = step ? step : o.step;
        if (!both) return true;
        const size_t apart = o.from >= from ? (o.from - from) % both : (both - (from - o.from) % both) % both;  // of o's columns behind this one's
        return apart < row || both - apart < o.row;
    }
};

// The arrays of a cache
struct CacheSpans {
    Span part[4];
    static int64_t blocks(const KvView &c) { return (int64_t)c.pages * c.heads * (c.page / KV_BLOCK); }
    explicit CacheSpans(const KvView &c)
        : part{Span(c.k, 1, 0, blocks(c) * KV_BLOCK * c.dim, 1), Span(c.v, 1, 0, blocks(c) * KV_BLOCK * c.dim, 1), Span(c.ks, 1, 0, blocks(c), 4), Span(c.vs, 1, 0, blocks(c), 4)} {}
    bool meets(const Span &o) const { return part[0].meets(o) || part[1].meets(o) || part[2].meets(o) || part[3].meets(o); }
};

extern "C" int ensi_clear_norm(ensi_ctx *ctx, const ensi_clear_norm_args *a, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!a) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear norm: no arguments");
    const int size = type_size(a->type);
    if (!size) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear norm: unknown type %d", a->type);
    if (a->d < 1 || a->d > 32768 || a->rows < 0 || a->rows > CLEAR_MAX_NORM_ROWS)
        ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear norm: %lld rows (up to %d) of %d elements (1 to 32768)", (long long)a->rows, CLEAR_MAX_NORM_ROWS, a->d);
    if (!(a->eps >= 0) || isinf(a->eps)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear norm: eps must not be negative or infinite");
    if (a->rows == 0) return ENSI_OK;
    if (!a->x || !a->gain) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear norm: x and gain are needed");
    if (!a->out && !a->codes) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear norm: neither codes nor out are wanted");
    if (!a->codes != !a->scales) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear norm: codes and scales go together");
    if (a->sum_out && !a->residual) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear norm: a sum needs a residual");
    if (a->rows > 1 && (a->x_stride < a->d || (a->residual && a->residual_stride < a->d) || (a->sum_out && a->sum_stride < a->d) || (a->out && a->out_stride < a->d)))
        ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear norm: rows overlap (a stride is below %d)", a->d);
    const Span x(a->x, a->rows, a->x_stride, a->d, size), r(a->residual, a->rows, a->residual_stride, a->d, size), s(a->sum_out, a->rows, a->sum_stride, a->d, size),
        o(a->out, a->rows, a->out_stride, a->d, size), c(a->codes, a->rows, a->d, a->d, 1), w(a->scales, a->rows, 1, 1, 4), g(a->gain, 1, a->d, a->d, size);
    const auto same = [&](const void *p, int64_t p_stride, const void *q, int64_t q_stride) { return p == q && (a->rows == 1 || p_stride == q_stride); };
    if ((s.meets(x) && !same(a->sum_out, a->sum_stride, a->x, a->x_stride)) || (s.meets(r) && !same(a->sum_out, a->sum_stride, a->residual, a->residual_stride)) ||
        (o.meets(x) && !same(a->out, a->out_stride, a->x, a->x_stride)) || o.meets(r) || o.meets(s) || c.meets(x) || c.meets(r) || c.meets(s) || c.meets(o) || c.meets(g) ||
        w.meets(x) || w.meets(r) || w.meets(s) || w.meets(o) || w.meets(c) || w.meets(g) || g.meets(s) || g.meets(o))
        ENSI_FAIL(ctx, ENSI_E_BADARG, "clear norm: an output overlaps another array (sum may be x or the residual, out may be x)");
    if (int rc = current_device(ctx)) return rc;
    launch_clear_norm(ctx, *a, (hipStream_t)stream);
    ENSI_HIP(ctx, hipGetLastError());
    return ENSI_OK;
}

extern "C" int ensi_clear_weights_prepare(ensi_ctx *ctx, const int8_t *W, const float *w_scales, int32_t d, int32_t m, int32_t group, ensi_cw **out) {
    if (!ctx) return ENSI_E_BADARG;
    if (!W || !w_scales || !out) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear weights: a null argument");
    *out = nullptr;
    if (d < 1 || d > 131072 || m < 1 || m > (1 << 24)) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear weights: %d x %d (up to 131072 x 2^24)", d, m);
    if (group < 0 || group % 64) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear weights: groups of %d rows (a multiple of 64, or 0)", group);
    if (int rc = current_device(ctx)) return rc;
    if (int rc = clear_workspace(ctx)) return rc;
    const int groups = group ? (int)(((int64_t)d + group - 1) / group) : 1;
    ensi_cw *cw = new (std::nothrow) ensi_cw();
    if (!cw) ENSI_FAIL(ctx, ENSI_E_NOMEM, "no host memory");
    cw->ctx = ctx;
    cw->d = d;
    cw->m = m;
    cw->group = group;
    cw->units = (d + 127) / 128;
    cw->m_pad = (m + 127) & ~127;  // whole workgroups of either kernel's tiles
    cw->m_tiles = cw->m_pad / 16;
    // on the default stream, which the copies and the wait below order
    DevBuf raw;
    int wrong = 0;
    hipError_t e = raw.alloc(ctx, (size_t)d * m + 8 + sizeof(int));
    int *bad = (int *)((char *)raw.p + (((size_t)d * m + 7) & ~(size_t)7));
    if (e == hipSuccess) e = ctx->pool->alloc((void **)&cw->w, (size_t)cw->m_tiles * cw->units * 512);
    if (e == hipSuccess) e = ctx->pool->alloc((void **)&cw->scales, (size_t)groups * cw->m_pad * sizeof(float));
    if (e != hipSuccess) {
        ensi_clear_weights_free(cw);
        ENSI_FAIL(ctx, ENSI_E_NOMEM, "clear weights: device allocation failed: %s", hipGetErrorString(e));
    }
    e = hipMemcpy(raw.p, W, (size_t)d * m, hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipMemcpy(bad, &wrong, sizeof wrong, hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipMemset(cw->scales, 0, (size_t)groups * cw->m_pad * sizeof(float));
    if (e == hipSuccess) e = hipMemcpy2D(cw->scales, (size_t)cw->m_pad * 4, w_scales, (size_t)m * 4, (size_t)m * 4, groups, hipMemcpyHostToDevice);
    if (e == hipSuccess) {
        launch_clear_pack((const int8_t *)raw.p, d, m, cw->units, cw->m_tiles, cw->w, bad, nullptr);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipMemcpy(&wrong, bad, sizeof wrong, hipMemcpyDeviceToHost);
    if (e != hipSuccess || wrong) {
        ensi_clear_weights_free(cw);
        if (e != hipSuccess) ENSI_FAIL(ctx, ENSI_E_HIP, "clear weights: %s", hipGetErrorString(e));
        ENSI_FAIL(ctx, ENSI_E_BADARG, "weights must be -1, 0 or 1");
    }
    *out = cw;
    return ENSI_OK;
}

extern "C" void ensi_clear_weights_free(ensi_cw *cw) {
    if (!cw) return;
    if (cw->w) (void)hipFree(cw->w);  // waits for the device
    if (cw->scales) (void)hipFree(cw->scales);
    delete cw;
}

extern "C" int ensi_clear_matmul(ensi_ctx *ctx, const ensi_cw *cw, const int8_t *codes, int64_t codes_stride, const float *scales, void *out, int64_t out_stride, int64_t rows, int32_t type,
                                 void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!cw || cw->ctx != ctx) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear matmul: no weights, or those of another context");
    const int size = type_size(type);
    if (!size) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear matmul: unknown type %d", type);
    if (rows < 0 || rows > (1 << 20)) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear matmul: %lld rows (up to 2^20)", (long long)rows);
    if (rows == 0) return ENSI_OK;
    if (!codes || !scales || !out) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear matmul: a null array");
    if (rows > 1 && (codes_stride < cw->d || out_stride < cw->m)) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear matmul: rows overlap");
    const Span c(codes, rows, codes_stride, cw->d, 1), s(scales, rows, 1, 1, 4), o(out, rows, out_stride, cw->m, size);
    if (o.meets(c) || o.meets(s)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear matmul: out overlaps an input");
    if (int rc = current_device(ctx)) return rc;
    launch_clear_matmul(ctx, cw, codes, codes_stride, scales, out, out_stride, rows, type, (hipStream_t)stream);
    ENSI_HIP(ctx, hipGetLastError());
    return ENSI_OK;
}

extern "C" int ensi_clear_cache_wrap(ensi_ctx *ctx, void *k, void *v, float *k_scale, float *v_scale, int32_t pages, int32_t heads, int32_t page, int32_t dim, ensi_kv **out) {
    if (!ctx) return ENSI_E_BADARG;
    if (!k || !v || !k_scale || !v_scale || !out) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear cache: a null argument");
    *out = nullptr;
    if (dim != 64 && dim != 96 && dim != 128 && dim != 192 && dim != 256) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear cache: heads of %d (64, 96, 128, 192 or 256)", dim);
    if (pages < 1 || heads < 1 || heads > CLEAR_MAX_HEADS || page < KV_BLOCK || page % KV_BLOCK || (int64_t)heads * page > INT32_MAX ||
        (int64_t)pages * ((int64_t)heads * page / KV_BLOCK) > INT32_MAX)
        ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear cache: %d pages of %d heads and %d tokens (pages of whole blocks of 16, fewer than 2^31 of these)", pages, heads, page);
    if (((uintptr_t)k | (uintptr_t)v) & 15 || ((uintptr_t)k_scale | (uintptr_t)v_scale) & 3) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear cache: arrays are not aligned");
    const KvView view = {(unsigned char *)k, (unsigned char *)v, k_scale, v_scale, pages, heads, page, dim, nullptr};
    const CacheSpans a(view);
    for (int i = 0; i < 4; i++)
        for (int j = 0; j < i; j++)
            if (a.part[i].meets(a.part[j])) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear cache: its arrays overlap");
    if (int rc = current_device(ctx)) return rc;
    if (int rc = clear_workspace(ctx)) return rc;
    ensi_kv *kv = new (std::nothrow) ensi_kv();
    if (!kv) ENSI_FAIL(ctx, ENSI_E_NOMEM, "no host memory");
    kv->ctx = ctx;
    kv->view = view;
    const int zero = 0;
    hipError_t e = ctx->pool->alloc((void **)&kv->view.status, sizeof(int));
    if (e == hipSuccess) e = hipMemcpy(kv->view.status, &zero, sizeof zero, hipMemcpyHostToDevice);
    if (e != hipSuccess) {
        ensi_clear_cache_free(kv);
        ENSI_FAIL(ctx, ENSI_E_NOMEM, "clear cache: device allocation failed: %s", hipGetErrorString(e));
    }
    *out = kv;
    return ENSI_OK;
}

extern "C" void ensi_clear_cache_free(ensi_kv *kv) {
    if (!kv) return;
    if (kv->view.status) (void)hipFree(kv->view.status);  // waits for the device
    delete kv;
}

extern "C" int ensi_clear_cache_status(ensi_ctx *ctx, ensi_kv *kv, int32_t *bits, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!kv || !bits || kv->ctx != ctx) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear cache: no cache, or that of another context");
    if (int rc = current_device(ctx)) return rc;
    int found = 0;
    const int zero = 0;
    ENSI_HIP(ctx, hipStreamSynchronize((hipStream_t)stream));
    ENSI_HIP(ctx, hipMemcpy(&found, kv->view.status, sizeof found, hipMemcpyDeviceToHost));
    if (found) ENSI_HIP(ctx, hipMemcpy(kv->view.status, &zero, sizeof zero, hipMemcpyHostToDevice));
    *bits = found;
    return ENSI_OK;
}

static int check_seqs(ensi_ctx *ctx, const char *who, const ensi_clear_seqs &s) {
    if (s.seqs < 0 || s.seqs > CLEAR_MAX_SEQS || s.tokens < 0 || s.tokens > INT32_MAX || s.max_new < 0 || s.max_new > CLEAR_MAX_NEW || s.table_width < 0)
        ENSI_FAIL(ctx, ENSI_E_SHAPE, "%s: %d sequences (up to %d) with %lld new tokens, at most %d each (up to %d), tables of %d pages", who, s.seqs, CLEAR_MAX_SEQS, (long long)s.tokens, s.max_new,
                  CLEAR_MAX_NEW, s.table_width);
    if (s.seqs && s.tokens && s.max_new && (!s.begin || !s.lengths || !s.table || s.table_width < 1 || (s.seqs > 1 && s.table_stride < s.table_width)))
        ENSI_FAIL(ctx, ENSI_E_BADARG, "%s: begin, lengths and a table are needed, its rows apart", who);
    return ENSI_OK;
}

// A tree's parents, where a call takes one
static int check_tree(ensi_ctx *ctx, const char *who, const ensi_clear_seqs &s) {
    if (s.max_new > TREE_MAX) ENSI_FAIL(ctx, ENSI_E_SHAPE, "%s: trees of up to %d tokens, not %d", who, TREE_MAX, s.max_new);
    return ENSI_OK;
}

static int append(ensi_ctx *ctx, ensi_kv *kv, const ensi_clear_append_args *a, const int32_t *parents, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!kv || !a || kv->ctx != ctx) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear append: no cache, or that of another context, or no arguments");
    const KvView &c = kv->view;
    const int size = type_size(a->type);
    if (!size) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear append: unknown type %d", a->type);
    if (a->pairs != ENSI_ROT_HALF && a->pairs != ENSI_ROT_NEIGHBOURS) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear append: unknown layout of pairs %d", a->pairs);
    if (a->rot < 0 || a->rot > c.dim || a->rot % 16) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear append: %d rotated elements (a multiple of 16, up to %d)", a->rot, c.dim);
    if (a->positions < 0 || !a->q != !a->q_out || (a->q && (a->q_heads < 1 || a->q_heads > CLEAR_MAX_HEADS)))
        ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear append: %d positions, %d query heads (up to %d), queries with q_out", a->positions, a->q_heads, CLEAR_MAX_HEADS);
    if (int rc = check_seqs(ctx, "clear append", a->s)) return rc;
    if (parents)
        if (int rc = check_tree(ctx, "clear append", a->s)) return rc;
    if (!a->s.seqs || !a->s.tokens || !a->s.max_new) return ENSI_OK;
    if (!a->k || !a->v || (a->rot && (!a->cos || !a->sin))) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear append: a null array");
    const int64_t kw = (int64_t)c.heads * c.dim, qw = (int64_t)a->q_heads * c.dim, t = a->s.tokens;
    if (t > 1 && (a->k_stride < kw || a->v_stride < kw || (a->q && (a->q_stride < qw || a->q_out_stride < qw)))) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear append: tokens overlap");
    const Span q(a->q, t, a->q_stride, qw, size), o(a->q_out, t, a->q_out_stride, qw, size), k(a->k, t, a->k_stride, kw, size), v(a->v, t, a->v_stride, kw, size);
    const bool same = a->q == a->q_out && (t == 1 || a->q_stride == a->q_out_stride);
    if ((o.meets(q) && !same)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear append: q_out overlaps q without being it");
    // (slices of one array with gaps between the rows of each: their ranges meet, their rows do not)
    if (o.meets(k) || o.meets(v)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear append: q_out overlaps k or v");
    const CacheSpans cache(c);
    if (cache.meets(q) || cache.meets(o) || cache.meets(k) || cache.meets(v)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear append: q, k, v or q_out overlaps the cache");
    const Span p(parents, 1, 0, t, 4);
    if (o.meets(p) || cache.meets(p)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear append: parents overlaps q_out or the cache");
    if (int rc = current_device(ctx)) return rc;
    launch_clear_append(ctx, c, *a, parents, (hipStream_t)stream);
    ENSI_HIP(ctx, hipGetLastError());
    return ENSI_OK;
}
extern "C" int ensi_clear_append(ensi_ctx *ctx, ensi_kv *kv, const ensi_clear_append_args *a, void *stream) { return append(ctx, kv, a, nullptr, stream); }
extern "C" int ensi_clear_append_tree(ensi_ctx *ctx, ensi_kv *kv, const ensi_clear_append_args *a, const int32_t *parents, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!parents) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear append: a tree needs parents");
    return append(ctx, kv, a, parents, stream);
}

static int attention(ensi_ctx *ctx, ensi_kv *kv, const ensi_clear_attention_args *a, const int32_t *parents, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!kv || !a || kv->ctx != ctx) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: no cache, or that of another context, or no arguments");
    const KvView &c = kv->view;
    if (a->type != ENSI_T_BF16 && a->type != ENSI_T_F16) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: type %d (bf16 or f16)", a->type);
    if (a->score != ENSI_SCORE_SOFTMAX && a->score != ENSI_SCORE_SIGMOID) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: unknown score %d", a->score);
    if (a->q_heads < 1 || a->q_heads > CLEAR_MAX_HEADS || a->q_heads % c.heads) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear attention: %d query heads over %d key heads", a->q_heads, c.heads);
    if (a->window < 0 || a->max_length < 0 || a->max_length > (1 << 30) || !(a->cap >= 0) || isinf(a->cap) || !isfinite(a->bias))
        ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: window %d, cap %g, bias %g, max_length %d", a->window, a->cap, a->bias, a->max_length);
    if (int rc = check_seqs(ctx, "clear attention", a->s)) return rc;
    if (parents)
        if (int rc = check_tree(ctx, "clear attention", a->s)) return rc;
    if (!a->s.seqs || !a->s.tokens || !a->s.max_new) return ENSI_OK;
    if (!a->q || !a->out) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: a null array");
    const int64_t w = (int64_t)a->q_heads * c.dim, t = a->s.tokens;
    if (t > 1 && (a->q_stride < w || a->out_stride < w)) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear attention: tokens overlap");
    const Span q(a->q, t, a->q_stride, w, 2), o(a->out, t, a->out_stride, w, 2);
    if (q.meets(o)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: out overlaps q");
    if (Span(parents, 1, 0, t, 4).meets(o)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: out overlaps parents");
    if (CacheSpans(c).meets(o)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: out overlaps the cache");
    if ((int64_t)a->s.max_new * a->q_heads > INT32_MAX / 16) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear attention: %d new tokens of %d heads are too many", a->s.max_new, a->q_heads);
    if (int rc = current_device(ctx)) return rc;
    if (parents) launch_clear_attention_tree(ctx, c, *a, parents, (hipStream_t)stream);
    else launch_clear_attention(ctx, c, *a, (hipStream_t)stream);
    ENSI_HIP(ctx, hipGetLastError());
    return ENSI_OK;
}
extern "C" int ensi_clear_attention(ensi_ctx *ctx, ensi_kv *kv, const ensi_clear_attention_args *a, void *stream) { return attention(ctx, kv, a, nullptr, stream); }
extern "C" int ensi_clear_attention_tree(ensi_ctx *ctx, ensi_kv *kv, const ensi_clear_attention_args *a, const int32_t *parents, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!parents) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: a tree needs parents");
    return attention(ctx, kv, a, parents, stream);
}

extern "C" int ensi_clear_sample(ensi_ctx *ctx, const ensi_clear_sample_args *a, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!a) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear sample: no arguments");
    const int size = type_size(a->type);
    if (!size) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear sample: unknown type %d", a->type);
    if (a->rows < 0 || a->rows > (1 << 20) || a->vocab < 1 || a->vocab > (1 << 24))
        ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear sample: %lld rows (up to 2^20) of %d logits (1 to 2^24)", (long long)a->rows, a->vocab);
    if (a->rows == 0) return ENSI_OK;
    if (!a->logits || !a->uniform || !a->out) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear sample: logits, uniform and out are needed");
    if (a->rows > 1 && a->stride < a->vocab) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear sample: rows overlap (their stride is below %d)", a->vocab);
    if ((!a->temperature && !(a->all_temperature >= 0 && isfinite(a->all_temperature))) || (!a->top_p && isnan(a->all_top_p)) || (!a->min_p && isnan(a->all_min_p)))
        ENSI_FAIL(ctx, ENSI_E_BADARG, "clear sample: temperature %g, top_p %g, min_p %g", a->all_temperature, a->all_top_p, a->all_min_p);
    const Span o(a->out, 1, 0, a->rows, 4);
    const auto meets = [&](const void *p) { return Span(p, 1, 0, a->rows, 4).meets(o); };
    if (Span(a->logits, a->rows, a->stride, a->vocab, size).meets(o) || meets(a->uniform) || meets(a->temperature) || meets(a->top_k) || meets(a->top_p) || meets(a->min_p))
        ENSI_FAIL(ctx, ENSI_E_BADARG, "clear sample: out overlaps an input");
    if (int rc = current_device(ctx)) return rc;
    // Rows are split over workgroups where there is a workspace; the first call of a context makes it, unless it is captured or there is no memory: without one
    // the tokens are the same.  It is asked for once: an allocation that fails takes as long as the call, or more (the next cache or weights try again).
    if (!ctx->ws_clear && !ctx->ws_clear_refused) {
        hipStreamCaptureStatus capture = hipStreamCaptureStatusActive;
        if (hipStreamIsCapturing((hipStream_t)stream, &capture) == hipSuccess && capture == hipStreamCaptureStatusNone) ctx->ws_clear_refused = clear_workspace(ctx) != ENSI_OK;
        (void)hipGetLastError();
    }
    launch_clear_sample(ctx, *a, (hipStream_t)stream);
    ENSI_HIP(ctx, hipGetLastError());
    return ENSI_OK;
}

extern "C" int ensi_clear_accept(ensi_ctx *ctx, const ensi_clear_accept_args *a, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!a) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear accept: no arguments");
    if (a->seqs < 0 || a->seqs > CLEAR_MAX_SEQS || a->tokens < 0 || a->tokens > INT32_MAX || a->max_new < 0 || a->max_new > TREE_MAX)
        ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear accept: %d sequences (up to %d) with %lld new tokens, at most %d each (up to %d)", a->seqs, CLEAR_MAX_SEQS, (long long)a->tokens, a->max_new, TREE_MAX);
    if (a->seqs == 0) return ENSI_OK;
    if (!a->begin || !a->count || !a->following || (a->max_new && !a->path) || (a->tokens && (!a->drafted || !a->sampled))) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear accept: a null array");
    if (a->seqs > 1 && a->path_stride < a->max_new) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear accept: paths overlap (their stride is below %d)", a->max_new);
    const Span in[] = {Span(a->begin, 1, 0, (int64_t)a->seqs + 1, 4), Span(a->parents, 1, 0, a->tokens, 4), Span(a->drafted, 1, 0, a->tokens, 4), Span(a->sampled, 1, 0, a->tokens, 4)};
    const Span out[] = {Span(a->path, a->seqs, a->path_stride, a->max_new, 4), Span(a->count, 1, 0, a->seqs, 4), Span(a->following, 1, 0, a->seqs, 4)};
    for (int i = 0; i < 3; i++) {
        for (const Span &s : in)
            if (s.meets(out[i])) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear accept: an output overlaps an input");
        for (int j = 0; j < i; j++)
            if (out[i].meets(out[j])) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear accept: outputs overlap");
    }
    if (int rc = current_device(ctx)) return rc;
    launch_clear_accept(ctx, *a, (hipStream_t)stream);
    ENSI_HIP(ctx, hipGetLastError());
    return ENSI_OK;
}

// The caches of a call: this context's, with pages of one size, no array of one within another's: waves and workgroups of different caches have no order between them.
static int check_caches(ensi_ctx *ctx, const char *who, ensi_kv *const *kv, int caches) {
    if (!kv || caches < 1 || caches > CLEAR_MAX_CACHES) ENSI_FAIL(ctx, kv ? ENSI_E_SHAPE : ENSI_E_BADARG, "%s: %d caches (1 to %d)", who, caches, CLEAR_MAX_CACHES);
    struct Range {
        uintptr_t from, to;
    } ranges[4 * CLEAR_MAX_CACHES];
    for (int i = 0; i < caches; i++) {
        if (!kv[i] || kv[i]->ctx != ctx) ENSI_FAIL(ctx, ENSI_E_BADARG, "%s: no cache, or that of another context", who);
        if (kv[i]->view.page != kv[0]->view.page) ENSI_FAIL(ctx, ENSI_E_SHAPE, "%s: caches with pages of %d and of %d tokens", who, kv[0]->view.page, kv[i]->view.page);
        const CacheSpans spans(kv[i]->view);
        for (int j = 0; j < 4; j++) ranges[4 * i + j] = {spans.part[j].from, spans.part[j].to};
    }
    if (caches == 1) return ENSI_OK;  // (one cache's arrays are apart: it was wrapped so)
    std::sort(ranges, ranges + 4 * caches, [](const Range &a, const Range &b) { return a.from < b.from; });
    for (int i = 1; i < 4 * caches; i++)
        if (ranges[i].from < ranges[i - 1].to) ENSI_FAIL(ctx, ENSI_E_BADARG, "%s: a cache is there twice, or arrays of two caches overlap", who);
    return ENSI_OK;
}

extern "C" int ensi_clear_keep(ensi_ctx *ctx, ensi_kv *const *kv, int32_t caches, const ensi_clear_keep_args *a, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!a) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear keep: no arguments");
    if (int rc = check_caches(ctx, "clear keep", kv, caches)) return rc;
    if (int rc = check_seqs(ctx, "clear keep", a->s)) return rc;
    if (int rc = check_tree(ctx, "clear keep", a->s)) return rc;
    if (!a->s.seqs || !a->s.tokens || !a->s.max_new) return ENSI_OK;
    if (!a->path || !a->count) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear keep: path and count are needed");
    if (a->s.seqs > 1 && a->path_stride < a->s.max_new) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear keep: paths overlap (their stride is below %d)", a->s.max_new);
    if (int rc = current_device(ctx)) return rc;
    launch_clear_keep(ctx, kv, caches, *a, (hipStream_t)stream);
    ENSI_HIP(ctx, hipGetLastError());
    return ENSI_OK;
}

extern "C" int ensi_clear_fork(ensi_ctx *ctx, ensi_kv *const *kv, int32_t caches, const ensi_clear_fork_args *a, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!a) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear fork: no arguments");
    if (int rc = check_caches(ctx, "clear fork", kv, caches)) return rc;
    if (a->seqs < 0 || a->seqs > CLEAR_MAX_SEQS || a->rows < 0 || a->rows > CLEAR_MAX_SEQS || a->table_width < 1)
        ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear fork: %d sequences and %d rows (up to %d), tables of %d pages", a->seqs, a->rows, CLEAR_MAX_SEQS, a->table_width);
    if (a->rows == 0) return ENSI_OK;
    if (!a->source || !a->fresh || !a->table_out || !a->lengths_out || (a->seqs && (!a->table || !a->lengths))) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear fork: a null array");
    if ((a->seqs > 1 && a->table_stride < a->table_width) || (a->rows > 1 && a->out_stride < a->table_width)) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear fork: rows of a table overlap");
    const Span table(a->table, a->seqs, a->table_stride, a->table_width, 4), lengths(a->lengths, 1, 0, a->seqs, 4), source(a->source, 1, 0, a->rows, 4), fresh(a->fresh, 1, 0, a->rows, 4);
    const Span table_out(a->table_out, a->rows, a->out_stride, a->table_width, 4), lengths_out(a->lengths_out, 1, 0, a->rows, 4);
    for (const Span *in : {&table, &lengths, &source, &fresh})
        if (in->meets(table_out) || in->meets(lengths_out)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear fork: an output overlaps an input");
    if (table_out.meets(lengths_out)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear fork: outputs overlap");
    for (int i = 0; i < caches; i++)
        if (CacheSpans(kv[i]->view).meets(table_out) || CacheSpans(kv[i]->view).meets(lengths_out)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear fork: an output overlaps a cache");
    if (int rc = current_device(ctx)) return rc;
    launch_clear_fork(ctx, kv, caches, *a, (hipStream_t)stream);
    ENSI_HIP(ctx, hipGetLastError());
    return ENSI_OK;
}
