// C ABI of the decoder layer on clear activations: argument checks, handles; the kernels are in clear_*.hip.
#include <math.h>

#include <new>

#include "api_util.h"
#include "clear.h"

#define CLEAR_MAX_HEADS 4096
#define CLEAR_MAX_NORM_ROWS (1 << 21)  // a grid has fewer than 2^32 threads, a row up to 1024 of them
#define CLEAR_MAX_SEQS 65535      // a grid's third dimension
#define CLEAR_MAX_NEW (1 << 20)   // its second one, in blocks of 16 tokens

static int current_device(ensi_ctx *ctx) {
    int cur = -1;
    if (hipGetDevice(&cur) != hipSuccess || cur != ctx->device) ENSI_FAIL(ctx, ENSI_E_HIP, "the context's device is not current");
    return ENSI_OK;
}
// The workspace of the clear calls, made with the first cache or the first weights of a context.
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

extern "C" int ensi_clear_append(ensi_ctx *ctx, ensi_kv *kv, const ensi_clear_append_args *a, void *stream) {
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
    if (int rc = current_device(ctx)) return rc;
    launch_clear_append(ctx, c, *a, (hipStream_t)stream);
    ENSI_HIP(ctx, hipGetLastError());
    return ENSI_OK;
}

extern "C" int ensi_clear_attention(ensi_ctx *ctx, ensi_kv *kv, const ensi_clear_attention_args *a, void *stream) {
    if (!ctx) return ENSI_E_BADARG;
    if (!kv || !a || kv->ctx != ctx) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: no cache, or that of another context, or no arguments");
    const KvView &c = kv->view;
    if (a->type != ENSI_T_BF16 && a->type != ENSI_T_F16) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: type %d (bf16 or f16)", a->type);
    if (a->score != ENSI_SCORE_SOFTMAX && a->score != ENSI_SCORE_SIGMOID) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: unknown score %d", a->score);
    if (a->q_heads < 1 || a->q_heads > CLEAR_MAX_HEADS || a->q_heads % c.heads) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear attention: %d query heads over %d key heads", a->q_heads, c.heads);
    if (a->window < 0 || a->max_length < 0 || a->max_length > (1 << 30) || !(a->cap >= 0) || isinf(a->cap) || !isfinite(a->bias))
        ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: window %d, cap %g, bias %g, max_length %d", a->window, a->cap, a->bias, a->max_length);
    if (int rc = check_seqs(ctx, "clear attention", a->s)) return rc;
    if (!a->s.seqs || !a->s.tokens || !a->s.max_new) return ENSI_OK;
    if (!a->q || !a->out) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: a null array");
    const int64_t w = (int64_t)a->q_heads * c.dim, t = a->s.tokens;
    if (t > 1 && (a->q_stride < w || a->out_stride < w)) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear attention: tokens overlap");
    const Span q(a->q, t, a->q_stride, w, 2), o(a->out, t, a->out_stride, w, 2);
    if (q.meets(o)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: out overlaps q");
    if (CacheSpans(c).meets(o)) ENSI_FAIL(ctx, ENSI_E_BADARG, "clear attention: out overlaps the cache");
    if ((int64_t)a->s.max_new * a->q_heads > INT32_MAX / 16) ENSI_FAIL(ctx, ENSI_E_SHAPE, "clear attention: %d new tokens of %d heads are too many", a->s.max_new, a->q_heads);
    if (int rc = current_device(ctx)) return rc;
    launch_clear_attention(ctx, c, *a, (hipStream_t)stream);
    ENSI_HIP(ctx, hipGetLastError());
    return ENSI_OK;
}
