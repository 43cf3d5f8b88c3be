// Shared by the kernels of the layer on clear activations: element types, 8 elements at a time, the sequences of a call.
#pragma once
#include "common.h"

template <int TYPE>
struct Elem;
template <>
struct Elem<ENSI_T_F32> {
    typedef float type;
};
template <>
struct Elem<ENSI_T_BF16> {
    typedef __bf16 type;
};
template <>
struct Elem<ENSI_T_F16> {
    typedef _Float16 type;
};

// Eight neighbouring elements in one or two wide accesses.  Rows of any stride are read: global memory takes wide accesses at any address of
// whole elements, so these types claim no more alignment than an element has.
template <int TYPE>
struct Chunk {
    typedef typename Elem<TYPE>::type T;
    typedef T vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    static __device__ __forceinline__ void load(float (&f)[8], const T *p) {
        const vec v = *(const vec *)p;
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = (float)v[i];
    }
    static __device__ __forceinline__ void store(T *p, const float (&f)[8]) {
        vec v;
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = (T)f[i];
        *(vec *)p = v;
    }
};

typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

#define KV_BLOCK 16  // tokens that share a scale

// Four floats of at most 448 to e4m3, nearest, ties to even.
__device__ __forceinline__ u32 to_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (u32)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// A cache as the kernels see it.
struct KvView {
    unsigned char *k, *v;
    float *ks, *vs;
    int pages, heads, page, dim;
    int *status;
};

// A sequence's part of a call, checked: count = 0 where it has nothing to do or does not fit (which the status then says).
struct SeqPart {
    int first, count, ctx;  // first new token, number of them, tokens before them
};
__device__ __forceinline__ SeqPart seq_part(const ensi_clear_seqs &s, int seq, int page, int64_t most, int *status, bool notes) {
    const int64_t b0 = s.begin[seq], b1 = s.begin[seq + 1], ctx = s.lengths[seq], n = b1 - b0;
    const bool ok = b0 >= 0 && n >= 0 && b1 <= s.tokens && n <= s.max_new && ctx >= 0 && ctx + n <= most && ctx + n <= (int64_t)s.table_width * page;
    SeqPart p = {(int)b0, (int)n, (int)ctx};
    if (!ok) {
        if (notes) atomicOr(status, ENSI_KV_BAD_LENGTH);
        p.count = 0;
    }
    return p;
}
__device__ __forceinline__ SeqPart seq_part(const ensi_clear_seqs &s, int seq, int page, int64_t most, int *status) { return seq_part(s, seq, page, most, status, threadIdx.x == 0); }

// A tree of a sequence's new tokens, a wave's width of them at most: each names an earlier one as its parent, or none (-1).  Lane t of a wave gets token t's line, the bits
// of itself and its ancestors, in as many steps as the number of tokens has bits: every step adds the line of the first ancestor that is not in it yet.
#define TREE_MAX 64
struct Tree {
    u64 line;
    int depth;   // ancestors
    bool good;   // of the whole tree: no parent behind its child or below -1 (the status then says so)
};
__device__ __forceinline__ Tree tree_of(const int32_t *parents, const SeqPart &part, int *status) {
    const int lane = threadIdx.x % 64;
    int up = lane < part.count ? parents[part.first + lane] : -1;
    Tree t;
    t.good = !__any(up < -1 || up >= lane);
    if (!t.good) {
        if (lane == 0) atomicOr(status, ENSI_KV_BAD_TREE);
        up = -1;
    }
    u32 lo = lane < 32 ? 1u << lane : 0, hi = lane < 32 ? 0 : 1u << (lane - 32);
    for (int k = 1; k < part.count; k *= 2) {
        const int from = max(up, 0);
        const u32 add_lo = __shfl(lo, from), add_hi = __shfl(hi, from);
        const int next = __shfl(up, from);
        if (up >= 0) {
            lo |= add_lo;
            hi |= add_hi;
            up = next;
        }
    }
    t.line = (u64)hi << 32 | lo;
    t.depth = __popcll(t.line) - 1;
    return t;
}

// ---- handles
// Ternary weights of a clear product on the device.
struct ensi_cw {
    ensi_ctx *ctx;
    int d, m, group;
    int units, m_tiles;     // units of 128 rows, tiles of 16 columns
    u32 *w = nullptr;       // two bits a weight, 512 bytes a tile and unit: k_clear_pack
    float *scales = nullptr;  // [groups][m_pad], m_pad = 16 m_tiles, a multiple of 128
    int m_pad;
};
struct ensi_kv {
    ensi_ctx *ctx;
    KvView view;
};

// ---- launchers
void launch_clear_norm(ensi_ctx *ctx, const ensi_clear_norm_args &a, hipStream_t st);
void launch_clear_matmul(ensi_ctx *ctx, const ensi_cw *cw, const int8_t *codes, int64_t codes_stride, const float *scales, void *out,
                         int64_t out_stride, int64_t rows, int type, hipStream_t st);
void launch_clear_pack(const int8_t *d_W, int d, int m, int units, int m_tiles, u32 *w, int *bad, hipStream_t st);
void launch_clear_append(ensi_ctx *ctx, const KvView &kv, const ensi_clear_append_args &a, const int32_t *parents, hipStream_t st);
void launch_clear_attention(ensi_ctx *ctx, const KvView &kv, const ensi_clear_attention_args &a, hipStream_t st);
void launch_clear_attention_tree(ensi_ctx *ctx, const KvView &kv, const ensi_clear_attention_args &a, const int32_t *parents, hipStream_t st);
void launch_clear_accept(ensi_ctx *ctx, const ensi_clear_accept_args &a, hipStream_t st);
void launch_clear_keep(ensi_ctx *ctx, const ensi_kv *const *kv, int caches, const ensi_clear_keep_args &a, hipStream_t st);
void launch_clear_fork(ensi_ctx *ctx, const ensi_kv *const *kv, int caches, const ensi_clear_fork_args &a, hipStream_t st);
void launch_clear_sample(ensi_ctx *ctx, const ensi_clear_sample_args &a, hipStream_t st);

// Raises a kernel's limit of dynamic LDS, once in a context.
inline void clear_lds(ensi_ctx *ctx, const void *kernel, int bytes) {
    for (int i = 0; i < ctx->clear_lds_n; i++)
        if (ctx->clear_lds[i] == kernel) return;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess && ctx->clear_lds_n < CLEAR_LDS_KERNELS) ctx->clear_lds[ctx->clear_lds_n++] = kernel;
}

// Workspace of the clear calls: partial results of keys split over workgroups (attention), aligned copies of codes (matmul), what the workgroups of a row leave for each other
// (sampling).  One allocation of fixed size, made with the first cache, weights or sampling call of a context and never moved, so that other calls allocate nothing and a captured graph's
// pointers stay good.
#define CLEAR_WS_FLOATS ((size_t)16 << 20)
