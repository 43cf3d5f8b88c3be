// Attention over a paged cache of 8-bit keys and values with one scale for 16 tokens of a head.
//
// Keys are codes c with a power of two s as scale, so q k = s (q c): codes widen to the queries' 16 bits without rounding, the matrix instruction
// forms q c in 32 bits, and the scale enters with the factor that the exponent needs anyway.  Values v = s' c' are folded the other way round: their
// scale multiplies the weight.  With t the score in units of log2 e, the running reference M is the maximum of t + log2 s'; e = 2^(t - M) is what the
// softmax's sum adds up, w = e s' <= 1 the weight of the code c'.  The matrix instruction takes weights as two terms of bf16, the nearest one and the nearest to what
// is left, 16 bits together with the exponents of 32 (f16 would end 2^-40 below the largest weight at best, and where the largest one's values are 0 the small ones
// are the result).  Both are held lifted: scales are 2^-64 to 2^120, so the largest e 2^32 is 2^-88 to 2^96 and sums of 2^30 of them stay in range,
// and w 2^69 leaves 2^-195 of the largest weight and sums of 2^30 products with codes in range.
//   sigmoid scores need no sum; w = sigmoid(t) s' 2^-M with the same reference.
// A tile of scores is held as [key][query]: a lane has one query, so the statistics of a row are per lane, and the weights leave the score's
// registers in the order in which the second product reads them; the order of its keys is that of the registers, for the values too.
//
// Masks are applied to scores; a masked weight is 0, and 0 times a value that is NaN must not count: NaN codes of values are taken as 0, and where a token of the
// sequence has one, the rows that see it get their NaN at the end, from a second look at the tiles that had any.
#pragma once
#include "clear.h"

struct AttentionView {
    KvView kv;
    ensi_clear_seqs s;
    const void *q;
    void *out;
    int64_t q_stride, out_stride;
    int q_heads, group;     // query heads, of them per key head
    int window, max_length;
    float cap, cap_inv, factor;  // t = factor q c s: 1 / sqrt(dim), times log2 e where the softmax needs nothing else
    float bias;
    int row_tiles, splits;
    float *ws;
};

#define LOG2E 1.4426950408889634f

template <int TYPE>
struct Wide;  // codes and queries in 16 bits, and their product
template <>
struct Wide<ENSI_T_BF16> {
    typedef bf16x8 vec;
    static __device__ __forceinline__ vec widen(u32 lo, u32 hi) {
        union {
            bf16x2 p[4];
            vec v;
        } u;
        u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
        u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
        u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
        u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
        return u.v;
    }
    static __device__ __forceinline__ f32x4 mfma16(vec a, vec b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16 mfma32(vec a, vec b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Wide<ENSI_T_F16> {
    typedef f16x8 vec;
    static __device__ __forceinline__ vec widen(u32 lo, u32 hi) {
        union {
            f16x2 p[4];
            vec v;
        } u;
        u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
        u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
        u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
        u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
        return u.v;
    }
    static __device__ __forceinline__ f32x4 mfma16(vec a, vec b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16 mfma32(vec a, vec b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// Bytes (k, j) of four words of keys to words of places: e[j] holds byte j of d[0..3]
__device__ __forceinline__ void transpose4(u32 (&d)[4]) {
    const u32 t0 = __builtin_amdgcn_perm(d[1], d[0], 0x05010400), t1 = __builtin_amdgcn_perm(d[1], d[0], 0x07030602);
    const u32 t2 = __builtin_amdgcn_perm(d[3], d[2], 0x05010400), t3 = __builtin_amdgcn_perm(d[3], d[2], 0x07030602);
    d[0] = __builtin_amdgcn_perm(t2, t0, 0x05040100);
    d[1] = __builtin_amdgcn_perm(t2, t0, 0x07060302);
    d[2] = __builtin_amdgcn_perm(t3, t1, 0x05040100);
    d[3] = __builtin_amdgcn_perm(t3, t1, 0x07060302);
}
// The larger one, NaN if either is: a row that sees NaN is NaN whatever its other scores are.  (The maximum that passes over NaN costs one more
// instruction for every operand.)
__device__ __forceinline__ float most_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float most_of(float a, float b, float c) { return most_of(most_of(a, b), c); }

// Bit 7 of every byte whose code is NaN
__device__ __forceinline__ u32 nan_bytes(u32 w) { return (w & 0x7f7f7f7f) + 0x01010101; }

// cap tanh(t / cap) of all of a lane's scores.  Below half a cap t (1 + P((t / cap)^2)), the first seven terms of the series (2^-23 of it are left out at one half), beyond
// cap (1 - 2 / (1 + exp(2 |t| / cap))): that difference would cancel for small scores, by 2^-23 of the cap.  A wave without a score beyond takes the series alone.
template <int B, int E>
__device__ __forceinline__ void cap_scores(float (&t)[B][E], float cap, float cap_inv) {
    float most = 0;
#pragma unroll
    for (int b = 0; b < B; b++)
#pragma unroll
        for (int e = 0; e < E; e++) most = fmaxf(most, fabsf(t[b][e]));
    const bool beyond = __any(most * cap_inv >= 0.5f);
#pragma unroll
    for (int b = 0; b < B; b++)
#pragma unroll
        for (int e = 0; e < E; e++) {
            const float x = t[b][e] * cap_inv, y = x * x;
            float p = __builtin_fmaf(y, 21844.0f / 6081075, -1382.0f / 155925);
            p = __builtin_fmaf(y, p, 62.0f / 2835);
            p = __builtin_fmaf(y, p, -17.0f / 315);
            p = __builtin_fmaf(y, p, 2.0f / 15);
            p = __builtin_fmaf(y, p, -1.0f / 3);
            float capped = __builtin_fmaf(t[b][e] * y, p, t[b][e]);
            if (beyond) {
                const float far = cap * __builtin_fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(fabsf(x) * (2 * LOG2E))), 1.0f);
                if (fabsf(x) >= 0.5f) capped = __builtin_copysignf(far, x);
            }
            t[b][e] = capped;
        }
}

// Products q c to scores t in units of the exponent: softmax log2 e t, sigmoid t log2 e + bias log2 e
template <int SCORE, bool CAP, int B, int E>
__device__ __forceinline__ void scores_of(float (&u)[B][E], const float (&scale)[B], const AttentionView &a) {
#pragma unroll
    for (int b = 0; b < B; b++)
#pragma unroll
        for (int e = 0; e < E; e++) u[b][e] *= a.factor * scale[b];
    if (CAP) cap_scores(u, a.cap, a.cap_inv);
    if (CAP || SCORE == ENSI_SCORE_SIGMOID)
#pragma unroll
        for (int b = 0; b < B; b++)
#pragma unroll
            for (int e = 0; e < E; e++) {
                if (CAP) u[b][e] *= LOG2E;
                if (SCORE == ENSI_SCORE_SIGMOID) u[b][e] += a.bias;
            }
}

// Where the rows of a tile (query tokens times the heads that share a key head, token by token) look: from key lo, rounded down to a tile of 32, to key `last`.
struct RowTile {
    int rows;             // of the tile; 0: none
    int first, last;      // positions of its first and last row
    int lo, tiles;        // tiles of 32 keys
};
__device__ __forceinline__ RowTile row_tile(const SeqPart &part, int row0, int most, int group, int window) {
    RowTile r;
    const int rows = part.count * group;
    r.rows = max(0, min(most, rows - row0));
    r.first = part.ctx + row0 / group;
    r.last = part.ctx + (row0 + max(r.rows, 1) - 1) / group;
    r.lo = window > 0 ? max(0, r.first - window + 1) & ~31 : 0;
    r.tiles = (r.last + 1 - r.lo + 31) / 32;
    return r;
}
// Whether a row of the tile sees a key of the block that begins at `key`: what lies before a window may have been given back, its page and scales are not looked at.
__device__ __forceinline__ bool sees_block(const RowTile &r, int key, int window) { return key <= r.last && (window <= 0 || key + KV_BLOCK - 1 > r.first - window); }

// The block of 16 keys that holds a key, as a row of the scales; -1: its page is outside the cache.
__device__ __forceinline__ int block_of(const AttentionView &a, int seq, int head, int key) {
    const int page = a.s.table[seq * a.s.table_stride + key / a.kv.page];
    if (page < 0 || page >= a.kv.pages) return -1;
    return (int)(((page * (int64_t)a.kv.heads + head) * a.kv.page + key % a.kv.page) / KV_BLOCK);
}
// Whether any key that the row at `pos` sees is in the cache: for rows whose softmax has a sum of 0, a page after the other.
__device__ __forceinline__ bool sees_any(const AttentionView &a, int seq, int pos) {
    for (int key = a.window > 0 ? max(0, pos - a.window + 1) : 0; key <= pos; key = (key / a.kv.page + 1) * a.kv.page)
        if (block_of(a, seq, 0, key) >= 0) return true;
    return false;
}
__device__ __forceinline__ bool is_nan(unsigned char code) { return (code & 0x7f) == 0x7f; }
// Which of a lane's keys its row sees, without a branch: places from low + 1 to high behind key0.
struct Seen {
    int low;
    __device__ __forceinline__ Seen(const AttentionView &a, int reach) : low(a.window > 0 ? reach - a.window : INT32_MIN) {}
    __device__ __forceinline__ bool at(int place, int high) const { return (place <= high) & (place > low); }
};

// How a lane holds its dims: PIECE of one load, then REST of a second one, for widths that are no power of two times 16; in bytes of a row, and
// of the whole row the first MAIN.
template <int DIM>
struct Split {
    static constexpr int PIECE = DIM == 64 || DIM == 96 ? 4 : DIM == 128 || DIM == 192 ? 8 : 16;
    static constexpr int REST = DIM / 16 - PIECE, MAIN = 16 * PIECE;
};

// One wave's softmax state and output for 16 queries: tile j, register r of lane (n, g) is query n and
// place PIECE (4 g + r) + j of the main part, or of the rest.
template <int DIM>
struct Rows16 {
    f32x4 o[DIM / 16];
    float m, l;
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < DIM / 16; j++) o[j] = (f32x4){0, 0, 0, 0};
        m = -__builtin_inff();
        l = 0;
    }
    __device__ __forceinline__ void scale(float f) {
#pragma unroll
        for (int j = 0; j < DIM / 16; j++)
#pragma unroll
            for (int r = 0; r < 4; r++) o[j][r] *= f;
    }
};
// 2^62 on a term e (2^64 at most, so that two add up within range), 2^32 on the softmax's sum, 2^69 on the weights: a value's scale, 2^120 at most, takes the 2^7 between
#define TERM_LIFT 62
#define SUM_LIFT 32
#define WEIGHT_LIFT 69
__device__ __forceinline__ float add_terms(float sum, float e0, float e1) { return __builtin_fmaf(e0 + e1, 0x1p-30f, sum); }
__device__ __forceinline__ float scale_of_terms(float scale) { return scale * 0x1p7f; }
static_assert(SUM_LIFT - TERM_LIFT == -30 && WEIGHT_LIFT - TERM_LIFT == 7, "factors between the lifts");
// Eight weights in two terms of bf16, set in twos: either term of both in one conversion
struct Weights {
    union {
        u32 w[4];
        bf16x8 v;
    } hi, lo;
    static __device__ __forceinline__ u32 pack(float a, float b) {
        const bf16x2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(u32, v);
    }
    __device__ __forceinline__ void set(int i, float a, float b) {
        u32 w = pack(a, b);
        asm("" : "+v"(w));  // (the compiler would convert `a` once more by itself)
        hi.w[i / 2] = w;
        lo.w[i / 2] = pack(a - __builtin_bit_cast(float, w << 16), b - __builtin_bit_cast(float, w & 0xffff0000));
    }
};
// What turns a row's sums into its outputs, 2^e f: the reference of sigmoid scores, or the softmax's sum l.  Factor and exponent apart, as their product can leave the range.
// A sum of 0: the row has no score (all of its pages are outside the cache) and gets 0, or none but -inf, which leaves its softmax undefined: NaN.  `any` tells.
struct Last {
    float f;
    int e;
    __device__ __forceinline__ float operator()(float o) const { return __builtin_ldexpf(o * f, e); }
};
template <int SCORE, class ANY>
__device__ __forceinline__ Last last_of(float m, float l, const ANY &any) {
    if (SCORE == ENSI_SCORE_SIGMOID) {
        const float whole = floorf(m);
        return {__builtin_amdgcn_exp2f(m - whole), (int)whole - WEIGHT_LIFT};
    }
    if (l == 0) return {any() ? __builtin_nanf("") : 0.0f, 0};
    return {1.0f / __builtin_amdgcn_frexp_mantf(l), SUM_LIFT - WEIGHT_LIFT - __builtin_amdgcn_frexp_expf(l)};
}
// 2^(from - to) in two equal factors: references may be 184 apart by their scales alone, which sums have to survive: the factors enter one after the other
// where their product would be small
#define HALF_LIFT_DEEP 0x1p-32f
__device__ __forceinline__ float half_lift(float from, float to) { return from == to ? 1.0f : __builtin_amdgcn_exp2f(0.5f * (from - to)); }

#define JOIN_MAX 256  // parts of a row that a join takes

// A tile of 64 keys and their values in LDS, widened to 16 bits
template <int DIM>
struct RowsLds {
    static constexpr int KEYS = 64, K_ROW = DIM * 2 + 16, V_ROW = KEYS * 2 + 16;  // bytes; 16 more keep the rows of a fragment on different banks,
    // and the chunks of 8 keys of a row of values are permuted with the row's number by 16, which does so for the rows, 4 apart, that a wave writes
    static constexpr int K_BYTES = KEYS * K_ROW, V_BYTES = DIM * V_ROW, BUFFER = K_BYTES + V_BYTES;
    static constexpr int BUFFERS = 2 * BUFFER <= 80 * 1024 ? 2 : 1;
};

inline AttentionView attention_view(ensi_ctx *ctx, const KvView &kv, const ensi_clear_attention_args &a) {
    AttentionView v = {kv, a.s, a.q, a.out, a.q_stride, a.out_stride, a.q_heads, a.q_heads / kv.heads, a.window, a.max_length, a.cap, 0, 0, a.bias * LOG2E, 0, 0, ctx->ws_clear};
    const float root = 1.0f / sqrtf((float)kv.dim);
    v.factor = a.cap > 0 ? root : root * LOG2E;
    // 1 / cap and cap log2 e stay finite: scores below 2^-120 are as good as 0, and of scores that a cap beyond 2^126 reaches only which are equal matters
    if (a.cap > 0) v.cap = std::min(std::max(a.cap, 0x1p-120f), 0x1p126f);
    v.cap_inv = a.cap > 0 ? 1.0f / v.cap : 0.0f;
    return v;
}
