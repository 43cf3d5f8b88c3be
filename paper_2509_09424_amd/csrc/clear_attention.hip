// Attention over a paged cache of 8-bit keys and values with one scale for 16 tokens of a head.
//
// Keys are codes c with a power of two s as scale, so q k = s (q c): codes widen to the queries' 16 bits without rounding, the matrix instruction
// forms q c in 32 bits, and the scale enters with the factor that the exponent needs anyway.  Values v = s' c' are folded the other way round: their
// scale multiplies the weight.  With t the score in units of log2 e, the running reference M is the maximum of t + log2 s'; e = 2^(t - M) is what the
// softmax's sum adds up, w = e s' <= 1 the weight of the code c'.  Scales are 2^-64 to 2^120, so the largest e of a row is 2^-120 to 2^64 and
// its sum in 32 bits loses nothing, and the largest weight is 1: weights in 16 bits lose only what is 2^-24 of the row's largest contribution.
//   sigmoid scores need no sum; w = sigmoid(t) s' 2^-M with the same reference.
// A tile of scores is held as [key][query]: a lane has one query, so the statistics of a row are per lane, and the weights leave the score's
// registers in the order in which the second product reads them; the order of its keys is that of the registers, for the values too.
//
// Masks are applied to scores; a masked weight is 0, and 0 times a value that is NaN must not count: tiles that hold such codes (any lane sees one)
// take a second, rare path.
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
// Bit 7 of every byte whose code is NaN
__device__ __forceinline__ u32 nan_bytes(u32 w) { return (w & 0x7f7f7f7f) + 0x01010101; }

// The score t of a product q c, in units of the exponent: softmax log2 e t, sigmoid t log2 e + bias log2 e
template <int SCORE>
__device__ __forceinline__ float score_of(float qc, float scale, const AttentionView &a) {
    float t = qc * (a.factor * scale);
    if (a.cap > 0) {
        // cap tanh(t / cap) = cap (1 - 2 / (1 + exp(2 t / cap)))
        const float e = __builtin_amdgcn_exp2f(t * a.cap_inv);  // cap_inv = 2 log2 e / cap
        t = a.cap - 2.0f * a.cap * __builtin_amdgcn_rcpf(1.0f + e);
        t *= LOG2E;
    }
    return SCORE == ENSI_SCORE_SIGMOID ? t + a.bias : t;
}

// Where the rows of a tile of 16 (query tokens times the heads that share a key head) look: keys [lo, hi), lo rounded down to a tile of 32.
struct RowTile {
    int rows;             // of the tile; 0: none
    int first, last;      // positions of its first and last row
    int lo, tiles;
};
__device__ __forceinline__ RowTile row_tile(const SeqPart &part, int tile, int group, int window) {
    RowTile r;
    const int row0 = 16 * tile, rows = part.count * group;
    r.rows = max(0, min(16, rows - row0));
    r.first = part.ctx + row0 / group;
    r.last = part.ctx + (row0 + max(r.rows, 1) - 1) / group;
    r.lo = window > 0 ? max(0, r.first - window + 1) & ~31 : 0;
    r.tiles = (r.last + 1 - r.lo + 31) / 32;
    return r;
}

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
// 2^(from - to) in two equal factors: references may be 184 apart by their scales alone, which a sum has to survive
__device__ __forceinline__ float half_lift(float from, float to) { return from == to ? 1.0f : __builtin_amdgcn_exp2f(0.5f * (from - to)); }

// Keys split over waves and workgroups: few rows, long caches.  A workgroup has one tile of 16 rows of a key head and `split` of its keys; its four
// waves take tiles of 32 keys in turn, straight from memory into registers, and are joined in LDS; parts of several workgroups are joined by
// k_clear_attention_join.  The cache has to be read once: bound by memory.
template <int TYPE, int DIM, int SCORE>
__global__ __launch_bounds__(256) void k_clear_attention_keys(AttentionView a, int split_tiles) {
    typedef typename Elem<TYPE>::type T;
    typedef Wide<TYPE> W;
    typedef typename W::vec vec;
    constexpr int STEPS = DIM / 32, TILES = DIM / 16, PIECE = Split<DIM>::PIECE, REST = Split<DIM>::REST, MAIN = Split<DIM>::MAIN;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 16, g = lane / 16;
    const int seq = blockIdx.z, head = blockIdx.x / a.row_tiles, tile = blockIdx.x % a.row_tiles, split = blockIdx.y;
    const SeqPart part = seq_part(a.s, seq, a.kv.page, a.max_length, a.kv.status);
    const RowTile rt = row_tile(part, tile, a.group, a.window);
    const int tile0 = split * split_tiles, tile1 = min(tile0 + split_tiles, rt.tiles);
    if (rt.rows == 0 || tile0 >= tile1) return;
    const int row = 16 * tile + min(n, rt.rows - 1), token = part.first + row / a.group, pos = part.ctx + row / a.group;
    const int q_head = head * a.group + row % a.group;
    vec q[STEPS];
    {
        typedef vec loose __attribute__((aligned(2)));
        const T *p = (const T *)a.q + (int64_t)token * a.q_stride + (int64_t)q_head * DIM + g * (DIM / 4);
#pragma unroll
        for (int s = 0; s < STEPS; s++) q[s] = *(const loose *)(p + 8 * s);
    }
    Rows16<DIM> st;
    st.clear();
    for (int batch = tile0 + wave; batch < tile1; batch += 4 * 32) {
        // 32 tiles of this wave at once: lane l looks up the block of 16 keys of half l % 2 of tile l / 2
        int my_block = 0, my_good = 0;
        float my_k = 1, my_v = 1;
        {
            const int t = batch + 4 * (lane / 2), key = rt.lo + 32 * t + 16 * (lane % 2);
            if (t < tile1 && key <= rt.last) {
                const int page = a.s.table[seq * a.s.table_stride + key / a.kv.page];
                if (page >= 0 && page < a.kv.pages) {
                    my_block = ((page * (int64_t)a.kv.heads + head) * a.kv.page + key % a.kv.page) / KV_BLOCK;
                    my_good = 1;
                    my_k = a.kv.ks[my_block];
                    my_v = fmaxf(a.kv.vs[my_block], 0x1p-64f);
                } else
                    atomicOr(a.kv.status, ENSI_KV_BAD_PAGE);
            }
        }
        const int turns = min(32, (tile1 - batch + 3) / 4);
        for (int i = 0; i < turns; i++) {
            const int key0 = rt.lo + 32 * (batch + 4 * i);
            int block[2], good[2];
            float ks[2], vs[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                block[h] = __builtin_amdgcn_readlane(my_block, 2 * i + h);
                good[h] = __builtin_amdgcn_readlane(my_good, 2 * i + h);
                ks[h] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_k), 2 * i + h));
                vs[h] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_v), 2 * i + h));
            }
            // keys: lane (n, g) has places DIM / 4 g .. of key n
            u32x2 kc[2][STEPS];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const unsigned char *p = a.kv.k + ((int64_t)block[h] * KV_BLOCK + n) * DIM + g * (DIM / 4);
#pragma unroll
                for (int s = 0; s < STEPS; s++) kc[h][s] = *(const u32x2 *)(p + 8 * s);
            }
            // values: lane (n, g) has places PIECE n .. of keys 4 g .. 4 g + 3 of either half
            constexpr int WORDS = (PIECE + REST + 3) / 4;
            u32 vc[2][WORDS][4];
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const unsigned char *p = a.kv.v + ((int64_t)block[h] * KV_BLOCK + 4 * g + r) * DIM;
                    typedef u32 piece __attribute__((ext_vector_type(PIECE / 4)));
                    const piece v = *(const piece *)(p + PIECE * n);
#pragma unroll
                    for (int w = 0; w < PIECE / 4; w++) vc[h][w][r] = v[w];
                    if (REST == 4) vc[h][WORDS - 1][r] = *(const u32 *)(p + MAIN + 4 * n);
                    if (REST == 2) vc[h][WORDS - 1][r] = *(const unsigned short *)(p + MAIN + 2 * n);
                }
            f32x4 qk[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                qk[h] = (f32x4){0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < STEPS; s++) qk[h] = W::mfma16(W::widen(kc[h][s][0], kc[h][s][1]), q[s], qk[h]);
            }
            float u[2][4];
            const bool masked = key0 + 31 > rt.first || (a.window > 0 && key0 <= rt.last - a.window) || !good[0] || !good[1];
            const auto sees = [&](int h, int r) {
                const int key = key0 + 16 * h + 4 * g + r;
                return good[h] && key <= pos && (a.window <= 0 || key > pos - a.window);
            };
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    u[h][r] = score_of<SCORE>(qk[h][r], ks[h], a);
                    if (SCORE == ENSI_SCORE_SIGMOID) u[h][r] = vs[h] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-u[h][r]));
                }
            if (masked) {
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int r = 0; r < 4; r++)
                        if (!sees(h, r)) u[h][r] = SCORE == ENSI_SCORE_SIGMOID ? 0 : -__builtin_inff();
            }
            float lv[2], most = SCORE == ENSI_SCORE_SIGMOID ? 0 : -__builtin_inff();
#pragma unroll
            for (int h = 0; h < 2; h++) {
                lv[h] = SCORE == ENSI_SCORE_SIGMOID ? 0 : __builtin_amdgcn_logf(vs[h]);
                float top = fmaxf(fmaxf(u[h][0], u[h][1]), fmaxf(u[h][2], u[h][3]));
                most = fmaxf(most, top + lv[h]);
            }
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            if (SCORE == ENSI_SCORE_SIGMOID) most = fmaxf(__builtin_amdgcn_logf(most), -120.0f);
            const float m = fmaxf(st.m, most), base = m == -__builtin_inff() ? 0.0f : m;
            const float lift = half_lift(st.m, base);
            st.m = m;
            if (__any(lift != 1.0f)) {
                st.scale(lift * lift);
                st.l = st.l * lift * lift;
            }
            union {
                _Float16 e[8];
                f16x8 v;
            } p, p_lo;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const float to = SCORE == ENSI_SCORE_SIGMOID ? __builtin_amdgcn_exp2f(-base) : vs[h];
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const float e = SCORE == ENSI_SCORE_SIGMOID ? u[h][r] : __builtin_amdgcn_exp2f(u[h][r] - base), w = e * to;
                    st.l += e;
                    p.e[4 * h + r] = (_Float16)w;
                    p_lo.e[4 * h + r] = (_Float16)(w - (float)p.e[4 * h + r]);
                }
            }
            u32 nans = 0;
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int x = 0; x < WORDS; x++)
#pragma unroll
                    for (int r = 0; r < 4; r++) nans |= nan_bytes(vc[h][x][r]);
            const bool any_nan = __any((nans & 0x80808080) != 0);
            f16x8 visible;
            if (any_nan) {
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int r = 0; r < 4; r++) visible[4 * h + r] = sees(h, r) ? (_Float16)1.0f : (_Float16)0.0f;
            }
#pragma unroll
            for (int x = 0; x < WORDS; x++) {
#pragma unroll
                for (int h = 0; h < 2; h++) transpose4(vc[h][x]);
#pragma unroll
                for (int b = 0; b < 4; b++) {
                    const int j = 4 * x + b;
                    if (j >= TILES) continue;
                    u32 c0 = vc[0][x][b], c1 = vc[1][x][b];
                    if (any_nan) {
                        const u32 n0 = nan_bytes(c0) & 0x80808080, n1 = nan_bytes(c1) & 0x80808080;
                        // 0x38 is 1.0 in e4m3: ones where the code is NaN
                        const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(Wide<ENSI_T_F16>::widen((n0 >> 7) * 0x38, (n1 >> 7) * 0x38), visible, (f32x4){0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                        for (int r = 0; r < 4; r++)
                            if (hit[r] > 0) st.o[j][r] = __builtin_nanf("");
                        c0 &= ~((n0 >> 7) * 0xff);
                        c1 &= ~((n1 >> 7) * 0xff);
                    }
                    const f16x8 v = Wide<ENSI_T_F16>::widen(c0, c1);
                    st.o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p.v, st.o[j], 0, 0, 0);
                    if (TYPE == ENSI_T_F16) st.o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p_lo.v, st.o[j], 0, 0, 0);
                }
            }
        }
    }
    // a lane has the sum of its keys only
    st.l += __shfl_xor(st.l, 16);
    st.l += __shfl_xor(st.l, 32);
    // waves 2 and 3 into 0 and 1, wave 1 into 0
    __shared__ f32x4 part_o[2][TILES][64];
    __shared__ float part_m[2][64], part_l[2][64];
#pragma unroll
    for (int half = 2; half >= 1; half /= 2) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int j = 0; j < TILES; j++) part_o[wave - half][j][lane] = st.o[j];
            part_m[wave - half][lane] = st.m;
            part_l[wave - half][lane] = st.l;
        }
        __syncthreads();
        if (wave < half) {
            const float om = part_m[wave][lane], m = fmaxf(st.m, om), base = m == -__builtin_inff() ? 0.0f : m;
            const float h0 = half_lift(st.m, base), h1 = half_lift(om, base), mine = h0 * h0, other = h1 * h1;
#pragma unroll
            for (int j = 0; j < TILES; j++) {
                const f32x4 o = part_o[wave][j][lane];
#pragma unroll
                for (int r = 0; r < 4; r++) st.o[j][r] = st.o[j][r] * mine + o[r] * other;
            }
            st.l = st.l * h0 * h0 + part_l[wave][lane] * h1 * h1;
            st.m = m;
        }
        __syncthreads();
    }
    if (wave != 0 || n >= rt.rows) return;
    const bool whole = rt.tiles <= split_tiles;
    const float f = !whole ? 1.0f : SCORE == ENSI_SCORE_SIGMOID ? __builtin_amdgcn_exp2f(st.m) : st.l == 0 ? 0.0f : 1.0f / st.l;
    float *ws = a.ws + (((int64_t)seq * gridDim.x + blockIdx.x) * a.splits + split) * (16 * DIM + 32);
    T *out = (T *)a.out + (int64_t)token * a.out_stride + (int64_t)q_head * DIM;
    const auto put = [&](int at, auto first, auto count) {  // registers r of tiles first .. first + count - 1, at place `at` of the row
#pragma unroll
        for (int r = 0; r < 4; r++)
#pragma unroll
            for (int j = 0; j < decltype(count)::value; j++) {
                const float v = st.o[decltype(first)::value + j][r] * f;
                const int d = at + decltype(count)::value * (4 * g + r) + j;
                if (whole) out[d] = (T)v;
                else ws[n * DIM + d] = v;
            }
    };
    put(0, std::integral_constant<int, 0>(), std::integral_constant<int, PIECE>());
    if constexpr (REST > 0) put(MAIN, std::integral_constant<int, PIECE>(), std::integral_constant<int, REST>());
    if (!whole && g == 0) {
        ws[16 * DIM + n] = st.m;
        ws[16 * DIM + 16 + n] = st.l;
    }
}

// Joins the parts of a row: a workgroup of DIM threads to a row.
template <int TYPE, int DIM, int SCORE>
__global__ __launch_bounds__(DIM) void k_clear_attention_join(AttentionView a, int split_tiles) {
    typedef typename Elem<TYPE>::type T;
    const int seq = blockIdx.z, head = blockIdx.x / a.row_tiles, tile = blockIdx.x % a.row_tiles, n = blockIdx.y, d = threadIdx.x;
    const SeqPart part = seq_part(a.s, seq, a.kv.page, a.max_length, a.kv.status);
    const RowTile rt = row_tile(part, tile, a.group, a.window);
    if (n >= rt.rows || rt.tiles <= split_tiles) return;
    const int splits = (rt.tiles + split_tiles - 1) / split_tiles;
    const float *ws = a.ws + ((int64_t)seq * gridDim.x + blockIdx.x) * a.splits * (16 * DIM + 32);
    float m = -__builtin_inff();
    for (int s = 0; s < splits; s++) m = fmaxf(m, ws[(int64_t)s * (16 * DIM + 32) + 16 * DIM + n]);
    if (m == -__builtin_inff()) m = 0;
    float o = 0, l = 0;
    for (int s = 0; s < splits; s++) {
        const float *p = ws + (int64_t)s * (16 * DIM + 32);
        const float h = half_lift(p[16 * DIM + n], m);
        l += p[16 * DIM + 16 + n] * h * h;
        o += p[n * DIM + d] * (h * h);
    }
    const int row = 16 * tile + n, token = part.first + row / a.group, q_head = head * a.group + row % a.group;
    const float f = SCORE == ENSI_SCORE_SIGMOID ? __builtin_amdgcn_exp2f(m) : l == 0 ? 0.0f : 1.0f / l;
    ((T *)a.out)[(int64_t)token * a.out_stride + (int64_t)q_head * DIM + d] = (T)(o * f);
}

template <int TYPE, int DIM, int SCORE>
static void attention_go(ensi_ctx *ctx, AttentionView v, hipStream_t st) {
    const int heads = v.kv.heads;
    v.row_tiles = (int)(((int64_t)v.s.max_new * v.group + 15) / 16);
    const int64_t base = (int64_t)v.s.seqs * heads * v.row_tiles;
    // the most tiles of 32 keys that a tile of rows looks at: those of its window, begun within a tile and ended within one
    const int tokens = min(v.s.max_new, 15 / v.group + 2);
    const int span = v.window > 0 ? (int)min((int64_t)v.max_length, (int64_t)v.window + tokens - 1 + 31) : v.max_length;
    const int tiles = (span + 31) / 32;
    int splits = (int)min((int64_t)(tiles + 3) / 4, max((int64_t)1, 2048 / base));
    const int64_t room = (int64_t)CLEAR_WS_FLOATS / (base * (16 * DIM + 32));
    if (splits > room) splits = (int)max((int64_t)1, room);
    int split_tiles = (tiles + splits - 1) / splits;
    split_tiles = (split_tiles + 3) & ~3;  // a tile for every wave
    splits = (tiles + split_tiles - 1) / split_tiles;
    v.splits = splits;
    const dim3 grid(heads * v.row_tiles, splits, v.s.seqs);
    {
        ScopedTimer timer(ctx, "k_clear_attention", st);
        hipLaunchKernelGGL((k_clear_attention_keys<TYPE, DIM, SCORE>), grid, dim3(256), 0, st, v, split_tiles);
    }
    if (splits == 1) return;
    ScopedTimer timer(ctx, "k_clear_attention_join", st);
    const int rows = (int)min((int64_t)16, (int64_t)v.s.max_new * v.group);
    hipLaunchKernelGGL((k_clear_attention_join<TYPE, DIM, SCORE>), dim3(heads * v.row_tiles, rows, v.s.seqs), dim3(DIM), 0, st, v, split_tiles);
}

template <int TYPE, int SCORE>
static void attention_dim(ensi_ctx *ctx, const AttentionView &v, hipStream_t st) {
    switch (v.kv.dim) {
    case 64: return attention_go<TYPE, 64, SCORE>(ctx, v, st);
    case 96: return attention_go<TYPE, 96, SCORE>(ctx, v, st);
    case 128: return attention_go<TYPE, 128, SCORE>(ctx, v, st);
    case 192: return attention_go<TYPE, 192, SCORE>(ctx, v, st);
    default: return attention_go<TYPE, 256, SCORE>(ctx, v, st);
    }
}

void launch_clear_attention(ensi_ctx *ctx, const KvView &kv, const ensi_clear_attention_args &a, hipStream_t st) {
    AttentionView v = {kv, a.s, a.q, a.out, a.q_stride, a.out_stride, a.q_heads, a.q_heads / kv.heads, a.window, a.max_length, a.cap, 0, 0, a.bias * LOG2E, 0, 0, ctx->ws_clear};
    const float root = 1.0f / sqrtf((float)kv.dim);
    v.factor = a.cap > 0 ? root : root * LOG2E;
    v.cap_inv = a.cap > 0 ? 2.0f * LOG2E / a.cap : 0.0f;
    if (a.type == ENSI_T_BF16) {
        if (a.score == ENSI_SCORE_SOFTMAX) return attention_dim<ENSI_T_BF16, ENSI_SCORE_SOFTMAX>(ctx, v, st);
        return attention_dim<ENSI_T_BF16, ENSI_SCORE_SIGMOID>(ctx, v, st);
    }
    if (a.score == ENSI_SCORE_SOFTMAX) return attention_dim<ENSI_T_F16, ENSI_SCORE_SOFTMAX>(ctx, v, st);
    attention_dim<ENSI_T_F16, ENSI_SCORE_SIGMOID>(ctx, v, st);
}
