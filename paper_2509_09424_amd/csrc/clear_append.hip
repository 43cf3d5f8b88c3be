// New tokens into a paged cache of 8-bit keys and values, with the rotation of queries and keys on the way.
//
// The pair (a, b) of a head becomes (a cos - b sin, b cos + a sin), each product and difference rounded to 32 bits by itself, so that what is stored does
// not hang on how a compiler joins them.  A block of 16 tokens and a head has one scale, the smallest power of two that brings its largest value to
// 448: a wave owns the block of a head, whichever of the block's tokens are new, so that nothing is shared and nothing added up in an order of
// its own.  Every element is read once and written once: prompts are bound by memory (5177 tokens of 16 heads of 96 in f16: 22 us, 3.6 TB/s), a decoding step by the
// launch and the chain length, page, scale (64 sequences: 5.8 us).  Drafted tokens of a tree are stored one behind the other and rotated by the position that they
// would have if accepted: the length and their depth.
#include <type_traits>

#include "clear.h"

struct AppendView {
    KvView kv;
    ensi_clear_seqs s;
    const void *q, *k, *v;
    void *q_out;
    const float *cos, *sin;
    const int32_t *parents;  // of a tree of new tokens
    int64_t q_stride, q_out_stride, k_stride, v_stride;
    int q_heads, rot, positions, neighbours;
};

// One wave: the tokens of one block of 16 positions, one head of the queries, keys or values.  An item is 16 elements of a token in two chunks of 8:
// the two halves of 8 pairs, or 16 neighbours where pairs are neighbours or nothing is rotated.  ITEMS = ceil(dim / 64) of them to a lane.
template <int TYPE, int ITEMS, bool TREE>
__global__ __launch_bounds__(256) void k_clear_append(AppendView a) {
#pragma clang fp contract(off)
    typedef typename Elem<TYPE>::type T;
    const int lane = threadIdx.x % 64, seq = blockIdx.z, dim = a.kv.dim;
    int slot = blockIdx.x * 4 + threadIdx.x / 64;
    slot = __builtin_amdgcn_readfirstlane(slot);
    if (slot >= a.q_heads + 2 * a.kv.heads) return;
    const SeqPart part = seq_part(a.s, seq, a.kv.page, a.rot && !TREE ? min(a.positions, 1 << 30) : 1 << 30, a.kv.status);
    int depth = 0;  // lane t: of new token t
    if (TREE && part.count > 0) {
        const Tree tree = tree_of(a.parents, part, a.kv.status);
        if (!tree.good) return;
        depth = tree.depth;
        if (a.rot && __any(lane < part.count && part.ctx + depth >= a.positions)) {
            if (lane == 0) atomicOr(a.kv.status, ENSI_KV_BAD_LENGTH);
            return;
        }
    }
    const int block = part.ctx / KV_BLOCK + blockIdx.y, start = block * KV_BLOCK;
    if (part.count == 0 || start >= part.ctx + part.count) return;
    const int from = max(part.ctx, start), to = min(part.ctx + part.count, start + KV_BLOCK);  // the new positions in this block
    const bool is_q = slot < a.q_heads, is_k = !is_q && slot < a.q_heads + a.kv.heads;
    const int head = is_q ? slot : slot - a.q_heads - (is_k ? 0 : a.kv.heads);
    const T *src = (const T *)(is_q ? a.q : is_k ? a.k : a.v) + (int64_t)head * dim;
    const int64_t stride = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
    const int rot = is_q || is_k ? a.rot : 0, units = dim / 16;
    int64_t page = 0;
    if (!is_q) {
        const int p = a.s.table[seq * a.s.table_stride + start / a.kv.page];
        if (p < 0 || p >= a.kv.pages) {
            if (lane == 0) atomicOr(a.kv.status, ENSI_KV_BAD_PAGE);
            return;
        }
        page = p;
    }
    float x[ITEMS][2][8];
    int at[ITEMS][2], pos[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; i++) {
        const int item = lane + 64 * i, unit = item % units;
        pos[i] = start + item / units;
        const int place = TREE ? part.ctx + __shfl(depth, (pos[i] - part.ctx) & 63) : pos[i];  // (asked for by every lane, used by those with a new token)
        at[i][0] = at[i][1] = 0;
#pragma unroll
        for (int c = 0; c < 2; c++)
#pragma unroll
            for (int j = 0; j < 8; j++) x[i][c][j] = 0;
        if (pos[i] < from || pos[i] >= to) {  // (items past the block's 16 tokens among them)
            pos[i] = -1;
            continue;
        }
        const bool turned = unit < rot / 16, apart = turned && !a.neighbours;
        at[i][0] = apart ? 8 * unit : 16 * unit;
        at[i][1] = apart ? 8 * unit + rot / 2 : 16 * unit + 8;
        const T *row = src + (int64_t)(part.first + pos[i] - part.ctx) * stride;
        Chunk<TYPE>::load(x[i][0], row + at[i][0]);
        Chunk<TYPE>::load(x[i][1], row + at[i][1]);
        if (turned) {
            float c[8], s[8];
            const int64_t angle = (int64_t)place * (rot / 2) + 8 * unit;
            Chunk<ENSI_T_F32>::load(c, a.cos + angle);
            Chunk<ENSI_T_F32>::load(s, a.sin + angle);
            const auto turn = [](float &u, float &w, float cosine, float sine) {
                const float u1 = u * cosine - w * sine;
                w = w * cosine + u * sine;
                u = u1;
            };
            if (a.neighbours) {
#pragma unroll
                for (int j = 0; j < 8; j++) turn(x[i][j / 4][2 * (j % 4)], x[i][j / 4][2 * (j % 4) + 1], c[j], s[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; j++) turn(x[i][0][j], x[i][1][j], c[j], s[j]);
            }
        }
    }
    if (is_q) {
        T *out = (T *)a.q_out + (int64_t)head * dim;
#pragma unroll
        for (int i = 0; i < ITEMS; i++) {
            if (pos[i] < 0) continue;
            T *row = out + (int64_t)(part.first + pos[i] - part.ctx) * a.q_out_stride;
            Chunk<TYPE>::store(row + at[i][0], x[i][0]);
            Chunk<TYPE>::store(row + at[i][1], x[i][1]);
        }
        return;
    }
    float most = 0;
#pragma unroll
    for (int i = 0; i < ITEMS; i++)
#pragma unroll
        for (int c = 0; c < 2; c++)
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const float m = fabsf(x[i][c][j]);
                if (m < __builtin_inff()) most = fmaxf(most, m);
            }
#pragma unroll
    for (int k = 1; k < 64; k *= 2) most = fmaxf(most, __shfl_xor(most, k));
    // the exponent e of the smallest 2^e with most / 2^e <= 448 = 1.75 2^8
    const u32 bits = __builtin_bit_cast(u32, most);
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    if (e < -64) e = -64;
    float scale = __builtin_bit_cast(float, (u32)(e + 127) << 23);
    const int64_t line = (page * a.kv.heads + head) * a.kv.page + start % a.kv.page;  // the block's first row of the cache
    unsigned char *codes = (is_k ? a.kv.k : a.kv.v) + line * dim;
    float *scales = (is_k ? a.kv.ks : a.kv.vs) + line / KV_BLOCK;
    if (from > start) {
        const float old = *scales;
        if (old >= scale) {
            scale = old;
        } else {  // the earlier tokens are rounded again to the larger scale
            const float ratio = old / scale;
            for (int c = lane; c < (from - start) * dim / 8; c += 64) {
                u32x2 w = *(const u32x2 *)(codes + 8 * c), o;
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    const u32 u = w[k];
                    o[k] = to_e4m3(__builtin_amdgcn_cvt_f32_fp8(u, 0) * ratio, __builtin_amdgcn_cvt_f32_fp8(u, 1) * ratio,
                                   __builtin_amdgcn_cvt_f32_fp8(u, 2) * ratio, __builtin_amdgcn_cvt_f32_fp8(u, 3) * ratio);
                }
                *(u32x2 *)(codes + 8 * c) = o;
            }
        }
    }
    const float inverse = 1.0f / scale;  // exact: a power of two
#pragma unroll
    for (int i = 0; i < ITEMS; i++) {
        if (pos[i] < 0) continue;
        unsigned char *row = codes + (pos[i] - start) * dim;
#pragma unroll
        for (int c = 0; c < 2; c++) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const float m = x[i][c][j];
                y[j] = fabsf(m) < __builtin_inff() ? m * inverse : __builtin_nanf("");
            }
            *(u32x2 *)(row + at[i][c]) = (u32x2){to_e4m3(y[0], y[1], y[2], y[3]), to_e4m3(y[4], y[5], y[6], y[7])};
        }
    }
    if (lane == 0) *scales = scale;
}

template <int TYPE>
static void append_type(const AppendView &v, hipStream_t st) {
    const int slots = v.q_heads + 2 * v.kv.heads;
    // the new tokens of a sequence touch at most this many blocks, wherever they begin
    const dim3 grid((slots + 3) / 4, (v.s.max_new + 2 * KV_BLOCK - 2) / KV_BLOCK, v.s.seqs), block(256);
    const auto go = [&](auto tree) {
        constexpr bool TREE = decltype(tree)::value;
        if (v.kv.dim <= 64) hipLaunchKernelGGL((k_clear_append<TYPE, 1, TREE>), grid, block, 0, st, v);
        else if (v.kv.dim <= 128) hipLaunchKernelGGL((k_clear_append<TYPE, 2, TREE>), grid, block, 0, st, v);
        else if (v.kv.dim <= 192) hipLaunchKernelGGL((k_clear_append<TYPE, 3, TREE>), grid, block, 0, st, v);
        else hipLaunchKernelGGL((k_clear_append<TYPE, 4, TREE>), grid, block, 0, st, v);
    };
    if (v.parents) go(std::true_type());
    else go(std::false_type());
}

void launch_clear_append(ensi_ctx *ctx, const KvView &kv, const ensi_clear_append_args &a, const int32_t *parents, hipStream_t st) {
    ScopedTimer timer(ctx, "k_clear_append", st);
    const AppendView v = {kv, a.s, a.q, a.k, a.v, a.q_out, a.cos, a.sin, parents, a.q_stride, a.q_out_stride, a.k_stride, a.v_stride, a.q ? a.q_heads : 0, a.rot, a.positions, a.pairs == ENSI_ROT_NEIGHBOURS};
    if (a.type == ENSI_T_F32) return append_type<ENSI_T_F32>(v, st);
    if (a.type == ENSI_T_BF16) return append_type<ENSI_T_BF16>(v, st);
    append_type<ENSI_T_F16>(v, st);
}
