// Attention of trees of drafted tokens over a paged cache (the mathematics: clear_attention.h).  New token t of a sequence sees the cached tokens, itself and its ancestors; its
// position is the length and its depth.
//
// A sequence has up to 64 new tokens, so one word of 64 bits holds what a row sees of them, and the rows of a sequence and key head read the same long cache.  Two kernels: up to
// 64 rows (a few tokens each) are bound by the cache's bytes, so a workgroup takes 16 or 32 of them and its four waves a quarter of its keys each, a tile of 32 widened once for all
// of a wave's rows and the next one under way (48 sequences of 8 tokens behind up to 8191 on 20 over 5 heads of 128: 223 MB in 62 us, and the join 6); more rows are bound by vector
// instructions, and share keys that are widened once for 128 of them.  Either splits long caches over workgroups; a third kernel joins the parts.
#include "clear_attention.h"

// Which of the 32 keys from key0 on a row sees: cached ones within the window of its place, and those of its line.
__device__ __forceinline__ u32 seen_keys(const SeqPart &part, int window, u64 line, int place, int key0) {
    const int old = part.ctx - key0;  // keys of the tile that are cached ones
    u32 seen = old >= 32 ? ~0u : old > 0 ? (1u << old) - 1 : 0;
    if (window > 0) {
        const int dark = place - window + 1 - key0;  // of its first keys lie before the window
        if (dark > 0) seen = dark >= 32 ? 0 : seen & (~0u << dark);
    }
    if (old <= 0) {
        if (old > -64) seen |= (u32)(line >> -old);
    } else if (old < 32)
        seen |= (u32)line << old;
    return seen;
}
// Whether any key that a row sees is in the cache.
__device__ __forceinline__ bool sees_any_of(const AttentionView &a, int seq, const SeqPart &part, u64 line, int place) {
    for (int key = a.window > 0 ? max(0, place - a.window + 1) : 0; key < part.ctx; key = (key / a.kv.page + 1) * a.kv.page)
        if (block_of(a, seq, 0, key) >= 0) return true;
    for (int t = 0; t < part.count; t++)
        if ((line >> t & 1) && block_of(a, seq, 0, part.ctx + t) >= 0) return true;
    return false;
}
// The keys that a sequence's trees look at, in tiles of 32.
struct TreeKeys {
    int lo, last, tiles;
};
__device__ __forceinline__ TreeKeys tree_keys(const SeqPart &part, int window) {
    TreeKeys k;
    k.lo = window > 0 ? max(0, part.ctx - window + 1) & ~31 : 0;
    k.last = part.ctx + part.count - 1;
    k.tiles = (k.last + 1 - k.lo + 31) / 32;
    return k;
}
// The part of a line within the window: ancestors come before their children, so the nearest ones are its highest bits.
__device__ __forceinline__ u64 near_line(u64 line, int window) {
    if (window > 0)
        for (int more = __popcll(line) - window; more > 0; more--) line &= line - 1;
    return line;
}

// Products q c to what the exponent takes, and the factor with which it takes them.  Softmax without a cap: the products as they are, a key's scale enters with the exponent.
template <int SCORE, int B, int E>
__device__ __forceinline__ void tree_scores(float (&u)[B][E], float (&factor)[B], const float (&ks)[B], const float (&vs)[B], const AttentionView &a) {
    const bool capped = a.cap > 0;
#pragma unroll
    for (int b = 0; b < B; b++) factor[b] = a.factor * ks[b];
    if (capped) {
#pragma unroll
        for (int b = 0; b < B; b++)
#pragma unroll
            for (int e = 0; e < E; e++) u[b][e] *= factor[b];
        cap_scores(u, a.cap, a.cap_inv);
#pragma unroll
        for (int b = 0; b < B; b++) factor[b] = LOG2E;
    }
    if (SCORE == ENSI_SCORE_SIGMOID)
#pragma unroll
        for (int b = 0; b < B; b++)
#pragma unroll
            for (int e = 0; e < E; e++) u[b][e] = vs[b] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-__builtin_fmaf(u[b][e], factor[b], a.bias)));
}
// A lane's largest one of a block, against the reference: log2 of the weight, or the weight of the sigmoid
template <int SCORE, int E>
__device__ __forceinline__ float tree_most(const float (&u)[E], float factor, float log_v) {
    float top = u[0];
#pragma unroll
    for (int e = 1; e < E; e++) top = most_of(top, u[e]);
    return SCORE == ENSI_SCORE_SIGMOID ? top : __builtin_fmaf(top, factor, log_v);
}

template <int DIM, int RT>
struct TreeLds {
    static constexpr int ROWS = 16 * RT, ROW = DIM + 4;  // floats of a row; 4 more put the rows that are written at once on different banks
    static constexpr int BYTES = 4 * ROWS * (ROW + 2) * 4;
};

template <int TYPE, int DIM, int SCORE, int RT>
__global__ __launch_bounds__(256) void k_clear_attention_tree(AttentionView a, const int32_t *parents, int split_tiles) {
    typedef typename Elem<TYPE>::type T;
    typedef Wide<TYPE> W;
    typedef typename W::vec vec;
    typedef TreeLds<DIM, RT> L;
    constexpr int STEPS = DIM / 32, TILES = DIM / 16, PIECE = Split<DIM>::PIECE, REST = Split<DIM>::REST, MAIN = Split<DIM>::MAIN;
    extern __shared__ __align__(16) float tree_lds[];
    __shared__ u64 lines[TREE_MAX];
    __shared__ int places[TREE_MAX];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 16, g = lane / 16;
    const int blocks = (a.row_tiles + RT - 1) / RT;
    const int seq = blockIdx.z, head = blockIdx.x / blocks, row0 = 16 * RT * (blockIdx.x % blocks), split = blockIdx.y;
    const SeqPart part = seq_part(a.s, seq, a.kv.page, a.max_length, a.kv.status);
    const int rows = part.count * a.group;
    const TreeKeys keys = tree_keys(part, a.window);
    const int tile0 = split * split_tiles, tile1 = min(tile0 + split_tiles, keys.tiles);
    if (row0 >= rows || tile0 >= tile1) return;
    int index[RT];  // of the row's token among the new ones
    vec q[RT][STEPS];
    Rows16<DIM> st[RT];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        const int row = min(row0 + 16 * rt + n, rows - 1);
        index[rt] = row / a.group;
        typedef vec loose __attribute__((aligned(2)));
        const T *p = (const T *)a.q + (int64_t)(part.first + index[rt]) * a.q_stride + (int64_t)(head * a.group + row % a.group) * DIM + g * (DIM / 4);
#pragma unroll
        for (int s = 0; s < STEPS; s++) q[rt][s] = *(const loose *)(p + 8 * s);
        st[rt].clear();
    }
    // 32 tiles of this wave at once: lane l looks up the block of 16 keys of half l % 2 of tile l / 2
    int my_block = 0, my_good = 0;
    float my_k = 1, my_v = 1;
    const auto look_up = [&](int batch) {
        const int t = batch + 4 * (lane / 2), key = keys.lo + 32 * t + 16 * (lane % 2);
        my_block = my_good = 0;
        my_k = my_v = 1;
        if (t < tile1 && key <= keys.last && (a.window <= 0 || key + KV_BLOCK - 1 > part.ctx - a.window)) {
            const int block = block_of(a, seq, head, key);
            if (block >= 0) {
                my_block = block;
                my_good = 1;
                my_k = a.kv.ks[block];
                my_v = fmaxf(a.kv.vs[block], 0x1p-64f);
            } else
                atomicOr(a.kv.status, ENSI_KV_BAD_PAGE);
        }
    };
    look_up(tile0 + wave);
    // lines and positions, where a tile has new tokens or the edge of a window (what is left out for its tree is left out by those workgroups and the join)
    if (keys.lo + 32 * tile1 > part.ctx || a.window > 0) {
        const Tree tree = tree_of(parents, part, a.kv.status);
        if (!tree.good) return;
        if (wave == 0) {
            lines[lane] = near_line(tree.line, a.window);
            places[lane] = part.ctx + tree.depth;
        }
        __syncthreads();
    }
    int nan_from = INT32_MAX, nan_to = -1;  // keys between which values had NaN
    for (int batch = tile0 + wave; batch < tile1; batch += 4 * 32) {
        if (batch != tile0 + wave) look_up(batch);
        const int turns = min(32, (tile1 - batch + 3) / 4);
        // keys: lane (n, g) has places DIM / 4 g .. of key n; values: places PIECE n .. of keys 4 g .. 4 g + 3 of either half
        constexpr int WORDS = (PIECE + REST + 3) / 4;
        struct Codes {
            u32x2 k[2][STEPS];
            u32 v[2][WORDS][4];
        };
        const int k_at = n * DIM + g * (DIM / 4), v_at = 4 * g * DIM + PIECE * n, rest_at = 4 * g * DIM + MAIN + REST * n;
        const auto fetch_keys = [&](Codes &to, int i) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                // a wave's base and a lane's offset of 32 bits: no registers for 64-bit addresses
                const unsigned char *p = a.kv.k + (int64_t)__builtin_amdgcn_readlane(my_block, 2 * i + h) * (KV_BLOCK * DIM);
#pragma unroll
                for (int s = 0; s < STEPS; s++) to.k[h][s] = *(const u32x2 *)(p + (u32)(k_at + 8 * s));
            }
        };
        const auto fetch_values = [&](Codes &to, int i) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const unsigned char *p = a.kv.v + (int64_t)__builtin_amdgcn_readlane(my_block, 2 * i + h) * (KV_BLOCK * DIM);
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    typedef u32 piece __attribute__((ext_vector_type(PIECE / 4)));
                    const piece v = *(const piece *)(p + (u32)(v_at + r * DIM));
#pragma unroll
                    for (int w = 0; w < PIECE / 4; w++) to.v[h][w][r] = v[w];
                    if (REST == 4) to.v[h][WORDS - 1][r] = *(const u32 *)(p + (u32)(rest_at + r * DIM));
                    if (REST == 2) to.v[h][WORDS - 1][r] = *(const unsigned short *)(p + (u32)(rest_at + r * DIM));
                }
            }
        };
        Codes now;
        fetch_keys(now, 0);
        for (int i = 0; i < turns; i++) {
            const int key0 = keys.lo + 32 * (batch + 4 * i);
            int good[2];
            float ks[2], vs[2], lv[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                good[h] = __builtin_amdgcn_readlane(my_good, 2 * i + h);
                ks[h] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_k), 2 * i + h));
                vs[h] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_v), 2 * i + h));
                lv[h] = SCORE == ENSI_SCORE_SIGMOID ? 0 : __builtin_amdgcn_logf(vs[h]);
            }
            fetch_values(now, i);
            const bool masked = key0 + 31 >= part.ctx || (a.window > 0 && key0 <= keys.last - a.window) || !good[0] || !good[1];
            vec k[2][STEPS];
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int s = 0; s < STEPS; s++) k[h][s] = W::widen(now.k[h][s][0], now.k[h][s][1]);
            // the next tile's keys are under way while this one is computed (its values too would not fit two waves' registers)
            if (i + 1 < turns) fetch_keys(now, i + 1);
            Weights p[RT];
#pragma unroll
            for (int rt = 0; rt < RT; rt++) {
                f32x4 qk[2];
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    qk[h] = (f32x4){0, 0, 0, 0};
#pragma unroll
                    for (int s = 0; s < STEPS; s++) qk[h] = W::mfma16(k[h][s], q[rt][s], qk[h]);
                }
                float u[2][4];
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int r = 0; r < 4; r++) u[h][r] = qk[h][r];
                float factor[2];
                tree_scores<SCORE>(u, factor, ks, vs, a);
                if (masked) {
                    u32 seen = seen_keys(part, a.window, lines[index[rt]], places[index[rt]], key0);
                    seen &= (good[0] ? 0xffffu : 0) | (good[1] ? 0xffff0000u : 0);
                    seen >>= 4 * g;
#pragma unroll
                    for (int h = 0; h < 2; h++)
#pragma unroll
                        for (int r = 0; r < 4; r++) u[h][r] = seen >> (16 * h + r) & 1 ? u[h][r] : SCORE == ENSI_SCORE_SIGMOID ? 0 : -__builtin_inff();
                }
                float most = SCORE == ENSI_SCORE_SIGMOID ? 0 : -__builtin_inff();
#pragma unroll
                for (int h = 0; h < 2; h++) most = most_of(most, tree_most<SCORE>(u[h], factor[h], lv[h]));
                most = most_of(most, __shfl_xor(most, 16));
                most = most_of(most, __shfl_xor(most, 32));
                if (SCORE == ENSI_SCORE_SIGMOID) most = most_of(__builtin_amdgcn_logf(most), -120.0f);
                const float m = most_of(st[rt].m, most), base = m == -__builtin_inff() ? 0.0f : m;
                const float lift = half_lift(st[rt].m, base);
                st[rt].m = m;
                if (__any(lift != 1.0f)) {
                    const bool deep = __any(lift < HALF_LIFT_DEEP);
                    if (deep) st[rt].scale(lift);
                    st[rt].scale(deep ? lift : lift * lift);
                    st[rt].l = st[rt].l * lift * lift;
                }
                const float unit = __builtin_amdgcn_exp2f(0.5f * (WEIGHT_LIFT - base));  // sigmoid: half of the way to the reference
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        if (SCORE == ENSI_SCORE_SIGMOID) {
                            p[rt].set(4 * h + r, u[h][r] * unit * unit, u[h][r + 1] * unit * unit);
                        } else {
                            const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(u[h][r], factor[h], TERM_LIFT - base)), e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(u[h][r + 1], factor[h], TERM_LIFT - base)), scale = scale_of_terms(vs[h]);
                            st[rt].l = add_terms(st[rt].l, e0, e1);
                            p[rt].set(4 * h + r, e0 * scale, e1 * scale);
                        }
                    }
            }
            // values that some row does not see: NaN among them is taken as 0 (elsewhere it finds its way through the products)
            if (masked) {
                u32 nans = 0;
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int x = 0; x < WORDS; x++)
#pragma unroll
                        for (int r = 0; r < 4; r++) nans |= nan_bytes(now.v[h][x][r]);
                if (__any((nans & 0x80808080) != 0)) {
                    bool inside = false;  // of a token of the sequence, not of what lies behind its end
#pragma unroll
                    for (int h = 0; h < 2; h++)
#pragma unroll
                        for (int x = 0; x < WORDS; x++)
#pragma unroll
                            for (int r = 0; r < 4; r++) {
                                const u32 hit = nan_bytes(now.v[h][x][r]) & 0x80808080;
                                inside |= hit && key0 + 16 * h + 4 * g + r <= keys.last;
                                now.v[h][x][r] &= ~((hit >> 7) * 0xff);
                            }
                    if (__any(inside)) {
                        nan_from = min(nan_from, key0);
                        nan_to = key0 + 31;
                    }
                }
            }
#pragma unroll
            for (int x = 0; x < WORDS; x++) {
#pragma unroll
                for (int h = 0; h < 2; h++) transpose4(now.v[h][x]);
#pragma unroll
                for (int b = 0; b < 4; b++) {
                    const int j = 4 * x + b;
                    if (j >= TILES) continue;
                    const bf16x8 v = Wide<ENSI_T_BF16>::widen(now.v[0][x][b], now.v[1][x][b]);
#pragma unroll
                    for (int rt = 0; rt < RT; rt++) {
                        st[rt].o[j] = Wide<ENSI_T_BF16>::mfma16(v, p[rt].hi.v, st[rt].o[j]);
                        st[rt].o[j] = Wide<ENSI_T_BF16>::mfma16(v, p[rt].lo.v, st[rt].o[j]);
                    }
                }
            }
        }
    }
    for (int key = nan_from; key <= min(nan_to, keys.last); key++) {
        // rare, and of this wave's tiles only
        const int block = (key - keys.lo) / 32 % 4 == (tile0 + wave) % 4 ? block_of(a, seq, head, key) : -1;
        if (block < 0) continue;
        const unsigned char *v = a.kv.v + ((int64_t)block * KV_BLOCK + key % KV_BLOCK) * DIM;
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            if (!(seen_keys(part, a.window, lines[index[rt]], places[index[rt]], key) & 1)) continue;
#pragma unroll
            for (int j = 0; j < TILES; j++)
#pragma unroll
                for (int r = 0; r < 4; r++)
                    if (is_nan(v[j < PIECE ? PIECE * (4 * g + r) + j : MAIN + REST * (4 * g + r) + j - PIECE])) st[rt].o[j][r] = __builtin_nanf("");
        }
    }
    // the four waves' sums through LDS, a row's floats side by side; every thread then joins and stores neighbouring ones
    float *const ms = tree_lds + 4 * L::ROWS * L::ROW, *const ls = ms + 4 * L::ROWS;
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        Rows16<DIM> &s = st[rt];
        // a lane has the sum of its keys only
        s.l += __shfl_xor(s.l, 16);
        s.l += __shfl_xor(s.l, 32);
        const int row = wave * L::ROWS + 16 * rt + n;
        float *to = tree_lds + row * L::ROW;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            typedef float piece __attribute__((ext_vector_type(PIECE)));
            piece v;
#pragma unroll
            for (int j = 0; j < PIECE; j++) v[j] = s.o[j][r];
            *(piece *)(to + PIECE * (4 * g + r)) = v;
            if constexpr (REST > 0) {
                typedef float rest __attribute__((ext_vector_type(REST), aligned(8)));
                rest w;
#pragma unroll
                for (int j = 0; j < REST; j++) w[j] = s.o[PIECE + j][r];
                *(rest *)(to + MAIN + REST * (4 * g + r)) = w;
            }
        }
        if (g == 0) {
            ms[row] = s.m;
            ls[row] = s.l;
        }
    }
    __syncthreads();
    const bool whole = keys.tiles <= split_tiles;
    constexpr int QUADS = DIM / 4;
#pragma unroll 2
    for (int i = threadIdx.x; i < L::ROWS * QUADS; i += 256) {
        const int r = i / QUADS, quad = i % QUADS, row = row0 + r;
        if (row >= rows) break;
        float m = ms[r], l = 0;
#pragma unroll
        for (int w = 1; w < 4; w++) m = most_of(m, ms[w * L::ROWS + r]);
        const float base = m == -__builtin_inff() ? 0.0f : m;
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; w++) {
            const float h = half_lift(ms[w * L::ROWS + r], base);
            const f32x4 v = *(const f32x4 *)(tree_lds + (w * L::ROWS + r) * L::ROW + 4 * quad);
#pragma unroll
            for (int e = 0; e < 4; e++) o[e] += v[e] * h * h;
            l += ls[w * L::ROWS + r] * h * h;
        }
        const int token = row / a.group;
        if (whole) {
            const Last end = last_of<SCORE>(m, l, [&] { return sees_any_of(a, seq, part, lines[token], places[token]); });
            typedef T quad_t __attribute__((ext_vector_type(4), aligned(sizeof(T))));
            quad_t w;
#pragma unroll
            for (int e = 0; e < 4; e++) w[e] = (T)end(o[e]);
            *(quad_t *)((T *)a.out + (int64_t)(part.first + token) * a.out_stride + (int64_t)(head * a.group + row % a.group) * DIM + 4 * quad) = w;
        } else {
            float *ws = a.ws + ((((int64_t)seq * a.kv.heads + head) * a.row_tiles + row / 16) * a.splits + split) * (16 * DIM + 32);
            *(f32x4 *)(ws + row % 16 * DIM + 4 * quad) = o;
            if (quad == 0) {
                ws[16 * DIM + row % 16] = m;
                ws[16 * DIM + 16 + row % 16] = l;
            }
        }
    }
}

// Many rows: 128 of them to a workgroup, 32 to a wave, and tiles of 64 keys widened once for all of them in LDS (RowsLds; a wave fetches and widens a block of 16 keys and values while
// the tile before is computed).  Widening a tile in every wave takes a third of the kernel above's vector instructions: 64 sequences of up to 64 tokens behind up to 300 on 20 over 5 heads of
// 128 59 us there, 37 here; 16 behind 2048 60 and 47.  What bounds it: 64 sequences of 64 tokens behind 300 each (47 us) are 640 workgroups on 512 places, 1.2 waves a SIMD of 2 on the average;
// vector instructions have 32 % of the SIMDs' cycles, matrix ones 18 %, LDS 16 % of the CUs'.
template <int TYPE, int DIM, int SCORE>
__global__ __launch_bounds__(256, DIM <= 128 ? 2 : 1) void k_clear_attention_tree_rows(AttentionView a, const int32_t *parents, int split_tiles) {
    typedef typename Elem<TYPE>::type T;
    typedef Wide<TYPE> W;
    typedef typename W::vec vec;
    typedef RowsLds<DIM> L;
    constexpr int STEPS = DIM / 16, TILES = DIM / 32, ITEMS = (DIM / 2 + 63) / 64;  // of the values: 8 keys x 4 places
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ int nan_tiles[2];  // first and last tile whose values had NaN
    __shared__ u64 lines[TREE_MAX];
    __shared__ int places[TREE_MAX];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 32, half = lane / 32;
    const int blocks = (a.row_tiles + 7) / 8;
    const int seq = blockIdx.z, head = blockIdx.x / blocks, block_row = 128 * (blockIdx.x % blocks), split = blockIdx.y;
    const SeqPart part = seq_part(a.s, seq, a.kv.page, a.max_length, a.kv.status);
    const int rows = part.count * a.group;
    const TreeKeys keys = tree_keys(part, a.window);
    const int tile0 = split * split_tiles, tile1 = min(tile0 + split_tiles, keys.tiles);  // of 32 keys, two of which are a tile here
    if (block_row >= rows || tile0 >= tile1) return;
    const int row0 = block_row + 32 * wave, lo = keys.lo + 32 * tile0, tiles = (tile1 - tile0 + 1) / 2;
    const int row = min(row0 + n, rows - 1), index = row / a.group, token = part.first + index;
    const int q_head = head * a.group + row % a.group;
    vec q[STEPS];
    {
        typedef vec loose __attribute__((aligned(2)));
        const T *p = (const T *)a.q + (int64_t)token * a.q_stride + (int64_t)q_head * DIM + 8 * half;
#pragma unroll
        for (int s = 0; s < STEPS; s++) q[s] = *(const loose *)(p + 16 * s);
    }
    f32x16 o[TILES];
#pragma unroll
    for (int j = 0; j < TILES; j++)
#pragma unroll
        for (int r = 0; r < 16; r++) o[j][r] = 0;
    float st_m = -__builtin_inff(), st_l = 0;
    // what 16 tiles need to know of their blocks of 16 keys: lane l has block l % 4 of tile l / 4
    int my_block = 0, my_good = 0;
    float my_k = 1, my_v = 1;
    const auto look_up = [&](int first) {
        const int key = lo + 64 * first + 16 * lane;
        my_block = my_good = 0;
        my_k = my_v = 1;
        if (key < keys.lo + 32 * tile1 && key <= keys.last && (a.window <= 0 || key + KV_BLOCK - 1 > part.ctx - a.window)) {
            const int block = block_of(a, seq, head, key);
            if (block >= 0) {
                my_block = block;
                my_good = 1;
                my_k = a.kv.ks[block];
                my_v = fmaxf(a.kv.vs[block], 0x1p-64f);
            } else
                atomicOr(a.kv.status, ENSI_KV_BAD_PAGE);
        }
    };
    // a wave's block of a tile: keys, DIM / 4 bytes of row lane / 4; values, items (half of the block's keys, 4 places)
    u32x2 kc[DIM / 32];
    u32 vc[ITEMS][8];
    const auto fetch = [&](int t) {
        const int64_t block = __builtin_amdgcn_readlane(my_block, 4 * (t % 16) + wave);
        const unsigned char *k = a.kv.k + block * (KV_BLOCK * DIM), *v = a.kv.v + block * (KV_BLOCK * DIM);
#pragma unroll
        for (int i = 0; i < DIM / 32; i++) kc[i] = *(const u32x2 *)(k + (u32)(lane * (DIM / 4) + 8 * i));
#pragma unroll
        for (int i = 0; i < ITEMS; i++) {
            const int item = lane + 64 * i, h = item / (DIM / 4), places = 4 * (item % (DIM / 4));
            if (DIM / 2 % 64 == 0 || item < DIM / 2) {
#pragma unroll
                for (int e = 0; e < 8; e++) vc[i][e] = *(const u32 *)(v + (u32)((4 * h + 8 * (e / 4) + e % 4) * DIM + places));
            }
        }
    };
    const auto put = [&](int t) {
        unsigned char *at = lds + (L::BUFFERS == 2 ? t % 2 * L::BUFFER : 0);
        unsigned char *k = at + (16 * wave + lane / 4) * L::K_ROW + (lane % 4) * (DIM / 2);
#pragma unroll
        for (int i = 0; i < DIM / 32; i++) *(vec *)(k + 16 * i) = W::widen(kc[i][0], kc[i][1]);
        // values that some row does not see: NaN among them is taken as 0 (elsewhere it finds its way through the products)
        u32 nans = 0;
        if (lo + 64 * t + 63 >= part.ctx || (a.window > 0 && lo + 64 * t <= keys.last - a.window) || !__builtin_amdgcn_readlane(my_good, 4 * (t % 16) + wave))
#pragma unroll
            for (int i = 0; i < ITEMS; i++)
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (DIM / 2 % 64 == 0 || lane + 64 * i < DIM / 2) nans |= nan_bytes(vc[i][e]);
        if (__any((nans & 0x80808080) != 0)) {
            bool inside = false;  // of a token of the sequence, not of what lies behind its end
#pragma unroll
            for (int i = 0; i < ITEMS; i++) {
                const int item = lane + 64 * i, h = item / (DIM / 4);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const u32 hit = item < DIM / 2 ? nan_bytes(vc[i][e]) & 0x80808080 : 0;
                    inside |= hit && lo + 64 * t + 16 * wave + 4 * h + 8 * (e / 4) + e % 4 <= keys.last;
                    vc[i][e] &= ~((hit >> 7) * 0xff);
                }
            }
            if (inside) {
                atomicMin(&nan_tiles[0], t);
                atomicMax(&nan_tiles[1], t);
            }
        }
#pragma unroll
        for (int i = 0; i < ITEMS; i++) {
            const int item = lane + 64 * i, h = item / (DIM / 4), places = 4 * (item % (DIM / 4));
            if (DIM / 2 % 64 == 0 || item < DIM / 2) {
                u32 x[2][4];
#pragma unroll
                for (int e = 0; e < 8; e++) x[e / 4][e % 4] = vc[i][e];
                transpose4(x[0]);
                transpose4(x[1]);
#pragma unroll
                for (int j = 0; j < 4; j++) *(bf16x8 *)(at + L::K_BYTES + (places + j) * L::V_ROW + 16 * ((2 * wave + h) ^ (places / 16 % 4))) = Wide<ENSI_T_BF16>::widen(x[0][j], x[1][j]);
            }
        }
    };
    if (threadIdx.x == 0) {
        nan_tiles[0] = INT32_MAX;
        nan_tiles[1] = -1;
    }
    look_up(0);
    fetch(0);
    // lines and positions, where a tile has new tokens or the edge of a window (what is left out for its tree is left out by those workgroups and the join)
    if (keys.lo + 32 * tile1 > part.ctx || a.window > 0) {
        const Tree tree = tree_of(parents, part, a.kv.status);
        if (!tree.good) return;
        if (wave == 0) {
            lines[lane] = near_line(tree.line, a.window);
            places[lane] = part.ctx + tree.depth;
        }
    }
    __syncthreads();
    put(0);
    __syncthreads();
    for (int t = 0; t < tiles; t++) {
        const int key0 = lo + 64 * t;
        int good[4];
        float ks[4], vs[4];
#pragma unroll
        for (int b = 0; b < 4; b++) {
            good[b] = __builtin_amdgcn_readlane(my_good, 4 * (t % 16) + b);
            ks[b] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_k), 4 * (t % 16) + b));
            vs[b] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_v), 4 * (t % 16) + b));
        }
        if (t + 1 < tiles) {
            if ((t + 1) % 16 == 0) look_up(t + 1);
            fetch(t + 1);
        }
        if (row0 < rows) {
            const unsigned char *at = lds + (L::BUFFERS == 2 ? t % 2 * L::BUFFER : 0);
            // fragments of AHEAD steps under way: left to itself, the compiler keeps two reads under way, and a wave waits for LDS most of its time
            f32x16 qk[2];
            constexpr int AHEAD = STEPS < 4 ? STEPS : 4;
            vec kf[AHEAD][2];
            const auto read_keys = [&](int s) {
#pragma unroll
                for (int x = 0; x < 2; x++) kf[s % AHEAD][x] = *(const vec *)(at + (32 * x + n) * L::K_ROW + 32 * s + 16 * half);
            };
#pragma unroll
            for (int s = 0; s < AHEAD; s++) read_keys(s);
#pragma unroll
            for (int x = 0; x < 2; x++)
#pragma unroll
                for (int r = 0; r < 16; r++) qk[x][r] = 0;
#pragma unroll
            for (int s = 0; s < STEPS; s++) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < 2; x++) qk[x] = W::mfma32(kf[s % AHEAD][x], q[s], qk[x]);
                if (s + AHEAD < STEPS) read_keys(s + AHEAD);
            }
            __builtin_amdgcn_sched_barrier(0);
            // register r of half x, block b = 2 x + r / 8: key 16 b + 8 (r % 8 / 4) + 4 half + r % 4 of the wave's
            bool masked = key0 + 63 >= part.ctx || (a.window > 0 && key0 <= keys.last - a.window);
            float u[4][8], most = SCORE == ENSI_SCORE_SIGMOID ? 0 : -__builtin_inff();
#pragma unroll
            for (int b = 0; b < 4; b++) {
                masked |= !good[b];
#pragma unroll
                for (int e = 0; e < 8; e++) u[b][e] = qk[b / 2][8 * (b % 2) + e];
            }
            float factor[4], lv[4];
            tree_scores<SCORE>(u, factor, ks, vs, a);
            if (masked) {
                const u64 line = lines[index];
                const int place = places[index];
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    u32 seen = seen_keys(part, a.window, line, place, key0 + 32 * x);
                    seen &= (good[2 * x] ? 0xffffu : 0) | (good[2 * x + 1] ? 0xffff0000u : 0);
                    seen >>= 4 * half;
#pragma unroll
                    for (int b = 0; b < 2; b++)
#pragma unroll
                        for (int e = 0; e < 8; e++) u[2 * x + b][e] = seen >> (16 * b + 8 * (e / 4) + e % 4) & 1 ? u[2 * x + b][e] : SCORE == ENSI_SCORE_SIGMOID ? 0 : -__builtin_inff();
                }
            }
#pragma unroll
            for (int b = 0; b < 4; b++) {
                lv[b] = __builtin_amdgcn_logf(vs[b]);
                most = most_of(most, tree_most<SCORE>(u[b], factor[b], lv[b]));
            }
            most = most_of(most, __shfl_xor(most, 32));
            if (SCORE == ENSI_SCORE_SIGMOID) most = most_of(__builtin_amdgcn_logf(most), -120.0f);
            const float m = most_of(st_m, most), base = m == -__builtin_inff() ? 0.0f : m;
            const float lift = half_lift(st_m, base);
            st_m = m;
            if (__any(lift != 1.0f)) {
                const bool deep = __any(lift < HALF_LIFT_DEEP);
                const auto scale = [&](float f) {
#pragma unroll
                    for (int j = 0; j < TILES; j++)
#pragma unroll
                        for (int r = 0; r < 16; r++) o[j][r] *= f;
                };
                if (deep) scale(lift);
                scale(deep ? lift : lift * lift);
                st_l = st_l * lift * lift;
            }
            // A block of 16 keys at a time: its values are read and its weights formed while the matrix cores have the block before (the weights of all four in two terms
            // would not fit the registers at 128 places).
            bf16x8 vf[2][TILES];
            const auto read_values = [&](int b) {
#pragma unroll
                for (int j = 0; j < TILES; j++) vf[b % 2][j] = *(const bf16x8 *)(at + L::K_BYTES + (32 * j + n) * L::V_ROW + 16 * ((2 * b + half) ^ (2 * (j % 2) + n / 16)));
            };
            const float unit = __builtin_amdgcn_exp2f(0.5f * (WEIGHT_LIFT - base));  // sigmoid: half of the way to the reference
            Weights p[2];
            const auto weigh = [&](int b) {
                Weights &to = p[b % 2];
                if (SCORE == ENSI_SCORE_SIGMOID) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) to.set(e, u[b][e] * unit * unit, u[b][e + 1] * unit * unit);
                } else {
                    const float scale = scale_of_terms(vs[b]);
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(u[b][e], factor[b], TERM_LIFT - base)), e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(u[b][e + 1], factor[b], TERM_LIFT - base));
                        st_l = add_terms(st_l, e0, e1);
                        to.set(e, e0 * scale, e1 * scale);
                    }
                }
            };
            read_values(0);
            __builtin_amdgcn_sched_barrier(0);
            weigh(0);
#pragma unroll
            for (int b = 0; b < 4; b++) {
                if (b + 1 < 4) read_values(b + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < TILES; j++) o[j] = Wide<ENSI_T_BF16>::mfma32(vf[b % 2][j], p[b % 2].hi.v, o[j]);
#pragma unroll
                for (int j = 0; j < TILES; j++) o[j] = Wide<ENSI_T_BF16>::mfma32(vf[b % 2][j], p[b % 2].lo.v, o[j]);
                if (b + 1 < 4) weigh(b + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (L::BUFFERS == 1) __syncthreads();  // everybody has read this tile
        if (t + 1 < tiles) put(t + 1);
        __syncthreads();
    }
    if (nan_tiles[1] >= 0)
        for (int key = lo + 64 * nan_tiles[0]; key <= min(lo + 64 * nan_tiles[1] + 63, keys.last); key++) {
            const int block = block_of(a, seq, head, key);
            if (block < 0 || !(seen_keys(part, a.window, lines[index], places[index], key) & 1)) continue;
            const unsigned char *v = a.kv.v + ((int64_t)block * KV_BLOCK + key % KV_BLOCK) * DIM + 4 * half;
#pragma unroll
            for (int j = 0; j < TILES; j++)
#pragma unroll
                for (int r = 0; r < 16; r++)
                    if (is_nan(v[32 * j + 8 * (r / 4) + r % 4])) o[j][r] = __builtin_nanf("");
        }
    st_l += __shfl_xor(st_l, 32);
    if (row0 + n >= rows) return;
    if (keys.tiles > split_tiles) {
        float *ws = a.ws + ((((int64_t)seq * a.kv.heads + head) * a.row_tiles + row / 16) * a.splits + split) * (16 * DIM + 32);
#pragma unroll
        for (int j = 0; j < TILES; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) *(f32x4 *)(ws + row % 16 * DIM + 32 * j + 8 * e + 4 * half) = (f32x4){o[j][4 * e], o[j][4 * e + 1], o[j][4 * e + 2], o[j][4 * e + 3]};
        if (half == 0) {
            ws[16 * DIM + row % 16] = st_m;
            ws[16 * DIM + 16 + row % 16] = st_l;
        }
        return;
    }
    const Last end = last_of<SCORE>(st_m, st_l, [&] { return sees_any_of(a, seq, part, lines[index], places[index]); });
    T *out = (T *)a.out + (int64_t)token * a.out_stride + (int64_t)q_head * DIM;
#pragma unroll
    for (int j = 0; j < TILES; j++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            typedef T quad __attribute__((ext_vector_type(4), aligned(sizeof(T))));
            quad w;
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = (T)end(o[j][4 * e + i]);
            *(quad *)(out + 32 * j + 8 * e + 4 * half) = w;
        }
}

// Joins the parts of a row, a wave to a row: the references first, a lane to a part, then the outputs, DIM / 4 lanes to a part and as many parts side by side as
// there are lanes.
#define TREE_SPLITS 64
template <int TYPE, int DIM, int SCORE>
__global__ __launch_bounds__(256) void k_clear_attention_tree_join(AttentionView a, const int32_t *parents, int split_tiles) {
    typedef typename Elem<TYPE>::type T;
    constexpr int QUADS = DIM / 4, SLICES = 64 / QUADS;
    const int lane = threadIdx.x % 64, seq = blockIdx.z, head = blockIdx.x / a.row_tiles, tile = blockIdx.x % a.row_tiles;
    const int n = __builtin_amdgcn_readfirstlane(4 * blockIdx.y + threadIdx.x / 64), row = 16 * tile + n;
    const SeqPart part = seq_part(a.s, seq, a.kv.page, a.max_length, a.kv.status);
    const TreeKeys keys = tree_keys(part, a.window);
    if (row >= part.count * a.group || keys.tiles <= split_tiles) return;
    const int splits = (keys.tiles + split_tiles - 1) / split_tiles, index = row / a.group;
    const float *ws = a.ws + ((int64_t)seq * gridDim.x + blockIdx.x) * a.splits * (16 * DIM + 32);
    const int up = lane < part.count ? parents[part.first + lane] : -1;
    if (__any(up < -1 || up >= lane)) return;  // (the status says so by now)
    const float m = lane < splits ? ws[(int64_t)lane * (16 * DIM + 32) + 16 * DIM + n] : -__builtin_inff();
    float l = lane < splits ? ws[(int64_t)lane * (16 * DIM + 32) + 16 * DIM + 16 + n] : 0, most = m;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) most = most_of(most, __shfl_xor(most, k));
    if (most == -__builtin_inff()) most = 0;
    const float h = half_lift(m, most);
    l *= h * h;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) l += __shfl_xor(l, k);
    f32x4 o = {0, 0, 0, 0};
    const int quad = lane % QUADS, slice = lane / QUADS;
    constexpr int AHEAD = 8;
    for (int s = 0; s < splits; s += AHEAD * SLICES) {
        f32x4 v[AHEAD];
        // (the last part in place of those behind it, which do not count)
#pragma unroll
        for (int e = 0; e < AHEAD; e++) v[e] = *(const f32x4 *)(ws + (int64_t)min(s + e * SLICES + slice, splits - 1) * (16 * DIM + 32) + n * DIM + 4 * quad);
#pragma unroll
        for (int e = 0; e < AHEAD; e++) {
            const int mine = s + e * SLICES + slice;
            const float f = __shfl(h, mine & 63);
            if (slice < SLICES && mine < splits)
#pragma unroll
                for (int i = 0; i < 4; i++) o[i] = __builtin_fmaf(v[e][i] * f, f, o[i]);
        }
    }
#pragma unroll
    for (int k = SLICES / 2; k >= 1; k /= 2)
#pragma unroll
        for (int i = 0; i < 4; i++) o[i] += __shfl(o[i], (lane + k * QUADS) & 63);
    if (lane >= QUADS) return;
    const int q_head = head * a.group + row % a.group;
    const Last end = last_of<SCORE>(most, l, [&] {
        u64 line = 0;  // of the row's token
        for (int t = index; t >= 0; t = parents[part.first + t]) line |= (u64)1 << t;
        return sees_any_of(a, seq, part, near_line(line, a.window), part.ctx + __popcll(line) - 1);
    });
    typedef T quad_t __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    quad_t w;
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = (T)end(o[i]);
    *(quad_t *)((T *)a.out + (int64_t)(part.first + index) * a.out_stride + (int64_t)q_head * DIM + 4 * quad) = w;
}

template <int TYPE, int DIM, int SCORE>
static void tree_go(ensi_ctx *ctx, AttentionView v, const int32_t *parents, hipStream_t st) {
    const int heads = v.kv.heads;
    const int span = v.window > 0 ? (int)min((int64_t)v.max_length, (int64_t)v.window + v.s.max_new - 1 + 31) : v.max_length;
    v.row_tiles = (v.s.max_new * v.group + 15) / 16;
    const int tiles = (span + 31) / 32;
    const int rows = v.s.max_new * v.group, rt = v.row_tiles == 1 ? 1 : 2;
    // Keys shared through LDS from 65 rows on; with up to 64 half the waves would have none there (16 sequences of 64 tokens behind up to 1000 on 16 heads of 64 28 us by rows and 19; 48 of 16 behind
    // up to 4096 on 20 over 5 heads of 128 81 and 65).  32 rows to a workgroup where its waves have keys of their own, 16 where there are no more (64 leave one wave to a SIMD: 16 sequences of 64
    // tokens behind 2048 81 us instead of 60).
    const bool by_rows = rows > 64;
    const int width = by_rows ? 8 : rt;  // tiles of 16 rows to a workgroup
    const int64_t base = (int64_t)v.s.seqs * heads * ((v.row_tiles + width - 1) / width);
    // Parts of a row's keys.  A CU has room for two workgroups, for one from 192 places on.  Keys of one length, of one sequence or within a window: as many parts as fill that room once.
    // Sequences of different lengths, of which only the longest is known here: 9/16 more.  Each part is also written and read again, so there are no more than 1.6 sqrt(tiles), where turns of a
    // wave and parts of a row cost about the same; but of different lengths at least tiles / 40, rounded down (the tiles of a part are rounded up to fours).
    // Against four turns a workgroup wherever CUs stand idle, and otherwise parts of 12 to 32 tiles: one sequence
    // of 16 tokens behind 4096 on 20 over 5 heads of 128 19 -> 16 us; 48 behind up to 1000 36 -> 25; the kernel of 48 of 8 tokens behind up to 8191 66 -> 62; 16 of 64 tokens with a window of 2048 on 16
    // heads of 96 63 -> 54; 8 behind up to 4096 on 16 over 4 heads of 256 84 -> 66 (and on 32 over 4 heads of 64 43 -> 47).
    const int room_for = v.kv.dim <= 128 ? 512 : 256;
    const bool even = v.s.seqs == 1 || span < v.max_length;
    int splits = (int)min((int64_t)(even ? room_for : room_for + room_for * 9 / 16) / base, (int64_t)sqrtf(2.56f * tiles));
    if (!even) splits = max(splits, tiles / 40);
    splits = max(min(splits, TREE_SPLITS), 1);
    const int64_t room = (int64_t)CLEAR_WS_FLOATS / ((int64_t)v.s.seqs * heads * v.row_tiles * (16 * DIM + 32));
    if (splits > room) splits = (int)max((int64_t)1, room);
    int split_tiles = (tiles + splits - 1) / splits;
    split_tiles = max((split_tiles + 3) & ~3, 4);  // a tile for every wave
    splits = max((tiles + split_tiles - 1) / split_tiles, 1);
    v.splits = splits;
    {
        ScopedTimer timer(ctx, "k_clear_attention_tree", st);
        const auto go = [&](auto kernel, int bytes) {
            if (bytes > 48 * 1024) clear_lds(ctx, (const void *)kernel, bytes);
            hipLaunchKernelGGL(kernel, dim3(heads * ((v.row_tiles + width - 1) / width), splits, v.s.seqs), dim3(256), bytes, st, v, parents, split_tiles);
        };
        constexpr int rows_bytes = RowsLds<DIM>::BUFFERS * RowsLds<DIM>::BUFFER;
        if (by_rows) go(k_clear_attention_tree_rows<TYPE, DIM, SCORE>, rows_bytes);
        else if (rt == 1) go(k_clear_attention_tree<TYPE, DIM, SCORE, 1>, TreeLds<DIM, 1>::BYTES);
        else go(k_clear_attention_tree<TYPE, DIM, SCORE, 2>, TreeLds<DIM, 2>::BYTES);
    }
    if (splits == 1) return;
    ScopedTimer timer(ctx, "k_clear_attention_tree_join", st);
    hipLaunchKernelGGL((k_clear_attention_tree_join<TYPE, DIM, SCORE>), dim3(heads * v.row_tiles, (min(rows, 16) + 3) / 4, v.s.seqs), dim3(256), 0, st, v, parents, split_tiles);
}

template <int TYPE, int SCORE>
static void tree_dim(ensi_ctx *ctx, const AttentionView &v, const int32_t *parents, hipStream_t st) {
    switch (v.kv.dim) {
    case 64: return tree_go<TYPE, 64, SCORE>(ctx, v, parents, st);
    case 96: return tree_go<TYPE, 96, SCORE>(ctx, v, parents, st);
    case 128: return tree_go<TYPE, 128, SCORE>(ctx, v, parents, st);
    case 192: return tree_go<TYPE, 192, SCORE>(ctx, v, parents, st);
    default: return tree_go<TYPE, 256, SCORE>(ctx, v, parents, st);
    }
}

void launch_clear_attention_tree(ensi_ctx *ctx, const KvView &kv, const ensi_clear_attention_args &a, const int32_t *parents, hipStream_t st) {
    const AttentionView v = attention_view(ctx, kv, a);
    if (a.type == ENSI_T_BF16) {
        if (a.score == ENSI_SCORE_SOFTMAX) return tree_dim<ENSI_T_BF16, ENSI_SCORE_SOFTMAX>(ctx, v, parents, st);
        return tree_dim<ENSI_T_BF16, ENSI_SCORE_SIGMOID>(ctx, v, parents, st);
    }
    if (a.score == ENSI_SCORE_SOFTMAX) return tree_dim<ENSI_T_F16, ENSI_SCORE_SOFTMAX>(ctx, v, parents, st);
    tree_dim<ENSI_T_F16, ENSI_SCORE_SIGMOID>(ctx, v, parents, st);
}
