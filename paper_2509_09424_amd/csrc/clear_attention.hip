// The kernels of the attention over a paged cache (the mathematics: clear_attention.h): keys split over waves, the join of its parts, rows split over waves.
#include "clear_attention.h"

// Keys split over waves and workgroups: few rows, long caches.  A workgroup has one tile of 16 rows of a key head and `split` of its keys; its four
// waves take tiles of 32 keys in turn, straight from memory into registers, and are joined in LDS; parts of several workgroups are joined by
// k_clear_attention_join.  The cache has to be read once: bound by memory.
template <int TYPE, int DIM, int SCORE, bool CAP>
__global__ __launch_bounds__(256) void k_clear_attention_keys(AttentionView a, int split_tiles) {
    typedef typename Elem<TYPE>::type T;
    typedef Wide<TYPE> W;
    typedef typename W::vec vec;
    constexpr int STEPS = DIM / 32, TILES = DIM / 16, PIECE = Split<DIM>::PIECE, REST = Split<DIM>::REST, MAIN = Split<DIM>::MAIN;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 16, g = lane / 16;
    const int seq = blockIdx.z, head = blockIdx.x / a.row_tiles, tile = blockIdx.x % a.row_tiles, split = blockIdx.y;
    const SeqPart part = seq_part(a.s, seq, a.kv.page, a.max_length, a.kv.status);
    const RowTile rt = row_tile(part, 16 * tile, 16, a.group, a.window);
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
    int nan_from = INT32_MAX, nan_to = -1;  // keys between which values had NaN
    for (int batch = tile0 + wave; batch < tile1; batch += 4 * 32) {
        // 32 tiles of this wave at once: lane l looks up the block of 16 keys of half l % 2 of tile l / 2
        int my_block = 0, my_good = 0;
        float my_k = 1, my_v = 1;
        {
            const int t = batch + 4 * (lane / 2), key = rt.lo + 32 * t + 16 * (lane % 2);
            if (t < tile1 && sees_block(rt, key, a.window)) {
                const int block = block_of(a, seq, head, key);
                if (block >= 0) {
                    my_block = block;
                    my_good = 1;
                    my_k = a.kv.ks[block];
                    my_v = fmaxf(a.kv.vs[block], 0x1p-64f);
                } else
                    atomicOr(a.kv.status, ENSI_KV_BAD_PAGE);
            }
        }
        const int turns = min(32, (tile1 - batch + 3) / 4);
        // keys: lane (n, g) has places DIM / 4 g .. of key n; values: places PIECE n .. of keys 4 g .. 4 g + 3 of either half
        constexpr int WORDS = (PIECE + REST + 3) / 4;
        struct Codes {
            u32x2 k[2][STEPS];
            u32 v[2][WORDS][4];
        };
        const int k_at = n * DIM + g * (DIM / 4), v_at = 4 * g * DIM + PIECE * n, rest_at = 4 * g * DIM + MAIN + REST * n;
        const auto fetch = [&](Codes &to, int i) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                // a wave's base and a lane's offset of 32 bits: no registers for 64-bit addresses
                const unsigned char *p = a.kv.k + (int64_t)__builtin_amdgcn_readlane(my_block, 2 * i + h) * (KV_BLOCK * DIM);
#pragma unroll
                for (int s = 0; s < STEPS; s++) to.k[h][s] = *(const u32x2 *)(p + (u32)(k_at + 8 * s));
            }
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
        for (int i = 0; i < turns; i++) {
            const int key0 = rt.lo + 32 * (batch + 4 * i);
            int good[2];
            float ks[2], vs[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                good[h] = __builtin_amdgcn_readlane(my_good, 2 * i + h);
                ks[h] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_k), 2 * i + h));
                vs[h] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_v), 2 * i + h));
            }
            Codes now;
            fetch(now, i);
            f32x4 qk[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                qk[h] = (f32x4){0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < STEPS; s++) qk[h] = W::mfma16(W::widen(now.k[h][s][0], now.k[h][s][1]), q[s], qk[h]);
            }
            float u[2][4];
            const bool masked = key0 + 31 > rt.first || (a.window > 0 && key0 <= rt.last - a.window) || !good[0] || !good[1];
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int r = 0; r < 4; r++) u[h][r] = qk[h][r];
            scores_of<SCORE, CAP>(u, ks, a);
            if (SCORE == ENSI_SCORE_SIGMOID)
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int r = 0; r < 4; r++) u[h][r] = vs[h] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-u[h][r]));
            if (masked) {
                const int reach = pos - key0 - 4 * g;
                const Seen seen(a, reach);
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const int high = good[h] ? reach : INT32_MIN;
#pragma unroll
                    for (int r = 0; r < 4; r++) u[h][r] = seen.at(16 * h + r, high) ? u[h][r] : SCORE == ENSI_SCORE_SIGMOID ? 0 : -__builtin_inff();
                }
            }
            float lv[2], most = SCORE == ENSI_SCORE_SIGMOID ? 0 : -__builtin_inff();
#pragma unroll
            for (int h = 0; h < 2; h++) {
                lv[h] = SCORE == ENSI_SCORE_SIGMOID ? 0 : __builtin_amdgcn_logf(vs[h]);
                const float top = most_of(most_of(u[h][0], u[h][1], u[h][2]), u[h][3]);
                most = most_of(most, top + lv[h]);
            }
            most = most_of(most, __shfl_xor(most, 16));
            most = most_of(most, __shfl_xor(most, 32));
            if (SCORE == ENSI_SCORE_SIGMOID) most = most_of(__builtin_amdgcn_logf(most), -120.0f);
            const float m = most_of(st.m, most), base = m == -__builtin_inff() ? 0.0f : m;
            const float lift = half_lift(st.m, base);
            st.m = m;
            if (__any(lift != 1.0f)) {
                const bool deep = __any(lift < HALF_LIFT_DEEP);
                if (deep) st.scale(lift);
                st.scale(deep ? lift : lift * lift);
                st.l = st.l * lift * lift;
            }
            Weights p;
            const float unit = __builtin_amdgcn_exp2f(0.5f * (WEIGHT_LIFT - base));  // sigmoid: half of the way to the reference
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    if (SCORE == ENSI_SCORE_SIGMOID) {
                        p.set(4 * h + r, u[h][r] * unit * unit, u[h][r + 1] * unit * unit);
                    } else {
                        const float e0 = __builtin_amdgcn_exp2f(u[h][r] - (base - TERM_LIFT)), e1 = __builtin_amdgcn_exp2f(u[h][r + 1] - (base - TERM_LIFT)), scale = scale_of_terms(vs[h]);
                        st.l = add_terms(st.l, e0, e1);
                        p.set(4 * h + r, e0 * scale, e1 * scale);
                    }
                }
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
                            inside |= hit && key0 + 16 * h + 4 * g + r <= rt.last;
                            now.v[h][x][r] &= ~((hit >> 7) * 0xff);
                        }
                if (__any(inside)) {
                    nan_from = min(nan_from, key0);
                    nan_to = key0 + 31;
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
                    st.o[j] = Wide<ENSI_T_BF16>::mfma16(v, p.hi.v, st.o[j]);
                    st.o[j] = Wide<ENSI_T_BF16>::mfma16(v, p.lo.v, st.o[j]);
                }
            }
        }
    }
    for (int key = nan_from; key <= min(nan_to, rt.last); key++) {
        // rare, and of this wave's tiles only
        const int block = (key - rt.lo) / 32 % 4 == (tile0 + wave) % 4 ? block_of(a, seq, head, key) : -1;
        if (block < 0 || key > pos || (a.window > 0 && key <= pos - a.window)) continue;
        const unsigned char *v = a.kv.v + ((int64_t)block * KV_BLOCK + key % KV_BLOCK) * DIM;
#pragma unroll
        for (int j = 0; j < TILES; j++)
#pragma unroll
            for (int r = 0; r < 4; r++)
                if (is_nan(v[j < PIECE ? PIECE * (4 * g + r) + j : MAIN + REST * (4 * g + r) + j - PIECE])) st.o[j][r] = __builtin_nanf("");
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
            const float om = part_m[wave][lane], m = most_of(st.m, om), base = m == -__builtin_inff() ? 0.0f : m;
            const float h0 = half_lift(st.m, base), h1 = half_lift(om, base);
#pragma unroll
            for (int j = 0; j < TILES; j++) {
                const f32x4 o = part_o[wave][j][lane];
#pragma unroll
                for (int r = 0; r < 4; r++) st.o[j][r] = st.o[j][r] * h0 * h0 + o[r] * h1 * h1;
            }
            st.l = st.l * h0 * h0 + part_l[wave][lane] * h1 * h1;
            st.m = m;
        }
        __syncthreads();
    }
    if (wave != 0 || n >= rt.rows) return;
    const bool whole = rt.tiles <= split_tiles;
    const Last end = last_of<SCORE>(st.m, st.l, [&] { return whole && sees_any(a, seq, pos); });
    float *ws = a.ws + (((int64_t)seq * gridDim.x + blockIdx.x) * a.splits + split) * (16 * DIM + 32);
    T *out = (T *)a.out + (int64_t)token * a.out_stride + (int64_t)q_head * DIM;
    const auto put = [&](int at, auto first, auto count) {  // registers r of tiles first .. first + count - 1, at place `at` of the row
#pragma unroll
        for (int r = 0; r < 4; r++)
#pragma unroll
            for (int j = 0; j < decltype(count)::value; j++) {
                const float v = st.o[decltype(first)::value + j][r];
                const int d = at + decltype(count)::value * (4 * g + r) + j;
                if (whole) out[d] = (T)end(v);
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

// Joins the parts of a row: a workgroup to a row.  The references first, a thread to a part, then the outputs: DIM / 4 threads to a part, as many
// parts side by side as there are threads, added in LDS.
template <int TYPE, int DIM, int SCORE>
__global__ __launch_bounds__(256) void k_clear_attention_join(AttentionView a, int split_tiles) {
    typedef typename Elem<TYPE>::type T;
    constexpr int QUADS = DIM / 4, SLICES = 256 / QUADS;
    const int seq = blockIdx.z, head = blockIdx.x / a.row_tiles, tile = blockIdx.x % a.row_tiles, n = blockIdx.y, t = threadIdx.x;
    const SeqPart part = seq_part(a.s, seq, a.kv.page, a.max_length, a.kv.status);
    const RowTile rt = row_tile(part, 16 * tile, 16, a.group, a.window);
    if (n >= rt.rows || rt.tiles <= split_tiles) return;
    const int splits = (rt.tiles + split_tiles - 1) / split_tiles;
    const float *ws = a.ws + ((int64_t)seq * gridDim.x + blockIdx.x) * a.splits * (16 * DIM + 32);
    __shared__ float factor[JOIN_MAX], top[4], sums[4];
    __shared__ f32x4 parts[SLICES][QUADS];
    const int quad = t % QUADS, slice = t / QUADS;
    float m = -__builtin_inff(), l = 0;
    if (t < splits) {
        m = ws[(int64_t)t * (16 * DIM + 32) + 16 * DIM + n];
        l = ws[(int64_t)t * (16 * DIM + 32) + 16 * DIM + 16 + n];
    }
    float most = m;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) most = fmaxf(most, __shfl_xor(most, k));
    if (t % 64 == 0) top[t / 64] = most;
    __syncthreads();
    most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    if (most == -__builtin_inff()) most = 0;
    const float h = half_lift(m, most);
    if (t < splits) factor[t] = h;
    l = t < splits ? l * h * h : 0;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) l += __shfl_xor(l, k);
    if (t % 64 == 0) sums[t / 64] = l;
    __syncthreads();
    f32x4 o = {0, 0, 0, 0};
    if (slice < SLICES) {
#pragma unroll 4
        for (int s = slice; s < splits; s += SLICES) {
            const f32x4 v = *(const f32x4 *)(ws + (int64_t)s * (16 * DIM + 32) + n * DIM + 4 * quad);
            const float f = factor[s];
#pragma unroll
            for (int i = 0; i < 4; i++) o[i] = __builtin_fmaf(v[i] * f, f, o[i]);
        }
        parts[slice][quad] = o;
    }
    __syncthreads();
    if (t >= QUADS) return;
    l = sums[0] + sums[1] + sums[2] + sums[3];
    o = (f32x4){0, 0, 0, 0};
    for (int s = 0; s < SLICES; s++) o += parts[s][t];
    const int row = 16 * tile + n, token = part.first + row / a.group, q_head = head * a.group + row % a.group;
    const Last end = last_of<SCORE>(most, l, [&] { return sees_any(a, seq, part.ctx + row / a.group); });
    typedef T quad_t __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    quad_t w;
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = (T)end(o[i]);
    *(quad_t *)((T *)a.out + (int64_t)token * a.out_stride + (int64_t)q_head * DIM + 4 * t) = w;
}

// Rows split over waves, keys shared: many rows (prompts).  A workgroup has 128 rows of a key head, 32 to a wave, and walks their keys in tiles of 64.
// A wave fetches one block of 16 keys and values of a tile (the codes of the next tile are under way while one is computed), widens them to 16 bits and puts them into
// LDS, values transposed and in the order in which the score's registers hold their keys; two buffers, one barrier a tile.  Matrix instructions (48 a wave and tile at
// 128 places, a third of them for the weights' second term: 258 us without it, 317 with it for 2048 + 4096 tokens of 20 over 5 heads) and the softmax's vector
// instructions (three more a weight for the two terms) decide; LDS reads are 32 KB a wave and tile.
template <int TYPE, int DIM, int SCORE, bool CAP>
__global__ __launch_bounds__(256, DIM <= 128 ? 2 : 1) void k_clear_attention_rows(AttentionView a) {
    typedef typename Elem<TYPE>::type T;
    typedef Wide<TYPE> W;
    typedef typename W::vec vec;
    typedef RowsLds<DIM> L;
    constexpr int STEPS = DIM / 16, TILES = DIM / 32, ITEMS = (DIM / 2 + 63) / 64;  // of the values: 8 keys x 4 places
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ int nan_tiles[2];  // first and last tile whose values had NaN
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 32, half = lane / 32;
    const int seq = blockIdx.z, head = blockIdx.x % a.kv.heads, tile = a.row_tiles - 1 - blockIdx.x / a.kv.heads;  // the longest rows first
    const SeqPart part = seq_part(a.s, seq, a.kv.page, a.max_length, a.kv.status);
    const RowTile all = row_tile(part, 128 * tile, 128, a.group, a.window);
    if (all.rows == 0) return;
    const int row0 = 128 * tile + 32 * wave;
    const RowTile mine = row_tile(part, row0, 32, a.group, a.window);  // rows may be 0: such a wave only fetches
    const int row = min(row0 + n, part.count * a.group - 1), token = part.first + row / a.group, pos = part.ctx + row / a.group;
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
    const int tiles = (all.last + 1 - all.lo + 63) / 64;
    // what 16 tiles need to know of their blocks of 16 keys: lane l has block l % 4 of tile l / 4
    int my_block = 0, my_good = 0;
    float my_k = 1, my_v = 1;
    const auto look_up = [&](int first) {
        const int key = all.lo + 64 * first + 16 * lane;
        my_block = my_good = 0;
        my_k = my_v = 1;
        if (sees_block(all, key, a.window)) {
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
        u32 nans = 0;
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
                    inside |= hit && all.lo + 64 * t + 16 * wave + 4 * h + 8 * (e / 4) + e % 4 <= all.last;
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
    __syncthreads();
    look_up(0);
    fetch(0);
    put(0);
    __syncthreads();
    for (int t = 0; t < tiles; t++) {
        const int key0 = all.lo + 64 * t;
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
        // a wave whose rows see nothing of the tile goes on
        if (mine.rows > 0 && key0 <= mine.last && (a.window <= 0 || key0 + 63 > mine.first - a.window)) {
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
            // register r of half x, block b = 2 x + r / 8: key 16 b + 8 (r % 8 / 4) + 4 half + r % 4
            const bool masked = key0 + 63 > mine.first || (a.window > 0 && key0 <= mine.last - a.window) || !(good[0] & good[1] & good[2] & good[3]);
            float u[4][8], most = SCORE == ENSI_SCORE_SIGMOID ? 0 : -__builtin_inff();
#pragma unroll
            for (int b = 0; b < 4; b++)
#pragma unroll
                for (int e = 0; e < 8; e++) u[b][e] = qk[b / 2][8 * (b % 2) + e];
            // softmax without a cap: the product itself, its factor enters with the exponent
            if (CAP || SCORE == ENSI_SCORE_SIGMOID) scores_of<SCORE, CAP>(u, ks, a);
            if (SCORE == ENSI_SCORE_SIGMOID)
#pragma unroll
                for (int b = 0; b < 4; b++)
#pragma unroll
                    for (int e = 0; e < 8; e++) u[b][e] = vs[b] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-u[b][e]));
            if (masked) {
                const int reach = pos - key0 - 4 * half;
                const Seen seen(a, reach);
#pragma unroll
                for (int b = 0; b < 4; b++) {
                    const int high = good[b] ? reach : INT32_MIN;
#pragma unroll
                    for (int e = 0; e < 8; e++) u[b][e] = seen.at(16 * b + 8 * (e / 4) + e % 4, high) ? u[b][e] : SCORE == ENSI_SCORE_SIGMOID ? 0 : -__builtin_inff();
                }
            }
            float factor[4], lv[4];
#pragma unroll
            for (int b = 0; b < 4; b++) {
                factor[b] = CAP || SCORE == ENSI_SCORE_SIGMOID ? 1.0f : a.factor * ks[b];
                lv[b] = __builtin_amdgcn_logf(vs[b]);
                const float top = most_of(most_of(most_of(u[b][0], u[b][1], u[b][2]), u[b][3], u[b][4]), most_of(u[b][5], u[b][6], u[b][7]));
                most = most_of(most, SCORE == ENSI_SCORE_SOFTMAX ? __builtin_fmaf(top, factor[b], lv[b]) : top);
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
    for (int key = all.lo + 64 * nan_tiles[0]; key <= min(all.lo + 64 * nan_tiles[1] + 63, all.last); key++) {
        const int block = block_of(a, seq, head, key);
        if (block < 0 || key > pos || (a.window > 0 && key <= pos - a.window)) continue;
        const unsigned char *v = a.kv.v + ((int64_t)block * KV_BLOCK + key % KV_BLOCK) * DIM + 4 * half;
#pragma unroll
        for (int j = 0; j < TILES; j++)
#pragma unroll
            for (int r = 0; r < 16; r++)
                if (is_nan(v[32 * j + 8 * (r / 4) + r % 4])) o[j][r] = __builtin_nanf("");
    }
    st_l += __shfl_xor(st_l, 32);
    if (row0 + n >= part.count * a.group) return;
    const Last end = last_of<SCORE>(st_m, st_l, [&] { return sees_any(a, seq, pos); });
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

// Whether rows are split over waves and their keys shared, or keys over waves: microseconds of either as measured (bf16, no cap).  Rows: for a tile of 64 keys 1.5 at 64
// places of a head, 1.8 at 96, 2.1 at 128, 2.75 at 192, 3.85 at 256, while two workgroups of 128 rows find room on a CU (one from 192 on); 500 + 1024 tokens of 20 over 5
// heads of 128 55, 100 + 2048 78, 2048 + 4096 312.  Keys: 50e6 to 90e6 products of a query, a key and a place in 1: these three 56, 101 and 501; 500 + 512 tokens 27 (rows 38),
// five prompts of 77 behind up to 1500 on 16 heads of 96 22 (49), 500 + 2000 of these 78 (77), 1000 + 1000 of 16 over 4 heads of 256 92 (126).
static bool attention_by_rows(const AttentionView &v, int span) {
    const int dim = v.kv.dim;
    const double blocks = (double)v.s.seqs * v.kv.heads * (((int64_t)v.s.max_new * v.group + 127) / 128);
    const double rows_us = 4 + (span + 63) / 64 * (0.72 + 0.0115 * dim) * std::max(1.0, blocks / (dim <= 128 ? 400 : 256));
    const double pairs = (double)v.s.seqs * v.s.max_new * v.q_heads * (v.window > 0 ? span : std::max(span - v.s.max_new / 2, 1));
    const double keys_us = 6 + pairs * dim / 60e6;
    return v.s.max_new > 1 && rows_us < keys_us;
}

template <int TYPE, int DIM, int SCORE>
static void attention_go(ensi_ctx *ctx, AttentionView v, hipStream_t st) {
    const int heads = v.kv.heads;
    // the most keys that a tile of 16 rows looks at: those of its window, begun within a tile of 32 and ended within one
    const int tokens = min(v.s.max_new, 15 / v.group + 2);
    const int span = v.window > 0 ? (int)min((int64_t)v.max_length, (int64_t)v.window + tokens - 1 + 31) : v.max_length;
    if (attention_by_rows(v, span)) {
        v.row_tiles = (int)(((int64_t)v.s.max_new * v.group + 127) / 128);
        ScopedTimer timer(ctx, "k_clear_attention", st);
        const auto go = [&](auto kernel) {
            constexpr int bytes = RowsLds<DIM>::BUFFERS * RowsLds<DIM>::BUFFER;
            clear_lds(ctx, (const void *)kernel, bytes);
            hipLaunchKernelGGL(kernel, dim3(heads * v.row_tiles, 1, v.s.seqs), dim3(256), bytes, st, v);
        };
        if (v.cap > 0) go(k_clear_attention_rows<TYPE, DIM, SCORE, true>);
        else go(k_clear_attention_rows<TYPE, DIM, SCORE, false>);
        return;
    }
    v.row_tiles = (int)(((int64_t)v.s.max_new * v.group + 15) / 16);
    const int64_t base = (int64_t)v.s.seqs * heads * v.row_tiles;
    const int tiles = (span + 31) / 32;
    // Parts of a row's keys.  A decoding step: 8 tiles for a wave, which evens out sequences of different lengths (48 sequences of up to 8192 tokens 66.5 us, in one part 96).
    // More where the CUs would stand idle, two workgroups for each of them (one sequence of 32768 tokens: 18.7 us with 102 parts, 19.6 with 128 or 38), unless a wave has no
    // more than 4 tiles: joining the parts costs 5 us for few rows and 10 for the thousands of a prompt (5 prompts of 77 tokens: 17.4 us in one part, 23.9 in two).
    const bool idle = base < (v.s.max_new > 1 ? 128 : 256) && tiles > 16;
    int splits = max(v.s.max_new > 1 ? 1 : (tiles + 31) / 32, idle ? (int)(512 / base) : 1);
    splits = min(splits, min((tiles + 3) / 4, JOIN_MAX));
    splits = max(splits, 1);
    const int64_t room = (int64_t)CLEAR_WS_FLOATS / (base * (16 * DIM + 32));
    if (splits > room) splits = (int)max((int64_t)1, room);
    int split_tiles = (tiles + splits - 1) / splits;
    split_tiles = max((split_tiles + 3) & ~3, 4);  // a tile for every wave
    splits = max((tiles + split_tiles - 1) / split_tiles, 1);
    v.splits = splits;
    const dim3 grid(heads * v.row_tiles, splits, v.s.seqs);
    {
        ScopedTimer timer(ctx, "k_clear_attention", st);
        if (v.cap > 0) hipLaunchKernelGGL((k_clear_attention_keys<TYPE, DIM, SCORE, true>), grid, dim3(256), 0, st, v, split_tiles);
        else hipLaunchKernelGGL((k_clear_attention_keys<TYPE, DIM, SCORE, false>), grid, dim3(256), 0, st, v, split_tiles);
    }
    if (splits == 1) return;
    ScopedTimer timer(ctx, "k_clear_attention_join", st);
    const int rows = (int)min((int64_t)16, (int64_t)v.s.max_new * v.group);
    hipLaunchKernelGGL((k_clear_attention_join<TYPE, DIM, SCORE>), dim3(heads * v.row_tiles, rows, v.s.seqs), dim3(256), 0, st, v, split_tiles);
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
    const AttentionView v = attention_view(ctx, kv, a);
    if (a.type == ENSI_T_BF16) {
        if (a.score == ENSI_SCORE_SOFTMAX) return attention_dim<ENSI_T_BF16, ENSI_SCORE_SOFTMAX>(ctx, v, st);
        return attention_dim<ENSI_T_BF16, ENSI_SCORE_SIGMOID>(ctx, v, st);
    }
    if (a.score == ENSI_SCORE_SOFTMAX) return attention_dim<ENSI_T_F16, ENSI_SCORE_SOFTMAX>(ctx, v, st);
    attention_dim<ENSI_T_F16, ENSI_SCORE_SIGMOID>(ctx, v, st);
}
