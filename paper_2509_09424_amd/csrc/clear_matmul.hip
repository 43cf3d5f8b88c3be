// Products of 8-bit codes with ternary weights: out[t][i] = s_t sum_g w_gi sum_{j in g} W_ji c_tj.
//
// The inner sums are whole numbers (at most 128 d < 2^24) and are formed exactly, by the int8 matrix instruction; they are rounded first when a group's
// scale multiplies them.  Weights lie in memory at two bits each, in the order in which a wave's lanes feed them to the instruction, so that a lane
// loads 64 of them with one 16-byte access and widens four at a time with a shift, a mask and one byte permutation.
#include "clear.h"
#include "ensi_dma.h"

struct MatmulView {
    const u32x2 *w;
    const float *w_scales;
    const signed char *codes;
    const float *scales;
    void *out;
    int64_t codes_stride, out_stride;
    int rows, d, m, m_pad, units, m_tiles, group;  // group 0: one scale a column
};

// Columns of a tile of 16: four tiles share 64 columns so that the four neighbouring results that a lane (n, g) has of each are 16 neighbours together,
// the first of them here.  Row 4 g + r of tile t is column tile_column(t, g) + r.
__device__ __forceinline__ int tile_column(int tile, int g) { return 64 * (tile / 4) + 16 * g + 4 * (tile % 4); }

// Weights lie as [64 columns][128 rows of W][tile of 16 columns][lane][two words]: word s of lane l, tile t and unit u has row l % 16 of the tile, rows
// 128 u + 64 s + 16 (l / 16) + 4 i + b of W at bits 8 b + 2 i, plus one; 1 (weight 0) past the ends.
__global__ __launch_bounds__(256) void k_clear_pack(const signed char *W, int d, int m, int units, int64_t words, u32 *w, int *bad) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= words) return;
    const int s = at % 2, lane = at / 2 % 64, tile = at / 128 % 4;
    const int64_t group = at / 512 / units, unit = at / 512 % units;
    const int64_t col = tile_column((int)(4 * group + tile), lane % 16 / 4) + lane % 4, row = unit * 128 + s * 64 + lane / 16 * 16;
    u32 word = 0;
    bool wrong = false;
    for (int i = 0; i < 4; i++)
        for (int b = 0; b < 4; b++) {
            const int64_t k = row + 4 * i + b;
            const int v = k < d && col < m ? W[k * m + col] : 0;
            wrong |= v < -1 || v > 1;
            word |= (u32)(v + 1) << (8 * b + 2 * i);
        }
    w[at] = word;
    if (wrong) atomicOr(bad, 1);
}

// 16 two-bit weights to 16 signed bytes: byte 0, 1 or 2 of the table 0xff, 0, 1 by every selector byte
__device__ __forceinline__ i32x4 widen(u32 w) {
    i32x4 v;
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = (int)__builtin_amdgcn_perm(0, 0x000100ff, (w >> (2 * i)) & 0x03030303);
    return v;
}

// 16 codes of a row from k on; past the row's end whatever is left of it (weights are 0 there), and nothing past it is read
__device__ __forceinline__ i32x4 codes16(const signed char *row, int k, int d) {
    typedef i32x4 loose __attribute__((aligned(1)));
    if (k + 16 <= d) return *(const loose *)(row + k);
    i32x4 v = {0, 0, 0, 0};
    if (k < d) {
#pragma unroll
        for (int j = 0; j < 16; j++)
            if (k + j < d) v[j / 4] |= ((int)row[k + j] & 255) << (8 * (j % 4));
    }
    return v;
}

// Few rows: a workgroup has a tile of 16 rows and TILES tiles of 16 columns, its four waves take the units of 128 weights in turn and are added in LDS.
// With one row the weights are what has to be read, once, and the launch takes longer than that; with more, the codes that every workgroup reads again, from L2: more
// tiles of columns share them where there are workgroups enough.
template <int TYPE, int TILES, bool GROUPED>
__global__ __launch_bounds__(256) void k_clear_matmul_few(MatmulView a) {
    typedef typename Elem<TYPE>::type T;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 16, g = lane / 16;
    const int tile0 = blockIdx.x * TILES, at = blockIdx.y * 16 + n;
    const u32x2 *w = a.w + ((int64_t)(tile0 / 4) * a.units * 4 + tile0 % 4) * 64 + lane;  // unit u: 256 u further, tile i of these: 64 i
    const signed char *row = a.codes + (int64_t)min(at, a.rows - 1) * a.codes_stride;
    i32x4 acc[TILES];
    f32x4 sum[TILES];
#pragma unroll
    for (int i = 0; i < TILES; i++) {
        acc[i] = (i32x4){0, 0, 0, 0};
        sum[i] = (f32x4){0, 0, 0, 0};
    }
    const float row_scale = a.scales[min(at, a.rows - 1)];
    f32x4 col_scale[TILES];
    if (!GROUPED)
#pragma unroll
        for (int i = 0; i < TILES; i++) col_scale[i] = *(const f32x4 *)(a.w_scales + tile_column(tile0 + i, g));
    for (int u = wave; u < a.units; u += 4) {
        // all of a unit's weights, scales and codes on their way before the first is used
        u32x2 ww[TILES];
        f32x4 scale[2][TILES];
        i32x4 x[2];
#pragma unroll
        for (int i = 0; i < TILES; i++) ww[i] = w[((int64_t)(i / 4) * a.units + u) * 256 + 64 * (i % 4)];
        if (128 * u + 128 <= a.d) {
            typedef i32x4 loose __attribute__((aligned(1)));
#pragma unroll
            for (int s = 0; s < 2; s++) x[s] = *(const loose *)(row + (128 * u + 64 * s + 16 * g));
        } else {
#pragma unroll
            for (int s = 0; s < 2; s++) x[s] = codes16(row, 128 * u + 64 * s + 16 * g, a.d);
        }
        if (GROUPED)
#pragma unroll
            for (int s = 0; s < 2; s++)
#pragma unroll
                for (int i = 0; i < TILES; i++)
                    scale[s][i] = *(const f32x4 *)(a.w_scales + (int64_t)(min(128 * u + 64 * s, a.d - 1) / a.group) * a.m_pad + tile_column(tile0 + i, g));
#pragma unroll
        for (int s = 0; s < 2; s++) {
#pragma unroll
            for (int i = 0; i < TILES; i++) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(widen(ww[i][s]), x[s], acc[i], 0, 0, 0);
            if (GROUPED && (s == 1 || (128 * u + 64) % a.group == 0)) {  // a group's sum, or a unit's part of it, times its scale
#pragma unroll
                for (int i = 0; i < TILES; i++)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        sum[i][r] = __builtin_fmaf((float)acc[i][r], scale[s][i][r], sum[i][r]);
                        acc[i][r] = 0;
                    }
            }
        }
    }
    __shared__ u32x4 part[4][TILES][64];
#pragma unroll
    for (int i = 0; i < TILES; i++) part[wave][i][lane] = GROUPED ? __builtin_bit_cast(u32x4, sum[i]) : __builtin_bit_cast(u32x4, acc[i]);
    __syncthreads();
    if (at >= a.rows) return;
#pragma unroll
    for (int i = 0; i < TILES; i++) {
        if (i % 4 != wave) continue;  // a wave to a tile
        f32x4 y;
        if (GROUPED) {
            y = (f32x4){0, 0, 0, 0};
#pragma unroll
            for (int p = 0; p < 4; p++) y += __builtin_bit_cast(f32x4, part[p][i][lane]);
        } else {
            i32x4 whole = {0, 0, 0, 0};
#pragma unroll
            for (int p = 0; p < 4; p++) whole += __builtin_bit_cast(i32x4, part[p][i][lane]);
#pragma unroll
            for (int r = 0; r < 4; r++) y[r] = (float)whole[r] * col_scale[i][r];
        }
        const int col = tile_column(tile0 + i, g);
        T *out = (T *)a.out + (int64_t)at * a.out_stride + col;
        if (col + 4 <= a.m) {
            typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
            vec v;
#pragma unroll
            for (int r = 0; r < 4; r++) v[r] = (T)(y[r] * row_scale);
            *(vec *)out = v;
        } else {
#pragma unroll
            for (int r = 0; r < 4; r++)
                if (col + r < a.m) out[r] = (T)(y[r] * row_scale);
        }
    }
}

// Many rows: the matrix cores decide.  A workgroup of eight waves has 128 rows and 256 columns, a wave 64 (TM tiles) and 64.  Codes and weights reach LDS by
// asynchronous copies, by units of 128 places, two units ahead (three buffers); nothing in the loop loads from memory to registers, as the compiler would then
// wait for every copy under way.  The codes need rows that begin and end on 16 bytes (others are copied first).  Two workgroups share a CU: one multiplies
// where the other waits at its barrier or stores.  Weights are widened by the wave that multiplies them: 44 vector instructions for 16 matrix
// instructions.  A tile of columns is the instruction's rows, so that a lane ends with neighbouring outputs of a row.
// The 8 chunks of 16 codes of a row are permuted in LDS with half the row's number: 16 rows of a fragment lie on different banks.
// Workgroups that follow each other on one XCD have the same rows.
#define MANY_COLS 256
#define MANY_ROWS 128
template <bool GROUPED>
struct ManyLds {
    static constexpr int CODES = MANY_ROWS * 128, WEIGHTS = MANY_COLS * 32, SCALES = GROUPED ? 2 * MANY_COLS * 4 : 0, BUFFER = CODES + WEIGHTS + SCALES;
};
template <int TYPE, bool GROUPED>
__global__ __launch_bounds__(512, GROUPED ? 2 : 4) void k_clear_matmul_many(MatmulView a) {
    typedef typename Elem<TYPE>::type T;
    typedef ManyLds<GROUPED> L;
    constexpr int ROWS = MANY_ROWS, TM = ROWS / 32, COPIES = TM / 2;  // copies of 8 rows a wave and unit
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 16, g = lane / 16;
    const int row_tiles = (a.rows + ROWS - 1) / ROWS, col_tiles = (a.m_tiles + 15) / 16, blocks = row_tiles * col_tiles, share = (blocks + 7) / 8;
    const int id = blockIdx.x % 8 * share + blockIdx.x / 8;
    if (id >= blocks) return;
    const int row0 = id / col_tiles * ROWS, block_tile = id % col_tiles * 16, tile0 = block_tile + 4 * (wave / 2);  // first tiles of columns of the workgroup and the wave
    const int wave_row = 16 * TM * (wave % 2);
    const u32 lds_base = __builtin_amdgcn_readfirstlane(lds_addr(lds));
    const signed char *src[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; i++) {
        const int row = 8 * (COPIES * wave + i) + lane / 8;
        src[i] = a.codes + (int64_t)min(row0 + row, a.rows - 1) * a.codes_stride + 16 * ((lane % 8) ^ (row / 2 % 8));
    }
    // 1 KB of the weights of 64 columns to a wave; columns past the last ones: those again
    const u32x4 *weights = (const u32x4 *)(a.w + (int64_t)min(block_tile / 4 + wave / 2, a.m_tiles / 4 - 1) * a.units * 256) + 64 * (wave % 2) + lane;
    const auto copy = [&](int unit) {
        const u32 to = lds_base + unit % 3 * L::BUFFER;
        dma_load16(weights + unit * 128, to + L::CODES + wave * 1024);
        if (GROUPED) {  // the scales of either step, one to a wave (and to three more: the same again)
            const int s = wave % 2, group = min(128 * unit + 64 * s, a.d - 1) / a.group;
            dma_load16(a.w_scales + (int64_t)group * a.m_pad + min(16 * block_tile + 4 * lane, a.m_pad - 4), to + L::CODES + L::WEIGHTS + s * 1024);
        }
#pragma unroll
        for (int i = 0; i < COPIES; i++) {
            const signed char *p = src[i] + 128 * unit;
            if (128 * unit + 128 > a.d) {  // past a row's end its last 16 codes, which meet weights of 0
                const int at = 128 * unit + 16 * ((lane % 8) ^ ((8 * (COPIES * wave + i) + lane / 8) / 2 % 8));
                p -= max(at - (a.d - 16), 0);
            }
            dma_load16(p, to + (COPIES * wave + i) * 1024);
        }
    };
    i32x4 acc[4][TM];
    f32x4 sum[GROUPED ? 4 : 1][GROUPED ? TM : 1];
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int t = 0; t < TM; t++) {
            acc[i][t] = (i32x4){0, 0, 0, 0};
            if (GROUPED) sum[i][t] = (f32x4){0, 0, 0, 0};
        }
    copy(0);
    if (a.units > 1) copy(1);
    for (int unit = 0; unit < a.units; unit++) {
        // the youngest copies are the next unit's; this one's have landed, and behind the barrier everybody's, and nobody reads the unit before any more
        if (unit + 1 < a.units) wait_vmcnt<COPIES + 1 + GROUPED>();
        else wait_vmcnt<0>();
        __syncthreads();
        if (unit + 2 < a.units) copy(unit + 2);
        const unsigned char *at = lds + unit % 3 * L::BUFFER;
        u32x2 w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = *(const u32x2 *)(at + L::CODES + (tile0 - block_tile + i) * 512 + 8 * lane);
#pragma unroll
        for (int s = 0; s < 2; s++) {
            i32x4 x[TM];
#pragma unroll
            for (int t = 0; t < TM; t++) x[t] = *(const i32x4 *)(at + (wave_row + 16 * t + n) * 128 + 16 * ((4 * s + g) ^ (n / 2)));
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const i32x4 v = widen(w[i][s]);
#pragma unroll
                for (int t = 0; t < TM; t++) acc[i][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, x[t], acc[i][t], 0, 0, 0);
            }
            if (GROUPED && ((128 * unit + 64 * s + 64) % a.group == 0 || (unit + 1 == a.units && s == 1))) {
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const f32x4 scale = *(const f32x4 *)(at + L::CODES + L::WEIGHTS + s * 1024 + 64 * (tile0 - block_tile) + 64 * g + 16 * i);
#pragma unroll
                    for (int t = 0; t < TM; t++)
#pragma unroll
                        for (int r = 0; r < 4; r++) {
                            sum[i][t][r] = __builtin_fmaf((float)acc[i][t][r], scale[r], sum[i][t][r]);
                            acc[i][t][r] = 0;
                        }
                }
            }
        }
    }
    // all scales before the first store: a load behind stores would wait for them
    float row_scale[TM];
    f32x4 scale[4];
#pragma unroll
    for (int t = 0; t < TM; t++) row_scale[t] = a.scales[min(row0 + wave_row + 16 * t + n, a.rows - 1)];
    if (tile0 >= a.m_tiles) return;
    const int col = tile_column(tile0, g);  // of 16 neighbours
    if (!GROUPED)
#pragma unroll
        for (int i = 0; i < 4; i++) scale[i] = *(const f32x4 *)(a.w_scales + col + 4 * i);
#pragma unroll
    for (int t = 0; t < TM; t++) {
        const int at = row0 + wave_row + 16 * t + n;
        if (at >= a.rows) continue;
        T *out = (T *)a.out + (int64_t)at * a.out_stride + col;
        float y[2][8];
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int r = 0; r < 4; r++) y[i / 2][4 * (i % 2) + r] = (GROUPED ? sum[GROUPED ? i : 0][GROUPED ? t : 0][r] : (float)acc[i][t][r] * scale[i][r]) * row_scale[t];
        if (col + 16 <= a.m) {
            Chunk<TYPE>::store(out, y[0]);
            Chunk<TYPE>::store(out + 8, y[1]);
        } else {
#pragma unroll
            for (int r = 0; r < 16; r++)
                if (col + r < a.m) out[r] = (T)y[r / 8][r % 8];
        }
    }
}

// Rows of codes that do not begin and end on 16 bytes, copied to rows that do.
__global__ __launch_bounds__(256) void k_clear_align(const signed char *codes, int64_t stride, int64_t rows, int d, int d_pad, signed char *to) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, parts = d_pad / 16;
    if (at >= rows * parts) return;
    const int64_t row = at / parts;
    const int part = (int)(at % parts);
    *(i32x4 *)(to + row * d_pad + 16 * part) = codes16(codes + row * stride, 16 * part, d);
}

// Which kernel: microseconds of either as measured (bf16).  Few rows, 8 tiles to a workgroup: 500 x 2560 x 2560 12.6, 1000 x 2560 x 6912 45, 4096 x 2560 x 6912 170, with groups
// 1000 x 2560 x 2560 33 and 2000 x 2560 x 6912 119: 3 and 1 for 0.43e9 products (0.30e9).  Many rows: 200 and 500 x 2560 x 2560 21, 1000 x 2560 x 6912
// 26, 2000 of them 40, 4096 74, with groups 100 x 2560 x 2560 32, 1000 of them 40 and 2000 x 2560 x 6912 72: for a unit of 128 places 1 (1.6) while the
// workgroups have a CU to themselves, then 1 for 230 (120) of them; the copy of unaligned codes 4 on top.
static bool matmul_is_many(const MatmulView &v, bool aligned) {
    const double few_us = 3 + (double)v.rows * v.d * v.m / (v.group ? 0.30e9 : 0.43e9);
    const double blocks = (double)((v.rows + MANY_ROWS - 1) / MANY_ROWS) * ((v.m + MANY_COLS - 1) / MANY_COLS);
    const double many_us = v.units * (v.group ? std::max(1.6, blocks / 120) : std::max(1.0, blocks / 230)) + (aligned ? 0 : 4);
    return many_us < few_us;
}
template <int TYPE, int TILES>
static void matmul_few(const MatmulView &v, hipStream_t st) {
    const dim3 grid(v.m_tiles / TILES, (v.rows + 15) / 16), block(256);
    if (v.group) hipLaunchKernelGGL((k_clear_matmul_few<TYPE, TILES, true>), grid, block, 0, st, v);
    else hipLaunchKernelGGL((k_clear_matmul_few<TYPE, TILES, false>), grid, block, 0, st, v);
}
template <int TYPE, bool GROUPED>
static void matmul_many(ensi_ctx *ctx, const MatmulView &v, hipStream_t st) {
    const int blocks = (int)((int64_t)((v.rows + MANY_ROWS - 1) / MANY_ROWS) * ((v.m + MANY_COLS - 1) / MANY_COLS));
    const int bytes = 3 * ManyLds<GROUPED>::BUFFER;
    clear_lds(ctx, (const void *)k_clear_matmul_many<TYPE, GROUPED>, bytes);
    hipLaunchKernelGGL((k_clear_matmul_many<TYPE, GROUPED>), dim3((u32)((blocks + 7) / 8 * 8)), dim3(512), bytes, st, v);
}
template <int TYPE>
static void matmul_type(ensi_ctx *ctx, const MatmulView &v, hipStream_t st) {
    const bool aligned = v.d % 16 == 0 && v.codes_stride % 16 == 0 && (uintptr_t)v.codes % 16 == 0;
    if (matmul_is_many(v, aligned)) {
        const auto many = [&](const MatmulView &u) {
            ScopedTimer timer(ctx, "k_clear_matmul", st);
            if (u.group) return matmul_many<TYPE, true>(ctx, u, st);
            matmul_many<TYPE, false>(ctx, u, st);
        };
        if (aligned) return many(v);
        // slices of the rows that the workspace holds
        const int d_pad = (v.d + 15) & ~15;
        const int slice = (int)min((size_t)v.rows, CLEAR_WS_FLOATS * sizeof(float) / d_pad);
        for (int from = 0; from < v.rows; from += slice) {
            MatmulView u = v;
            u.rows = min(slice, v.rows - from);
            u.codes = (const signed char *)ctx->ws_clear;
            u.codes_stride = u.d = d_pad;
            u.scales = v.scales + from;
            u.out = (typename Elem<TYPE>::type *)v.out + from * v.out_stride;
            {
                ScopedTimer timer(ctx, "k_clear_align", st);
                const int64_t parts = (int64_t)u.rows * (d_pad / 16);
                hipLaunchKernelGGL(k_clear_align, dim3((u32)((parts + 255) / 256)), dim3(256), 0, st, v.codes + from * v.codes_stride, v.codes_stride, (int64_t)u.rows, v.d, d_pad, (signed char *)ctx->ws_clear);
            }
            many(u);
        }
        return;
    }
    ScopedTimer timer(ctx, "k_clear_matmul", st);
    // one tile of rows: every tile of columns to a workgroup of its own (5 x 8192 x 8192: 9.2 us, with two 9.7, with four 10.9); more: as many tiles as leave the CUs
    // workgroups (64 x 4096 x 4096: 10 us with one, 7.5 with two, 6.1 with four, 8.4 with eight; 300 x 8192 x 8192: 161, 63 with four, 52 with eight)
    const int64_t tiles = (int64_t)v.m_tiles * ((v.rows + 15) / 16);
    if (v.rows > 16 && tiles >= 8 * 256) return matmul_few<TYPE, 8>(v, st);
    if (v.rows > 16 && tiles >= 4 * 128) return matmul_few<TYPE, 4>(v, st);
    if (v.rows > 16 && tiles >= 2 * 128) return matmul_few<TYPE, 2>(v, st);
    matmul_few<TYPE, 1>(v, st);
}

void launch_clear_matmul(ensi_ctx *ctx, const ensi_cw *cw, const int8_t *codes, int64_t codes_stride, const float *scales, void *out, int64_t out_stride, int64_t rows, int type,
                         hipStream_t st) {
    const MatmulView v = {(const u32x2 *)cw->w, cw->scales, (const signed char *)codes, scales, out, codes_stride, out_stride, (int)rows, cw->d, cw->m, cw->m_pad, cw->units, cw->m_tiles, cw->group};
    if (type == ENSI_T_F32) return matmul_type<ENSI_T_F32>(ctx, v, st);
    if (type == ENSI_T_BF16) return matmul_type<ENSI_T_BF16>(ctx, v, st);
    matmul_type<ENSI_T_F16>(ctx, v, st);
}

void launch_clear_pack(const int8_t *d_W, int d, int m, int units, int m_tiles, u32 *w, int *bad, hipStream_t st) {
    const int64_t words = (int64_t)m_tiles * units * 128;
    hipLaunchKernelGGL(k_clear_pack, dim3((u32)((words + 255) / 256)), dim3(256), 0, st, (const signed char *)d_W, d, m, units, words, w, bad);
}
