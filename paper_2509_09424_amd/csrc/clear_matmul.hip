// Products of 8-bit codes with ternary weights: out[t][i] = s_t sum_g w_gi sum_{j in g} W_ji c_tj.
//
// The inner sums are whole numbers (at most 128 d < 2^24) and are formed exactly, by the int8 matrix instruction; they are rounded first when a group's
// scale multiplies them.  Weights lie in memory at two bits each, in the order in which a wave's lanes feed them to the instruction, so that a lane
// loads 64 of them with one 16-byte access and widens four at a time with a shift, a mask and one byte permutation.
#include "clear.h"

struct MatmulView {
    const u32x4 *w;
    const float *w_scales;
    const signed char *codes;
    const float *scales;
    void *out;
    int64_t codes_stride, out_stride;
    int rows, d, m, m_pad, k_chunks, m_tiles, group;  // group 0: one scale a column
};

// The weights of lane l, tile t (16 columns), chunk c (256 rows), dword s: column 16 t + l % 16, rows 256 c + 64 s + 16 (l / 16) + 4 i + b at bits
// 8 b + 2 i, plus one; 1 (weight 0) past the ends.
__global__ __launch_bounds__(256) void k_clear_pack(const signed char *W, int d, int m, int k_chunks, int64_t words, u32 *w, int *bad) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= words) return;
    const int s = at % 4, lane = at / 4 % 64;
    const int64_t tile = at / 256 / k_chunks, chunk = at / 256 % k_chunks;
    const int64_t col = tile * 16 + lane % 16, row = chunk * 256 + s * 64 + lane / 16 * 16;
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

// Few rows: a workgroup has 16 columns and NT tiles of 16 rows, its four waves take the chunks of 256 weights in turn and are added in LDS.
// The weights are what has to be read, once: bound by memory, and for the smallest by the launch.
template <int TYPE, int NT, bool GROUPED>
__global__ __launch_bounds__(256) void k_clear_matmul_few(MatmulView a) {
    typedef typename Elem<TYPE>::type T;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 16, g = lane / 16;
    const int tile = blockIdx.x, row0 = blockIdx.y * 16 * NT;
    const u32x4 *w = a.w + ((int64_t)tile * a.k_chunks) * 64 + lane;
    const signed char *row[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) row[t] = a.codes + (int64_t)min(row0 + 16 * t + n, a.rows - 1) * a.codes_stride;
    i32x4 acc[NT];
    f32x4 sum[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        acc[t] = (i32x4){0, 0, 0, 0};
        sum[t] = (f32x4){0, 0, 0, 0};
    }
    // whole sums of a group, or of a chunk's part of it, times its scale
    const int steps = GROUPED ? min(a.group / 64, 4) : 4;
    for (int c = wave; c < a.k_chunks; c += 4) {
        const u32x4 ww = w[c * 64];
#pragma unroll
        for (int s = 0; s < 4; s++) {
            const int k = 256 * c + 64 * s;
            const i32x4 v = widen(ww[s]);
#pragma unroll
            for (int t = 0; t < NT; t++) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, codes16(row[t], k + 16 * g, a.d), acc[t], 0, 0, 0);
            if (GROUPED && (s % steps == steps - 1 || s == 3 || (k + 64) % a.group == 0)) {
                const f32x4 scale = *(const f32x4 *)(a.w_scales + (int64_t)(min(k, a.d - 1) / a.group) * a.m_pad + 16 * tile + 4 * g);
#pragma unroll
                for (int t = 0; t < NT; t++)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        sum[t][r] = __builtin_fmaf((float)acc[t][r], scale[r], sum[t][r]);
                        acc[t][r] = 0;
                    }
            }
        }
    }
    __shared__ u32x4 part[4][NT][64];
#pragma unroll
    for (int t = 0; t < NT; t++) part[wave][t][lane] = GROUPED ? __builtin_bit_cast(u32x4, sum[t]) : __builtin_bit_cast(u32x4, acc[t]);
    __syncthreads();
    for (int t = wave; t < NT; t += 4) {
        f32x4 y;
        if (GROUPED) {
            y = (f32x4){0, 0, 0, 0};
#pragma unroll
            for (int p = 0; p < 4; p++) y += __builtin_bit_cast(f32x4, part[p][t][lane]);
        } else {
            i32x4 whole = {0, 0, 0, 0};
#pragma unroll
            for (int p = 0; p < 4; p++) whole += __builtin_bit_cast(i32x4, part[p][t][lane]);
            const f32x4 scale = *(const f32x4 *)(a.w_scales + 16 * tile + 4 * g);
#pragma unroll
            for (int r = 0; r < 4; r++) y[r] = (float)whole[r] * scale[r];
        }
        const int at = row0 + 16 * t + n, col = 16 * tile + 4 * g;
        if (at >= a.rows) continue;
        const float scale = a.scales[at];
        T *out = (T *)a.out + (int64_t)at * a.out_stride + col;
        if (col + 4 <= a.m) {
            typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
            vec v;
#pragma unroll
            for (int r = 0; r < 4; r++) v[r] = (T)(y[r] * scale);
            *(vec *)out = v;
        } else {
#pragma unroll
            for (int r = 0; r < 4; r++)
                if (col + r < a.m) out[r] = (T)(y[r] * scale);
        }
    }
}

template <int TYPE, int NT>
static void matmul_few(const MatmulView &v, hipStream_t st) {
    const dim3 grid(v.m_tiles, (v.rows + 16 * NT - 1) / (16 * NT)), block(256);
    if (v.group) hipLaunchKernelGGL((k_clear_matmul_few<TYPE, NT, true>), grid, block, 0, st, v);
    else hipLaunchKernelGGL((k_clear_matmul_few<TYPE, NT, false>), grid, block, 0, st, v);
}
template <int TYPE>
static void matmul_type(const MatmulView &v, hipStream_t st) {
    if (v.rows <= 16) return matmul_few<TYPE, 1>(v, st);
    if (v.rows <= 32) return matmul_few<TYPE, 2>(v, st);
    matmul_few<TYPE, 4>(v, st);
}

void launch_clear_matmul(ensi_ctx *ctx, const ensi_cw *cw, const int8_t *codes, int64_t codes_stride, const float *scales, void *out, int64_t out_stride, int64_t rows, int type,
                         hipStream_t st) {
    ScopedTimer timer(ctx, "k_clear_matmul", st);
    const MatmulView v = {(const u32x4 *)cw->w, cw->scales, (const signed char *)codes, scales, out, codes_stride, out_stride, (int)rows, cw->d, cw->m, cw->m_pad, cw->k_chunks, cw->m_tiles, cw->group};
    if (type == ENSI_T_F32) return matmul_type<ENSI_T_F32>(v, st);
    if (type == ENSI_T_BF16) return matmul_type<ENSI_T_BF16>(v, st);
    matmul_type<ENSI_T_F16>(v, st);
}

void launch_clear_pack(const int8_t *d_W, int d, int m, int k_chunks, int m_tiles, u32 *w, int *bad, hipStream_t st) {
    const int64_t words = (int64_t)m_tiles * k_chunks * 256;
    hipLaunchKernelGGL(k_clear_pack, dim3((u32)((words + 255) / 256)), dim3(256), 0, st, (const signed char *)d_W, d, m, k_chunks, words, w, bad);
}
