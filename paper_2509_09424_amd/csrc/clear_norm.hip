// Root-mean-square norm of rows with the residual's addition, and the 8-bit codes that a ternary product multiplies.
//
// Per row: h = x + r (rounded to the type), p = h g, most = max |p|; codes = rint(p (127 (1 / most))), scale = most / (127 rms), out = p / rms.
// The root cancels in the codes, so they need the row's maximum only, and both row values come from one pass over the row: it is read
// once and p stays in registers.  Many rows are bound by memory (4096 x 2560 bf16 with a residual, 7 bytes an element: 14.6 us, 5.0 TB/s, where a copy of 4 GiB reaches 4.8), few
// by the launch and three latencies (1 x 2560: 2.8 us).
#include "clear.h"

struct NormView {
    const void *x, *residual, *gain;
    void *sum_out, *out;
    signed char *codes;
    float *scales;
    int64_t rows, x_stride, residual_stride, sum_stride, out_stride;
    int d;
    float eps;
};

// LANES threads hold a row, V chunks of 8 elements each: thread t has chunks t, t + LANES, ...
template <int TYPE, int LANES, int V>
__global__ __launch_bounds__(LANES == 64 ? 256 : LANES) void k_clear_norm(NormView a) {
    typedef typename Elem<TYPE>::type T;
    constexpr int PER_BLOCK = LANES == 64 ? 4 : 1;  // rows
    const int t = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * PER_BLOCK + threadIdx.x / LANES;
    if (PER_BLOCK > 1 && row >= a.rows) return;  // a whole wave: nothing is shared between the rows of a block
    const int d = a.d;
    const T *x = (const T *)a.x + row * a.x_stride;
    const T *r = a.residual ? (const T *)a.residual + row * a.residual_stride : nullptr;
    const T *g = (const T *)a.gain;
    T *sum = a.sum_out ? (T *)a.sum_out + row * a.sum_stride : nullptr;
    float p[V][8];
    float squares = 0, most = 0, check = 0;
#pragma unroll
    for (int i = 0; i < V; i++) {
        const int at = (t + i * LANES) * 8;
        float h[8], gain[8];
        if (at + 8 <= d) {
            Chunk<TYPE>::load(h, x + at);
            Chunk<TYPE>::load(gain, g + at);
            if (r) {
                float more[8];
                Chunk<TYPE>::load(more, r + at);
#pragma unroll
                for (int j = 0; j < 8; j++) h[j] = (float)(T)(h[j] + more[j]);
                if (sum) Chunk<TYPE>::store(sum + at, h);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                h[j] = gain[j] = 0;
                if (at + j < d) {
                    h[j] = (float)x[at + j];
                    gain[j] = (float)g[at + j];
                    if (r) {
                        h[j] = (float)(T)(h[j] + (float)r[at + j]);
                        if (sum) sum[at + j] = (T)h[j];
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const float v = h[j] * gain[j];
            p[i][j] = v;
            squares = __builtin_fmaf(h[j], h[j], squares);
            most = fmaxf(most, fabsf(v));
            check = __builtin_fmaf(v, 0.0f, check);  // NaN from the first infinity or NaN on
        }
    }
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        squares += __shfl_xor(squares, k);
        most = fmaxf(most, __shfl_xor(most, k));
        check += __shfl_xor(check, k);
    }
    if constexpr (LANES > 64) {
        __shared__ float part[LANES / 64][3];
        if (threadIdx.x % 64 == 0) {
            part[threadIdx.x / 64][0] = squares;
            part[threadIdx.x / 64][1] = most;
            part[threadIdx.x / 64][2] = check;
        }
        __syncthreads();
        squares = most = check = 0;
#pragma unroll
        for (int w = 0; w < LANES / 64; w++) {
            squares += part[w][0];
            most = fmaxf(most, part[w][1]);
            check += part[w][2];
        }
    }
    const bool fine = check == 0 && squares < __builtin_inff();
    float root = fine ? rsqrtf(squares / (float)d + a.eps) : __builtin_nanf(""), lift = 1;
    if (fine && squares < 0x1p-100f && a.eps < 0x1p-100f) {
        // Squares below the range of 32 bits, with no eps to hide them: once more, of h taken 2^100 times (the row's threads agree).  p and the root
        // take half of that each, which keeps both in range.  A row of zeros without an eps is 0.
        const T *from = sum ? sum : x, *more = sum ? nullptr : r;  // (x or the residual may be where the sum is)
        squares = 0;
        for (int i = 0; i < V; i++)
            for (int j = 0; j < 8; j++) {
                const int at = (t + i * LANES) * 8 + j;
                if (at >= d) break;
                float h = (float)from[at];
                if (more) h = (float)(T)(h + (float)more[at]);
                h *= 0x1p100f;
                squares = __builtin_fmaf(h, h, squares);
            }
        for (int k = 1; k < 64; k *= 2) squares += __shfl_xor(squares, k);
        if constexpr (LANES > 64) {
            __shared__ float part[LANES / 64];
            if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = squares;
            __syncthreads();
            squares = 0;
            for (int w = 0; w < LANES / 64; w++) squares += part[w];
        }
        lift = 0x1p50f;
        const float mean = squares / (float)d + a.eps * 0x1p100f * 0x1p100f;
        root = mean == 0 ? 0.0f : rsqrtf(mean) * lift;
    }
    if (a.out) {
        T *out = (T *)a.out + row * a.out_stride;
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int at = (t + i * LANES) * 8;
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; j++) o[j] = p[i][j] * lift * root;
            if (at + 8 <= d)
                Chunk<TYPE>::store(out + at, o);
            else
#pragma unroll
                for (int j = 0; j < 8; j++)
                    if (at + j < d) out[at + j] = (T)o[j];
        }
    }
    if (!a.codes) return;
    // 127 / most would leave the range of 32 bits below 2^-121: there both are taken 2^100 times, which changes no code
    const float up = most < 0x1p-100f ? 0x1p100f : 1.0f;
    const float factor = !fine || most == 0 ? 0.0f : 127.0f * (1.0f / (most * up));
    signed char *codes = a.codes + row * d;
#pragma unroll
    for (int i = 0; i < V; i++) {
        const int at = (t + i * LANES) * 8;
        u32 w[2] = {0, 0};
        if (fine) {
#pragma unroll
            for (int j = 0; j < 8; j++) w[j / 4] |= ((u32)(int)__builtin_rintf(p[i][j] * up * factor) & 255) << (8 * (j % 4));
        }
        if (at + 8 <= d) {
            typedef u32 pair __attribute__((ext_vector_type(2), aligned(1)));
            *(pair *)(codes + at) = (pair){w[0], w[1]};
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (at + j < d) codes[at + j] = (signed char)(w[j / 4] >> (8 * (j % 4)));
        }
    }
    most *= lift;
    if (t == 0) a.scales[row] = most < 0x1p-100f ? root * most / 127.0f : root * (most / 127.0f);  // (most / 127 could leave the range of 32 bits)
}

template <int TYPE, int LANES, int V>
static void norm_go(const NormView &v, hipStream_t st) {
    constexpr int PER_BLOCK = LANES == 64 ? 4 : 1;  // rows
    hipLaunchKernelGGL((k_clear_norm<TYPE, LANES, V>), dim3((u32)((v.rows + PER_BLOCK - 1) / PER_BLOCK)), dim3(PER_BLOCK * LANES), 0, st, v);
}

template <int TYPE>
static void norm_type(const NormView &v, hipStream_t st) {
    const int chunks = (v.d + 7) / 8;
    // Few chunks to a thread for few rows, whose latency decides (1 x 2560 with a residual: 2.8 us with 512 threads to a row, 3.2 with 256, 5.0 with 64; 512 rows 5.0, 5.0 and
    // 6.6), a wave to a row without a barrier for many (4096 rows: 17.2, 16.8 and 14.6 us; 2048: 10.8, 10.1 and 10.6).  200 x 8192: 5.4 us with 512, 6.4 with 256;
    // 1024 x 8191 14.5 with either.  5 chunks to a thread from 1025 to 2560 wide (4096 rows of 1040, 1536, 2048 and 2560: 10.8, 11.5, 13.0 and 14.3 us; with 8 17.8, 18.1, 19.5
    // and 21.0, with 256 threads to a row 12.4, 12.5, 15.2 and 16.1).
    if (chunks <= 64) return norm_go<TYPE, 64, 1>(v, st);
    if (v.rows > 2048 && chunks <= 8 * 64) {
        if (chunks <= 2 * 64) return norm_go<TYPE, 64, 2>(v, st);
        if (chunks <= 5 * 64) return norm_go<TYPE, 64, 5>(v, st);
        return norm_go<TYPE, 64, 8>(v, st);
    }
    if (chunks <= 128) return norm_go<TYPE, 128, 1>(v, st);
    if (v.rows > 1024 && chunks <= 2 * 256) return norm_go<TYPE, 256, 2>(v, st);
    if (chunks <= 512) return norm_go<TYPE, 512, 1>(v, st);
    if (chunks <= 2 * 512) return norm_go<TYPE, 512, 2>(v, st);
    return norm_go<TYPE, 1024, 4>(v, st);
}

void launch_clear_norm(ensi_ctx *ctx, const ensi_clear_norm_args &a, hipStream_t st) {
    ScopedTimer timer(ctx, "k_clear_norm", st);
    const NormView v = {a.x, a.residual, a.gain, a.residual ? a.sum_out : nullptr, a.out, (signed char *)a.codes, a.scales, a.rows, a.x_stride, a.residual_stride, a.sum_stride, a.out_stride, a.d, a.eps};
    if (a.type == ENSI_T_F32) return norm_type<ENSI_T_F32>(v, st);
    if (a.type == ENSI_T_BF16) return norm_type<ENSI_T_BF16>(v, st);
    norm_type<ENSI_T_F16>(v, st);
}
