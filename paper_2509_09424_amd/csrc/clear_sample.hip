// Tokens from rows of logits: temperature, top-k, top-p and min-p, with given random numbers.
//
// Weights are whole multiples of 2^-S of the row's largest one, S as large as sums of the vocabulary leave room for in 64 bits (45 for 2^17 tokens): sums are then exact, do
// not hang on their order, and compare with top_p and the random number as they are.  exp in 64 bits: 2^(y / 64) = 2^(k / 64) 2^(r / 64) with k the nearest whole number,
// 64 values of the first in LDS, four terms of the second beside its 1 (2^-44 of it are left out), and the addition of 2^52 rounds to a whole number of units.
//
// The filters keep the front part of the order (value falling, index rising), so that what is kept is a bound: a key, and an index among those equal to it.  A bound is found
// with histograms of counts and sums, 2048 bins over the distance to the largest value first, then over the keys of the bin where the bound lies.
#include "clear.h"

#define SAMPLE_THREADS 1024
#define SAMPLE_WAVES (SAMPLE_THREADS / 64)
#define SAMPLE_BINS 2048
#define SAMPLE_SEGMENTS 2048

struct SampleLds {
    double roots[64];  // 2^(k / 64)
    u32 count[SAMPLE_BINS + 1];
    u64 sum[SAMPLE_BINS];  // of the bins, or of the segments of a row
    u64 part[SAMPLE_WAVES];
    u32 low[SAMPLE_WAVES], high[SAMPLE_WAVES];
    int found, found_count;
    u64 found_before;
};

// Numbers in their order as unsigned ones; both zeros are one
__device__ __forceinline__ u32 key_of(float x) {
    const u32 b = __builtin_bit_cast(u32, x + 0.0f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(u32 k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffff : ~k); }

// floor(w f), and the same rounded up, for 0 <= f < 1
__device__ __forceinline__ u64 part_of(u64 w, float f, bool up) {
    const u32 b = __builtin_bit_cast(u32, f);
    const int e = (int)(b >> 23);
    const u64 m = e ? (b & 0x7fffff) | 0x800000 : b & 0x7fffff;
    const int shift = 150 - max(e, 1);  // f = m 2^-shift, 24 to 149
    const unsigned __int128 p = (unsigned __int128)w * m;
    if (shift >= 128) return up && p ? 1 : 0;
    const u64 whole = (u64)(p >> shift);
    return up && (p & (((unsigned __int128)1 << shift) - 1)) ? whole + 1 : whole;
}

template <int TYPE>
struct SampleRow {
    typedef typename Elem<TYPE>::type T;
    static constexpr int E = TYPE == ENSI_T_F32 ? 4 : 8, TILE = 64 * E;  // elements of a lane and of a wave
    const T *x;
    int vocab, tiles, per;  // tiles of a row, tiles to a segment
    SampleLds &lds;
    int lane, wave;
    // weights
    double largest, rate;  // y = (x - largest) rate, 64 to a power of two
    double least;          // y below: weight 0 by min_p
    int shift;             // S
    // kept so far: keys above `key`, and of the equal ones those up to index `last`
    u32 key;
    int last;

    __device__ __forceinline__ void load(float (&f)[E], int tile) const {
        const int at = tile * TILE + lane * E;
        if (at + E <= vocab) {
            typedef T vec __attribute__((ext_vector_type(E), aligned(sizeof(T))));
            const vec v = *(const vec *)(x + at);
#pragma unroll
            for (int i = 0; i < E; i++) f[i] = (float)v[i];
        } else {
#pragma unroll
            for (int i = 0; i < E; i++) f[i] = at + i < vocab ? (float)x[at + i] : -__builtin_inff();
        }
    }
    __device__ __forceinline__ bool kept(float f, int index) const {
        const u32 k = key_of(f);
        return k > key || (k == key && index <= last);
    }
    __device__ __forceinline__ u64 weight(float f) const {
        const double y = fmax(((double)f - largest) * rate, -4096.0), z = y + 0x1.8p52, r = y - (z - 0x1.8p52);
        if (y < least) return 0;
        const int k = (int)__builtin_bit_cast(u64, z);
        const double a = 0.69314718055994530942 / 64;
        double p = fma(r, a * a * a * a / 24, a * a * a / 6);
        p = fma(r, p, a * a / 2);
        p = fma(r, p, a);
        p = fma(r, p, 1.0);
        const double root = __builtin_bit_cast(double, __builtin_bit_cast(u64, lds.roots[k & 63]) + ((u64)(int64_t)(shift + (k >> 6)) << 52));
        return __builtin_bit_cast(u64, fma(root, p, 0x1p52)) - __builtin_bit_cast(u64, 0x1p52);
    }
    // Sum over the workgroup
    __device__ __forceinline__ u64 total(u64 v) const {
#pragma unroll
        for (int k = 1; k < 64; k *= 2) v += (u64)__shfl_xor((unsigned long long)v, k);
        __syncthreads();
        if (lane == 0) lds.part[wave] = v;
        __syncthreads();
        u64 sum = 0;
#pragma unroll
        for (int w = 0; w < SAMPLE_WAVES; w++) sum += lds.part[w];
        return sum;
    }
    __device__ __forceinline__ u64 scan(u64 v) const {  // inclusive, over the wave
#pragma unroll
        for (int k = 1; k < 64; k *= 2) {
            const u64 o = (u64)__shfl_up((unsigned long long)v, k);
            if (lane >= k) v += o;
        }
        return v;
    }
    // The first of lds.sum[0 .. n) (or of lds.count, by COUNTS) at which the running sum reaches `target` >= 1: into lds.found, with the sum before it; n if none does
    template <bool COUNTS>
    __device__ __forceinline__ void find(int n, u64 target) const {
        __syncthreads();
        if (wave == 0) {
            u64 before = 0;
            int found = n;
            for (int at = 0; at < n; at += 64) {
                const u64 v = at + lane < n ? (COUNTS ? (u64)lds.count[at + lane] : lds.sum[at + lane]) : 0, s = scan(v);
                const u64 reached = __ballot(before + s >= target);
                if (reached) {
                    const int l = __ffsll((unsigned long long)reached) - 1;
                    found = at + l;
                    before += (u64)__shfl((unsigned long long)(s - v), l);
                    break;
                }
                before += (u64)__shfl((unsigned long long)s, 63);
            }
            if (lane == 0) {
                lds.found = found;
                lds.found_before = before;
            }
        }
        __syncthreads();
    }
    // The first index at which the running sum of `of` reaches `target` >= 1, which it does
    template <class OF>
    __device__ __forceinline__ void sums(const OF &of) const {  // of every segment
        __syncthreads();
        for (int segment = wave; segment * per < tiles; segment += SAMPLE_WAVES) {
            u64 s = 0;
            for (int tile = segment * per; tile < min((segment + 1) * per, tiles); tile++) {
                float f[E];
                load(f, tile);
#pragma unroll
                for (int i = 0; i < E; i++) s += of(f[i], tile * TILE + lane * E + i);
            }
#pragma unroll
            for (int k = 1; k < 64; k *= 2) s += (u64)__shfl_xor((unsigned long long)s, k);
            if (lane == 0) lds.sum[segment] = s;
        }
        __syncthreads();
    }
    template <class OF>
    __device__ __forceinline__ int pick(const OF &of, u64 target) const {
        find<false>((tiles + per - 1) / per, target);
        const int segment = lds.found;
        u64 before = lds.found_before;
        __syncthreads();
        if (wave == 0 && segment * per < tiles) {
            for (int tile = segment * per; tile < min((segment + 1) * per, tiles); tile++) {
                float f[E];
                load(f, tile);
                u64 w[E], mine = 0;
#pragma unroll
                for (int i = 0; i < E; i++) mine += w[i] = of(f[i], tile * TILE + lane * E + i);
                const u64 s = scan(mine), reached = __ballot(before + s >= target);
                if (reached) {
                    if (lane == __ffsll((unsigned long long)reached) - 1) {
                        u64 run = before + s - mine;
                        int at = 0;
#pragma unroll
                        for (int i = 0; i < E; i++) {
                            if (run < target) at = i;
                            run += w[i];
                        }
                        lds.found = tile * TILE + lane * E + at;
                    }
                    break;
                }
                before += (u64)__shfl((unsigned long long)s, 63);
            }
        }
        __syncthreads();
        return lds.found;
    }
    // Moves the bound to where the running sum of counts or weights, in the order, reaches `target` >= 1; leaves it where the whole is less.
    template <bool COUNTS>
    __device__ __forceinline__ void bound(u64 target) {
        // bins over the distance to the largest value: what lies beyond the last has no weight
        const float top = (float)largest, scale = (float)fmin(SAMPLE_BINS / (0.69314718055994530942 * (shift + 2)) * rate * (0.69314718055994530942 / 64), 3e38);
        const auto bin = [&](float f) { return (int)fminf((top - f) * scale, (float)SAMPLE_BINS); };
        const auto clear = [&] {
            __syncthreads();
            for (int i = threadIdx.x; i < SAMPLE_BINS; i += SAMPLE_THREADS) {
                lds.count[i] = 0;
                lds.sum[i] = 0;
            }
            __syncthreads();
        };
        const auto each = [&](const auto &todo) {
            for (int tile = wave; tile < tiles; tile += SAMPLE_WAVES) {
                float f[E];
                load(f, tile);
#pragma unroll
                for (int i = 0; i < E; i++)
                    if (kept(f[i], tile * TILE + lane * E + i)) todo(f[i]);
            }
        };
        const auto add = [&](int b, float f) {
            atomicAdd(&lds.count[b], 1u);
            if (!COUNTS) atomicAdd((unsigned long long *)&lds.sum[b], (unsigned long long)weight(f));
        };
        clear();
        each([&](float f) {
            const int b = bin(f);
            if (b < SAMPLE_BINS) add(b, f);
        });
        find<COUNTS>(SAMPLE_BINS, target);
        const int border = lds.found;
        if (border == SAMPLE_BINS) return;
        target -= lds.found_before;
        // its keys
        u32 low = ~0u, high = 0;
        each([&](float f) {
            if (bin(f) == border) {
                low = min(low, key_of(f));
                high = max(high, key_of(f));
            }
        });
#pragma unroll
        for (int k = 1; k < 64; k *= 2) {
            low = min(low, (u32)__shfl_xor(low, k));
            high = max(high, (u32)__shfl_xor(high, k));
        }
        if (lane == 0) {
            lds.low[wave] = low;
            lds.high[wave] = high;
        }
        __syncthreads();
        for (int w = 0; w < SAMPLE_WAVES; w++) {
            low = min(low, lds.low[w]);
            high = max(high, lds.high[w]);
        }
        int ties;
        for (;;) {
            const int bits = 32 - __clz((int)((high - low) | 1)), step = max(0, bits - 11);
            clear();
            each([&](float f) {
                const u32 k = key_of(f);
                if (k >= low && k <= high) add((int)((high - k) >> step), f);
            });
            find<COUNTS>(SAMPLE_BINS, target);
            const u32 b = lds.found;
            target -= lds.found_before;
            ties = (int)lds.count[b];
            const u32 top_key = high - (b << step);
            if (step == 0) {
                if (key != top_key) last = INT32_MAX;  // (equal ones may have been cut before)
                key = top_key;
                break;
            }
            const u32 width = (1u << step) - 1;
            low = top_key - low > width ? top_key - width : low;
            high = top_key;
        }
        u64 needed = target;
        if (!COUNTS) {
            const u64 w = weight(of_key(key));
            needed = w ? (target + w - 1) / w : ties;
        }
        if (needed >= (u64)ties) return;
        const u32 at = key;
        const auto one = [&](float f, int) { return (u64)(key_of(f) == at ? 1 : 0); };
        sums(one);
        last = pick(one, needed);
    }
};

template <int TYPE>
__global__ __launch_bounds__(SAMPLE_THREADS) void k_clear_sample(ensi_clear_sample_args a) {
    typedef typename Elem<TYPE>::type T;
    __shared__ SampleLds lds;
    const int64_t row = blockIdx.x;
    const float t = a.temperature ? a.temperature[row] : a.all_temperature, p = a.top_p ? a.top_p[row] : a.all_top_p, m = a.min_p ? a.min_p[row] : a.all_min_p;
    const float u = a.uniform[row];
    const int k = a.top_k ? a.top_k[row] : a.all_top_k;
    const int E = SampleRow<TYPE>::E, TILE = SampleRow<TYPE>::TILE, tiles = (a.vocab + TILE - 1) / TILE;
    SampleRow<TYPE> r = {(const T *)a.logits + row * a.stride, a.vocab, tiles, (tiles + SAMPLE_SEGMENTS - 1) / SAMPLE_SEGMENTS, lds, (int)threadIdx.x % 64, (int)threadIdx.x / 64};
    if (threadIdx.x < 64) lds.roots[threadIdx.x] = exp2(threadIdx.x / 64.0);
    float most = -__builtin_inff();
    bool nan = false;
    for (int tile = r.wave; tile < tiles; tile += SAMPLE_WAVES) {
        float f[SampleRow<TYPE>::E];
        r.load(f, tile);
#pragma unroll
        for (int i = 0; i < E; i++) {
            most = fmaxf(most, f[i]);
            nan |= f[i] != f[i];
        }
    }
#pragma unroll
    for (int j = 1; j < 64; j *= 2) most = fmaxf(most, __shfl_xor(most, j));
    if (r.lane == 0) lds.high[r.wave] = key_of(most);
    nan = __syncthreads_or(nan);
    u32 high = 0;
    for (int w = 0; w < SAMPLE_WAVES; w++) high = max(high, lds.high[w]);
    most = of_key(high);
    // no distribution: NaN or +inf among the logits, nothing but -inf, numbers out of range
    if (nan || !(fabsf(most) < __builtin_inff()) || !(t >= 0) || !(t < __builtin_inff()) || p != p || m != m || u != u) {
        if (threadIdx.x == 0) a.out[row] = -1;
        return;
    }
    r.largest = most;
    r.key = 0;
    r.last = INT32_MAX;
    const bool greedy = t == 0;
    int bits = 1;
    while (a.vocab >> bits) bits++;
    r.shift = min(50, 62 - bits);
    r.rate = greedy ? 0 : 64 * 1.44269504088896340736 / (double)t;
    r.least = m > 0 ? 64 * log2((double)fminf(m, 1.0f)) : -1e30;
    if (greedy) r.key = high;  // the largest ones, of which the first is taken
    else {
        if (k > 0 && k < a.vocab) r.template bound<true>(k);
        if (p < 1) {
            const auto kept = [&](float f, int at) { return r.kept(f, at) ? r.weight(f) : (u64)0; };
            const double least = r.least;
            r.least = -1e30;
            // (min_p does not enter the sum that top_p is a part of)
            u64 mine = 0;
            for (int tile = r.wave; tile < tiles; tile += SAMPLE_WAVES) {
                float f[SampleRow<TYPE>::E];
                r.load(f, tile);
#pragma unroll
                for (int i = 0; i < E; i++) mine += kept(f[i], tile * TILE + r.lane * E + i);
            }
            const u64 whole = r.total(mine), target = p > 0 ? part_of(whole, p, true) : 1;
            r.template bound<false>(target > 0 ? target : 1);
            r.least = least;
        }
    }
    const auto of = [&](float f, int at) { return r.kept(f, at) ? greedy ? (u64)1 : r.weight(f) : (u64)0; };
    r.sums(of);
    u64 sum = 0;
    for (int i = threadIdx.x; i * r.per < tiles; i += SAMPLE_THREADS) sum += lds.sum[i];
    sum = r.total(sum);
    const u64 target = greedy || !(u > 0) ? 0 : u >= 1 ? sum - 1 : part_of(sum, u, false);
    const int token = r.pick(of, target + 1);
    if (threadIdx.x == 0) a.out[row] = token;
}

void launch_clear_sample(ensi_ctx *ctx, const ensi_clear_sample_args &a, hipStream_t st) {
    ScopedTimer timer(ctx, "k_clear_sample", st);
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((u32)a.rows), dim3(SAMPLE_THREADS), 0, st, a); };
    if (a.type == ENSI_T_F32) go(k_clear_sample<ENSI_T_F32>);
    else if (a.type == ENSI_T_BF16) go(k_clear_sample<ENSI_T_BF16>);
    else go(k_clear_sample<ENSI_T_F16>);
}
