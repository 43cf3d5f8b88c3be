// Tokens from rows of logits: temperature, top-k, top-p and min-p, with given random numbers.
//
// Weights are whole multiples of 2^-S of the row's largest one, S as large as sums of the vocabulary leave room for in 64 bits (45 for 2^17 tokens): sums are then exact, do
// not hang on their order or on how a row is split, and compare with top_p and the random number as they are.  exp in 64 bits: 2^(y / 512) = 2^(k / 512) 2^(r / 512) with k the
// nearest whole number, 512 values of the first in LDS, three terms of the second beside its 1 (2^-46 of it are left out), and the addition of 2^52 rounds to a whole number of
// units.  That is about 24 instructions, 8 of them in 64 bits, and what a row without top_k costs: 21 us for 128000 of them on one CU.
//
// The filters keep the front part of the order (value falling, index rising), so that what is kept is a bound: a value, and an index among those equal to it.  It is looked for
// among few candidates, which are gathered in LDS:
//   top_k: counts in 2048 bins over the distance to the largest value show up to which bin the first k reach; for a small k the largest values of the threads do (the k-th of them
//          is not above the row's k-th);
//   top_p of all tokens: sums in these bins show in which one the bound lies; what is above it is kept.
// Where there are more candidates than room (flat rows, thousands of equal logits) the bound is found in the row itself, by bins over the bits of the values where it lies.
#include "clear.h"

#define SAMPLE_THREADS 1024
#define SAMPLE_WAVES (SAMPLE_THREADS / 64)
#define SAMPLE_BINS 2048
#define SAMPLE_SEGMENTS 512  // of a row: one wave looks through one of them at the end
#define SAMPLE_LIST 4096     // candidates
#define SAMPLE_PAIRS 256     // candidates that are compared each with each
#define SAMPLE_FEW 512       // top_k up to which the threads' largest values choose the candidates
#define SAMPLE_PARTS 8       // workgroups to a row
#define LN2 0.69314718055994530942

struct SampleLds {
    double roots[512];     // 2^(k / 512)
    u64 sum[SAMPLE_BINS];  // of the bins, of the segments of a row, or the candidates' weights
    u32 count[SAMPLE_BINS];
    u64 list[SAMPLE_LIST];  // bits of the value in their order, and inverted index: the order of the filters is the falling one of these
    u64 part[2 * SAMPLE_WAVES];
    u32 low[SAMPLE_WAVES], high[SAMPLE_WAVES];
    int found, listed;
    u64 found_before;
};

// What the workgroups of a row leave for each other, in the workspace
struct SamplePart {
    u64 bins[SAMPLE_BINS];
    u64 list[SAMPLE_LIST];
    int listed, first;
    float most;
    int pad;
};
struct SampleShared {
    u64 sum[SAMPLE_SEGMENTS];
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
// The running sum at which top_p's part ends, and the one that the random number exceeds by less than a token
__device__ __forceinline__ u64 part_target(u64 sum, float p) { return p > 0 ? max(part_of(sum, p, true), (u64)1) : 1; }
__device__ __forceinline__ u64 draw_target(u64 sum, float u) { return !(u > 0) ? 0 : u >= 1 ? sum - 1 : part_of(sum, u, false); }

enum SampleMode { SAMPLE_NONE, SAMPLE_FIRST, SAMPLE_TOP, SAMPLE_PART, SAMPLE_ALL, SAMPLE_SLOW };

template <int TYPE>
struct SampleRow {
    typedef typename Elem<TYPE>::type T;
    static constexpr int E = TYPE == ENSI_T_F32 ? 4 : 8, TILE = 64 * E, AHEAD = 4;  // elements of a lane and of a wave; tiles under way
    typedef T vec __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    SampleLds &lds;
    const T *x;
    int vocab, tiles, per;  // tiles of a row, tiles to a segment
    int lane, wave;
    float t, p, m, u;
    int k;
    // weights
    float top;             // the largest value
    double rate;           // y = (x - top) rate, 512 to a power of two
    int shift;             // S
    float bins;            // to a unit of distance
    // kept so far: values above `edge`, and of the equal ones those up to index `last`
    float edge, small;     // small: the smallest value that min_p leaves
    int last;

    __device__ SampleRow(const ensi_clear_sample_args &a, int64_t row, SampleLds &l) : lds(l) {
        x = (const T *)a.logits + row * a.stride;
        vocab = a.vocab;
        tiles = (vocab + TILE - 1) / TILE;
        per = (tiles + SAMPLE_SEGMENTS - 1) / SAMPLE_SEGMENTS;
        lane = threadIdx.x % 64;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        t = a.temperature ? a.temperature[row] : a.all_temperature;
        p = a.top_p ? a.top_p[row] : a.all_top_p;
        m = a.min_p ? a.min_p[row] : a.all_min_p;
        k = a.top_k ? a.top_k[row] : a.all_top_k;
        u = a.uniform[row];
    }
    // With the row's largest value (NaN where it has one): what is to be done, and the constants for it
    __device__ __forceinline__ SampleMode begin(float most) {
        // no distribution: NaN or +inf among the logits, nothing but -inf, numbers out of range
        if (!(fabsf(most) < __builtin_inff()) || !(t >= 0) || !(t < __builtin_inff()) || p != p || m != m || u != u) return SAMPLE_NONE;
        top = most;
        edge = small = -__builtin_inff();
        last = INT32_MAX;
        if (t == 0) return SAMPLE_FIRST;
        const int bits = 32 - __clz(vocab);
        shift = min(50, 62 - bits);
        rate = 512 / LN2 / (double)t;
        bins = (float)fmin(SAMPLE_BINS / (LN2 * (shift + 2)) / (double)t, 3e38);
        if (m > 0) {
            // min_p keeps values from some place on: found by all lanes, a 64th of what is left at a time
            const double least = 512 * log2((double)fminf(m, 1.0f));
            u32 low = 0, high = key_of(top);  // not kept, kept
            while (high - low > 1) {
                const u32 step = (high - low - 1) / 64 + 1, probe = high - low > (u32)lane * step + step ? low + ((u32)lane + 1) * step : high;
                const u64 hit = __ballot(place(of_key(probe)) >= least);  // (values below -inf are NaN)
                const int l = __ffsll((unsigned long long)hit) - 1;
                high = __shfl(probe, l);
                low += (u32)l * step;
            }
            small = of_key(high);
        }
        if (k <= 0 || k >= vocab) k = 0;
        if (!k && p >= 1) edge = small;
        return k ? (k <= SAMPLE_LIST ? SAMPLE_TOP : SAMPLE_SLOW) : p < 1 ? SAMPLE_PART : SAMPLE_ALL;
    }
    __device__ __forceinline__ void set_roots() const {
        if (threadIdx.x < 512) lds.roots[threadIdx.x] = exp2(threadIdx.x / 512.0);
    }

    __device__ __forceinline__ void load(float (&f)[E], int tile) const {
        const int at = tile * TILE + lane * E;
        if (at + E <= vocab) {
            const vec v = *(const vec *)(x + at);
#pragma unroll
            for (int i = 0; i < E; i++) f[i] = (float)v[i];
        } else {
#pragma unroll
            for (int i = 0; i < E; i++) f[i] = at + i < vocab ? (float)x[at + i] : -__builtin_inff();
        }
    }
    // todo(values, index of the first) for the tiles that `step` apart follow `first`, up to `end`: little work, AHEAD whole tiles at a time ...
    template <class TODO>
    __device__ __forceinline__ void walk(int first, int end, int step, const TODO &todo) const {
        const int whole = min(end, vocab / TILE);
        int tile = first;
        for (; tile + (AHEAD - 1) * step < whole; tile += AHEAD * step) {
            vec v[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; a++) v[a] = *(const vec *)(x + (tile + a * step) * TILE + lane * E);
#pragma unroll
            for (int a = 0; a < AHEAD; a++) {
                float f[E];
#pragma unroll
                for (int i = 0; i < E; i++) f[i] = (float)v[a][i];
                todo(f, (tile + a * step) * TILE + lane * E);
            }
        }
        for (; tile < end; tile += step) {
            float f[E];
            load(f, tile);
            todo(f, tile * TILE + lane * E);
        }
    }
    // ... or much: the next tile is under way while one is worked on
    template <class TODO>
    __device__ __forceinline__ void walk_slowly(int first, int end, int step, const TODO &todo) const {
        const int whole = min(end, vocab / TILE);
        int tile = first;
        if (tile < whole) {
            vec now = *(const vec *)(x + tile * TILE + lane * E);
            for (; tile < whole; tile += step) {
                vec next = now;
                if (tile + step < whole) next = *(const vec *)(x + (tile + step) * TILE + lane * E);
                float f[E];
#pragma unroll
                for (int i = 0; i < E; i++) f[i] = (float)now[i];
                todo(f, tile * TILE + lane * E);
                now = next;
            }
        }
        for (; tile < end; tile += step) {
            float f[E];
            load(f, tile);
            todo(f, tile * TILE + lane * E);
        }
    }
    __device__ __forceinline__ bool kept(float f, int index) const { return (f > edge) | ((f == edge) & (index <= last)); }
    __device__ __forceinline__ double place(float f) const { return ((double)f - (double)top) * rate; }
    // The weights of N values, 0 where `in` is not set; each 2^52 more than it is in its bits.  All at once, so that they hide each other's latencies.
    template <int N>
    __device__ __forceinline__ void weights(u64 (&w)[N], const float (&f)[N], const bool (&in)[N]) const {
        double r[N], root[N];
        int e[N];
#pragma unroll
        for (int i = 0; i < N; i++) {
            const double y = fmax(place(f[i]), -32768.0), z = y + 0x1.8p52;
            const int k = (int)__builtin_bit_cast(u64, z);
            r[i] = y - (z - 0x1.8p52);
            root[i] = lds.roots[k & 511];
            e[i] = (in[i] ? shift : -512) + (k >> 9);
        }
        const double a = LN2 / 512;
#pragma unroll
        for (int i = 0; i < N; i++) {
            double p = fma(r[i], a * a * a / 6, a * a / 2);
            p = fma(r[i], p, a);
            p = fma(r[i], p, 1.0);
            const double high = __builtin_bit_cast(double, __builtin_bit_cast(u64, root[i]) + ((u64)(u32)e[i] << 52));
            w[i] = __builtin_bit_cast(u64, fma(high, p, 0x1p52));
        }
    }
    static constexpr u64 NO_WEIGHT = 0x4330000000000000;  // 2^52
    __device__ __forceinline__ u64 weight(float f) const {
        u64 w[1];
        const float v[1] = {f};
        const bool in[1] = {true};
        weights<1>(w, v, in);
        return w[0] - NO_WEIGHT;
    }
    // Bins over the distance to the largest value: what lies beyond the last has no weight
    __device__ __forceinline__ int bin(float f) const { return (int)fminf((top - f) * bins, (float)SAMPLE_BINS); }

    // ---- over the workgroup
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
    template <class OP>
    __device__ __forceinline__ u32 reduce(u32 v, u32 (&each)[SAMPLE_WAVES], const OP &op) const {  // (a barrier before `each` is written again is the caller's)
#pragma unroll
        for (int k = 1; k < 64; k *= 2) v = op(v, (u32)__shfl_xor(v, k));
        if (lane == 0) each[wave] = v;
        __syncthreads();
        for (int w = 0; w < SAMPLE_WAVES; w++) v = op(v, each[w]);
        return v;
    }
    __device__ __forceinline__ u64 scan(u64 v) const {  // inclusive, over the wave
#pragma unroll
        for (int k = 1; k < 64; k *= 2) {
            const u64 o = (u64)__shfl_up((unsigned long long)v, k);
            if (lane >= k) v += o;
        }
        return v;
    }
    // The first of lds.sum[0 .. n) (or of lds.count, by COUNTS) at which the running sum reaches `target` >= 1: into lds.found, with the sum before it; n if none does.  Two to a thread
    template <bool COUNTS>
    __device__ __forceinline__ void find(int n, u64 target) const {
        __syncthreads();
        const int at = 2 * threadIdx.x;
        const u64 v0 = at < n ? (COUNTS ? (u64)lds.count[at] : lds.sum[at]) : 0, v1 = at + 1 < n ? (COUNTS ? (u64)lds.count[at + 1] : lds.sum[at + 1]) : 0;
        const u64 s = scan(v0 + v1);
        if (lane == 63) lds.part[SAMPLE_WAVES + wave] = s;
        if (threadIdx.x == 0) lds.found = n;
        __syncthreads();
        u64 before = s - v0 - v1;
        for (int w = 0; w < wave; w++) before += lds.part[SAMPLE_WAVES + w];
        if (before < target && before + v0 + v1 >= target) {  // (of one thread)
            const bool second = before + v0 < target;
            lds.found = at + second;
            lds.found_before = before + (second ? v0 : 0);
        }
        __syncthreads();
    }
    __device__ __forceinline__ void clear_bins() const {
        __syncthreads();
        for (int i = threadIdx.x; i < SAMPLE_BINS; i += SAMPLE_THREADS) {
            lds.count[i] = 0;
            lds.sum[i] = 0;
        }
        __syncthreads();
    }
    // Of the elements that each(todo) hands over as todo(key, weight), with keys from low to high: the key at which the running sum of counts or weights, from the largest key on, reaches
    // `target` >= 1, which it does; `target` becomes what is left of it there, `ties` how many have that key.
    template <bool COUNTS, class EACH>
    __device__ __forceinline__ u32 select(u32 low, u32 high, u64 &target, int &ties, const EACH &each) const {
        for (;;) {
            const int bits = 32 - __clz((int)((high - low) | 1)), step = max(0, bits - 11);
            clear_bins();
            each([&](u32 k, const auto &weight) {
                if (k >= low && k <= high) {
                    const u32 b = (high - k) >> step;
                    atomicAdd(&lds.count[b], 1u);
                    if (!COUNTS) atomicAdd((unsigned long long *)&lds.sum[b], (unsigned long long)weight());
                }
            });
            find<COUNTS>(SAMPLE_BINS, target);
            const u32 b = lds.found, first = high - (b << step);
            target -= lds.found_before;
            ties = (int)lds.count[b];
            if (step == 0) return first;
            const u32 width = (1u << step) - 1;
            if (first - low > width) low = first - width;
            high = first;
        }
    }
    // ---- in the tiles from `first` to `end`
    __device__ __forceinline__ float largest(int first, int end) const {  // of a thread; NaN where it has one
        float most = -__builtin_inff();
        walk(first + wave, end, SAMPLE_WAVES, [&](const float (&f)[E], int) {
#pragma unroll
            for (int i = 0; i < E; i++) most = __builtin_elementwise_maximum(most, f[i]);
        });
        return most;
    }
    __device__ __forceinline__ int first_largest(int first, int end) const {
        int index = INT32_MAX;
        walk(first + wave, end, SAMPLE_WAVES, [&](const float (&f)[E], int at) {
#pragma unroll
            for (int i = 0; i < E; i++)
                if (f[i] == top) index = min(index, at + i);
        });
        return (int)reduce((u32)index, lds.high, [](u32 a, u32 b) { return min(a, b); });
    }
    __device__ __forceinline__ void count_bins(int first, int end) const {
        clear_bins();
        walk(first + wave, end, SAMPLE_WAVES, [&](const float (&f)[E], int) {
#pragma unroll
            for (int i = 0; i < E; i++) {
                const int b = bin(f[i]);
                if (b < SAMPLE_BINS) atomicAdd(&lds.count[b], 1u);
            }
        });
        __syncthreads();
    }
    __device__ __forceinline__ void sum_bins(int first, int end) const {
        clear_bins();
        walk_slowly(first + wave, end, SAMPLE_WAVES, [&](const float (&f)[E], int at) {
            u64 w[E];
            bool in[E];
#pragma unroll
            for (int i = 0; i < E; i++) in[i] = kept(f[i], at + i);
            weights<E>(w, f, in);
#pragma unroll
            for (int i = 0; i < E; i++) {
                const int b = bin(f[i]);
                if (b < SAMPLE_BINS) atomicAdd((unsigned long long *)&lds.sum[b], (unsigned long long)(w[i] - NO_WEIGHT));
            }
        });
        __syncthreads();
    }
    // Puts what `in` holds for into the list
    template <class IN>
    __device__ __forceinline__ void gather(int first, int end, const IN &in) const {
        walk(first + wave, end, SAMPLE_WAVES, [&](const float (&f)[E], int at) {
#pragma unroll
            for (int i = 0; i < E; i++)
                if (in(f[i])) {
                    const int n = atomicAdd(&lds.listed, 1);
                    if (n < SAMPLE_LIST) lds.list[n] = (u64)key_of(f[i]) << 32 | ~(u32)(at + i);
                }
        });
        __syncthreads();
    }
    // Weights of what `in` holds for, summed over each segment
    template <class IN>
    __device__ __forceinline__ void sums(int first_segment, int end_segment, u64 *into, const IN &in) const {
        for (int segment = first_segment + wave; segment < end_segment; segment += SAMPLE_WAVES) {
            u64 s = 0;
            walk_slowly(segment * per, min((segment + 1) * per, tiles), 1, [&](const float (&f)[E], int at) {
                u64 w[E];
                bool is[E], any = false;
#pragma unroll
                for (int i = 0; i < E; i++) any |= is[i] = in(f[i], at + i);
                if (!__any(any)) return;
                weights<E>(w, f, is);
#pragma unroll
                for (int i = 0; i < E; i++) s += w[i];
                s -= E * NO_WEIGHT;
            });
#pragma unroll
            for (int k = 1; k < 64; k *= 2) s += (u64)__shfl_xor((unsigned long long)s, k);
            if (lane == 0) into[segment] = s;
        }
    }
    // The first index at which the running sum of `of`, whose sums over segments are in lds.sum, reaches `target` >= 1, which it does
    template <class OF>
    __device__ __forceinline__ int pick(const OF &of, u64 target) const {
        find<false>((tiles + per - 1) / per, target);
        const int segment = lds.found;
        u64 before = lds.found_before;
        __syncthreads();
        if (wave == 0) {
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
    // The token, once the bound is known and the sums of the segments are in lds.sum
    __device__ __forceinline__ int draw() const {
        __syncthreads();
        u64 sum = 0;
        for (int i = threadIdx.x; i * per < tiles; i += SAMPLE_THREADS) sum += lds.sum[i];
        sum = total(sum);
        return pick([&](float f, int at) { return kept(f, at) ? weight(f) : (u64)0; }, draw_target(sum, u) + 1);
    }
    // min_p leaves the front part of what is kept
    __device__ __forceinline__ void keep_small() {
        if (small > edge) {
            edge = small;
            last = INT32_MAX;
        }
    }
    // Moves the bound to where the running sum of counts or weights, in the order, reaches `target` >= 1; leaves it where the whole is less.  In the whole row.
    template <bool COUNTS>
    __device__ __forceinline__ void bound(u64 target) {
        const auto each = [&](const auto &todo) {
            walk(wave, tiles, SAMPLE_WAVES, [&](const float (&f)[E], int at) {
#pragma unroll 1
                for (int i = 0; i < E; i++) {
                    float v = f[0];
#pragma unroll
                    for (int j = 1; j < E; j++) v = j == i ? f[j] : v;
                    if (kept(v, at + i)) todo(key_of(v), [&] { return weight(v); });
                }
            });
        };
        if (COUNTS) count_bins(0, tiles);  // (nothing is cut before)
        else sum_bins(0, tiles);
        find<COUNTS>(SAMPLE_BINS, target);
        const int border = lds.found;
        if (border == SAMPLE_BINS) return;
        target -= lds.found_before;
        // the values in that bin
        u32 low = ~0u, high = 0;
        walk(wave, tiles, SAMPLE_WAVES, [&](const float (&f)[E], int at) {
#pragma unroll
            for (int i = 0; i < E; i++)
                if (bin(f[i]) == border && kept(f[i], at + i)) {
                    low = min(low, key_of(f[i]));
                    high = max(high, key_of(f[i]));
                }
        });
        low = reduce(low, lds.low, [](u32 a, u32 b) { return min(a, b); });
        high = reduce(high, lds.high, [](u32 a, u32 b) { return max(a, b); });
        int ties;
        const float at = of_key(select<COUNTS>(low, high, target, ties, each));
        if (edge != at) last = INT32_MAX;  // (equal ones may have been cut before)
        edge = at;
        u64 needed = target;
        if (!COUNTS) {
            const u64 w = weight(edge);
            needed = w ? (target + w - 1) / w : ties;
        }
        if (needed >= (u64)ties) return;
        // how many of the equal ones each segment has
        __syncthreads();
        for (int segment = wave; segment * per < tiles; segment += SAMPLE_WAVES) {
            u32 n = 0;
            walk(segment * per, min((segment + 1) * per, tiles), 1, [&](const float (&f)[E], int) {
#pragma unroll
                for (int i = 0; i < E; i++) n += f[i] == at;
            });
#pragma unroll
            for (int k = 1; k < 64; k *= 2) n += __shfl_xor(n, k);
            if (lane == 0) lds.sum[segment] = n;
        }
        last = pick([&](float f, int) { return (u64)(f == at ? 1 : 0); }, needed);
    }
    __device__ __forceinline__ int slowly() {
        if (k) bound<true>(k);
        if (p < 1) {
            u64 sum = 0;
            if (k) {
                walk_slowly(wave, tiles, SAMPLE_WAVES, [&](const float (&f)[E], int at) {
                    u64 w[E];
                    bool is[E];
#pragma unroll
                    for (int i = 0; i < E; i++) is[i] = kept(f[i], at + i);
                    weights<E>(w, f, is);
#pragma unroll
                    for (int i = 0; i < E; i++) sum += w[i] - NO_WEIGHT;
                });
            } else {
                sum_bins(0, tiles);
                sum = lds.sum[threadIdx.x] + lds.sum[threadIdx.x + SAMPLE_THREADS];
            }
            bound<false>(part_target(total(sum), p));
        }
        keep_small();
        __syncthreads();
        sums(0, (tiles + per - 1) / per, lds.sum, [&](float f, int at) { return kept(f, at); });
        return draw();
    }
    // ---- in the list of candidates
    template <class TODO>
    __device__ __forceinline__ void each_listed(const TODO &todo) const {
        for (int i = threadIdx.x; i < lds.listed; i += SAMPLE_THREADS) {
            const u64 e = lds.list[i];
            if (kept(of_key((u32)(e >> 32)), (int)~(u32)e)) todo((u32)(e >> 32), ~(u32)e);
        }
    }
    // Moves the bound as above, to one among the candidates.
    template <bool COUNTS>
    __device__ __forceinline__ void bound_listed(u64 target) {
        int ties;
        u32 low = ~0u, high = 0;
        each_listed([&](u32 key, u32) {
            low = min(low, key);
            high = max(high, key);
        });
        __syncthreads();
        low = reduce(low, lds.low, [](u32 a, u32 b) { return min(a, b); });
        high = reduce(high, lds.high, [](u32 a, u32 b) { return max(a, b); });
        const u32 key = select<COUNTS>(low, high, target, ties, [&](const auto &todo) { each_listed([&](u32 key, u32) { todo(key, [&] { return weight(of_key(key)); }); }); });
        const float value = of_key(key);
        u64 needed = target;
        if (!COUNTS) {
            const u64 w = weight(value);
            needed = w ? (target + w - 1) / w : ties;
        }
        int index = edge == value ? last : INT32_MAX;
        if (needed < (u64)ties)
            index = (int)~select<true>(~(u32)(vocab - 1), ~0u, needed, ties, [&](const auto &todo) {
                each_listed([&](u32 k, u32 i) {
                    if (k == key) todo(~i, [] { return 1; });
                });
            });
        edge = value;
        last = index;
    }
    // The token of a row whose top k are among the candidates
    __device__ __forceinline__ int finish_listed() {
        const int n = lds.listed;
        if (n <= SAMPLE_PAIRS) {
            // four threads to a candidate: how many come before it and what they weigh
            const int mine = threadIdx.x / 4, sub = threadIdx.x % 4;
            const bool there = mine < n;
            const u64 e = there ? lds.list[mine] : 0;
            const float f = of_key((u32)(e >> 32));
            u64 w = 0;
            if (there) w = weight(f);
            if (sub == 0) lds.sum[mine] = w;
            __syncthreads();
            int rank = 0;
            u64 before = 0;
            for (int i = sub; i < n; i += 4) {
                const bool ahead = lds.list[i] > e;
                rank += ahead;
                before += ahead ? lds.sum[i] : 0;
            }
#pragma unroll
            for (int s = 1; s < 4; s *= 2) {
                rank += __shfl_xor(rank, s);
                before += (u64)__shfl_xor((unsigned long long)before, s);
            }
            bool in = there && rank < k;
            if (p < 1) {
                const u64 target = part_target(total(sub == 0 && in ? w : 0), p);
                in = in && before < target;
            }
            in = in && f >= small;
            if (!in) w = 0;
            __syncthreads();
            if (sub == 0) lds.sum[mine] = w;
            if (threadIdx.x == 0) lds.found = 0;
            const u64 at = draw_target(total(sub == 0 ? w : 0), u);
            before = 0;
            for (int i = sub; i < n; i += 4) before += (u32)lds.list[i] > (u32)e ? lds.sum[i] : 0;  // (indices are inverted)
#pragma unroll
            for (int s = 1; s < 4; s *= 2) before += (u64)__shfl_xor((unsigned long long)before, s);
            if (sub == 0 && before <= at && at < before + w) lds.found = (int)~(u32)e;
            __syncthreads();
            return lds.found;
        }
        const auto sum = [&] {
            u64 s = 0;
            each_listed([&](u32 key, u32) { s += weight(of_key(key)); });
            return total(s);
        };
        if (k < n) bound_listed<true>(k);
        if (p < 1) bound_listed<false>(part_target(sum(), p));
        keep_small();
        u64 target = draw_target(sum(), u) + 1;
        int ties;
        return (int)~select<false>(~(u32)(vocab - 1), ~0u, target, ties, [&](const auto &todo) { each_listed([&](u32 key, u32 i) { todo(~i, [&] { return weight(of_key(key)); }); }); });
    }
    // The token of a row whose bound by top_p is among the candidates, where it leaves `rest` of the sum; the segments' sums of what is above are in lds.sum
    __device__ __forceinline__ int finish_part(u64 rest, u64 *sums) {
        bound_listed<false>(rest);  // (it works in lds.sum)
        keep_small();
        __syncthreads();
        for (int i = threadIdx.x; i * per < tiles; i += SAMPLE_THREADS) lds.sum[i] = sums[i];
        __syncthreads();
        each_listed([&](u32 key, u32 i) { atomicAdd((unsigned long long *)&lds.sum[i / TILE / per], (unsigned long long)weight(of_key(key))); });
        return draw();
    }
};

// A workgroup to a row
template <int TYPE>
__global__ __launch_bounds__(SAMPLE_THREADS) void k_clear_sample(ensi_clear_sample_args a) {
    __shared__ SampleLds lds;
    __shared__ u64 above[SAMPLE_SEGMENTS];
    SampleRow<TYPE> r(a, blockIdx.x, lds);
    r.set_roots();
    if (threadIdx.x == 0) lds.listed = 0;
    const float mine = r.largest(0, r.tiles);
    const auto larger = [](u32 a, u32 b) { return __builtin_bit_cast(u32, __builtin_elementwise_maximum(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b))); };
    SampleMode mode = r.begin(__builtin_bit_cast(float, r.reduce(__builtin_bit_cast(u32, mine), lds.low, larger)));
    const int tiles = r.tiles, segments = (tiles + r.per - 1) / r.per;
    int token = -1;
    if (mode == SAMPLE_FIRST) token = r.first_largest(0, tiles);
    if (mode == SAMPLE_TOP) {
        int limit = SAMPLE_BINS - 1;  // candidates: the bins up to this one
        if (a.vocab > SAMPLE_LIST) {
            if (r.k <= SAMPLE_FEW) {
                r.clear_bins();
                const int b = r.bin(mine);
                if (b < SAMPLE_BINS) atomicAdd(&lds.count[b], 1u);
            } else
                r.count_bins(0, tiles);
            r.template find<true>(SAMPLE_BINS, r.k);
            limit = min(lds.found, limit);
        }
        r.gather(0, tiles, [&](float f) { return r.bin(f) <= limit; });
        if (lds.listed <= SAMPLE_LIST) token = r.finish_listed();
        else mode = SAMPLE_SLOW;
    }
    if (mode == SAMPLE_PART) {
        r.sum_bins(0, tiles);
        const u64 target = part_target(r.total(lds.sum[threadIdx.x] + lds.sum[threadIdx.x + SAMPLE_THREADS]), r.p);
        r.template find<false>(SAMPLE_BINS, target);
        const int border = lds.found;
        const u64 rest = target - lds.found_before;
        r.gather(0, tiles, [&](float f) { return r.bin(f) == border; });
        if (lds.listed <= SAMPLE_LIST) {
            r.sums(0, segments, above, [&](float f, int) { return r.bin(f) < border && f >= r.small; });
            token = r.finish_part(rest, above);
        } else
            mode = SAMPLE_SLOW;
    }
    if (mode == SAMPLE_ALL) {
        r.sums(0, segments, lds.sum, [&](float f, int at) { return r.kept(f, at); });
        token = r.draw();
    }
    if (mode == SAMPLE_SLOW) token = r.slowly();
    if (threadIdx.x == 0) a.out[blockIdx.x] = token;
}

void launch_clear_sample(ensi_ctx *ctx, const ensi_clear_sample_args &a, hipStream_t st) {
    ScopedTimer timer(ctx, "k_clear_sample", st);
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((u32)a.rows), dim3(SAMPLE_THREADS), 0, st, a); };
    if (a.type == ENSI_T_F32) go(k_clear_sample<ENSI_T_F32>);
    else if (a.type == ENSI_T_BF16) go(k_clear_sample<ENSI_T_BF16>);
    else go(k_clear_sample<ENSI_T_F16>);
}
